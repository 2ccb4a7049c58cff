// Pieces shared by the inner products on microscaled operands: operand fragments, the matrix instructions and the end of a result.
//
// Accuracy of the instructions (measured, one instruction against 64-bit sums).  The scaled f8f6f4 forms multiply 4-bit elements
// exactly and add them and the scales' powers as float32 does (2e-8).  With an 8-bit operand the products of eight consecutive k are
// aligned to the largest of them, 13 bits behind its leading one, before they are added: normal values come out 1.5e-5 off (2-norm),
// any one sum at most 7 * 2^-13 of the largest products of its groups of eight.  Where such products cancel, nothing of what is left
// need be right, so products with an 8-bit operand are computed from bfloat16 (an element times its scale fits its eight bits) by the
// bfloat16 instructions (4e-8) at half the rate of the f8f6f4 ones, unless the caller asks for these (DFQ_LINEAR_ALIGNED).
#pragma once
#include <type_traits>

#include "dfq_host.hpp"
#include "mx_device.hpp"

namespace dfq {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

__host__ inline void advance_tokens(LinearMxArgs &a, size_t m)
{
    a.x += m * a.ldx;
    a.xs += m * a.ldxs;
    if (a.y) a.y = (char *)a.y + m * a.ldy * (a.dtype == kF32 ? 4 : 2);
    if (a.q.codes) {
        a.q.codes += m * a.q.ldc;
        a.q.scales += m * a.q.lds;
    }
}

// eight codes times their scale as bfloat16, which holds their digits and, from scale byte 3 (E2M1: 0) on and below 2^128, their powers
__device__ __forceinline__ v8bf bf16_of_mx8(int lo, int hi, float scale)
{
    const v2bf a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const v2bf c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return v8bf{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

__device__ __forceinline__ v8bf bf16_of_mx4(int w, float scale)
{
    const v2bf a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
    const v2bf c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
    return v8bf{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// One lane's share of a row's 128 values for the 16x16 instructions.  EXACT: the 16 values 16g .. and 64 + 16g .. for both element
// types, so that mixed operands meet; otherwise what the f8f6f4 instruction wants.
template <int ELEM, bool EXACT>
struct Frag16 {
    static constexpr bool kWide = ELEM == kMx8;
    v4i lo, hi;                // hi: 8-bit elements only; EXACT 4-bit: lo[0..1] the first, lo[2..3] the second 16 values
    unsigned scales;           // the step's four scale bytes; not EXACT: shifted so that this lane's is the lowest

    // left: blocks the row still has in this step (4: all); the codes and scales of the others are zeros
    __device__ __forceinline__ void load(const uint8_t *row, const uint8_t *srow, int s, int g, int left)
    {
        const uint8_t *p = row + (size_t)s * (kWide ? 128 : 64);
        scales = left > 0 ? *(const unsigned *)(srow + (size_t)s * 4) : 0u;
        if (left < 4) scales &= (1u << 8 * max(left, 0)) - 1u;
        const v4i none = {0, 0, 0, 0};
        if constexpr (kWide) {
            lo = (g >> 1) < left ? *(const v4i *)(p + 16 * g) : none;
            hi = 2 + (g >> 1) < left ? *(const v4i *)(p + 64 + 16 * g) : none;
        } else if constexpr (EXACT) {
            typedef int v2i __attribute__((ext_vector_type(2)));
            const v2i nil = {0, 0};
            const v2i a = (g >> 1) < left ? *(const v2i *)(p + 8 * g) : nil, b = 2 + (g >> 1) < left ? *(const v2i *)(p + 32 + 8 * g) : nil;
            lo = v4i{a[0], a[1], b[0], b[1]};
        } else {
            lo = g < left ? *(const v4i *)(p + 16 * g) : none;
        }
        if constexpr (!EXACT) scales >>= 8 * g;
        else scales >>= 8 * (g >> 1);
    }
    // the same from a row in LDS whose pieces are XOR-ed with `key`; step j of the row, scales at srow
    __device__ __forceinline__ void read(const char *row, int key, const char *srow, int j, int g, int left)
    {
        typedef int v2i __attribute__((ext_vector_type(2)));
        if constexpr (kWide) {
            lo = *(const v4i *)(row + (((8 * j + g) ^ key) * 16));
            hi = *(const v4i *)(row + (((8 * j + 4 + g) ^ key) * 16));
        } else if constexpr (EXACT) {
            const v2i a = *(const v2i *)(row + (((4 * j + (g >> 1)) ^ key) * 16) + 8 * (g & 1)), b = *(const v2i *)(row + (((4 * j + 2 + (g >> 1)) ^ key) * 16) + 8 * (g & 1));
            lo = v4i{a[0], a[1], b[0], b[1]};
        } else {
            lo = *(const v4i *)(row + (((4 * j + g) ^ key) * 16));
        }
        scales = *(const unsigned *)(srow + 4 * j) & (left >= 4 ? ~0u : (1u << 8 * max(left, 0)) - 1u);
        scales >>= EXACT ? 8 * (g >> 1) : 8 * g;
    }
    __device__ __forceinline__ v8i codes() const
    {
        if constexpr (kWide) return v8i{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        else return v8i{lo[0], lo[1], lo[2], lo[3], 0, 0, 0, 0};
    }
    // values 8i .. 8i+7 of the lane's 32, as bfloat16
    __device__ __forceinline__ v8bf bf16(int i) const
    {
        const unsigned byte = i < 2 ? scales & 255u : (scales >> 16) & 255u;
        const float scale = __uint_as_float(byte << 23);
        v8bf r;
        if constexpr (kWide) r = i < 2 ? bf16_of_mx8(lo[2 * i], lo[2 * i + 1], scale) : bf16_of_mx8(hi[2 * i - 4], hi[2 * i - 3], scale);
        else r = bf16_of_mx4(lo[i], scale);
        return r;
    }
};

template <int EW, int EX, bool EXACT>
__device__ __forceinline__ v4f multiply16(const Frag16<EW, EXACT> &w, const Frag16<EX, EXACT> &x, v4f acc)
{
    if constexpr (EXACT) {
#pragma unroll
        for (int i = 0; i < 4; i++) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.bf16(i), x.bf16(i), acc, 0, 0, 0);
        return acc;
    } else {
        constexpr int FW = EW == kMx8 ? 0 : 4, FX = EX == kMx8 ? 0 : 4;
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w.codes(), x.codes(), acc, FW, FX, 0, (int)w.scales, 0, (int)x.scales);
    }
}

// What becomes of results: dfq_dtype's types, or converted.
constexpr int kToMx4 = 3, kToMx8 = 4;

// f(kind) with the kind of a call's results as a type
template <class F>
__device__ __forceinline__ void with_kind(const LinearMxArgs &a, F &&f)
{
    const int kind = a.q.codes ? (a.q.elem == kMx8 ? kToMx8 : kToMx4) : a.dtype;
    if (kind == kBF16) f(std::integral_constant<int, kBF16>{});
    else if (kind == kF16) f(std::integral_constant<int, kF16>{});
    else if (kind == kF32) f(std::integral_constant<int, kF32>{});
    else if (kind == kToMx8) f(std::integral_constant<int, kToMx8>{});
    else f(std::integral_constant<int, kToMx4>{});
}

// The end of results, an octet (features 8o .. 8o + 7) of one token at a time: bias, ReLU, rounding and the store.  A lane keeps its
// octet from token to token.  Converted results: the four lanes of a quad hold a block and come here together.
struct OctetEnd {
    float bias[8];
    int o, blocks;

    __device__ __forceinline__ OctetEnd(const LinearMxArgs &a, int octet) : o(octet), blocks((a.N + kMxBlock - 1) / kMxBlock)
    {
#pragma unroll
        for (int j = 0; j < 8; j++) bias[j] = a.bias && o * 8 + j < a.N ? a.bias[o * 8 + j] : 0.0f;
    }
    // WHOLE: the octet and its block are within N, and no scales' padding is to be cleared here
    template <int KIND, bool WHOLE, bool NT = false>
    __device__ __forceinline__ void put(float (&v)[8], const LinearMxArgs &a, size_t m) const
    {
        if (a.bias) {
#pragma unroll
            for (int j = 0; j < 8; j++) v[j] += bias[j];
        }
        if (a.relu) {
#pragma unroll
            for (int j = 0; j < 8; j++) v[j] = relu_f32(v[j]);
        }
        if constexpr (KIND == kToMx4 || KIND == kToMx8) {
            if (!WHOLE) {
                if (o >= blocks * 4) return;                      // (whole quads)
#pragma unroll
                for (int j = 0; j < 8; j++) v[j] = o * 8 + j < a.N ? v[j] : 0.0f;
            }
            mx_store_octet<KIND == kToMx8 ? kMx8 : kMx4, NT>(v, a.q.codes + m * a.q.ldc, a.q.scales + m * a.q.lds, o, WHOLE ? -1 : blocks, a.cover);
        } else if constexpr (WHOLE) {
            store_octet<KIND, NT>(v, (char *)a.y + m * a.ldy * dtype_bytes<KIND>(), o, o * 8 + 8);
        } else if (o * 8 < a.N) {
            store_octet<KIND>(v, (char *)a.y + m * a.ldy * dtype_bytes<KIND>(), o, a.N);
        }
    }
};

}  // namespace dfq
