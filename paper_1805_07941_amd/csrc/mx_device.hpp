// Microscaled tensors on the device: rows of 4- or 8-bit elements with one power-of-two scale for 32 values along the row.
//   element E2M1 (4 bits, two to a byte, the even one in the low half): the paper's (4, 1) code at alpha = 1/2 (Eq. 1-2)
//   element E4M3 (8 bits): its (8, 3) code, but for the last code of each sign, which is NaN
//   scale byte s: 2^(s - 127); 255: the block holds NaN
// A row of K values is ceil(K / 32) blocks of 16 or 32 bytes, what lies behind K in the last block is zero codes.
//
// The gfx950 conversion instructions take the scale as the exponent field of a float (all other bits ignored, field 0 is 2^-127,
// checked against the formats' enumeration over every scale), round to nearest even and saturate E2M1; E4M3 overflows to NaN,
// so magnitudes are limited first where the scale rule lets them exceed the largest element.
#pragma once
#include "dfq_device.hpp"

namespace dfq {

constexpr int kF32 = 0, kBF16 = 1, kF16 = 2;      // dfq_dtype
constexpr int kMx4 = 0, kMx8 = 1;                 // dfq_mx_elem
constexpr int kMxBlock = 32;

typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef short v2s __attribute__((ext_vector_type(2)));

template <int DT>
constexpr int dtype_bytes() { return DT == kF32 ? 4 : 2; }

// bytes of a block's codes
__host__ __device__ constexpr int mx_block_bytes(int elem) { return elem == kMx8 ? 32 : 16; }

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
// the same at any address of their element type: global memory takes 16-byte accesses at any
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));

// ---- eight consecutive values of a row as floats; past K: zeros
template <int DT>
__device__ __forceinline__ void load_octet(float (&v)[8], const void *row, int o, int K)
{
    const char *p = (const char *)row + (size_t)o * 8 * dtype_bytes<DT>();
    const int left = K - o * 8;
    if (left >= 8) {
        if constexpr (DT == kF32) {
            const f32x4 a = ((const f32x4_any *)p)[0], b = ((const f32x4_any *)p)[1];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                v[i] = a[i];
                v[4 + i] = b[i];
            }
        } else {
            const u32x4 u = *(const u32x4_any *)p;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                if constexpr (DT == kBF16) {
                    v[2 * i] = __uint_as_float(u[i] << 16);
                    v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
                } else {
                    const uint32_t w = u[i];
                    const v2h h = __builtin_bit_cast(v2h, w);
                    v[2 * i] = (float)h[0];
                    v[2 * i + 1] = (float)h[1];
                }
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; i++) {
        float x = 0.0f;
        if (i < left) {
            if constexpr (DT == kF32) x = ((const float *)p)[i];
            else if constexpr (DT == kBF16) x = __uint_as_float((uint32_t)((const uint16_t *)p)[i] << 16);
            else x = (float)((const _Float16 *)p)[i];
        }
        v[i] = x;
    }
}

// two floats rounded to the two 16-bit values of a word
template <int DT>
__device__ __forceinline__ uint32_t pack_pair(float a, float b)
{
    static_assert(DT != kF32, "16-bit types");
    if constexpr (DT == kBF16) {
        const v2bf h = {(__bf16)a, (__bf16)b};
        return __builtin_bit_cast(uint32_t, h);
    } else {
        const v2h h = {(_Float16)a, (_Float16)b};
        return __builtin_bit_cast(uint32_t, h);
    }
}

// NT: results that are written once and too many for a cache to hold go past it
template <bool NT, class T>
__device__ __forceinline__ void store_as(T *p, const T &v)
{
    if constexpr (NT) __builtin_nontemporal_store(v, p);
    else *p = v;
}
// 16 bytes at any address of their element type (no template of the pointer's: a template's argument loses the alignment)
template <bool NT>
__device__ __forceinline__ void store_any(u32x4_any *p, u32x4 v)
{
    if constexpr (NT) __builtin_nontemporal_store(v, p);
    else *p = v;
}
template <bool NT>
__device__ __forceinline__ void store_any(f32x4_any *p, f32x4 v)
{
    if constexpr (NT) __builtin_nontemporal_store(v, p);
    else *p = v;
}

// the values of an octet rounded to the row's type and stored; nothing past K.  (float32: two stores that take turns in a cache line,
// which do not go past the cache: a conversion back of 8192 x 8192 by such stores took 64 us, past it 104.)
template <int DT, bool NT = false>
__device__ __forceinline__ void store_octet(const float (&v)[8], void *row, int o, int K)
{
    char *p = (char *)row + (size_t)o * 8 * dtype_bytes<DT>();
    const int left = K - o * 8;
    if (left >= 8) {
        if constexpr (DT == kF32) {
            ((f32x4_any *)p)[0] = f32x4{v[0], v[1], v[2], v[3]};
            ((f32x4_any *)p)[1] = f32x4{v[4], v[5], v[6], v[7]};
        } else {
            store_any<NT>((u32x4_any *)p, u32x4{pack_pair<DT>(v[0], v[1]), pack_pair<DT>(v[2], v[3]), pack_pair<DT>(v[4], v[5]), pack_pair<DT>(v[6], v[7])});
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; i++) {
        if (i >= left) break;
        if constexpr (DT == kF32) ((float *)p)[i] = v[i];
        else ((uint16_t *)p)[i] = (uint16_t)pack_pair<DT>(v[i], v[i]);
    }
}

// the bits of |v|: ordered like the magnitudes, infinities and NaNs above every number
__device__ __forceinline__ uint32_t magnitude_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// ---- the scale byte of a block whose largest magnitude has the bits u.
// floor: e = floor(log2 amax) - emax.  cover: the smallest e with amax <= top * 2^e; the largest element's significand (1.5 or 1.75)
// is where the exponent steps up: adding what it lacks of the next binade carries into the exponent field exactly above it.
template <int ELEM>
__device__ __forceinline__ int mx_scale_byte(uint32_t u, bool cover)
{
    constexpr uint32_t kTopSignificand = ELEM == kMx8 ? 0x600000u : 0x400000u;
    constexpr int kEmax = ELEM == kMx8 ? 8 : 2;
    if (u >= 0x7f800000u) return 255;
    const int field = (int)((u + (cover ? 0x7fffffu - kTopSignificand : 0u)) >> 23);
    return max(field - kEmax, 0);
}

// ---- eight values as codes at scale byte s: two words of E4M3 or one of E2M1.  The code of -0 is never written.
template <int ELEM>
__device__ __forceinline__ uint2 mx_codes(const float (&v)[8], int s, bool cover)
{
    const float scale = __uint_as_float((uint32_t)s << 23);
    if constexpr (ELEM == kMx4) {
        uint32_t w = 0;
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], scale, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], scale, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], scale, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], scale, 3);
        w &= (((w & 0x77777777u) + 0x77777777u) & 0x88888888u) | 0x77777777u;      // a sign without a magnitude goes
        return make_uint2(s == 255 ? 0u : w, 0u);
    } else {
        float t[8];
        // at most top * 2^e; a finite block's s is at most 247 without the cover rule and the product finite
        const float top = ldexpf(448.0f, s - 127);
#pragma unroll
        for (int i = 0; i < 8; i++) t[i] = cover ? v[i] : __builtin_amdgcn_fmed3f(v[i], -top, top);
        uint32_t w[2];
#pragma unroll
        for (int i = 0; i < 2; i++) {
            v2s z = {0, 0};
            z = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(z, t[4 * i], t[4 * i + 1], scale, false);
            z = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(z, t[4 * i + 2], t[4 * i + 3], scale, true);
            w[i] = __builtin_bit_cast(uint32_t, z);
            w[i] &= (((w[i] & 0x7f7f7f7fu) + 0x7f7f7f7fu) & 0x80808080u) | 0x7f7f7f7fu;
        }
        return s == 255 ? make_uint2(0u, 0u) : make_uint2(w[0], w[1]);
    }
}

// ---- N codes (8 or 4; the words that hold them) at scale byte s as floats (exact; products below 2^-149 do not occur)
template <int ELEM, int N>
__device__ __forceinline__ void mx_values(float (&v)[N], uint2 w, int s)
{
    const float scale = __uint_as_float((uint32_t)s << 23);
    v2f f[N / 2];
    if constexpr (ELEM == kMx4) {
        f[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w.x, scale, 0);
        f[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w.x, scale, 1);
        if constexpr (N == 8) {
            f[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w.x, scale, 2);
            f[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w.x, scale, 3);
        }
    } else {
        f[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.x, scale, false);
        f[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.x, scale, true);
        if constexpr (N == 8) {
            f[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.y, scale, false);
            f[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w.y, scale, true);
        }
    }
#pragma unroll
    for (int i = 0; i < N / 2; i++) {
        v[2 * i] = s == 255 ? __uint_as_float(0x7fc00000u) : f[i][0];
        v[2 * i + 1] = s == 255 ? __uint_as_float(0x7fc00000u) : f[i][1];
    }
}

// max(v, 0) that lets a NaN through
__device__ __forceinline__ float relu_f32(float v) { return v < 0.0f ? 0.0f : v; }

// the largest of a value over the four lanes of a quad, in all of them
__device__ __forceinline__ uint32_t quad_max(uint32_t u)
{
    u = max(u, (uint32_t)__builtin_amdgcn_mov_dpp((int)u, 0xB1, 0xf, 0xf, true));    // lanes 1 0 3 2
    return max(u, (uint32_t)__builtin_amdgcn_mov_dpp((int)u, 0x4E, 0xf, 0xf, true)); // lanes 2 3 0 1
}

// Octet o of a row, held by lane o % 4 of a quad with the other octets of its block: converted and stored.  All four lanes of the
// quad come here (those behind K with zeros).  nb: blocks of the row; the last one's first lane clears the scales' padding too (nb < 0:
// there is none).
template <int ELEM, bool NT = false>
__device__ __forceinline__ void mx_store_octet(const float (&v)[8], uint8_t *codes, uint8_t *scales, int o, int nb, bool cover)
{
    uint32_t u = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) u = max(u, magnitude_bits(v[i]));
    const int s = mx_scale_byte<ELEM>(quad_max(u), cover);
    const uint2 w = mx_codes<ELEM>(v, s, cover);
    if constexpr (ELEM == kMx4) store_as<NT>((uint32_t *)codes + o, w.x);
    else store_as<NT>((u32x2 *)codes + o, u32x2{w.x, w.y});
    if ((o & 3) == 0) {
        const int b = o >> 2;
        scales[b] = (uint8_t)s;
        if (b == nb - 1)
            for (int i = nb; i & 3; i++) scales[i] = 0;
    }
}

}  // namespace dfq
