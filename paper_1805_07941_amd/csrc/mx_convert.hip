// Conversion of float rows to microscaled ones and back, and the root-mean-square norm whose result is converted on the way out.
// All three move bytes: a lane takes eight values (16 bytes of a 16-bit type), the four lanes of a quad a block of 32, whose largest
// magnitude is found by two lane exchanges inside the quad.
#include <type_traits>

#include "dfq_host.hpp"
#include "mx_device.hpp"
#include "conv_epilogue.hpp"

namespace dfq {

namespace {

constexpr int kBlock = 256;

// rows * octets of one launch: 32-bit thread numbers and grids
constexpr long long kMostOctets = 1LL << 30;

template <int DT, int ELEM>
__global__ void __launch_bounds__(kBlock) quantize_mx_kernel(const char *__restrict__ x, size_t ldx, uint8_t *__restrict__ codes, size_t ldc,
                                                             uint8_t *__restrict__ scales, size_t lds, int K, int nb, unsigned total, FastDiv div, int cover)
{
    const unsigned t = blockIdx.x * kBlock + threadIdx.x;
    if (t >= total) return;                          // (total is a multiple of 4: whole quads)
    const int row = fastdiv((int)t, div), o = (int)t - row * nb * 4;
    float v[8];
    load_octet<DT>(v, x + (size_t)row * ldx, o, K);
    mx_store_octet<ELEM>(v, codes + (size_t)row * ldc, scales + (size_t)row * lds, o, nb, cover);
}

// A lane stores 16 bytes: eight values of a 16-bit type or four floats (`units` of them in a row)
template <int DT, int ELEM>
__global__ void __launch_bounds__(kBlock) dequantize_mx_kernel(const uint8_t *__restrict__ codes, size_t ldc, const uint8_t *__restrict__ scales, size_t lds,
                                                               char *__restrict__ x, size_t ldx, int K, int units, unsigned total, FastDiv div)
{
    constexpr int N = DT == kF32 ? 4 : 8;
    const unsigned t = blockIdx.x * kBlock + threadIdx.x;
    if (t >= total) return;
    const int row = fastdiv((int)t, div), o = (int)t - row * units;
    const uint8_t *c = codes + (size_t)row * ldc + (size_t)o * (N * (ELEM == kMx8 ? 8 : 4) / 8);
    uint2 w = make_uint2(0u, 0u);
    if constexpr (ELEM == kMx8 && N == 8) w = *(const uint2 *)c;
    else if constexpr (ELEM == kMx4 && N == 4) w.x = *(const uint16_t *)c;
    else w.x = *(const uint32_t *)c;
    float v[N];
    mx_values<ELEM>(v, w, scales[(size_t)row * lds + o * N / kMxBlock]);
    char *to = x + (size_t)row * ldx;
    if constexpr (DT == kF32) {
        float *p = (float *)to + o * 4;
        const int left = K - o * 4;
        if (left >= 4) {
            store_any<true>((f32x4_any *)p, f32x4{v[0], v[1], v[2], v[3]});
        } else {
#pragma unroll
            for (int i = 0; i < 4; i++)
                if (i < left) p[i] = v[i];
        }
    } else {
        store_octet<DT, true>(v, to, o, K);
    }
}

template <int DT>
hipError_t run_quantize(const MxRows &x, const MxTensor &q, bool cover, hipStream_t st)
{
    const int nb = (x.K + kMxBlock - 1) / kMxBlock;
    const size_t most = (size_t)(kMostOctets / (nb * 4LL));
    for (size_t r = 0; r < x.rows; r += most) {
        const size_t rows = x.rows - r < most ? x.rows - r : most;
        const unsigned total = (unsigned)(rows * nb * 4);
        const char *xp = (const char *)x.p + r * x.ld * dtype_bytes<DT>();
        const auto kernel = q.elem == kMx8 ? quantize_mx_kernel<DT, kMx8> : quantize_mx_kernel<DT, kMx4>;
        kernel<<<(total + kBlock - 1) / kBlock, kBlock, 0, st>>>(xp, x.ld * dtype_bytes<DT>(), q.codes + r * q.ldc, q.ldc, q.scales + r * q.lds, q.lds, x.K,
                                                                 nb, total, make_fastdiv(nb * 4), cover);
    }
    return hipGetLastError();
}

template <int DT>
hipError_t run_dequantize(const MxTensor &q, const MxRows &x, hipStream_t st)
{
    constexpr int N = DT == kF32 ? 4 : 8;
    const int units = (x.K + N - 1) / N;
    const size_t most = (size_t)(kMostOctets / units);
    for (size_t r = 0; r < x.rows; r += most) {
        const size_t rows = x.rows - r < most ? x.rows - r : most;
        const unsigned total = (unsigned)(rows * units);
        char *xp = (char *)x.p + r * x.ld * dtype_bytes<DT>();
        const auto kernel = q.elem == kMx8 ? dequantize_mx_kernel<DT, kMx8> : dequantize_mx_kernel<DT, kMx4>;
        kernel<<<(total + kBlock - 1) / kBlock, kBlock, 0, st>>>(q.codes + r * q.ldc, q.ldc, q.scales + r * q.lds, q.lds, xp, x.ld * dtype_bytes<DT>(), x.K, units,
                                                                 total, make_fastdiv(units));
    }
    return hipGetLastError();
}

// ---- root-mean-square norm: s = x + add, y = s / sqrt(mean(s^2) + eps) * weight.
// R threads to a row (a wavefront's part, a wavefront or a workgroup), V octets of the sum held in registers between the two passes
// over it; V == 0: rows too long for that, the second pass reads x and add again.  Bound by the bytes: x and add read, the sum and the
// codes written (8192 x 8192 bfloat16 to 8 bits, 472 MB: 88 us, 5.4 TB/s; a copy of that size 5.1 to 5.3).
// The sum of squares is a float32 one (in 64 bits that call took a ninth longer), but for a thread's part of the longest rows.
// Squares that leave float32's range (values of 2^50 and above, 2^-40 and below) are added again, of values times a power of two.
// The sum goes past the cache; the codes stay, the product behind the norm reads them: 8192 x 8192 codes past it 78 us, but norm and
// product 518 for 509, 16384 x 4096 with its product 314 for 295.
struct NormParams {
    RmsNormArgs a;
    int nb;
    size_t row0;             // the launch's first row
};

template <int DT>
__device__ __forceinline__ void load_sum(float (&s)[8], const NormParams &p, size_t row, int o)
{
    constexpr int B = dtype_bytes<DT>();
    load_octet<DT>(s, (const char *)p.a.x.p + row * p.a.x.ld * B, o, p.a.x.K);
    if (p.a.add) {
        float t[8];
        load_octet<DT>(t, (const char *)p.a.add + row * p.a.ldadd * B, o, p.a.x.K);
#pragma unroll
        for (int i = 0; i < 8; i++) s[i] += t[i];
    }
}

template <int DT>
__device__ __forceinline__ void load_weight(float (&w)[8], const NormParams &p, int o)
{
    if (!p.a.weight) {
#pragma unroll
        for (int i = 0; i < 8; i++) w[i] = 1.0f;
    } else if (p.a.weight_f32) {
        load_octet<kF32>(w, p.a.weight, o, p.a.x.K);
    } else {
        load_octet<DT>(w, p.a.weight, o, p.a.x.K);
    }
}

// T threads to a workgroup
template <int DT, int ELEM, int T, int R, int V>
__global__ void __launch_bounds__(T) rms_norm_mx_kernel(NormParams p)
{
    constexpr int B = dtype_bytes<DT>();
    static_assert(R <= T && (R <= 64 || R == T), "a row's threads");
    constexpr bool EARLY = V == 1;                       // the weight is asked for before the sum of squares is known (V == 2: 104 for 95 us)
    __shared__ float part[T / 64];
    const size_t row = p.row0 + (size_t)blockIdx.x * (T / R) + threadIdx.x / R;
    if (row >= p.a.x.rows) return;                       // (R < T: whole groups of threads, and no barrier below)
    const int K = p.a.x.K, octets = p.nb * 4, first = threadIdx.x % R;
    float s[V > 0 ? V : 1][8], w[EARLY ? V : 1][8];
    // the sum of the squares of the row's values times c
    auto squares = [&](float c, auto again) __attribute__((always_inline)) {
        float sq = 0.0f;
        auto visit = [&](const float (&v)[8]) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 8; i++) sq += (v[i] * c) * (v[i] * c);
        };
        if constexpr (V > 0) {
#pragma unroll
            for (int j = 0; j < V; j++)
                if (j * R + first < octets) {
                    if constexpr (!decltype(again)::value) load_sum<DT>(s[j], p, row, j * R + first);
                    visit(s[j]);
                }
            if constexpr (EARLY && !decltype(again)::value) {
#pragma unroll
                for (int j = 0; j < V; j++)
                    if (j * R + first < octets) load_weight<DT>(w[j], p, j * R + first);
            }
        } else {
            // up to 512 octets to a thread: each is added up on its own and they meet in 64 bits, where thousands of additions that round
            // the same way gather nothing (2^22 equal values: 2 steps of float32 off, 260 without)
            double wide = 0.0;
            for (int o = first; o < octets; o += R) {
                load_sum<DT>(s[0], p, row, o);
                sq = 0.0f;
                visit(s[0]);
                wide += (double)sq;
            }
            sq = (float)wide;
        }
#pragma unroll
        for (int off = (R < 64 ? R : 64) / 2; off >= 1; off >>= 1) sq += __shfl_xor(sq, off, kWave);
        if constexpr (R > 64) {
            if constexpr (decltype(again)::value) __syncthreads();
            if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sq;
            __syncthreads();
            sq = 0.0f;
#pragma unroll
            for (int i = 0; i < T / 64; i++) sq += part[i];
        }
        return sq;
    };
    float c = 1.0f, lift = 1.0f, sq = squares(1.0f, std::false_type{}), mean = sq / (float)K + p.a.eps;
    if (!(sq <= 0x1p100f) || mean < 0x1p-80f) {          // (the same for all of a row's threads)
        // 2^22 squares of values up to 2^128 or a single one of 2^-149 stay normal; the mean of such a one among zeros does times 2^24
        c = sq <= 0x1p100f ? 0x1p90f : 0x1p-76f;
        lift = c > 1.0f ? 0x1p24f : 1.0f;
        mean = squares(c, std::true_type{}) * (lift / (float)K) + p.a.eps * c * c * lift;
    }
    const float r = (lift > 1.0f ? 0x1p12f : 1.0f) / sqrtf(mean);
    // A value times c times r: the factor above 1 before r and the one below 1 behind it, so that nothing between leaves float32's range
    // (a row with 2^51 has c = 2^-76, and its values below 2^-50 must not be multiplied by that first).
    const float before = fmaxf(c, 1.0f), behind = fminf(c, 1.0f);

    auto finish = [&](float (&v)[8], float (&g)[8], int o) __attribute__((always_inline)) {
        if (!EARLY) load_weight<DT>(g, p, o);
        if (p.a.sum) store_octet<DT, true>(v, (char *)p.a.sum + row * p.a.ldsum * B, o, K);
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = o * 8 + i < K ? v[i] * before * r * behind * g[i] : 0.0f;      // (zeros behind K whatever r is)
        if (p.a.y) store_octet<DT, true>(v, (char *)p.a.y + row * p.a.ldy * B, o, K);
        if (p.a.q.codes) mx_store_octet<ELEM>(v, p.a.q.codes + row * p.a.q.ldc, p.a.q.scales + row * p.a.q.lds, o, p.nb, p.a.cover);
    };
    if constexpr (V > 0) {
#pragma unroll
        for (int j = 0; j < V; j++)
            if (j * R + first < octets) finish(s[j], w[EARLY ? j : 0], j * R + first);
    } else {
        for (int o = first; o < octets; o += R) {
            load_sum<DT>(s[0], p, row, o);
            finish(s[0], w[0], o);
        }
    }
}

template <int DT, int ELEM, int T, int R, int V>
hipError_t run_norm(NormParams p, hipStream_t st)
{
    constexpr size_t rows = T / R, most = kMostThreads / T * rows;
    for (; p.row0 < p.a.x.rows; p.row0 += most) {
        const size_t n = p.a.x.rows - p.row0 < most ? p.a.x.rows - p.row0 : most;
        rms_norm_mx_kernel<DT, ELEM, T, R, V><<<(unsigned)((n + rows - 1) / rows), T, 0, st>>>(p);
    }
    return hipGetLastError();
}

// Rows of up to 512 values several to a workgroup (16384 x 100: 7.2 us, a workgroup of one wavefront each 16.6); as many threads as
// leave one or two octets to each (1 x 4096 by 512 threads 3.2 us, by 256 4.1; 64 x 16384 by 1024 5.8, by 512 7.1)
template <int DT, int ELEM>
hipError_t run_norm(const NormParams &p, hipStream_t st)
{
    const int octets = p.nb * 4;
    if (octets <= 16) return run_norm<DT, ELEM, 256, 16, 1>(p, st);
    if (octets <= 32) return run_norm<DT, ELEM, 256, 32, 1>(p, st);
    if (octets <= 64) return run_norm<DT, ELEM, 256, 64, 1>(p, st);
    if (octets <= 256) return run_norm<DT, ELEM, 256, 256, 1>(p, st);
    if (octets <= 512) return run_norm<DT, ELEM, 512, 512, 1>(p, st);
    if (octets <= 1024) return run_norm<DT, ELEM, 512, 512, 2>(p, st);
    if (octets <= 2048) return run_norm<DT, ELEM, 1024, 1024, 2>(p, st);
    if (octets <= 4096) return run_norm<DT, ELEM, 1024, 1024, 4>(p, st);
    return run_norm<DT, ELEM, 1024, 1024, 0>(p, st);
}

}  // namespace

hipError_t launch_quantize_mx(const MxRows &x, const MxTensor &q, bool cover, hipStream_t st)
{
    return x.dtype == kF32 ? run_quantize<kF32>(x, q, cover, st) : x.dtype == kBF16 ? run_quantize<kBF16>(x, q, cover, st) : run_quantize<kF16>(x, q, cover, st);
}

hipError_t launch_dequantize_mx(const MxTensor &q, const MxRows &x, hipStream_t st)
{
    return x.dtype == kF32 ? run_dequantize<kF32>(q, x, st) : x.dtype == kBF16 ? run_dequantize<kBF16>(q, x, st) : run_dequantize<kF16>(q, x, st);
}

hipError_t launch_rms_norm_mx(const RmsNormArgs &a, hipStream_t st)
{
    const NormParams p{a, (a.x.K + kMxBlock - 1) / kMxBlock, 0};
    const bool mx8 = a.q.elem == kMx8;
    if (a.x.dtype == kF32) return mx8 ? run_norm<kF32, kMx8>(p, st) : run_norm<kF32, kMx4>(p, st);
    if (a.x.dtype == kBF16) return mx8 ? run_norm<kBF16, kMx8>(p, st) : run_norm<kBF16, kMx4>(p, st);
    return mx8 ? run_norm<kF16, kMx8>(p, st) : run_norm<kF16, kMx4>(p, st);
}

}  // namespace dfq
