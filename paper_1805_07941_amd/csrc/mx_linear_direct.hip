// The inner product on microscaled operands, y[m][n] = sum_k x[m][k] * w[n][k], without staging: a wavefront reads its operands from
// global memory straight into the registers of the matrix instruction, the wavefronts of a workgroup share the reduction axis and
// their sums meet in LDS in a fixed order.  64-bit addresses throughout: for rows further apart than the other kernels' 31-bit
// offsets reach.
//
// v_mfma_scale_f32_16x16x128_f8f6f4: rows of the first operand are features, columns of the second tokens; lane l holds row l % 16
// and, with g = l / 16, of 4-bit elements the block g of the step's four (16 bytes), of 8-bit ones bytes 16g..16g+15 of the step's
// first 64 and of its last 64; its scale byte is block g's.
#include "dfq_host.hpp"
#include "mx_linear.hpp"

namespace dfq {

namespace {

// EXACT: the elements times their scales as bfloat16 (they fit its significand) on the bfloat16 matrix instructions, whose products
// and sums keep float32's accuracy (mx_linear.hpp).
template <int EX, int EW, bool EXACT, int FT, int TT, int NW, int U>
__global__ void __launch_bounds__(NW * 64) linear_mx_direct_kernel(LinearMxArgs a)
{
    constexpr int F = FT * 16, T = TT * 16;
    constexpr int kPad = F + 4;                          // floats between tokens of the partial sums
    __shared__ float part[NW][T][kPad];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * F;
    const size_t m0 = (size_t)blockIdx.y * T;
    const int nb = (a.K + kMxBlock - 1) / kMxBlock;
    const int steps = (nb + 3) / 4;

    // rows past the last one read it again; what comes of them is not stored
    const uint8_t *wp[FT], *wsp[FT], *xp[TT], *xsp[TT];
#pragma unroll
    for (int f = 0; f < FT; f++) {
        const size_t n = (size_t)min(n0 + f * 16 + l16, a.N - 1);
        wp[f] = a.w + n * a.ldw;
        wsp[f] = a.ws + n * a.ldws;
    }
#pragma unroll
    for (int t = 0; t < TT; t++) {
        size_t m = m0 + t * 16 + l16;
        m = m < a.M ? m : a.M - 1;
        xp[t] = a.x + m * a.ldx;
        xsp[t] = a.xs + m * a.ldxs;
    }

    v4f acc[FT][TT];
#pragma unroll
    for (int f = 0; f < FT; f++)
#pragma unroll
        for (int t = 0; t < TT; t++) acc[f][t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

    // U steps at a time, so that their loads are in flight together; the wavefront's last ones, among them a last step of fewer than
    // four blocks, as one group whose missing blocks are zeros
    auto group = [&](int s, int end, auto whole) __attribute__((always_inline)) {
        Frag16<EW, EXACT> fw[U][FT];
        Frag16<EX, EXACT> fx[U][TT];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int left = decltype(whole)::value ? 4 : s + u < end ? min(nb - (s + u) * 4, 4) : 0;
#pragma unroll
            for (int f = 0; f < FT; f++) fw[u][f].load(wp[f], wsp[f], s + u, g, left);
#pragma unroll
            for (int t = 0; t < TT; t++) fx[u][t].load(xp[t], xsp[t], s + u, g, left);
        }
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
            for (int f = 0; f < FT; f++)
#pragma unroll
                for (int t = 0; t < TT; t++) acc[f][t] = multiply16(fw[u][f], fx[u][t], acc[f][t]);
    };
    const int per = (steps + NW - 1) / NW, s1 = min(steps, (wave + 1) * per), whole = min(s1, nb / 4);
    int s = wave * per;
    for (; s + U <= whole; s += U) group(s, s1, std::true_type{});
    for (; s < s1; s += U) group(s, s1, std::false_type{});

    // lane: features 4g .. 4g+3 of token l16 of each tile
#pragma unroll
    for (int f = 0; f < FT; f++)
#pragma unroll
        for (int t = 0; t < TT; t++) *(v4f *)&part[wave][t * 16 + l16][f * 16 + g * 4] = acc[f][t];
    __syncthreads();

    constexpr int kOctets = F / 8;
    with_kind(a, [&](auto kind) __attribute__((always_inline)) {
        for (int i = threadIdx.x; i < T * kOctets; i += NW * 64) {
            const int t = i / kOctets, o = i % kOctets;
            const size_t m = m0 + t;
            float v[8] = {};
    #pragma unroll 2
            for (int w = 0; w < NW; w++) {
                const v4f *p = (const v4f *)&part[w][t][o * 8];
    #pragma unroll
                for (int j = 0; j < 4; j++) {
                    v[j] += p[0][j];
                    v[4 + j] += p[1][j];
                }
            }
            if (m < a.M) OctetEnd(a, n0 / 8 + o).put<decltype(kind)::value, false>(v, a, m);
        }
    });
}

template <int EX, int EW, bool EXACT, int FT, int TT, int NW, int U>
hipError_t run(const LinearMxArgs &a, hipStream_t st)
{
    const size_t most = 65535;                           // rows of the grid
    for (size_t m = 0; m < a.M; m += most * TT * 16) {
        LinearMxArgs b = a;
        advance_tokens(b, m);
        b.M = a.M - m < most * TT * 16 ? a.M - m : most * TT * 16;
        const dim3 grid((unsigned)((a.N + FT * 16 - 1) / (FT * 16)), (unsigned)((b.M + TT * 16 - 1) / (TT * 16)));
        linear_mx_direct_kernel<EX, EW, EXACT, FT, TT, NW, U><<<grid, NW * 64, 0, st>>>(b);
    }
    return hipGetLastError();
}

template <int EX, int EW>
hipError_t by_accuracy(const LinearMxArgs &a, hipStream_t st)
{
    if constexpr (EX == kMx8 || EW == kMx8)
        if (a.exact()) return run<EX, EW, true, 2, 1, 4, 2>(a, st);
    return run<EX, EW, false, 2, 1, 4, 2>(a, st);
}

}  // namespace

hipError_t launch_linear_mx_direct(const LinearMxArgs &a, hipStream_t st)
{
    if (a.elem_x == kMx4) return a.elem_w == kMx4 ? by_accuracy<kMx4, kMx4>(a, st) : by_accuracy<kMx4, kMx8>(a, st);
    return a.elem_w == kMx4 ? by_accuracy<kMx8, kMx4>(a, st) : by_accuracy<kMx8, kMx8>(a, st);
}

}  // namespace dfq
