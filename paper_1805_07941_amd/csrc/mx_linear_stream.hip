// The inner product on microscaled operands for few results: what bounds it is the bytes of the weights and a call's latency.
//
// A workgroup has FT * 16 features and TT * 16 tokens; its wavefronts share the reduction axis, each with chunks of 256 values of its
// own, and their sums meet in LDS in a fixed order at the end.  A chunk comes by direct global -> LDS loads into a ring of one or
// two stages that belongs to the wavefront alone: nothing but its own count of outstanding loads is waited for.  (Loads straight into the
// registers of the matrix instruction have 16 rows in 16 neighbouring lanes, four cache lines to every four lanes: 41 cache accesses
// an instruction; one token through 8192 x 8192 weights of 4 bits took 12.6 us with the same bytes in flight, 11.7 with fewer.)
//
// v_mfma_scale_f32_16x16x128_f8f6f4: see Frag16.  Rows past the last token or feature and blocks past the last bring zeros from
// outside the buffers.
#include "conv_ring.hpp"
#include "mx_linear.hpp"

namespace dfq {

namespace {

template <int ELEM>
struct StreamRow {
    static constexpr int kBytes = ELEM == kMx8 ? 256 : 128;            // of a chunk
    static constexpr int kPieces16 = kBytes / 16, kRows = 64 / kPieces16;   // rows of a wavefront-wide load
    // physical place of a row's logical piece: 16 rows put one piece on all banks
    __device__ static __forceinline__ int key(int row) { return ELEM == kMx8 ? row & 15 : (row >> 1) & 7; }
};

template <int EX, int EW, bool EXACT, int FT, int TT, int NW, int NST>
__global__ void __launch_bounds__(NW * 64) linear_mx_stream_kernel(LinearMxArgs a)
{
    using RX = StreamRow<EX>;
    using RW = StreamRow<EW>;
    constexpr int F = FT * 16, T = TT * 16;
    constexpr int SW = (F + 31) / 32, SX = (T + 31) / 32;                      // loads of scales: 32 rows each
    constexpr int WL = F / RW::kRows, XL = T / RX::kRows, L = WL + XL + SW + SX;      // loads of a chunk
    constexpr int kX = F * RW::kBytes, kWS = kX + T * RX::kBytes, kXS = kWS + SW * 256, kStage = kXS + SX * 256;
    static_assert(NST * L < 64, "outstanding loads fit the counter");
    constexpr int kPad = F + 4;                          // floats between tokens of the partial sums
    static_assert(T * kPad * 4 <= NST * kStage, "partial sums in the wavefront's own stages");
    extern __shared__ char lds[];                        // NW rings of NST stages

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, g = lane >> 4;
    const int n0 = blockIdx.x * F;
    const size_t m0 = (size_t)blockIdx.y * T;
    const int nb = (a.K + kMxBlock - 1) / kMxBlock, chunks = (nb + 7) / 8;
    const int mrows = (int)(a.M - m0 < T ? a.M - m0 : T), nrows = min(a.N - n0, F);
    const unsigned xrow = (unsigned)(nb * mx_block_bytes(EX)), wrow = (unsigned)(nb * mx_block_bytes(EW)), srow = (unsigned)(nb + 3) & ~3u;
    const unsigned ldx = (unsigned)a.ldx, ldw = (unsigned)a.ldw, ldxs = (unsigned)a.ldxs, ldws = (unsigned)a.ldws;
    const v4i xr = make_rsrc(a.x + m0 * a.ldx, (unsigned)(mrows - 1) * ldx + xrow), wr = make_rsrc(a.w + (size_t)n0 * a.ldw, (unsigned)(nrows - 1) * ldw + wrow);
    const v4i xsr = make_rsrc(a.xs + m0 * a.ldxs, (unsigned)(mrows - 1) * ldxs + srow), wsr = make_rsrc(a.ws + (size_t)n0 * a.ldws, (unsigned)(nrows - 1) * ldws + srow);
    char *ring = lds + wave * NST * kStage;
    const unsigned ring_base = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(size_t)(__attribute__((address_space(3))) char *)ring);

    // ---- loads of chunk c of the row.  A load's rows: the ones behind the last lie past the buffer's end by themselves.
    auto issue = [&](int c, int stage) __attribute__((always_inline)) {
        const unsigned at = ring_base + (unsigned)stage * kStage;
        auto codes = [&](auto row, int loads, const v4i &rsrc, unsigned ld, unsigned bytes, unsigned dst) __attribute__((always_inline)) {
            using R = decltype(row);
#pragma unroll
            for (int q = 0; q < loads; q++) {
                const int r = R::kRows * q + lane / R::kPieces16;
                const unsigned k = (unsigned)c * R::kBytes + (unsigned)((lane % R::kPieces16) ^ R::key(r)) * 16;
                load_piece_to_lds(k < bytes ? (unsigned)r * ld + k : kOutOfRange, rsrc, dst + q * 1024);
            }
        };
        codes(RW{}, WL, wr, ldw, wrow, at);
        codes(RX{}, XL, xr, ldx, xrow, at + kX);
        // scales: two words of 32 rows
        const unsigned s = (unsigned)c * 8 + (lane & 1) * 4;
#pragma unroll
        for (int q = 0; q < SW; q++) {
            const int r = 32 * q + lane / 2;
            load_word_to_lds(r < F && s < srow ? (unsigned)r * ldws + s : kOutOfRange, wsr, at + kWS + q * 256);
        }
#pragma unroll
        for (int q = 0; q < SX; q++) {
            const int r = 32 * q + lane / 2;
            load_word_to_lds(r < T && s < srow ? (unsigned)r * ldxs + s : kOutOfRange, xsr, at + kXS + q * 256);
        }
    };

    v4f acc[FT][TT];
#pragma unroll
    for (int f = 0; f < FT; f++)
#pragma unroll
        for (int t = 0; t < TT; t++) acc[f][t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

    // wavefront w has chunks w, w + NW, ..; those past the last bring zeros without touching memory
#pragma unroll
    for (int i = 0; i < NST; i++) issue(wave + i * NW, i);
    for (int c = wave, stage = 0; c < chunks; c += NW, stage = stage + 1 == NST ? 0 : stage + 1) {
        wait_loads<(NST - 1) * L>();
        asm volatile("" ::: "memory");
        const char *s = ring + stage * kStage;
        Frag16<EW, EXACT> fw[2][FT];
        Frag16<EX, EXACT> fx[2][TT];
#pragma unroll
        for (int j = 0; j < 2; j++) {
            const int left = nb - (c * 2 + j) * 4;       // blocks of this step, at least 4: all
#pragma unroll
            for (int f = 0; f < FT; f++)
                fw[j][f].read(s + (f * 16 + l16) * RW::kBytes, RW::key(l16), s + kWS + (f * 16 + l16) * 8, j, g, left);
#pragma unroll
            for (int t = 0; t < TT; t++)
                fx[j][t].read(s + kX + (t * 16 + l16) * RX::kBytes, RX::key(l16), s + kXS + (t * 16 + l16) * 8, j, g, left);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the stage has been read: it is filled again while its values are multiplied
        issue(c + NST * NW, stage);
#pragma unroll
        for (int j = 0; j < 2; j++)
#pragma unroll
            for (int f = 0; f < FT; f++)
#pragma unroll
                for (int t = 0; t < TT; t++) acc[f][t] = multiply16(fw[j][f], fx[j][t], acc[f][t]);
    }
    wait_loads<0>();

    // ---- lane: features 4g .. 4g+3 of token l16 of each tile
    float *part = (float *)ring;
#pragma unroll
    for (int f = 0; f < FT; f++)
#pragma unroll
        for (int t = 0; t < TT; t++) *(v4f *)&part[(t * 16 + l16) * kPad + f * 16 + g * 4] = acc[f][t];
    __syncthreads();
    constexpr int kOctets = F / 8;
    with_kind(a, [&](auto kind) __attribute__((always_inline)) {
        for (int i = threadIdx.x; i < T * kOctets; i += NW * 64) {
            const int t = i / kOctets, o = i % kOctets;
            float v[8] = {};
    #pragma unroll 2
            for (int w = 0; w < NW; w++) {
                const v4f *p = (const v4f *)(lds + w * NST * kStage + (t * kPad + o * 8) * 4);
    #pragma unroll
                for (int j = 0; j < 4; j++) {
                    v[j] += p[0][j];
                    v[4 + j] += p[1][j];
                }
            }
            if (m0 + t < a.M) OctetEnd(a, n0 / 8 + o).put<decltype(kind)::value, false>(v, a, m0 + t);
        }
    });
}

template <int EX, int EW, bool EXACT, int FT, int TT, int NW, int NST>
hipError_t run(const LinearMxArgs &a, hipStream_t st)
{
    constexpr int kLds = NW * NST * (FT * 16 * StreamRow<EW>::kBytes + TT * 16 * StreamRow<EX>::kBytes + ((FT + 1) / 2 + (TT + 1) / 2) * 256);
    static_assert(kLds <= kLdsBytes, "LDS of a compute unit");
    const auto kernel = linear_mx_stream_kernel<EX, EW, EXACT, FT, TT, NW, NST>;
    static std::atomic<unsigned long long> devices{0};
    const hipError_t allowed = allow_lds((const void *)kernel, kLds, devices);
    if (allowed != hipSuccess) return allowed;
    const size_t most = (size_t)65535 * TT * 16;         // rows of the grid
    for (size_t m = 0; m < a.M; m += most) {
        LinearMxArgs b = a;
        advance_tokens(b, m);
        b.M = a.M - m < most ? a.M - m : most;
        const dim3 grid((unsigned)((a.N + FT * 16 - 1) / (FT * 16)), (unsigned)((b.M + TT * 16 - 1) / (TT * 16)));
        kernel<<<grid, NW * 64, kLds, st>>>(b);
    }
    return hipGetLastError();
}

template <int EX, int EW, bool EXACT>
hipError_t by_shape(const LinearMxArgs &a, LinearMxForm form, hipStream_t st)
{
    switch (form) {
        case LinearMxForm::Stream16x16: return run<EX, EW, EXACT, 1, 1, 4, 2>(a, st);
        case LinearMxForm::Stream16x32: return run<EX, EW, EXACT, 2, 1, 4, 2>(a, st);
        case LinearMxForm::Stream32x32: return run<EX, EW, EXACT, 2, 2, 4, 2>(a, st);
        case LinearMxForm::Stream32x64: return run<EX, EW, EXACT, 4, 2, 4, 1>(a, st);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace

hipError_t launch_linear_mx_stream(const LinearMxArgs &a, LinearMxForm form, hipStream_t st)
{
    const bool exact = a.exact();
    if (a.elem_x == kMx4 && a.elem_w == kMx4) return by_shape<kMx4, kMx4, false>(a, form, st);
    if (a.elem_x == kMx4) return exact ? by_shape<kMx4, kMx8, true>(a, form, st) : by_shape<kMx4, kMx8, false>(a, form, st);
    if (a.elem_w == kMx4) return exact ? by_shape<kMx8, kMx4, true>(a, form, st) : by_shape<kMx8, kMx4, false>(a, form, st);
    return exact ? by_shape<kMx8, kMx8, true>(a, form, st) : by_shape<kMx8, kMx8, false>(a, form, st);
}

}  // namespace dfq
