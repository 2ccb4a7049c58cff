// The inner product on microscaled operands for results that fill the chip: tiles of tokens x features from operands staged in LDS.
//
// acc[n][m] = sum_k w[n][k] * x[m][k]: features are the rows of the matrix instruction's first operand and tokens the columns of its
// second; feature rows lie in LDS in an order that leaves 16 consecutive features of one token in each lane.  A workgroup walks the
// reduction axis in steps of 128 bytes of an operand row (256 values of 4 bits, 128 where an operand has 8) through a ring of LDS
// stages that direct global -> LDS loads fill, one barrier to a step.  A wavefront waits for its own loads of the step it is about to
// read only, and reads the next 64 values' operands while the matrix pipe is busy with these.
//
// Scales come in chunks of 16 bytes of a row (512 values): a row's four bytes of one step would cost as many cache lines as its 128
// bytes of codes.  Chunk c + 1 is loaded in equal parts with the steps of chunk c, into a ring of its own.  What lies behind a row's
// last block is masked twice: codes by an offset past the buffer (zeros arrive), scales by a comparison when they are read, so that
// neither the next row's bytes nor padding count.
#include "conv_ring.hpp"
#include "mx_linear.hpp"

namespace dfq {

namespace {

typedef float v16f __attribute__((ext_vector_type(16)));

struct TileParams {
    LinearMxArgs a;
    int nb;                  // blocks of a row
    int steps;
    int tiles_m, tiles_n;
};

// f(0), f(1), .. f(N - 1) with the number as a type
template <int N, int I = 0, class F>
__device__ __forceinline__ void static_for(F &&f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        static_for<N, I + 1>(f);
    }
}

template <int ELEM, int KS>
struct Operand {
    static constexpr int kRow = KS * (ELEM == kMx8 ? 8 : 4) / 8;      // bytes of a row in a stage
    static constexpr int kPieces16 = kRow / 16;
    static_assert(kRow == 64 || kRow == 128, "LDS rows");
    // physical place of a row's logical piece: 16 consecutive rows put one piece on all banks
    __device__ static __forceinline__ int place(int row, int piece) { return kRow == 128 ? piece ^ ((row >> 1) & 7) : piece ^ ((row >> 2) & 3); }
};

// chunks of scales in LDS: chunk s / SPC + 1 is loaded with step s, up to NST steps ahead of the one that is read
constexpr int scale_chunks(int nst, int spc) { return (nst + spc - 1) / spc + 2 <= 4 ? 4 : 8; }

// where a row's words of a chunk of scales are
__device__ __forceinline__ int scale_key(int row) { return (row >> 3) & 3; }

// One lane's operands of a 32-row group for 64 values: what v_mfma_scale_f32_32x32x64_f8f6f4 wants (with h = lane / 32: of 4-bit
// elements block h, of 8-bit ones bytes 16h.. of both blocks).  EXACT: bytes 16h.. (4 bits: 8h..) of both blocks, and both scales.
// (Otherwise scales are words, the bytes of four blocks, shifted so that block h's is the lowest: two parts take its bytes 0 and 2.)
template <int ELEM, bool EXACT>
struct Frag32 {
    v4i lo, hi;
    unsigned scale, scale1;
};

template <int EX, int EW, bool EXACT, int BM, int BN, int WM, int WN, int OCC, int NST, bool WHOLE>
__global__ void __launch_bounds__(WM * WN * 64, OCC) linear_mx_tiles_kernel(TileParams prm)
{
    constexpr int NW = WM * WN;
    constexpr int KS = EX == kMx4 && EW == kMx4 ? 256 : 128;
    constexpr int KK = KS / 64;                                        // matrix instructions along a step
    using OX = Operand<EX, KS>;
    using OW = Operand<EW, KS>;
    constexpr int TM = BM / WM / 32, TN = BN / WN / 32;
    constexpr int XL = BM * OX::kRow / 1024 / NW, WL = BN * OW::kRow / 1024 / NW;     // code loads of a wavefront in a step
    constexpr int SPC = 512 / KS;                                      // steps of a chunk of scales
    constexpr int SL = ((BM + BN) / 16 + SPC * NW - 1) / (SPC * NW);   // scale loads of a wavefront in a step
    static_assert(XL * NW * 1024 == BM * OX::kRow && WL * NW * 1024 == BN * OW::kRow, "whole loads");
    constexpr int LPS = XL + WL + SL;
    static_assert(NST >= 2 && SPC * SL + NST * LPS < 64, "outstanding loads fit the counter");
    constexpr int NCH = scale_chunks(NST, SPC);
    constexpr int kStage = BM * OX::kRow + BN * OW::kRow;
    constexpr int kChunk = SL * SPC * NW * 256;                        // (rows past the tile's: loads to keep their number even)

    extern __shared__ char lds[];                                      // NST stages, then NCH chunks of scales
    const LinearMxArgs &a = prm.a;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, h = lane >> 5;

    // ---- this workgroup's tile.  Workgroups are dealt round-robin to the 8 XCDs: each gets a contiguous run of tiles, in groups of
    // four token tiles that share the feature tiles they pass
    int t = blockIdx.x;
    {
        const int G = gridDim.x, per = G / 8, rem = G % 8, xcd = t % 8, idx = t / 8;
        t = (xcd < rem ? xcd * (per + 1) : rem * (per + 1) + (xcd - rem) * per) + idx;
    }
    constexpr int kGroup = 4;
    const int group = t / (kGroup * prm.tiles_n), in = t - group * kGroup * prm.tiles_n;
    const int rows = min(kGroup, prm.tiles_m - group * kGroup);
    const size_t m0 = (size_t)(group * kGroup + in % rows) * BM;
    const int n0 = in / rows * BN;

    const int mrows = (int)(a.M - m0 < BM ? a.M - m0 : BM), nrows = min(a.N - n0, BN);
    const unsigned xrow = (unsigned)(prm.nb * mx_block_bytes(EX)), wrow = (unsigned)(prm.nb * mx_block_bytes(EW));
    const unsigned srow = (unsigned)(prm.nb + 3) & ~3u;
    const unsigned ldx = (unsigned)a.ldx, ldw = (unsigned)a.ldw, ldxs = (unsigned)a.ldxs, ldws = (unsigned)a.ldws;
    const v4i xr = make_rsrc(a.x + m0 * a.ldx, (unsigned)(mrows - 1) * ldx + xrow);
    const v4i wr = make_rsrc(a.w + (size_t)n0 * a.ldw, (unsigned)(nrows - 1) * ldw + wrow);
    const v4i xsr = make_rsrc(a.xs + m0 * a.ldxs, (unsigned)(mrows - 1) * ldxs + srow);
    const v4i wsr = make_rsrc(a.ws + (size_t)n0 * a.ldws, (unsigned)(nrows - 1) * ldws + srow);
    const unsigned lds_base = (unsigned)(size_t)(__attribute__((address_space(3))) char *)(char *)&lds[0];

    // feature of LDS row r of the weights (within the tile): row 8g + 4h + e of a group of 32 holds feature 16h + 4g + e
    auto feature_of = [](int r) { return (r & ~31) + 16 * ((r >> 2) & 1) + 4 * ((r & 31) >> 3) + (r & 3); };

    // ---- producer: a wavefront-wide load fills 1024 bytes of a stage, rows lane / pieces of it.  From one load of a wavefront to its
    // next the lane's logical piece stays the same (the number of wavefronts is even) and its row, a feature's too, moves by a
    // multiple of 32: one offset in a register serves them all.  Rows past the last lie behind the buffer's end by themselves.
    constexpr int XR = 64 / OX::kPieces16, WR = 64 / OW::kPieces16;    // rows of a load
    static_assert(XR * NW % 32 == 0 && WR * NW % 32 == 0 && 16 * NW % 32 == 0, "rows from load to load");
    const int xp = OX::place(XR * wave + lane / OX::kPieces16, lane % OX::kPieces16) * 16;
    const int wp = OW::place(WR * wave + lane / OW::kPieces16, lane % OW::kPieces16) * 16;
    const unsigned xoff = (unsigned)(XR * wave + lane / OX::kPieces16) * ldx + xp;
    const unsigned woff = (unsigned)feature_of(WR * wave + lane / OW::kPieces16) * ldw + wp;
    // scales: a load fills 16 rows of a chunk, rows 0 .. BM-1 the tokens', then the features' in their LDS order.  Which of a row's
    // four words a lane brings is XOR-ed with bits of the row, so that one word of 32 rows lies on 32 banks.
    static_assert(BM % (16 * NW) == 0 && BN % (16 * NW) == 0, "a load of scales has rows of one operand");
    const unsigned sword = (unsigned)((lane & 3) ^ scale_key(16 * wave + lane / 4)) * 4;
    const unsigned xsoff = (unsigned)(16 * wave + lane / 4) * ldxs + sword, wsoff = (unsigned)feature_of(16 * wave + lane / 4) * ldws + sword;
    // load j of a chunk
    auto issue_scales = [&](int j, int chunk) __attribute__((always_inline)) {
        const unsigned dst = (unsigned)__builtin_amdgcn_readfirstlane(
            (int)(lds_base + NST * kStage + (unsigned)(chunk & (NCH - 1)) * kChunk + (unsigned)(wave + NW * j) * 256u));
        const bool x = j < BM / (16 * NW);
        const v4i r = {x ? xsr.x : wsr.x, x ? xsr.y : wsr.y, x ? xsr.z : wsr.z, wsr.w};
        const unsigned moved = x ? (unsigned)j * (16 * NW) * ldxs : (unsigned)(j - BM / (16 * NW)) * (16 * NW) * ldws;
        load_word_to_lds((x ? xsoff : wsoff) + (moved + (unsigned)chunk * 16), r, dst);
    };
    // loads FROM .. TO-1 of a wavefront's LPS for a step (without a branch: the compiler would sink the matrix instructions in front of
    // one behind it)
    auto issue = [&](int step, int stage, auto from, auto to) __attribute__((always_inline)) {
        constexpr int kFrom = decltype(from)::value, kTo = decltype(to)::value;
        const unsigned base = (unsigned)__builtin_amdgcn_readfirstlane((int)(lds_base + (unsigned)stage * kStage + (unsigned)wave * 1024u));
        // (offsets stay below 2^31: out of range is a bit more to add)
        unsigned kx = (unsigned)step * OX::kRow, kw = (unsigned)step * OW::kRow;
        kx += kx + xp < xrow ? 0u : kOutOfRange;
        kw += kw + wp < wrow ? 0u : kOutOfRange;
#pragma unroll
        for (int q = kFrom; q < kTo; q++) {
            const int j = q < XL ? q : q < XL + WL ? q - XL : q - XL - WL;
            if (q < XL) load_piece_to_lds(xoff + j * (XR * NW) * ldx + kx, xr, base + (unsigned)j * (NW * 1024u));
            else if (q < XL + WL) load_piece_to_lds(woff + j * (WR * NW) * ldw + kw, wr, base + (unsigned)(BM * OX::kRow) + (unsigned)j * (NW * 1024u));
            else issue_scales(step % SPC * SL + j, step / SPC + 1);
        }
    };
    // A step's loads are issued one or two at a time between matrix instructions - a burst of them fills the memory pipeline's queue and
    // holds up the wavefront - from slot 0 behind the barrier that frees the stage on: over the rest of the step's last part, and with
    // four parts to a step over the first part of the next step too.  (EXACT: registers for one burst only.)
    constexpr int kLate = EXACT || WHOLE || TM == 1 ? 1 : TM - 1, kSlots = kLate + (KK == 4 && !EXACT && !WHOLE ? TM : 0);
    auto issue_slot = [&](int step, int stage, auto slot) __attribute__((always_inline)) {
        constexpr int s = decltype(slot)::value;
        issue(step, stage, std::integral_constant<int, s * LPS / kSlots>{}, std::integral_constant<int, (s + 1) * LPS / kSlots>{});
    };
    constexpr int kFirst = kLate * LPS / kSlots;                       // loads of a step issued before the next one begins
    using None = std::integral_constant<int, 0>;

    // ---- consumer
    const int wm0 = wave % WM * (BM / WM), wn0 = wave / WM * (BN / WN);
    // Addresses: a lane's row and the key of its pieces are the same in every group of 32 rows; the groups differ by constants.
    const unsigned xlane = (unsigned)(wm0 + l32) * OX::kRow, wlane = (unsigned)(BM * OX::kRow + (wn0 + l32) * OW::kRow);
    const unsigned xkey = OX::place(l32, 0) * 16, wkey = OW::place(l32, 0) * 16;
    const unsigned skey = scale_key(l32) * 4;
    const unsigned xslane = (unsigned)(NST * kStage + (wm0 + l32) * 16), wslane = (unsigned)(NST * kStage + (BM + wn0 + l32) * 16);
    auto read_rows = [&](auto &f, auto op, unsigned at, unsigned key, unsigned scale_at, int kk) __attribute__((always_inline)) {
        constexpr bool wide = decltype(op)::kRow * 8 / KS == 8;
        if constexpr (wide) {
            f.lo = *(const v4i *)(lds + at + (((4 * kk + h) * 16) ^ key));
            f.hi = *(const v4i *)(lds + at + (((4 * kk + 2 + h) * 16) ^ key));
        } else if constexpr (EXACT) {
            typedef int v2i __attribute__((ext_vector_type(2)));
            const v2i p0 = *(const v2i *)(lds + at + ((2 * kk * 16) ^ key) + 8 * h), p1 = *(const v2i *)(lds + at + (((2 * kk + 1) * 16) ^ key) + 8 * h);
            f.lo = v4i{p0[0], p0[1], p1[0], p1[1]};
        } else {
            f.lo = *(const v4i *)(lds + at + (((2 * kk + h) * 16) ^ key));
        }
        if constexpr (EXACT) {
            f.scale = *(const unsigned char *)(lds + scale_at);
            f.scale1 = *(const unsigned char *)(lds + scale_at + 1);
        }
    };
    // 64 values of the reduction axis: part kk of a step
    struct Part {
        int kk;
        unsigned rows, scales;
    };
    auto part_of = [&](int step, int stage, int kk) __attribute__((always_inline)) {
        const int block = (step * KK + kk) * 2;                        // the first of the two
        return Part{kk, (unsigned)stage * kStage, (unsigned)((step / SPC & (NCH - 1)) * kChunk) + ((unsigned)(block & 12) ^ skey) + (unsigned)(block & 2)};
    };
    auto read_w = [&](Frag32<EW, EXACT> &f, int n, const Part &p) __attribute__((always_inline)) {
        read_rows(f, OW{}, p.rows + wlane + n * 32 * OW::kRow, wkey, p.scales + wslane + n * 512, p.kk);
    };
    auto read_x = [&](Frag32<EX, EXACT> &f, int m, const Part &p) __attribute__((always_inline)) {
        read_rows(f, OX{}, p.rows + xlane + m * 32 * OX::kRow, xkey, p.scales + xslane + m * 512, p.kk);
    };
    auto word_w = [&](int n, const Part &p) __attribute__((always_inline)) { return *(const unsigned *)(lds + p.scales + wslane + n * 512); };
    auto word_x = [&](int m, const Part &p) __attribute__((always_inline)) { return *(const unsigned *)(lds + p.scales + xslane + m * 512); };
    // which bytes of this lane's scales count in a part (taken where they are used, not where they are read: no wait there).  Steps with
    // all their blocks go without, their instructions are many beside the few products of a small tile's step (512 x 4096 x 10240 on
    // 4 bits, tiles of 64 x 128: 25.2 us with masks in every step, 22.8 without, 22.1 with the scales as words).
    struct Counts {
        unsigned b0, b1;
    };
    auto counts_of = [&](auto full, int step, int kk) __attribute__((always_inline)) {
        if constexpr (decltype(full)::value) return std::true_type{};
        else {
            const int block = (step * KK + kk) * 2;
            return Counts{block + (EXACT ? 0 : h) < prm.nb ? ~0u : 0u, block + 1 < prm.nb ? ~0u : 0u};
        }
    };
    auto counted = [](unsigned scale, const auto &c, unsigned Counts::*which) __attribute__((always_inline)) {
        if constexpr (std::is_same_v<std::decay_t<decltype(c)>, Counts>) return scale & c.*which;
        else return scale;
    };
    v16f acc[TN][TM] = {};
    auto multiply = [&](auto part, const Frag32<EW, EXACT> (&w)[TN], const unsigned (&ws)[TN], const Frag32<EX, EXACT> &x, unsigned xs, int m, const auto &c) __attribute__((always_inline)) {
        if constexpr (EXACT) {
            auto bf16 = [&](const auto &g, bool wide, int i) __attribute__((always_inline)) {
                const float s = __uint_as_float((i < 2 ? counted(g.scale, c, &Counts::b0) : counted(g.scale1, c, &Counts::b1)) << 23);
                const v4i q = wide && i >= 2 ? g.hi : g.lo;
                return wide ? bf16_of_mx8(q[2 * (i & 1)], q[2 * (i & 1) + 1], s) : bf16_of_mx4(q[i], s);
            };
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const v8bf xb = bf16(x, EX == kMx8, i);
#pragma unroll
                for (int n = 0; n < TN; n++) acc[n][m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bf16(w[n], EW == kMx8, i), xb, acc[n][m], 0, 0, 0);
            }
        } else {
            constexpr int FW = EW == kMx8 ? 0 : 4, FX = EX == kMx8 ? 0 : 4, kByte = decltype(part)::value % 2 * 2;
            auto codes = [](const v4i &lo, const v4i &hi, bool wide) __attribute__((always_inline)) {
                return wide ? v8i{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]} : v8i{lo[0], lo[1], lo[2], lo[3], 0, 0, 0, 0};
            };
#pragma unroll
            for (int n = 0; n < TN; n++)
                acc[n][m] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(codes(w[n].lo, w[n].hi, EW == kMx8), codes(x.lo, x.hi, EX == kMx8), acc[n][m], FW, FX, kByte,
                                                                            (int)counted(ws[n], c, &Counts::b0), kByte, (int)counted(xs, c, &Counts::b0));
        }
    };
    // completes this wavefront's LDS reads, waits for no vector-memory operation
    auto ring_barrier = [&]() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };

    const int steps = prm.steps, full = prm.nb / (2 * KK);             // of them with all their blocks
#pragma unroll
    for (int j = 0; j < SPC * SL; j++) issue_scales(j, 0);
#pragma unroll
    for (int i = 0; i < NST - 1; i++) issue(i, i, None{}, std::integral_constant<int, LPS>{});
    issue(NST - 1, NST - 1, None{}, std::integral_constant<int, kFirst>{});
    wait_loads<(NST - 2) * LPS + kFirst>();
    ring_barrier();
    if constexpr (WHOLE) {
        // Small tiles: a step's operands are read while the step before it is multiplied, into the other of two sets, a few reads and
        // loads behind every matrix instruction (in blocks of reads, loads and products, which the wavefronts go through in step:
        // 256 x 4096 x 4096 on 8 by 4 bits, aligned, a tenth more time).
        struct Set {
            Frag32<EW, EXACT> w[KK][TN];
            Frag32<EX, EXACT> x[KK][TM];
            unsigned ws[KK / 2][TN], xs[KK / 2][TM];
        };
        Set sets[2];
        auto read_part = [&](Set &f, auto part, auto group, int step, int stage) __attribute__((always_inline)) {
            constexpr int kk = decltype(part)::value, m = decltype(group)::value;
            const Part p = part_of(step, stage, kk);
            if constexpr (m == 0) {
#pragma unroll
                for (int n = 0; n < TN; n++) {
                    read_w(f.w[kk][n], n, p);
                    if constexpr (!EXACT && kk % 2 == 0) f.ws[kk / 2][n] = word_w(n, p);
                }
            }
            read_x(f.x[kk][m], m, p);
            if constexpr (!EXACT && kk % 2 == 0) f.xs[kk / 2][m] = word_x(m, p);
        };
        auto do_step = [&](auto whole, Set &now, Set &then, int i, int stage, int next) __attribute__((always_inline)) {
            wait_loads<(NST - 2) * LPS>();
            ring_barrier();                                            // (and every wavefront has read step i)
            static_for<KK>([&](auto part) __attribute__((always_inline)) {
                const auto c = counts_of(whole, i, decltype(part)::value);
                static_for<TM>([&](auto group) __attribute__((always_inline)) {
                    constexpr int kk = decltype(part)::value, m = decltype(group)::value, slot = kk * TM + m;
                    if constexpr (!EXACT && kk % 2 == 0) {
                        if constexpr (m == 0) {
#pragma unroll
                            for (int n = 0; n < TN; n++) now.ws[kk / 2][n] >>= 8 * h;
                        }
                        now.xs[kk / 2][m] >>= 8 * h;
                    }
                    multiply(part, now.w[kk], now.ws[kk / 2], now.x[kk][m], now.xs[kk / 2][m], m, c);
                    __builtin_amdgcn_sched_barrier(0);
                    read_part(then, part, group, i + 1, next);
                    issue(i + NST, stage, std::integral_constant<int, slot * LPS / (KK * TM)>{}, std::integral_constant<int, (slot + 1) * LPS / (KK * TM)>{});
                    __builtin_amdgcn_sched_barrier(0);
                });
            });
        };
        static_for<KK>([&](auto part) __attribute__((always_inline)) {
            static_for<TM>([&](auto group) __attribute__((always_inline)) { read_part(sets[0], part, group, 0, 0); });
        });
        int stage = 0, i = 0;
        auto two_steps = [&](auto whole) __attribute__((always_inline)) {
            const int s1 = stage + 1 == NST ? 0 : stage + 1, s2 = s1 + 1 == NST ? 0 : s1 + 1;
            do_step(whole, sets[0], sets[1], i, stage, s1);
            do_step(whole, sets[1], sets[0], i + 1, s1, s2);
            stage = s2;
        };
        for (; i + 2 <= full; i += 2) two_steps(std::true_type{});
        for (; i < steps; i += 2) two_steps(std::false_type{});        // (a step past the last multiplies zeros)
    } else {
        Frag32<EW, EXACT> fw[2][TN];                                   // this part's and the next one's
        Frag32<EX, EXACT> fx[TM];                                      // each read again as soon as it is multiplied
        unsigned ws[TN], xs[TM], next_ws[TN], next_xs[TM];             // two parts' scales, and the next two's as they are read
        {
            const Part p = part_of(0, 0, 0);
#pragma unroll
            for (int n = 0; n < TN; n++) {
                read_w(fw[0][n], n, p);
                if constexpr (!EXACT) next_ws[n] = word_w(n, p);
            }
#pragma unroll
            for (int m = 0; m < TM; m++) {
                read_x(fx[m], m, p);
                if constexpr (!EXACT) next_xs[m] = word_x(m, p);
            }
        }
        // A step's KK parts.  A token group's operands are read again for the next part as soon as they are multiplied, the features'
        // into the other of two sets.  Behind the first products of a step's last part every read of this step has been made: the
        // wavefronts meet there, the next step having arrived, and the stage is filled again.  Steps past the last are all out of
        // range: their loads bring zeros, touch no memory, and keep one form of the loop.
        int stage = 0, i = 0;
        auto do_step = [&](auto whole) __attribute__((always_inline)) {
            const int next = stage + 1 == NST ? 0 : stage + 1, last = stage == 0 ? NST - 1 : stage - 1;
            static_for<KK>([&](auto part) __attribute__((always_inline)) {
                constexpr int kk = decltype(part)::value;
                const Part p = kk + 1 < KK ? part_of(i, stage, kk + 1) : part_of(i + 1, next, 0);
                const auto c = counts_of(whole, i, kk);
                static_for<TM>([&](auto group) __attribute__((always_inline)) {
                    constexpr int m = decltype(group)::value;
                    if constexpr (!EXACT && kk % 2 == 0) {
                        if constexpr (m == 0) {
#pragma unroll
                            for (int n = 0; n < TN; n++) ws[n] = next_ws[n] >> 8 * h;
                        }
                        xs[m] = next_xs[m] >> 8 * h;
                    }
                    multiply(part, fw[kk & 1], ws, fx[m], xs[m], m, c);
                    __builtin_amdgcn_sched_barrier(0);
                    if constexpr (m == 0) {
                        if constexpr (kk == KK - 1) {
                            wait_loads<(NST - 2) * LPS>();
                            ring_barrier();
                        }
#pragma unroll
                        for (int n = 0; n < TN; n++) {
                            read_w(fw[~kk & 1][n], n, p);
                            if constexpr (!EXACT && kk % 2 == 1) next_ws[n] = word_w(n, p);
                        }
                    }
                    read_x(fx[m], m, p);
                    if constexpr (!EXACT && kk % 2 == 1) next_xs[m] = word_x(m, p);
                    constexpr int late = TM == 1 ? m : m - 1;
                    if constexpr (kk == KK - 1 && late >= 0 && late < kLate) issue_slot(i + NST, stage, std::integral_constant<int, late < 0 ? 0 : late>{});
                    if constexpr (kk == 0 && kSlots > kLate) issue_slot(i + NST - 1, last, std::integral_constant<int, kLate + m>{});
                    __builtin_amdgcn_sched_barrier(0);
                });
            });
            stage = next;
        };
        for (; i < full; i++) do_step(std::true_type{});
        for (; i < steps; i++) do_step(std::false_type{});
    }
    wait_loads<0>();

    // ---- results: lane holds features wn0 + 32n + 16h + 0..15 of token wm0 + 32m + l32.  32 tokens at a time go through the
    // wavefront's own part of LDS, so that a row's features leave in whole cache lines, an octet to a lane.
    constexpr int F = TN * 32, kPad = F + 4;
    static_assert(NW * 32 * kPad * 4 <= NST * kStage + NCH * kChunk, "LDS for the results");
    __syncthreads();                                                   // every wavefront has read its last operands
    float *mine = (float *)lds + wave * 32 * kPad;
    constexpr int kOctets = F / 8, kTokens = 64 / kOctets;             // octets of a token, tokens at a time
    const OctetEnd end(a, (n0 + wn0) / 8 + lane % kOctets);
    const bool inside = mrows == BM && n0 + BN <= a.N && (!a.q.codes || n0 + BN < a.N || a.N % 128 == 0);
    // the largest tiles' results go past the cache where their rows are whole cache lines (8192 x 8192 x 8192 on 4 bits: 14 of 270 us)
    const bool past = BM == 256 && (a.q.codes ? ((uintptr_t)a.q.codes | a.q.ldc) % 128 == 0 : ((uintptr_t)a.y | a.ldy * 2) % 128 == 0);
    with_kind(a, [&](auto kind) __attribute__((always_inline)) {
        static_for<TM>([&](auto group) __attribute__((always_inline)) {
            constexpr int m = decltype(group)::value;
#pragma unroll
            for (int n = 0; n < TN; n++)
#pragma unroll
                for (int q = 0; q < 4; q++)
                    *(v4f *)&mine[l32 * kPad + n * 32 + 16 * h + 4 * q] = v4f{acc[n][m][4 * q], acc[n][m][4 * q + 1], acc[n][m][4 * q + 2], acc[n][m][4 * q + 3]};
            __builtin_amdgcn_wave_barrier();
            auto octet = [&](float (&v)[8], int token) __attribute__((always_inline)) {
                const v4f *p = (const v4f *)&mine[token * kPad + lane % kOctets * 8];
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    v[j] = p[0][j];
                    v[4 + j] = p[1][j];
                }
            };
            const int first = wm0 + m * 32 + lane / kOctets;
            if (inside) {
                float v[32 / kTokens][8];
#pragma unroll
                for (int it = 0; it < 32 / kTokens; it++) octet(v[it], it * kTokens + lane / kOctets);
                if (past) {
#pragma unroll
                    for (int it = 0; it < 32 / kTokens; it++) end.put<decltype(kind)::value, true, BM == 256>(v[it], a, m0 + first + it * kTokens);
                } else {
#pragma unroll
                    for (int it = 0; it < 32 / kTokens; it++) end.put<decltype(kind)::value, true>(v[it], a, m0 + first + it * kTokens);
                }
            } else {
#pragma unroll 1
                for (int it = 0; it < 32; it += kTokens) {
                    float v[8];
                    octet(v, it + lane / kOctets);
                    if (first + it < mrows) end.put<decltype(kind)::value, false>(v, a, m0 + first + it);
                }
            }
            __builtin_amdgcn_wave_barrier();
        });
    });
}

template <int EX, int EW, bool EXACT, int BM, int BN, int WM, int WN, int OCC, int NST, bool WHOLE>
hipError_t run(const LinearMxArgs &a, hipStream_t st)
{
    constexpr int KS = EX == kMx4 && EW == kMx4 ? 256 : 128;
    constexpr int kParts = 512 / KS * WM * WN;                         // loads of scales come in multiples of this
    constexpr int kLds = NST * (BM * Operand<EX, KS>::kRow + BN * Operand<EW, KS>::kRow) + scale_chunks(NST, 512 / KS) * (((BM + BN) / 16 + kParts - 1) / kParts * kParts * 256);
    static_assert(kLds <= kLdsBytes, "LDS of a compute unit");
    const auto kernel = linear_mx_tiles_kernel<EX, EW, EXACT, BM, BN, WM, WN, OCC, NST, WHOLE>;
    static std::atomic<unsigned long long> devices{0};
    const hipError_t allowed = allow_lds((const void *)kernel, kLds, devices);
    if (allowed != hipSuccess) return allowed;
    TileParams p{a, (a.K + kMxBlock - 1) / kMxBlock};
    p.steps = (a.K + KS - 1) / KS;
    p.tiles_n = (a.N + BN - 1) / BN;
    const size_t most = (size_t)(kMostThreads / (WM * WN * 64) / p.tiles_n) * BM;     // token rows of one launch
    for (size_t m = 0; m < a.M; m += most) {
        p.a = a;
        advance_tokens(p.a, m);
        p.a.M = a.M - m < most ? a.M - m : most;
        p.tiles_m = (int)((p.a.M + BM - 1) / BM);
        kernel<<<(unsigned)(p.tiles_m * p.tiles_n), WM * WN * 64, kLds, st>>>(p);
    }
    return hipGetLastError();
}

template <int EX, int EW, bool EXACT>
hipError_t by_shape(const LinearMxArgs &a, LinearMxForm form, hipStream_t st)
{
    switch (form) {
        case LinearMxForm::Tile64x64: return run<EX, EW, EXACT, 64, 64, 2, 2, 3, 3, true>(a, st);
        case LinearMxForm::Tile64x128: return run<EX, EW, EXACT, 64, 128, 2, 2, 2, 3, true>(a, st);
        case LinearMxForm::Tile128x128Deep: return run<EX, EW, EXACT, 128, 128, 2, 4, 2, 3, true>(a, st);
        case LinearMxForm::Tile128x128: return run<EX, EW, EXACT, 128, 128, 2, 2, 2, 2, !(EX == kMx4 && EW == kMx4) && !EXACT>(a, st);
        case LinearMxForm::Tile256x256: return run<EX, EW, EXACT, 256, 256, 2, 4, 2, 2, false>(a, st);
        default: return hipErrorInvalidValue;
    }
}

}  // namespace

hipError_t launch_linear_mx_tiles(const LinearMxArgs &a, LinearMxForm form, hipStream_t st)
{
    const bool exact = a.exact();
    if (a.elem_x == kMx4 && a.elem_w == kMx4) return by_shape<kMx4, kMx4, false>(a, form, st);
    if (a.elem_x == kMx4) return exact ? by_shape<kMx4, kMx8, true>(a, form, st) : by_shape<kMx4, kMx8, false>(a, form, st);
    if (a.elem_w == kMx4) return exact ? by_shape<kMx8, kMx4, true>(a, form, st) : by_shape<kMx8, kMx4, false>(a, form, st);
    return exact ? by_shape<kMx8, kMx8, true>(a, form, st) : by_shape<kMx8, kMx8, false>(a, form, st);
}

}  // namespace dfq
