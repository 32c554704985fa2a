// Product of two tensors held in 8 bits with one scale a row, as a linear layer at serving time reads them:
//     y_mn = sx_m sw_n sum_k x8_mk w8_nk + b_n          x8 [M, K], w8 [N, K] e4m3, sums in fp32, y rounded once
// The scales belong to whole rows, so they leave the sum over k: the contraction runs on the 8-bit values alone
// (v_mfma_f32_32x32x64 / 16x16x128_f8f6f4, twice the rate of 16-bit operands) and the scales meet the finished sums.
//
// Precision: accumulators are fp32.  Within a contraction the unit first adds 8 products of neighbouring k, of each of which it
// drops, towards zero, what lies below 2^-13 of the largest one's power of two (measured: 448 * 448 - 448 * 448 + s gives 0 for
// |s| < 8 and loses the bits below 8 beyond; across groups the sum behaves as fp32).  The price of the doubled rate: 1.5e-5 of the
// result on random data (16-bit outputs round by 2e-4 and 1.6e-3, the operands' own rounding to 8 bits by 2e-2).
//
// Both operands of a contraction hold, in lane l, 32 bytes of row l%32 (l%16): which k a slot stands for is free as long as
// both sides agree.  The weights are the A operand, so a lane's accumulators are consecutive n of one row of y.
#pragma once
#include "avion_common.h"
#include "avion_ln.h"

typedef __attribute__((ext_vector_type(8))) int i32x8;

DEVINL i32x8 join16(u32x4 a, u32x4 b)
{
    return i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
}
// scale operands 0: the form without scales
DEVINL f32x16 mfma8(i32x8 a, i32x8 b, f32x16 c) { return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, 0, 0, 0); }
DEVINL f32x4 mfma8_16(i32x8 a, i32x8 b, f32x4 c) { return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, 0, 0, 0); }

// ------------------------------------------------------------------------------------- few rows
// Bound by the weights' bytes (one token: N K bytes for 2 N K operations) or by latency.  A workgroup takes 16 rows of w8 and
// all rows of x8 (MT tiles of 16); its eight wavefronts take every eighth 128-byte step of K, four steps in flight each, straight
// from memory into the operands (nothing is read twice by a workgroup, so LDS has nothing to give), and add their sums through
// LDS in a fixed order.  1 x 6144 x 4096: 8.0 us, 3.1 TB/s of w8 (25 MB: a launch this short does not reach the copy's 5.2).
constexpr int kFewWaves = 8;
template <int MT, typename E>
__global__ void __launch_bounds__(kFewWaves * 64)
avion_linear_fp8_few_kernel(const char* __restrict__ x8, const float* __restrict__ x_scale, const char* __restrict__ w8,
                            const float* __restrict__ w_scale, const float* __restrict__ bias, raw16* __restrict__ y, int M, int N,
                            int K)
{
    constexpr int FLY = 4;
    __shared__ f32x4 sh[kFewWaves - 1][MT][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, l16 = lane % 16, G = lane / 16;
    const int n0 = blockIdx.x * 16;
    const long wrow = n0 + l16 < N ? n0 + l16 : N - 1;  // a row past the end: any, its sums are not stored
    const char* wp = w8 + wrow * K;
    const char* xp[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) xp[t] = x8 + (long)(16 * t + l16 < M ? 16 * t + l16 : M - 1) * K;
    f32x4 acc[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    const u32x4 zero = {0u, 0u, 0u, 0u};
    const int steps = (K + 127) / 128;
    for (int s0 = wave; s0 < steps; s0 += kFewWaves * FLY) {
        i32x8 w[FLY], x[FLY][MT];
#pragma unroll
        for (int f = 0; f < FLY; ++f) {
            const int k = (s0 + f * kFewWaves) * 128 + 16 * G;  // K is a multiple of 16
            const bool a = k < K, b = k + 64 < K;
            w[f] = join16(a ? *reinterpret_cast<const u32x4*>(wp + k) : zero, b ? *reinterpret_cast<const u32x4*>(wp + k + 64) : zero);
#pragma unroll
            for (int t = 0; t < MT; ++t)
                x[f][t] = join16(a ? *reinterpret_cast<const u32x4*>(xp[t] + k) : zero,
                                 b ? *reinterpret_cast<const u32x4*>(xp[t] + k + 64) : zero);
        }
#pragma unroll
        for (int f = 0; f < FLY; ++f)
#pragma unroll
            for (int t = 0; t < MT; ++t) acc[t] = mfma8_16(w[f], x[f][t], acc[t]);
    }
    if (wave > 0)
#pragma unroll
        for (int t = 0; t < MT; ++t) sh[wave - 1][t][lane] = acc[t];
    __syncthreads();
    const int n = n0 + 4 * G;
    if (wave > 0 || n >= N) return;
    const f32x4 sw = *reinterpret_cast<const f32x4*>(w_scale + n);
    f32x4 b = {0.f, 0.f, 0.f, 0.f};
    if (bias) b = *reinterpret_cast<const f32x4*>(bias + n);
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int m = 16 * t + l16;
        if (m >= M) continue;
#pragma unroll
        for (int w = 0; w < kFewWaves - 1; ++w) acc[t] += sh[w][t][lane];
        const float sx = x_scale[m];
        float o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = fmaf(acc[t][e] * sx, sw[e], b[e]);
        *reinterpret_cast<u32x2*>(y + (long)m * N + n) = u32x2{E::pack(o[0], o[1]), E::pack(o[2], o[3])};
    }
}

// ------------------------------------------------------------------------------------ many rows
// Tiles of TM rows of x8 by TN rows of w8, 128 bytes of K (whole cache lines) at a time, moved global -> LDS by LDS-direct loads
// into one of ST buffers: while a step is multiplied, the next ones are on their way.  With KG = 2 two groups of wavefronts
// take every other step each, for launches whose time is the chain of steps, and add their sums at the end.
// LDS: rows of 128 bytes; the eight 16-byte chunks of a row are permuted by a XOR with bits 1..3 of the row number, so that a
// fragment read (16 consecutive lanes: 16 rows, one chunk) meets 16 different places.
template <int TM, int TN, int WM, int WN, int ST, int KG>
struct Fp8Cfg {
    static constexpr int BK = 128, STAGES = ST, NT = WM * WN * KG * 64;
    static constexpr int MI = TM / WM / 32, NI = TN / WN / 32;  // 32 x 32 tiles of a wavefront
    static constexpr int BLOCKS = (TM + TN) / 8;                // 1 KB loads of a step
    static constexpr int LOADS = BLOCKS / (WM * WN);            // of a wavefront
    static constexpr int STAGE = (TM + TN) * BK;
    static constexpr int LDS_BYTES = STAGE * STAGES * KG;
    static_assert(BLOCKS % (WM * WN) == 0 && TM % 8 == 0 && ST >= 2 && ST <= 6 && (ST - 1) * LOADS < 64, "");
};

// Between the lanes of one wavefront: LDS takes its accesses in the order of the program, which the compiler, looking at one
// lane, is told to keep.
DEVINL void own_lds_written() { asm volatile("" ::: "memory"); }

template <int LOADS>
DEVINL void fp8_landed_barrier()
{
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_waitcnt lgkmcnt(0)\n\ts_barrier" ::"i"(LOADS) : "memory");
}

// This wavefront's reads of LDS are done, and so are everybody's.
DEVINL void read_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <int TM, int TN, int WM, int WN, int ST, int KG, typename E>
__global__ void __launch_bounds__(WM* WN* KG * 64, KG > 1 ? 1 : 2)
avion_linear_fp8_kernel(const char* __restrict__ x8, const float* __restrict__ x_scale, const char* __restrict__ w8,
                        const float* __restrict__ w_scale, const float* __restrict__ bias, raw16* __restrict__ y, int M, int N, int K,
                        int ntn, int ntiles)
{
    using Cfg = Fp8Cfg<TM, TN, WM, WN, ST, KG>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int lane = threadIdx.x % 64, l32 = lane % 32, g = lane / 32;
    const int group = __builtin_amdgcn_readfirstlane(threadIdx.x / (WM * WN * 64)), wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64) % (WM * WN);
    // consecutive tiles on one XCD (workgroups go round the 8 of them): the tiles of one block of x8 share its L2
    const int per = gridDim.x / 8, tile = (blockIdx.x % 8) * per + blockIdx.x / 8;
    if (tile >= ntiles) return;
    const int m0 = tile / ntn * TM, n0 = tile % ntn * TN;
    const int rows_m = M - m0 < TM ? M - m0 : TM, rows_n = N - n0 < TN ? N - n0 : TN;
    const RawBuffer xb(x8 + (long)m0 * K, (unsigned)rows_m * (unsigned)K), wb(w8 + (long)n0 * K, (unsigned)rows_n * (unsigned)K);
    const unsigned lds = lds_address(smem) + group * (Cfg::STAGE * ST);  // each group of wavefronts has its own steps and buffers

    // 1 KB block b of a step: rows 8 b .. 8 b + 7 (x8's, then w8's); lane i brings the chunk that lies at 16 i
    const unsigned ch = ((lane & 7) ^ (lane >> 4 & 3)) * 16;
    unsigned voff[Cfg::LOADS];
#pragma unroll
    for (int i = 0; i < Cfg::LOADS; ++i) {
        const int b = wave + i * WM * WN;
        const int row = (b < TM / 8 ? b : b - TM / 8) * 8 + lane / 8;
        voff[i] = (unsigned)row * (unsigned)K;
    }
    auto fetch = [&](int step, int buf) {
        const unsigned k = (unsigned)(step * KG + group) * Cfg::BK;
#pragma unroll
        for (int i = 0; i < Cfg::LOADS; ++i) {
            const int b = wave + i * WM * WN;
            const unsigned at = k + (ch ^ ((b & 1) * 64));
            load_to_lds16(pick(b < TM / 8, xb, wb), lds + buf * Cfg::STAGE + b * 1024, at < (unsigned)K ? voff[i] + at : kOutOfRangeBase);
        }
    };

    const int wm = wave / WN, wn = wave % WN;
    const unsigned swz = (l32 >> 1 & 7);
    const unsigned a0 = lds + TM * Cfg::BK + (wn * Cfg::NI * 32 + l32) * Cfg::BK, b0 = lds + (wm * Cfg::MI * 32 + l32) * Cfg::BK;
    const unsigned c0 = (g ^ swz) * 16, c1 = ((g + 2) ^ swz) * 16;  // of the first 64 bytes; the second: bit 6 turned
    typedef const __attribute__((address_space(3))) u32x4* ptr;

    f32x16 acc[Cfg::MI][Cfg::NI];
#pragma unroll
    for (int i = 0; i < Cfg::MI; ++i)
#pragma unroll
        for (int j = 0; j < Cfg::NI; ++j) acc[i][j] = f32x16_zero();

    const int steps = (K + Cfg::BK * KG - 1) / (Cfg::BK * KG);
#pragma unroll
    for (int i = 0; i < ST; ++i)
        if (i < steps) fetch(i, i);
    // `left`: steps behind the awaited one that have been asked for
    auto landed = [&](int left) {
        switch (min(left, ST - 1)) {
            case 5: fp8_landed_barrier<5 * Cfg::LOADS>(); break;
            case 4: fp8_landed_barrier<4 * Cfg::LOADS>(); break;
            case 3: fp8_landed_barrier<3 * Cfg::LOADS>(); break;
            case 2: fp8_landed_barrier<2 * Cfg::LOADS>(); break;
            case 1: fp8_landed_barrier<Cfg::LOADS>(); break;
            default: fp8_landed_barrier<0>();
        }
    };
    auto read = [&](unsigned base, unsigned half) { return join16(*(ptr)(base + (c0 ^ half)), *(ptr)(base + (c1 ^ half))); };
    i32x8 a[2][Cfg::NI], b;
    landed(min(steps - 1, ST - 1));
#pragma unroll
    for (int j = 0; j < Cfg::NI; ++j) a[0][j] = read(a0 + j * 32 * Cfg::BK, 0);
    b = read(b0, 0);
    int buf = 0;
    // The operands of each group of contractions are read while the group before runs.  Before the last group of a step the
    // next step's tile is awaited (by then this step's has been read by everybody: its buffer is filled again).
    for (int s = 0; s < steps; ++s) {
        const unsigned at = buf * Cfg::STAGE;
#pragma unroll
        for (int gr = 0; gr < 2 * Cfg::MI; ++gr) {
            const int i = gr % Cfg::MI, half = gr / Cfg::MI;
            i32x8 b_next = b;
            if (i + 1 < Cfg::MI) {
                b_next = read(b0 + at + (i + 1) * 32 * Cfg::BK, half * 64);
            } else if (half == 0) {
#pragma unroll
                for (int j = 0; j < Cfg::NI; ++j) a[1][j] = read(a0 + at + j * 32 * Cfg::BK, 64);
                b_next = read(b0 + at, 64);
            } else if (s + 1 < steps) {
                landed(min(steps - 2 - s, ST - 2));
                if (s + ST < steps) fetch(s + ST, buf);
                const unsigned next = (buf + 1 == ST ? 0 : buf + 1) * Cfg::STAGE;
#pragma unroll
                for (int j = 0; j < Cfg::NI; ++j) a[0][j] = read(a0 + next + j * 32 * Cfg::BK, 0);
                b_next = read(b0 + next, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < Cfg::NI; ++j) acc[i][j] = mfma8(a[half][j], b, acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
            b = b_next;
        }
        buf = buf + 1 == ST ? 0 : buf + 1;
    }

    // Lane l holds row l%32 of a 32 x 32 tile of y; registers 4 q .. 4 q + 3 are its columns 8 q + 4 g ...  The scaled and
    // rounded tile goes through LDS (rows 16 bytes longer than their data: an odd multiple of 16 bytes), so that the stores
    // write whole rows of the wavefront's tile: 64 to 128 consecutive bytes each.
    constexpr int ROW = Cfg::NI * 64 + 16, LANES = Cfg::NI * 4, ROWS = 64 / LANES;  // bytes of a row, lanes and rows of a store
    static_assert(WM * WN * 32 * ROW <= Cfg::LDS_BYTES, "");
    const int n_wave = n0 + wn * Cfg::NI * 32, m_wave = m0 + wm * Cfg::MI * 32;
    f32x4 sw[Cfg::NI][4], bb[Cfg::NI][4];
    float sx[Cfg::MI];
#pragma unroll
    for (int j = 0; j < Cfg::NI; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int n = min(n_wave + 32 * j + 8 * q + 4 * g, N - 4);  // (past the end: anything)
            sw[j][q] = *reinterpret_cast<const f32x4*>(w_scale + n);
            bb[j][q] = bias ? *reinterpret_cast<const f32x4*>(bias + n) : f32x4{0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll
    for (int i = 0; i < Cfg::MI; ++i) sx[i] = x_scale[min(m_wave + 32 * i + l32, M - 1)];
    __syncthreads();  // everybody has read the last step's buffer
    if constexpr (KG > 1) {
        // the groups' sums, in the groups' order
        static_assert(Cfg::MI * Cfg::NI * WM * WN * 4096 <= Cfg::STAGE * ST && KG == 2, "");
        f32x16* sums = reinterpret_cast<f32x16*>(smem + Cfg::STAGE * ST) + wave * (Cfg::MI * Cfg::NI * 64) + lane;
#pragma unroll
        for (int i = 0; i < Cfg::MI; ++i)
#pragma unroll
            for (int j = 0; j < Cfg::NI; ++j)
                if (group == 1) sums[(i * Cfg::NI + j) * 64] = acc[i][j];
        __syncthreads();
        if (group == 1) return;
#pragma unroll
        for (int i = 0; i < Cfg::MI; ++i)
#pragma unroll
            for (int j = 0; j < Cfg::NI; ++j) acc[i][j] += sums[(i * Cfg::NI + j) * 64];
    }
    char* out = smem + wave * (32 * ROW);
    const int n = n_wave + lane % LANES * 8;
#pragma unroll
    for (int i = 0; i < Cfg::MI; ++i) {
#pragma unroll
        for (int j = 0; j < Cfg::NI; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float o[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = fmaf(acc[i][j][4 * q + e] * sx[i], sw[j][q][e], bb[j][q][e]);
                *reinterpret_cast<u32x2*>(out + l32 * ROW + 64 * j + 16 * q + 8 * g) = u32x2{E::pack(o[0], o[1]), E::pack(o[2], o[3])};
            }
        own_lds_written();
#pragma unroll
        for (int r = 0; r < 32; r += ROWS) {
            const int row = r + lane / LANES, m = m_wave + 32 * i + row;
            const u32x4 v = *reinterpret_cast<const u32x4*>(out + row * ROW + lane % LANES * 16);
            if (m < M && n < N) *reinterpret_cast<u32x4*>(y + (long)m * N + n) = v;
        }
        own_lds_written();
    }
}

// ---------------------------------------------------------------------------------- whole chip
// Tiles of 256 x 256 by one workgroup of eight wavefronts (128 x 64 each) per compute unit, which walks over its tiles without
// a pause between them: the tiles' steps form one stream, two steps of 128 bytes of K in LDS, and the next tile's first steps
// are on their way while a tile's sums are scaled, rounded and stored.
//   Tile size: LDS reads for a step's 2048 MFMA cycles are 1536 (128 x 64 a wavefront), reads from L2 half of what tiles of
//   128 x 128 ask for.  128 bytes of K: whole cache lines; with 64 the same bytes took twice the requests.
//   Order: an XCD owns a run of tiles, and its workgroups' 32 tiles at a time are 8 blocks of x8 by 4 of w8, so that what they
//   share stays in its L2.
//   Waits: a step's loads are awaited with everything older; stores of a tile are younger than the loads that the next tile's
//   first step awaits, so that wait leaves them (kWideStores of them, all issued always) on their way.
//   AHEAD, for long K: w8's half of a buffer, whose rows are all in registers from the middle of a step on, is filled again from
//   there, behind a barrier of its own.  50176 x 1024 x 4096 220 -> 202 us, 50176 x 768 x 2304 99 -> 92, 8192 cubed 434 -> 416;
//   with fewer steps a tile it gives nothing or costs: 25088 x 2048 x 1536 89 and 90, 12544 x 4096 x 1024 65 and 68.
// Bound by two things in turn.  50176 x 2304 x K, back to back and without AHEAD, takes 65, 82, 102, 122 and 166 us at K = 256, 512,
// 768, 1024 and 1536: 9.6 us a step of K and 46 that do not depend on it.  A step of a tile is 1.4 us, 0.85 of them contractions; the rest
// waits for its loads, all that two buffers of 64 KB leave in flight.  The 46, 6.6 us for each of a workgroup's seven tiles, are the
// scaling, exchange and stores of y (44 at the copy's rate), beside which nobody contracts.  No part alone is the bound: at K = 768
// it takes 80 us without loads, 69 without contractions, 7 less without stores.  That case: 93 (in the profiler) to 102 us, 1.9 to
// 1.7 PFLOP/s, matrix units 35 % of the cycles, LDS reads 24 %.  8192 cubed: 2.64 PFLOP/s.
constexpr int kWideM = 256, kWideN = 256, kWideK = 128, kWideWaves = 8, kWideGroup = 8;
constexpr int kWideStage = (kWideM + kWideN) * kWideK, kWideScales = 3 * 1024, kWideRow = 144;
constexpr int kWideLds = 2 * kWideStage + 3 * kWideScales + kWideWaves * 16 * kWideRow;
constexpr int kWideStores = 16;
constexpr int kWideAhead = 2048;  // AHEAD from this K on
constexpr int kNontemporal = 2;  // of a buffer access's cache policy

template <typename E, bool STREAM, bool AHEAD>
__global__ void __launch_bounds__(kWideWaves * 64)
avion_linear_fp8_wide_kernel(const char* __restrict__ x8, const float* __restrict__ x_scale, const char* __restrict__ w8,
                             const float* __restrict__ w_scale, const float* __restrict__ bias, raw16* __restrict__ y, int M, int N,
                             int K, int ntm, int ntn)
{
    extern __shared__ __attribute__((aligned(16))) char smem[];
    constexpr int MI = 4, NI = 2, LOADS = (kWideM + kWideN) / 8 / kWideWaves;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l32 = lane % 32, g = lane / 32;
    const int wm = wave / 4, wn = wave % 4;
    const int ntiles = ntm * ntn, per = (ntiles + 7) / 8, xcd = blockIdx.x % 8, together = gridDim.x / 8;
    const int first = xcd * per + blockIdx.x / 8, end = min(ntiles, (xcd + 1) * per);
    if (first >= end) return;
    const int steps = (K + kWideK - 1) / kWideK, total = ((end - first + together - 1) / together) * steps;
    const unsigned lds = lds_address(smem);

    // tile number -> its rows of x8 and of w8: groups of kWideGroup blocks of x8, block by block of w8
    auto place = [&](int tile, int& m0, int& n0) {
        const int group = tile / (kWideGroup * ntn), in = tile - group * kWideGroup * ntn;
        const int blocks = min(kWideGroup, ntm - group * kWideGroup), n = in / blocks;
        n0 = n * kWideN;
        m0 = (group * kWideGroup + in - n * blocks) * kWideM;
    };

    // The stream of loads.  1 KB block b of a step: rows 8 b .. 8 b + 7 (x8's, then w8's), 128 bytes each; lane i brings the
    // chunk that lies at 16 i: the eight chunks of a row are permuted by a XOR with bits 1..3 of the row number.  A wavefront
    // brings every eighth block.
    const unsigned ch = ((lane & 7) ^ (lane >> 4 & 3) ^ (wave & 1) * 4) * 16, row_at = (unsigned)(wave * 8 + lane / 8) * (unsigned)K + ch;
    int f_tile = first, f_step = 0, f_buf = 0, f_scales = 0;
    RawBuffer xb(x8, 0), wb(w8, 0);
    auto fetch_tile = [&] {  // before a step's loads: the next tile, if this is its first step
        if (f_step == 0) {
            int m0, n0;
            place(f_tile, m0, n0);
            const int rows_m = min(kWideM, M - m0), rows_n = min(kWideN, N - n0);
            xb = RawBuffer(x8 + (long)m0 * K, (unsigned)rows_m * (unsigned)K);
            wb = RawBuffer(w8 + (long)n0 * K, (unsigned)rows_n * (unsigned)K);
            // the tile's scales and biases, 1 KB each
            const unsigned into = lds + 2 * kWideStage + f_scales * kWideScales;
            if (wave == 0) load_to_lds16(RawBuffer(x_scale + m0, rows_m * 4), into, lane * 16);
            if (wave == 1) load_to_lds16(RawBuffer(w_scale + n0, rows_n * 4), into + 1024, lane * 16);
            if (wave == 2 && bias) load_to_lds16(RawBuffer(bias + n0, rows_n * 4), into + 2048, lane * 16);
        }
    };
    auto fetch_half = [&](const RawBuffer& buffer, unsigned to) {
        const unsigned k = (unsigned)f_step * kWideK, v = k + ch < (unsigned)K ? row_at + k : kOutOfRangeBase;
        const unsigned down = 8 * kWideWaves * (unsigned)K;
        load_to_lds16_x4<kWideWaves * 1024>(buffer, buffer, buffer, buffer, lds + f_buf * kWideStage + to + wave * 1024, v, v + down,
                                            v + 2 * down, v + 3 * down);
    };
    auto fetch_w = [&] { fetch_half(wb, kWideM * kWideK); };
    auto fetch_x = [&] { fetch_half(xb, 0); };
    auto fetched = [&] {
        f_buf ^= 1;
        if (++f_step == steps) {
            f_step = 0;
            f_tile += together;
            f_scales = f_scales == 2 ? 0 : f_scales + 1;
        }
    };

    const unsigned swz = l32 >> 1 & 7, c0 = (g ^ swz) * 16, c1 = ((g + 2) ^ swz) * 16;  // of a row's first 64 bytes; the second: bit 6 turned
    const unsigned a0 = lds + kWideM * kWideK + (wn * NI * 32 + l32) * kWideK, b0 = lds + (wm * MI * 32 + l32) * kWideK;
    typedef const __attribute__((address_space(3))) u32x4* ptr;
    auto read = [&](unsigned base, unsigned half) { return join16(*(ptr)(base + (c0 ^ half)), *(ptr)(base + (c1 ^ half))); };

    f32x16 acc[MI][NI];
    i32x8 a[2][NI], b;
    auto fetch = [&] {
        fetch_tile();
        fetch_x();
        fetch_w();
        fetched();
    };
    fetch();
    if (total > 1) {
        fetch();
        fp8_landed_barrier<LOADS>();  // (the second step's loads are the youngest; scales among them are waited for with the first)
    } else {
        fp8_landed_barrier<0>();
    }
#pragma unroll
    for (int j = 0; j < NI; ++j) a[0][j] = read(a0 + j * 32 * kWideK, 0);
    b = read(b0, 0);
    int buf = 0, scales = 0, q = 0;
    for (int tile = first; tile < end; tile += together) {
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[i][j] = f32x16_zero();
        // The operands of each group of contractions are read while the group before runs.  Before the last group of a step the
        // next step is awaited (by then this one has been read by everybody: its buffer is filled again).
        for (int s = 0; s < steps; ++s, ++q) {
            const unsigned at = buf * kWideStage, next = kWideStage - at;
#pragma unroll
            for (int gr = 0; gr < 2 * MI; ++gr) {
                const int i = gr % MI, half = gr / MI;
                i32x8 b_next = b;
                if (AHEAD && gr == MI + 1 && q + 2 < total) {
                    read_barrier();  // w8's rows of this step are in everybody's registers
                    fetch_tile();
                    fetch_w();
                }
                if (i + 1 < MI) {
                    b_next = read(b0 + at + (i + 1) * 32 * kWideK, half * 64);
                } else if (half == 0) {
#pragma unroll
                    for (int j = 0; j < NI; ++j) a[1][j] = read(a0 + at + j * 32 * kWideK, 64);
                    b_next = read(b0 + at, 64);
                } else if (q + 1 < total) {
                    const bool after = s == 0 && q > 0;  // a tile's stores
                    if (AHEAD && q + 2 < total) {
                        if (after) fp8_landed_barrier<kWideStores + LOADS / 2>();
                        else fp8_landed_barrier<LOADS / 2>();
                    } else {
                        if (after) fp8_landed_barrier<kWideStores>();
                        else fp8_landed_barrier<0>();
                    }
#pragma unroll
                    for (int j = 0; j < NI; ++j) a[0][j] = read(a0 + next + j * 32 * kWideK, 0);
                    b_next = read(b0 + next, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = 0; j < NI; ++j) acc[i][j] = mfma8(a[half][j], b, acc[i][j]);
                __builtin_amdgcn_sched_barrier(0);
                b = b_next;
            }
            if (q + 2 < total) {
                if (!AHEAD) fetch_tile();
                fetch_x();
                if (!AHEAD) fetch_w();
                fetched();
            }
            buf ^= 1;
        }

        // Lane l holds row l%32 of a 32 x 32 tile of y; registers 4 q .. 4 q + 3 are its columns 8 q + 4 g ...  16 rows at a
        // time go through LDS (rows of 144 bytes), so that the stores write 128 consecutive bytes a row.
        int m0, n0;
        place(tile, m0, n0);
        const int rows_m = min(kWideM, M - m0);
        const __amdgpu_buffer_rsrc_t out =
            __builtin_amdgcn_make_buffer_rsrc(y + (long)m0 * N, 0, (int)((unsigned)rows_m * (unsigned)N * 2), 0x00020000);
        const char* sc = smem + 2 * kWideStage + scales * kWideScales;
        char* stage = smem + 2 * kWideStage + 3 * kWideScales + wave * (16 * kWideRow);
        const int col = n0 + wn * 64 + lane % 8 * 8;
        const unsigned col_at = col < N ? (unsigned)col * 2 : kOutOfRangeBase;
        f32x4 sw[NI][4], bb[NI][4];
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const char* at = sc + 1024 + (wn * 64 + 32 * j + 8 * c + 4 * g) * 4;
                sw[j][c] = *reinterpret_cast<const f32x4*>(at);
                bb[j][c] = bias ? *reinterpret_cast<const f32x4*>(at + 1024) : f32x4{0.f, 0.f, 0.f, 0.f};
            }
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const float sx = *reinterpret_cast<const float*>(sc + (wm * 128 + 32 * i + l32) * 4);
            u32x4 p[NI][2];
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                u32x2 d[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    float o[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] = fmaf(acc[i][j][4 * c + e] * sx, sw[j][c][e], bb[j][c][e]);
                    d[c] = u32x2{E::pack(o[0], o[1]), E::pack(o[2], o[3])};
                }
                // quarters exchanged between the wavefront's halves: 8 consecutive columns a lane
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const auto r0 = __builtin_amdgcn_permlane32_swap(d[2 * c][0], d[2 * c + 1][0], false, false);
                    const auto r1 = __builtin_amdgcn_permlane32_swap(d[2 * c][1], d[2 * c + 1][1], false, false);
                    p[j][c] = u32x4{r0[0], r1[0], r0[1], r1[1]};
                }
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                if (l32 / 16 == half)
#pragma unroll
                    for (int j = 0; j < NI; ++j)
#pragma unroll
                        for (int c = 0; c < 2; ++c)
                            *reinterpret_cast<u32x4*>(stage + l32 % 16 * kWideRow + 64 * j + 32 * c + 16 * g) = p[j][c];
                own_lds_written();
#pragma unroll
                for (int r = 0; r < 16; r += 8) {
                    const u32x4 v = *reinterpret_cast<const u32x4*>(stage + (r + lane / 8) * kWideRow + lane % 8 * 16);
                    const unsigned row = wm * 128 + 32 * i + 16 * half + r + lane / 8;
                    __builtin_amdgcn_raw_buffer_store_b128(v, out, col_at == kOutOfRangeBase ? kOutOfRangeBase : row * (unsigned)N * 2 + col_at,
                                                           0, STREAM ? kNontemporal : 0);
                }
                own_lds_written();
            }
        }
        scales = scales == 2 ? 0 : scales + 1;
    }
}
