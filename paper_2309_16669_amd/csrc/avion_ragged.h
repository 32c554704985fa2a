// Attention over sequences of different lengths that lie one after the other, with query heads that share key heads.
//
//   q [Tq, Hq, d], k and v [Tk, Hk, d], G = Hq / Hk query heads a key head; sequence s owns queries bq[s] .. bq[s+1]-1 and keys
//   bk[s] .. bk[s+1]-1 (nq and nk of them).  Per sequence and head O = softmax(scale Q K^T) V; under a causal mask query i sees the
//   keys up to i + nk - nq: the last query stands beside the last key, whether the queries are a whole prompt, its end, or one
//   token behind a cache.  A query that sees no key has O = 0 and LSE = -inf, and no gradient.
//
// Rows.  For one key head all G heads of a query read the same keys, so the kernels' rows are (query, head) pairs, row r = query
// r / G, head r % G: one token of 8 heads is a tile of 8 rows that reads the cache once, and a prompt's tile of 32 rows is 8
// queries of 4 heads, which all end at nearly the same key.
//
// Slots.  How many blocks of BM rows a sequence has is known on the device only.  A launch has floor(T / BM) + S + 2 slots a head,
// of which sequence s owns those from floor(begin_s / BM) + s on: at least as many as it has blocks.  A workgroup finds its
// sequence by a search over the offsets of which a wavefront probes 63 at a time, and leaves if its block is past the
// end.  The rows before the first and behind the last offset are two more "sequences", whose outputs become zeros.  Offsets are
// read as they come: each border is held inside the tensor, so that no content of them leads out of it.
//
// Masks.  All keys of a tile beyond the sequence arrive as zero rows; the scores that a query must not see start from -1e30 as in the
// other kernels, in the units that need it.  Nothing of a sequence is ever multiplied with another's rows, so what one holds
// (infinities, NaN, an unused slot) cannot reach the next.  Within a sequence a masked key's weight is 0, which NaN and infinity
// in its value survive, as in avion_attn_fwd.
#pragma once
#include "avion_bwd.h"
#include "avion_common.h"
#include "avion_ragged_search.h"

struct RaggedArgs {
    const raw16 *q, *k, *v;
    const int *off_q, *off_k;
    long rs_q, rs_k, rs_v;  // token rows of q, k, v, elements apart; of o and the gradients Hq d and Hk d
    int S, Tq, Tk, Hq, Hk, G;
    unsigned g_mul, g_shift;  // of over_heads()
    int slots;
    int done;               // forward: sequences of at most so many rows are avion_ragged_few_kernel's, the others the next launch's (0:
                            // one of the two has all); backward: those of at most so many queries and keys are
                            // avion_ragged_whole_kernel's (0: none)
    int* more;              // and whether there are others, as that kernel has found
    int causal;
    float cs, scale;        // scale * log2 e, scale
    // r / G for 0 <= r < 2^31: multiplication by 2^(32 + shift) / G, whose 33rd bit is the addition (a division by a number known at run
    // time is some 25 instructions, of which a wavefront with one short sequence would spend more than on the softmax)
    DEVINL int over_heads(int r) const { return (int)((__umulhi(g_mul, (unsigned)r) + (unsigned)r) >> g_shift); }
};

// The lanes of a wavefront that search in device memory (see ragged_search)
struct RaggedLanes {
    const int* off;
    int S, T, lane, border;
    DEVINL void load(int lo, int step) { border = ragged_border(off, S, T, lo + lane * step); }
    template <typename F>
    DEVINL int count(F begun) const
    {
        return (int)__popcll(__ballot(begun(lane, border)));
    }
    DEVINL int at(int l) const { return __builtin_amdgcn_readlane(border, l); }
};
// The interval that owns `slot`, for blocks of 2^SHIFT rows and `mul` rows a token.  Wavefront-uniform.
template <int SHIFT>
DEVINL RaggedPlace ragged_place(const int* off, int S, int T, int mul, long slot, int lane)
{
    RaggedLanes lanes{off, S, T, lane, 0};
    return ragged_search<SHIFT>(lanes, S, mul, slot);
}
// Over the lanes up to each: the sum, the largest
DEVINL int lanes_sum(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // 1, 2, 4 and 8 lanes down a row of 16
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // a row's last lane to the next row, the second row's to both behind
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    return x;
}
DEVINL int lanes_max(int x)
{
    x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x111, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x112, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x114, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x118, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x142, 0xa, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(x, x, 0x143, 0xc, 0xf, false));
    return x;
}
// The block whose turn it is, the `turn`th of those that begin.  Up to kRaggedOrdered sequences, of which a lane holds one, begin in up
// to eight classes by the tokens on the other side, the most first (the three highest bits that there are), rows of no sequence in the last
// one; all blocks of a sequence together, the last of them first where it sees the most (BACK).  The launch then ends with its
// shortest workgroups.  More sequences keep their order, from the last one on with BACK.
// 16 sequences of 196 to 3136 tokens, 12 heads, 64 channels, forward, dQ and dK/dV, best launches: 80 + 92 + 113 us, in four classes
// 83 + 95 + 118, in their own order 103 + 116 + 132; 37 of 400 to 1100, 16 heads on 2 of 80, all passes 125, wholly sorted (40 steps of a search
// in every wavefront) 130
constexpr int kRaggedOrdered = 61;
template <int SHIFT, bool BACK>
DEVINL RaggedPlace ragged_turn(const int* off, int S, int T, int mul, const int* other, int others, int slots, int turn, int lane)
{
    if (S > kRaggedOrdered) return ragged_place<SHIFT>(off, S, T, mul, BACK ? slots - 1 - turn : turn, lane);
    const int begin = ragged_border(off, S, T, lane), n = lane > S + 1 ? 0 : max(ragged_border(off, S, T, lane + 1) - begin, 0);
    const bool sequence = lane > 0 && lane <= S;
    const int seen = sequence ? max(ragged_border(other, S, others, lane + 1) - ragged_border(other, S, others, lane), 0) : -1;
    const int blocks = (int)(((long)n * mul + (1 << SHIFT) - 1) >> SHIFT);
    const int most = __builtin_amdgcn_readlane(lanes_max(seen), 63), shift = max(29 - __clz(most | 1), 0), rank = min((most >> shift) - (seen >> shift), 7);
    int before = 0, begun = 0;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const int upto = lanes_sum(rank == c ? blocks : 0);
        before = rank == c ? begun + upto - blocks : before;
        begun += __builtin_amdgcn_readlane(upto, 63);
    }
    const unsigned long long owner = __ballot(turn >= before && turn - before < blocks);
    if (owner == 0) return RaggedPlace{0, 0, 0, 0};
    const int i = __builtin_ctzll(owner), in = turn - __builtin_amdgcn_readlane(before, i);
    return RaggedPlace{i, __builtin_amdgcn_readlane(begin, i), __builtin_amdgcn_readlane(n, i), BACK ? __builtin_amdgcn_readlane(blocks, i) - 1 - in : in};
}
// The other side's tokens of the interval: begin and number
DEVINL int2 ragged_tokens(const int* off, int S, int T, int i)
{
    const int begin = ragged_border(off, S, T, i);
    return int2{begin, max(ragged_border(off, S, T, i + 1) - begin, 0)};
}

// How a kernel cuts its work.  A workgroup: NW wavefronts of 32 rows (keys in dK/dV) each, in KG groups that walk over a share of the
// other side's tiles through buffers of their own and add their sums up at the end; tiles of ROWS tokens in NBUF buffers.
//   RaggedWide   the usual one
//   RaggedSplit, RaggedSplitHalf, RaggedSplit4   where such workgroups would leave compute units without work, or with one of two:
//                shorter walks of fewer rows
//   RaggedShort  sequences of less than two wavefronts' rows: one wavefront with one buffer of 32 rows, so that 16 of a compute unit
//                wait for their loads at once; four of them, which know nothing of each other, to a workgroup (JOBS)
//   RaggedLone   single tokens behind long caches
template <int NW_, int KG_, int ROWS_, int NBUF_, int JOBS_>
struct RaggedCut {
    static constexpr int NW = NW_, KG = KG_, ROWS = ROWS_, NBUF = NBUF_, JOBS = JOBS_;
    static constexpr int BLOCK = 32 * NW, SHIFT = NW == 4 ? 7 : NW == 2 ? 6 : 5, NT = NW * KG * 64;  // rows, their logarithm, threads of a job
    static_assert(NBUF == 2 || KG == 1, "");
};
using RaggedWide = RaggedCut<4, 1, 64, 2, 1>;
using RaggedSplit = RaggedCut<2, 2, 64, 2, 1>;
using RaggedSplitHalf = RaggedCut<2, 2, 32, 2, 1>;
using RaggedSplit4 = RaggedCut<1, 4, 32, 2, 1>;
using RaggedShort = RaggedCut<1, 1, 32, 1, 4>;
using RaggedLone = RaggedCut<1, 1, 64, 2, 1>;

// NBUF buffers in LDS of an A and a B tile of ROWS token rows each (and, with SCALARS, ROWS + ROWS floats), filled by LDS-direct loads
// as TileRing's.  The descriptors begin at the tile's own first row, so that no length of a sequence and no row stride takes a
// byte offset past 32 bits; rows past the end arrive as zeros.
// Layout of a tile: at 64 channels quad_at's (no bank conflicts, and two addresses a lane for the loads of both tensors instead of one
// for each load: where registers are scarce, in dK/dV, that is what keeps the accumulators out of scratch), at 128 two such halves one
// after the other (padded rows' bank conflicts took 30 % of the cycles: prompts of 500 to 8000 tokens, 32 heads on 8, 690 -> 665 us a call on one card), else
// padded rows.
template <int D, typename Cut, bool SCALARS>
struct RaggedRing {
    static constexpr int NW = Cut::NW, ROWS = Cut::ROWS, NBUF = Cut::NBUF, STRIDE = tile_stride<D>();
    static constexpr bool QUAD = D % 64 == 0;
    static constexpr int HALF = ROWS / 8;  // blocks of 64 channels of a tile
    // 1 KB blocks of a tile (the last one's rows past the tile, where there are any, are not read)
    static constexpr int NTI = QUAD ? D / 64 * HALF : (ROWS * STRIDE + 1023) / 1024, NBLK = 2 * NTI, NPW = (NBLK + NW - 1) / NW;
    static_assert(!QUAD || (HALF % NW == 0 && HALF % 2 == 0 && (NW == 1 || NW % 2 == 0)), "a load's blocks belong to 64 channels of one tensor, a wavefront's are all even or all odd");
    static constexpr int OFF_B = NTI * 1024, OFF_SCALARS = 2 * NTI * 1024;
    static constexpr int BUF_BYTES = NBLK * 1024 + (SCALARS ? 1024 : 0);
    static constexpr int LDS_BYTES = NBUF * BUF_BYTES + (D % 32 != 0 ? 64 : 0);

    const raw16 *a, *b;
    const float* scalars;
    long rs_a, rs_b;
    int n, wave;
    unsigned smem_addr, npad_bytes, scalar_voff;
    unsigned place[QUAD ? 3 : NPW];  // of this lane: rows of a and b, and the chunk; or each load's byte offset

    // a, b: first rows, rs_a and rs_b elements apart, n of them; scalars: two arrays npad floats apart
    DEVINL RaggedRing(const raw16* a_, long rs_a_, const raw16* b_, long rs_b_, const float* scalars_, int npad, int n_, char* smem,
                      int wave_, int lane)
        : a(a_), b(b_), scalars(scalars_), rs_a(rs_a_), rs_b(rs_b_), n(n_), wave(wave_), smem_addr(lds_address(smem)),
          npad_bytes((unsigned)npad * 4)
    {
        if constexpr (QUAD) {
            const unsigned row = 8 * wave + lane / 32 * 4 + lane / 4 % 4;
            place[0] = row * (unsigned)(rs_a * 2);
            place[1] = row * (unsigned)(rs_b * 2);
            place[2] = (lane / 16 % 2 * 4 + ((lane ^ (row >> 2)) & 3)) * 16;
        } else {
#pragma unroll
            for (int j = 0; j < NPW; ++j) {
                const int blk = wave + NW * j;
                const bool first = blk < NTI;
                place[j] = padded_block_voff<D>(first ? blk : blk - NTI, lane, (unsigned)((first ? rs_a : rs_b) * 2));
            }
        }
        if constexpr (SCALARS)
            scalar_voff = lane < ROWS / 4 ? (unsigned)lane * 16 : lane < ROWS / 2 ? npad_bytes + (lane - ROWS / 4) * 16 : kOutOfRangeBase;
    }
    // this lane's byte offset in load j
    DEVINL unsigned voff(int j) const
    {
        if constexpr (QUAD) {
            const bool first = NW * j < NTI;
            const int blk = NW * j - (first ? 0 : NTI);
            const unsigned down = (unsigned)(8 * (blk % HALF)) * (unsigned)((first ? rs_a : rs_b) * 2) + (unsigned)(blk / HALF) * 128;
            return place[first ? 0 : 1] + down + (NW == 1 ? place[2] ^ (32 * (j & 1)) : place[2]);
        } else {
            return place[j];
        }
    }
    // this wavefront's share of the loads of tile t, into buffer `to` (t % NBUF)
    DEVINL void fetch(int t) const { fetch(t, t & (NBUF - 1)); }
    DEVINL void fetch(int t, int to) const
    {
        const int r0 = t * ROWS, left = min(n - r0, ROWS);
        const RawBuffer ab(a + (long)r0 * rs_a, left > 0 ? slice_bytes(rs_a, left, D) : 0);
        const RawBuffer bb(b + (long)r0 * rs_b, left > 0 ? slice_bytes(rs_b, left, D) : 0);
        const unsigned base = smem_addr + to * BUF_BYTES + wave * 1024;
        // load j's descriptor: known from j where all wavefronts' blocks of it belong to one tensor
        auto desc = [&](int j) { return NW * j + NW - 1 < NTI ? ab : NW * j >= NTI ? bb : pick(wave + NW * j < NTI, ab, bb); };
        constexpr int WHOLE = NBLK / NW, FOURS = WHOLE / 4 * 4;  // loads that every wavefront has
#pragma unroll
        for (int j = 0; j < FOURS; j += 4)
            load_to_lds16_x4<NW * 1024>(desc(j), desc(j + 1), desc(j + 2), desc(j + 3), base + NW * j * 1024, voff(j), voff(j + 1), voff(j + 2),
                                        voff(j + 3));
        if constexpr (WHOLE - FOURS >= 2)
            load_to_lds16_x2<NW * 1024>(desc(FOURS), desc(FOURS + 1), base + NW * FOURS * 1024, voff(FOURS), voff(FOURS + 1));
#pragma unroll
        for (int j = FOURS + (WHOLE - FOURS) / 2 * 2; j < NPW; ++j)
            if (j < WHOLE || wave + NW * j < NBLK) load_to_lds16(desc(j), base + NW * j * 1024, voff(j));
        if constexpr (SCALARS)
            // (the arrays go on to the next multiple of 64 rows)
            if (wave == NW - 1) load_to_lds16(RawBuffer(scalars + r0, npad_bytes + ROWS * 4), smem_addr + to * BUF_BYTES + OFF_SCALARS, scalar_voff);
    }
    DEVINL char* at(char* smem, int t) const { return smem + (t & (NBUF - 1)) * BUF_BYTES; }
    // what was asked for is in LDS, and nobody reads any more what was read (one wavefront has nobody to wait for)
    DEVINL static void landed_barrier()
    {
        if constexpr (NW * Cut::KG > 1) asm volatile("s_waitcnt vmcnt(0)\n\ts_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(0)\n\ts_waitcnt lgkmcnt(0)" ::: "memory");
    }
    // before tile t is computed on, from t0 on: with two buffers the next one is asked for, with one this one
    DEVINL void before(int t, int t0, int t1) const
    {
        if constexpr (NBUF == 2) {
            if (t + 1 < t1) fetch(t + 1);
        } else if (t > t0) {
            fetch(t);
            landed_barrier();
        }
    }
};

// A lane's fragments of a tile: rows 32 * hk .. of it (natural) and 16 tokens of step `step` (transposed)
template <int D, int ROWS>
struct RaggedLane {
    unsigned nat, tr;
    DEVINL explicit RaggedLane(int lane)
        : nat((unsigned)(lane % 32 * tile_stride<D>() + lane / 32 * 16)), tr((unsigned)tr_lane_offset(lane, tile_stride<D>()))
    {
    }
    DEVINL frag8 natural(const char* tile, int hk, int ks) const
    {
        return *reinterpret_cast<const frag8*>(tile + nat + 32 * hk * tile_stride<D>() + ks * 32);
    }
    DEVINL frag8 transposed(const char* tile, int ct, int step) const { return tr_frag(tile, tile_stride<D>(), (int)tr, ct, step); }
};
template <int D, int ROWS>
struct RaggedQuadLane : QuadLane {
    static constexpr int HALF = ROWS * 128;
    DEVINL explicit RaggedQuadLane(int lane) : QuadLane(lane, 0) {}
    DEVINL frag8 natural(const char* tile, int hk, int ks) const
    {
        return *reinterpret_cast<const frag8*>(tile + nat[ks & 1] + hk * 4096 + (ks / 2 & 1) * 256 + ks / 4 * HALF);
    }
    DEVINL frag8 transposed(const char* tile, int ct, int step) const
    {
        const lds_char* p = (const lds_char*)tile + step * 2048 + (ct & 1) * 256 + ct / 2 * HALF;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + tr[0]));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + tr[1]));
        const u32x2 l2 = __builtin_bit_cast(u32x2, lo), h2 = __builtin_bit_cast(u32x2, hi);
        return as_frag8(u32x4{l2[0], l2[1], h2[0], h2[1]});
    }
};
template <int ROWS>
struct RaggedLane<64, ROWS> : RaggedQuadLane<64, ROWS> {
    using RaggedQuadLane<64, ROWS>::RaggedQuadLane;
};
template <int ROWS>
struct RaggedLane<128, ROWS> : RaggedQuadLane<128, ROWS> {
    using RaggedQuadLane<128, ROWS>::RaggedQuadLane;
};

// The work of a workgroup, or, with several jobs, of each of its wavefronts
template <typename Cut>
struct RaggedJob {
    int id, wave, group, tid;
    char *all, *smem;  // the job's LDS, the group's
    DEVINL RaggedJob(char* shared, int ring_bytes)
    {
        const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        if constexpr (Cut::JOBS > 1) {
            id = blockIdx.x * Cut::JOBS + w;
            wave = group = 0;
            tid = threadIdx.x % 64;
            all = smem = shared + w * ring_bytes;
        } else {
            id = blockIdx.x;
            wave = w % Cut::NW;
            group = Cut::KG == 1 ? 0 : w / Cut::NW;
            tid = threadIdx.x;
            all = shared;
            smem = shared + group * ring_bytes;
        }
    }
};
// A group's share of the tiles 0 .. n - 1: all groups pass `per` of them
struct RaggedShare {
    int t0, t1, per;
    DEVINL RaggedShare(int n, int groups, int group)
    {
        per = (n + groups - 1) / groups;
        t0 = min(group * per, n);
        t1 = min(t0 + per, n);
    }
};

// Where a lane's row lies: token and head, and how many keys it sees.  Rows past the end stand for the last one.
struct RaggedRow {
    int token, head, keys;
    DEVINL RaggedRow(const RaggedArgs& a, int hk, int row, int rows, int nq, int nk)
    {
        const int r = min(row, rows - 1), i = a.over_heads(r);
        token = i;
        head = hk * a.G + r - i * a.G;
        keys = a.causal ? min(max(i + 1 + nk - nq, 0), nk) : nk;
    }
};

// 32 result rows (transposed accumulators, lane = row) to their places in a [T, Hq, D] tensor
template <int D, typename E>
struct RaggedStore {
    static constexpr int CT = (D + 31) / 32, STRIDE = D * 2 + 16, BYTES = 32 * STRIDE, CH = D / 8;
    DEVINL static void run(char* region, const f32x16 (&acc)[CT], float mul, raw16* out, const RaggedArgs& a, int hk, int begin, int row0,
                           int rows, int lane)
    {
        const int l32 = lane % 32, g = lane / 32;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int c0 = 32 * ct + 8 * q + 4 * g;
                if (c0 < D)
                    *reinterpret_cast<u32x2*>(region + l32 * STRIDE + c0 * 2) =
                        u32x2{E::pack(acc[ct][4 * q] * mul, acc[ct][4 * q + 1] * mul), E::pack(acc[ct][4 * q + 2] * mul, acc[ct][4 * q + 3] * mul)};
            }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
        for (int x = 0; x < (32 * CH + 63) / 64; ++x) {
            const int idx = lane + 64 * x, row = idx / CH, ch = idx % CH, r = row0 + row;
            if (idx < 32 * CH && r < rows) {
                const int i = a.over_heads(r);
                *reinterpret_cast<u32x4*>(out + ((long)(begin + i) * a.Hq + hk * a.G + r - i * a.G) * D + ch * 8) =
                    *reinterpret_cast<const u32x4*>(region + row * STRIDE + ch * 16);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
};

// Rows of no sequence: zeros in [T, H, D] for `count` heads from h0 on, tokens begin + t0 .. (n of them), by `threads` threads
template <int D>
DEVINL void ragged_zero(raw16* out, int H, int h0, int heads, long token0, int n, int tid, int threads)
{
    constexpr int CH = D / 8;
    const u32x4 zero = {0u, 0u, 0u, 0u};
    for (long x = tid; x < (long)n * heads * CH; x += threads) {
        const long t = x / (heads * CH);
        const int in = (int)(x - t * (heads * CH));
        *reinterpret_cast<u32x4*>(out + ((token0 + t) * H + h0 + in / CH) * D + in % CH * 8) = zero;
    }
}

// ------------------------------------------------------------------------------------------- forward
// One wavefront owns 32 rows, the workgroup's NW share (K | V) tiles of 64 keys; work in units of 32 keys as in avion_fwd_kernel,
// but with the running maximum: the accumulators are rescaled only where a row's maximum has grown by more than 2^8 (weights then
// stay below 2^8, which either format holds), a branch that after the first units is hardly ever taken.
// Bound by the vector issue port (63 % of the cycles at 64 channels, matrix units 33) and, at 128, by both (49 and 47).  Medians on two cards:
// 16 videos of 196 to 3136 tokens, 12 heads of 64, 91 and 95 us = 570 to 590 TFLOP/s (best launch 81); prompts of 500 to 8000, 32 heads on
// 8 of 128, 733 and 808 us = 760 to 830 (best 698); 2048 captions of 6 to 77, 8 heads of 64, 56 us, bound by memory.
constexpr float kRaggedLazy = 8.f;
constexpr float kRaggedNone = -3.0e38f;  // reference of a row that has seen nothing: finite, so that -inf - it is -inf

template <int D, typename Cut>
struct RaggedFwdCfg {
    using Ring = RaggedRing<D, Cut, false>;
    static constexpr int LDS_BYTES = Ring::LDS_BYTES * Cut::KG * Cut::JOBS;
    static_assert(LDS_BYTES <= 160 * 1024 && Cut::NW * RaggedStore<D, Bf16>::BYTES <= Ring::LDS_BYTES, "the rows on their way out take the ring's place");
    static constexpr int WAVES_PER_SIMD = Cut::KG > 1 || std::is_same<Cut, RaggedLone>::value ? 1 : D == 64 ? 4 : D == 80 ? 3 : 2;
};
template <int CT>
struct RaggedSums {
    f32x16 o[CT];
    f32x4 rs4;          // sums of the rounded weights, which multiplied V (four equal values)
    float m, l;         // reference, sum of the weights
    DEVINL RaggedSums()
    {
        acc_zero(o);
        rs4 = f32x4{0.f, 0.f, 0.f, 0.f};
        m = kRaggedNone;
        l = 0.f;
    }
};

// The tiles t0 .. t1 - 1 (and as many barriers as `per` tiles take) of one sequence's keys for the wavefront's rows row0 .. row0 + 31
template <int D, typename Cut, typename E>
DEVINL void ragged_fwd_walk(char* smem, const RaggedArgs& a, int hk, int begin_q, int nq, int begin_k, int nk, int row0, int rows, int t0,
                            int t1, int per, RaggedSums<(D + 31) / 32>& sums, int wave, int lane)
{
    using Ring = typename RaggedFwdCfg<D, Cut>::Ring;
    constexpr int KS = D / 16, CT = (D + 31) / 32, ROWS = Cut::ROWS;
    const int l32 = lane % 32, g = lane / 32;
    const RaggedLane<D, Ring::ROWS> at(lane);
    const Ring ring(a.k + (long)begin_k * a.rs_k + hk * D, a.rs_k, a.v + (long)begin_k * a.rs_v + hk * D, a.rs_v, nullptr, 0, nk, smem,
                    wave, lane);
    if (t0 < t1) ring.fetch(t0);
    const bool active = row0 < rows;
    const RaggedRow row(a, hk, row0 + l32, rows, nq, nk);
    const int seen_by_all = RaggedRow(a, hk, row0, rows, nq, nk).keys, seen_by_any = RaggedRow(a, hk, row0 + 31, rows, nq, nk).keys;
    frag8 qf[KS];
    const raw16* q = a.q + (long)(begin_q + row.token) * a.rs_q + row.head * D + g * 8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qf[ks] = *reinterpret_cast<const frag8*>(q + ks * 16);
    hold(qf);
    Ring::landed_barrier();

    const float cs = a.cs;
    // (one copy of the unit: with a copy for masked and one for whole units the accumulators took 20 registers' worth of spills)
    auto unit = [&](const char* kt, const char* vt, int hk32, int key_base) {
        f32x16 s = key_base + 32 > seen_by_all ? key_mask_block(key_base, g, row.keys) : f32x16_zero();
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) s = E::mfma(at.natural(kt, hk32, ks), qf[ks], s);
        frag8 vf[2][CT];
        if constexpr (D <= 96) {
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) vf[half][ct] = at.transposed(vt, ct, 2 * hk32 + half);
        }
        const float top = both_halves_max(max16(s)) * cs;
        if (__any(top > sums.m + kRaggedLazy)) {
            const float m = fmaxf(sums.m, top), shrink = fast_exp2(sums.m - m);
            sums.m = m;
            if (key_base > t0 * ROWS) {  // (the first unit finds zeros)
                sums.l *= shrink;
                sums.rs4 *= shrink;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int i = 0; i < 16; ++i) sums.o[ct][i] *= shrink;
            }
        }
        u32x4 pf[2];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float p = fast_exp2(fmaf(s[i], cs, -sums.m));
            s[i] = p;
            sums.l += p;
            if (i % 2 == 1) pf[i / 8][(i / 2) % 4] = E::pack(s[i - 1], p);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) sums.rs4 = E::add_four(u32x2{pf[i / 2][2 * (i % 2)], pf[i / 2][2 * (i % 2) + 1]}, sums.rs4);
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                if constexpr (D > 96) vf[half][ct] = at.transposed(vt, ct, 2 * hk32 + half);
                sums.o[ct] = E::mfma(vf[half][ct], as_frag8(pf[half]), sums.o[ct]);
            }
    };
    for (int t = t0; t < t0 + per; ++t) {
        ring.before(t, t0, t1);
        if (active && (Cut::KG == 1 || t < t1)) {
            const char* kt = ring.at(smem, t);
#pragma unroll
            for (int hk32 = 0; hk32 < ROWS / 32; ++hk32) {
                const int key_base = t * ROWS + 32 * hk32;
                if (key_base >= seen_by_any) continue;
                unit(kt, kt + Ring::OFF_B, hk32, key_base);
            }
        }
        Ring::landed_barrier();
    }
    // a row that none of these keys is for has met their masks only
    if (row.keys <= t0 * ROWS) sums = RaggedSums<CT>();
}

// What the sums come to: O's rows and LSE
template <int D, typename E>
DEVINL void ragged_fwd_store(char* region, const RaggedArgs& a, raw16* o, float* lse, int hk, int begin_q, int row0, int rows,
                             RaggedSums<(D + 31) / 32>& sums, int lane)
{
    const float l = both_halves_sum(sums.l), r = both_halves_sum(sums.rs4[0]);
    RaggedStore<D, E>::run(region, sums.o, r == 0.f ? 0.f : 1.f / r, o, a, hk, begin_q, row0, rows, lane);
    const int row = row0 + lane;
    if (lane < 32 && row < rows) {
        const int i = a.over_heads(row);
        lse[(long)(hk * a.G + row - i * a.G) * a.Tq + begin_q + i] = l == 0.f ? -INFINITY : (sums.m + __builtin_amdgcn_logf(l)) * kLn2;
    }
}
// Rows of no sequence
template <int D>
DEVINL void ragged_fwd_none(const RaggedArgs& a, raw16* o, float* lse, int hk, int token0, int n, int tid, int threads)
{
    ragged_zero<D>(o, a.Hq, hk * a.G, a.G, token0, n, tid, threads);
    for (long x = tid; x < (long)n * a.G; x += threads) lse[(long)(hk * a.G + x / n) * a.Tq + token0 + x % n] = -INFINITY;
}
// the tokens whose (token, head) rows a block of BM rows begins: each token belongs to one block
DEVINL int ragged_first_token(long row, int G) { return (int)((row + G - 1) / G); }

// The groups' sums of the same rows, in group order, each scaled to the larger reference: into group 0's
template <int CT, typename Cut>
DEVINL void ragged_fwd_join(char* area, RaggedSums<CT>& sums, int group, int wave, int lane)
{
    constexpr int VALS = CT * 16 + 3;
    if (group > 0) {
        float* mine = reinterpret_cast<float*>(area) + ((group - 1) * Cut::NW + wave) * VALS * 64 + lane;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int i = 0; i < 16; ++i) mine[(ct * 16 + i) * 64] = sums.o[ct][i];
        mine[(VALS - 3) * 64] = sums.l;
        mine[(VALS - 2) * 64] = sums.rs4[0];
        mine[(VALS - 1) * 64] = sums.m;
    }
    __syncthreads();
    if (group > 0) return;
#pragma unroll
    for (int og = 0; og < Cut::KG - 1; ++og) {
        const float* other = reinterpret_cast<const float*>(area) + (og * Cut::NW + wave) * VALS * 64 + lane;
        const float m = fmaxf(sums.m, other[(VALS - 1) * 64]), x = fast_exp2(sums.m - m), y = fast_exp2(other[(VALS - 1) * 64] - m);
        sums.l = sums.l * x + other[(VALS - 3) * 64] * y;
        sums.rs4[0] = sums.rs4[0] * x + other[(VALS - 2) * 64] * y;
        sums.m = m;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int i = 0; i < 16; ++i) sums.o[ct][i] = sums.o[ct][i] * x + other[(ct * 16 + i) * 64] * y;
    }
}

template <int D, typename Cut, typename E>
__global__ void __launch_bounds__(Cut::NT * Cut::JOBS, (RaggedFwdCfg<D, Cut>::WAVES_PER_SIMD))
avion_ragged_fwd_kernel(RaggedArgs a, raw16* __restrict__ o, float* __restrict__ lse)
{
    using Cfg = RaggedFwdCfg<D, Cut>;
    constexpr int CT = (D + 31) / 32, STORE = Cut::NW * RaggedStore<D, E>::BYTES;
    extern __shared__ __attribute__((aligned(16))) char shared[];
    const int lane = threadIdx.x % 64;
    const RaggedJob<Cut> job(shared, Cfg::Ring::LDS_BYTES);
    // (the key heads go round the XCDs)
    const int hk = job.id % a.Hk, turn = job.id / a.Hk;
    if (turn >= a.slots) return;
    const RaggedPlace p = ragged_turn<Cut::SHIFT, true>(a.off_q, a.S, a.Tq, a.G, a.off_k, a.Tk, a.slots, turn, lane);
    const int rows = p.n * a.G;
    if (p.block < 0 || p.block * Cut::BLOCK >= rows || rows <= a.done) return;
    const int block0 = (int)p.block * Cut::BLOCK;
    if (p.i == 0 || p.i == a.S + 1) {
        if (a.done) return;  // (these are avion_ragged_join_kernel's then)
        const int from = ragged_first_token(block0, a.G), to = min(ragged_first_token(block0 + Cut::BLOCK, a.G), p.n);
        ragged_fwd_none<D>(a, o, lse, hk, p.begin + from, to - from, job.tid, Cut::NT);
        return;
    }
    // (offsets that serve both sides are here already)
    const int2 keys = a.off_k == a.off_q && a.Tk == a.Tq ? int2{p.begin, p.n} : ragged_tokens(a.off_k, a.S, a.Tk, p.i);
    const int begin_k = keys.x, nk = keys.y;
    const int last_seen = RaggedRow(a, hk, block0 + Cut::BLOCK - 1, rows, p.n, nk).keys;
    const RaggedShare share((last_seen + Cut::ROWS - 1) / Cut::ROWS, Cut::KG, job.group);
    RaggedSums<CT> sums;
    const int row0 = block0 + job.wave * 32;
    ragged_fwd_walk<D, Cut, E>(job.smem, a, hk, p.begin, p.n, begin_k, nk, row0, rows, share.t0, share.t1, share.per, sums, job.wave, lane);
    if constexpr (Cut::KG > 1) {
        static_assert(STORE + (Cut::KG - 1) * Cut::NW * (CT * 16 + 3) * 256 <= Cfg::LDS_BYTES, "exchange area");
        ragged_fwd_join<CT, Cut>(job.all + STORE, sums, job.group, job.wave, lane);
        if (job.group > 0) return;
    }
    if (row0 >= rows) return;
    ragged_fwd_store<D, E>(job.all + job.wave * RaggedStore<D, E>::BYTES, a, o, lse, hk, p.begin, row0, rows, sums, lane);
}

// ------------------------------------------------------------------------------ few rows, many keys
// Single tokens behind long caches: bound by the keys' bytes, which must come from all of memory at once.  Slots are chunks of
// 2^SHIFT keys (found as above, in the keys' offsets): a wavefront takes the first 32 rows of a sequence through one chunk and
// leaves its sums; a second launch joins them.  A sequence with one chunk is finished here.  Rows past the first 32, which a launch of a
// few hundred rows may hold, take all keys in the wavefront of the first chunk; in larger ones such a sequence is a launch of
// avion_ragged_fwd_kernel's.  24 tokens behind up to 9000 keys, 32 heads on 8 of 128: 35 us for 182 MB, 5.2 TB/s, and 5 for the join.
template <int D>
struct RaggedPart {
    static constexpr int FLOATS = 32 * D + 3 * 32;  // O, then reference, sum, sum of the rounded weights
};
template <int D, typename E>
__global__ void __launch_bounds__(64, 1)
avion_ragged_few_kernel(RaggedArgs a, raw16* __restrict__ o, float* __restrict__ lse, float* __restrict__ parts, int shift)
{
    constexpr int CT = (D + 31) / 32;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int lane = threadIdx.x, hk = blockIdx.x % a.Hk, slot = blockIdx.x / a.Hk;
    // (the search knows shifts at compile time)
    RaggedPlace p;
    switch (shift) {
        case 8: p = ragged_place<8>(a.off_k, a.S, a.Tk, 1, slot, lane); break;
        case 9: p = ragged_place<9>(a.off_k, a.S, a.Tk, 1, slot, lane); break;
        case 10: p = ragged_place<10>(a.off_k, a.S, a.Tk, 1, slot, lane); break;
        default: p = ragged_place<11>(a.off_k, a.S, a.Tk, 1, slot, lane); break;
    }
    const int chunk = 1 << shift;
    if (p.i == 0 || p.i == a.S + 1 || p.block < 0 || (p.block > 0 && p.block * chunk >= p.n)) return;
    const int begin_q = ragged_border(a.off_q, a.S, a.Tq, p.i), nq = max(ragged_border(a.off_q, a.S, a.Tq, p.i + 1) - begin_q, 0);
    const int rows = nq * a.G, chunks = max((p.n + chunk - 1) >> shift, 1), tiles = (p.n + 63) / 64;
    if (a.done && rows > a.done) return;
    for (int row0 = 0; row0 < rows; row0 += 32) {
        const bool part = row0 == 0 && chunks > 1;
        if (!part && p.block > 0) return;
        const int t0 = part ? (int)p.block * (chunk / 64) : 0, t1 = part ? min(t0 + chunk / 64, tiles) : tiles;
        RaggedSums<CT> sums;
        ragged_fwd_walk<D, RaggedLone, E>(smem, a, hk, begin_q, nq, p.begin, p.n, row0, rows, t0, t1, t1 - t0, sums, 0, lane);
        if (!part) {
            ragged_fwd_store<D, E>(smem, a, o, lse, hk, begin_q, row0, rows, sums, lane);
            RaggedFwdCfg<D, RaggedLone>::Ring::landed_barrier();
            continue;
        }
        const int l32 = lane % 32, g = lane / 32;
        float* out = parts + ((long)slot * a.Hk + hk) * RaggedPart<D>::FLOATS;
        if (l32 < rows) {
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (32 * ct + 8 * q + 4 * g < D)
                        *reinterpret_cast<f32x4*>(out + l32 * D + 32 * ct + 8 * q + 4 * g) =
                            f32x4{sums.o[ct][4 * q], sums.o[ct][4 * q + 1], sums.o[ct][4 * q + 2], sums.o[ct][4 * q + 3]};
        }
        const float l = both_halves_sum(sums.l), r = both_halves_sum(sums.rs4[0]);
        if (g == 0) {
            out[32 * D + l32] = sums.m;
            out[32 * D + 32 + l32] = l;
            out[32 * D + 64 + l32] = r;
        }
        RaggedFwdCfg<D, RaggedLone>::Ring::landed_barrier();
    }
}

// Joins them: a wavefront a row, D / 4 lanes a chunk and as many chunks at a time as that leaves; groups in a fixed order.  Also the
// rows of no sequence.
template <int D, typename E>
__global__ void __launch_bounds__(256)
avion_ragged_join_kernel(RaggedArgs a, raw16* __restrict__ o, float* __restrict__ lse, const float* __restrict__ parts, int shift)
{
    constexpr int LANES = D / 4, GROUPS = 64 / LANES;
    const int hk = blockIdx.x % a.Hk, i = blockIdx.x / a.Hk;  // interval of the borders
    const int begin_q = ragged_border(a.off_q, a.S, a.Tq, i), nq = max(ragged_border(a.off_q, a.S, a.Tq, i + 1) - begin_q, 0);
    if (i == 0 || i == a.S + 1) {
        ragged_fwd_none<D>(a, o, lse, hk, begin_q, nq, threadIdx.x, 256);
        return;
    }
    const int begin_k = ragged_border(a.off_k, a.S, a.Tk, i), nk = max(ragged_border(a.off_k, a.S, a.Tk, i + 1) - begin_k, 0);
    const int chunks = (nk + (1 << shift) - 1) >> shift, rows = min(nq * a.G, 32);
    if (chunks < 2 || (a.done && nq * a.G > a.done)) return;
    const long slot = (begin_k >> shift) + i, step = (long)a.Hk * RaggedPart<D>::FLOATS;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, group = lane / LANES, col = lane % LANES * 4;
    for (int row = wave; row < rows; row += 4) {
        const float* at = parts + (slot * a.Hk + hk) * RaggedPart<D>::FLOATS;
        float m = kRaggedNone;
        for (int c = lane; c < chunks; c += 64) m = fmaxf(m, at[c * step + 32 * D + row]);
#pragma unroll
        for (int x = 1; x < 64; x *= 2) m = fmaxf(m, __shfl_xor(m, x));
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        float l = 0.f, r = 0.f;
        if (group < GROUPS) {
#pragma unroll 4
            for (int c = group; c < chunks; c += GROUPS) {
                const float* part = at + c * step;
                const float w = fast_exp2(part[32 * D + row] - m);
                l += w * part[32 * D + 32 + row];
                r += w * part[32 * D + 64 + row];
                acc += w * *reinterpret_cast<const f32x4*>(part + row * D + col);
            }
        }
        // the groups' sums, one after the other
        f32x4 sum = acc;
        float ls = l, rs = r;
#pragma unroll
        for (int x = 1; x < GROUPS; ++x) {
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] += __shfl(acc[e], lane % LANES + x * LANES);
            ls += __shfl(l, lane % LANES + x * LANES);
            rs += __shfl(r, lane % LANES + x * LANES);
        }
        const int q = a.over_heads(row), head = hk * a.G + row - q * a.G;
        const float inv = rs == 0.f ? 0.f : 1.f / rs;
        if (group == 0)
            *reinterpret_cast<u32x2*>(o + ((long)(begin_q + q) * a.Hq + head) * D + col) =
                u32x2{E::pack(sum[0] * inv, sum[1] * inv), E::pack(sum[2] * inv, sum[3] * inv)};
        if (lane == 0) lse[(long)head * a.Tq + begin_q + q] = ls == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(ls)) * kLn2;
    }
}

// ------------------------------------------------------------------------------------------------ dQ
// As avion_dq_kernel, on the rows above.  delta = rowsum(dO o O) from the O that the forward rounded is off by 2^-9 |dO| |O|, which
// counts where a row sees few keys; a workgroup with up to 128 keys (all of them in LDS, or in the caches) forms delta = sum_j P_j dP_j
// from them first: the rows that need it, and the ones that are not bound by contractions.
// Leaves lse * log2 e (+inf where a row sees nothing, so that its weights are 0; fp16: less kRaggedShift) and -delta for the second
// kernel: [Hq][2][npad], sequence s at (floor(begin / 64) + s) * 64.
//
// fp16 weights below 2^-14 lose bits: over thousands of keys most are.  The second kernel holds them 2^8 times larger where they
// are rounded for dV; in dS they stand beside dP, which is as large as the loss is scaled.
// The 16 videos 101 and 106 us (medians on two cards, best launch 95) = 770 to 800 TFLOP/s, the logits among them (matrix units 42 % of the
// cycles, vector issue 58).
template <typename E>
constexpr float kRaggedShift = std::is_same<E, F16>::value ? 8.f : 0.f;

template <int D, typename Cut>
struct RaggedDqCfg {
    using Ring = RaggedRing<D, Cut, false>;
    static constexpr int LDS_BYTES = Ring::LDS_BYTES * Cut::KG * Cut::JOBS;
    static_assert(LDS_BYTES <= 160 * 1024 && Cut::NW * RaggedStore<D, Bf16>::BYTES <= Ring::LDS_BYTES, "the rows on their way out take the ring's place");
    // (four of the lone wavefronts spill: both passes of 1000 sequences of 20 to 40 tokens, 16 heads on 8, 119 us, with three 109)
    static constexpr int WAVES_PER_SIMD = Cut::KG > 1 ? 1 : D == 64 ? (Cut::JOBS > 1 ? 3 : 4) : 2;
};
DEVINL long ragged_scalar_at(int begin, int i) { return ((long)(begin >> 6) + i) * 64; }

template <int D, typename Cut, typename E>
__global__ void __launch_bounds__(Cut::NT * Cut::JOBS, (RaggedDqCfg<D, Cut>::WAVES_PER_SIMD))
avion_ragged_dq_kernel(RaggedArgs a, const raw16* __restrict__ o, const raw16* __restrict__ dO, const float* __restrict__ lse,
                       raw16* __restrict__ dq, float* __restrict__ rowsc, int npad)
{
    using Cfg = RaggedDqCfg<D, Cut>;
    using Ring = typename Cfg::Ring;
    constexpr int KS = D / 16, CT = (D + 31) / 32;
    extern __shared__ __attribute__((aligned(16))) char shared[];
    const int lane = threadIdx.x % 64, l32 = lane % 32, g = lane / 32;
    const RaggedJob<Cut> job(shared, Ring::LDS_BYTES);
    const int wave = job.wave;
    char* smem = job.smem;
    const int hk = job.id % a.Hk, turn = job.id / a.Hk;
    if (turn >= a.slots || (a.done && !*a.more)) return;
    const RaggedPlace p = ragged_turn<Cut::SHIFT, true>(a.off_q, a.S, a.Tq, a.G, a.off_k, a.Tk, a.slots, turn, lane);
    const int rows = p.n * a.G, nq = p.n;
    if (p.block < 0 || p.block * Cut::BLOCK >= rows) return;
    const int block0 = (int)p.block * Cut::BLOCK;
    if (p.i == 0 || p.i == a.S + 1) {
        const int from = ragged_first_token(block0, a.G), to = min(ragged_first_token(block0 + Cut::BLOCK, a.G), p.n);
        ragged_zero<D>(dq, a.Hq, hk * a.G, a.G, p.begin + from, to - from, job.tid, Cut::NT);
        return;
    }
    // (offsets that serve both sides are here already)
    const int2 keys = a.off_k == a.off_q && a.Tk == a.Tq ? int2{p.begin, p.n} : ragged_tokens(a.off_k, a.S, a.Tk, p.i);
    const int begin_k = keys.x, nk = keys.y;
    if (max(nq, nk) <= a.done) return;
    constexpr int ROWS = Ring::ROWS;
    const int ntiles = (RaggedRow(a, hk, block0 + Cut::BLOCK - 1, rows, nq, nk).keys + ROWS - 1) / ROWS;
    const bool whole = Ring::NBUF == 1 ? ntiles * ROWS <= 128 : ntiles <= 2;  // (the first group's work then)
    const RaggedShare share(ntiles, Cut::KG == 1 || whole ? 1 : Cut::KG, job.group);
    const int t0 = share.t0, t1 = share.t1;
    const Ring ring(a.k + (long)begin_k * a.rs_k + hk * D, a.rs_k, a.v + (long)begin_k * a.rs_v + hk * D, a.rs_v, nullptr, 0, nk, smem,
                    wave, lane);
    if (t0 < t1) ring.fetch(t0);
    if (Ring::NBUF == 2 && whole && t1 == 2) ring.fetch(1);
    const int row0 = block0 + wave * 32;
    const RaggedLane<D, Ring::ROWS> at(lane);
    const bool active = row0 < rows, first = job.group == 0;
    const RaggedRow row(a, hk, row0 + l32, rows, nq, nk);
    const int seen_by_all = RaggedRow(a, hk, row0, rows, nq, nk).keys, seen_by_any = RaggedRow(a, hk, row0 + 31, rows, nq, nk).keys;
    frag8 qf[KS], gf[KS];
    float dl;
    {
        const raw16* q = a.q + (long)(p.begin + row.token) * a.rs_q + row.head * D + g * 8;
        const long out_at = ((long)(p.begin + row.token) * a.Hq + row.head) * D + g * 8;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            qf[ks] = *reinterpret_cast<const frag8*>(q + ks * 16);
            gf[ks] = *reinterpret_cast<const frag8*>(dO + out_at + ks * 16);
        }
        float part = 0.f;
        if (!whole) {
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const frag8 of = *reinterpret_cast<const frag8*>(o + out_at + ks * 16);
#pragma unroll
                for (int e = 0; e < 8; ++e) part = fmaf(E::widen(of, e), E::widen(gf[ks], e), part);
            }
        }
        dl = both_halves_sum(part);
    }
    const float saved = lse[(long)row.head * a.Tq + p.begin + row.token];
    const float lc = saved == -INFINITY ? INFINITY : saved * kLog2e, cs = a.cs;
    hold(qf);
    hold(gf);
    Ring::landed_barrier();

    // scores (far below all others where the row does not see the key) and dP of one unit
    auto products = [&](const char* kt, int hk32, int key_base, f32x16& sc, f32x16& dp) {
        const char* vt = kt + Ring::OFF_B;
        sc = key_base + 32 > seen_by_all ? key_mask_block(key_base, g, row.keys) : f32x16_zero();
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const frag8 ak = at.natural(kt, hk32, ks), av = at.natural(vt, hk32, ks);
            sc = E::mfma(ak, qf[ks], sc);
            dp = E::mfma(av, gf[ks], ks == 0 ? f32x16_zero() : dp);
        }
    };
    // weights in place of the scores
    auto weigh = [&](f32x16& sc) {
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[i] = fast_exp2(fmaf(sc[i], cs, -lc));
    };
    f32x16 s, dp;
    const bool single = Ring::NBUF == 1 && ntiles == 1;  // one unit: its products serve twice
    if (whole && active && first) {
        float sum = 0.f;
        for (int key_base = 0; key_base < seen_by_any; key_base += 32) {
            if (Ring::NBUF == 1) ring.before(key_base / ROWS, 0, 0);
            products(ring.at(smem, key_base / ROWS), key_base % ROWS / 32, key_base, s, dp);
            if (Ring::NBUF == 1) Ring::landed_barrier();
            weigh(s);
#pragma unroll
            for (int i = 0; i < 16; ++i) sum = fmaf(s[i], dp[i], sum);
        }
        dl = both_halves_sum(sum);
        if (Ring::NBUF == 1 && seen_by_any > ROWS) {
            ring.fetch(0);
            Ring::landed_barrier();
        }
    }
    if (active && first && g == 0 && row0 + l32 < rows) {
        float* ws = rowsc + (long)row.head * 2 * npad + ragged_scalar_at(p.begin, p.i) + row.token;
        ws[0] = lc - kRaggedShift<E>;
        ws[npad] = -dl;
    }
    // the rows up to the next multiple of 64: weight 0
    if (block0 + Cut::BLOCK >= rows)
        for (int x = job.tid; x < (-nq & 63) * a.G; x += Cut::NT) {
            const int i = a.over_heads(x);
            float* ws = rowsc + (long)(hk * a.G + x - i * a.G) * 2 * npad + ragged_scalar_at(p.begin, p.i) + nq + i;
            ws[0] = INFINITY;
            ws[npad] = 0.f;
        }
    f32x16 acc[CT];
    acc_zero(acc);
    auto unit = [&](const char* kt, int hk32, int key_base) {
        if (!single) {
            products(kt, hk32, key_base, s, dp);
            weigh(s);
        }
        frag8 kf[2][CT];
        if constexpr (D <= 96) {
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) kf[half][ct] = at.transposed(kt, ct, 2 * hk32 + half);
        }
        u32x4 df[2];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[i] *= dp[i] - dl;
            if (i % 2 == 1) df[i / 8][(i / 2) % 4] = E::pack(s[i - 1], s[i]);
        }
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                if constexpr (D > 96) kf[half][ct] = at.transposed(kt, ct, 2 * hk32 + half);
                acc[ct] = E::mfma(kf[half][ct], as_frag8(df[half]), acc[ct]);
            }
    };
    for (int t = t0; t < t0 + share.per; ++t) {
        if (Ring::NBUF == 1 || !whole) ring.before(t, t0, t1);
        if (active && (Cut::KG == 1 || t < t1)) {
            const char* kt = ring.at(smem, t);
#pragma unroll
            for (int hk32 = 0; hk32 < ROWS / 32; ++hk32) {
                const int key_base = t * ROWS + 32 * hk32;
                if (key_base >= seen_by_any) continue;
                unit(kt, hk32, key_base);
            }
        }
        Ring::landed_barrier();
    }
    if constexpr (Cut::KG > 1) {
        constexpr int STORE = Cut::NW * RaggedStore<D, E>::BYTES;
        static_assert(STORE + (Cut::KG - 1) * Cut::NW * (int)sizeof(acc) * 64 <= Cfg::LDS_BYTES, "exchange area");
        add_groups<Cut::NW, Cut::KG>(job.all + STORE, acc, job.group, wave, lane, active);
        if (!first) return;
    }
    if (!active) return;
    RaggedStore<D, E>::run(job.all + wave * RaggedStore<D, E>::BYTES, acc, a.scale, dq, a, hk, p.begin, row0, rows, lane_from_exec());
}

// -------------------------------------------------------------------------------------------- dK, dV
// As avion_dkdv_kernel: a wavefront owns 32 keys of one key head; the tiles of 64 queries of its query heads come one after the
// other.  With `parts` > 1 the query heads are dealt to that many workgroups, whose sums meet in fp32 (avion_ragged_sum_kernel).
template <int D, typename Cut>
struct RaggedDkvCfg {
    using Ring = RaggedRing<D, Cut, true>;
    static constexpr int LDS_BYTES = Ring::LDS_BYTES * Cut::KG * Cut::JOBS;
    static_assert(LDS_BYTES <= 160 * 1024 && Cut::NW * RowStore<D, Bf16>::BYTES <= Ring::LDS_BYTES, "the rows on their way out take the ring's place");
    static constexpr int WAVES_PER_SIMD = Cut::KG > 1 ? 1 : D == 64 ? 3 : D == 80 ? 2 : 1;
};
// 32 rows of fp32 sums, lane = row
template <int D>
DEVINL void ragged_store_part(const f32x16 (&acc)[(D + 31) / 32], float* out, long stride, int rows, int lane)
{
    const int l32 = lane % 32, g = lane / 32;
    if (l32 >= rows) return;
#pragma unroll
    for (int ct = 0; ct < (D + 31) / 32; ++ct)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (32 * ct + 8 * q + 4 * g < D)
                *reinterpret_cast<f32x4*>(out + l32 * stride + 32 * ct + 8 * q + 4 * g) =
                    f32x4{acc[ct][4 * q], acc[ct][4 * q + 1], acc[ct][4 * q + 2], acc[ct][4 * q + 3]};
}

// One unit: queries 32 * hq .. of the tiles qt (Q) and gt (dO), whose scalars (lse as avion_ragged_dq_kernel leaves it, then, `rows` further,
// -delta) stand at `scalars`; `from`: the first query that sees this lane's key, from_all: all keys of the wavefront
template <int D, typename E, typename Lane>
DEVINL void ragged_dkdv_unit(const Lane& at, const char* qt, const char* gt, const float* scalars, int rows, int hq, int query_base,
                             int from, int from_all, float cs, int g, const frag8 (&kf)[D / 16], const frag8 (&vf)[D / 16],
                             f32x16 (&dka)[(D + 31) / 32], f32x16 (&dva)[(D + 31) / 32])
{
    constexpr int KS = D / 16, CT = (D + 31) / 32;
    const float* rowv = scalars + 32 * hq + 4 * g;
            f32x16 dp, s = query_base < from_all ? query_mask_block(query_base, g, from) : f32x16_zero();
#pragma unroll
            for (int a4 = 0; a4 < 4; ++a4) {
                const f32x4 d4 = *reinterpret_cast<const f32x4*>(rowv + rows + 8 * a4);
#pragma unroll
                for (int e = 0; e < 4; ++e) dp[4 * a4 + e] = d4[e];
            }
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const frag8 aq = at.natural(qt, hq, ks), ag = at.natural(gt, hq, ks);
                s = E::mfma(aq, kf[ks], s);
                dp = E::mfma(ag, vf[ks], dp);
            }
            f32x4 l4[4];
#pragma unroll
            for (int a4 = 0; a4 < 4; ++a4) l4[a4] = *reinterpret_cast<const f32x4*>(rowv + 8 * a4);
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                frag8 tg[CT], tq[CT];
                if constexpr (D <= 96) {
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) {
                        tg[ct] = at.transposed(gt, ct, 2 * hq + half);
                        tq[ct] = at.transposed(qt, ct, 2 * hq + half);
                    }
                }
                u32x4 pf, df;
#pragma unroll
                for (int e = 8 * half; e < 8 * half + 8; ++e) {
                    const float pe = fast_exp2(fmaf(s[e], cs, -l4[e / 4][e % 4]));
                    const float ds = (std::is_same<E, F16>::value ? pe * (1.f / 256.f) : pe) * dp[e];
                    s[e] = pe;
                    dp[e] = ds;
                    if (e % 2 == 1) {
                        pf[(e / 2) % 4] = E::pack(s[e - 1], s[e]);
                        df[(e / 2) % 4] = E::pack(dp[e - 1], dp[e]);
                    }
                }
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    if constexpr (D > 96) {
                        tg[ct] = at.transposed(gt, ct, 2 * hq + half);
                        tq[ct] = at.transposed(qt, ct, 2 * hq + half);
                    }
                    dva[ct] = E::mfma(tg[ct], as_frag8(pf), dva[ct]);
                    dka[ct] = E::mfma(tq[ct], as_frag8(df), dka[ct]);
                }
            }
}

// dK and dV: 32 keys a wavefront, K and V in registers, (Q | dO) tiles of the query heads that share them one after the other.  The 16 videos
// 124 and 133 us (medians on two cards, best launch 116) = 820 to 880 TFLOP/s, the logits among them (matrix units 46 % of the cycles, LDS 36,
// vector issue 46).
template <int D, typename Cut, typename E>
__global__ void __launch_bounds__(Cut::NT * Cut::JOBS, (RaggedDkvCfg<D, Cut>::WAVES_PER_SIMD))
avion_ragged_dkdv_kernel(RaggedArgs a, const raw16* __restrict__ dO, const float* __restrict__ rowsc, int npad, raw16* __restrict__ dk,
                         raw16* __restrict__ dv, float* __restrict__ sums, int parts)
{
    using Cfg = RaggedDkvCfg<D, Cut>;
    using Ring = typename Cfg::Ring;
    constexpr int KS = D / 16, CT = (D + 31) / 32, OFF_G = Ring::OFF_B, ROWS = Ring::ROWS;
    extern __shared__ __attribute__((aligned(16))) char shared[];
    const int lane = threadIdx.x % 64, l32 = lane % 32, g = lane / 32;
    const RaggedJob<Cut> job(shared, Ring::LDS_BYTES);
    const int wave = job.wave;
    char* smem = job.smem;
    const int hk = job.id % a.Hk, part = job.id / a.Hk % parts, turn = job.id / (a.Hk * parts);
    if (turn >= a.slots || (a.done && !*a.more)) return;
    const RaggedPlace p = ragged_turn<Cut::SHIFT, false>(a.off_k, a.S, a.Tk, 1, a.off_q, a.Tq, a.slots, turn, lane);
    const int nk = p.n;
    if (p.block < 0 || p.block * Cut::BLOCK >= nk) return;
    const int block0 = (int)p.block * Cut::BLOCK, k0 = block0 + wave * 32;
    const int2 queries = a.off_k == a.off_q && a.Tk == a.Tq ? int2{p.begin, p.n} : ragged_tokens(a.off_q, a.S, a.Tq, p.i);
    const int begin_q = queries.x, nq = p.i == 0 || p.i == a.S + 1 ? 0 : queries.y;
    if (max(nq, nk) <= a.done && p.i > 0 && p.i <= a.S) return;
    const bool active = k0 < nk;
    // first query that sees a key: this lane's, the wavefront's first and last, the workgroup's first
    auto first_query = [&](int key) { return a.causal ? max(min(key, nk - 1) - nk + nq, 0) : 0; };
    const int key = min(k0 + l32, nk - 1), from = first_query(k0 + l32), from_all = first_query(k0 + 31), from_any = first_query(k0);
    const int tile0 = first_query(block0) / ROWS, tiles = nq == 0 ? 0 : (nq + ROWS - 1) / ROWS - tile0;
    const int heads = a.G / parts, h0 = hk * a.G + part * heads;

    const long q_at = (long)begin_q * a.rs_q, o_at = (long)begin_q * a.Hq * D;
    Ring ring(a.q + q_at, a.rs_q, dO + o_at, (long)a.Hq * D, rowsc + ragged_scalar_at(begin_q, p.i), npad, nq, smem, wave, lane);
    // the tiles of all heads, one after the other: this group's share
    const RaggedShare share(heads * tiles, Cut::KG, job.group);
    const int total = share.t1 - share.t0;
    int f_head = tiles > 0 ? share.t0 / tiles : 0, f_tile = share.t0 - f_head * tiles;  // next to fetch
    int tile = f_tile;
    auto fetch = [&](int n) {
        Ring r = ring;
        r.a += (h0 + f_head) * D;
        r.b += (h0 + f_head) * D;
        r.scalars += (long)(h0 + f_head) * 2 * npad;
        r.fetch(tile0 + f_tile, n & (Ring::NBUF - 1));
        if (++f_tile == tiles) {
            f_tile = 0;
            ++f_head;
        }
    };
    if (total > 0) fetch(0);
    frag8 kf[KS], vf[KS];
    {
        const raw16 *k = a.k + (long)(p.begin + key) * a.rs_k + hk * D + g * 8, *v = a.v + (long)(p.begin + key) * a.rs_v + hk * D + g * 8;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            kf[ks] = *reinterpret_cast<const frag8*>(k + ks * 16);
            vf[ks] = *reinterpret_cast<const frag8*>(v + ks * 16);
        }
    }
    f32x16 dka[CT], dva[CT];
    acc_zero(dka);
    acc_zero(dva);
    hold(kf);
    hold(vf);
    Ring::landed_barrier();
    const float cs = a.cs;
    const RaggedLane<D, Ring::ROWS> at(lane);

    for (int n = 0; n < (Cut::KG == 1 ? total : share.per); ++n) {
        if constexpr (Ring::NBUF == 2) {
            if (n + 1 < total) fetch(n + 1);
        } else if (n > 0) {
            fetch(n);
            Ring::landed_barrier();
        }
        if (active && (Cut::KG == 1 || n < total)) {
            const char* buf = ring.at(smem, n);
#pragma unroll
            for (int hq = 0; hq < ROWS / 32; ++hq) {
                const int query_base = (tile0 + tile) * ROWS + 32 * hq;
                if (query_base >= nq || query_base + 32 <= from_any) continue;
                ragged_dkdv_unit<D, E>(at, buf, buf + OFF_G, reinterpret_cast<const float*>(buf + Ring::OFF_SCALARS), ROWS, hq, query_base, from, from_all, cs, g, kf, vf,
                                       dka, dva);
            }
        }
        if (++tile == tiles) tile = 0;
        Ring::landed_barrier();
    }
    if constexpr (Cut::KG > 1) {
        constexpr int STORE = Cut::NW * RowStore<D, E>::BYTES;
        static_assert(STORE + (Cut::KG - 1) * Cut::NW * CT * 4096 <= Cfg::LDS_BYTES, "exchange area");
        add_groups<Cut::NW, Cut::KG>(job.all + STORE, dka, job.group, wave, lane, active);
        __syncthreads();
        add_groups<Cut::NW, Cut::KG>(job.all + STORE, dva, job.group, wave, lane, active);
        if (job.group > 0) return;
    }
    if (!active) return;
    const int lane_now = lane_from_exec();
    const float dv_mul = std::is_same<E, F16>::value ? 1.f / 256.f : 1.f;
    const long rs = (long)a.Hk * D, out_at = (long)(p.begin + k0) * rs + hk * D;
    if (parts > 1) {
        const long whole = (long)a.Tk * rs;
        float* out = sums + part * 2 * whole + out_at;
        ragged_store_part<D>(dka, out, rs, nk - k0, lane_now);
        ragged_store_part<D>(dva, out + whole, rs, nk - k0, lane_now);
        return;
    }
    char* region = job.all + wave * RowStore<D, E>::BYTES;
    RowStore<D, E>::run(region, dka, a.scale, dk + out_at, rs, nk - k0, lane_now);
    RowStore<D, E>::run(region, dva, dv_mul, dv + out_at, rs, nk - k0, lane_now);
}

// dK and dV from the parts' sums, part after part
template <typename E>
__global__ void __launch_bounds__(256)
avion_ragged_sum_kernel(const float* __restrict__ sums, int parts, long n, raw16* __restrict__ dk, raw16* __restrict__ dv, float dk_mul, float dv_mul)
{
    const long chunks = n / 4;
    for (long x = blockIdx.x * 256L + threadIdx.x; x < 2 * chunks; x += gridDim.x * 256L) {
        const bool second = x >= chunks;
        const long i = (second ? x - chunks : x) * 4;
        f32x4 t = {0.f, 0.f, 0.f, 0.f};
        for (int p = 0; p < parts; ++p) t += *reinterpret_cast<const f32x4*>(sums + (2L * p + second) * n + i);
        t *= second ? dv_mul : dk_mul;
        *reinterpret_cast<u32x2*>((second ? dv : dk) + i) = u32x2{E::pack(t[0], t[1]), E::pack(t[2], t[3])};
    }
}

// ------------------------------------------------------------------------------- whole short sequences
// The backward of a sequence of at most 32 W queries and keys (and more than 16 W), heads not shared, in one pass: W wavefronts hold Q, dO,
// K and V of one head in LDS, each first does 32 queries (dQ, and lse and delta for the others, as avion_ragged_dq_kernel), then 32
// keys (dK, dV).  Every tensor is read once and O not at all.
// A workgroup for each (sequence, head), which ends at once where the sequence is another launch's; but with four wavefronts and 65 KB of
// LDS, of which a compute unit ends two at a time, a grid that fills the chip once, whose workgroups look at the lengths of 512 sequences
// at a time and take the pairs number b, b + grid, ... of those that fit.  2048 captions of 6 to 77 tokens, 8 heads, 64 channels, in one and
// in the other way: W = 1 40 and 52 us, 2 51 and 62, 4 (145 of them) 50 and 38, of which the first two move 3.7 TB/s; in two passes
// 171 for all.
// The first launch clears `more`, the last one sets it where a sequence (or a row of none) is left for the two passes, which
// else end at once.
template <int D, int W>
struct RaggedWholeCfg {
    using Cut = RaggedCut<W, 1, 32 * W, 1, 1>;
    using Ring = RaggedRing<D, Cut, false>;
    static constexpr int SCALARS = 2 * Ring::BUF_BYTES, ROWS = 32 * W, SECOND = Ring::BUF_BYTES;
    static constexpr int LDS_BYTES = SCALARS + ROWS * 8 + (D % 32 != 0 ? 64 : 0);
    static_assert(W * RowStore<D, Bf16>::BYTES <= SCALARS, "");
};
// Head h of one sequence: its queries and keys, (begin, number)
template <int D, int W, typename E>
DEVINL void ragged_whole(char* smem, const RaggedArgs& a, const raw16* __restrict__ dO, const float* __restrict__ lse, raw16* __restrict__ dq,
                         raw16* __restrict__ dk, raw16* __restrict__ dv, int2 queries, int2 keys, int h, int wave, int lane)
{
    using Cfg = RaggedWholeCfg<D, W>;
    using Ring = typename Cfg::Ring;
    constexpr int KS = D / 16, CT = (D + 31) / 32;
    // (opaque: what is made of it is not kept over the caller's loop, where it took up to 80 registers)
    if constexpr (W == 4) asm volatile("" : "+v"(lane));
    const int l32 = lane % 32, g = lane / 32, nq = queries.y, nk = keys.y;
    const long o_at = (long)queries.x * a.Hq * D + h * D, k_at = (long)keys.x * a.Hq * D + h * D, rs = (long)a.Hq * D;
    const Ring first(a.q + (long)queries.x * a.rs_q + h * D, a.rs_q, dO + o_at, rs, nullptr, 0, nq, smem, wave, lane);
    const Ring second(a.k + (long)keys.x * a.rs_k + h * D, a.rs_k, a.v + (long)keys.x * a.rs_v + h * D, a.rs_v, nullptr, 0, nk,
                      smem + Cfg::SECOND, wave, lane);
    first.fetch(0);
    second.fetch(0);
    const char *qt = smem, *gt = smem + Ring::OFF_B, *kt = smem + Cfg::SECOND, *vt = kt + Ring::OFF_B;
    float* scalars = reinterpret_cast<float*>(smem + Cfg::SCALARS);
    const RaggedLane<D, Cfg::ROWS> at(lane);
    const int row0 = 32 * wave, row = row0 + l32;
    const bool active = row0 < nq, in = row < nq;
    const float saved = in ? lse[(long)h * a.Tq + queries.x + row] : -INFINITY;
    const float lc = saved == -INFINITY ? INFINITY : saved * kLog2e, cs = a.cs;
    auto seen = [&](int r) { return a.causal ? min(max(min(r, nq - 1) + 1 + nk - nq, 0), nk) : nk; };
    const int sees = seen(row), seen_by_all = seen(row0), seen_by_any = seen(row0 + 31);
    f32x16 acc[CT];
    acc_zero(acc);
    Ring::landed_barrier();
    if (active) {
        frag8 qf[KS], gf[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            qf[ks] = at.natural(qt, wave, ks);
            gf[ks] = at.natural(gt, wave, ks);
        }
        f32x16 s[W], dp[W];
        float sum = 0.f;
#pragma unroll
        for (int u = 0; u < W; ++u) {
            if (32 * u >= seen_by_any) continue;
            s[u] = 32 * u + 32 > seen_by_all ? key_mask_block(32 * u, g, sees) : f32x16_zero();
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const frag8 ak = at.natural(kt, u, ks), av = at.natural(vt, u, ks);
                s[u] = E::mfma(ak, qf[ks], s[u]);
                dp[u] = E::mfma(av, gf[ks], ks == 0 ? f32x16_zero() : dp[u]);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[u][e] = fast_exp2(fmaf(s[u][e], cs, -lc));
                sum = fmaf(s[u][e], dp[u][e], sum);
            }
        }
        const float dl = both_halves_sum(sum);
        if (g == 0) {
            scalars[row] = in ? lc - kRaggedShift<E> : INFINITY;
            scalars[Cfg::ROWS + row] = in ? -dl : 0.f;
        }
#pragma unroll
        for (int u = 0; u < W; ++u) {
            if (32 * u >= seen_by_any) continue;
            u32x4 df[2];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                s[u][e] *= dp[u][e] - dl;
                if (e % 2 == 1) df[e / 8][(e / 2) % 4] = E::pack(s[u][e - 1], s[u][e]);
            }
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) acc[ct] = E::mfma(at.transposed(kt, ct, 2 * u + half), as_frag8(df[half]), acc[ct]);
        }
    }
    __syncthreads();
    const bool owns = row0 < nk;
    f32x16 dka[CT], dva[CT];
    acc_zero(dka);
    acc_zero(dva);
    if (owns) {
        auto first_query = [&](int key) { return a.causal ? max(min(key, nk - 1) - nk + nq, 0) : 0; };
        const int from = first_query(row), from_all = first_query(row0 + 31), from_any = first_query(row0);
        frag8 kf[KS], vf[KS];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            kf[ks] = at.natural(kt, wave, ks);
            vf[ks] = at.natural(vt, wave, ks);
        }
#pragma unroll
        for (int hq = 0; hq < W; ++hq)
            if (32 * hq < nq && 32 * hq + 32 > from_any)
                ragged_dkdv_unit<D, E>(at, qt, gt, scalars, Cfg::ROWS, hq, 32 * hq, from, from_all, cs, g, kf, vf, dka, dva);
    }
    __syncthreads();  // the tiles are read: rows on their way out take their place
    char* region = smem + wave * RowStore<D, E>::BYTES;
    if (active) RowStore<D, E>::run(region, acc, a.scale, dq + o_at + row0 * rs, rs, nq - row0, lane);
    if (!owns) return;
    RowStore<D, E>::run(region, dka, a.scale, dk + k_at + row0 * rs, rs, nk - row0, lane);
    RowStore<D, E>::run(region, dva, std::is_same<E, F16>::value ? 1.f / 256.f : 1.f, dv + k_at + row0 * rs, rs, nk - row0, lane);
}
template <int D, int W, typename E>
__global__ void __launch_bounds__(W * 64, (RaggedWholeCfg<D, W>::LDS_BYTES > 80 * 1024 || D == 128 ? 1 : 2))
avion_ragged_whole_kernel(RaggedArgs a, const raw16* __restrict__ dO, const float* __restrict__ lse, raw16* __restrict__ dq,
                          raw16* __restrict__ dk, raw16* __restrict__ dv)
{
    using Cfg = RaggedWholeCfg<D, W>;
    constexpr int LEAST = W == 1 ? -1 : 16 * W;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const bool same = a.off_k == a.off_q && a.Tk == a.Tq;
    if (W == 1 && blockIdx.x == 0 && threadIdx.x == 0) *a.more = 0;
    bool left = false;
    // rows before the first sequence and behind the last one
    if (Cfg::ROWS == a.done && blockIdx.x == 0)
        left = ragged_border(a.off_q, a.S, a.Tq, 1) > 0 || ragged_border(a.off_k, a.S, a.Tk, 1) > 0 ||
               ragged_border(a.off_q, a.S, a.Tq, a.S + 1) < a.Tq || ragged_border(a.off_k, a.S, a.Tk, a.S + 1) < a.Tk;
    if constexpr (W < 4) {
        const int i = blockIdx.x / a.Hq + 1, h = blockIdx.x % a.Hq;
        const int2 queries = ragged_tokens(a.off_q, a.S, a.Tq, i), keys = same ? queries : ragged_tokens(a.off_k, a.S, a.Tk, i);
        const int longer = max(queries.y, keys.y);
        if (Cfg::ROWS == a.done && h == 0 && threadIdx.x == 0 && (left || longer > Cfg::ROWS)) *a.more = 1;
        if (longer > LEAST && longer <= Cfg::ROWS) ragged_whole<D, W, E>(smem, a, dO, lse, dq, dk, dv, queries, keys, h, wave, lane);
        return;
    }
    int before = 0, job = blockIdx.x;
    for (int base = 1; base <= a.S; base += 512) {
        unsigned long long mine[8];
        int found = 0;
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            const int i = base + 64 * x + lane;
            int longer = -1;
            if (i <= a.S) {
                longer = ragged_tokens(a.off_q, a.S, a.Tq, i).y;
                if (!same) longer = max(longer, ragged_tokens(a.off_k, a.S, a.Tk, i).y);
            }
            mine[x] = __ballot(longer > LEAST && longer <= Cfg::ROWS);
            found += __popcll(mine[x]);
            left = left || longer > Cfg::ROWS;
        }
        for (; job < (before + found) * a.Hq; job += gridDim.x) {
            int rank = job / a.Hq - before, i = base;
            unsigned long long m = mine[0];
#pragma unroll
            for (int x = 0; x < 7; ++x) {  // the word of it
                const int n = __popcll(m);
                if (rank >= n && i == base + 64 * x) {
                    rank -= n;
                    i += 64;
                    m = mine[x + 1];
                }
            }
            for (; rank > 0; --rank) m &= m - 1;
            i = __builtin_amdgcn_readfirstlane(i + __ffsll(m) - 1);
            const int2 queries = ragged_tokens(a.off_q, a.S, a.Tq, i), keys = same ? queries : ragged_tokens(a.off_k, a.S, a.Tk, i);
            ragged_whole<D, W, E>(smem, a, dO, lse, dq, dk, dv, queries, keys, job % a.Hq, wave, lane);
            __syncthreads();  // before the next one's tiles
        }
        before += found;
    }
    if (Cfg::ROWS == a.done && blockIdx.x == 0 && __any(left) && threadIdx.x == 0) *a.more = 1;
}
