// Token table: lookup with scaling, and the table's gradient by sorted tokens.
//     y_i = s W[t_i];     dW[v] = s sum over i with t_i = v of dy_i, in an order that n and the tokens fix
// A token outside [0, V) names no row: its y is zero and it adds to no gradient (padding, another device's share of a table).
//
// Lookup: bound by memory bandwidth, one read of a row and one write; a thread moves 16-byte pieces, four in flight, and writes
// past the caches (y is not read again before the next kernel, the table's rows are).  Captions of 512 columns from 50000 rows, us, past
// the caches and through them: 157696 slots 29.7 (5.4 TB/s written) and 41.8, 78848 16.4 and 18.6, 4928 3.7 and 3.7; together with
// the norm that reads y next 103 and 108, 54.5 and 49.3, 9.3 and 8.8: what y leaves in the caches is worth more than the lookup
// gains up to about 80 MB of it.
//
// Gradient: reads dy once and writes every row of dW once (rows that no token names: zeros).  Floating-point sums in a fixed
// order, no atomics on them: the same n and tokens give the same bits.
//   up to kEmbSmallTokens tokens: one launch.  A workgroup per (slot, 512 columns) ends at once unless its slot is the first
//   with its token; else it collects the slots with that token, in order, and sums their rows.  Further workgroups clear the
//   rows that no token names.
//   beyond: the slots are sorted by token, then a workgroup sums the rows of a chunk of sorted slots, writes the sums of the
//   tokens that begin and end among them, and leaves what spans a border to a last launch, as fp32 sums: a token that fills most
//   slots (padding) is spread over the chip like any others.
//   The sort, up to kEmbRankSlots: by counting, in one launch; else a stable radix sort with digits of 8 or 10 bits, per digit
//   one launch that counts and one that places: each of at most 96 workgroups adds up the counts of the ones before it itself,
//   so nothing waits for another workgroup.  The sort is bound by latency, so the unnamed rows are cleared by spare workgroups
//   of its placing launches (or of the sums, where it is one launch).
//   Whether a token is named: the counting launch writes each slot's number to stamp[token] (plain stores, any one of them is
//   right), and row v is named if stamp[v] is a slot whose token is v, so the stamps need no clearing before.
// Both sides at the borders (table 50000 x 512, us): one launch and sorted 700 slots 13.4 and 16.5, 1000 slots, 3/4 of them one
// token's, 19.3 and 18.0; counting and radix 8000 slots 32 and 36, 9000 34 and 35, 12000 40 and 36; 8 and 32 slots a wavefront in
// the sums 20000 slots 41 and 45, 40000 47 and 47, 130000 79 and 66.
// 157696 slots of 512 columns into 50000 rows: 71 us, of these the sums 34 (5.1 TB/s of dy and dW), counting and placing
// 4.2 + 9.8 and 4.1 + 10.2 (half of the unnamed rows cleared beside each placing), the join 9.0 (chains of latency: padding is one token's).
// First version 118.
#pragma once
#include "avion_common.h"
#include "avion_ln.h"

constexpr int kEmbThreads = 256;
constexpr int kEmbFly = 4;                // pieces in flight per thread in the lookup
constexpr int kEmbSmallTokens = 768;      // at most this many: gradient in one launch
constexpr int kEmbCols = 512;             // columns of a workgroup in the sums: 8 per lane
constexpr int kEmbSumWaves = 8;           // of a workgroup in the sums
constexpr int kEmbSumMost = 32;           // sorted slots of a wavefront there: this many, or
constexpr int kEmbSumFew = 8;             // where there are fewer than kEmbSumEnough
constexpr int kEmbSumEnough = 1 << 15;
constexpr int kEmbSortThreads = 1024;
constexpr int kEmbSortTile = 2048;        // slots that a sorting workgroup places at a time: 128 per wavefront
constexpr int kEmbSortGrid = 96;          // sorting workgroups at most
constexpr int kEmbClearBytes = 1 << 15;   // of the table that a clearing workgroup looks after

template <typename T>
DEVINL unsigned token_key(const T* tokens, long i, int V)
{
    const long t = (long)tokens[i];
    return t >= 0 && t < V ? (unsigned)t : (unsigned)V;  // V: no row
}

// 8 values of a row as they lie in memory
template <typename E>
struct EmbPiece {
    u32x4 c;
    DEVINL void load(const void* base, long at) { c = *reinterpret_cast<const u32x4*>(static_cast<const raw16*>(base) + at); }
    DEVINL float get(int e) const { return E::widen(as_frag8(c), e); }
};
template <>
struct EmbPiece<float> {
    f32x4 c[2];
    DEVINL void load(const void* base, long at)
    {
        const f32x4* p = reinterpret_cast<const f32x4*>(static_cast<const float*>(base) + at);
        c[0] = p[0];
        c[1] = p[1];
    }
    DEVINL float get(int e) const { return c[e / 4][e % 4]; }
};

template <typename E>
DEVINL void emb_store8(void* base, long at, const float (&v)[8])
{
    if constexpr (std::is_same_v<E, float>) {
        store8(static_cast<float*>(base) + at, v);
    } else {
        u32x4 w;
#pragma unroll
        for (int p = 0; p < 4; ++p) w[p] = E::pack(v[2 * p], v[2 * p + 1]);
        *reinterpret_cast<u32x4*>(static_cast<raw16*>(base) + at) = w;
    }
}

// T: token type, TE: table's format (16-bit or fp32), E: output's.  pieces = D / 8; magic = ceil(2^32 / pieces).
template <typename T, typename TE, typename E>
__global__ void __launch_bounds__(kEmbThreads)
avion_embedding_fwd_kernel(const T* __restrict__ tokens, const void* __restrict__ table, raw16* __restrict__ y, long n, int V,
                           int D, float scale, int pieces, unsigned magic)
{
    const long total = n * pieces, base = (long)blockIdx.x * (kEmbThreads * kEmbFly);
    const long row0 = base / pieces;
    const unsigned rem = (unsigned)(base - row0 * pieces);  // < pieces; rem + kEmbThreads * kEmbFly stays below 2^16
    unsigned key[kEmbFly], piece[kEmbFly];
    long row[kEmbFly];
#pragma unroll
    for (int k = 0; k < kEmbFly; ++k) {
        const unsigned at = rem + threadIdx.x + kEmbThreads * k;
        const unsigned down = pieces == 1 ? at : (unsigned)(((unsigned long)at * magic) >> 32);
        row[k] = row0 + down;
        piece[k] = at - down * pieces;
        key[k] = row[k] < n ? token_key(tokens, row[k], V) : (unsigned)V;
    }
    EmbPiece<TE> v[kEmbFly];
#pragma unroll
    for (int k = 0; k < kEmbFly; ++k)
        if (key[k] != (unsigned)V) v[k].load(table, (long)key[k] * D + piece[k] * 8);
#pragma unroll
    for (int k = 0; k < kEmbFly; ++k) {
        if (base + threadIdx.x + kEmbThreads * k >= total) continue;
        u32x4 w = {0u, 0u, 0u, 0u};
        if (key[k] != (unsigned)V)
#pragma unroll
            for (int p = 0; p < 4; ++p) w[p] = E::pack(v[k].get(2 * p) * scale, v[k].get(2 * p + 1) * scale);
        __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(y + row[k] * D + piece[k] * 8));
    }
}

// The rows [first, first + rows) of the table that `named` does not claim, cleared by this workgroup: a wavefront asks for 64
// rows at once (one lane each: the answers take two dependent loads).
template <typename TE, int WAVES, typename F>
DEVINL void emb_clear(void* dtable, long first, long rows, int D, F named)
{
    const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const long share = (rows + WAVES - 1) / WAVES, from = wave * share, to = from + share < rows ? from + share : rows;
    for (long r0 = from; r0 < to; r0 += 64) {
        unsigned long clear = __ballot(r0 + lane < to && !named(first + r0 + lane));
        while (clear) {
            const long r = first + r0 + __builtin_ctzl(clear);
            clear &= clear - 1;
            for (int c = lane * 8; c < D; c += 512) emb_store8<TE>(dtable, r * D + c, zero);
        }
    }
}

// ------------------------------------------------------------------------- gradient, few tokens
// grid: (ncol * n) workgroups of slots, then clearing ones of `rows` table rows each (rows <= kEmbSmallRows)
constexpr int kEmbSmallRows = 1024, kEmbSmallThreads = 512;
template <typename T, typename E, typename TE>
__global__ void __launch_bounds__(kEmbSmallThreads)
avion_embedding_bwd_small_kernel(const T* __restrict__ tokens, const raw16* __restrict__ dy, void* __restrict__ dtable, int n,
                                 int V, int D, float scale, int ncol, int rows)
{
    __shared__ unsigned keys[kEmbSmallTokens];
    __shared__ unsigned short slots[kEmbSmallTokens];
    __shared__ unsigned char flags[kEmbSmallRows];
    __shared__ int counts[kEmbSmallTokens / 64];
    constexpr int WAVES = kEmbSmallThreads / 64, FLY = 8;
    __shared__ float sums[WAVES - 1][kEmbCols];
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
    if ((int)blockIdx.x >= ncol * n) {
        const long first = (long)((int)blockIdx.x - ncol * n) * rows;
        const long here = V - first < rows ? V - first : rows;
        for (int i = tid; i < rows; i += kEmbSmallThreads) flags[i] = 0;
        __syncthreads();
        for (int i = tid; i < n; i += kEmbSmallThreads) {
            const long at = (long)token_key(tokens, i, V) - first;
            if (at >= 0 && at < here) flags[at] = 1;
        }
        __syncthreads();
        emb_clear<TE, WAVES>(dtable, first, here, D, [&](long r) { return flags[r - first] != 0; });
        return;
    }
    const int slot = blockIdx.x / ncol, col = (blockIdx.x % ncol) * kEmbCols + lane * 8;
    const unsigned key = token_key(tokens, slot, V);
    if (key == (unsigned)V) return;
    bool before = false;
    for (int i = tid; i < n; i += kEmbSmallThreads) {
        keys[i] = token_key(tokens, i, V);
        before |= i < slot && keys[i] == key;
    }
    if (__syncthreads_or(before)) return;
    // the slots with this token, in order: 64 at a time by vote, places by the votes before
    const int groups = (n + 63) / 64;
    for (int g = wave; g < groups; g += WAVES) {
        const int i = g * 64 + lane;
        const unsigned long hit = __ballot(i < n && keys[i] == key);
        if (lane == 0) counts[g] = __popcll(hit);
    }
    __syncthreads();
    int total = 0;
    for (int g = 0; g < groups; ++g) {
        if (g % (WAVES) == wave) {
            const int i = g * 64 + lane;
            const bool mine = i < n && keys[i] == key;
            const unsigned long hit = __ballot(mine);
            if (mine) slots[total + __popcll(hit & ((1ul << lane) - 1))] = (unsigned short)i;
        }
        total += counts[g];
    }
    __syncthreads();
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (col < D) {
        int i = wave;
        for (; i + (FLY - 1) * WAVES < total; i += FLY * WAVES) {
            EmbPiece<E> v[FLY];
#pragma unroll
            for (int k = 0; k < FLY; ++k) v[k].load(dy, (long)slots[i + WAVES * k] * D + col);
#pragma unroll
            for (int k = 0; k < FLY; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[e] += v[k].get(e);
        }
        for (; i < total; i += WAVES) {
            EmbPiece<E> v;
            v.load(dy, (long)slots[i] * D + col);
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] += v.get(e);
        }
    }
    if (total > 1) {
        if (wave > 0) store8(&sums[wave - 1][lane * 8], acc);
        __syncthreads();
        if (wave == 0)
            for (int w = 0; w < min(WAVES, total) - 1; ++w)
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[e] += sums[w][lane * 8 + e];
    }
    if (wave == 0 && col < D) {
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] *= scale;
        emb_store8<TE>(dtable, (long)key * D + col, acc);
    }
}

// ------------------------------------------------------------------------------------- the sort
// Each of gridDim.x (hist) workgroups owns `per` consecutive slots.  FIRST: keys come from the tokens, slots are their own
// numbers, and the stamps are written.  A digit has BITS bits.
template <typename T, bool FIRST, int BITS>
__global__ void __launch_bounds__(kEmbSortThreads)
avion_embedding_hist_kernel(const T* __restrict__ tokens, const unsigned* __restrict__ keys, unsigned* __restrict__ stamp,
                            unsigned* __restrict__ hist, long n, int V, long per, int shift)
{
    constexpr int BINS = 1 << BITS;
    __shared__ unsigned count[BINS];
    if (threadIdx.x < BINS) count[threadIdx.x] = 0;
    __syncthreads();
    const long from = (long)blockIdx.x * per, to = from + per < n ? from + per : n;
#pragma unroll 2
    for (long i = from + threadIdx.x; i < to; i += kEmbSortThreads) {
        unsigned key;
        if constexpr (FIRST) {
            key = token_key(tokens, i, V);
            if (key != (unsigned)V) stamp[key] = (unsigned)i;
        } else {
            key = keys[i];
        }
        atomicAdd(&count[(key >> shift) & (BINS - 1)], 1u);  // integers: the order does not matter
    }
    __syncthreads();
    if (threadIdx.x < BINS) hist[(long)blockIdx.x * BINS + threadIdx.x] = count[threadIdx.x];
}

// The first nsort workgroups place their slots by this digit, the others clear `rows` table rows each, from row clear_from to
// before clear_to.
template <typename T, bool FIRST, int BITS, typename TE>
__global__ void __launch_bounds__(kEmbSortThreads)
avion_embedding_place_kernel(const T* __restrict__ tokens, const unsigned* __restrict__ keys, const unsigned* __restrict__ slots,
                             const unsigned* __restrict__ hist, const unsigned* __restrict__ stamp, unsigned* __restrict__ keys_out,
                             unsigned* __restrict__ slots_out, void* __restrict__ dtable, long n, int V, int D, long per, int nsort,
                             int shift, int rows, long clear_from, long clear_to)
{
    constexpr int BINS = 1 << BITS, WAVES = kEmbSortThreads / 64, ROUNDS = kEmbSortTile / kEmbSortThreads, GROUPS = kEmbSortThreads / BINS,
                  FLY = 32;
    __shared__ unsigned short count[WAVES][BINS];        // of a tile, by wavefront; then what the wavefronts before have
    __shared__ unsigned total[GROUPS][BINS], ahead[GROUPS][BINS];
    __shared__ unsigned base[BINS];                      // where the next slot with this digit goes
    __shared__ unsigned part[WAVES];
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
    if ((int)blockIdx.x >= nsort) {
        const long first = clear_from + (long)((int)blockIdx.x - nsort) * rows;
        emb_clear<TE, WAVES>(dtable, first, clear_to - first < rows ? clear_to - first : rows, D, [&](long r) {
            const unsigned s = stamp[r];
            return s < n && token_key(tokens, s, V) == (unsigned)r;
        });
        return;
    }
    const long from = (long)blockIdx.x * per, to = from + per < n ? from + per : n;
    unsigned key[ROUNDS], slot[ROUNDS], rank[ROUNDS];
    auto load = [&](long tile) {
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const long i = tile + wave * (kEmbSortTile / WAVES) + r * 64 + lane;
            key[r] = slot[r] = 0;
            if (i < to) {
                key[r] = FIRST ? token_key(tokens, i, V) : keys[i];
                slot[r] = FIRST ? (unsigned)i : slots[i];
            }
        }
    };
    load(from);
    // a digit's first place: all slots with a smaller digit, then this digit's slots of the workgroups before.  The workgroups'
    // counts are read by GROUPS groups of threads, a digit a thread.
    {
        const int b = tid % BINS, group = tid / BINS, share = (nsort + GROUPS - 1) / GROUPS;
        const int g_from = group * share, g_to = min(g_from + share, nsort);
        unsigned t = 0, a = 0;
#pragma unroll 1
        for (int g0 = g_from; g0 < g_to; g0 += FLY) {
            unsigned c[FLY];
#pragma unroll
            for (int g = 0; g < FLY; ++g) c[g] = hist[min(g0 + g, nsort - 1) * BINS + b];
#pragma unroll
            for (int g = 0; g < FLY; ++g) {
                t += g0 + g < g_to ? c[g] : 0u;
                a += g0 + g < min(g_to, (int)blockIdx.x) ? c[g] : 0u;
            }
        }
        total[group][b] = t;
        ahead[group][b] = a;
    }
    __syncthreads();
    unsigned mine = 0, before = 0;
    if (tid < BINS)
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            mine += total[g][tid];
            before += ahead[g][tid];
        }
    unsigned upto = mine;  // sum over the threads of this wavefront up to this one
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const unsigned o = __shfl_up(upto, off, 64);
        if (lane >= off) upto += o;
    }
    if (lane == 63) part[wave] = upto;
    __syncthreads();
    if (tid < BINS) {
        unsigned start = upto - mine;
#pragma unroll
        for (int w = 0; w < BINS / 64; ++w) start += w < wave ? part[w] : 0u;
        base[tid] = start + before;
    }
    for (long tile = from; tile < to; tile += kEmbSortTile) {
        if (tile > from) load(tile);
        for (int b = tid; b < WAVES * BINS / 2; b += kEmbSortThreads) reinterpret_cast<unsigned*>(count)[b] = 0;
        __syncthreads();
        // a slot's rank among its wavefront's with the same digit: the lanes below that vote alike, and the rounds before
        unsigned long same[ROUNDS];
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const unsigned digit = (key[r] >> shift) & (BINS - 1);
            same[r] = __ballot(tile + wave * (kEmbSortTile / WAVES) + r * 64 + lane < to);
#pragma unroll
            for (int b = 0; b < BITS; ++b) {
                const unsigned long vote = __ballot((digit >> b) & 1);
                same[r] &= (digit >> b) & 1 ? vote : ~vote;
            }
        }
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const unsigned below = __popcll(same[r] & ((1ul << lane) - 1));
            rank[r] = 0;
            if (tile + wave * (kEmbSortTile / WAVES) + r * 64 + lane < to) {
                volatile unsigned short* c = &count[wave][(key[r] >> shift) & (BINS - 1)];
                rank[r] = *c + below;
                if (below == 0) *c = (unsigned short)(rank[r] + __popcll(same[r]));
            }
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
        unsigned here = 0;
        if (tid < BINS) {
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const unsigned c = count[w][tid];
                count[w][tid] = (unsigned short)here;
                here += c;
            }
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const long i = tile + wave * (kEmbSortTile / WAVES) + r * 64 + lane;
            if (i < to) {
                const unsigned d = (key[r] >> shift) & (BINS - 1), p = base[d] + count[wave][d] + rank[r];
                if (p < n) {  // always, unless the tokens change between the launches
                    keys_out[p] = key[r];
                    slots_out[p] = slot[r];
                }
            }
        }
        __syncthreads();
        if (tid < BINS) base[tid] += here;
    }
}

// Up to kEmbRankSlots slots: a slot's sorted place is the number of slots before it, counted: those with a smaller token, and
// those with the same one and a smaller number.  A workgroup places 64 slots; its 16 wavefronts each compare them with a share
// of the keys.  stamp[token]: the place of one of its slots.
constexpr int kEmbRankSlots = 8192;
template <typename T>
__global__ void __launch_bounds__(kEmbSortThreads)
avion_embedding_rank_kernel(const T* __restrict__ tokens, unsigned* __restrict__ keys_out, unsigned* __restrict__ slots_out,
                            unsigned* __restrict__ stamp, int n, int V)
{
    constexpr int WAVES = kEmbSortThreads / 64;
    __shared__ u32x4 keys4[kEmbRankSlots / 4];
    __shared__ unsigned part[WAVES][64];
    unsigned* keys = reinterpret_cast<unsigned*>(keys4);
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64, n4 = (n + 3) / 4;
    for (int i = tid; i < 4 * n4; i += kEmbSortThreads) keys[i] = i < n ? token_key(tokens, i, V) : ~0u;
    __syncthreads();
    const int first = blockIdx.x * 64, i = first + lane;
    const unsigned mine = i < n ? keys[i] : ~0u;
    unsigned below = 0;
    // all slots before the workgroup's (equal ones count), its own (equal ones with a smaller number), all behind
    for (int j = wave; j < first / 4; j += WAVES) {
        const u32x4 k = keys4[j];
#pragma unroll
        for (int e = 0; e < 4; ++e) below += k[e] <= mine ? 1u : 0u;
    }
    for (int j = first / 4 + 16 + wave; j < n4; j += WAVES) {
        const u32x4 k = keys4[j];
#pragma unroll
        for (int e = 0; e < 4; ++e) below += k[e] < mine ? 1u : 0u;
    }
    for (int j = first + wave; j < min(first + 64, n); j += WAVES) {
        const unsigned k = keys[j];
        below += k < mine || (k == mine && j < i) ? 1u : 0u;
    }
    part[wave][lane] = below;
    __syncthreads();
    if (wave > 0 || i >= n) return;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) below += part[w][lane];
    keys_out[below] = mine;
    slots_out[below] = (unsigned)i;
    if (mine != (unsigned)V) stamp[mine] = below;
}

// ------------------------------------------------------------------------------------- the sums
// Sums of kEmbSumWaves * PER sorted slots (a chunk) in 512 columns.  heads[chunk][D]: the sum of a token that began in a chunk
// before, tails: of one that begins here and goes on in the next.
template <int PER, typename E, typename TE>
__global__ void __launch_bounds__(kEmbSumWaves * 64)
avion_embedding_sum_kernel(const unsigned* __restrict__ keys, const unsigned* __restrict__ slots, const raw16* __restrict__ dy,
                           void* __restrict__ dtable, float* __restrict__ heads, float* __restrict__ tails, long n, int V, int D,
                           float scale, int nchunks, int ncol, const unsigned* __restrict__ stamp, int rows)
{
    constexpr int WAVES = kEmbSumWaves, FLY = PER < 16 ? PER : 16;
    const int sums = nchunks * ncol, chunk = blockIdx.x / ncol, block = blockIdx.x - chunk * ncol;
    if ((int)blockIdx.x >= sums) {  // (few slots: the table is cleared here)
        const long r0 = (long)((int)blockIdx.x - sums) * rows;
        emb_clear<TE, WAVES>(dtable, r0, V - r0 < rows ? V - r0 : rows, D, [&](long r) {
            const unsigned s = stamp[r];
            return s < n && keys[s] == (unsigned)r;
        });
        return;
    }
    __shared__ float sh_head[WAVES][kEmbCols], sh_tail[WAVES][kEmbCols];
    __shared__ unsigned sh_key[WAVES];  // of the tail
    __shared__ int sh_what[WAVES];      // 1: has a head, 2: the head ends here, 4: has a tail
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int col = block * kEmbCols + lane * 8, read_col = col < D ? col : 0;
    const bool in = col < D;
    const long first = ((long)chunk * WAVES + wave) * PER;
    const int count = first >= n ? 0 : n - first < PER ? (int)(n - first) : PER;
    const unsigned none = (unsigned)V;
    // lane l: key and slot of sorted place first + l, lane `count`: the key behind, lane 63: the key before.  (A key is at most
    // V and a slot below n, unless the tokens change between the launches.)
    unsigned key = none, slot = 0;
    const long place = lane == 63 ? first - 1 : first + lane;
    if (place >= 0 && place < n && (lane <= count || lane == 63)) {
        key = min(keys[place], none);
        slot = min(slots[place], (unsigned)(n - 1));
    }
    const unsigned behind = __shfl_down(key, 1, 64);
    const int valid = __popcll(__ballot(lane < count && key != none));  // the slots without a row are the last ones
    const int last = valid - 1;
    // after these places a sum is complete, or passed on
    const unsigned long cuts = __ballot(lane < valid && (lane == last || behind != key));
    const bool head = valid > 0 && __builtin_amdgcn_readlane(key, 63) == __builtin_amdgcn_readfirstlane(key);
    const bool on = valid > 0 && __builtin_amdgcn_readlane(behind, last < 0 ? 0 : last) == __builtin_amdgcn_readlane(key, last < 0 ? 0 : last);
    const int head_cut = head ? __builtin_ctzl(cuts | 1ul << 63) : -1;   // the sum that began before ends or is passed on here
    const int tail_cut = on && head_cut != last ? last : -1;             // the sum that begins here and goes on
    if (lane == 0) {
        sh_what[wave] = (head ? 1 : 0) | (head && !(on && head_cut == last) ? 2 : 0) | (tail_cut >= 0 ? 4 : 0);
        if (tail_cut >= 0) sh_key[wave] = __builtin_amdgcn_readlane(key, last);
    }
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    // (a loop: unrolled, the cuts' code is so long that small launches wait for instructions)
#pragma unroll 1
    for (int i0 = 0; i0 < valid; i0 += FLY) {
        u32x4 raw[FLY];
#pragma unroll
        for (int k = 0; k < FLY; ++k) {  // (places behind the last valid one: any row, their sum goes nowhere)
            const raw16* row = dy + (long)__builtin_amdgcn_readlane(slot, i0 + k) * D;
            raw[k] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(row + read_col));
        }
        const unsigned here = (unsigned)(cuts >> i0);
#pragma unroll
        for (int k = 0; k < FLY; ++k) {
#pragma unroll
            for (int e = 0; e < 8; ++e) acc[e] += E::widen(as_frag8(raw[k]), e);
            if (here >> k & 1) {
                if (i0 + k == head_cut || i0 + k == tail_cut) {
                    store8(i0 + k == head_cut ? &sh_head[wave][lane * 8] : &sh_tail[wave][lane * 8], acc);
                } else if (in) {
                    float o[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[e] = acc[e] * scale;
                    emb_store8<TE>(dtable, (long)__builtin_amdgcn_readlane(key, i0 + k) * D + col, o);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[e] = 0.f;
            }
        }
    }
    __syncthreads();
    // the parts that meet at the wavefronts' borders, in order
    if (wave != 0 || !in) return;
    bool running = false, began_here = false;
    unsigned run_key = none;
    float run[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int w = 0; w < WAVES; ++w) {
        const int f = sh_what[w];
        if (f & 1) {
#pragma unroll
            for (int e = 0; e < 8; ++e) run[e] += sh_head[w][lane * 8 + e];
            running = true;
            if (f & 2) {
                if (began_here) {
                    float o[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[e] = run[e] * scale;
                    emb_store8<TE>(dtable, (long)run_key * D + col, o);
                } else {
                    store8(heads + (long)chunk * D + col, run);
                }
                running = began_here = false;
#pragma unroll
                for (int e = 0; e < 8; ++e) run[e] = 0.f;
            }
        }
        if (f & 4) {
#pragma unroll
            for (int e = 0; e < 8; ++e) run[e] = sh_tail[w][lane * 8 + e];
            running = began_here = true;
            run_key = sh_key[w];
        }
    }
    if (running) store8((began_here ? tails : heads) + (long)chunk * D + col, run);
}

// The tokens that span chunks: the workgroup of the chunk where one begins adds its tail and the heads behind it, in a fixed
// order: 16 groups of threads each take every 16th, 128 columns a workgroup.
constexpr int kEmbJoinGroups = 16, kEmbJoinCols = 128;
template <typename TE>
__global__ void __launch_bounds__(kEmbJoinGroups * kEmbJoinCols / 4)
avion_embedding_join_kernel(const unsigned* __restrict__ keys, const float* __restrict__ heads, const float* __restrict__ tails,
                            void* __restrict__ dtable, long n, int V, int D, float scale, long nchunks, int chunk)
{
    constexpr int LANES = kEmbJoinCols / 4, THREADS = kEmbJoinGroups * LANES, FLY = 16;
    __shared__ f32x4 sh[kEmbJoinGroups][LANES];
    const long c = blockIdx.x, end = (c + 1) * chunk;
    if (end >= n) return;
    const unsigned key = keys[end - 1];
    if (key >= (unsigned)V || keys[end] != key) return;
    if (c > 0 && keys[c * chunk - 1] == key) return;  // began before this chunk
    // the chunks whose first slot has this token follow this one without a gap
    long behind = 0;
    for (long from = c + 1; from < nchunks; from += THREADS) {
        const long q = from + threadIdx.x;
        const int hits = __syncthreads_count(q < nchunks && keys[q * chunk] == key);
        behind += hits;
        if (hits < THREADS) break;
    }
    const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
    const int col = blockIdx.y * kEmbJoinCols + lane * 4;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    if (col < D) {
        const float* p = heads + (c + 1) * D + col;
        if (group == 0) acc = *reinterpret_cast<const f32x4*>(tails + c * D + col);
        long q = group;
        for (; q + (FLY - 1) * kEmbJoinGroups < behind; q += FLY * kEmbJoinGroups) {
            f32x4 v[FLY];
#pragma unroll
            for (int k = 0; k < FLY; ++k) v[k] = *reinterpret_cast<const f32x4*>(p + (q + k * kEmbJoinGroups) * D);
#pragma unroll
            for (int k = 0; k < FLY; ++k) acc += v[k];
        }
        for (; q < behind; q += kEmbJoinGroups) acc += *reinterpret_cast<const f32x4*>(p + q * D);
    }
    sh[group][lane] = acc;
    for (int half = kEmbJoinGroups / 2; half > 0; half /= 2) {
        __syncthreads();
        if (group < half) {
            acc += sh[group + half][lane];
            sh[group][lane] = acc;
        }
    }
    if (group == 0 && col < D) {
        acc *= scale;
        if constexpr (std::is_same_v<TE, float>) {
            *reinterpret_cast<f32x4*>(static_cast<float*>(dtable) + (long)key * D + col) = acc;
        } else {
            *reinterpret_cast<u32x2*>(static_cast<raw16*>(dtable) + (long)key * D + col) =
                u32x2{TE::pack(acc[0], acc[1]), TE::pack(acc[2], acc[3])};
        }
    }
}
