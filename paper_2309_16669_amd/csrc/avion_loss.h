// Softmax cross entropy of a linear layer's outputs that are never kept: rows x [T, D] against a table w [V, D] (the vocabulary of a
// text decoder, or the other side of a contrastive batch), z = s x w^T:
//     lse_m = ln sum_v exp z_mv,   loss_m = lse_m - z_{m, t_m}
//     dz = (softmax(z) - onehot(t)) dloss_m,   dx = s dz w,   dw = s dz^T x
// T V numbers do not fit what T D and V D do, so the forward forms z tile by tile and keeps a running maximum and sum a row; the
// backward forms it again, one piece of the vocabulary after the other, rounds dz of that piece to the operands' format (workspace,
// bounded) and multiplies it with w and with x.  2 T V D operations forward, 6 backward; all four products are bound by the matrix
// units, the forward of few rows by w's bytes.
//
// The product.  C [b, a] = sum_k B[b, k] A[a, k], tiles of TB x TA, 64 deep steps; an operand lies in memory either with k contiguous
// (rows x or w) or with its own index contiguous (its rows are k: dz and x in dw, w in dx).
//   Either comes to LDS by LDS-direct loads, 128 bytes of k a row or whole rows of the tile's width, and leaves it as fragments
//   of 8 consecutive k: rows of 128 bytes with ds_read_b128, their eight 16-byte chunks permuted by a XOR with bits 1..3 of the row
//   number; rows of k with two transposing ds_read_b64_tr_b16 (4 k each), their 64-byte units permuted by a XOR with the row
//   number mod 4.  Both meet distinct banks.
//   Two buffers of a step (four in tiles of 128 gained nothing where a compute unit has one workgroup: 2048 x 2048 x 512 forward 10.4 and
//   11.6 us); fragments of 16 k are read while the 16 before are multiplied; before a step's last ones the next step is awaited, and
//   this one's buffer, which everybody then holds in registers, is filled again.  Steps of a workgroup's tiles form one stream, so that
//   the next tile's first steps are on their way during the end of a tile.
//   8192 cubed: 1212 to 1258 TFLOP/s by the operands' layouts (the library's product 1301); matrix units busy 62 % of the cycles, LDS
//   reads 23 %, at 1.8 GHz.
//   A is the contiguous index of the result: a lane's accumulators are 4 consecutive a of one row b.
#pragma once
#include "avion_common.h"

enum class Along { kK, kIndex };  // what is contiguous in memory

struct LossOperand {
    const raw16* p;
    long ld;      // elements between rows
    int extent;   // of its own index
    int rows;     // kIndex: rows of k that there are (the others count as zeros)
};

constexpr int kLossStep = 64;  // k of a step

// One operand's tile in a buffer: how this wavefront brings it there and how a lane reads it
template <Along ALONG, int W, int WAVES>
struct LossTile {
    static constexpr int BYTES = W * 128, BLOCKS = W / 8, PER = (BLOCKS + WAVES - 1) / WAVES;
    static constexpr int CPR = ALONG == Along::kK ? 8 : W / 8, RPB = 64 / CPR, ROW = CPR * 16;  // chunks a row, rows a 1 KB block
    static_assert(ALONG == Along::kK || (W >= 128 && W <= 512), "a row of k holds whole groups of four 64-byte units");
    static_assert(WAVES % 2 == 0 || ALONG == Along::kIndex, "a wavefront's blocks are all even or all odd");
    LossOperand op;
    int K, wave;
    unsigned row_at, chunk;  // this lane's part of a load: byte offset of its row in block `wave`, byte offset in the row
    unsigned read_at;        // of a fragment
    unsigned turn;
    u32x4 desc;

    DEVINL LossTile(const LossOperand& op_, int K_, int wave_, int lane) : op(op_), K(K_), wave(wave_)
    {
        const unsigned row = (unsigned)(wave * RPB + lane / CPR);
        row_at = row * (unsigned)(op.ld * 2);
        if constexpr (ALONG == Along::kK) chunk = ((lane & 7) ^ (lane >> 4 & 3) ^ (wave & 1) * 4) * 16;
        else chunk = (((unsigned)lane % CPR) ^ (row & 3) * 4) * 16;
        const int l32 = lane % 32, g = lane / 32, G = lane >> 4, j = lane & 15;
        if constexpr (ALONG == Along::kK) {
            read_at = (unsigned)l32 * 128;
            turn = (g ^ (l32 >> 1 & 7)) * 16;
        } else {
            read_at = (unsigned)(8 * g + (j >> 2)) * ROW + (G & 1) * 32 + (j & 3) * 8;
            turn = (j >> 2) * 64;
        }
        desc = RawBuffer(op.p, 0).words;
    }
    // the tile begins at index i0
    DEVINL void tile(int i0)
    {
        if constexpr (ALONG == Along::kK) {
            const int rows = min(op.extent - i0, W);
            desc = RawBuffer(op.p + (long)i0 * op.ld, (unsigned)(((long)(rows - 1) * op.ld + K) * 2)).words;
        }
    }
    // its step from k0 on, to LDS address `to`
    DEVINL void fetch(int i0, int k0, unsigned to) const
    {
        u32x4 d = desc;
        unsigned v = row_at + chunk;
        if constexpr (ALONG == Along::kK) {
            v = (unsigned)k0 * 2 + chunk < (unsigned)K * 2 ? v + (unsigned)k0 * 2 : kOutOfRangeBase;
        } else {
            const int rows = min(op.rows - k0, kLossStep);
            d = RawBuffer(op.p + (long)k0 * op.ld + i0, rows > 0 ? (unsigned)(((long)(rows - 1) * op.ld + (op.extent - i0)) * 2) : 0).words;
        }
        const unsigned down = (unsigned)(WAVES * RPB) * (unsigned)(op.ld * 2);
        const RawBuffer b(d);
        const unsigned at = to + wave * 1024;
        if constexpr (PER % 4 == 0 && BLOCKS % WAVES == 0) {
#pragma unroll
            for (int i = 0; i < PER; i += 4)
                load_to_lds16_x4<WAVES * 1024>(b, b, b, b, at + i * WAVES * 1024, v + i * down, v + (i + 1) * down, v + (i + 2) * down, v + (i + 3) * down);
        } else {
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (BLOCKS % WAVES == 0 || wave + i * WAVES < BLOCKS) load_to_lds16(b, at + i * WAVES * 1024, v + i * down);
        }
    }
    // fragment of the 32 indexes from 32 * t on, k 16 * ks .. (the wavefront's lanes: index l % 32, 8 k of half l / 32)
    DEVINL frag8 read(unsigned from, int t, int ks) const
    {
        if constexpr (ALONG == Along::kK) {
            typedef const __attribute__((address_space(3))) frag8* ptr;
            return *(ptr)(from + read_at + (turn ^ (ks * 32)) + t * 4096);
        } else {
            const unsigned at = from + read_at + (((unsigned)t * 64) ^ turn) + ks * 16 * ROW;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)at);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(at + 4 * ROW));
            const u32x2 l2 = __builtin_bit_cast(u32x2, lo), h2 = __builtin_bit_cast(u32x2, hi);
            return as_frag8(u32x4{l2[0], l2[1], h2[0], h2[1]});
        }
    }
};

template <Along AA, Along AB, int TA_, int TB_, int WA_, int WB_>
struct LossCfg {
    static constexpr int TA = TA_, TB = TB_, WA = WA_, WB = WB_;
    static constexpr int WAVES = WA * WB, NT = WAVES * 64;
    static constexpr int NI = TA / WA / 32, MI = TB / WB / 32;  // 32 x 32 tiles of a wavefront
    using TileA = LossTile<AA, TA, WAVES>;
    using TileB = LossTile<AB, TB, WAVES>;
    static constexpr int STAGE = TileA::BYTES + TileB::BYTES;
    static constexpr int LOADS = TileA::PER + TileB::PER;  // of a wavefront for a step
    static constexpr int OUT_ROW = NI * 64 + 16, OUT_BYTES = (NI == 2 ? 16 : 32) * OUT_ROW;  // a wavefront's rows on their way out
    static constexpr int LDS_BYTES = 2 * STAGE + WAVES * OUT_BYTES;
    static_assert(LDS_BYTES <= 160 * 1024 && TileA::BLOCKS % WAVES == 0 && TileB::BLOCKS % WAVES == 0 && LOADS < 64, "");
};

// All but this wavefront's youngest `left` steps of LOADS loads have arrived (stores and other loads among them are younger than they
// count here: that waits for more, never for less), its LDS reads are done, and so everybody's.
template <int LOADS>
DEVINL void loss_landed_barrier(int left)
{
    if (left == 1) asm volatile("s_waitcnt vmcnt(%0)\n\ts_waitcnt lgkmcnt(0)\n\ts_barrier" ::"i"(LOADS) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)\n\ts_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Tile number -> its places: 8 blocks of b, then the next a.  What an XCD's workgroups hold at a time, neighbouring numbers, is then 8
// blocks of b by a few of a, whose operands fit its L2.
DEVINL void loss_place(int tile, int na, int nb, int& a, int& b)
{
    const int group = tile / (8 * na), in = tile - group * 8 * na, blocks = min(8, nb - group * 8);
    a = in / blocks;
    b = group * 8 + in - a * blocks;
}

// The tiles place(0) .. place(count - 1) of one workgroup, each an (a0, b0) and steps k0 .. k1 - 1 (k1 > k0); done(n, a0, b0, acc) takes
// the sums of tile n.
struct LossPlace {
    int a0, b0, k0, k1;
};
// begin(n, place) is called with the loads of the tile's first step: what it asks for in the same way has arrived when the tile is done.
template <typename Cfg, typename E, typename Place, typename Begin, typename Done>
DEVINL void loss_product(char* smem, const LossOperand& opa, const LossOperand& opb, int K, int count, int wave, int lane, Place place, Begin begin,
                         Done done)
{
    constexpr int MI = Cfg::MI, NI = Cfg::NI;
    if (count <= 0) return;
    const int wa = wave % Cfg::WA, wb = wave / Cfg::WA;
    typename Cfg::TileA ta(opa, K, wave, lane);
    typename Cfg::TileB tb(opb, K, wave, lane);
    const unsigned lds = lds_address(smem);
    // the next step to fetch
    int f_n = 0;
    LossPlace f = place(0);
    int f_k = f.k0;
    ta.tile(f.a0);
    tb.tile(f.b0);
    auto fetch = [&](int buf) {
        const unsigned to = lds + buf * Cfg::STAGE;
        if (f_k == f.k0) begin(f_n, f);
        ta.fetch(f.a0, f_k * kLossStep, to);
        tb.fetch(f.b0, f_k * kLossStep, to + Cfg::TileA::BYTES);
        if (++f_k == f.k1 && ++f_n < count) {
            f = place(f_n);
            f_k = f.k0;
            ta.tile(f.a0);
            tb.tile(f.b0);
        }
    };
    int ahead = 0;  // steps asked for behind the one that is awaited next
    fetch(0);
    if (f_n < count) {
        fetch(1);
        ++ahead;
    }
    loss_landed_barrier<Cfg::LOADS>(ahead);
    frag8 fa[NI], fb[MI];
    auto read = [&](int buf, int ks) {
        const unsigned from = lds + buf * Cfg::STAGE;
#pragma unroll
        for (int j = 0; j < NI; ++j) fa[j] = ta.read(from, wa * NI + j, ks);
#pragma unroll
        for (int i = 0; i < MI; ++i) fb[i] = tb.read(from + Cfg::TileA::BYTES, wb * MI + i, ks);
    };
    read(0, 0);
    int buf = 0;
    f32x16 acc[MI][NI];
    for (int n = 0; n < count; ++n) {
        const LossPlace p = place(n);
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[i][j] = f32x16_zero();
        for (int k = p.k0; k < p.k1; ++k) {
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                frag8 ca[NI], cb[MI];
#pragma unroll
                for (int j = 0; j < NI; ++j) ca[j] = fa[j];
#pragma unroll
                for (int i = 0; i < MI; ++i) cb[i] = fb[i];
                if (ks < 3) {
                    read(buf, ks + 1);
                } else if (k + 1 < p.k1 || n + 1 < count) {
                    loss_landed_barrier<Cfg::LOADS>(--ahead);  // the next step is there, and this one in everybody's registers
                    if (f_n < count) {
                        fetch(buf);
                        ++ahead;
                    }
                    read(buf ^ 1, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < MI; ++i)
#pragma unroll
                    for (int j = 0; j < NI; ++j) acc[i][j] = E::mfma(ca[j], cb[i], acc[i][j]);
                __builtin_amdgcn_sched_barrier(0);
            }
            buf ^= 1;
        }
        done(n, p.a0, p.b0, acc);
    }
    __syncthreads();  // (a second product may begin in the same buffers)
}

// A wavefront's 32 x (32 NI) part of a result with contiguous a, rounded, to rows of `out` (ld elements apart): through LDS, so that
// the stores write whole rows of it.  value(j, e): register e of tile j.  Columns from `cols` on and rows from `rows` on are not stored.
template <int NI, typename E, typename Value>
DEVINL void loss_store(char* stage, raw16* out, long ld, int rows, int cols, int lane, Value value)
{
    constexpr int ROW = NI * 64 + 16, LANES = NI * 4, STEP = 64 / LANES, BATCH = NI == 2 ? 16 : 32;
    const int l32 = lane % 32, g = lane / 32;
#pragma unroll
    for (int half = 0; half < 32 / BATCH; ++half) {
        if (l32 / BATCH == half) {
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    *reinterpret_cast<u32x2*>(stage + l32 % BATCH * ROW + 64 * j + 16 * c + 8 * g) =
                        u32x2{E::pack(value(j, 4 * c), value(j, 4 * c + 1)), E::pack(value(j, 4 * c + 2), value(j, 4 * c + 3))};
        }
        asm volatile("" ::: "memory");  // (LDS takes a wavefront's accesses in the order of the program)
#pragma unroll
        for (int r = 0; r < BATCH; r += STEP) {
            const int row = half * BATCH + r + lane / LANES, col = lane % LANES * 8;
            if (row < rows && col < cols)
                *reinterpret_cast<u32x4*>(out + (long)row * ld + col) = *reinterpret_cast<const u32x4*>(stage + (r + lane / LANES) * ROW + col * 2);
        }
        asm volatile("" ::: "memory");
    }
}

// ------------------------------------------------------------------------------------------- forward
struct LossArgs {
    const raw16 *x, *w;
    const void* targets;
    long rs_x, rs_w;
    int T, V, D;
    int wide;          // targets are int64
    long long ignore;
    float cs;          // scale * log2 e
    float scale;
};
// the target of row m, -1 where it has none
DEVINL int loss_target(const LossArgs& a, int m)
{
    if (m >= a.T) return -1;
    const long t = a.wide ? static_cast<const long*>(a.targets)[m] : (long)static_cast<const int*>(a.targets)[m];
    return t >= 0 && t < a.V && t != a.ignore ? (int)t : -1;
}

constexpr float kLossNone = -3.0e38f;

// A workgroup takes TB rows through one of `slabs` runs of vocabulary tiles.  A lane holds, for each of its MI rows, the maximum and sum
// (base 2, scaled) over the columns that its registers hold; they meet once, at the end: parts [slabs][T] of (maximum, sum).  The lane
// that holds a row's target leaves its logit.
// Medians on two cards: 16384 x 50000 x 768 1129 and 1179 us = 1.07 to 1.11 PFLOP/s, matrix units 52 % of the cycles; 5 x 50000 x 512 11 us for 51
// MB; 2048 x 2048 x 512 10.
template <int TA, int TB, int WA, int WB, typename E>
__global__ void __launch_bounds__(WA* WB * 64, 2)
avion_loss_fwd_kernel(LossArgs a, float2* __restrict__ parts, float* __restrict__ hit, int slabs, unsigned* __restrict__ ticket)
{
    using Cfg = LossCfg<Along::kK, Along::kK, TA, TB, WA, WB>;
    constexpr int MI = Cfg::MI, NI = Cfg::NI;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    __shared__ float2 meet[WA][TB];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l32 = lane % 32, g = lane / 32;
    const int wa = wave % WA, wb = wave / WA;
    const int blocks = (a.T + TB - 1) / TB, logical = xcd_local_id(blockIdx.x, blocks * slabs);
    if (blockIdx.x == 0 && threadIdx.x == 0) *ticket = 0;  // of the next launch
    if (logical < 0) return;
    int slab, block;
    loss_place(logical, slabs, blocks, slab, block);
    const int b0 = block * TB, ntiles = (a.V + TA - 1) / TA;
    const int first = (int)((long)ntiles * slab / slabs), last = (int)((long)ntiles * (slab + 1) / slabs);
    float m[MI], l[MI];
    int target[MI];
#pragma unroll
    for (int i = 0; i < MI; ++i) {
        m[i] = kLossNone;
        l[i] = 0.f;
        target[i] = loss_target(a, b0 + (wb * MI + i) * 32 + l32);
    }
    const LossOperand opa{a.w, a.rs_w, a.V, 0}, opb{a.x, a.rs_x, a.T, 0};
    loss_product<Cfg, E>(
        smem, opa, opb, a.D, last - first, wave, lane,
        [&](int n) { return LossPlace{(first + n) * TA, b0, 0, (a.D + kLossStep - 1) / kLossStep}; }, [](int, const LossPlace&) {},
        [&](int, int a0, int, f32x16(&acc)[MI][NI]) {
            const int from = a0 + wa * NI * 32;
            const bool ragged = from + NI * 32 > a.V;
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                // the target's logit: register e of tile j holds column from + 32 j + 8 (e / 4) + 4 g + e % 4
                const int at = target[i] - from;
                if (__any(target[i] >= 0 && at >= 0 && at < NI * 32)) {
                    float z = 0.f;
#pragma unroll
                    for (int j = 0; j < NI; ++j)
#pragma unroll
                        for (int e = 0; e < 16; ++e) z = at == 32 * j + 8 * (e / 4) + 4 * g + e % 4 ? acc[i][j][e] : z;
                    if (target[i] >= 0 && at >= 0 && at < NI * 32 && (at / 4) % 2 == g) hit[b0 + (wb * MI + i) * 32 + l32] = z * a.scale;
                }
                if (ragged) {
#pragma unroll
                    for (int j = 0; j < NI; ++j)
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            if (from + 32 * j + 8 * (e / 4) + 4 * g + e % 4 >= a.V) acc[i][j][e] = -INFINITY;
                }
                float top = max16(acc[i][0]);
#pragma unroll
                for (int j = 1; j < NI; ++j) top = fmaxf(top, max16(acc[i][j]));
                const float mn = fmaxf(m[i], top * a.cs);
                l[i] *= fast_exp2(m[i] - mn);
                m[i] = mn;
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < NI; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e) sum += fast_exp2(fmaf(acc[i][j][e], a.cs, -mn));
                l[i] += sum;
            }
        });
#pragma unroll
    for (int i = 0; i < MI; ++i) {
        const float mn = both_halves_max(m[i]), sum = both_halves_sum(l[i] * fast_exp2(m[i] - mn));
        if (g == 0) meet[wa][(wb * MI + i) * 32 + l32] = float2{mn, sum};
    }
    __syncthreads();
    for (int r = threadIdx.x; r < TB; r += Cfg::NT) {
        if (b0 + r >= a.T) continue;
        float mn = kLossNone, sum = 0.f;
#pragma unroll
        for (int x = 0; x < WA; ++x) mn = fmaxf(mn, meet[x][r].x);
#pragma unroll
        for (int x = 0; x < WA; ++x) sum += meet[x][r].y * fast_exp2(meet[x][r].x - mn);
        parts[(long)slab * a.T + b0 + r] = float2{mn, sum};
    }
}

// Rows joined over the runs, LANES lanes a row: lse, loss; and, for a mean or sum, the losses of 256 / LANES rows and how many of them
// have a target; the workgroup that comes last (a counter says which) adds these up, in their order.  (391 runs of 5 rows: one lane 70
// us, 16 lanes 8; the total in a launch of its own 3 to 5 us more.)
// total[0]: the mean over the rows with a target (0 where there is none) or the sum, total[1]: how many
template <int LANES>
__global__ void __launch_bounds__(256)
avion_loss_join_kernel(LossArgs a, const float2* __restrict__ parts, const float* __restrict__ hit, int slabs, float* __restrict__ loss,
                       float* __restrict__ lse, double2* __restrict__ sums, unsigned* __restrict__ ticket, bool mean, float* __restrict__ total)
{
    const int lane = threadIdx.x % LANES, m = blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    __shared__ double2 meet[256 / LANES];
    double2 mine{0., 0.};
    if (m < a.T) {
        float top = kLossNone, total = 0.f;
        #pragma unroll 4
        for (int s = lane; s < slabs; s += LANES) {
            const float2 p = parts[(long)s * a.T + m];
            const float mn = fmaxf(top, p.x);
            total = total * fast_exp2(top - mn) + p.y * fast_exp2(p.x - mn);
            top = mn;
        }
#pragma unroll
        for (int x = 1; x < LANES; x *= 2) {
            const float o = __shfl_xor(top, x), ot = __shfl_xor(total, x), mn = fmaxf(top, o);
            total = total * fast_exp2(top - mn) + ot * fast_exp2(o - mn);
            top = mn;
        }
        const float all = (top + __builtin_amdgcn_logf(total)) * kLn2;
        const bool has = loss_target(a, m) >= 0;
        const float of = has ? all - hit[m] : 0.f;
        if (lane == 0) {
            lse[m] = all;
            if (loss) loss[m] = of;
        }
        mine = double2{of, has ? 1. : 0.};
    }
    if (!total) return;
    __shared__ bool last;
    if (lane == 0) meet[threadIdx.x / LANES] = mine;
    __syncthreads();
    if (threadIdx.x == 0) {
        double2 t{0., 0.};
        for (int i = 0; i < 256 / LANES; ++i) {
            t.x += meet[i].x;
            t.y += meet[i].y;
        }
        // written through to where every XCD sees it, and there before the ticket; a fence would write the whole L2 back
        __hip_atomic_store(&sums[blockIdx.x].x, t.x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(&sums[blockIdx.x].y, t.y, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        last = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __shared__ double2 all[256];
    double2 t{0., 0.};
    for (int i = threadIdx.x; i < (int)gridDim.x; i += 256) {
        t.x += __hip_atomic_load(&sums[i].x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        t.y += __hip_atomic_load(&sums[i].y, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    all[threadIdx.x] = t;
    __syncthreads();
    for (int half = 128; half > 0; half /= 2) {
        if ((int)threadIdx.x < half) {
            all[threadIdx.x].x += all[threadIdx.x + half].x;
            all[threadIdx.x].y += all[threadIdx.x + half].y;
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) {
        total[0] = (float)(mean ? all[0].y > 0. ? all[0].x / all[0].y : 0. : all[0].x);
        total[1] = (float)all[0].y;
    }
}
// of no rows at all
__global__ void avion_loss_none_kernel(float* __restrict__ total) { total[threadIdx.x] = 0.f; }

// ------------------------------------------------------------------------------------------ backward
// dz is held as (softmax - onehot) r_m S with r_m = dloss_m / max |dloss|, S = 1 for bf16 and 2^14 for fp16 (a softmax over many
// columns has values below fp16's normal numbers; |dz| stays below 2^14), and the products are scaled back in fp32 by
// factors[0] = scale max|dloss| / S; factors[1] = max|dloss|.
template <typename E>
constexpr float kLossHeld = std::is_same<E, F16>::value ? 16384.f : 1.f;

// max |dloss| over the rows with a target (NaN if one of them is no finite number), where each row has its own
__global__ void __launch_bounds__(1024)
avion_loss_largest_kernel(LossArgs a, const float* __restrict__ dloss, float* __restrict__ factors)
{
    __shared__ float meet[16];
    float top = 0.f;
    bool nan = false;
    for (int m = threadIdx.x; m < a.T; m += 1024)
        if (loss_target(a, m) >= 0) {
            const float d = fabsf(dloss[m]);
            nan = nan || !(d <= 3.4028235e38f);
            top = fmaxf(top, d);
        }
    if (nan) top = __builtin_nanf("");
#pragma unroll
    for (int x = 1; x < 64; x *= 2) {
        const float o = __shfl_xor(top, x);
        top = top != top || o != o ? __builtin_nanf("") : fmaxf(top, o);
    }
    if (threadIdx.x % 64 == 0) meet[threadIdx.x / 64] = top;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 16; ++i) top = top != top || meet[i] != meet[i] ? __builtin_nanf("") : fmaxf(top, meet[i]);
        factors[1] = top;
    }
}
// What the dz kernel needs of a row, three arrays of `padded` (a multiple of 256) words: its target (-1: none), its lse in base 2 (+inf
// where it has none: weights 0) and r S; and factors[0], what the products are multiplied with.
__global__ void __launch_bounds__(256)
avion_loss_rows_kernel(LossArgs a, const float* __restrict__ lse, const float* __restrict__ dloss, const float* __restrict__ total, bool each,
                       bool mean, float held, float* __restrict__ factors, int* __restrict__ rows, int padded)
{
    const int m = blockIdx.x * 256 + threadIdx.x;
    const float top = each ? factors[1] : 1.f;
    if (m == 0) {
        float d = each ? top : dloss[0];
        if (!each && mean) d = total[1] > 0.f ? d / total[1] : 0.f;
        if (!(fabsf(d) <= 3.4028235e38f)) d = __builtin_nanf("");  // (infinity would leave infinities where a sum is not zero)
        factors[0] = d * a.scale / held;
    }
    if (m >= padded) return;
    const int target = loss_target(a, m);
    rows[m] = target;
    float* f = reinterpret_cast<float*>(rows);
    f[padded + m] = target >= 0 ? lse[m] * kLog2e : INFINITY;
    f[2 * padded + m] = target >= 0 ? (each ? (top == 0.f ? 0.f : dloss[m] / top) : 1.f) * held : 0.f;
}

// dz of the vocabulary's columns v0 .. v0 + n - 1, [T, ld]; columns from n to the next multiple of 8 are zeros
// What a tile's rows need (their targets, lse and factors, 1 KB each for 256 rows) comes to LDS with its first step: loaded where it is
// used, it made every tile wait once more.  Columns of a target are rare (a wavefront's 32 x 64 logits of 50000 columns hold one in 25),
// and so are columns past the end: both have a copy of the loop.  16384 x 25088 x 768: 742 and 771 us (medians on two
// cards), matrix units 38 % of the cycles; 822 MB are written.
constexpr int kLossRowBytes = 3 * 1024;
template <int TA, int TB, int WA, int WB, typename E>
__global__ void __launch_bounds__(WA* WB * 64, 2)
avion_loss_dz_kernel(LossArgs a, const int* __restrict__ rowdata, int padded, int v0, int n, raw16* __restrict__ dz, long ld)
{
    using Cfg = LossCfg<Along::kK, Along::kK, TA, TB, WA, WB>;
    constexpr int MI = Cfg::MI, NI = Cfg::NI;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), l32 = lane % 32, g = lane / 32;
    const int wa = wave % WA, wb = wave / WA;
    const int na = (n + TA - 1) / TA, nb = (a.T + TB - 1) / TB, ntiles = na * nb, per = (ntiles + 7) / 8, together = gridDim.x / 8;
    const int first = blockIdx.x % 8 * per + blockIdx.x / 8, end = min(ntiles, (blockIdx.x % 8 + 1) * per);
    char* stage = smem + 2 * Cfg::STAGE + wave * Cfg::OUT_BYTES;
    char* rowmem = smem + Cfg::LDS_BYTES;  // of three tiles: where a tile is one step, those of two more are on their way at its end
    static_assert(Cfg::LDS_BYTES + 3 * kLossRowBytes <= 160 * 1024 && TB <= 256, "");
    const LossOperand opa{a.w + (long)v0 * a.rs_w, a.rs_w, n, 0}, opb{a.x, a.rs_x, a.T, 0};
    loss_product<Cfg, E>(
        smem, opa, opb, a.D, first < end ? (end - first + together - 1) / together : 0, wave, lane,
        [&](int t) {
            LossPlace p{0, 0, 0, (a.D + kLossStep - 1) / kLossStep};
            loss_place(first + t * together, na, nb, p.a0, p.b0);
            p.a0 *= TA;
            p.b0 *= TB;
            return p;
        },
        [&](int t, const LossPlace& p) {
            if (wave < 3)
                load_to_lds16(RawBuffer(rowdata + (long)wave * padded + p.b0, TB * 4), lds_address(rowmem) + t % 3 * kLossRowBytes + wave * 1024, lane * 16);
        },
        [&](int t, int a0, int b0, f32x16(&acc)[MI][NI]) {
            const int from = a0 + wa * NI * 32;
            const bool ragged = from + NI * 32 > n;
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                const int in = (wb * MI + i) * 32, m0 = b0 + in;
                const char* data = rowmem + t % 3 * kLossRowBytes + (in + l32) * 4;
                const int target = *reinterpret_cast<const int*>(data), at = target >= 0 ? target - v0 - from : -1;
                const float lc = *reinterpret_cast<const float*>(data + 1024), r = *reinterpret_cast<const float*>(data + 2048);
                raw16* out = dz + (long)m0 * ld + from;
                const int cols = (int)min(ld - from, (long)NI * 32);
                if (ragged || __any(at >= 0 && at < NI * 32)) {
                    loss_store<NI, E>(stage, out, ld, a.T - m0, cols, lane, [&](int j, int e) {
                        const int col = 32 * j + 8 * (e / 4) + 4 * g + e % 4;
                        const float p = fast_exp2(fmaf(acc[i][j][e], a.cs, -lc)) - (col == at ? 1.f : 0.f);
                        return target >= 0 && from + col < n ? p * r : 0.f;
                    });
                } else {
                    loss_store<NI, E>(stage, out, ld, a.T - m0, cols, lane, [&](int j, int e) {
                        const float p = fast_exp2(fmaf(acc[i][j][e], a.cs, -lc)) * r;
                        return target >= 0 ? p : 0.f;
                    });
                }
            }
        });
}

// dx (+)= dz w and dw = dz^T x, one launch for both, so that the rounds of their tiles fill each other up (16384 x 25000 x 768: 192 tiles
// of 392 steps and 294 of 256 on 256 compute units).  C [b, a], its first `rows` b; each tile is cut into `splits` ranges of K.  One
// range and one piece of the vocabulary: the result, times factors[0], goes to `out`; else to planes of fp32, one a range (added to
// what earlier pieces left), of which avion_loss_sum_kernel makes it.  A plane holds whole tiles in the accumulators' order (tile,
// wavefront, 32 x 32 block, quarter, lane: 4 numbers), so that a wavefront reads and writes 1 KB at a time.
// 16384 x 25088 x 768: 1181 and 1202 us for both (medians on two cards) = 1.05 to 1.07 PFLOP/s, matrix units 50 % of the cycles (the library's
// two products 1495).
struct LossGrad {
    LossOperand a, b;
    int rows, K, splits;
    float* sum;
    int add;
    raw16* out;
};
template <typename Cfg, typename E>
DEVINL void loss_grad(char* smem, const LossGrad& p, float mul, int first, int step, int wave, int lane)
{
    constexpr int MI = Cfg::MI, NI = Cfg::NI;
    const int wa = wave % Cfg::WA, wb = wave / Cfg::WA, cols = p.a.extent;
    const int na = (cols + Cfg::TA - 1) / Cfg::TA, nb = (p.rows + Cfg::TB - 1) / Cfg::TB, items = na * nb * p.splits;
    const int steps = (p.K + kLossStep - 1) / kLossStep;
    char* stage = smem + 2 * Cfg::STAGE + wave * Cfg::OUT_BYTES;
    loss_product<Cfg, E>(
        smem, p.a, p.b, p.K, first < items ? (items - first + step - 1) / step : 0, wave, lane,
        [&](int n) {
            const int item = first + n * step, split = item / (na * nb);
            LossPlace at{0, 0, (int)((long)steps * split / p.splits), (int)((long)steps * (split + 1) / p.splits)};
            loss_place(item - split * na * nb, na, nb, at.a0, at.b0);
            at.a0 *= Cfg::TA;
            at.b0 *= Cfg::TB;
            return at;
        },
        [](int, const LossPlace&) {},
        [&](int n, int a0, int b0, f32x16(&acc)[MI][NI]) {
            const int from = a0 + wa * NI * 32;
            f32x4* plane = reinterpret_cast<f32x4*>(p.sum) + ((long)(first + n * step) * Cfg::WAVES + wave) * (MI * NI * 256) + lane;
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                const int m0 = b0 + (wb * MI + i) * 32;
                if (!p.out) {
#pragma unroll
                    for (int j = 0; j < NI; ++j)
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            f32x4* at = plane + ((i * NI + j) * 4 + c) * 64;
                            f32x4 v = {acc[i][j][4 * c], acc[i][j][4 * c + 1], acc[i][j][4 * c + 2], acc[i][j][4 * c + 3]};
                            if (p.add) v += *at;
                            *at = v;
                        }
                } else {
                    loss_store<NI, E>(stage, p.out + (long)m0 * cols + from, cols, p.rows - m0, min(cols - from, NI * 32), lane,
                                      [&](int j, int e) { return acc[i][j][e] * mul; });
                }
            }
        });
}
template <int TA, int TB, int WA, int WB, typename E>
__global__ void __launch_bounds__(WA* WB * 64, 2)
avion_loss_grad_kernel(LossGrad dx, LossGrad dw, const float* __restrict__ factors, int items_x)
{
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), groups = gridDim.x;
    // an XCD's workgroups (they go round) take neighbouring tiles
    const int id = groups % 8 == 0 ? (int)(blockIdx.x % 8) * (groups / 8) + blockIdx.x / 8 : blockIdx.x;
    const float mul = factors[0];
    loss_grad<LossCfg<Along::kIndex, Along::kK, TA, TB, WA, WB>, E>(smem, dx, mul, id < items_x ? id : items_x, groups, wave, lane);
    // dw's tiles follow dx's in the same round
    const int taken = items_x % groups, start = id >= taken ? id - taken : id - taken + groups;
    loss_grad<LossCfg<Along::kIndex, Along::kIndex, TA, TB, WA, WB>, E>(smem, dw, mul, start, groups, wave, lane);
}

// The planes' sum, in their order, times factors[0]: a wavefront a 32 x 32 block, of either product
struct LossPlanes {
    const float* sum;
    int planes, rows;
    raw16* out;
};
template <int TA, int TB, int WA, int WB, typename E>
__global__ void __launch_bounds__(256)
avion_loss_sum_kernel(LossPlanes x, LossPlanes w, int cols, const float* __restrict__ factors)
{
    using Cfg = LossCfg<Along::kK, Along::kK, TA, TB, WA, WB>;
    constexpr int MI = Cfg::MI, NI = Cfg::NI, BLOCKS = Cfg::WAVES * MI * NI;
    const int lane = threadIdx.x % 64, na = (cols + TA - 1) / TA;
    long unit = blockIdx.x * 4L + threadIdx.x / 64;
    const long of_x = (long)na * ((x.rows + TB - 1) / TB) * BLOCKS;
    const bool second = unit >= of_x;
    const LossPlanes& p = second ? w : x;
    if (second) unit -= of_x;
    const int nb = (p.rows + TB - 1) / TB;
    const long units = (long)na * nb * BLOCKS;
    if (unit >= units) return;
    const int tile = (int)(unit / BLOCKS), in = (int)(unit - (long)tile * BLOCKS), wave = in / (MI * NI), i = in / NI % MI, j = in % NI;
    int a0, b0;
    loss_place(tile, na, nb, a0, b0);
    const int row = b0 * TB + (wave / WA * MI + i) * 32 + lane % 32, col = a0 * TA + (wave % WA * NI + j) * 32 + 4 * (lane / 32);
    const f32x4* at = reinterpret_cast<const f32x4*>(p.sum) + unit * 256 + lane;
    f32x4 t[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) t[c] = at[c * 64];
    for (int k = 1; k < p.planes; ++k) {
        at += units * 256;
#pragma unroll
        for (int c = 0; c < 4; ++c) t[c] += at[c * 64];
    }
    const float mul = factors[0];
    if (row >= p.rows) return;
#pragma unroll
    for (int c = 0; c < 4; ++c)
        if (col + 8 * c < cols)
            *reinterpret_cast<u32x2*>(p.out + (long)row * cols + col + 8 * c) =
                u32x2{E::pack(t[c][0] * mul, t[c][1] * mul), E::pack(t[c][2] * mul, t[c][3] * mul)};
}
