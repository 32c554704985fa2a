// Root-mean-square normalisation together with the residual's addition in front of it, forward and backward, its form with
// an 8-bit output, and the same rounding to 8 bits for a tensor as it is.  Per token row, x, r in R^D, gains w:
//     h = x + r (rounded to the format of r: the norm is of what the residual stream holds; h = x without r)
//     rstd = 1 / sqrt(mean(h^2) + eps),  y = h rstd w
//     8 bits: s = max(max|y|, 2^-96) / 448,  q = e4m3(y / s): each row fills the format's range (largest value 448)
//     backward, with xhat = h rstd, g = dy w and dh the gradient that reaches h by its other use:
//     dw = sum_rows dy xhat,   dx = dr = rstd (g - xhat mean(g xhat)) + dh
// What the backward needs from the forward is h itself, which the stream keeps anyway, and one fp32 per row.
//
// Bound by memory bandwidth: forward two reads and two writes per element, backward three reads and one write (two with a
// stream in 32 bits).  LANES lanes own a row at a time (16 or 32 neighbours, a wavefront, or 4 or 8 wavefronts), lane j of
// them the 16-byte chunks j, j + LANES, ...: all of the row is in registers, so it is read once, and the next row is requested
// before the current one is worked on.  The grid is two workgroups a compute unit, more streams only meet in the memory (forward
// + backward of 50176 x 768 58 + 55 us, with 1024 workgroups 60 + 58; 157696 x 512 117 + 119, 125 + 130).  Sums and
// statistics are fp32, outputs are rounded once (nearest even).  max|y| is rstd max|h w|, so that the row's sum and its maximum
// travel through one exchange.  The gains' gradient is summed over each wavefront's rows in registers, over the workgroup's
// through LDS and over the workgroups by avion_ln_param_reduce_kernel in a fixed order: no atomics, bit-reproducible.
#pragma once
#include "avion_common.h"
#include "avion_ln.h"

constexpr int kRmsWaves = 4;            // wavefronts of a workgroup (as many as a row's, where a row has more)
constexpr int kRmsMaxGrid = 512;        // workgroups of a launch; also the number of partial sums of the gains' gradient
constexpr int kQuantizeMaxGrid = 1024;  // of avion_quantize_rows_kernel, for narrow rows
constexpr int kRmsMaxD = 16384;         // 8 wavefronts x 4 chunks x 64 lanes x 8
constexpr float kF8Max = 448.0f;        // largest finite e4m3 value
constexpr float kF8Least = 1.2621774483536189e-29f;  // 2^-96: a row's largest magnitude counts as at least this

// Sum and maximum over a wavefront by lane moves of the vector unit alone (a chain of LDS permutes takes about 600 cycles a
// row): pairs, quads, mirrored eights and sixteens, then the rows of sixteen and the halves exchanged.
template <int CTRL>
DEVINL float lane_move(float x)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
DEVINL void sixteens(float x, float& a, float& b)  // as `halves`, for the two rows of sixteen of each half
{
    const unsigned u = __builtin_bit_cast(unsigned, x);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    unsigned r0 = r[0], r1 = r[1];
    asm volatile("" : "+v"(r0), "+v"(r1));
    a = __builtin_bit_cast(float, r0);
    b = __builtin_bit_cast(float, r1);
}
// of LANES = 16, 32 or 64 neighbours
template <int LANES>
DEVINL float lanes_sum(float x)
{
    x += lane_move<0xB1>(x);   // lanes 1 0 3 2
    x += lane_move<0x4E>(x);   // 2 3 0 1
    x += lane_move<0x141>(x);  // 7 - l of each eight
    x += lane_move<0x140>(x);  // 15 - l of each sixteen
    if (LANES > 16) {
        float a, b;
        sixteens(x, a, b);
        x = a + b;
    }
    return LANES > 32 ? both_halves_sum(x) : x;
}
template <int LANES>
DEVINL float lanes_max(float x)
{
    x = fmaxf(x, lane_move<0xB1>(x));
    x = fmaxf(x, lane_move<0x4E>(x));
    x = fmaxf(x, lane_move<0x141>(x));
    x = fmaxf(x, lane_move<0x140>(x));
    if (LANES > 16) {
        float a, b;
        sixteens(x, a, b);
        x = fmaxf(a, b);
    }
    return LANES > 32 ? both_halves_max(x) : x;
}

// 1 / sqrt(x), also of x below 2^-126, which the unit takes for zero
DEVINL float rsqrt_of(float x)
{
    const bool least = x < 0x1p-126f;
    const float r = __builtin_amdgcn_rsqf(least ? x * 0x1p64f : x);
    return least ? r * 0x1p32f : r;
}

// 8 fp32 -> 8 e4m3 (nearest even).  |v| < 464 or NaN.
DEVINL u32x2 pack_fp8(const float (&v)[8])
{
    u32x2 w;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int p = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i], v[4 * i + 1], 0, false);
        p = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2], v[4 * i + 3], p, true);
        w[i] = (unsigned)p;
    }
    return w;
}

// 448 / (big + rest), rest < half a step of big, as the sum of two fp32: what a row's values are scaled by, without a rounding
// that shows before the last one, to 8 bits.
struct F8Factor {
    float hi, lo;
    DEVINL explicit F8Factor(float big, float rest = 0.f)
    {
        hi = kF8Max / big;
        const float l = fmaf(-hi, rest, fmaf(-hi, big, kF8Max)) / big;
        lo = fabsf(l) < hi ? l : 0.f;  // (not finite: left out)
    }
    DEVINL float times(float v) const { return fmaf(v, hi, v * lo); }
    // (a * b) times this, in fp32 rounded to odd: towards zero, the last bit set where something (to 2^-40) is left.  What is rounded
    // once more from there, to the 8-bit values of whatever size, goes to the side that the exact value would.
    DEVINL float times(float a, float b) const
    {
        const float t = a * b, e = fmaf(a, b, -t), c = fmaf(t, lo, e * hi), q = fmaf(t, hi, c), rest = fmaf(t, hi, -q) + c;
        const int below = (rest < 0.f) != (q < 0.f) ? 1 : 0, odd = (__builtin_bit_cast(int, q) - below) | 1;
        return fabsf(rest) > fabsf(q) * 0x1p-40f ? __builtin_bit_cast(float, odd) : q;
    }
};

// Products of these values are formed anew behind this (kept from before, they take a wide row's kernel from 202 to 220 registers).
template <int NCH>
DEVINL void apart(float (&v)[NCH][8])
{
#pragma unroll
    for (int j = 0; j < NCH; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e) asm volatile("" : "+v"(v[j][e]));
}

// A lane's share of a row: NCH chunks of 8 elements, 16-bit (E) or fp32
// LAST: nobody reads it again (all inputs of the backward).  Read past the caches, backward of 157696 x 512 142 -> 112 us; the
// forward, whose inputs are as dead, takes 101 or 121 then instead of 107, by turns, and reads them as usual.
template <bool LAST, typename V>
DEVINL V rms_load(const V* p)
{
    return LAST ? __builtin_nontemporal_load(p) : *p;
}
template <int NCH, int LANES, typename E>
struct RmsRow {
    u32x4 c[NCH];
    template <bool LAST = false>
    DEVINL void load(const void* base, long row, int D, int nchunks, int at)
    {
        const u32x4 zero = {0u, 0u, 0u, 0u};
        const raw16* p = static_cast<const raw16*>(base) + row * D;
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            const int ch = at + LANES * j;
            c[j] = ch < nchunks ? rms_load<LAST>(reinterpret_cast<const u32x4*>(p + ch * 8)) : zero;
        }
    }
    DEVINL float get(int j, int e) const { return E::widen(as_frag8(c[j]), e); }
    DEVINL static void store(void* base, long row, int D, int ch, const float (&v)[8])
    {
        u32x4 w;
#pragma unroll
        for (int p = 0; p < 4; ++p) w[p] = E::pack(v[2 * p], v[2 * p + 1]);
        *reinterpret_cast<u32x4*>(static_cast<raw16*>(base) + row * D + ch * 8) = w;
    }
    // v as the format holds it
    DEVINL static void round(float (&v)[8])
    {
        u32x4 w;
#pragma unroll
        for (int p = 0; p < 4; ++p) w[p] = E::pack(v[2 * p], v[2 * p + 1]);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = E::widen(as_frag8(w), e);
    }
};
template <int NCH, int LANES>
struct RmsRow<NCH, LANES, float> {
    f32x4 c[NCH][2];
    template <bool LAST = false>
    DEVINL void load(const void* base, long row, int D, int nchunks, int at)
    {
        const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
        const float* p = static_cast<const float*>(base) + row * D;
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            const int ch = at + LANES * j;
            c[j][0] = ch < nchunks ? rms_load<LAST>(reinterpret_cast<const f32x4*>(p + ch * 8)) : zero;
            c[j][1] = ch < nchunks ? rms_load<LAST>(reinterpret_cast<const f32x4*>(p + ch * 8 + 4)) : zero;
        }
    }
    DEVINL float get(int j, int e) const { return c[j][e / 4][e % 4]; }
    DEVINL static void store(void* base, long row, int D, int ch, const float (&v)[8])
    {
        store8(static_cast<float*>(base) + row * D + ch * 8, v);
    }
    DEVINL static void round(float (&)[8]) {}
};

// How a row lies over lanes: 16 or 32 neighbours (several rows a wavefront), a wavefront, or 4 or 8 wavefronts of a workgroup.
template <int LANES>
struct RmsWork {
    static constexpr int WPR = LANES / 64 > 1 ? LANES / 64 : 1;              // wavefronts a row
    static constexpr int SUB = LANES < 64 ? 64 / LANES : 1;                  // rows a wavefront
    static constexpr int WAVES = WPR > kRmsWaves ? WPR : kRmsWaves;
    static constexpr int ROWS = LANES <= 64 ? kRmsWaves * SUB : 1;           // rows of a workgroup at a time
    int lane, wave, at, sub;
    DEVINL RmsWork()
        : lane(threadIdx.x % 64), wave(threadIdx.x / 64), at(LANES <= 64 ? lane % LANES : (int)threadIdx.x),
          sub(LANES < 64 ? lane / LANES : 0) {}
    // the first of this wavefront's rows (the same in all its lanes); a lane's own is `sub` behind
    DEVINL long first() const { return (long)blockIdx.x * ROWS + (LANES <= 64 ? wave * SUB : 0); }
    DEVINL long stride() const { return (long)gridDim.x * ROWS; }
};

// Sum of a (and maximum of b) over the lanes of a row.  Through LDS where it has more than one wavefront; two places, used in
// turn by consecutive rows: a wavefront writes the other one only after the barrier that everybody's reads of the one before
// precede.
template <int LANES, bool MAX>
DEVINL void row_reduce(float& a, float& b, float (&sh)[2][RmsWork<LANES>::WPR][2], int wave, int lane, int& turn)
{
    constexpr int WPR = RmsWork<LANES>::WPR, IN = LANES < 64 ? LANES : 64;
    a = lanes_sum<IN>(a);
    if (MAX) b = lanes_max<IN>(b);
    if constexpr (WPR > 1) {
        if (lane == 0) {
            sh[turn][wave][0] = a;
            if (MAX) sh[turn][wave][1] = b;
        }
        __syncthreads();
        a = sh[turn][0][0];
        if (MAX) b = sh[turn][0][1];
#pragma unroll
        for (int w = 1; w < WPR; ++w) {
            a += sh[turn][w][0];
            if (MAX) b = fmaxf(b, sh[turn][w][1]);
        }
        turn ^= 1;
    }
}

// y (E), or y8 and scale with F8; h where there is a residual; rstd where it is asked for
// (two wavefronts a SIMD at least: 8 bits and an fp32 stream would take 262 registers at 4 chunks a lane)
template <int LANES, int NCH, typename E, typename R, bool F8>
__global__ void __launch_bounds__(RmsWork<LANES>::WAVES * 64, 2)
avion_rmsnorm_fwd_kernel(const raw16* __restrict__ x, const void* __restrict__ residual, const float* __restrict__ weight,
                         void* __restrict__ y, float* __restrict__ scale, void* __restrict__ h, float* __restrict__ rstd,
                         long M, int D, float eps)
{
    const RmsWork<LANES> rw;
    __shared__ float sh[2][RmsWork<LANES>::WPR][2];
    const int lane = rw.lane, wave = rw.wave, at = rw.at;
    const int nchunks = D / 8;
    const float inv_d = 1.0f / (float)D;
    const long stride = rw.stride();
    long row = rw.first();
    if (row >= M) return;
    float gain[NCH][8];
    int turn = 0;

    RmsRow<NCH, LANES, E> xa, xb;
    RmsRow<NCH, LANES, R> ra, rb;
    auto load = [&](RmsRow<NCH, LANES, E>& xr, RmsRow<NCH, LANES, R>& rr, long n) {
        n += rw.sub;
        const int chunks = n < M ? nchunks : 0;
        xr.load(x, n, D, chunks, at);
        if (residual) rr.load(residual, n, D, chunks, at);
    };
    load(xa, ra, row);
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
        const int ch = at + LANES * j;
#pragma unroll
        for (int e = 0; e < 8; ++e) gain[j][e] = 0.f;
        if (ch < nchunks) load8(weight + ch * 8, gain[j]);
    }

    auto finish = [&](const RmsRow<NCH, LANES, E>& xr, const RmsRow<NCH, LANES, R>& rr, long n) {
        n += rw.sub;
        const int chunks = n < M ? nchunks : 0;
        float v[NCH][8], ss = 0.f, big = 0.f;
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[j][e] = xr.get(j, e);
            if (residual) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[j][e] += rr.get(j, e);
                RmsRow<NCH, LANES, R>::round(v[j]);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                ss = fmaf(v[j][e], v[j][e], ss);  // chunks past the row are zeros
                if (F8) big = fmaxf(big, fabsf(v[j][e] * gain[j][e]));
            }
        }
        row_reduce<LANES, F8>(ss, big, sh, wave, lane, turn);
        const float rs = rsqrt_of(fmaf(ss, inv_d, eps));
        // 8 bits: y / scale = h w 448 / max|h w|, in which rstd has gone; it stays where the least scale holds, where max|h w|
        // is too small to divide by (with an eps below 1e-14), and where that maximum or something else is not finite (gains of
        // 1e30 on a stream of 1e10): max|y| is then taken of the products with rstd
        float big_y = big * rs;
        u32x2 in8[NCH];
        if constexpr (F8) {
            const bool gone = big >= 0x1p-90f && big < __builtin_inff() && big_y >= kF8Least;
            // five roundings at most lie between these and the exact quotients: where both ends of eight round alike, so do those
            const float by = kF8Max / big, by_more = by * (1.f + 0x1p-21f), by_less = by * (1.f - 0x1p-21f);
            bool again = !gone;
            apart(v);
#pragma unroll
            for (int j = 0; j < NCH; ++j) {
                float more[8], less[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float p = v[j][e] * gain[j][e];
                    more[e] = p * by_more;
                    less[e] = p * by_less;
                }
                in8[j] = pack_fp8(more);
                const u32x2 other = pack_fp8(less);
                again |= in8[j][0] != other[0] || in8[j][1] != other[1];
            }
            // A row with a value whose ends part (one row of 120 of 768 columns), or one that keeps rstd: once more, exactly.
            // (Against quotients rounded to fp32 before, some twenty of 50176 x 768 of which lie on the wrong side of a middle:
            // 54.1 us and 53 there, 4096 x 1024 9.2 and 8.6, 3000 x 8192, whose wavefronts have to agree, 39.6 and 36.  Finding the
            // rows by the bits of one quotient took 54.5, 9.4 and 39.6, spilled at 4 chunks a lane, and knew no middles below 2^-6.)
            if (LANES > 64 ? __syncthreads_or(again) : __any(again)) {
                // of the largest product: what its rounding took; or the largest product with rstd
                const float up = gone ? 1.f : rs;
                float none = 0.f, rest = gone ? -big : 0.f;
                apart(v);
#pragma unroll
                for (int j = 0; j < NCH; ++j)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float a = fabsf(v[j][e] * up), b = fabsf(gain[j][e]);
                        if (!gone || a * b == big) rest = fmaxf(rest, gone ? fmaf(a, b, -big) : a * b);
                    }
                row_reduce<LANES, true>(none, rest, sh, wave, lane, turn);
                if (!gone) big_y = rest;
                const F8Factor to8(gone ? big : fmaxf(big_y, kF8Least), gone ? rest : 0.f);
#pragma unroll
                for (int j = 0; j < NCH; ++j) {
                    float o[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[e] = to8.times(v[j][e] * up, gain[j][e]);
                    in8[j] = pack_fp8(o);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            const int ch = at + LANES * j;
            if (ch < chunks) {
                if (residual) RmsRow<NCH, LANES, R>::store(h, n, D, ch, v[j]);
                if constexpr (F8) {
                    *reinterpret_cast<u32x2*>(static_cast<char*>(y) + n * D + ch * 8) = in8[j];
                } else {
                    float o[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[e] = v[j][e] * rs * gain[j][e];
                    RmsRow<NCH, LANES, E>::store(y, n, D, ch, o);
                }
            }
        }
        if (at == 0 && n < M) {
            if (F8) scale[n] = fmaxf(big_y, kF8Least) * (1.0f / kF8Max);
            if (rstd) rstd[n] = rs;
        }
    };

    // two rows in registers: the next one is in flight while the current one is worked on
    while (true) {
        const long n1 = row + stride;
        if (n1 < M) load(xb, rb, n1);
        finish(xa, ra, row);
        if (n1 >= M) break;
        const long n2 = n1 + stride;
        if (n2 < M) load(xa, ra, n2);
        finish(xb, rb, n1);
        if (n2 >= M) break;
        row = n2;
    }
}

// Rows of x as they are, in 8 bits.  One read and half a write an element: with two workgroups a compute unit, narrow rows keep too
// little in flight; up to 1024 columns (two chunks a lane) that shows where x is read from memory.  512 and 1024 workgroups:
// 157696 x 512 59 and 48 us, 12544 x 512 6.8 and 6.5, 50176 x 768 26 and 23, 25088 x 1024 14.9 and 13.8, but 12544 x 1024 8.8 and
// 9.2, 8192 x 1024 6.9 and 7.2, 50176 x 1280 38.1 and 38.6.
template <int LANES, int NCH, typename E>
__global__ void __launch_bounds__(RmsWork<LANES>::WAVES * 64)
avion_quantize_rows_kernel(const raw16* __restrict__ x, void* __restrict__ y, float* __restrict__ scale, long M, int D)
{
    const RmsWork<LANES> rw;
    __shared__ float sh[2][RmsWork<LANES>::WPR][2];
    const int lane = rw.lane, wave = rw.wave, at = rw.at;
    const int nchunks = D / 8;
    const long stride = rw.stride();
    long row = rw.first();
    if (row >= M) return;
    int turn = 0;
    auto load = [&](RmsRow<NCH, LANES, E>& xr, long n) { xr.load(x, n + rw.sub, D, n + rw.sub < M ? nchunks : 0, at); };
    auto finish = [&](const RmsRow<NCH, LANES, E>& xr, long n) {
        n += rw.sub;
        const int chunks = n < M ? nchunks : 0;
        float none = 0.f, big = 0.f;
#pragma unroll
        for (int j = 0; j < NCH; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) big = fmaxf(big, fabsf(xr.get(j, e)));
        row_reduce<LANES, true>(none, big, sh, wave, lane, turn);
        big = fmaxf(big, kF8Least);
        const F8Factor to8(big);
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            const int ch = at + LANES * j;
            if (ch < chunks) {
                float o[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = to8.times(xr.get(j, e));
                *reinterpret_cast<u32x2*>(static_cast<char*>(y) + n * D + ch * 8) = pack_fp8(o);
            }
        }
        if (at == 0 && n < M) scale[n] = big * (1.0f / kF8Max);
    };
    RmsRow<NCH, LANES, E> a, b;
    load(a, row);
    while (true) {
        const long n1 = row + stride;
        if (n1 < M) load(b, n1);
        finish(a, row);
        if (n1 >= M) break;
        const long n2 = n1 + stride;
        if (n2 < M) load(a, n2);
        finish(b, n1);
        if (n2 >= M) break;
        row = n2;
    }
}

// dx (E; the gradient of both inputs where the stream has that format too), dr (fp32 stream), either may be absent, and this
// workgroup's partial sums of the gains' gradient into part[blockIdx.x][D].  dh may be absent.  FEW: few rows, in one launch:
// the workgroups behind the first row_wgs sum 64 columns of the gains' gradient each over all rows, which they read once more
// (rstd is known, so they need nothing of the others), into dweight.
constexpr int kRmsFewCols = 64, kRmsFewRows = 640;
template <int LANES, int NCH, typename E, typename R, bool FEW>
__global__ void __launch_bounds__(RmsWork<LANES>::WAVES * 64)
avion_rmsnorm_bwd_kernel(const void* __restrict__ h, const float* __restrict__ weight, const float* __restrict__ rstd,
                         const raw16* __restrict__ dy, const void* __restrict__ dh, void* __restrict__ dx,
                         float* __restrict__ dr, float* __restrict__ part, float* __restrict__ dweight, long M, int D, int row_wgs)
{
    const RmsWork<LANES> rw;
    extern __shared__ __attribute__((aligned(16))) char smem[];  // LANES <= 64: (kRmsWaves - 1) x D floats
    __shared__ float sh[2][RmsWork<LANES>::WPR][2];
    if constexpr (FEW) {
        constexpr int LPC = kRmsFewCols / 8, GROUPS = RmsWork<LANES>::WAVES * 64 / LPC, FLY = 4;
        __shared__ float sums[GROUPS][kRmsFewCols];
        if ((int)blockIdx.x >= row_wgs) {
            const int lane = threadIdx.x % LPC, group = threadIdx.x / LPC, ch = ((int)blockIdx.x - row_wgs) * LPC + lane;
            float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            for (long r0 = group; r0 < M; r0 += FLY * GROUPS) {
                RmsRow<1, 64, R> hh[FLY];
                RmsRow<1, 64, E> dd[FLY];
                float rs[FLY];
#pragma unroll
                for (int k = 0; k < FLY; ++k) {
                    const long n = r0 + k * GROUPS;
                    const int chunks = n < M ? D / 8 : 0;
                    hh[k].load(h, n, D, chunks, ch);
                    dd[k].load(dy, n, D, chunks, ch);
                    rs[k] = n < M ? rstd[n] : 0.f;
                }
#pragma unroll
                for (int k = 0; k < FLY; ++k)
#pragma unroll
                    for (int e = 0; e < 8; ++e) acc[e] = fmaf(dd[k].get(0, e), hh[k].get(0, e) * rs[k], acc[e]);
            }
            store8(&sums[group][lane * 8], acc);
            __syncthreads();
            const int col = ((int)blockIdx.x - row_wgs) * kRmsFewCols + threadIdx.x;
            if (threadIdx.x < kRmsFewCols && col < D) {
                float t = 0.f;
#pragma unroll
                for (int g = 0; g < GROUPS; ++g) t += sums[g][threadIdx.x];
                dweight[col] = t;
            }
            return;
        }
    }
    const int lane = rw.lane, wave = rw.wave, at = rw.at;
    const int nchunks = D / 8;
    const float inv_d = 1.0f / (float)D;
    const long stride = (long)row_wgs * RmsWork<LANES>::ROWS;
    long row = rw.first();
    float gain[NCH][8], dw[NCH][8];
    int turn = 0;
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
        const int ch = at + LANES * j;
#pragma unroll
        for (int e = 0; e < 8; ++e) gain[j][e] = dw[j][e] = 0.f;
        if (ch < nchunks) load8(weight + ch * 8, gain[j]);
    }

    struct Rows {
        RmsRow<NCH, LANES, R> h, dh;
        RmsRow<NCH, LANES, E> dy;
        float rs;
    };
    auto load = [&](Rows& t, long n) {
        n += rw.sub;
        const int chunks = n < M ? nchunks : 0;
        t.h.template load<!FEW>(h, n, D, chunks, at);
        t.dy.template load<!FEW>(dy, n, D, chunks, at);
        if (dh) t.dh.template load<!FEW>(dh, n, D, chunks, at);
        t.rs = n < M ? rstd[n] : 0.f;
    };
    auto finish = [&](const Rows& t, long n) {
        n += rw.sub;
        const int chunks = n < M ? nchunks : 0;
        float s = 0.f, none = 0.f;
#pragma unroll
        for (int j = 0; j < NCH; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float xh = t.h.get(j, e) * t.rs, gy = t.dy.get(j, e);
                s = fmaf(gy * gain[j][e], xh, s);  // zero in chunks past the row
                if (!FEW) dw[j][e] = fmaf(gy, xh, dw[j][e]);
            }
        row_reduce<LANES, false>(s, none, sh, wave, lane, turn);
        const float c = s * inv_d;
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            const int ch = at + LANES * j;
            if (ch < chunks) {
                float o[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    o[e] = t.rs * (t.dy.get(j, e) * gain[j][e] - t.h.get(j, e) * t.rs * c);
                    if (dh) o[e] += t.dh.get(j, e);
                }
                if (dx) RmsRow<NCH, LANES, E>::store(dx, n, D, ch, o);
                if (dr) store8(dr + n * D + ch * 8, o);
            }
        }
    };
    if (NCH > 2) {
        // (two rows in registers would leave one wavefront a SIMD)
        for (; row < M; row += stride) {
            Rows a;
            load(a, row);
            finish(a, row);
        }
    } else if (row < M) {
        Rows a, b;
        load(a, row);
        while (true) {
            const long n1 = row + stride;
            if (n1 < M) load(b, n1);
            finish(a, row);
            if (n1 >= M) break;
            const long n2 = n1 + stride;
            if (n2 < M) load(a, n2);
            finish(b, n1);
            if (n2 >= M) break;
            row = n2;
        }
    }
    if constexpr (FEW) return;
    float* out = part + (long)blockIdx.x * D;
    if constexpr (LANES <= 64) {
        // the rows that a wavefront held side by side, then the workgroup's sum in wavefront order (0 + 1 + 2 + 3)
        if (LANES < 64)
#pragma unroll
            for (int j = 0; j < NCH; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (LANES == 16) {
                        float a, b;
                        sixteens(dw[j][e], a, b);
                        dw[j][e] = a + b;
                    }
                    dw[j][e] = both_halves_sum(dw[j][e]);
                }
        float* sums = reinterpret_cast<float*>(smem);
        if (wave > 0) {
#pragma unroll
            for (int j = 0; j < NCH; ++j) {
                const int ch = at + LANES * j;
                if (ch < nchunks) store8(sums + (wave - 1) * D + ch * 8, dw[j]);
            }
        }
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int j = 0; j < NCH; ++j) {
            const int ch = at + LANES * j;
            if (ch < nchunks)
                for (int w = 0; w < kRmsWaves - 1; ++w) {
                    float a[8];
                    load8(sums + w * D + ch * 8, a);
#pragma unroll
                    for (int e = 0; e < 8; ++e) dw[j][e] += a[e];
                }
        }
    }
#pragma unroll
    for (int j = 0; j < NCH; ++j) {
        const int ch = at + LANES * j;
        if (ch < nchunks) store8(out + ch * 8, dw[j]);
    }
}
