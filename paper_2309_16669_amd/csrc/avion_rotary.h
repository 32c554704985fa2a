// Rotary positions: each pair of channels of a head is turned by the angle that its token's position on one axis (time, height
// or width of a video's token grid, place in a text) gives it:
//     theta_j = position[axis(j)] * freq_j,   y1 = x1 cos theta_j - x2 sin theta_j,   y2 = x2 cos theta_j + x1 sin theta_j
// The backward is the same with -theta.  Memory-bound: 4 bytes a channel for 3 operations, and an angle serves all heads of a
// token.
//
// Angles: position and frequency are exact in double; their product, and its quotient by 2 pi, are held as sums of two doubles, of which
// the whole turns go before the rest is rounded to fp32.  In fp32 the position 20000 would leave 1e-3 of an angle and 10^6 0.06; one
// double would leave 2e-4 at 2^40.
//
// Split: a workgroup takes kRotaryTokens (fewer in small launches) tokens, forms their cosines and sines once in LDS, and walks over
// their heads with 16-byte accesses; a thread holds both halves of its pairs, so that an output may lie on its input.  50176 tokens of 24 heads of
// 64 channels: 62 to 63 us, 4.9 TB/s of the 5.2 that a copy reaches; one token 2.3 us.
#pragma once
#include "avion_common.h"

constexpr int kRotaryThreads = 256, kRotaryAxes = 4, kRotaryMostPairs = 512;

struct RotarySide {
    const raw16* x;  // token rows rs elements apart, heads d apart
    raw16* y;        // [T, H, d]
    long rs;
    int H;
};
struct RotaryArgs {
    RotarySide side[2];  // queries and keys (the second: H 0 where there are none)
    const void* positions;  // [axes, P]
    const float* freqs;     // [pairs]
    long T, P;
    int d, pairs, tokens;  // tokens of a workgroup
    int ends[kRotaryAxes];  // pairs of the axes up to and with each
    float sign;
};

enum class RotaryPositions { kI64, kI32, kF32 };

template <RotaryPositions KIND>
DEVINL double rotary_position(const void* p, long i)
{
    if constexpr (KIND == RotaryPositions::kI64) return (double)static_cast<const long*>(p)[i];
    if constexpr (KIND == RotaryPositions::kI32) return (double)static_cast<const int*>(p)[i];
    return (double)static_cast<const float*>(p)[i];
}

// position * freq / (2 pi), less whole turns
DEVINL float rotary_turn(double position, double freq)
{
#pragma clang fp contract(off)  // (a product drawn into the difference behind it would count its rest twice)
    constexpr double kInv2Pi = 0x1.45f306dc9c883p-3, kInv2PiRest = -0x1.6b01ec5417056p-57;
    const double angle = position * freq, angle_rest = fma(position, freq, -angle);
    const double turns = angle * kInv2Pi, rest = fma(angle, kInv2Pi, -turns) + fma(angle, kInv2PiRest, angle_rest * kInv2Pi);
    return (float)((turns - rint(turns)) + rest);
}

template <typename E, RotaryPositions KIND, bool INTERLEAVED>
__global__ void __launch_bounds__(kRotaryThreads) avion_rotary_kernel(RotaryArgs a)
{
    extern __shared__ __attribute__((aligned(16))) float turns[];  // [tokens][cos of the pairs | sin]
    const long t0 = (long)blockIdx.x * a.tokens;
    const int n = (int)min((long)a.tokens, a.T - t0), m = a.pairs;
    for (int i = threadIdx.x; i < n * m; i += kRotaryThreads) {
        const int t = i / m, j = i - t * m;
        int axis = 0;
#pragma unroll
        for (int k = 0; k < kRotaryAxes - 1; ++k) axis += j >= a.ends[k];
        const double pos = rotary_position<KIND>(a.positions, axis * a.P + (t0 + t) % a.P);
        float s, c;
        sincospif(2.f * rotary_turn(pos, (double)a.freqs[j]), &s, &c);
        turns[t * 2 * m + j] = c;
        turns[t * 2 * m + m + j] = a.sign * s;
    }
    __syncthreads();
    // items of a head: its pairs of chunks (or, neighbouring pairs, its chunks), then the chunks that do not turn
    const int turned = INTERLEAVED ? m / 4 : m / 8, items = turned + (a.d - 2 * m) / 8;
    const int H = a.side[0].H + a.side[1].H, of_token = H * items;
    for (int i = threadIdx.x; i < n * of_token; i += kRotaryThreads) {
        const int t = i / of_token, in = i - t * of_token, head = in / items, item = in - head * items;
        const bool second = head >= a.side[0].H;
        const RotarySide& s = a.side[second];
        const int h = second ? head - a.side[0].H : head;
        const raw16* x = s.x + (t0 + t) * s.rs + (long)h * a.d;
        raw16* y = s.y + ((t0 + t) * s.H + h) * (long)a.d;
        const float* c = turns + t * 2 * m;
        if (item >= turned) {
            const int at = 2 * m + (item - turned) * 8;
            *reinterpret_cast<u32x4*>(y + at) = *reinterpret_cast<const u32x4*>(x + at);
        } else if constexpr (INTERLEAVED) {
            const frag8 v = *reinterpret_cast<const frag8*>(x + item * 8);
            const f32x4 cs = *reinterpret_cast<const f32x4*>(c + item * 4), sn = *reinterpret_cast<const f32x4*>(c + m + item * 4);
            u32x4 r;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float p = E::widen(v, 2 * e), q = E::widen(v, 2 * e + 1);
                r[e] = E::pack(p * cs[e] - q * sn[e], q * cs[e] + p * sn[e]);
            }
            *reinterpret_cast<u32x4*>(y + item * 8) = r;
        } else {
            const frag8 v = *reinterpret_cast<const frag8*>(x + item * 8), w = *reinterpret_cast<const frag8*>(x + m + item * 8);
            f32x4 cs[2], sn[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                cs[k] = *reinterpret_cast<const f32x4*>(c + item * 8 + 4 * k);
                sn[k] = *reinterpret_cast<const f32x4*>(c + m + item * 8 + 4 * k);
            }
            u32x4 r1, r2;
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                float o1[2], o2[2];
#pragma unroll
                for (int f = 0; f < 2; ++f) {
                    const float p = E::widen(v, e + f), q = E::widen(w, e + f), co = cs[(e + f) / 4][(e + f) % 4], si = sn[(e + f) / 4][(e + f) % 4];
                    o1[f] = p * co - q * si;
                    o2[f] = q * co + p * si;
                }
                r1[e / 2] = E::pack(o1[0], o1[1]);
                r2[e / 2] = E::pack(o2[0], o2[1]);
            }
            *reinterpret_cast<u32x4*>(y + item * 8) = r1;
            *reinterpret_cast<u32x4*>(y + m + item * 8) = r2;
        }
    }
}
