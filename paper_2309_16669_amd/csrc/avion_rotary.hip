// C ABI of the rotary positions.  See include/avion_attn.h for the contract.
#include "avion_attn.h"

#include <hip/hip_runtime.h>

#include <algorithm>

#include "avion_host.h"
#include "avion_rotary.h"

namespace {

template <typename E, RotaryPositions KIND, bool INTERLEAVED>
int launch_rotary(RotaryArgs a, hipStream_t st)
{
    a.tokens = (int)std::max<long>(1, std::min<long>(8, a.T / 2048));
    const long grid = (a.T + a.tokens - 1) / a.tokens;
    begin_launch();
    hipLaunchKernelGGL((avion_rotary_kernel<E, KIND, INTERLEAVED>), dim3((unsigned)grid), dim3(kRotaryThreads),
                       (size_t)a.tokens * a.pairs * 8, st, a);
    return end_launch("launch avion_rotary_kernel");
}

}  // namespace

extern "C" {

int avion_rotary(const void* q, const void* k, const void* positions, const float* freqs, void* yq, void* yk, long long T, long long P,
                 int Hq, int Hk, int d, int pairs, const int* sections, int axes, long long rs_q, long long rs_k, unsigned flags,
                 void* stream)
{
    const unsigned known = AVION_FLAG_F16 | AVION_FLAG_TOKENS_I32 | AVION_FLAG_POSITIONS_F32 | AVION_FLAG_INTERLEAVED | AVION_FLAG_INVERSE;
    if (T < 0 || P < 1 || Hq < 1 || Hk < 0 || d < 1 || pairs < 1 || axes < 1 || !sections || (flags & ~known)) return AVION_EINVAL;
    if ((flags & AVION_FLAG_TOKENS_I32) && (flags & AVION_FLAG_POSITIONS_F32)) return AVION_EINVAL;
    if (T % P != 0 || 2LL * pairs > d || rs_q < (long long)Hq * d || (Hk > 0 && rs_k < (long long)Hk * d)) return AVION_EINVAL;
    if (axes > kRotaryAxes || d % 8 != 0 || pairs % 8 != 0 || pairs > kRotaryMostPairs || d > 4096) return AVION_EUNSUPPORTED;
    RotaryArgs a{};
    long long sum = 0;
    for (int i = 0; i < axes; ++i) {
        if (sections[i] < 0) return AVION_EINVAL;
        sum += sections[i];
        for (int j = i; j < kRotaryAxes; ++j) a.ends[j] = (int)std::min<long long>(sum, 1 << 20);
    }
    if (sum != pairs) return AVION_EINVAL;
    if (T > (1LL << 27) - 8 || Hq > (1 << 16) || Hk > (1 << 16) || rs_q > (1LL << 31) || rs_k > (1LL << 31)) return AVION_EUNSUPPORTED;
    if (rs_q % 8 != 0 || (Hk > 0 && rs_k % 8 != 0)) return AVION_EUNSUPPORTED;
    if (T == 0) return AVION_OK;
    if (!q || !positions || !freqs || !yq || (Hk > 0 && (!k || !yk))) return AVION_EINVAL;
    const uintptr_t width = flags & (AVION_FLAG_TOKENS_I32 | AVION_FLAG_POSITIONS_F32) ? 4 : 8;
    if (!aligned16(q) || !aligned16(yq) || reinterpret_cast<uintptr_t>(positions) % width != 0 || reinterpret_cast<uintptr_t>(freqs) % 4 != 0)
        return AVION_EUNSUPPORTED;
    if (Hk > 0 && (!aligned16(k) || !aligned16(yk))) return AVION_EUNSUPPORTED;
    // an output on its own input is turned where it lies; its rows are then as far apart as the output's
    if ((q == yq && rs_q != (long long)Hq * d) || (Hk > 0 && k == yk && rs_k != (long long)Hk * d)) return AVION_EINVAL;
    a.side[0] = {static_cast<const raw16*>(q), static_cast<raw16*>(yq), (long)rs_q, Hq};
    a.side[1] = {static_cast<const raw16*>(k), static_cast<raw16*>(yk), (long)rs_k, Hk};
    a.positions = positions;
    a.freqs = freqs;
    a.T = T;
    a.P = P;
    a.d = d;
    a.pairs = pairs;
    a.sign = flags & AVION_FLAG_INVERSE ? -1.f : 1.f;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return by_element(flags, [&](auto fmt) {
        using E = typename decltype(fmt)::type;
        const auto by_pairs = [&](auto kind) {
            constexpr RotaryPositions KIND = decltype(kind)::value;
            return flags & AVION_FLAG_INTERLEAVED ? launch_rotary<E, KIND, true>(a, st) : launch_rotary<E, KIND, false>(a, st);
        };
        if (flags & AVION_FLAG_TOKENS_I32) return by_pairs(std::integral_constant<RotaryPositions, RotaryPositions::kI32>{});
        if (flags & AVION_FLAG_POSITIONS_F32) return by_pairs(std::integral_constant<RotaryPositions, RotaryPositions::kF32>{});
        return by_pairs(std::integral_constant<RotaryPositions, RotaryPositions::kI64>{});
    });
}

}  // extern "C"
