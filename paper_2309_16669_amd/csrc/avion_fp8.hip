// C ABI of the product of rows in 8 bits.  See include/avion_attn.h for its contract.
#include "avion_attn.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "avion_fp8.h"
#include "avion_host.h"

namespace {

constexpr long long kComputeUnits = 256;

// ------------------------------------------------------------------------------- 8-bit product
template <int MT, typename E>
int launch_few(const char* x8, const float* xs, const char* w8, const float* ws, const float* bias, raw16* y, int M, int N, int K,
               hipStream_t st)
{
    begin_launch();
    hipLaunchKernelGGL((avion_linear_fp8_few_kernel<MT, E>), dim3((N + 15) / 16), dim3(kFewWaves * 64), 0, st, x8, xs, w8, ws, bias, y,
                       M, N, K);
    return end_launch("launch avion_linear_fp8_few_kernel");
}
long long fp8_tiles(int M, int N, int tm, int tn) { return (long long)((M + tm - 1) / tm) * ((N + tn - 1) / tn); }
template <int TM, int TN, int WM, int WN, int ST, int KG, typename E>
int launch_fp8(const char* x8, const float* xs, const char* w8, const float* ws, const float* bias, raw16* y, int M, int N, int K,
               hipStream_t st)
{
    using Cfg = Fp8Cfg<TM, TN, WM, WN, ST, KG>;
    static std::atomic<unsigned long long> lds_allowed{0};
    const auto kernel = avion_linear_fp8_kernel<TM, TN, WM, WN, ST, KG, E>;
    const hipError_t attr = allow_lds_here(kernel, Cfg::LDS_BYTES, lds_allowed);
    if (attr != hipSuccess) return hip_fail(attr, "hipFuncSetAttribute(linear_fp8)");
    const long long tiles = fp8_tiles(M, N, TM, TN);
    const unsigned grid = (unsigned)((tiles + 7) / 8 * 8);
    begin_launch();
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(Cfg::NT), Cfg::LDS_BYTES, st, x8, xs, w8, ws, bias, y, M, N, K, (N + TN - 1) / TN,
                       (int)tiles);
    return end_launch("launch avion_linear_fp8_kernel");
}

// Which kernel (us, kernel alone):
//   up to 16 rows, and up to 32 where each compute unit has one workgroup at most (N up to 4096): straight from memory.  K = 1024
//     and 4096, then tiles of 64 x 64: 32 x 4096 3.9, 8.7 and 4.6, 9.9; 32 x 4608 5.2, 13.8 and 4.7, 9.9; 17 x 4608 4.5, 11.2 and
//     4.6, 9.9; 16 x 4608 4.0, 10.1 and 4.5, 9.8; 8 x 8192 4.0, 9.1 and 4.9, 10.0.  (Up to 16 rows and N past 8192 either may be
//     faster: 1 x 12288 6.0, 13.0 and 5.6, 10.4; 1 x 50000 14.7, 40 and 13.4, 53.)
//   else the smallest tiles that leave no more than one for a compute unit (latency), larger ones beyond (traffic):
//     64 x 64 and 128 x 64 on 1024 x 1024 x 1024 (256 tiles): 6.0 and 6.9, on 512 x 4096 x 4096 (512): 21.8 and 17.5;
//     with eight wavefronts, half of K each, where K is long: 64 x 2304 with K = 512 3.8 and 3.8, 768 4.4 and 4.2, 1024 5.0 and 4.6,
//     4096 12.7 and 9.9, 1024 x 1024 with K = 512 4.1 and 4.2, 1024 5.7 and 5.4;
//     128 x 64 in this way, where there is one for a compute unit at most: 2048 x 1024 with K = 1280 7.7 and 8.2, 2048 9.8 and 9.9,
//     3584 14.7 and 13.9, 4096 16.2 and 14.8; 1024 x 2048 with 3584 14.7 and 14.5; 3000 x 640 x 8192 28.6 and 24.9;
//     128 x 64 and 128 x 128 on 785 x 2304 x 768 (126 tiles of 128 x 128): 6.8 and 8.7, on 1570 x 3840 x 1280 (390): 19.3 and 16.2
//     and 128 x 128 only where y has more than 64 columns: 36864 x 64 x 1024 11.4 and 12.5, 36864 x 72 x 1024 13.5 and 12.6
//   256 x 256: a round of its 256 tiles takes about as long as 820 tiles of 128 x 128 in a long row and less to begin with, so it
//     needs rounds that are well filled, at any K (these tiles, then those of 128 x 128): 12544 x 768 (147 tiles) 13.5 and 15.6 with K = 768, 43 and 53
//     with 4096; 2048 x 4096 x 4096 (128): 46 and 38; 8448 x 2048 (264, a second round that is nearly empty) 26.1 and 22.8, 93 and 82;
//     11008 x 2048 (344) 26.5 and 26.3, 94.3 and 93.7; 12800 x 1792 (350) 26.6 and 26.3, 93 and 97; 25088 x 1024 (392) 26 and 30,
//     102 and 131
//     and tiles that are more than half inside y both ways: 65536 x 128 x 1024 18.9 and 16.5, 65536 x 136 x 1024 20.8 and 22.5;
//     128 x 50000 x 768 15.8 and 12.3, 160 x 50000 x 768 16.3 and 22.1
bool fp8_wide(int M, int N)
{
    if (M <= kWideM / 2 || N <= kWideN / 2) return false;
    const long long tiles = fp8_tiles(M, N, kWideM, kWideN), rounds = (tiles + kComputeUnits - 1) / kComputeUnits;
    return 5 * (tiles + 64) >= 4 * kComputeUnits * rounds;
}
template <typename E, bool STREAM, bool AHEAD>
int launch_wide_by(const char* x8, const float* xs, const char* w8, const float* ws, const float* bias, raw16* y, int M, int N, int K,
                   hipStream_t st)
{
    static std::atomic<unsigned long long> lds_allowed{0};
    const auto kernel = avion_linear_fp8_wide_kernel<E, STREAM, AHEAD>;
    const hipError_t attr = allow_lds_here(kernel, kWideLds, lds_allowed);
    if (attr != hipSuccess) return hip_fail(attr, "hipFuncSetAttribute(linear_fp8_wide)");
    const int ntm = (M + kWideM - 1) / kWideM, ntn = (N + kWideN - 1) / kWideN;
    const unsigned grid = (unsigned)std::min<long long>(kComputeUnits, ((long long)ntm * ntn + 7) / 8 * 8);
    begin_launch();
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(kWideWaves * 64), kWideLds, st, x8, xs, w8, ws, bias, y, M, N, K, ntm, ntn);
    return end_launch("launch avion_linear_fp8_wide_kernel");
}
template <typename E, bool STREAM>
int launch_wide(const char* x8, const float* xs, const char* w8, const float* ws, const float* bias, raw16* y, int M, int N, int K,
                hipStream_t st)
{
    if (K >= kWideAhead) return launch_wide_by<E, STREAM, true>(x8, xs, w8, ws, bias, y, M, N, K, st);
    return launch_wide_by<E, STREAM, false>(x8, xs, w8, ws, bias, y, M, N, K, st);
}

}  // namespace

extern "C" {

int avion_linear_fp8(const void* x8, const float* x_scale, const void* w8, const float* w_scale, const float* bias, void* y,
                     long long M, int N, int K, unsigned flags, void* stream)
{
    if (M < 0 || N < 1 || K < 1 || (flags & ~AVION_FLAG_F16)) return AVION_EINVAL;
    if (M >= (1LL << 31) - 256 || N % 8 != 0 || N > (1 << 20) || K % 16 != 0 || K > (1 << 16)) return AVION_EUNSUPPORTED;
    if (fp8_tiles((int)M, N, 64, 64) > (1LL << 24)) return AVION_EUNSUPPORTED;  // workgroups of a launch
    if (M == 0) return AVION_OK;
    if (!x8 || !x_scale || !w8 || !w_scale || !y) return AVION_EINVAL;
    const void* ptrs[] = {x8, w8, w_scale, bias, y};
    for (const void* p : ptrs)
        if (!aligned16(p)) return AVION_EUNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(x_scale) % 4 != 0) return AVION_EUNSUPPORTED;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const char *x = static_cast<const char*>(x8), *w = static_cast<const char*>(w8);
    raw16* out = static_cast<raw16*>(y);
    const int m = (int)M;
    return by_element(flags, [&](auto fmt) {
        using E = typename decltype(fmt)::type;
        if (m <= 16) return launch_few<1, E>(x, x_scale, w, w_scale, bias, out, m, N, K, st);
        if (m <= 32 && N <= 16 * kComputeUnits) return launch_few<2, E>(x, x_scale, w, w_scale, bias, out, m, N, K, st);
        // (stores past the caches only where rows are whole cache lines: 30000 x 1544 x 768 65.9 us with them, 55.4 without,
        // 50176 x 2304 x 768 106 and 116, 50176 x 2304 x 2304 244 and 243, 12544 x 4096 x 1024 65.6 and 64.4)
        if (fp8_wide(m, N) && N % 64 == 0) return launch_wide<E, true>(x, x_scale, w, w_scale, bias, out, m, N, K, st);
        if (fp8_wide(m, N)) return launch_wide<E, false>(x, x_scale, w, w_scale, bias, out, m, N, K, st);
        if (N > 64 && fp8_tiles(m, N, 128, 128) >= kComputeUnits)
            return launch_fp8<128, 128, 2, 2, 2, 1, E>(x, x_scale, w, w_scale, bias, out, m, N, K, st);
        if (fp8_tiles(m, N, 64, 64) > kComputeUnits && fp8_tiles(m, N, 128, 64) <= kComputeUnits && K >= 4096)
            return launch_fp8<128, 64, 2, 2, 3, 2, E>(x, x_scale, w, w_scale, bias, out, m, N, K, st);
        if (fp8_tiles(m, N, 64, 64) > kComputeUnits)
            return launch_fp8<128, 64, 2, 2, 3, 1, E>(x, x_scale, w, w_scale, bias, out, m, N, K, st);
        if (K >= 1024) return launch_fp8<64, 64, 2, 2, 3, 2, E>(x, x_scale, w, w_scale, bias, out, m, N, K, st);
        return launch_fp8<64, 64, 2, 2, 3, 1, E>(x, x_scale, w, w_scale, bias, out, m, N, K, st);
    });
}

}  // extern "C"
