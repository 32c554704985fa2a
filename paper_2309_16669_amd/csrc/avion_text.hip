// C ABI of the text encoder's entry: token table, RMS normalisation with the residual's addition, rows in 8 bits.  See
// include/avion_attn.h for the contract of every entry point.
#include "avion_attn.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "avion_embed.h"
#include "avion_host.h"
#include "avion_rms.h"

namespace {

template <int N>
using Int = std::integral_constant<int, N>;

// ------------------------------------------------------------------------------ RMS normalisation
int rms_check(long long M, int D, unsigned flags, unsigned allowed)
{
    if (M < 0 || D < 1) return AVION_EINVAL;
    if (flags & ~allowed) return AVION_EINVAL;
    if (D % 8 != 0 || D > kRmsMaxD) return AVION_EUNSUPPORTED;
    if (M > (1LL << 40)) return AVION_EUNSUPPORTED;
    return AVION_OK;
}
// Lanes a row.  A wavefront holds up to 2048 columns (4 chunks a lane) and needs no exchange through LDS; narrow rows take 16
// or 32 lanes (forward and backward of 600000 x 128 111 + 112 us with 16, 214 + 208 with 64; 100000 x 256 39 + 38 and 45 + 46),
// wide ones four wavefronts, or eight beyond 8192.  So few rows that each has a workgroup of its own take four wavefronts as
// well: 1 x 1024 2.3 and 2.5 us, 300 x 1024 2.9 and 3.0; with more rows than workgroups, 1000 x 768, 3.8 and 3.3.
int rms_lanes(long long M, int D)
{
    if (D > 8192) return 512;
    if (D > 2048 || (D > 512 && M <= kRmsMaxGrid)) return 256;
    return D <= 128 ? 16 : D <= 256 ? 32 : 64;
}
unsigned rms_grid(long long M, int D, int most = kRmsMaxGrid)
{
    const int lanes = rms_lanes(M, D), rows = lanes <= 64 ? kRmsWaves * (64 / lanes) : 1;
    return (unsigned)std::min<long long>((M + rows - 1) / rows, most);
}
// f(lanes a row, chunks a lane)
template <typename F>
int rms_by_width(long long M, int D, F f)
{
    const int lanes = rms_lanes(M, D), per_lane = (D / 8 + lanes - 1) / lanes;
    if (lanes == 16) return f(Int<16>{}, Int<1>{});
    if (lanes == 32) return f(Int<32>{}, Int<1>{});
    if (lanes == 512) return f(Int<512>{}, Int<4>{});
    if (lanes == 256) {
        if (per_lane <= 1) return f(Int<256>{}, Int<1>{});
        if (per_lane <= 2) return f(Int<256>{}, Int<2>{});
        return f(Int<256>{}, Int<4>{});
    }
    if (per_lane <= 1) return f(Int<64>{}, Int<1>{});
    if (per_lane <= 2) return f(Int<64>{}, Int<2>{});
    return f(Int<64>{}, Int<4>{});
}
// f(stream's format): E, or fp32
template <typename E, typename F>
int rms_by_stream(unsigned flags, F f)
{
    if (flags & AVION_FLAG_WIDE_F32) return f(TypeTag<float>{});
    return f(TypeTag<E>{});
}

template <bool F8>
int rmsnorm_fwd_impl(const void* x, const void* residual, const float* weight, void* y, float* scale, void* h, float* rstd, long long M,
                     int D, float eps, unsigned flags, void* stream)
{
    const int rc = rms_check(M, D, flags, AVION_FLAG_F16 | AVION_FLAG_WIDE_F32);
    if (rc != AVION_OK) return rc;
    if (!(eps >= 0.f) || !std::isfinite(eps)) return AVION_EINVAL;
    if (M == 0) return AVION_OK;
    if (!x || !weight || !y || (F8 && !scale) || (residual == nullptr) != (h == nullptr)) return AVION_EINVAL;
    if (!residual && (flags & AVION_FLAG_WIDE_F32)) return AVION_EINVAL;
    const void* ptrs[] = {x, residual, weight, y, scale, h, rstd};
    for (const void* p : ptrs)
        if (!aligned16(p)) return AVION_EUNSUPPORTED;
    if (F8 && D % 16 != 0) return AVION_EUNSUPPORTED;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return by_element(flags, [&](auto fmt) {
        using E = typename decltype(fmt)::type;
        return rms_by_stream<E>(flags, [&](auto wide) {
            return rms_by_width(M, D, [&](auto lanes, auto nch) {
                constexpr int LANES = decltype(lanes)::value;
                begin_launch();
                hipLaunchKernelGGL((avion_rmsnorm_fwd_kernel<LANES, decltype(nch)::value, E, typename decltype(wide)::type, F8>),
                                   dim3(rms_grid(M, D)), dim3(RmsWork<LANES>::WAVES * 64), 0, st, static_cast<const raw16*>(x),
                                   residual, weight, y, scale, h, rstd, (long)M, D, eps);
                return end_launch("launch avion_rmsnorm_fwd_kernel");
            });
        });
    });
}

// --------------------------------------------------------------------------------- token table
constexpr unsigned kEmbFlags = AVION_FLAG_F16 | AVION_FLAG_WIDE_F32 | AVION_FLAG_TOKENS_I32;
constexpr int kEmbMaxD = 65536;
constexpr long long kEmbMax = 1LL << 28;  // slots, and rows of the table

int embedding_check(long long n, long long V, int D, unsigned flags)
{
    if (n < 0 || V < 1 || D < 1) return AVION_EINVAL;
    if (flags & ~kEmbFlags) return AVION_EINVAL;
    if (D % 8 != 0 || D > kEmbMaxD || V > kEmbMax || n > kEmbMax) return AVION_EUNSUPPORTED;
    if (n * (D / 8) > (1LL << 33)) return AVION_EUNSUPPORTED;  // threads of the lookup: below 2^32
    return AVION_OK;
}
// f(token type, table's format, output's format)
template <typename F>
int embedding_by_type(unsigned flags, F f)
{
    return by_element(flags, [&](auto fmt) {
        auto by_table = [&](auto tok) {
            if (flags & AVION_FLAG_WIDE_F32) return f(tok, TypeTag<float>{}, fmt);
            return f(tok, fmt, fmt);
        };
        if (flags & AVION_FLAG_TOKENS_I32) return by_table(TypeTag<int>{});
        return by_table(TypeTag<long>{});
    });
}
// How the gradient of n slots is cut: digits of the sort, its workgroups, chunks of the sums, and where all of it lies.
struct EmbeddingPlan {
    int passes, bits, nsort, chunk;
    long long per, nchunks;
    size_t keys[2], slots[2], hist, stamp, heads, tails, bytes;
    EmbeddingPlan(long long n, long long V, int D)
    {
        if (n <= kEmbSmallTokens) {
            bytes = 256;
            return;
        }
        const bool radix = n > kEmbRankSlots;
        int need = 0;  // keys 0 .. V
        while ((V >> need) != 0) ++need;
        passes = (need + 9) / 10;
        bits = need <= 8 * passes ? 8 : 10;
        // whole tiles a workgroup, at most kEmbSortGrid workgroups
        const long long tiles = (n + kEmbSortTile - 1) / kEmbSortTile;
        per = (tiles + kEmbSortGrid - 1) / kEmbSortGrid * kEmbSortTile;
        nsort = (int)((n + per - 1) / per);
        chunk = kEmbSumWaves * (n < kEmbSumEnough ? kEmbSumFew : kEmbSumMost);
        nchunks = (n + chunk - 1) / chunk;
        size_t at = 0;
        auto take = [&](size_t b) {
            const size_t here = at;
            at += round256(b);
            return here;
        };
        for (int i = 0; i < (radix ? 2 : 1); ++i) keys[i] = take(n * 4);
        for (int i = 0; i < (radix ? 2 : 1); ++i) slots[i] = take(n * 4);
        if (!radix) {
            passes = 1;  // the result lies where one pass would leave it
            keys[1] = keys[0];
            slots[1] = slots[0];
        }
        hist = take(radix ? (size_t)nsort * 4 << bits : 0);
        stamp = take(V * 4);
        heads = take((size_t)nchunks * D * 4);
        tails = take((size_t)nchunks * D * 4);
        bytes = at;
    }
};
// table rows of a clearing workgroup
int clear_rows(long long V, int D, size_t element, int most)
{
    const long long fits = kEmbClearBytes / ((long long)D * (long long)element);
    return (int)std::min<long long>(std::max({fits, 1LL, (V >> 20) + 1}), most);
}

}  // namespace

extern "C" {

int avion_rmsnorm_fwd(const void* x, const void* residual, const float* weight, void* y, void* h, float* rstd, long long M, int D,
                      float eps, unsigned flags, void* stream)
{
    return rmsnorm_fwd_impl<false>(x, residual, weight, y, nullptr, h, rstd, M, D, eps, flags, stream);
}

int avion_rmsnorm_fwd_fp8(const void* x, const void* residual, const float* weight, void* y8, float* scale, void* h, long long M,
                          int D, float eps, unsigned flags, void* stream)
{
    return rmsnorm_fwd_impl<true>(x, residual, weight, y8, scale, h, nullptr, M, D, eps, flags, stream);
}

size_t avion_rmsnorm_bwd_workspace_bytes(long long M, int D)
{
    if (rms_check(M, D, 0, 0) != AVION_OK) return 0;
    return round256(std::max<size_t>((size_t)rms_grid(M, D) * D * sizeof(float), 1));
}

int avion_rmsnorm_bwd(const void* h, const float* weight, const float* rstd, const void* dy, const void* dh, void* dx, float* dresidual,
                      float* dweight, long long M, int D, unsigned flags, void* workspace, size_t workspace_bytes, void* stream)
{
    const int rc = rms_check(M, D, flags, AVION_FLAG_F16 | AVION_FLAG_WIDE_F32);
    if (rc != AVION_OK) return rc;
    if (!dweight) return AVION_EINVAL;
    if (M > 0 && (!h || !weight || !rstd || !dy)) return AVION_EINVAL;
    if (dresidual && !(flags & AVION_FLAG_WIDE_F32)) return AVION_EINVAL;
    const void* ptrs[] = {h, weight, rstd, dy, dh, dx, dresidual, dweight};
    for (const void* p : ptrs)
        if (!aligned16(p)) return AVION_EUNSUPPORTED;
    if (!workspace_fits(workspace, workspace_bytes, avion_rmsnorm_bwd_workspace_bytes(M, D))) return AVION_EWORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    float* part = static_cast<float*>(workspace);
    const unsigned grid = rms_grid(M, D);
    // One launch where the gains' gradient can read the rows once more at little cost (they are in the caches then): a launch
    // and its kernel less (this call on 4 x 64: 7.6 -> 4.0 us of the host's time).  On the GPU, one launch and two: 300 x 1024 4.0
    // and 6.6, 640 x 64 5.1 and 5.0, x 768 5.4 and 6.2, x 2048 7.9 and 8.8, x 16384 22.4 and 34.9; 704 x 64 5.8 and 5.0, x 768 6.0
    // and 6.6, x 1536 8.1 and 8.0; 800 x 768 7.2 and 6.7; 1024 x 64 7.1 and 5.0, x 768 9.4 and 7.0 (a chain of 8 loads).
    const bool few = M > 0 && M <= kRmsFewRows;
    if (M > 0) {
        const int r1 = by_element(flags, [&](auto fmt) {
            using E = typename decltype(fmt)::type;
            return rms_by_stream<E>(flags, [&](auto wide) {
                return rms_by_width(M, D, [&](auto lanes, auto nch) {
                    constexpr int LANES = decltype(lanes)::value, NCH = decltype(nch)::value;
                    using R = typename decltype(wide)::type;
                    const raw16* g = static_cast<const raw16*>(dy);
                    const dim3 block(RmsWork<LANES>::WAVES * 64);
                    begin_launch();
                    if (few)
                        hipLaunchKernelGGL((avion_rmsnorm_bwd_kernel<LANES, NCH, E, R, true>),
                                           dim3(grid + (D + kRmsFewCols - 1) / kRmsFewCols), block, 0, st, h, weight, rstd, g, dh, dx, dresidual,
                                           part, dweight, (long)M, D, (int)grid);
                    else
                        hipLaunchKernelGGL((avion_rmsnorm_bwd_kernel<LANES, NCH, E, R, false>), dim3(grid), block,
                                           LANES <= 64 ? (kRmsWaves - 1) * D * sizeof(float) : 0, st, h, weight, rstd, g, dh, dx, dresidual, part,
                                           dweight, (long)M, D, (int)grid);
                    return end_launch("launch avion_rmsnorm_bwd_kernel");
                });
            });
        });
        if (r1 != AVION_OK || few) return r1;
    }
    // sums over the workgroups (none: zeros); the reduction kernel splits its 2 * (D / 2) columns into two outputs
    begin_launch();
    hipLaunchKernelGGL((avion_ln_param_reduce_kernel<void>), dim3((D + kLnReduceCols - 1) / kLnReduceCols),
                       dim3(kLnReduceCols * kLnReduceGroups), 0, st, part, dweight, dweight + D / 2, (int)grid, D / 2);
    return end_launch("launch avion_ln_param_reduce_kernel");
}

int avion_quantize_rows(const void* x, void* x8, float* scale, long long M, int D, unsigned flags, void* stream)
{
    const int rc = rms_check(M, D, flags, AVION_FLAG_F16);
    if (rc != AVION_OK) return rc;
    if (M == 0) return AVION_OK;
    if (!x || !x8 || !scale) return AVION_EINVAL;
    if (!aligned16(x) || !aligned16(x8) || !aligned16(scale) || D % 16 != 0) return AVION_EUNSUPPORTED;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int grid = D <= 512 || (D <= 1024 && M * D >= (1 << 24)) ? kQuantizeMaxGrid : kRmsMaxGrid;
    return by_element(flags, [&](auto fmt) {
        return rms_by_width(M, D, [&](auto lanes, auto nch) {
            constexpr int LANES = decltype(lanes)::value;
            begin_launch();
            hipLaunchKernelGGL((avion_quantize_rows_kernel<LANES, decltype(nch)::value, typename decltype(fmt)::type>),
                               dim3(rms_grid(M, D, grid)), dim3(RmsWork<LANES>::WAVES * 64), 0, st,
                               static_cast<const raw16*>(x), x8, scale, (long)M, D);
            return end_launch("launch avion_quantize_rows_kernel");
        });
    });
}

int avion_embedding_fwd(const void* tokens, const void* table, void* y, long long n, long long V, int D, float scale, unsigned flags,
                        void* stream)
{
    const int rc = embedding_check(n, V, D, flags);
    if (rc != AVION_OK) return rc;
    if (!std::isfinite(scale)) return AVION_EINVAL;
    if (n == 0) return AVION_OK;
    if (!tokens || !table || !y) return AVION_EINVAL;
    if (!aligned16(table) || !aligned16(y)) return AVION_EUNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(tokens) % (flags & AVION_FLAG_TOKENS_I32 ? 4 : 8) != 0) return AVION_EUNSUPPORTED;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const int pieces = D / 8;
    const unsigned magic = (unsigned)(((1ULL << 32) + pieces - 1) / pieces);
    const long long per = kEmbThreads * kEmbFly, grid = (n * pieces + per - 1) / per;
    return embedding_by_type(flags, [&](auto tok, auto tab, auto fmt) {
        using T = typename decltype(tok)::type;
        begin_launch();
        hipLaunchKernelGGL((avion_embedding_fwd_kernel<T, typename decltype(tab)::type, typename decltype(fmt)::type>),
                           dim3((unsigned)grid), dim3(kEmbThreads), 0, st, static_cast<const T*>(tokens), table,
                           static_cast<raw16*>(y), (long)n, (int)V, D, scale, pieces, magic);
        return end_launch("launch avion_embedding_fwd_kernel");
    });
}

size_t avion_embedding_bwd_workspace_bytes(long long n, long long V, int D)
{
    if (embedding_check(n, V, D, 0) != AVION_OK) return 0;
    return EmbeddingPlan(n, V, D).bytes;
}

int avion_embedding_bwd(const void* tokens, const void* dy, void* dtable, long long n, long long V, int D, float scale, unsigned flags,
                        void* workspace, size_t workspace_bytes, void* stream)
{
    const int rc = embedding_check(n, V, D, flags);
    if (rc != AVION_OK) return rc;
    if (!std::isfinite(scale) || !dtable || (n > 0 && (!tokens || !dy))) return AVION_EINVAL;
    if (!aligned16(dy) || !aligned16(dtable)) return AVION_EUNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(tokens) % (flags & AVION_FLAG_TOKENS_I32 ? 4 : 8) != 0) return AVION_EUNSUPPORTED;
    const EmbeddingPlan p(n, V, D);
    if (!workspace_fits(workspace, workspace_bytes, p.bytes)) return AVION_EWORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return embedding_by_type(flags, [&](auto tok, auto tab, auto fmt) -> int {
        using T = typename decltype(tok)::type;
        using TE = typename decltype(tab)::type;
        using E = typename decltype(fmt)::type;
        const T* t = static_cast<const T*>(tokens);
        const raw16* g = static_cast<const raw16*>(dy);
        const size_t element = std::is_same_v<TE, float> ? 4 : 2;
        const int ncol = (D + kEmbCols - 1) / kEmbCols;
        if (n <= kEmbSmallTokens) {
            const int rows = clear_rows(V, D, element, kEmbSmallRows);
            begin_launch();
            hipLaunchKernelGGL((avion_embedding_bwd_small_kernel<T, E, TE>), dim3((unsigned)(ncol * n + (V + rows - 1) / rows)),
                               dim3(kEmbSmallThreads), 0, st, t, g, dtable, (int)n, (int)V, D, scale, ncol, rows);
            return end_launch("launch avion_embedding_bwd_small_kernel");
        }
        char* ws = static_cast<char*>(workspace);
        unsigned *keys[2], *slots[2];
        for (int i = 0; i < 2; ++i) {
            keys[i] = reinterpret_cast<unsigned*>(ws + p.keys[i]);
            slots[i] = reinterpret_cast<unsigned*>(ws + p.slots[i]);
        }
        unsigned *hist = reinterpret_cast<unsigned*>(ws + p.hist), *stamp = reinterpret_cast<unsigned*>(ws + p.stamp);
        float *heads = reinterpret_cast<float*>(ws + p.heads), *tails = reinterpret_cast<float*>(ws + p.tails);
        const int rows = clear_rows(V, D, element, 1 << 28);
        auto sort = [&](auto first, auto width, int pass) {
            constexpr bool FIRST = decltype(first)::value;
            constexpr int BITS = decltype(width)::value;
            const int to = pass % 2, from = 1 - to, shift = pass * BITS;
            const dim3 threads(kEmbSortThreads);
            begin_launch();
            hipLaunchKernelGGL((avion_embedding_hist_kernel<T, FIRST, BITS>), dim3(p.nsort), threads, 0, st, t, keys[from], stamp, hist,
                               (long)n, (int)V, (long)p.per, shift);
            const int rh = end_launch("launch avion_embedding_hist_kernel");
            if (rh != AVION_OK) return rh;
            // each placing launch clears its share of the table
            const long clear_from = (long)(V * pass / p.passes), clear_to = (long)(V * (pass + 1) / p.passes);
            const unsigned clearing = (unsigned)((clear_to - clear_from + rows - 1) / rows);
            begin_launch();
            hipLaunchKernelGGL((avion_embedding_place_kernel<T, FIRST, BITS, TE>), dim3(p.nsort + clearing), threads, 0, st, t, keys[from],
                               slots[from], hist, stamp, keys[to], slots[to], dtable, (long)n, (int)V, D, (long)p.per, p.nsort, shift, rows,
                               clear_from, clear_to);
            return end_launch("launch avion_embedding_place_kernel");
        };
        const bool ranked = n <= kEmbRankSlots;
        if (ranked) {
            begin_launch();
            hipLaunchKernelGGL((avion_embedding_rank_kernel<T>), dim3((unsigned)((n + 63) / 64)), dim3(kEmbSortThreads), 0, st, t, keys[0],
                               slots[0], stamp, (int)n, (int)V);
            const int rr = end_launch("launch avion_embedding_rank_kernel");
            if (rr != AVION_OK) return rr;
        }
        for (int pass = 0; !ranked && pass < p.passes; ++pass) {
            const int rk = pass == 0 ? (p.bits == 8 ? sort(std::true_type{}, Int<8>{}, 0) : sort(std::true_type{}, Int<10>{}, 0))
                                     : (p.bits == 8 ? sort(std::false_type{}, Int<8>{}, pass) : sort(std::false_type{}, Int<10>{}, pass));
            if (rk != AVION_OK) return rk;
        }
        const int last = (p.passes - 1) % 2;
        auto sums = [&](auto per) {
            const unsigned clearing = ranked ? (unsigned)((V + rows - 1) / rows) : 0u;
            begin_launch();
            hipLaunchKernelGGL((avion_embedding_sum_kernel<decltype(per)::value, E, TE>), dim3((unsigned)p.nchunks * ncol + clearing),
                               dim3(kEmbSumWaves * 64), 0, st, keys[last], slots[last], g, dtable, heads, tails, (long)n, (int)V, D, scale,
                               (int)p.nchunks, ncol, stamp, rows);
            return end_launch("launch avion_embedding_sum_kernel");
        };
        const int rs = n < kEmbSumEnough ? sums(Int<kEmbSumFew>{}) : sums(Int<kEmbSumMost>{});
        if (rs != AVION_OK) return rs;
        begin_launch();
        hipLaunchKernelGGL((avion_embedding_join_kernel<TE>), dim3((unsigned)p.nchunks, (D + kEmbJoinCols - 1) / kEmbJoinCols),
                           dim3(kEmbJoinGroups * kEmbJoinCols / 4), 0, st, keys[last], heads, tails, dtable, (long)n, (int)V, D, scale,
                           (long)p.nchunks, p.chunk);
        return end_launch("launch avion_embedding_join_kernel");
    });
}

}  // extern "C"
