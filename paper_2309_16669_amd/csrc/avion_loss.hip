// C ABI of the loss over a vocabulary.  See include/avion_attn.h for its contract.
#include "avion_attn.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "avion_host.h"
#include "avion_loss.h"

namespace {

constexpr long long kComputeUnits = 256;

struct LossShape {
    long long T, V;
    int D;
};
int loss_check(const LossShape& s)
{
    if (s.T < 0 || s.V < 1 || s.D < 1) return AVION_EINVAL;
    if (s.D % 8 != 0 || s.D > (1 << 16) || s.T >= (1 << 28) || s.V > (1 << 28)) return AVION_EUNSUPPORTED;
    return AVION_OK;
}
long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

enum class LossTiles { kFew, kLow, kSmall, kLarge };  // 32 rows x 128 columns, 64 x 128, 128 x 128, 256 x 256
// Forward: 256 x 256 where they are a compute unit's at least, 128 x 128 where they are more than the compute units, else 64 x 128.
//   Of 128 and 64 rows, in a graph, us: 2048 x 2048 x 512 19.4, 18.6; 997 x 10007 x 776 41.7, 42.5; 4000 x 3700 x 1024 46, 54; 200 x 50000 x 768 36, 42
// dz: 64 x 128, whose stores the other workgroups of a compute unit fill up, below 1.4 tiles of 256 x 256 for one.
//   Whole backward with 128 and 64 rows: 2048 x 2048 x 512 46, 42; 997 x 10007 x 776 110, 102; 4000 x 3700 x 1024 178, 156; 200 x 50000 x 768 129, 114;
//   with 256 and 64: 1000 x 20000 x 768 163, 149; 4200 x 4200 x 2048 343, 321; 4096 x 10000 x 1024 335, 337; 5000 x 5000 x 4096 585, 654; 16384 x 50000 x
//   768 3655, 4108
LossTiles loss_tiles(long long rows, long long cols)
{
    if (rows <= 32) return LossTiles::kFew;
    if (ceil_div(rows, 256) * ceil_div(cols, 256) >= kComputeUnits) return LossTiles::kLarge;
    return ceil_div(rows, 128) * ceil_div(cols, 128) > kComputeUnits ? LossTiles::kSmall : LossTiles::kLow;
}
LossTiles dz_tiles(long long rows, long long cols)
{
    if (rows <= 32) return LossTiles::kFew;
    return rows * cols >= kComputeUnits * 7 / 5 * 256 * 256 ? LossTiles::kLarge : LossTiles::kLow;
}
// tile height and width, wavefronts
template <int TB_>
struct Tile {
    static constexpr int TB = TB_, TA = TB == 256 ? 256 : 128, WA = TB == 128 ? 2 : 4, WB = TB < 128 ? 1 : 2;
};
template <bool DZ, typename F>
int by_tiles(LossTiles t, F f)
{
    if (t == LossTiles::kFew) return f(Tile<32>{});
    if (t == LossTiles::kLow) return f(Tile<64>{});
    if constexpr (!DZ)
        if (t == LossTiles::kSmall) return f(Tile<128>{});
    return f(Tile<256>{});
}

// runs of vocabulary tiles in the forward: enough workgroups for the chip, whole rounds of them where there are many
int loss_slabs(const LossShape& s)
{
    const LossTiles t = loss_tiles(s.T, s.V);
    const long long tb = t == LossTiles::kFew ? 32 : t == LossTiles::kLow ? 64 : t == LossTiles::kSmall ? 128 : 256, ta = t == LossTiles::kLarge ? 256 : 128;
    const long long blocks = std::max<long long>(1, ceil_div(s.T, tb)), tiles = ceil_div(s.V, ta), at_once = t == LossTiles::kLarge ? kComputeUnits : 2 * kComputeUnits;
    return (int)std::max<long long>(1, std::min<long long>(tiles, at_once / blocks));
}
struct LossForward {  // offsets of its workspace
    size_t hit, sums, ticket, bytes;
    LossForward(const LossShape& s)
    {
        hit = round256((size_t)loss_slabs(s) * s.T * sizeof(float2));
        sums = hit + round256((size_t)s.T * 4);
        ticket = sums + round256((size_t)ceil_div(s.T, 4) * sizeof(double2));
        bytes = ticket + 256;
    }
};

// A piece of the vocabulary in the backward: dz of it is at most kLossPiece bytes (or 256 columns), in pieces of equal size
constexpr long long kLossPiece = 1LL << 30;
long long loss_piece(const LossShape& s)
{
    const long long most = std::max<long long>(256, kLossPiece / (2 * std::max<long long>(1, s.T)) / 256 * 256);
    const long long pieces = ceil_div(s.V, most);
    return std::min<long long>(most, ceil_div(ceil_div(s.V, pieces), 256) * 256);
}
long long loss_ld(const LossShape& s) { return std::min(loss_piece(s), ceil_div(s.V, 64) * 64); }
// The two gradients' tiles: 256 x 256 where both together have one for each compute unit and no side is narrower than one, else 128 x
// 128.  Both passes in a graph with 256 and with 128, us: 16384 x 50000 x 768 4787, 5242; 65536 x 8192 x 768 3315, 3581; 8192 x 8192 x 1024 519, 549;
// in between by how full the last round is (8192 x 20000 x 768 1049, 1089; 8192 x 32000 x 1024 2238, 2119); below, 997 x 10007 x 776 157, 142;
// 2048 x 2048 x 512 67, 60.  Either way a product whose steps are more than a workgroup's fair share of all (few tiles, long K) is cut along K, at
// least 4 steps a range: 213 x 112000 x 72, dx of which is two tiles of 1750 steps, 2540 us without.  A range's plane is written and
// read again, so there are no more of them than that.
bool grads_large(const LossShape& s, long long n)
{
    return s.T >= 256 && n >= 256 && s.D > 128 && (ceil_div(s.T, 256) + ceil_div(n, 256)) * ceil_div(s.D, 256) >= kComputeUnits;
}
int grad_splits(const LossShape& s, long long n, bool dw)
{
    const long long t = grads_large(s, n) ? 256 : 128, at_once = t == 256 ? kComputeUnits : 2 * kComputeUnits;
    const long long of_x = ceil_div(n, kLossStep), of_w = ceil_div(s.T, kLossStep), steps = dw ? of_w : of_x;
    const long long all = (ceil_div(s.T, t) * of_x + ceil_div(n, t) * of_w) * ceil_div(s.D, t), fair = std::max<long long>(4, ceil_div(all, at_once));
    return (int)std::max<long long>(1, std::min<long long>(ceil_div(steps, fair), steps / 4));
}
// floats of a plane: whole tiles
long long plane_floats(const LossShape& s, long long n, long long rows)
{
    const long long t = grads_large(s, n) ? 256 : 128;
    return ceil_div(rows, t) * ceil_div(s.D, t) * t * t;
}
int loss_padded(const LossShape& s) { return (int)(ceil_div(s.T, 256) * 256); }
struct LossBackward {
    size_t rows, dz, sum_x, sum_w, bytes;
    bool planes_x, planes_w;
    LossBackward(const LossShape& s)
    {
        const long long n = loss_piece(s);
        const int sx = grad_splits(s, n, false), sw = grad_splits(s, n, true);
        planes_x = n < s.V || sx > 1;
        planes_w = sw > 1;
        rows = 256;
        dz = rows + round256((size_t)loss_padded(s) * 12);
        sum_x = dz + round256((size_t)s.T * loss_ld(s) * 2);
        sum_w = sum_x + (planes_x ? round256((size_t)sx * plane_floats(s, n, s.T) * 4) : 0);
        bytes = sum_w + (planes_w ? round256((size_t)sw * plane_floats(s, n, std::min(n, s.V)) * 4) : 0);
    }
};

template <typename K, typename... Args>
int launch(K kernel, int lds, std::atomic<unsigned long long>& allowed, long long grid, int threads, hipStream_t st, const char* what, Args... args)
{
    const hipError_t attr = lds > 32 * 1024 ? allow_lds_here(kernel, lds, allowed) : hipSuccess;
    if (attr != hipSuccess) return hip_fail(attr, "hipFuncSetAttribute(loss)");
    begin_launch();
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(threads), lds, st, args...);
    return end_launch(what);
}
long long persistent(long long tiles, int tb) { return ceil_div(std::min(tiles, tb == 256 ? kComputeUnits : 2 * kComputeUnits), 8) * 8; }

int loss_inputs(const LossShape& s, const void* x, const void* w, const void* targets, long long rs_x, long long rs_w, float scale,
                unsigned flags, unsigned allowed)
{
    if (flags & ~allowed) return AVION_EINVAL;
    if (!std::isfinite(scale) || !(scale > 0.f)) return AVION_EINVAL;
    const int rc = loss_check(s);
    if (rc != AVION_OK) return rc;
    if (rs_x < s.D || rs_w < s.D) return AVION_EINVAL;
    if (rs_x % 8 != 0 || rs_w % 8 != 0 || rs_x > (1 << 20) || rs_w > (1 << 20)) return AVION_EUNSUPPORTED;
    if (!w || (s.T > 0 && (!x || !targets))) return AVION_EINVAL;
    if (!aligned16(x) || !aligned16(w) || reinterpret_cast<uintptr_t>(targets) % (flags & AVION_FLAG_TOKENS_I32 ? 4 : 8) != 0)
        return AVION_EUNSUPPORTED;
    return AVION_OK;
}
LossArgs loss_args(const LossShape& s, const void* x, const void* w, const void* targets, long long rs_x, long long rs_w, long long ignore,
                   float scale, unsigned flags)
{
    LossArgs a{};
    a.x = static_cast<const raw16*>(x);
    a.w = static_cast<const raw16*>(w);
    a.targets = targets;
    a.rs_x = rs_x;
    a.rs_w = rs_w;
    a.T = (int)s.T;
    a.V = (int)s.V;
    a.D = s.D;
    a.wide = flags & AVION_FLAG_TOKENS_I32 ? 0 : 1;
    a.ignore = ignore;
    a.cs = scale * kLog2e;
    a.scale = scale;
    return a;
}

}  // namespace

extern "C" {

size_t avion_linear_ce_fwd_workspace_bytes(long long T, long long V, int D)
{
    const LossShape s{T, V, D};
    return loss_check(s) == AVION_OK ? LossForward(s).bytes : 0;
}

int avion_linear_ce_fwd(const void* x, const void* w, const void* targets, float* loss, float* lse, float* total, long long T, long long V,
                        int D, long long rs_x, long long rs_w, float scale, long long ignore_index, unsigned flags, void* workspace,
                        size_t workspace_bytes, void* stream)
{
    const LossShape s{T, V, D};
    const int rc = loss_inputs(s, x, w, targets, rs_x, rs_w, scale, flags, AVION_FLAG_F16 | AVION_FLAG_TOKENS_I32 | AVION_FLAG_MEAN);
    if (rc != AVION_OK) return rc;
    if (T > 0 && (!lse || (!loss && !total))) return AVION_EINVAL;
    for (const void* p : {(const void*)loss, (const void*)lse, (const void*)total})
        if (reinterpret_cast<uintptr_t>(p) % 4 != 0) return AVION_EUNSUPPORTED;
    const LossForward at(s);
    if (!workspace_fits(workspace, workspace_bytes, at.bytes)) return AVION_EWORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const LossArgs a = loss_args(s, x, w, targets, rs_x, rs_w, ignore_index, scale, flags);
    char* ws = static_cast<char*>(workspace);
    float2* parts = reinterpret_cast<float2*>(ws);
    float* hit = reinterpret_cast<float*>(ws + at.hit);
    double2* sums = reinterpret_cast<double2*>(ws + at.sums);
    unsigned* ticket = reinterpret_cast<unsigned*>(ws + at.ticket);
    const bool mean = (flags & AVION_FLAG_MEAN) != 0;
    static std::atomic<unsigned long long> none{0};
    if (T > 0) {
        const int slabs = loss_slabs(s);
        const int first = by_element(flags, [&](auto fmt) {
            using E = typename decltype(fmt)::type;
            const LossTiles t = loss_tiles(T, V);
            return by_tiles<false>(t, [&](auto tile) {
                using X = decltype(tile);
                using Cfg = LossCfg<Along::kK, Along::kK, X::TA, X::TB, X::WA, X::WB>;
                static std::atomic<unsigned long long> allowed{0};
                return launch(avion_loss_fwd_kernel<X::TA, X::TB, X::WA, X::WB, E>, 2 * Cfg::STAGE, allowed,
                              ceil_div(ceil_div(T, X::TB) * slabs, 8) * 8, Cfg::NT, st, "launch avion_loss_fwd_kernel", a, parts, hit, slabs, ticket);
            });
        });
        if (first != AVION_OK) return first;
        const auto join = [&](auto lanes) {
            constexpr int LANES = decltype(lanes)::value;
            return launch(avion_loss_join_kernel<LANES>, 0, none, ceil_div(T, 256 / LANES), 256, st, "launch avion_loss_join_kernel", a,
                          (const float2*)parts, (const float*)hit, slabs, loss, lse, sums, ticket, mean, total);
        };
        return slabs > 32 ? join(std::integral_constant<int, 64>{}) : join(std::integral_constant<int, 16>{});
    }
    if (!total) return AVION_OK;
    return launch(avion_loss_none_kernel, 0, none, 1, 2, st, "launch avion_loss_none_kernel", total);
}

size_t avion_linear_ce_bwd_workspace_bytes(long long T, long long V, int D)
{
    const LossShape s{T, V, D};
    return loss_check(s) == AVION_OK ? LossBackward(s).bytes : 0;
}

int avion_linear_ce_bwd(const void* x, const void* w, const void* targets, const float* lse, const float* dloss, const float* total, void* dx,
                        void* dw, long long T, long long V, int D, long long rs_x, long long rs_w, float scale, long long ignore_index,
                        unsigned flags, void* workspace, size_t workspace_bytes, void* stream)
{
    const LossShape s{T, V, D};
    const int rc = loss_inputs(s, x, w, targets, rs_x, rs_w, scale, flags,
                               AVION_FLAG_F16 | AVION_FLAG_TOKENS_I32 | AVION_FLAG_MEAN | AVION_FLAG_ONE_GRADIENT);
    if (rc != AVION_OK) return rc;
    const bool each = !(flags & AVION_FLAG_ONE_GRADIENT), mean = (flags & AVION_FLAG_MEAN) != 0;
    if ((T > 0 && (!dloss || !lse || (!dx && !dw))) || (!each && !dloss) || (mean && (each || !total))) return AVION_EINVAL;
    if (!aligned16(dx) || !aligned16(dw)) return AVION_EUNSUPPORTED;
    for (const void* p : {(const void*)lse, (const void*)dloss, (const void*)total})
        if (reinterpret_cast<uintptr_t>(p) % 4 != 0) return AVION_EUNSUPPORTED;
    const LossBackward at(s);
    if (!workspace_fits(workspace, workspace_bytes, at.bytes)) return AVION_EWORKSPACE;
    if (!dx && !dw) return AVION_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const LossArgs a = loss_args(s, x, w, targets, rs_x, rs_w, ignore_index, scale, flags);
    char* ws = static_cast<char*>(workspace);
    float* factors = reinterpret_cast<float*>(ws);
    raw16* dz = reinterpret_cast<raw16*>(ws + at.dz);
    const long long piece = loss_piece(s), ld = loss_ld(s);
    return by_element(flags, [&](auto fmt) {
        using E = typename decltype(fmt)::type;
        static std::atomic<unsigned long long> none{0};
        int rc2 = AVION_OK;
        if (each) rc2 = launch(avion_loss_largest_kernel, 0, none, 1, 1024, st, "launch avion_loss_largest_kernel", a, dloss, factors);
        int* rows = reinterpret_cast<int*>(ws + at.rows);
        const int padded = loss_padded(s);
        if (rc2 == AVION_OK)
            rc2 = launch(avion_loss_rows_kernel, 0, none, std::max(1, padded / 256), 256, st, "launch avion_loss_rows_kernel", a, lse, dloss, total,
                         each, mean, kLossHeld<E>, factors, rows, padded);
        for (long long v0 = 0; v0 < V && rc2 == AVION_OK; v0 += piece) {
            const long long n = std::min(piece, V - v0), held = std::min(ld, ceil_div(n, 8) * 8);
            if (T > 0)
                rc2 = by_tiles<true>(dz_tiles(T, n), [&](auto tile) {
                    using X = decltype(tile);
                    using Cfg = LossCfg<Along::kK, Along::kK, X::TA, X::TB, X::WA, X::WB>;
                    static std::atomic<unsigned long long> allowed{0};
                    return launch(avion_loss_dz_kernel<X::TA, X::TB, X::WA, X::WB, E>, Cfg::LDS_BYTES + 3 * kLossRowBytes, allowed,
                                  persistent(ceil_div(T, X::TB) * ceil_div(n, X::TA), X::TB), Cfg::NT, st, "launch avion_loss_dz_kernel", a,
                                  (const int*)rows, padded, (int)v0, (int)n, dz, (long)ld);
                });
            if (rc2 != AVION_OK) break;
            // (the last piece may be smaller; all use the first one's way)
            const bool last = v0 + n >= V;
            LossGrad gx{{a.w + v0 * rs_w, (long)rs_w, D, (int)n}, {dz, (long)ld, (int)T, 0}, (int)T, (int)held, grad_splits(s, piece, false),
                        reinterpret_cast<float*>(ws + at.sum_x), v0 > 0, at.planes_x ? nullptr : static_cast<raw16*>(dx)};
            LossGrad gw{{a.x, (long)rs_x, D, (int)T}, {dz, (long)ld, (int)held, (int)T}, (int)n, (int)std::max<long long>(1, T),
                        grad_splits(s, piece, true), reinterpret_cast<float*>(ws + at.sum_w), 0,
                        at.planes_w ? nullptr : static_cast<raw16*>(dw) + v0 * D};
            // (a smaller last piece may have fewer steps than planes: the others keep what they have)
            gx.splits = (int)std::min<long long>(gx.splits, ceil_div(held, kLossStep));
            if (!dx || T == 0) gx.rows = 0;
            if (!dw) gw.rows = 0;
            const auto by_grads = [&](auto f) { return grads_large(s, piece) ? f(Tile<256>{}) : f(Tile<128>{}); };
            if (gx.rows > 0 || gw.rows > 0)
                rc2 = by_grads([&](auto tile) {
                    using X = decltype(tile);
                    using Cfg = LossCfg<Along::kIndex, Along::kIndex, X::TA, X::TB, X::WA, X::WB>;
                    static std::atomic<unsigned long long> allowed{0};
                    const long long items_x = ceil_div(gx.rows, X::TB) * ceil_div(D, X::TA) * gx.splits;
                    const long long items_w = ceil_div(gw.rows, X::TB) * ceil_div(D, X::TA) * gw.splits;
                    return launch(avion_loss_grad_kernel<X::TA, X::TB, X::WA, X::WB, E>, Cfg::LDS_BYTES, allowed,
                                  persistent(items_x + items_w, X::TB), Cfg::NT, st, "launch avion_loss_grad_kernel", gx, gw,
                                  (const float*)factors, (int)items_x);
                });
            const LossPlanes px{gx.sum, grad_splits(s, piece, false), at.planes_x && last ? gx.rows : 0, static_cast<raw16*>(dx)};
            const LossPlanes pw{gw.sum, gw.splits, at.planes_w ? gw.rows : 0, static_cast<raw16*>(dw) + v0 * D};
            if (rc2 == AVION_OK && (px.rows > 0 || pw.rows > 0))
                rc2 = by_grads([&](auto tile) {
                    using X = decltype(tile);
                    const long long blocks = (ceil_div(px.rows, X::TB) + ceil_div(pw.rows, X::TB)) * ceil_div(D, X::TA) * (X::TA / 32) * (X::TB / 32);
                    return launch(avion_loss_sum_kernel<X::TA, X::TB, X::WA, X::WB, E>, 0, none, ceil_div(blocks, 4), 256, st,
                                  "launch avion_loss_sum_kernel", px, pw, D, (const float*)factors);
                });
        }
        return rc2;
    });
}

}  // extern "C"
