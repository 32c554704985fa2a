// C ABI of the attention over sequences of different lengths.  See include/avion_attn.h for its contract.
#include "avion_attn.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "avion_host.h"
#include "avion_ragged.h"

namespace {

template <int N>
using Int = std::integral_constant<int, N>;

constexpr float kMinScale = 8.673617379884035e-19f;  // 2^-60, as avion_attn_fwd
constexpr long long kComputeUnits = 256, kMostTokens = 1 << 28, kMostSequences = 1 << 20, kMostStride = 1 << 23;

struct RaggedShape {
    long long Tq, Tk, S;
    int Hq, Hk, d;
};
int ragged_check(const RaggedShape& s)
{
    if (s.Tq < 0 || s.Tk < 0 || s.S < 0 || s.Hq < 1 || s.Hk < 1 || s.d < 1 || s.Hq % s.Hk != 0) return AVION_EINVAL;
    if ((s.d != 64 && s.d != 80 && s.d != 128) || s.Tq > kMostTokens || s.Tk > kMostTokens || s.S > kMostSequences) return AVION_EUNSUPPORTED;
    const long long G = s.Hq / s.Hk;
    if (s.Hq > (1 << 16) || s.Tq * G > (1LL << 30)) return AVION_EUNSUPPORTED;  // (rows of up to kMostStride elements, rows' numbers in an int)
    if ((s.Tq * G / 128 + s.Tk / 128 + s.S + 4) * s.Hk * 256 > 0xffffffffLL) return AVION_EUNSUPPORTED;  // threads of a launch
    return AVION_OK;
}
bool stride_ok(long long rs, int H, int d) { return rs >= (long long)H * d; }

// Few rows a sequence and many keys, or a batch most of whose sequences may be such: a wavefront per chunk of keys.  2^shift keys a chunk,
// 0: not this way.  63 single tokens and a prompt of 1000, each with 9000 keys, 32 heads on 8 of 128: 648 us, in one launch 665; 15 tokens and
// 500 with 4000 keys, 8 heads of 64: 60, 118.
// Not cut over workgroups: the keys of a sequence's rows past the first 32, and those of three or fewer sequences of more than 32 rows each.  64
// heads on 8 of 128 behind 9000 keys, 4 and 8 tokens: one sequence 40 and 349 us (32 tokens 105), four 62 and 272, 64 502 and 516.
int few_shift(const RaggedShape& s)
{
    const long long G = s.Hq / s.Hk;
    const bool few = s.Tq * G <= 32 * s.S && s.Tk >= 256 * s.S, mixed = s.S >= 4 && s.Tk >= 1024 * s.S && s.Tk >= 4 * s.Tq;
    if (s.S < 1 || !(few || mixed)) return 0;
    int shift = 8;
    while (shift < 11 && (s.Tk >> shift) * s.Hk > 8 * kComputeUnits) ++shift;
    return shift;
}
// whether sequences of more than 32 rows get a launch of their own beside it: where they may have more than a few hundred (the 63 tokens
// with a prompt of 400: 597 us, without 10300; 128 tokens with 2000 keys, which need none, 217 and 213)
bool few_apart(const RaggedShape& s) { return s.Tq * (s.Hq / s.Hk) > 256; }
long long few_slots(const RaggedShape& s, int shift) { return (s.Tk >> shift) + s.S + 2; }
size_t few_bytes(const RaggedShape& s)
{
    const int shift = few_shift(s);
    return shift == 0 ? 0 : round256((size_t)few_slots(s, shift) * s.Hk * (32 * s.d + 96) * 4);
}

enum class RaggedWay { kShort, kWide, kSplitHalf, kSplit, kSplit4 };
// rows: of one head, over S sequences; heads: that are worked on apart.  By how many whole blocks there are (wide, split, split4; forward
// and backward, us):
//   from two for a compute unit on the wide cut: 1092 blocks (17 x 500 tokens, 16 heads on 4, causal) 26 + 88, 37 + 102, 60 + 133; 608
//   (4000 and 5700, 8 heads) 148 + 377, 164 + 409, 220 + 504; 416 (300, 2000, 900, 16 heads, causal) 39 + 97, 26 + 70, 38 + 101; 410
//   (1000 to 5000, 4 on 2 of 128 channels, causal) 125 + 372, 131 + 358, 181 + 464; 160 (2000 and 500, 8 of 128) 52 + 148, 36 + 96, 46 + 120;
//   split of more than 64 channels with tiles of 32 keys from one block for a compute unit, as two workgroups of one then work at a time and
//   else one does: 410 (1000 to 5000, as above) 93 + 275; 386 (12 x 500, 8 on 2 of 80) 19 + 62, 31 + 83; 284 (2000 and 1000, 12 on 4 of 80)
//   34 + 94, 37 + 100, wide 43 + 115; 218 (200 to 1000, 8 on 2 of 80) 19 + 61, 19 + 58; 160 (as above) 40 + 111;
//   split4 below 96: 112 (1000, 16 heads) 22 + 56, 15 + 54, 16 + 55; 60 (700 and 1200, 4 of 80) 26 + 67, 18 + 55, 16 + 54; 39 (5000, one
//   head) 82 + 192, 48 + 115, 38 + 86
// and sequences of less than 80 rows on average by lone wavefronts: 2048 of 6 to 77 tokens (28 on average), 8 heads, forward 54, wide 130;
// 131000 tokens in sequences of 40, 64, 77, 96, 128: 120, 115, 129, 181, 137, wide 164, 134, 160, 126, 172.
// The rule sees totals, as the lengths are on the device: one sequence of 3136 tokens (8 heads of 64, causal, forward 35 us alone) among 1000 of
// 28 (22 us) is a lone wavefronts' too, and both together take 97 us.
RaggedWay ragged_way(int d, long long rows, long long S, long long heads)
{
    if (rows < 80 * S) return RaggedWay::kShort;
    const long long blocks = (rows / 128 + S / 2) * heads;
    if (blocks >= 2 * kComputeUnits) return RaggedWay::kWide;
    if (d > 64 && blocks >= kComputeUnits) return RaggedWay::kSplitHalf;
    return blocks >= 96 ? RaggedWay::kSplit : RaggedWay::kSplit4;
}
template <int D, typename F>
int by_way(RaggedWay way, F f)
{
    if constexpr (D > 64)
        if (way == RaggedWay::kSplitHalf) return f(RaggedSplitHalf{});
    switch (way) {
        case RaggedWay::kShort: return f(RaggedShort{});
        case RaggedWay::kWide: return f(RaggedWide{});
        case RaggedWay::kSplit: return f(RaggedSplit{});
        default: return f(RaggedSplit4{});
    }
}

// dK and dV of a shared key head: by how many workgroups the query heads are walked, whose fp32 sums are added up afterwards.  Up to four
// workgroups for a compute unit, but past one only while the sums (16 bytes a channel and part, at the memory's 5 TB/s) cost less than a
// quarter of the walk (10 operations for a query, head and channel, at 0.7 PFLOP/s).  Whole backward, 1, 2, 4 and 8 parts, us: 400 tokens,
// 2 heads on one, 432 blocks 67, 81; 500, 4 on one, 220 blocks 101, 98, 109; 9000, 8 on one, 140 blocks 2055, 1451, 1318, 1115; 760, 8 on one,
// 474 blocks 298, 252, 253, 288
int dkdv_parts(const RaggedShape& s)
{
    const int G = s.Hq / s.Hk;
    const long long blocks = (s.Tk / (s.Tk < 80 * s.S ? 32 : 128) + s.S) * s.Hk;
    int parts = 1;
    for (int p = 2; p <= G && p <= 8; ++p)
        if (G % p == 0 && blocks * parts < 4 * kComputeUnits && (blocks * parts < kComputeUnits || 900 * p * s.S <= s.Tq * G)) parts = p;
    return parts;
}
long long ragged_npad(const RaggedShape& s) { return (s.Tq / 64 + s.S + 2) * 64; }
size_t scalar_bytes(const RaggedShape& s) { return round256((size_t)s.Hq * 2 * ragged_npad(s) * 4); }
size_t parts_bytes(const RaggedShape& s)
{
    const int parts = dkdv_parts(s);
    return parts == 1 ? 0 : round256((size_t)parts * 2 * s.Tk * s.Hk * s.d * 4);
}

// f(head channels, element format)
template <typename F>
int by_head(int d, unsigned flags, F f)
{
    return by_element(flags, [&](auto fmt) {
        if (d == 64) return f(Int<64>{}, fmt);
        if (d == 80) return f(Int<80>{}, fmt);
        return f(Int<128>{}, fmt);
    });
}
RaggedArgs ragged_args(const RaggedShape& s, const void* q, const void* k, const void* v, const int* off_q, const int* off_k, long long rs_q,
                       long long rs_k, long long rs_v, float scale, unsigned flags)
{
    RaggedArgs a{};
    a.q = static_cast<const raw16*>(q);
    a.k = static_cast<const raw16*>(k);
    a.v = static_cast<const raw16*>(v);
    a.off_q = off_q;
    a.off_k = off_k;
    a.rs_q = rs_q;
    a.rs_k = rs_k;
    a.rs_v = rs_v;
    a.S = (int)s.S;
    a.Tq = (int)s.Tq;
    a.Tk = (int)s.Tk;
    a.Hq = s.Hq;
    a.Hk = s.Hk;
    a.G = s.Hq / s.Hk;
    while ((1LL << a.g_shift) < a.G) ++a.g_shift;
    a.g_mul = (unsigned)((1ULL << 32) * ((1ULL << a.g_shift) - a.G) / a.G + 1);
    a.causal = flags & AVION_FLAG_CAUSAL ? 1 : 0;
    a.cs = scale * kLog2e;
    a.scale = scale;
    return a;
}

template <typename K, typename... Args>
int launch(K kernel, int lds, std::atomic<unsigned long long>& allowed, long long grid, int threads, hipStream_t st, const char* what, Args... args)
{
    const hipError_t attr = lds ? allow_lds_here(kernel, lds, allowed) : hipSuccess;
    if (attr != hipSuccess) return hip_fail(attr, "hipFuncSetAttribute(ragged attention)");
    begin_launch();
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(threads), lds, st, args...);
    return end_launch(what);
}

template <typename Cut>
long long workgroups(long long jobs)
{
    return (jobs + Cut::JOBS - 1) / Cut::JOBS;
}

int ragged_inputs(const RaggedShape& s, const void* q, const void* k, const void* v, const int* off_q, const int* off_k, long long rs_q,
                  long long rs_k, long long rs_v, float scale, unsigned flags)
{
    if (flags & ~(AVION_FLAG_F16 | AVION_FLAG_CAUSAL)) return AVION_EINVAL;
    if (!(scale >= kMinScale) || !std::isfinite(scale)) return AVION_EINVAL;
    const int rc = ragged_check(s);
    if (rc != AVION_OK) return rc;
    if (!stride_ok(rs_q, s.Hq, s.d) || !stride_ok(rs_k, s.Hk, s.d) || !stride_ok(rs_v, s.Hk, s.d)) return AVION_EINVAL;
    for (const long long rs : {rs_q, rs_k, rs_v})
        if (rs > kMostStride || rs % 8 != 0) return AVION_EUNSUPPORTED;
    if (!off_q || !off_k || (s.Tq > 0 && !q) || (s.Tk > 0 && (!k || !v))) return AVION_EINVAL;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v)) return AVION_EUNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(off_q) % 4 != 0 || reinterpret_cast<uintptr_t>(off_k) % 4 != 0) return AVION_EUNSUPPORTED;
    return AVION_OK;
}

}  // namespace

extern "C" {

size_t avion_ragged_fwd_workspace_bytes(long long Tq, long long Tk, long long S, int Hq, int Hk, int d)
{
    const RaggedShape s{Tq, Tk, S, Hq, Hk, d};
    return ragged_check(s) == AVION_OK ? std::max<size_t>(256, few_bytes(s)) : 0;
}

int avion_ragged_fwd(const void* q, const void* k, const void* v, const int* offsets_q, const int* offsets_k, void* o, float* lse,
                     long long Tq, long long Tk, long long S, int Hq, int Hk, int d, long long rs_q, long long rs_k, long long rs_v,
                     float scale, unsigned flags, void* workspace, size_t workspace_bytes, void* stream)
{
    const RaggedShape s{Tq, Tk, S, Hq, Hk, d};
    const int rc = ragged_inputs(s, q, k, v, offsets_q, offsets_k, rs_q, rs_k, rs_v, scale, flags);
    if (rc != AVION_OK) return rc;
    if (Tq > 0 && (!o || !lse)) return AVION_EINVAL;
    if (!aligned16(o) || reinterpret_cast<uintptr_t>(lse) % 4 != 0) return AVION_EUNSUPPORTED;
    const size_t need = few_bytes(s);
    if (need && !workspace_fits(workspace, workspace_bytes, need)) return AVION_EWORKSPACE;
    if (Tq == 0) return AVION_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    RaggedArgs a = ragged_args(s, q, k, v, offsets_q, offsets_k, rs_q, rs_k, rs_v, scale, flags);
    raw16* out = static_cast<raw16*>(o);
    return by_head(d, flags, [&](auto dim, auto fmt) {
        constexpr int D = decltype(dim)::value;
        using E = typename decltype(fmt)::type;
        const auto forward = [&](RaggedWay way) {
            return by_way<D>(way, [&](auto cut) {
                using Cut = decltype(cut);
                using Cfg = RaggedFwdCfg<D, Cut>;
                static std::atomic<unsigned long long> allowed{0};
                a.slots = (int)(Tq * a.G / Cut::BLOCK + S + 2);
                return launch(avion_ragged_fwd_kernel<D, Cut, E>, Cfg::LDS_BYTES, allowed, workgroups<Cut>((long long)a.slots * Hk),
                              Cut::NT * Cut::JOBS, st, "launch avion_ragged_fwd_kernel", a, out, lse);
            });
        };
        const int shift = few_shift(s);
        if (!shift) return forward(ragged_way(d, Tq * a.G, S, Hk));
        static std::atomic<unsigned long long> allowed{0}, none{0};
        float* parts = static_cast<float*>(workspace);
        a.done = few_apart(s) ? 32 : 0;
        if (a.done) {  // (how many sequences these are is not known: as if all rows were one's)
            const int apart = forward(ragged_way(d, Tq * a.G, 1, Hk));
            if (apart != AVION_OK) return apart;
        }
        const int first = launch(avion_ragged_few_kernel<D, E>, RaggedFwdCfg<D, RaggedLone>::LDS_BYTES, allowed, few_slots(s, shift) * Hk, 64, st,
                                 "launch avion_ragged_few_kernel", a, out, lse, parts, shift);
        if (first != AVION_OK) return first;
        return launch(avion_ragged_join_kernel<D, E>, 0, none, (S + 2) * Hk, 256, st, "launch avion_ragged_join_kernel", a, out, lse,
                      (const float*)parts, shift);
    });
}

size_t avion_ragged_bwd_workspace_bytes(long long Tq, long long Tk, long long S, int Hq, int Hk, int d)
{
    const RaggedShape s{Tq, Tk, S, Hq, Hk, d};
    return ragged_check(s) == AVION_OK ? scalar_bytes(s) + parts_bytes(s) + 256 : 0;
}

int avion_ragged_bwd(const void* q, const void* k, const void* v, const int* offsets_q, const int* offsets_k, const void* o,
                     const float* lse, const void* dO, void* dq, void* dk, void* dv, long long Tq, long long Tk, long long S, int Hq,
                     int Hk, int d, long long rs_q, long long rs_k, long long rs_v, float scale, unsigned flags, void* workspace,
                     size_t workspace_bytes, void* stream)
{
    const RaggedShape s{Tq, Tk, S, Hq, Hk, d};
    const int rc = ragged_inputs(s, q, k, v, offsets_q, offsets_k, rs_q, rs_k, rs_v, scale, flags);
    if (rc != AVION_OK) return rc;
    if ((Tq > 0 && (!o || !lse || !dO || !dq)) || (Tk > 0 && (!dk || !dv))) return AVION_EINVAL;
    for (const void* p : {o, dO, (const void*)dq, (const void*)dk, (const void*)dv})
        if (!aligned16(p)) return AVION_EUNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(lse) % 4 != 0) return AVION_EUNSUPPORTED;
    if (!workspace_fits(workspace, workspace_bytes, avion_ragged_bwd_workspace_bytes(Tq, Tk, S, Hq, Hk, d))) return AVION_EWORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    RaggedArgs a = ragged_args(s, q, k, v, offsets_q, offsets_k, rs_q, rs_k, rs_v, scale, flags);
    float* rowsc = static_cast<float*>(workspace);
    float* sums = reinterpret_cast<float*>(static_cast<char*>(workspace) + scalar_bytes(s));
    const int npad = (int)ragged_npad(s), parts = dkdv_parts(s);
    return by_head(d, flags, [&](auto dim, auto fmt) {
        constexpr int D = decltype(dim)::value;
        using E = typename decltype(fmt)::type;
        // short sequences whose heads are their own: whole, up to 64 tokens or 128; the two passes below take the others.  Beyond 64 tokens
        // of 80 channels a compute unit holds one such workgroup: 16 heads, 1024 sequences of 77, 512 (8 heads) of 100 and 1024 of 128 tokens
        // 785, 255 and 1058 us, in two passes 633, 232 and 1554; of 64 channels two, 2048 (8 heads) of 77, 1000 of 100 and of 128 384, 231 and 250,
        // 479, 270 and 467
        if (a.G == 1 && S > 0 && std::max(Tq, Tk) <= 128 * S) {
            a.done = D == 128 || (D == 80 && std::max(Tq, Tk) < 112 * S) ? 64 : 128;
            a.more = reinterpret_cast<int*>(static_cast<char*>(workspace) + scalar_bytes(s) + parts_bytes(s));
            int rc3 = AVION_OK;
            const auto whole = [&](auto w) {
                constexpr int W = decltype(w)::value;
                static std::atomic<unsigned long long> allowed{0};
                if (rc3 == AVION_OK)
                    rc3 = launch(avion_ragged_whole_kernel<D, W, E>, RaggedWholeCfg<D, W>::LDS_BYTES, allowed,
                                 W < 4 ? S * Hq : std::min<long long>(S * Hq, kComputeUnits * (160 * 1024 / RaggedWholeCfg<D, W>::LDS_BYTES)),
                                 W * 64, st,
                                 "launch avion_ragged_whole_kernel", a, static_cast<const raw16*>(dO), lse, static_cast<raw16*>(dq),
                                 static_cast<raw16*>(dk), static_cast<raw16*>(dv));
            };
            whole(Int<1>{});
            whole(Int<2>{});
            if constexpr (D < 128)
                if (a.done == 128) whole(Int<4>{});
            if (rc3 != AVION_OK) return rc3;
        }
        if (Tq > 0) {
            const int first = by_way<D>(ragged_way(d, Tq * a.G, S, Hk), [&](auto cut) {
                using Cut = decltype(cut);
                using Cfg = RaggedDqCfg<D, Cut>;
                static std::atomic<unsigned long long> allowed{0};
                a.slots = (int)(Tq * a.G / Cut::BLOCK + S + 2);
                return launch(avion_ragged_dq_kernel<D, Cut, E>, Cfg::LDS_BYTES, allowed, workgroups<Cut>((long long)a.slots * Hk),
                          Cut::NT * Cut::JOBS, st,
                              "launch avion_ragged_dq_kernel", a, static_cast<const raw16*>(o), static_cast<const raw16*>(dO), lse,
                              static_cast<raw16*>(dq), rowsc, npad);
            });
            if (first != AVION_OK) return first;
        }
        if (Tk == 0) return AVION_OK;
        const int second = by_way<D>(ragged_way(d, Tk, S, (long long)Hk * parts), [&](auto cut) {
            using Cut = decltype(cut);
            using Cfg = RaggedDkvCfg<D, Cut>;
            static std::atomic<unsigned long long> allowed{0};
            a.slots = (int)(Tk / Cut::BLOCK + S + 2);
            return launch(avion_ragged_dkdv_kernel<D, Cut, E>, Cfg::LDS_BYTES, allowed, workgroups<Cut>((long long)a.slots * Hk * parts),
                          Cut::NT * Cut::JOBS, st,
                          "launch avion_ragged_dkdv_kernel", a, static_cast<const raw16*>(dO), (const float*)rowsc, npad,
                          static_cast<raw16*>(dk), static_cast<raw16*>(dv), sums, parts);
        });
        if (second != AVION_OK || parts == 1) return second;
        static std::atomic<unsigned long long> none{0};
        const long long n = Tk * Hk * D;
        return launch(avion_ragged_sum_kernel<E>, 0, none, std::min<long long>(2048, (n / 2 + 255) / 256), 256, st,
                      "launch avion_ragged_sum_kernel", (const float*)sums, parts, (long)n, static_cast<raw16*>(dk), static_cast<raw16*>(dv),
                      scale, std::is_same<E, F16>::value ? 1.f / 256.f : 1.f);
    });
}

}  // extern "C"
