// Host-side helpers shared by the C ABI's files: error text, launch status, argument checks, compile-time tags.
#pragma once
#include <hip/hip_runtime.h>

#include <atomic>
#include <cstdint>
#include <cstdio>

#include "avion_attn.h"
#include "avion_common.h"

// one text per thread for the whole library (avion_last_hip_error)
inline thread_local char g_hip_error[256] = "";

namespace {

[[maybe_unused]] int hip_fail(hipError_t e, const char* what)
{
    std::snprintf(g_hip_error, sizeof g_hip_error, "%s: %s", what, hipGetErrorString(e));
    return AVION_EHIP;
}

[[maybe_unused]] bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
[[maybe_unused]] bool workspace_fits(const void* p, size_t have, size_t need)
{
    return p && (reinterpret_cast<uintptr_t>(p) & 255u) == 0 && have >= need;
}
[[maybe_unused]] size_t round256(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

// Raises the kernel's dynamic LDS limit once; `done` is the caller's per-instance flag.  A failure
// is not remembered, so the next call tries again.
template <typename K>
hipError_t allow_lds(K kernel, int bytes, std::atomic<bool>& done)
{
    if (done.load(std::memory_order_acquire)) return hipSuccess;
    const hipError_t e =
        hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess) done.store(true, std::memory_order_release);
    return e;
}

// The same, remembered for each GPU (bit = device number; beyond 64 of them each call asks again).
template <typename K>
hipError_t allow_lds_here(K kernel, int bytes, std::atomic<unsigned long long>& done)
{
    int dev = -1;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const unsigned long long bit = dev >= 0 && dev < 64 ? 1ull << dev : 0;
    if (done.load(std::memory_order_acquire) & bit) return hipSuccess;
    e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess) done.fetch_or(bit, std::memory_order_release);
    return e;
}

// Result of the launch just made on this thread.  Errors left behind by earlier, unrelated work of
// the caller are cleared before the launch (begin_launch) so that they are not mistaken for it.
[[maybe_unused]] void begin_launch() { (void)hipGetLastError(); }
[[maybe_unused]] int end_launch(const char* what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? AVION_OK : hip_fail(e, what);
}

template <typename T>
struct TypeTag {
    using type = T;
};

// f(element format) by AVION_FLAG_F16
template <typename F>
int by_element(unsigned flags, F f)
{
    if (flags & AVION_FLAG_F16) return f(TypeTag<F16>{});
    return f(TypeTag<Bf16>{});
}

}  // namespace
