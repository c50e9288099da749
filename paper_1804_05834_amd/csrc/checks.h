// What the C entry points of the recurrent network's operators share: errors, checks of arguments, LDS beyond 64 KB.
#pragma once
#include <hip/hip_runtime.h>

#include <atomic>

#include "../../include/dqn.h"
#include "seq_common.h"

namespace {

constexpr int64_t MOST = 1ll << 48;   // no size, stride or product of sizes beyond this: byte offsets stay far below 2^63
[[maybe_unused]] int32_t bad(const char *call, const char *why) { return dqn_seq_fail(DQN_ERR_INVALID_ARG, call, why); }

[[maybe_unused]] int32_t launched(const char *call)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? (int32_t)DQN_OK : dqn_seq_fail(DQN_ERR_HIP, call, hipGetErrorString(e));
}

[[maybe_unused]] bool dtype_ok(int32_t d) { return d == DQN_F32 || d == DQN_BF16; }
[[maybe_unused]] size_t bytes_of(int32_t d) { return d == DQN_F32 ? 4 : 2; }
[[maybe_unused]] bool at(const void *p, size_t a) { return (uintptr_t)p % a == 0; }
[[maybe_unused]] bool size_ok(int64_t a, int64_t b, int64_t c) { return a >= 0 && b >= 0 && c >= 0 && (!a || !b || a * b <= MOST) && (!a || !b || !c || a * b <= MOST / c); }

[[maybe_unused]] const char *check_rows(const void *p, int64_t rs, int64_t M, int32_t C, int32_t dtype, bool written)
{
    if (!p || !at(p, bytes_of(dtype))) return "a tensor is NULL or not aligned to its elements";
    if (rs < 0 || rs > MOST || (rs > 0 && M - 1 > MOST / rs)) return "a stride is negative or too large";
    return !written || M == 1 || rs >= C ? nullptr : "rows of an output lie on top of each other";
}

// More LDS than a workgroup gets without asking: asked for once per kernel and device (and again by a racing thread, which does no harm).
// granted: the kernel's own, a bit per device.
[[maybe_unused]] bool lds_granted(const void *kernel, int bytes, std::atomic<uint64_t> &granted)
{
    if (bytes <= 65536) return true;
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev > 63) return false;
    if (!(granted.load(std::memory_order_relaxed) >> dev & 1)) {
        if (hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess) {
            (void)hipGetLastError();
            return false;
        }
        granted.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    return true;
}

}  // namespace
