// What the C entry points of the reader and of its training share on the host.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "plaid.h"

int plaid_fail(int code, const char *fmt, ...);  // sets plaid_last_error's text and returns code

#define FAIL(...) return plaid_fail(PLAID_EINVAL, __VA_ARGS__)

namespace {

struct OnDevice {  // the calling thread's device for the length of a call
    int before = -1;
    bool ok = false, moved = false;
    explicit OnDevice(int device)
    {
        ok = hipGetDevice(&before) == hipSuccess;
        if (ok && before != device) ok = moved = hipSetDevice(device) == hipSuccess;
    }
    ~OnDevice()
    {
        if (moved) (void)hipSetDevice(before);
    }
};

[[maybe_unused]] int launched()
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? PLAID_OK : plaid_fail(PLAID_EHIP, "kernel launch: %s", hipGetErrorString(e));
}
constexpr int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
constexpr int64_t round16(int64_t x) { return (x + 15) & ~(int64_t)15; }
[[maybe_unused]] bool misaligned(const void *p, size_t to) { return ((uintptr_t)p & (to - 1)) != 0; }

[[maybe_unused]] int check_workspace(const void *p, int64_t have, int64_t need)
{
    if (need > 0 && (!p || misaligned(p, 16) || have < need))
        FAIL("workspace: %lld bytes, 16-byte aligned, are needed, %lld given", (long long)need, (long long)have);
    return PLAID_OK;
}

}  // namespace
