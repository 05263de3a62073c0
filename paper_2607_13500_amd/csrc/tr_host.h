// What the entry points of the C ABI share on the host: HIP errors as status
// codes, the marker ranges, the device guard and the counted allocations.
#pragma once

#include <dlfcn.h>
#include <stdint.h>
#include <stdlib.h>
#include <string.h>

#include <hip/hip_runtime.h>

#include "tr_plan.h"

namespace tr {

inline tr_status hip_fail(hipError_t e, const char* what)
{
    return fail(TR_EDEVICE, "%s: %s", what, hipGetErrorString(e));
}

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

// Optional roctx ranges: with the environment variable TR_ROCTX = 1 the
// marker library is opened once (dlopen, no link-time dependency) and every
// entry point that enqueues work brackets its enqueue in a range named after
// itself, so a marker trace ties each call to the kernels it launched.
struct Roctx {
    int (*push)(const char*) = nullptr;
    int (*pop)() = nullptr;
};

inline const Roctx& roctx()
{
    static const Roctx r = [] {
        Roctx x;
        const char* v = getenv("TR_ROCTX");
        if (!v || strcmp(v, "1") != 0) return x;
        void* h = dlopen("librocprofiler-sdk-roctx.so.1", RTLD_NOW | RTLD_LOCAL);
        if (!h) h = dlopen("libroctx64.so.4", RTLD_NOW | RTLD_LOCAL);
        if (!h) {
            log_line("TR_ROCTX=1 but no roctx library could be opened");
            return x;
        }
        x.push = reinterpret_cast<int (*)(const char*)>(dlsym(h, "roctxRangePushA"));
        x.pop = reinterpret_cast<int (*)()>(dlsym(h, "roctxRangePop"));
        if (!x.push || !x.pop) {
            x.push = nullptr;
            x.pop = nullptr;
            log_line("TR_ROCTX=1 but the roctx library lacks its range functions");
        } else {
            log_line("roctx ranges on");
        }
        return x;
    }();
    return r;
}

struct Range {
    bool on;
    explicit Range(const char* name) : on(roctx().push != nullptr)
    {
        if (on) roctx().push(name);
    }
    ~Range()
    {
        if (on) roctx().pop();
    }
};

// The device allocations of one tr_create call.  Test hook: with the
// environment variable TR_FAIL_ALLOC = k (k >= 1), the k-th allocation fails
// as if the device were out of memory (nothing is allocated for it), so that
// the clean-up path of tr_create can be exercised on a real device.
struct CtxAlloc {
    int count = 0;
    int fail_at = 0;
    CtxAlloc()
    {
        const char* v = getenv("TR_FAIL_ALLOC");
        if (v) fail_at = atoi(v);
    }
    template <typename T>
    hipError_t operator()(T** ptr, size_t bytes)
    {
        if (++count == fail_at) {
            *ptr = nullptr;
            return hipErrorOutOfMemory;
        }
        return hipMalloc(reinterpret_cast<void**>(ptr), bytes);
    }
};

struct DeviceGuard {
    int prev = -1;
    bool ok = true;
    explicit DeviceGuard(int dev)
    {
        if (hipGetDevice(&prev) != hipSuccess) prev = -1;
        if (prev != dev) ok = hipSetDevice(dev) == hipSuccess;
    }
    ~DeviceGuard()
    {
        int cur = -1;
        if (prev >= 0 && hipGetDevice(&cur) == hipSuccess && cur != prev) (void)hipSetDevice(prev);
    }
};

}  // namespace tr
