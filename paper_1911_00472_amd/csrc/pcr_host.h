// What the entry points of the operators behind the decode share on the host.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/pcr.h"

namespace pcr {

constexpr int64_t kMaxGrid = 2147483647;

// The calling thread's device while a call enqueues its work, and the one it had behind it.
struct OnDevice {
    int before = -1;
    bool ok;
    explicit OnDevice(int device) {
        ok = hipGetDevice(&before) == hipSuccess && (before == device || hipSetDevice(device) == hipSuccess);
        if (!ok) (void)hipGetLastError();
        if (before == device) before = -1;
    }
    ~OnDevice() { if (before >= 0) (void)hipSetDevice(before); }
};

// f(first, count) for ranges of a grid of `groups` workgroups: a launch holds fewer than 2^32 threads.
inline int64_t groups_of_a_launch(int threads) { return 4294967295ll / threads; }
template <typename F> void in_ranges(int64_t groups, int threads, F f) {
    const int64_t most = groups_of_a_launch(threads);
    for (int64_t first = 0; first < groups; first += most) f(first, (unsigned)std::min(most, groups - first));
}

inline int launched() { return hipGetLastError() == hipSuccess ? PCR_OK : PCR_E_DEVICE; }

// The type that a dtype stands for, as an argument of f.
template <typename F> void with_type(int dtype, F f) {
    if (dtype == PCR_FLOAT) f(float());
    else if (dtype == PCR_HALF) f((_Float16)0);
    else f((__bf16)0);
}

}  // namespace pcr
