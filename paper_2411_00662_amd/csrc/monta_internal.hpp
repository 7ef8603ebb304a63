// What the entry points of all translation units share on the host: the checked problem statement, launch timing and
// the last HIP error.  monta.hip defines the functions; nothing here is visible outside the library.
#pragma once

#include "monta.h"

#include <hip/hip_runtime.h>

#include <atomic>

#include "monta_device.hpp"

#pragma GCC visibility push(hidden)
namespace monta {

// A monta_cfg that has passed the checks of every entry point.
struct Call {
    Shape s;
    int64_t max_rows;      // rows of STAGE, FINAL and the experts' output
    int64_t kept_bound;    // rows that can be kept
    int64_t row_bytes;     // of an activation row
    int64_t ws_bytes;
    int H;
    bool bf16;
    PlanPtrs p;            // tables of the workspace, if the call has one
};
int open_call(const monta_cfg *cfg, const void *ws, Call *out);

// The rows of each expert that a call works on, and nothing else of its arguments: slice = -1, its whole kept segment
// [offsets[e], offsets[e] + kept[e]), or the part of it filled by the slice's units, which starts at unit_base[first unit
// of the slice][e] and ends where the next slice's starts.
void expert_ranges(const Shape &s, const PlanPtrs &p, int slice, ExpertArgs *a);
int64_t slice_kept_bound(const Shape &s, int64_t kept_bound, int slice);

// Notes the error for monta_last_hip_error() and clears it.
int hip_failed(hipError_t e);
#define MONTA_HIP_TRY(expr)                                              \
    do {                                                                 \
        const hipError_t e__ = (expr);                                   \
        if (e__ != hipSuccess) return monta::hip_failed(e__);            \
    } while (0)

// Event profiling of the launches between its construction and its end.
struct LaunchTimer {
    hipStream_t st;
    int kid;
    hipEvent_t a = nullptr;
    bool on;
    LaunchTimer(int kid_, hipStream_t st_);
    ~LaunchTimer();
    LaunchTimer(const LaunchTimer &) = delete;
    LaunchTimer &operator=(const LaunchTimer &) = delete;
};

inline bool misaligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

// Do the bytes [a, a + na) and [b, b + nb) share any?
inline bool overlap(const void *a, int64_t na, const void *b, int64_t nb)
{
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
    return pa < pb + (uintptr_t)nb && pb < pa + (uintptr_t)na;
}

// Does HIP launch that many workgroups?  A dimension has fewer than 2^32 threads; of a greater number it launches the low 32 bits' worth
// and reports no error.
inline bool launchable(int64_t workgroups, int threads) { return workgroups < (1ll << 32) / threads; }

// Dynamic LDS above the default limit has to be asked for once per kernel and device.
struct LdsOptIn {
    std::atomic<int> done[64];
};

inline int opt_in_lds(const void *kernel, int bytes, LdsOptIn &state)
{
    int dev = 0;
    MONTA_HIP_TRY(hipGetDevice(&dev));
    if (dev < 0 || dev >= 64) return MONTA_ERR_UNSUPPORTED;
    if (!state.done[dev].load()) {
        MONTA_HIP_TRY(hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
        state.done[dev].store(1);
    }
    return MONTA_OK;
}

}  // namespace monta
#pragma GCC visibility pop
