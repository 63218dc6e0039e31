// Error state, argument checks and schedule overrides shared by the
// translation units that implement the C ABI.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

#include <atomic>
#include <cstdarg>
#include <cstdio>

#include "lce.h"

namespace lce {

// The message of the calling thread's last failure ("" after a success).  A
// plain array: setting it allocates nothing and cannot throw.
inline thread_local char g_error_text[512];

inline const char *last_error_text() { return g_error_text; }

__attribute__((format(printf, 2, 3))) inline lce_status fail(lce_status st, const char *fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_error_text, sizeof g_error_text, fmt, ap);
    va_end(ap);
    return st;
}

inline lce_status ok() {
    g_error_text[0] = 0;
    return LCE_OK;
}

inline lce_status check_launch(const char *what) {
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(LCE_EHIP, "%s: %s", what, hipGetErrorString(e));
    return ok();
}

// What the calling thread's last convolution or attention launched (lce_last_schedule).
inline thread_local const char *g_last_schedule = "";

inline bool aligned(const void *p, uintptr_t a) {
    return (reinterpret_cast<uintptr_t>(p) % a) == 0;
}

// Schedule overrides (lce_set_tuning): 0 = the library's own choice.  Each
// launch reads every value it uses once, with a relaxed atomic load, so a
// concurrent lce_set_tuning is never a data race (a launch sees the old or
// the new value).
inline std::atomic<int32_t> g_tuning[LCE_TUNE_COUNT];

inline int tuning(lce_tuning_key key) { return g_tuning[key].load(std::memory_order_relaxed); }

}  // namespace lce
