// What the C entry points share: the last HIP error of a thread, the measurement hook around a launch, alignment.
#pragma once

#include "../../include/floe.h"

#include <hip/hip_runtime.h>

namespace floe {

inline thread_local int g_last_hip_error = 0;

inline int hip_fail(hipError_t e) {
    g_last_hip_error = (int)e;
    return FLOE_EHIP;
}

#define FLOE_HIP(call)                             \
    do {                                           \
        hipError_t e__ = (call);                   \
        if (e__ != hipSuccess) return hip_fail(e__); \
    } while (0)

// Optional measurement hook: when armed for kernel `id`, the next launches of that kernel are bracketed
// by the two events on the launch stream (see floe_profile_kernel in floe.h).
struct ProfileHook {
    int id = 0;
    hipEvent_t start = nullptr, stop = nullptr;
};
inline thread_local ProfileHook g_hook;

struct Bracket {
    bool on;
    hipStream_t st;
    Bracket(int id, hipStream_t s) : on(g_hook.id == id && g_hook.start && g_hook.stop), st(s) {
        if (on) (void)hipEventRecord(g_hook.start, st);
    }
    ~Bracket() {
        if (on) (void)hipEventRecord(g_hook.stop, st);
    }
};

#define FLOE_LAUNCH(id, stream, call) \
    do {                              \
        Bracket br__((id), (stream)); \
        FLOE_HIP(call);               \
    } while (0)

constexpr size_t kAlign = 256;
inline size_t align_up(size_t n) { return (n + kAlign - 1) / kAlign * kAlign; }
inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

}  // namespace floe
