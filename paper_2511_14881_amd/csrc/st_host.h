// Host-side pieces that the library's translation units share: the error text of a call, the guard at a C
// entry and the timing of launches.
#pragma once
#include "../../include/silvertorch.h"

#include <hip/hip_runtime.h>

#include <new>
#include <vector>

namespace st {

// Records the text that st_last_error() gives the calling thread, and returns the code.
int fail(int code, const char* fmt, ...);

// The C ABI never lets an exception out: host allocations that fail become ST_ENOMEM.
template <class F>
int guarded(F&& body)
{
    try {
        return body();
    } catch (const std::bad_alloc&) {
        return fail(ST_ENOMEM, "out of host memory");
    } catch (...) {
        return fail(ST_EINVAL, "unexpected failure in host code");
    }
}

#define ST_HIP(call)                                                                       \
    do {                                                                                   \
        hipError_t e_ = (call);                                                            \
        if (e_ != hipSuccess)                                                              \
            return st::fail(e_ == hipErrorOutOfMemory ? ST_ENOMEM : ST_EHIP,               \
                            "%s failed: %s (%s:%d)", #call, hipGetErrorString(e_),         \
                            __FILE__, __LINE__);                                           \
    } while (0)

// Optional per-kernel timing with HIP events recorded on the caller's stream around each launch
// (state of the calling thread: the thread that begins a measurement makes the calls and ends it).
struct Timing {
    bool on = false;
    std::vector<hipEvent_t> ev;  // pairs: [2i] before, [2i+1] after launch i
    std::vector<int> kind;       // 0 scan, 1 select, 2 rescue, 3 filter expressions
    size_t used = 0;             // launches recorded
    size_t dropped = 0;
};
extern thread_local Timing g_timing;

struct TimedLaunch {
    hipStream_t stream;
    bool active;
    size_t slot;
    TimedLaunch(int kind, hipStream_t s) : stream(s), active(false), slot(0)
    {
        if (!g_timing.on) return;
        if (2 * (g_timing.used + 1) > g_timing.ev.size()) { ++g_timing.dropped; return; }
        slot = g_timing.used++;
        g_timing.kind[slot] = kind;
        active = hipEventRecord(g_timing.ev[2 * slot], stream) == hipSuccess;
    }
    ~TimedLaunch()
    {
        if (active) (void)hipEventRecord(g_timing.ev[2 * slot + 1], stream);
    }
};

}  // namespace st
