// The library's workspace and the lease that hands it from call to call (host side).
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>
#include <mutex>

namespace nt {

// Workspace of the k splits (convolution, skinny GEMM), of the copies and the unfolded input of a convolution, and of attention whose
// keys are shared out over programs: one allocation
// per device, made by the first call on that device that needs it and kept until the process ends (never freed or moved, so work
// in flight never loses it).  It is cut into lanes, one of kSplitWsMax bytes and kSmallLanes of kSmallLane bytes for what fits
// those, so that calls on a few streams overlap as calls without workspace do.  A call holds a lane through a WorkspaceLease from
// before its first launch that touches it until after its last: the lease serialises host threads (a mutex) and streams (an event
// recorded behind the last consumer, which a call on any other stream makes its stream wait for before its own first launch), so
// calls that meet on one lane queue up instead of racing.  A stream keeps to the small lane it has used before, a new one takes
// the lane that has not been taken for the longest time.  (Two streams of (2,64,56,56)*(64,64,3,3) from two threads, us a call: 30
// on one lane, 14; alternating (4,256,14,14)*(256,256,3,3) 32 and 19.)
// Calls captured into a graph never touch those lanes or their events: a replay takes no lease, so nothing would order it against
// the calls around it.  They share an allocation of their own (kSplitWsMax bytes, made by the first that needs it); within a
// capture the event between two streams becomes an edge of the graph, and replays that overlap each other are the caller's to avoid.
// The event carries no system-scope fence: it only orders kernels of one device, and what it orders is the last consumer's reads
// before the next caller's writes (a consumer's input left the writer's caches at the launch boundary between the two).  The
// fence cost every call 2 us on the device (the paper's conv task 29.5 -> 27.6 us).
constexpr size_t kSplitWsMax = 256u << 20, kSmallLane = 32u << 20;
constexpr int kSmallLanes = 3;

// the capture (a number above 0) that work on the stream goes into, 0: none
inline unsigned long long capture_of(hipStream_t stream)
{
    hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
    unsigned long long id = 0;
    if (hipStreamGetCaptureInfo(stream, &st, &id) != hipSuccess) { (void)hipGetLastError(); return ~0ull; }
    return st == hipStreamCaptureStatusNone ? 0 : id;
}

class WorkspaceLease {
public:
    WorkspaceLease() = default;
    WorkspaceLease(const WorkspaceLease &) = delete;
    WorkspaceLease &operator=(const WorkspaceLease &) = delete;
    // nullptr: more than the workspace holds, no memory, or no device -- the caller then runs without it
    void *acquire(size_t bytes, hipStream_t stream)
    {
        int dev = 0;
        if (lane_ || bytes > kSplitWsMax || hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return nullptr;
        Device &d = table()[dev];
        const unsigned long long capture = capture_of(stream);
        if (capture == ~0ull) return nullptr;
        if (!(capture ? ready_for_captures(d) : ready(d))) return nullptr;
        Lane *w = capture ? &d.captures : bytes <= kSmallLane ? small_lane(d, stream) : &d.lane[0];
        w->mu.lock();
        // (an event recorded in another capture says nothing about this one)
        if (w->used && w->last != stream && w->capture == capture && (!w->marked || hipStreamWaitEvent(stream, w->done, 0) != hipSuccess)) {
            (void)hipGetLastError();
            w->mu.unlock();
            return nullptr;
        }
        lane_ = w;
        stream_ = stream;
        w->capture = capture;
        return w->p;
    }
    ~WorkspaceLease()
    {
        if (!lane_) return;
        lane_->last = stream_;
        lane_->used = lane_->marked = hipEventRecord(lane_->done, stream_) == hipSuccess;
        if (!lane_->marked) {
            // without the marker a later call on another stream could not wait for this one's work: wait for it here (in a capture,
            // where there is nothing to wait for yet, such a call runs without the workspace)
            (void)hipGetLastError();
            if (lane_->capture) lane_->used = true;
            else (void)hipStreamSynchronize(stream_);
        }
        lane_->mu.unlock();
    }

private:
    // (owner and stamp -- who was given the lane last, and when -- under the device's mutex, the rest under the lane's)
    struct Lane {
        void *p = nullptr;
        hipEvent_t done = nullptr;
        hipStream_t last = nullptr, owner = nullptr;
        bool used = false, marked = false;
        uint64_t stamp = 0;
        unsigned long long capture = 0;
        std::mutex mu;
    };
    struct Device { Lane lane[1 + kSmallLanes], captures; void *p = nullptr; uint64_t clock = 0; std::mutex mu; };
    static Device *table() { static Device t[64]; return t; }

    // the device's allocation, made if need be
    static bool ready(Device &d)
    {
        std::lock_guard<std::mutex> lock(d.mu);
        if (d.p) return true;
        void *p = nullptr;
        hipEvent_t ev[1 + kSmallLanes] = {};
        bool ok = hipMalloc(&p, kSplitWsMax + kSmallLanes * kSmallLane) == hipSuccess;
        for (hipEvent_t &e : ev) ok = ok && hipEventCreateWithFlags(&e, hipEventDisableTiming | hipEventDisableSystemFence) == hipSuccess;
        if (!ok) {
            (void)hipGetLastError();
            for (hipEvent_t e : ev)
                if (e) (void)hipEventDestroy(e);
            if (p) (void)hipFree(p);
            return false;
        }
        for (int i = 0; i <= kSmallLanes; ++i) {
            d.lane[i].p = (char *)p + (i ? kSplitWsMax + (size_t)(i - 1) * kSmallLane : 0);
            d.lane[i].done = ev[i];
        }
        d.p = p;
        return true;
    }
    // ... and the captured calls', which a thread in relaxed mode may make during a capture
    static bool ready_for_captures(Device &d)
    {
        std::lock_guard<std::mutex> lock(d.mu);
        if (d.captures.p) return true;
        hipStreamCaptureMode mode = hipStreamCaptureModeRelaxed;
        if (hipThreadExchangeStreamCaptureMode(&mode) != hipSuccess) { (void)hipGetLastError(); return false; }
        void *p = nullptr;
        bool ok = hipMalloc(&p, kSplitWsMax) == hipSuccess;
        ok = ok && hipEventCreateWithFlags(&d.captures.done, hipEventDisableTiming | hipEventDisableSystemFence) == hipSuccess;
        if (!ok) (void)hipGetLastError();
        if (!ok && p) (void)hipFree(p);
        (void)hipThreadExchangeStreamCaptureMode(&mode);
        if (ok) d.captures.p = p;
        return ok;
    }
    // the small lane of this stream
    static Lane *small_lane(Device &d, hipStream_t stream)
    {
        std::lock_guard<std::mutex> lock(d.mu);
        Lane *w = &d.lane[1];
        for (int i = 1; i <= kSmallLanes; ++i) {
            Lane &l = d.lane[i];
            if (l.stamp && l.owner == stream) { w = &l; break; }
            if (l.stamp < w->stamp) w = &l;
        }
        w->owner = stream;
        w->stamp = ++d.clock;
        return w;
    }
    Lane *lane_ = nullptr;
    hipStream_t stream_ = nullptr;
};

}  // namespace nt
