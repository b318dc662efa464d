// Which streams have a step's kernel (tokens, attention) in front of the next copy.
//
// Those kernels let later kernels of their stream in early, so a copy that would not wait for the kernel before
// it (pdl = 3) has to wait for them.  What is remembered is a matter of streams, not of handles: a step and the
// copy behind it may come from different handles, and copies on other streams change nothing.
//   - A stream is marked by a step's call and cleared by a copy that waited on it, once that has been launched.
//   - What is being captured goes by the capture: streams of one capture may depend on one another in ways that only
//     the graph knows, and what is captured has not run, so a capture that holds a step stays marked.
//   - A handle value that several streams share (the per-thread default stream) is never cleared.
//   - Where the table is full, all streams count as marked.  A stream that takes the handle of a destroyed one
//     inherits its mark.  Either costs a copy its overlap with the kernel before it, never a result.
#ifndef KVC_STEP_ORDER_H
#define KVC_STEP_ORDER_H

#include <stdint.h>

class KvcStepOrder {
public:
    // capture: the stream's capture id, 0 outside a capture
    void step(int device, uint64_t stream, uint64_t capture)
    {
        if (capture) {
            if (holds_capture(capture))
                return;
            const uint64_t old = captures_[next_capture_];
            captures_[next_capture_] = capture;
            next_capture_ = (next_capture_ + 1) % CAPTURES;
            if (old > forgotten_)
                forgotten_ = old;
            return;
        }
        if (full_ || find(device, stream) < used_)
            return;
        if (used_ == STREAMS) {
            full_ = true;
            return;
        }
        marks_[used_].device = device;
        marks_[used_].stream = stream;
        ++used_;
    }

    // Whether a copy has to wait for the kernel before it.
    bool pending(int device, uint64_t stream, uint64_t capture) const
    {
        if (capture)  // (ids ascend, so one that is no larger than a forgotten one may have been it)
            return capture <= forgotten_ || holds_capture(capture);
        return full_ || find(device, stream) < used_;
    }

    // A copy that waited was launched.
    void waited(int device, uint64_t stream, uint64_t capture)
    {
        if (capture || stream == PER_THREAD)
            return;
        const uint32_t i = find(device, stream);
        if (i < used_)
            marks_[i] = marks_[--used_];
    }

    static constexpr uint64_t LEGACY = 1, PER_THREAD = 2;  // the runtime's handles of its default streams

private:
    static constexpr uint32_t STREAMS = 256, CAPTURES = 32;
    struct Mark {
        int device;
        uint64_t stream;
    };
    Mark marks_[STREAMS];
    uint32_t used_ = 0, next_capture_ = 0;
    bool full_ = false;
    uint64_t captures_[CAPTURES] = {}, forgotten_ = 0;

    static uint64_t name(uint64_t stream) { return stream ? stream : LEGACY; }
    uint32_t find(int device, uint64_t stream) const
    {
        uint32_t i = 0;
        while (i < used_ && (marks_[i].device != device || name(marks_[i].stream) != name(stream)))
            ++i;
        return i;
    }
    bool holds_capture(uint64_t capture) const
    {
        for (uint64_t c : captures_)
            if (c == capture)
                return true;
        return false;
    }
};

#endif
