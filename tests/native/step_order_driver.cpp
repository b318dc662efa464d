// Which copies have to wait for a step's kernels (kvc_step_order.h): hand-worked sequences, and a random walk
// against a plain record of what was queued on every stream.
#include <stdio.h>
#include <stdlib.h>

#include <map>
#include <memory>

#include "kvc_step_order.h"

#define CHECK(x)                                          \
    do {                                                  \
        if (!(x)) {                                       \
            printf("FAILED line %d: %s\n", __LINE__, #x); \
            exit(1);                                      \
        }                                                 \
    } while (0)

// A copy on the stream: whether it waits; if so it was launched, and clears the mark.
static bool copy(KvcStepOrder &o, int dev, uint64_t stream, uint64_t capture = 0)
{
    const bool wait = o.pending(dev, stream, capture);
    if (wait)
        o.waited(dev, stream, capture);
    return wait;
}

int main()
{
    const uint64_t A = 0xA000, B = 0xB000;
    {
        KvcStepOrder o;
        CHECK(!copy(o, 0, A));
        o.step(0, A, 0);
        CHECK(!copy(o, 0, B));  // a copy on another stream neither waits ...
        CHECK(copy(o, 0, A));   // ... nor takes the mark away
        CHECK(!copy(o, 0, A));  // behind a copy that waited none has to
        o.step(0, A, 0);
        o.step(0, A, 0);
        CHECK(o.pending(0, A, 0));  // a launch that failed: the next copy still waits
        CHECK(copy(o, 0, A) && !copy(o, 0, A));
        o.step(1, A, 0);  // the same handle value on another device
        CHECK(!copy(o, 0, A) && copy(o, 1, A));
        o.step(0, 0, 0);  // the default stream under either of its names
        CHECK(copy(o, 0, KvcStepOrder::LEGACY) && !copy(o, 0, 0));
        o.step(0, KvcStepOrder::PER_THREAD, 0);  // one handle, a stream a thread
        CHECK(copy(o, 0, KvcStepOrder::PER_THREAD) && copy(o, 0, KvcStepOrder::PER_THREAD));
    }
    {
        KvcStepOrder o;
        o.step(0, A, 7);  // captured
        CHECK(copy(o, 0, A, 7) && copy(o, 0, B, 7) && copy(o, 0, A, 7));
        CHECK(!copy(o, 0, A) && !copy(o, 0, A, 8));
        o.step(0, A, 0);
        CHECK(!copy(o, 0, A, 9));  // a copy in a capture says nothing about the stream ...
        CHECK(copy(o, 0, A));      // ... whose next copy waits
        for (uint64_t c = 10; c < 200; ++c)
            o.step(0, A, c);
        for (uint64_t c = 10; c < 200; ++c)
            CHECK(copy(o, 0, A, c));
        CHECK(!copy(o, 0, A, 1000));
    }
    {
        auto o = std::make_unique<KvcStepOrder>();
        for (uint64_t s = 0; s < 1000; ++s)
            o->step(0, 0x1000 + s * 16, 0);
        for (uint64_t s = 0; s < 1000; ++s)
            CHECK(copy(*o, 0, 0x1000 + s * 16));  // more streams than there is room for: all wait
    }
    srand(1);
    for (int round = 0; round < 200; ++round) {
        KvcStepOrder o;
        std::map<uint64_t, bool> marked;  // the last thing queued on the stream that later kernels may overtake
        for (int i = 0; i < 2000; ++i) {
            const uint64_t s = 0x1000 + (uint64_t)(rand() % 40) * 16;
            if (rand() % 3 == 0) {
                o.step(0, s, 0);
                marked[s] = true;
            } else {
                CHECK(copy(o, 0, s) == marked[s]);
                marked[s] = false;
            }
        }
    }
    printf("ok\n");
    return 0;
}
