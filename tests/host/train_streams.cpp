// The order that calls on a list of tensors are put in over several streams,
// without a GPU: HIP's events are replaced by a record of what each stream has
// to run after.  Exit status 0 = every check held.
#include <stdio.h>
#include <stdlib.h>

#include <map>
#include <random>
#include <set>
#include <vector>

#include "dd_train.h"

typedef std::set<int> Seen;                        // pieces of work, by number
static std::map<hipStream_t, Seen> seen;           // what runs before the next work of a stream
struct Event {
    Seen before;
    bool captured = false;
};
static int events = 0, works = 0, bad = 0;
static hipStream_t capturing = nullptr;

#define EXPECT(c)                                                         \
    do {                                                                  \
        if (!(c)) {                                                       \
            fprintf(stderr, "FAILED: %s (line %d)\n", #c, __LINE__);      \
            bad++;                                                        \
        }                                                                 \
    } while (0)

static int work_on(hipStream_t s) {
    seen[s].insert(works);
    return works++;
}
static bool after(const Seen &a, const Seen &b) {  // a holds all of b
    for (int w : b)
        if (!a.count(w)) return false;
    return true;
}

extern "C" {
hipError_t hipEventCreateWithFlags(hipEvent_t *e, unsigned) {
    events++;
    *e = reinterpret_cast<hipEvent_t>(new Event);
    return hipSuccess;
}
hipError_t hipEventDestroy(hipEvent_t e) {
    events--;
    delete reinterpret_cast<Event *>(e);
    return hipSuccess;
}
hipError_t hipEventRecord(hipEvent_t e, hipStream_t s) {
    Event *v = reinterpret_cast<Event *>(e);
    v->before = seen[s];
    v->captured = s == capturing && capturing;
    return hipSuccess;
}
hipError_t hipStreamWaitEvent(hipStream_t s, hipEvent_t e, unsigned) {
    Event *v = reinterpret_cast<Event *>(e);
    EXPECT(v->captured == (s == capturing && capturing));    // (else HIP refuses it, and the capture fails)
    seen[s].insert(v->before.begin(), v->before.end());
    return hipSuccess;
}
hipError_t hipStreamIsCapturing(hipStream_t s, hipStreamCaptureStatus *st) {
    *st = s == capturing && capturing ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone;
    return hipSuccess;
}
hipError_t hipGetDevice(int *d) {
    *d = 0;
    return hipSuccess;
}
hipError_t hipMalloc(void **p, size_t n) {
    *p = malloc(n);
    return hipSuccess;
}
hipError_t hipMemcpyAsync(void *, const void *, size_t, hipMemcpyKind, hipStream_t) { return hipSuccess; }
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
const char *hipGetErrorString(hipError_t) { return "error"; }
}

namespace dd {
hipError_t launch_tensor_chunks(const TensorPlace *, int, const dd_tensors *, hipStream_t) { return hipSuccess; }
hipError_t launch_grad_norm(const dd_tensors *, double, const float *, float *, hipStream_t s) {
    work_on(s);
    return hipSuccess;
}
hipError_t launch_grad_clip(const dd_tensors *, const dd_tensors *, const float *, hipStream_t s) {
    work_on(s);
    return hipSuccess;
}
hipError_t launch_adam(const dd_tensors *, int64_t *, const float *, const AdamParams &, hipStream_t s) {
    work_on(s);
    return hipSuccess;
}
}  // namespace dd

static hipStream_t stream(int i) { return reinterpret_cast<hipStream_t>((uintptr_t)(0x100 * i)); }
static float room[16];
static int64_t step;

static dd_tensors *load(hipStream_t s) {
    dd_tensor t = {};
    t.grad = t.param = t.m = t.v = room;
    t.n = 16;
    dd_tensors *x = nullptr;
    EXPECT(dd_tensors_load(1, &t, s, &x) == DD_OK && x);
    return x;
}
static dd_status norm(dd_tensors *t, hipStream_t s) { return dd_grad_norm(t, 1.0f, nullptr, room, s); }
static dd_status adam(dd_tensors *t, hipStream_t s) {
    return dd_adam_step(t, &step, nullptr, 1e-3, 0.9, 0.999, 1e-8, 0.0, 1, s);
}

int main() {
    // any mixture of streams: every call that uses the list's working memory
    // after all before it, and the list's own stream after all calls when it
    // is freed there
    std::mt19937 rng(1);
    for (int round = 0; round < 200; round++) {
        seen.clear();
        const hipStream_t own = stream((int)(rng() % 4));
        dd_tensors *t = load(own);
        Seen turns, all;
        for (int k = 0; k < 30; k++) {
            const hipStream_t s = stream((int)(rng() % 4));
            const int what = (int)(rng() % 4), before = works;
            if (what == 0) EXPECT(norm(t, s) == DD_OK);
            else if (what == 1) EXPECT(adam(t, s) == DD_OK);
            else if (what == 2) EXPECT(dd_grad_clip(t, t, room, s) == DD_OK);
            else work_on(s);
            if (what < 2) {
                EXPECT(after(seen[s], turns));
                turns.insert(before);
            }
            if (what < 3) all.insert(before);
        }
        dd_tensors_free(t);
        EXPECT(after(seen[own], all));
        EXPECT(events == 0);
    }

    // calls on one other stream: it and the list's stream go on independently
    seen.clear();
    const hipStream_t own = stream(1), side = stream(2), third = stream(3);
    dd_tensors *t = load(own);
    Seen unrelated, on_side;
    for (int k = 0; k < 5; k++) {
        unrelated.insert(work_on(own));
        on_side.insert(works);
        EXPECT(norm(t, side) == DD_OK);
        on_side.insert(works);
        EXPECT(adam(t, side) == DD_OK);
    }
    for (int w : unrelated) EXPECT(!seen[side].count(w));
    for (int w : on_side) EXPECT(!seen[own].count(w));
    EXPECT(norm(t, third) == DD_OK);                     // a third follows the second alone
    EXPECT(after(seen[third], on_side));
    for (int w : unrelated) EXPECT(!seen[third].count(w));
    EXPECT(norm(t, own) == DD_OK && after(seen[own], on_side));

    // a graph takes calls on the list's own stream, and clipping on any
    capturing = own;
    EXPECT(norm(t, own) == DD_OK && adam(t, own) == DD_OK);
    capturing = third;
    const int before = works;
    EXPECT(norm(t, third) == DD_EINVAL && adam(t, third) == DD_EINVAL && works == before);
    EXPECT(dd_grad_clip(t, t, room, third) == DD_OK && works == before + 1);
    capturing = nullptr;
    EXPECT(norm(t, own) == DD_OK && norm(t, side) == DD_OK);
    dd_tensors_free(t);
    EXPECT(events == 0);
    if (!bad) printf("ALL OK\n");
    return bad ? 1 : 0;
}
