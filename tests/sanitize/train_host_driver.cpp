// Host-side checks of the weight update's and the norm's entry points under
// AddressSanitizer and UBSan, without a GPU: refusals, and the clean-up after a
// device call that fails.  The passes are replaced by stubs that are never
// reached.  Exit status 0 = every check held.
#include <stdio.h>
#include <string.h>

#include <thread>
#include <vector>

#include "dd_train.h"

namespace dd {
#define STUB return hipErrorNoDevice
hipError_t launch_tensor_chunks(const TensorPlace *, int, const dd_tensors *, hipStream_t) { STUB; }
hipError_t launch_grad_norm(const dd_tensors *, double, const float *, float *, hipStream_t) { STUB; }
hipError_t launch_grad_clip(const dd_tensors *, const dd_tensors *, const float *, hipStream_t) { STUB; }
hipError_t launch_adam(const dd_tensors *, int64_t *, const float *, const AdamParams &, hipStream_t) { STUB; }
size_t rms_grad_work(int64_t, int64_t cols) { return (size_t)cols * 4; }
hipError_t launch_rms_norm(const RmsArgs &, hipStream_t) { STUB; }
hipError_t launch_rms_norm_grad(const RmsGradArgs &, float *, hipStream_t) { STUB; }
// of the simulation's passes (the API layer refers to them)
dd_status levelize_device(const dd_graph *, uint64_t, int32_t, dd_sched *, hipStream_t, char *, size_t) { return DD_EHIP; }
hipError_t launch_simulate(const dd_graph *, const dd_sched *, const dd_variants *, int64_t *, int64_t *, int64_t *, int,
                           hipStream_t) { STUB; }
hipError_t simulate_noalloc(const dd_graph *, const dd_sched *, const dd_variants *, int64_t *, int64_t *, int64_t *,
                            hipStream_t, size_t *, size_t *) { STUB; }
int split_width(const dd_sched *, const dd_variants *) { return 0; }
hipError_t launch_split(const dd_graph *, const dd_sched *, const dd_variants *, int64_t *, int64_t *, int64_t *, int,
                        hipStream_t) { STUB; }
void split_set_polls(int32_t) {}
hipError_t launch_breakdown(const dd_graph *, const dd_variants *, const uint8_t *, const int64_t *, const int64_t *,
                            int64_t *, hipStream_t) { STUB; }
hipError_t build_event_lists(const dd_graph *, EventLists *, hipStream_t) { STUB; }
void free_event_lists(EventLists *, hipStream_t) {}
hipError_t launch_sim_event(const dd_graph *, const EventLists &, const dd_variants *, int32_t, const uint8_t *,
                            const int32_t *, int32_t *, int64_t *, uint32_t **, int64_t *, int64_t *, int64_t *, uint32_t *,
                            hipStream_t) { STUB; }
}  // namespace dd

static int g_bad = 0;
#define EXPECT(cond, what)                                                  \
    do {                                                                    \
        if (!(cond)) {                                                      \
            fprintf(stderr, "FAILED: %s (line %d)\n", what, __LINE__);      \
            g_bad++;                                                        \
        }                                                                   \
    } while (0)

static bool failed_on_device(dd_status st) { return (st == DD_EHIP || st == DD_ENOMEM) && dd_last_error()[0]; }

int main() {
    alignas(16) float room[64] = {};
    dd_tensors *t = (dd_tensors *)0x1;
    // lists of many sizes get as far as the device, and are cleaned up
    for (int count : {0, 1, 3, 1000}) {
        std::vector<dd_tensor> v((size_t)count);
        for (int i = 0; i < count; i++) {
            memset(&v[i], 0, sizeof(dd_tensor));
            v[i].grad = v[i].param = v[i].m = v[i].v = room;
            v[i].n = i % 7 ? (int64_t)i * 10007 : 0;
        }
        EXPECT(failed_on_device(dd_tensors_load(count, v.data(), nullptr, &t)) && t == nullptr, "load without a device");
        t = (dd_tensors *)0x1;
    }
    dd_tensor one;
    memset(&one, 0, sizeof(one));
    one.grad = room;
    one.n = 5;
    EXPECT(dd_tensors_load(1, &one, nullptr, nullptr) == DD_EINVAL, "out NULL");
    EXPECT(dd_tensors_load(-1, &one, nullptr, &t) == DD_EINVAL && t == nullptr, "count < 0");
    EXPECT(dd_tensors_load(1, nullptr, nullptr, &t) == DD_EINVAL, "t NULL");
    std::vector<dd_tensor> mixed(2, one);
    mixed[1].param = mixed[1].m = mixed[1].v = room;
    EXPECT(dd_tensors_load(2, mixed.data(), nullptr, &t) == DD_EINVAL && strstr(dd_last_error(), "some tensors"), "mixed list");
    mixed.assign(2, one);
    mixed[0].n = mixed[1].n = (int64_t(1) << 61) + 5;
    EXPECT(dd_tensors_load(2, mixed.data(), nullptr, &t) == DD_EINVAL, "total past 2^62");
    dd_tensors_free(nullptr);
    EXPECT(dd_grad_norm(nullptr, 1.0f, nullptr, room, nullptr) == DD_EINVAL, "norm of NULL");
    EXPECT(dd_grad_clip(nullptr, nullptr, room, nullptr) == DD_EINVAL, "clip of NULL");
    int64_t step = 0;
    EXPECT(dd_adam_step(nullptr, &step, nullptr, 1e-3, 0.9, 0.999, 1e-8, 0.0, 1, nullptr) == DD_EINVAL, "step of NULL");

    dd_rms_norm_args n;
    memset(&n, 0, sizeof(n));
    n.rows = 2;
    n.cols = 8;
    n.x_stride = n.out_stride = 8;
    n.x = n.out = room;
    EXPECT(failed_on_device(dd_rms_norm(&n, nullptr)), "norm without a device");
    n.out_stride = 7;
    EXPECT(dd_rms_norm(&n, nullptr) == DD_EINVAL, "rows that overlap");
    n.rows = 0;
    EXPECT(dd_rms_norm(&n, nullptr) == DD_OK, "no rows");
    EXPECT(dd_rms_norm(nullptr, nullptr) == DD_EINVAL, "args NULL");

    dd_rms_norm_grad_args g;
    memset(&g, 0, sizeof(g));
    g.rows = 2;
    g.cols = 8;
    g.dy_stride = g.h_stride = g.dx_stride = 8;
    g.dy = g.h = g.dx = room;
    g.rstd = room;
    EXPECT(failed_on_device(dd_rms_norm_grad(&g, nullptr)), "gradient without a device");
    g.dw = room;
    EXPECT(failed_on_device(dd_rms_norm_grad(&g, nullptr)), "gradient without memory for its sums");
    g.work = room;
    EXPECT(failed_on_device(dd_rms_norm_grad(&g, nullptr)), "gradient with the caller's work");
    g.rstd = nullptr;
    EXPECT(dd_rms_norm_grad(&g, nullptr) == DD_EINVAL, "rstd NULL");
    EXPECT(dd_rms_norm_grad_work(-1, 1) == 0 && dd_rms_norm_grad_work(3, 5) == 20, "work");

    // error messages are per host thread
    EXPECT(dd_rms_norm(nullptr, nullptr) == DD_EINVAL, "args NULL");
    char mine[512];
    snprintf(mine, sizeof(mine), "%s", dd_last_error());
    std::thread other([] { (void)dd_grad_norm(nullptr, 0.0f, nullptr, nullptr, nullptr); });
    other.join();
    EXPECT(strcmp(mine, dd_last_error()) == 0, "thread-local message");
    if (g_bad == 0) printf("ALL OK\n");
    return g_bad ? 1 : 0;
}
