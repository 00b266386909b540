// Host-side checks of the product, dropout and embedding entry points under
// AddressSanitizer and UBSan, without a GPU: refusals, the largest sizes, and the
// clean-up after a device call that fails.  The passes are replaced by stubs.
// Exit status 0 = every check held.
#include <stdio.h>
#include <string.h>

#include "dd_layers.h"

namespace dd {
#define STUB return hipErrorNoDevice
size_t product_work(int64_t m, int64_t n, int64_t k, bool) { return k > 1000 ? (size_t)m * (size_t)n * 8 : 0; }
bool product_fits(int64_t m, int64_t n, int64_t, bool) { return m < (1 << 30) && n < (1 << 30); }
hipError_t launch_product(const Product &, void *, hipStream_t) { STUB; }
bool goes_together(const Product &dw, const Product &) { return dw.m < 64; }
hipError_t launch_together(const Product &, const Product &, hipStream_t) { STUB; }
bool small_gradients(int64_t rows, int64_t, int64_t, bool) { return rows < 64; }
size_t padded_size(int64_t rows, int64_t cols) { return (size_t)rows * (size_t)cols * 2; }
size_t pad_rows(const void *&, int64_t &, int64_t rows, int64_t cols, void *, PadRows *r) {
    *r = PadRows{};
    return padded_size(rows, cols);
}
bool few_rows(int64_t, int64_t) { return true; }
bool loads_directly(const void *, int64_t, bool, int64_t, int64_t) { return false; }
size_t product_need(const Product &p) { return product_work(p.m, p.n, p.k, true); }
size_t grad_copies_work(int64_t rows, int64_t k, int64_t n) { return n % 8 && rows > 64 ? (size_t)(rows * (n + k) + k * n) * 2 : 0; }
GradCopies grad_copies(int64_t rows, int64_t k, int64_t n, bool, const GradCopies &needed) { return grad_copies_work(rows, k, n) ? needed : GradCopies{}; }
hipError_t launch_pad_rows(const PadRows &, const PadRows &, const PadRows &, const FewSums &, hipStream_t) { STUB; }
size_t column_sum_work(int64_t, int64_t cols) { return (size_t)cols * 4; }
hipError_t launch_column_sum(const void *, int64_t, int64_t, int64_t, int32_t, void *, int32_t, void *, hipStream_t) { STUB; }
hipError_t launch_act_grad(const dd_act_grad_args &, hipStream_t) { STUB; }
hipError_t launch_dropout(const dd_dropout_args &, hipStream_t) { STUB; }
hipError_t launch_embed(const dd_embed_args &, hipStream_t) { STUB; }
size_t embed_grad_work(int64_t tokens, int64_t, int64_t) { return (size_t)tokens * 16; }
hipError_t launch_embed_grad(const dd_embed_grad_args &, void *, hipStream_t) { STUB; }
// of the other passes (the API layer refers to them)
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
            fprintf(stderr, "FAILED: %s (line %d): %s\n", what, __LINE__, dd_last_error()); \
            g_bad++;                                                        \
        }                                                                   \
    } while (0)

static bool failed_on_device(dd_status st) { return (st == DD_EHIP || st == DD_ENOMEM) && dd_last_error()[0]; }

int main() {
    alignas(16) float room[64] = {};
    alignas(16) uint64_t state[4] = {};
    dd_linear_args l;
    memset(&l, 0, sizeof(l));
    l.rows = 2;
    l.k = l.n = 8;
    l.x_stride = l.w_stride = l.y_stride = 8;
    l.x = l.w = l.y = room;
    l.type = l.bias_type = DD_BF16;
    EXPECT(failed_on_device(dd_linear(&l, nullptr)), "product without a device");
    l.k = l.x_stride = 2000;
    EXPECT(failed_on_device(dd_linear(&l, nullptr)), "product without memory for its parts");
    l.work = room;
    EXPECT(failed_on_device(dd_linear(&l, nullptr)), "product with the caller's work");
    l.k = l.n = l.rows = (int64_t(1) << 31) - 1;
    l.x_stride = l.w_stride = l.y_stride = int64_t(1) << 29;
    EXPECT(dd_linear(&l, nullptr) == DD_EINVAL, "rows that overlap");
    l.y_stride = INT64_MAX;
    EXPECT(dd_linear(&l, nullptr) == DD_EINVAL, "the largest stride");
    l.x_stride = INT64_MIN;
    EXPECT(dd_linear(&l, nullptr) == DD_EINVAL, "the least stride");
    EXPECT(dd_linear_work(INT64_MAX, INT64_MAX, INT64_MAX) == 0 && dd_linear_grad_work(INT64_MIN, 1, 1) == 0, "work of no sizes");
    EXPECT(dd_linear_grad_work(2, 3, 5) == 20, "work");

    dd_linear_grad_args g;
    memset(&g, 0, sizeof(g));
    g.rows = 2;
    g.k = g.n = 8;
    g.dy_stride = g.x_stride = g.w_stride = g.dx_stride = g.dw_stride = 8;
    g.dy = g.x = g.w = room;
    g.type = g.bias_type = DD_F16;
    EXPECT(dd_linear_grad(&g, nullptr) == DD_OK, "nothing wanted");
    g.dx = room;
    EXPECT(failed_on_device(dd_linear_grad(&g, nullptr)), "dx without a device");
    g.dw = room;
    EXPECT(failed_on_device(dd_linear_grad(&g, nullptr)), "dw without a device");
    g.db = room;
    EXPECT(failed_on_device(dd_linear_grad(&g, nullptr)), "db without a device");
    g.rows = 0;
    g.work = room;
    EXPECT(failed_on_device(dd_linear_grad(&g, nullptr)), "dw of no rows");
    g.in_act = DD_ACT_GELU;
    EXPECT(dd_linear_grad(&g, nullptr) == DD_EINVAL, "in_act without in_z");
    g.in_act = DD_ACT_NONE;
    g.rows = 100;
    g.n = 81;
    g.dy_stride = g.w_stride = g.dw_stride = 81;
    g.work = nullptr;
    EXPECT(failed_on_device(dd_linear_grad(&g, nullptr)), "copies without a device");
    g.work = room;
    EXPECT(failed_on_device(dd_linear_grad(&g, nullptr)), "copies in given memory without a device");

    dd_act_grad_args a;
    memset(&a, 0, sizeof(a));
    a.rows = a.cols = 4;
    a.dy_stride = a.z_stride = a.dz_stride = 4;
    a.dy = a.z = a.dz = room;
    EXPECT(failed_on_device(dd_act_grad(&a, nullptr)), "activation gradient without a device");
    a.dz_stride = 3;
    EXPECT(dd_act_grad(&a, nullptr) == DD_EINVAL, "rows that overlap");

    dd_dropout_args d;
    memset(&d, 0, sizeof(d));
    d.rows = d.cols = 4;
    d.x_stride = d.out_stride = 4;
    d.x = d.out = room;
    d.d_state = state;
    d.d_used = state + 2;
    EXPECT(failed_on_device(dd_dropout(&d, nullptr)), "dropout without a device");
    d.d_used = state;
    EXPECT(dd_dropout(&d, nullptr) == DD_EINVAL, "used is state");

    dd_embed_args e;
    memset(&e, 0, sizeof(e));
    e.tokens = e.vocab = e.cols = 4;
    e.table_stride = e.out_stride = 4;
    e.ids = e.table = e.out = room;
    e.id_bytes = 8;
    EXPECT(failed_on_device(dd_embed(&e, nullptr)), "lookup without a device");
    dd_embed_grad_args b;
    memset(&b, 0, sizeof(b));
    b.tokens = b.vocab = b.cols = 4;
    b.dy_stride = b.dtable_stride = 4;
    b.ids = b.dy = b.dtable = room;
    b.id_bytes = 4;
    b.pad = 3;
    EXPECT(failed_on_device(dd_embed_grad(&b, nullptr)), "gradient without memory");
    b.work = room;
    EXPECT(failed_on_device(dd_embed_grad(&b, nullptr)), "gradient without a device");
    b.pad = 4;
    EXPECT(dd_embed_grad(&b, nullptr) == DD_EINVAL, "pad is no row");
    EXPECT(dd_embed_grad_work(int64_t(1) << 28, 4, 4) == 0 && dd_embed_grad_work(3, 4, 4) == 48, "work");
    if (g_bad == 0) printf("ALL OK\n");
    return g_bad ? 1 : 0;
}
