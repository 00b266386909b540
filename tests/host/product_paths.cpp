// Which kernels a product and its gradients go to, without a GPU: the argument checks, the plan and the working memory
// are the library's own, launches are written down.
//
//   product_paths          reads calls, "fwd" or "grad", rows, k, n, pad (elements between rows), turned, type
//                          (0: bf16, 1: f16), wanted (1 dx, 2 dw, 4 db), a line each; writes a line for each
//   product_paths draw N   N drawn calls: what is loaded to LDS directly lies within the reach of a load's
//                          offset, all that is written to working memory within the bytes that the call needs and its sizes ask for, and a
//                          gradient alone is cut as it is beside the others where operands load directly
#include "k_linear.hip"

#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <random>
#include <string>
#include <vector>

#include "dd_layers.hip"

using dd::Plan;
using dd::Product;

static char *const kWork = reinterpret_cast<char *>(uintptr_t(1) << 50);       // (never touched)
static size_t room = 0, need = 0, used = 0;       // by sizes, of the call, and written
static std::string said;
static int bad = 0;
static const void *y_at, *dx_at, *dw_at, *given[3];

#define EXPECT(c)                                                                    \
    do {                                                                             \
        if (!(c)) {                                                                  \
            fprintf(stderr, "FAILED: %s (line %d), %s\n", #c, __LINE__, said.c_str()); \
            bad++;                                                                   \
        }                                                                            \
    } while (0)

static void uses(const void *p, size_t bytes) {
    const size_t end = (size_t)(static_cast<const char *>(p) - kWork) + bytes;
    if (end > used) used = end;
}
// a load to LDS has 64 lines by sums, or a tile's rows, below 2 GiB
static void check_reach(int64_t stride, bool by_rows, int64_t lines, int64_t width) {
    EXPECT(((lines - 1) * stride + (by_rows ? 64 : width)) * 2 <= int64_t(1) << 31);
}
// tile and parts of dx and dw, as launched last
struct Cut {
    int tile, splits;
    bool operator==(const Cut &o) const { return tile == o.tile && splits == o.splits; }
};
static Cut cut_dx, cut_dw;
static char operand(const void *p) {
    for (const void *g : given)
        if (p == g) return 'g';
    return 'c';         // (copied)
}
static void say(const Product &a, const Plan &p, bool direct, const char *how) {
    char line[200];
    const char *what = a.e.out == y_at ? "y" : a.e.out == dx_at ? "dx" : "dw";
    const int64_t tiles = (int64_t)p.tm * p.tn * p.splits;
    (a.e.out == dx_at ? cut_dx : cut_dw) = Cut{p.tile, p.splits};
    snprintf(line, sizeof(line), " %s:%d%s%s%s%c%c%s", what, p.tile, how, p.splits > 1 ? "/cut" : "", direct ? "/direct" : "/any", operand(a.p), operand(a.q),
             tiles > dd::kUnits ? "/rounds" : "");
    said += line;
}
static void check_direct(const Product &a, const Plan &p) {
    const int64_t rows = p.tile, cols = p.tile <= 64 ? 64 : p.tile;
    if (a.k == 0) return;
    check_reach(a.p_stride, a.p_by_rows, a.p_by_rows ? (rows < a.m ? rows : a.m) : (a.k < 64 ? a.k : 64), rows);
    check_reach(a.q_stride, a.q_by_rows, a.q_by_rows ? (cols < a.n ? cols : a.n) : (a.k < 64 ? a.k : 64), cols);
}

namespace dd {
template <class T, bool DIRECT>
void launch_tiles(const Product &a, const Plan &p, float *part, hipStream_t) {
    if (p.splits > 1) uses(part, (size_t)p.splits * (size_t)a.m * (size_t)a.n * sizeof(float));
    say(a, p, DIRECT, "");
    if (DIRECT) check_direct(a, p);
}
template void launch_tiles<bf16_t, true>(const Product &, const Plan &, float *, hipStream_t);
template void launch_tiles<bf16_t, false>(const Product &, const Plan &, float *, hipStream_t);
template void launch_tiles<f16_t, true>(const Product &, const Plan &, float *, hipStream_t);
template void launch_tiles<f16_t, false>(const Product &, const Plan &, float *, hipStream_t);
template <class T>
void launch_two(const Product &a, const Product &b, hipStream_t) {
    for (const Product *x : {&a, &b}) {
        const Plan p{64, (int)((x->m + 63) / 64), (int)((x->n + 63) / 64), 1, 0, 0.0};
        say(*x, p, true, "two");
        check_direct(*x, p);
    }
}
template void launch_two<bf16_t>(const Product &, const Product &, hipStream_t);
template void launch_two<f16_t>(const Product &, const Product &, hipStream_t);

dd_status fail(dd_status s, const char *, ...) { return s; }
dd_status hip_fail(hipError_t, const char *) { return DD_EHIP; }
void no_error() {}
hipError_t dalloc(void **p, size_t, hipStream_t) { *p = nullptr; return hipErrorOutOfMemory; }
void dfree(void *, hipStream_t) {}
hipError_t launch_dropout(const dd_dropout_args &, hipStream_t) { return hipSuccess; }
hipError_t launch_embed(const dd_embed_args &, hipStream_t) { return hipSuccess; }
size_t embed_grad_work(int64_t, int64_t, int64_t) { return 0; }
hipError_t launch_embed_grad(const dd_embed_grad_args &, void *, hipStream_t) { return hipSuccess; }
}  // namespace dd

extern "C" {
void **__hipRegisterFatBinary(const void *) { static void *h; return &h; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *, char *, const char *, unsigned, void *, void *, void *, void *, int *) {}
hipError_t __hipPushCallConfiguration(dim3, dim3, size_t, hipStream_t) { return hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3 *, dim3 *, size_t *, hipStream_t *) { return hipSuccess; }
hipError_t hipLaunchKernel(const void *f, dim3, dim3, void **args, size_t, hipStream_t) {
    if (f == (const void *)dd::k_pad_rows)
        for (int i = 0; i < 3; i++) {
            const dd::PadRows &r = *static_cast<const dd::PadRows *>(args[i]);
            if (r.rows) uses(r.to, dd::padded_size(r.rows, r.cols));
        }
    if (f == (const void *)dd::k_column_sum<dd::bf16_t> || f == (const void *)dd::k_column_sum<dd::f16_t>) {
        const size_t bytes = dd::column_sum_work(*static_cast<int64_t *>(args[2]), *static_cast<int64_t *>(args[3]));
        if (bytes) uses(*static_cast<float **>(args[7]), bytes);
    }
    return hipSuccess;
}
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus *s) { *s = hipStreamCaptureStatusNone; return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
const char *hipGetErrorString(hipError_t) { return "error"; }
}

struct Call {
    bool grad;
    long long rows, k, n, pad;
    int turned, type, wanted;
};

// odd: operand i lies 2 bytes further than 16 bytes divide, if its bit is set
static dd_status run(const Call &c, unsigned odd = 0) {
    auto at = [odd](int i) { return reinterpret_cast<char *>((uintptr_t(1) << 52) + ((uintptr_t)i << 48) + (odd >> i & 1 ? 2 : 0)); };
    const int64_t wr = c.turned ? c.n : c.k, wc = c.turned ? c.k : c.n;
    char line[200];
    snprintf(line, sizeof(line), "%s %lld %lld %lld pad %lld turned %d wanted %d:", c.grad ? "grad" : "fwd", c.rows, c.k, c.n, c.pad, c.turned, c.wanted);
    used = 0;
    said = line;
    given[0] = at(0);
    given[1] = at(1);
    given[2] = at(2);
    y_at = at(3);
    dx_at = at(4);
    dw_at = at(5);
    if (!c.grad) {
        dd_linear_args a;
        memset(&a, 0, sizeof(a));
        a.rows = c.rows;
        a.k = c.k;
        a.n = c.n;
        a.x_stride = c.k + c.pad;
        a.w_stride = wc + c.pad;
        a.y_stride = c.n;
        a.x = at(0);
        a.w = at(1);
        a.y = at(3);
        a.work = kWork;
        a.type = a.bias_type = c.type ? DD_F16 : DD_BF16;
        a.turned = c.turned;
        room = dd_linear_work(c.rows, c.k, c.n);
        need = dd_linear_need(&a);
        return dd_linear(&a, nullptr);
    }
    dd_linear_grad_args a;
    memset(&a, 0, sizeof(a));
    a.rows = c.rows;
    a.k = c.k;
    a.n = c.n;
    a.dy_stride = c.n + c.pad;
    a.x_stride = c.k + c.pad;
    a.w_stride = wc + c.pad;
    a.dx_stride = c.k;
    a.dw_stride = wc;
    a.dy = at(0);
    a.x = at(1);
    a.w = at(2);
    if (c.wanted & 1) a.dx = at(4);
    if (c.wanted & 2) a.dw = at(5);
    if (c.wanted & 4) a.db = at(6);
    a.work = kWork;
    a.type = a.bias_type = c.type ? DD_F16 : DD_BF16;
    a.turned = c.turned;
    room = dd_linear_grad_work(c.rows, c.k, c.n);
    need = dd_linear_grad_need(&a);
    return dd_linear_grad(&a, nullptr);
}

int main(int argc, char **argv) {
    if (argc == 3 && !strcmp(argv[1], "draw")) {
        std::mt19937_64 gen(7);
        int alike = 0;
        auto size = [&](double most) { return (long long)exp2(std::uniform_real_distribution<double>(0.0, most)(gen)); };
        for (int i = 0; i < atoi(argv[2]); i++) {
            Call c{gen() % 2 == 0, 0, 0, 0, 0, (int)(gen() % 2), (int)(gen() % 2), (int)(gen() % 8)};
            const int wide = gen() % 8;       // (one of the sizes may be very large)
            c.rows = size(wide == 0 ? 30 : 14);
            c.k = size(wide == 1 ? 30 : 14);
            c.n = size(wide == 2 ? 30 : 14);
            c.pad = gen() % 3 == 0 ? (long long)(gen() % 20) : gen() % 5 == 0 ? 8 : 0;
            if (gen() % 3 == 0) c.rows = (c.rows + 7) / 8 * 8, c.k = (c.k + 7) / 8 * 8, c.n = (c.n + 7) / 8 * 8;
            const dd_status st = run(c, gen() % 3 ? 0 : gen() % 8);
            EXPECT(st == DD_OK || st == DD_EINVAL);
            EXPECT(used <= need && need <= room);
            EXPECT(st == DD_OK || need == 0);
            // operands that load directly: what is wanted alone has the tiles and parts that it has beside the other
            if (!c.grad || st != DD_OK || c.k % 8 || c.n % 8 || c.pad % 8) continue;
            c.wanted = 7;
            run(c);
            const Cut dx = cut_dx, dw = cut_dw;
            c.wanted = 1;
            run(c);
            EXPECT(cut_dx == dx);
            c.wanted = 2;
            run(c);
            EXPECT(cut_dw == dw);
            alike++;
        }
        EXPECT(alike > atoi(argv[2]) / 100);
        if (!bad) printf("ALL OK\n");
        return bad ? 1 : 0;
    }
    char op[8];
    Call c;
    while (scanf("%7s %lld %lld %lld %lld %d %d %d", op, &c.rows, &c.k, &c.n, &c.pad, &c.turned, &c.type, &c.wanted) == 8) {
        c.grad = !strcmp(op, "grad");
        const dd_status st = run(c);
        printf("%d %zu %zu %zu %s\n", (int)st, used, need, room, said.c_str());
    }
    return bad ? 1 : 0;
}
