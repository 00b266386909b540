// C-ABI of a layer's product and its gradient, of dropout and of the embedding:
// argument checks, working memory, and which passes run.

#include "dd_layers.h"

#include <math.h>
#include <string.h>

#include "dd_args.h"

namespace {

using dd::aligned;
using dd::check_rows;
using dd::fail;
using dd::float_type;
using dd::guarded;
using dd::hip_fail;

constexpr int64_t kMost = int64_t(1) << 31;

bool act_type(int32_t act) { return act >= DD_ACT_NONE && act <= DD_ACT_SILU; }

// f(work) with `need` bytes of the caller's working memory or, if that is NULL, of the
// library's for the time of the call (a graph would keep writing to it: refused).
template <class F>
dd_status with_work(void *given, size_t need, hipStream_t s, const char *what, const F &f) {
    if (!aligned(given, 16)) return fail(DD_EINVAL, "work is not aligned to 16 bytes");
    void *taken = nullptr;
    hipError_t e = hipSuccess;
    if (need && !given) {
        bool graph = false;
        e = dd::captured(s, &graph);
        if (e != hipSuccess) return hip_fail(e, what);
        if (graph) return fail(DD_EINVAL, "a captured %s of this size needs work from the caller", what);
        e = dd::dalloc(&taken, need, s);
        if (e != hipSuccess) return hip_fail(e, what);
        given = taken;
    }
    e = f(given);
    dd::dfree(taken, s);
    return e == hipSuccess ? DD_OK : hip_fail(e, what);
}

dd_status check_layer(int64_t rows, int64_t k, int64_t n, int32_t type, int32_t bias_type, int32_t turned) {
    if (rows < 0 || k < 1 || n < 1) return fail(DD_EINVAL, "rows must be at least 0, k and n at least 1");
    if (rows >= kMost || k >= kMost || n >= kMost) return fail(DD_EINVAL, "rows, k and n must be below 2^31");
    if (type != DD_BF16 && type != DD_F16) return fail(DD_EINVAL, "type must be DD_BF16 or DD_F16 (got %d)", type);
    if (bias_type != DD_F32 && bias_type != type) return fail(DD_EINVAL, "bias_type must be DD_F32 or type");
    if (turned != 0 && turned != 1) return fail(DD_EINVAL, "turned must be 0 or 1");
    return DD_OK;
}

dd_status check_product(int64_t m, int64_t n, int64_t k, bool p_by_rows) {
    return dd::product_fits(m, n, k, p_by_rows) ? DD_OK : fail(DD_EINVAL, "a product of %lld by %lld is too large for one launch", (long long)m, (long long)n);
}

// Whether two arrays of rows of 16-bit elements have bytes in common (or rows that lie between each other's).
bool overlap(const void *x, int64_t x_stride, const void *y, int64_t y_stride, int64_t rows, int64_t cols) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(x), b = reinterpret_cast<uintptr_t>(y);
    auto bytes = [&](int64_t stride) { return (uintptr_t)((rows > 1 ? (rows - 1) * stride : 0) + cols) * 2; };
    return a < b + bytes(y_stride) && b < a + bytes(x_stride);
}

bool sizes_known(int64_t rows, int64_t k, int64_t n) { return rows >= 0 && k >= 1 && n >= 1 && rows < kMost && k < kMost && n < kMost; }

// Bytes of a gradient whose products share the copies of their operands: those copies, and behind them what the
// products and the sums over rows need then, whose operands load directly but for w, which dx may read as it is.
// (Tiles and parts of dw are those of its transpose.)
size_t shared_work(int64_t rows, int64_t k, int64_t n) {
    if (!dd::grad_copies_work(rows, k, n)) return 0;
    auto longer = [](size_t x, size_t y) { return x > y ? x : y; };
    auto padded = [](int64_t x) { return (x + 7) / 8 * 8; };
    const char *at = reinterpret_cast<const char *>(uintptr_t(16));
    const int32_t small = dd::small_gradients(rows, k, n, false);
    const dd::Product dw{at, at, k, n, rows, padded(k), padded(n), 0, 0, DD_BF16, 3, small, {}};
    dd::Product dx{at, at, rows, k, n, padded(n), padded(n), 1, 1, DD_BF16, 3, small, {}};
    const size_t behind = longer(longer(dd::product_need(dw), dd::product_need(dx)), dd::column_sum_work(rows, n));
    dx.q = at + 2;
    const size_t by_rows = dd::product_need(dx);
    dx.q_by_rows = 0;
    const size_t by_sums = dd::product_need(dx), with_w = longer(dd::padded_size(k, n), dd::padded_size(n, k)) + behind;
    return dd::padded_size(rows, n) + dd::padded_size(rows, k) + longer(with_w, longer(by_rows, by_sums));
}

dd_status check_linear(const dd_linear_args *a) {
    if (!a) return fail(DD_EINVAL, "args is NULL");
    CHECK(check_layer(a->rows, a->k, a->n, a->type, a->bias_type, a->turned));
    if (!act_type(a->act)) return fail(DD_EINVAL, "unknown act %d", a->act);
    if (!aligned(a->bias, dd::elem_size(a->bias_type))) return fail(DD_EINVAL, "bias is not aligned to its elements");
    if (a->rows == 0) return DD_OK;
    CHECK(check_rows("x", a->x, a->rows, a->k, a->x_stride, a->type, false));
    CHECK(check_rows("w", a->w, a->turned ? a->n : a->k, a->turned ? a->k : a->n, a->w_stride, a->type, false));
    if (a->residual) CHECK(check_rows("residual", a->residual, a->rows, a->n, a->residual_stride, a->type, false));
    CHECK(check_rows("y", a->y, a->rows, a->n, a->y_stride, a->type, true));
    if (a->z) CHECK(check_rows("z", a->z, a->rows, a->n, a->z_stride, a->type, true));
    return check_product(a->rows, a->n, a->k, true);
}

dd::Product product_of(const dd_linear_args &a) {
    dd::Product p{a.x, a.w, a.rows, a.n, a.k, a.x_stride, a.w_stride, 1, a.turned, a.type, 0, 0, {}};
    p.e.bias = a.bias;
    p.e.bias_type = a.bias_type;
    p.e.act = a.act;
    p.e.residual = a.residual;
    p.e.side_stride = a.residual_stride;
    p.e.z = a.z;
    p.e.z_stride = a.z_stride;
    p.e.out = a.y;
    p.e.out_stride = a.y_stride;
    return p;
}

dd_status check_linear_grad(const dd_linear_grad_args *a) {
    if (!a) return fail(DD_EINVAL, "args is NULL");
    CHECK(check_layer(a->rows, a->k, a->n, a->type, a->bias_type, a->turned));
    if (!act_type(a->in_act)) return fail(DD_EINVAL, "unknown in_act %d", a->in_act);
    if (!a->in_z && a->in_act != DD_ACT_NONE) return fail(DD_EINVAL, "in_act needs in_z");
    const int64_t wr = a->turned ? a->n : a->k, wc = a->turned ? a->k : a->n;
    if (a->rows > 0) {
        if (a->dx || a->dw || a->db) CHECK(check_rows("dy", a->dy, a->rows, a->n, a->dy_stride, a->type, false));
        if (a->dw) CHECK(check_rows("x", a->x, a->rows, a->k, a->x_stride, a->type, false));
        if (a->dx) {
            CHECK(check_rows("w", a->w, wr, wc, a->w_stride, a->type, false));
            if (a->in_z) CHECK(check_rows("in_z", a->in_z, a->rows, a->k, a->in_z_stride, a->type, false));
            CHECK(check_rows("dx", a->dx, a->rows, a->k, a->dx_stride, a->type, true));
            CHECK(check_product(a->rows, a->k, a->n, true));
        }
    }
    if (a->dw) {
        CHECK(check_rows("dw", a->dw, wr, wc, a->dw_stride, a->type, true));
        CHECK(check_product(wr, wc, a->rows, false));
    }
    if (!aligned(a->db, dd::elem_size(a->bias_type))) return fail(DD_EINVAL, "db is not aligned to its elements");
    return DD_OK;
}

// The two products of a gradient, and the copies of operands that they share.
struct Gradients {
    const dd_linear_grad_args &a;
    dd::GradCopies copies{};
    int32_t small;
    dd::Product dw{}, dx{};
    dd::PadRows pads[3];
    size_t copied;                  // bytes of the copies

    explicit Gradients(const dd_linear_grad_args &args) : a(args) {
        if (a.dw && a.dx && a.rows > 0) {
            const bool of_dy = !dd::loads_directly(a.dy, a.dy_stride, true, a.rows, a.n) || !dd::loads_directly(a.dy, a.dy_stride, false, a.n, a.rows);
            copies = dd::grad_copies(a.rows, a.k, a.n, a.turned, dd::GradCopies{of_dy, !dd::loads_directly(a.x, a.x_stride, false, a.k, a.rows),
                                                                             !dd::loads_directly(a.w, a.w_stride, !a.turned, a.k, a.n)});
        }
        small = a.rows > 0 && dd::small_gradients(a.rows, a.k, a.n, a.turned);
        copied = lay_out(reinterpret_cast<char *>(uintptr_t(16)));      // (an address as aligned as the memory's)
    }
    // with the copies in `work` (of which the size is returned)
    size_t lay_out(char *work) {
        const char *begin = work;
        const int64_t wr = a.turned ? a.n : a.k, wc = a.turned ? a.k : a.n;
        const void *dy = a.dy, *x = a.x, *w = a.w;
        int64_t dy_stride = a.dy_stride, x_stride = a.x_stride, w_stride = a.w_stride;
        for (dd::PadRows &r : pads) r = dd::PadRows{};
        dd::PadRows *r = pads;
        if (copies.dy) work += dd::pad_rows(dy, dy_stride, a.rows, a.n, work, r++);
        if (copies.x) work += dd::pad_rows(x, x_stride, a.rows, a.k, work, r++);
        if (copies.w) work += dd::pad_rows(w, w_stride, wr, wc, work, r++);
        dw = dd::Product{x, dy, wr, wc, a.rows, x_stride, dy_stride, 0, 0, a.type, copies.x | copies.dy << 1, small, {}};
        if (a.turned) dw = dd::Product{dy, x, wr, wc, a.rows, dy_stride, x_stride, 0, 0, a.type, copies.dy | copies.x << 1, small, {}};
        dw.e.out = a.dw;
        dw.e.out_stride = a.dw_stride;
        dx = dd::Product{dy, w, a.rows, a.k, a.n, dy_stride, w_stride, 1, !a.turned, a.type, copies.dy | copies.w << 1, small, {}};
        dx.e.in_z = a.in_z;
        dx.e.side_stride = a.in_z_stride;
        dx.e.in_act = a.in_act;
        dx.e.out = a.dx;
        dx.e.out_stride = a.dx_stride;
        return (size_t)(work - begin);
    }
    size_t need() const {
        size_t most = 0;
        auto needs = [&](size_t x) { most = x > most ? x : most; };
        if (a.dw) needs(dd::product_need(dw));
        if (a.db) needs(dd::column_sum_work(a.rows, a.n));
        if (a.dx && a.rows > 0) needs(dd::product_need(dx));
        return copied + most;
    }
};

dd_status check_table(int64_t tokens, int64_t vocab, int64_t cols, int32_t type, const void *ids, int32_t id_bytes, float scale, int32_t reserved) {
    if (tokens < 0 || vocab < 1 || cols < 1) return fail(DD_EINVAL, "tokens must be at least 0, vocab and cols at least 1");
    if (tokens >= (int64_t(1) << 28) || vocab >= kMost || cols >= kMost)
        return fail(DD_EINVAL, "tokens must be below 2^28, vocab and cols below 2^31");
    if (!float_type(type)) return fail(DD_EINVAL, "unknown type %d", type);
    if (id_bytes != 8 && id_bytes != 4) return fail(DD_EINVAL, "id_bytes must be 8 or 4");
    if (tokens > 0 && (!ids || !aligned(ids, id_bytes))) return fail(DD_EINVAL, "ids is NULL or not aligned to its elements");
    if (isnan(scale)) return fail(DD_EINVAL, "scale is not a number");
    if (reserved) return fail(DD_EINVAL, "reserved must be 0");
    return DD_OK;
}

}  // namespace

extern "C" {

size_t dd_linear_work(int64_t rows, int64_t k, int64_t n) { return sizes_known(rows, k, n) && rows > 0 ? dd::product_work(rows, n, k, true) : 0; }

size_t dd_linear_need(const dd_linear_args *a) {
    size_t need = 0;
    guarded([&] {
        CHECK(check_linear(a));
        if (a->rows) need = dd::product_need(product_of(*a));
        return DD_OK;
    });
    return need;
}

dd_status dd_linear(const dd_linear_args *a, void *stream) {
    return guarded([&] {
        CHECK(check_linear(a));
        if (a->rows == 0) return DD_OK;
        const dd::Product p = product_of(*a);
        hipStream_t s = (hipStream_t)stream;
        return with_work(a->work, dd::product_need(p), s, "linear", [&](void *work) { return dd::launch_product(p, work, s); });
    });
}

size_t dd_linear_grad_work(int64_t rows, int64_t k, int64_t n) {
    if (!sizes_known(rows, k, n)) return 0;
    // each product by itself, or both with copies that they share: never the copies of either
    size_t most = dd::column_sum_work(rows, n);
    for (size_t x : {rows > 0 ? dd::product_work(rows, k, n, true) : 0, dd::product_work(k, n, rows, false), dd::product_work(n, k, rows, false)}) most = x > most ? x : most;
    const size_t shared = rows > 0 ? shared_work(rows, k, n) : 0;
    return shared > most ? shared : most;
}

size_t dd_linear_grad_need(const dd_linear_grad_args *a) {
    size_t need = 0;
    guarded([&] {
        CHECK(check_linear_grad(a));
        Gradients g(*a);
        need = g.need();
        return DD_OK;
    });
    return need;
}

dd_status dd_linear_grad(const dd_linear_grad_args *a, void *stream) {
    return guarded([&] {
        CHECK(check_linear_grad(a));
        hipStream_t s = (hipStream_t)stream;
        Gradients g(*a);
        return with_work(a->work, g.need(), s, "linear gradient", [&](void *given) {
            char *work = static_cast<char *>(given);
            hipError_t e = hipSuccess;
            bool summed = false;
            if (g.copied) {
                work += g.lay_out(work);
                dd::FewSums sums{};
                if (a->db && dd::few_rows(a->rows, a->n)) {
                    sums = dd::FewSums{a->dy, a->db, a->dy_stride, a->n, (int32_t)a->rows, a->type, a->bias_type};
                    summed = true;
                }
                e = dd::launch_pad_rows(g.pads[0], g.pads[1], g.pads[2], sums, s);
            }
            const dd::Product &dw = g.dw, &dx = g.dx;
            const void *x = a->turned ? dw.q : dw.p;
            const int64_t x_stride = a->turned ? dw.q_stride : dw.p_stride;
            const bool both = a->dw && a->dx && a->rows > 0 && dd::goes_together(dw, dx) && !overlap(a->dx, a->dx_stride, x, x_stride, a->rows, a->k);
            if (e == hipSuccess && both) e = dd::launch_together(dw, dx, s);
            if (e == hipSuccess && a->dw && !both) e = dd::launch_product(dw, work, s);
            if (e == hipSuccess && a->db && !summed) e = dd::launch_column_sum(a->dy, a->dy_stride, a->rows, a->n, a->type, a->db, a->bias_type, work, s);
            if (e == hipSuccess && a->dx && a->rows > 0 && !both) e = dd::launch_product(dx, work, s);      // (last: it may be x)
            return e;
        });
    });
}

dd_status dd_act_grad(const dd_act_grad_args *a, void *stream) {
    return guarded([&] {
        if (!a) return fail(DD_EINVAL, "args is NULL");
        if (a->rows < 0 || a->cols < 1) return fail(DD_EINVAL, "rows must be at least 0 and cols at least 1");
        if (a->rows >= kMost || a->cols >= kMost) return fail(DD_EINVAL, "rows and cols must be below 2^31");
        if (!float_type(a->type)) return fail(DD_EINVAL, "unknown type %d", a->type);
        if (!act_type(a->act)) return fail(DD_EINVAL, "unknown act %d", a->act);
        if (a->rows == 0) return DD_OK;
        CHECK(check_rows("dy", a->dy, a->rows, a->cols, a->dy_stride, a->type, false));
        CHECK(check_rows("z", a->z, a->rows, a->cols, a->z_stride, a->type, false));
        CHECK(check_rows("dz", a->dz, a->rows, a->cols, a->dz_stride, a->type, true));
        const hipError_t e = dd::launch_act_grad(*a, (hipStream_t)stream);
        return e == hipSuccess ? DD_OK : hip_fail(e, "activation gradient");
    });
}

dd_status dd_dropout(const dd_dropout_args *a, void *stream) {
    return guarded([&] {
        if (!a) return fail(DD_EINVAL, "args is NULL");
        if (a->rows < 0 || a->cols < 1) return fail(DD_EINVAL, "rows must be at least 0 and cols at least 1");
        if (a->rows >= kMost || a->cols >= kMost) return fail(DD_EINVAL, "rows and cols must be below 2^31");
        if (!float_type(a->type)) return fail(DD_EINVAL, "unknown type %d", a->type);
        if (!(a->p >= 0.0 && a->p <= 1.0)) return fail(DD_EINVAL, "p must lie in [0, 1]");
        if (!a->d_state || !aligned(a->d_state, 8) || !aligned(a->d_used, 8)) return fail(DD_EINVAL, "d_state is NULL, or it or d_used not aligned to 8 bytes");
        if (a->d_used && a->d_used < a->d_state + 2 && a->d_state < a->d_used + 2) return fail(DD_EINVAL, "d_used is d_state, or overlaps it");
        if (a->reserved) return fail(DD_EINVAL, "reserved must be 0");
        if (a->rows > 0) {
            CHECK(check_rows("x", a->x, a->rows, a->cols, a->x_stride, a->type, false));
            if (a->residual) CHECK(check_rows("residual", a->residual, a->rows, a->cols, a->residual_stride, a->type, false));
            CHECK(check_rows("out", a->out, a->rows, a->cols, a->out_stride, a->type, true));
        }
        const hipError_t e = dd::launch_dropout(*a, (hipStream_t)stream);
        return e == hipSuccess ? DD_OK : hip_fail(e, "dropout");
    });
}

dd_status dd_embed(const dd_embed_args *a, void *stream) {
    return guarded([&] {
        if (!a) return fail(DD_EINVAL, "args is NULL");
        CHECK(check_table(a->tokens, a->vocab, a->cols, a->type, a->ids, a->id_bytes, a->scale, a->reserved));
        if (a->tokens == 0) return DD_OK;
        CHECK(check_rows("table", a->table, a->vocab, a->cols, a->table_stride, a->type, false));
        CHECK(check_rows("out", a->out, a->tokens, a->cols, a->out_stride, a->type, true));
        const hipError_t e = dd::launch_embed(*a, (hipStream_t)stream);
        return e == hipSuccess ? DD_OK : hip_fail(e, "embedding");
    });
}

size_t dd_embed_grad_work(int64_t tokens, int64_t vocab, int64_t cols) {
    return sizes_known(tokens, vocab, cols) && tokens < (int64_t(1) << 28) && vocab < (int64_t(1) << 29) ? dd::embed_grad_work(tokens, vocab, cols) : 0;
}

dd_status dd_embed_grad(const dd_embed_grad_args *a, void *stream) {
    return guarded([&] {
        if (!a) return fail(DD_EINVAL, "args is NULL");
        CHECK(check_table(a->tokens, a->vocab, a->cols, a->type, a->ids, a->id_bytes, a->scale, a->reserved));
        if (a->vocab >= (int64_t(1) << 29)) return fail(DD_EINVAL, "vocab must be below 2^29");
        if (a->pad < -1 || a->pad >= a->vocab) return fail(DD_EINVAL, "pad must be -1 or a row of the table");
        if (a->tokens > 0) CHECK(check_rows("dy", a->dy, a->tokens, a->cols, a->dy_stride, a->type, false));
        CHECK(check_rows("dtable", a->dtable, a->vocab, a->cols, a->dtable_stride, a->type, true));
        hipStream_t s = (hipStream_t)stream;
        return with_work(a->work, dd::embed_grad_work(a->tokens, a->vocab, a->cols), s, "embedding gradient",
                         [&](void *work) { return dd::launch_embed_grad(*a, work, s); });
    });
}

}  // extern "C"
