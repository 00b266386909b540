// C-ABI of the weight update and of the root-mean-square norm: argument
// checks, the list handle, and which pass runs.

#include <math.h>
#include <string.h>

#include "dd_args.h"

namespace {

using dd::aligned;
using dd::captured;
using dd::check_rows;
using dd::fail;
using dd::float_type;
using dd::guarded;
using dd::hip_fail;

// A graph has no place among the calls of other streams: one that uses the
// working memory is captured on the list's own stream.
dd_status check_capture(const dd_tensors *t, hipStream_t s) {
    bool graph = false;
    const hipError_t e = s == t->stream ? hipSuccess : captured(s, &graph);
    if (e != hipSuccess) return hip_fail(e, "stream state");
    return graph ? fail(DD_EINVAL, "captured on another stream than the list was loaded on") : DD_OK;
}

// The handle's working memory is one, so calls on it run one after the other
// on whatever streams they are made.  Its own stream waits for the uses noted on
// others; another stream for those, and for the own stream only where that has
// had a call since (what else is queued there is none of its business).
hipError_t take_turn(const dd_tensors *t, hipStream_t s) {
    if (s == t->stream) {
        dd::join_uses(t->uses, s);
        return hipSuccess;
    }
    hipError_t e = dd::follow_uses(t->uses, s);
    if (e != hipSuccess || !t->own_turn) return e;
    hipEvent_t ev = nullptr;
    e = hipEventCreateWithFlags(&ev, hipEventDisableTiming);
    if (e != hipSuccess) return e;
    e = hipEventRecord(ev, t->stream);
    if (e == hipSuccess) e = hipStreamWaitEvent(s, ev, 0);
    (void)hipEventDestroy(ev);
    return e;
}
hipError_t end_turn(const dd_tensors *t, hipStream_t s) {
    const hipError_t e = dd::note_use(t->uses, t->stream, s);
    if (e == hipSuccess) t->own_turn = s == t->stream;
    return e;
}

dd_status check_tensor(int32_t i, const dd_tensor &t) {
    if (t.n < 0) return fail(DD_EINVAL, "tensor %d: n < 0", i);
    if (!float_type(t.grad_type)) return fail(DD_EINVAL, "tensor %d: unknown grad_type %d", i, t.grad_type);
    if (t.reserved || (t.no_decay != 0 && t.no_decay != 1))
        return fail(DD_EINVAL, "tensor %d: no_decay must be 0 or 1 and reserved 0", i);
    if (!aligned(t.grad, dd::elem_size(t.grad_type))) return fail(DD_EINVAL, "tensor %d: grad is not aligned to its elements", i);
    if (t.n > 0 && !t.grad) return fail(DD_EINVAL, "tensor %d: grad is NULL", i);
    if (!t.param) {
        if (t.master || t.m || t.v) return fail(DD_EINVAL, "tensor %d: master, m and v need a param", i);
        return DD_OK;
    }
    if (!float_type(t.param_type)) return fail(DD_EINVAL, "tensor %d: unknown param_type %d", i, t.param_type);
    if (!t.m || !t.v) return fail(DD_EINVAL, "tensor %d: param needs m and v", i);
    if ((t.param_type == DD_F32) != !t.master)
        return fail(DD_EINVAL, "tensor %d: a param of 16 bits needs a master, one of 32 has none", i);
    if (!aligned(t.param, dd::elem_size(t.param_type)) || !aligned(t.master, 4) || !aligned(t.m, 4) || !aligned(t.v, 4))
        return fail(DD_EINVAL, "tensor %d: param, master, m or v is not aligned to its elements", i);
    return DD_OK;
}

void free_tensors(dd_tensors *x) {
    dd::join_uses(x->uses, x->stream);
    dd::dfree(x->work, x->stream);
    delete x;
}

dd_status load_tensors(int32_t count, const dd_tensor *t, hipStream_t s, dd_tensors *x) {
    // total below 2^62 and chunks below 2^31: no count of them wraps
    int64_t total = 0, chunks = 0;
    int32_t with = 0, without = 0;
    for (int32_t i = 0; i < count; i++) {
        const dd_status st = check_tensor(i, t[i]);
        if (st != DD_OK) return st;
        if (t[i].n >= (int64_t(1) << 62) - total) return fail(DD_EINVAL, "more than 2^62 elements");
        total += t[i].n;
        if (t[i].n > 0) (t[i].param ? with : without)++;
        x->sizes.push_back(t[i].n);
    }
    if (with && without) return fail(DD_EINVAL, "some tensors have params and some have none");
    for (int32_t i = 0; i < count; i++) chunks += (t[i].n + dd::kChunkLen - 1) / dd::kChunkLen;
    if (chunks >= (int64_t(1) << 31)) return fail(DD_EINVAL, "too many elements for one list");
    x->n_chunks = (int32_t)chunks;
    x->total = total;
    x->params = without == 0;
    std::vector<dd::TensorPlace> h;
    h.reserve((size_t)count);
    int64_t first = 0;
    for (int32_t i = 0; i < count; i++) {
        const dd_tensor &a = t[i];
        if (a.n == 0) continue;
        dd::TensorPlace c;
        memset(&c, 0, sizeof(c));
        c.whole.grad = a.grad;
        c.whole.param = a.param;
        c.whole.w = a.master ? a.master : static_cast<float *>(a.param);
        c.whole.m = a.m;
        c.whole.v = a.v;
        c.whole.grad_type = (uint8_t)a.grad_type;
        c.whole.param_type = (uint8_t)a.param_type;
        c.whole.decay = !a.no_decay;
        c.n = a.n;
        c.first = first;
        first += (a.n + dd::kChunkLen - 1) / dd::kChunkLen;
        h.push_back(c);
    }
    void *mem = nullptr, *places = nullptr;
    hipError_t e = dd::dalloc(&mem, sizeof(dd::TensorWork) + sizeof(dd::TensorChunk) * (size_t)chunks, s);
    if (e != hipSuccess) return hip_fail(e, "alloc tensor list");
    x->work = static_cast<dd::TensorWork *>(mem);
    x->chunks = reinterpret_cast<dd::TensorChunk *>(x->work + 1);
    if (!h.empty()) {
        e = dd::dalloc(&places, sizeof(dd::TensorPlace) * h.size(), s);
        if (e == hipSuccess)
            e = hipMemcpyAsync(places, h.data(), sizeof(dd::TensorPlace) * h.size(), hipMemcpyHostToDevice, s);
    }
    if (e == hipSuccess)
        e = dd::launch_tensor_chunks(static_cast<dd::TensorPlace *>(places), (int)h.size(), x, s);
    const hipError_t done = hipStreamSynchronize(s);      // (h is read until here)
    if (e == hipSuccess) e = done;
    dd::dfree(places, s);
    return e == hipSuccess ? DD_OK : hip_fail(e, "copy tensor list");
}

dd_status check_norm(int64_t rows, int64_t cols, int32_t type, int32_t weight_type, const void *weight) {
    if (rows < 0 || cols < 1) return fail(DD_EINVAL, "rows must be at least 0 and cols at least 1");
    if (rows >= (int64_t(1) << 31) || cols >= (int64_t(1) << 31)) return fail(DD_EINVAL, "rows and cols must be below 2^31");
    if (!float_type(type)) return fail(DD_EINVAL, "unknown type %d", type);
    if (weight_type != DD_F32 && weight_type != type) return fail(DD_EINVAL, "weight_type must be DD_F32 or type");
    if (!aligned(weight, dd::elem_size(weight_type))) return fail(DD_EINVAL, "weight is not aligned to its elements");
    return DD_OK;
}

}  // namespace

extern "C" {

dd_status dd_tensors_load(int32_t count, const dd_tensor *t, void *stream, dd_tensors **out) {
    return guarded([&] {
        if (!out) return fail(DD_EINVAL, "out is NULL");
        *out = nullptr;
        if (count < 0) return fail(DD_EINVAL, "count < 0");
        if (count > 0 && !t) return fail(DD_EINVAL, "t is NULL");
        hipStream_t s = (hipStream_t)stream;
        dd_tensors *x = new dd_tensors();
        x->stream = s;
        dd_status st;
        try {
            st = load_tensors(count, t, s, x);
        } catch (...) {
            free_tensors(x);
            throw;
        }
        if (st != DD_OK) {
            free_tensors(x);
            return st;
        }
        *out = x;
        return DD_OK;
    });
}

void dd_tensors_free(dd_tensors *t) {
    if (t) free_tensors(t);
}

dd_status dd_grad_norm(const dd_tensors *t, float max_norm, const float *d_inv_scale, float *d_stats, void *stream) {
    return guarded([&] {
        if (!t) return fail(DD_EINVAL, "NULL handle");
        if (!d_stats) return fail(DD_EINVAL, "d_stats is NULL");
        if (isnan(max_norm)) return fail(DD_EINVAL, "max_norm is not a number");
        hipStream_t s = (hipStream_t)stream;
        CHECK(check_capture(t, s));
        std::lock_guard<std::mutex> lk(t->mu);
        hipError_t e = take_turn(t, s);
        if (e == hipSuccess) e = dd::launch_grad_norm(t, max_norm, d_inv_scale, d_stats, s);
        if (e == hipSuccess) e = end_turn(t, s);
        return e == hipSuccess ? DD_OK : hip_fail(e, "gradient norm");
    });
}

dd_status dd_grad_clip(const dd_tensors *src, const dd_tensors *dst, const float *d_stats, void *stream) {
    return guarded([&] {
        if (!src || !dst) return fail(DD_EINVAL, "NULL handle");
        if (!d_stats) return fail(DD_EINVAL, "d_stats is NULL");
        if (src != dst && src->sizes != dst->sizes) return fail(DD_EMISMATCH, "the lists differ in their tensors' sizes");
        hipStream_t s = (hipStream_t)stream;
        bool graph = false;
        hipError_t e = s == src->stream && s == dst->stream ? hipSuccess : captured(s, &graph);
        if (e == hipSuccess) e = dd::launch_grad_clip(src, dst, d_stats, s);
        // (a point inside a graph is none that a stream could wait for)
        if (e == hipSuccess && !graph) e = dd::note_use(src->uses, src->stream, s);
        if (e == hipSuccess && !graph) e = dd::note_use(dst->uses, dst->stream, s);
        return e == hipSuccess ? DD_OK : hip_fail(e, "clip gradients");
    });
}

dd_status dd_adam_step(const dd_tensors *t, int64_t *d_step, const float *d_stats, double lr, double beta1, double beta2,
                       double eps, double weight_decay, int32_t decoupled, void *stream) {
    return guarded([&] {
        if (!t) return fail(DD_EINVAL, "NULL handle");
        if (!d_step) return fail(DD_EINVAL, "d_step is NULL");
        if (!t->params) return fail(DD_EINVAL, "the list has gradients only");
        if (!(lr >= 0.0 && isfinite(lr) && eps >= 0.0 && isfinite(eps) && weight_decay >= 0.0 && isfinite(weight_decay)))
            return fail(DD_EINVAL, "lr, eps and weight_decay must be finite and not negative");
        if (!(beta1 >= 0.0 && beta1 < 1.0 && beta2 >= 0.0 && beta2 < 1.0))
            return fail(DD_EINVAL, "beta1 and beta2 must lie in [0, 1)");
        if (decoupled != 0 && decoupled != 1) return fail(DD_EINVAL, "decoupled must be 0 or 1");
        hipStream_t s = (hipStream_t)stream;
        CHECK(check_capture(t, s));
        const dd::AdamParams p{lr, beta1, beta2, eps, weight_decay, decoupled};
        std::lock_guard<std::mutex> lk(t->mu);
        hipError_t e = take_turn(t, s);
        if (e == hipSuccess) e = dd::launch_adam(t, d_step, d_stats, p, s);
        if (e == hipSuccess) e = end_turn(t, s);
        return e == hipSuccess ? DD_OK : hip_fail(e, "adam step");
    });
}

dd_status dd_rms_norm(const dd_rms_norm_args *a, void *stream) {
    return guarded([&] {
        if (!a) return fail(DD_EINVAL, "args is NULL");
        CHECK(check_norm(a->rows, a->cols, a->type, a->weight_type, a->weight));
        const bool narrow = a->out_type == DD_E4M3 || a->out_type == DD_I8;
        if (!narrow && a->out_type != a->type) return fail(DD_EINVAL, "out_type must be type, DD_E4M3 or DD_I8");
        if (a->group != 0 && a->group != 32 && a->group != 64 && a->group != 128)
            return fail(DD_EINVAL, "group must be 0, 32, 64 or 128 (got %d)", a->group);
        if (!narrow && (a->group || a->scales)) return fail(DD_EINVAL, "group and scales belong to an output of 8 bits");
        if (a->reserved) return fail(DD_EINVAL, "reserved must be 0");
        if (!(a->eps >= 0.0f && isfinite(a->eps))) return fail(DD_EINVAL, "eps must be finite and not negative");
        if (a->rows == 0) return DD_OK;
        CHECK(check_rows("x", a->x, a->rows, a->cols, a->x_stride, a->type, false));
        if (a->residual) CHECK(check_rows("residual", a->residual, a->rows, a->cols, a->residual_stride, a->type, false));
        if (a->h) CHECK(check_rows("h", a->h, a->rows, a->cols, a->h_stride, a->type, true));
        CHECK(check_rows("out", a->out, a->rows, a->cols, a->out_stride, a->out_type, true));
        if (narrow && (!a->scales || !aligned(a->scales, 4)))
            return fail(DD_EINVAL, "an output of 8 bits needs scales, aligned to 4 bytes");
        if (!aligned(a->rstd, 4)) return fail(DD_EINVAL, "rstd is not aligned to its elements");
        const hipError_t e = dd::launch_rms_norm(*a, (hipStream_t)stream);
        return e == hipSuccess ? DD_OK : hip_fail(e, "rms norm");
    });
}

size_t dd_rms_norm_grad_work(int64_t rows, int64_t cols) {
    return rows < 0 || cols < 1 || rows >= (int64_t(1) << 31) || cols >= (int64_t(1) << 31) ? 0 : dd::rms_grad_work(rows, cols);
}

dd_status dd_rms_norm_grad(const dd_rms_norm_grad_args *a, void *stream) {
    return guarded([&] {
        if (!a) return fail(DD_EINVAL, "args is NULL");
        CHECK(check_norm(a->rows, a->cols, a->type, a->weight_type, a->weight));
        if (a->rows > 0) {
            CHECK(check_rows("dy", a->dy, a->rows, a->cols, a->dy_stride, a->type, false));
            CHECK(check_rows("h", a->h, a->rows, a->cols, a->h_stride, a->type, false));
            if (a->dh) CHECK(check_rows("dh", a->dh, a->rows, a->cols, a->dh_stride, a->type, false));
            CHECK(check_rows("dx", a->dx, a->rows, a->cols, a->dx_stride, a->type, true));
            if (!a->rstd || !aligned(a->rstd, 4)) return fail(DD_EINVAL, "rstd is NULL or not aligned to its elements");
        }
        if (!aligned(a->dw, dd::elem_size(a->weight_type))) return fail(DD_EINVAL, "dw is not aligned to its elements");
        if (!aligned(a->work, 16)) return fail(DD_EINVAL, "work is not aligned to 16 bytes");
        if (a->rows == 0 && !a->dw) return DD_OK;
        hipStream_t s = (hipStream_t)stream;
        void *work = a->work, *taken = nullptr;
        hipError_t e = hipSuccess;
        if (a->dw && !work) {
            // (the block goes back to the cache, a graph would keep writing to it)
            bool graph = false;
            e = captured(s, &graph);
            if (e != hipSuccess) return hip_fail(e, "alloc partial sums");
            if (graph) return fail(DD_EINVAL, "a captured gradient needs work from the caller");
            e = dd::dalloc(&taken, dd::rms_grad_work(a->rows, a->cols), s);
            if (e != hipSuccess) return hip_fail(e, "alloc partial sums");
            work = taken;
        }
        e = dd::launch_rms_norm_grad(*a, static_cast<float *>(work), s);
        dd::dfree(taken, s);
        return e == hipSuccess ? DD_OK : hip_fail(e, "rms norm gradient");
    });
}

}  // extern "C"
