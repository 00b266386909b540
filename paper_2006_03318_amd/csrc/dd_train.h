// Declarations shared by the sources of the weight update and the
// root-mean-square norm.
#pragma once

#include "dd_internal.h"

// A list of tensors for the weight update (k_update.hip).
namespace dd {
// Part of one tensor, with the part's own addresses.
struct alignas(64) TensorChunk {
    void *grad, *param;
    float *w, *m, *v;             // w: the f32 weights (master, or param itself)
    int32_t n;
    uint8_t grad_type, param_type, decay, pad;
    uint64_t pad2[2];
};
static_assert(sizeof(TensorChunk) == 64, "record size");
constexpr int64_t kChunkLen = 8192;
// A tensor of n elements, whose chunks start at `first`.
struct TensorPlace {
    TensorChunk whole;
    int64_t n, first;
};
constexpr int kNormParts = 1024;  // workgroups of the norm, at most
struct AdamFactors {
    float f;                      // factor of the gradients
    float b1, c1, b2, c2;         // beta1, 1 - beta1, beta2, 1 - beta2
    float l2, shrink;             // weight decay: weight * l2 added to the gradient, weight * shrink taken off
    float lr, rv, eps;            // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
    int32_t skip;                 // nothing is applied
};
// Working memory of a list.
struct TensorWork {
    uint32_t ticket;              // workgroups that are done; 0 between calls
    AdamFactors factors;
    alignas(64) double part[kNormParts];
};
}  // namespace dd

struct dd_tensors {
    int32_t n_chunks = 0;
    int64_t total = 0;            // elements
    bool params = false;          // weights and moments are there (dd_adam_step)
    hipStream_t stream = nullptr;
    std::vector<int64_t> sizes;
    dd::TensorWork *work = nullptr;   // one block of memory, the chunks behind it
    dd::TensorChunk *chunks = nullptr;
    mutable std::mutex mu;        // held while a call that uses work is queued
    mutable bool own_turn = false;    // the last of them was on `stream`
    mutable dd::ForeignUses uses;
};

namespace dd {

// the message of dd_last_error() for this host thread
dd_status fail(dd_status s, const char *fmt, ...) __attribute__((format(printf, 2, 3)));
dd_status hip_fail(hipError_t e, const char *what);
void no_error();

// make s wait for every use recorded on another stream
hipError_t follow_uses(ForeignUses &u, hipStream_t s);

// weight update over a list of tensors (k_update.hip)
struct AdamParams {
    double lr, beta1, beta2, eps, weight_decay;
    int32_t decoupled;
};
// the list's chunks from its tensors (of n > 0), and its working memory
hipError_t launch_tensor_chunks(const TensorPlace *p, int count, const dd_tensors *t, hipStream_t s);
hipError_t launch_grad_norm(const dd_tensors *t, double max_norm, const float *inv_scale, float *stats, hipStream_t s);
hipError_t launch_grad_clip(const dd_tensors *src, const dd_tensors *dst, const float *stats, hipStream_t s);
hipError_t launch_adam(const dd_tensors *t, int64_t *step, const float *stats, const AdamParams &p, hipStream_t s);

// root-mean-square norm over rows (k_rms.hip); rows and cols at least 1 (the
// gradient takes rows == 0: dw is zero then), work of rms_grad_work bytes
typedef dd_rms_norm_args RmsArgs;
typedef dd_rms_norm_grad_args RmsGradArgs;
constexpr int kRmsParts = 512;         // partial sums of a weight's gradient, at most
size_t rms_grad_work(int64_t rows, int64_t cols);
hipError_t launch_rms_norm(const RmsArgs &a, hipStream_t s);
hipError_t launch_rms_norm_grad(const RmsGradArgs &a, float *work, hipStream_t s);

}  // namespace dd
