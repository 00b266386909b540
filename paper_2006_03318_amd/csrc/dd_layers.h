// Declarations shared by the sources of a layer's product, of dropout and of
// the embedding.
#pragma once

#include "dd_train.h"

namespace dd {

typedef dd_linear_args LinearArgs;
typedef dd_linear_grad_args LinearGradArgs;

// What becomes of a sum s of products before it is stored (k_linear.hip):
//   t = s + bias,  z = t,  out = act(t) + residual     or
//   out = s * in_act'(in_z)
struct Epilogue {
    const void *bias, *residual, *in_z;     // (the last two: one of them at most)
    void *z, *out;
    int64_t side_stride, z_stride, out_stride;      // (the first: of residual or in_z)
    int32_t bias_type, act, in_act;
};

// out[i][j] = sum over l of p(i, l) q(l, j).  An operand lies by its rows (i or
// j: l is consecutive) or by its sums (i or j is consecutive); its stride is
// between the others.
struct Product {
    const void *p, *q;
    int64_t m, n, k;
    int64_t p_stride, q_stride;
    int32_t p_by_rows, q_by_rows;
    int32_t type;
    int32_t padded;             // 1: p's, 2: q's rows are padded with zeros to 16 bytes, whatever their length
    int32_t small;              // 1: aligned operands go in tiles of 64 x 64, uncut
    Epilogue e;
};

// Rows of 16-bit elements copied end to end, padded with zeros to 16 bytes (no rows: nothing).
struct PadRows {
    const void *from;
    void *to;
    int64_t stride, rows, cols;
};
size_t padded_size(int64_t rows, int64_t cols);
// an operand, `count` rows (or columns) of k sums, needs no copy
bool loads_directly(const void *p, int64_t stride, bool by_rows, int64_t count, int64_t k);
// Operands of a layer's gradients that are copied once for both products.  needed: those that do not load directly
// as they are; grad_copies_work bytes hold all (0: none is copied).
struct GradCopies {
    bool dy, x, w;
};
GradCopies grad_copies(int64_t rows, int64_t k, int64_t n, bool turned, const GradCopies &needed);
size_t grad_copies_work(int64_t rows, int64_t k, int64_t n);
// x and its stride become those of the copy in `to`; the size of the copy
size_t pad_rows(const void *&x, int64_t &stride, int64_t rows, int64_t cols, void *to, PadRows *r);
// Sums over few rows of an array (type), into out (out_type).  No columns: none.
struct FewSums {
    const void *x;
    void *out;
    int64_t stride, cols;
    int32_t rows, type, out_type;
};
bool few_rows(int64_t rows, int64_t cols);
hipError_t launch_pad_rows(const PadRows &x, const PadRows &y, const PadRows &z, const FewSums &sums, hipStream_t s);

// bytes of working memory of an m by n product of k sums (0: none), and the product
size_t product_work(int64_t m, int64_t n, int64_t k, bool p_by_rows);
size_t product_need(const Product &p);      // of these operands: at most that
bool product_fits(int64_t m, int64_t n, int64_t k, bool p_by_rows);      // one launch takes it
hipError_t launch_product(const Product &p, void *work, hipStream_t s);
// Whether the products of a layer's gradients take less in one launch, by their sizes (both are `small` then, which one
// alone is too: where operands load directly, its bits do not depend on whether the other is wanted), and by their
// operands; that launch, without working memory.
bool small_gradients(int64_t rows, int64_t k, int64_t n, bool turned);
bool goes_together(const Product &dw, const Product &dx);
hipError_t launch_together(const Product &dw, const Product &dx, hipStream_t s);

// sums over the rows of an array (type, rows) into out (out_type), with
// column_sum_work bytes
size_t column_sum_work(int64_t rows, int64_t cols);
hipError_t launch_column_sum(const void *x, int64_t stride, int64_t rows, int64_t cols, int32_t type, void *out, int32_t out_type,
                             void *work, hipStream_t s);

// dz = dy * act'(z)
hipError_t launch_act_grad(const dd_act_grad_args &a, hipStream_t s);

// dropout (k_dropout.hip)
hipError_t launch_dropout(const dd_dropout_args &a, hipStream_t s);

// embedding (k_embed.hip)
hipError_t launch_embed(const dd_embed_args &a, hipStream_t s);
size_t embed_grad_work(int64_t tokens, int64_t vocab, int64_t cols);
hipError_t launch_embed_grad(const dd_embed_grad_args &a, void *work, hipStream_t s);

}  // namespace dd
