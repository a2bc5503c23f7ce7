// Arguments of the residual-norm kernels (residual_norm.hip).
#pragma once

#include "philox.h"

namespace lsp {

struct ResidualNormArgs {
    const void *x, *f, *post_w, *post_b, *gate, *pre_w, *pre_b, *dy, *dh;
    void *y, *h, *dx, *df;
    float* stats;                                        // [4][rows]
    float* partial;                                      // backward: [workgroups][sums][width]
    float* grads[5];                                     // of pre_w, pre_b, gate, post_w, post_b; NULL: not asked for
    int64_t x_stride, f_stride, y_stride, h_stride, dy_stride, dh_stride, dx_stride, df_stride;
    int64_t rows;
    int32_t width, post, pre, many;                      // many: backward, see many_rows()
    int32_t whole, whole_too;                            // see may_read_whole()
    float   eps, residual_scale, branch_scale;
    Dropout drop;
};

hipError_t launch_residual_norm_forward(const ResidualNormArgs& a, lsp_dtype dtype, hipStream_t st);
hipError_t launch_residual_norm_backward(const ResidualNormArgs& a, lsp_dtype dtype, hipStream_t st);
size_t residual_norm_partial_bytes(int64_t rows, int32_t width);   // backward: the parts of the sums over the rows

}  // namespace lsp
