// Launchers of the microscaled-format kernels (each enqueues on `stream`, returns the launch's status).
#pragma once

#include <algorithm>

#include "mg_mx.h"

namespace mg {

hipError_t launch_mx_pack(Mx f, Num t, int64_t rows, int64_t cols, const void *x, int64_t row_stride,
                          uint8_t *codes, uint8_t *scales, hipStream_t stream);
hipError_t launch_mx_unpack(Mx f, Num t, int64_t rows, int64_t cols, const uint8_t *codes, const uint8_t *scales,
                            void *x, int64_t row_stride, hipStream_t stream);

size_t mx_gradient_workspace(int64_t M, int64_t T, int64_t E);
hipError_t launch_mx_gradient(Mx f, Num t, int B, int N, int T, int E, const void *grad, int64_t grad_stride,
                              const uint8_t *codes, const uint8_t *scales, const int32_t *natoms, float *weight,
                              float *bias, void *workspace, hipStream_t stream);

// C[m][n] = sum_k A[m][k] B[n][k] + bias[n], A and B in e2m1
hipError_t launch_mx4_product(Num out, int M, int N, int K, const uint8_t *a_codes, const uint8_t *a_scales,
                              const uint8_t *b_codes, const uint8_t *b_scales, const float *bias, void *c,
                              int64_t c_stride, hipStream_t stream);
// the same with A in plain numbers (type t, also the type of C), taken to e2m1 on the way
size_t mx4_linear_workspace(int M, int N, int K);
hipError_t launch_mx4_linear(Num t, int M, int N, int K, const void *x, int64_t x_stride, const uint8_t *w_codes,
                             const uint8_t *w_scales, const float *bias, void *c, int64_t c_stride, void *workspace,
                             hipStream_t stream);

}  // namespace mg
