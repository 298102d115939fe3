// Row quantisation to 8-bit levels and the product of such levels: what net.hip and the C entries of quant.hip share.
#pragma once
#include "common.h"

namespace dqn {

// Enqueue only; arguments have been checked.
int enqueue_quantize_rows(const void* x, int32_t type, int64_t ldx, int64_t rows, int64_t cols, int8_t* q, int64_t ldq, float* scale, void* values, int64_t ldv,
                          hipStream_t st);
int enqueue_q8_linear(const int8_t* x, int64_t ldx, const float* sx, const int8_t* w, int64_t ldw, const float* sw, const float* bias, bool relu, int64_t M,
                      int64_t N, int64_t K, void* y, int32_t type, int64_t ldy, hipStream_t st);

}  // namespace dqn
