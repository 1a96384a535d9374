// What the experts of dispatched rows (mw_ffn.hip) take from the products in 8-bit integers (mw_int8.hip).
#ifndef MW_FFN_H_
#define MW_FFN_H_

#include "mw_internal.h"

// mw_ffn with experts of 8-bit codes; arguments are checked.  act: [n_rows][inter] bf16, codes: [n_rows][max(hidden, inter)], scales: [n_rows].
int32_t mw_ffn_int8(const mw_experts *experts, int32_t hidden, const void *x, int64_t x_stride, const int64_t *offsets, int32_t n_local,
                    int64_t n_rows, const float *row_weights, void *y, int64_t y_stride, void *act, int8_t *codes, float *scales, float *parts, hipStream_t s);

#endif  // MW_FFN_H_
