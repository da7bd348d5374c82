// Interface between the kernels of the products of 8-bit floating point numbers.
#pragma once

#include "hikonv_linear.h"

namespace hikonv {

// A few rows (hikonv_linear_f8_rows.cu).  LinearParams: x, w and their scales, epilogue; xs_row: elements from block to block
// of x_scale.
bool linear_f8_rows_takes(const LinearParams &p);
int launch_linear_f8_rows(const LinearParams &p, int x_f8, int w_f8, long long xs_row, cudaStream_t st);

}  // namespace hikonv
