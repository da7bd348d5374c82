// Interface between the entry points of the linear layers (hikonv_linear.cu) and their kernels.
#pragma once

#include <cuda_runtime.h>

#include "hikonv_internal.h"

namespace hikonv {

// A linear layer as its kernels see it.  A plain layer is one group that holds all rows (offsets == nullptr, E == 1).
struct LinearParams {
    const uint8_t *x, *w;
    const int32_t *offsets;
    long long x_row, w_row;             // bytes from row to row
    int M, N, K, E;
    int x_signed, w_signed;
    int x_u8, w_u8;                     // bytes that only unsigned arithmetic reads right (unsigned 8-bit codes)
    int w_bits;                         // 8, or 4 / 2 / 1 dense
    int down;                           // sums hold the products times 2^down (signed dense weights sit in a byte's upper bits)
    int out_type, act;
    void *out;
    const void *residual, *bias;
    const float *x_scale, *w_scale;
    long long out_row, res_row;         // elements from row to row
    int shift, lo, hi;
};

// A few rows (per group) at a time (hikonv_linear_rows.cu); `rows`: how many a group has on average, since the host does not see the bounds of
// the groups.  A group that has most of the rows is walked over eight rows at a time by its own CTAs alone: 64 rows over eight groups of
// 2048 x 2048 8-bit weights take 8.3 us where every group has eight, 37 us where one has all.
constexpr int kLinearFewRows = 16;
bool linear_rows_takes(const LinearParams &p, int rows);
int launch_linear_rows(const LinearParams &p, cudaStream_t st);

int sm_count_here();                                         // of the current device

// All others (hikonv_linear_tc.cu).
size_t linear_tc_workspace(const LinearParams &p);           // bytes, 16-byte aligned, for rows that do not start on such boundaries
int launch_linear_tc(LinearParams p, void *workspace, size_t workspace_bytes, cudaStream_t st);
int read_linear_timeouts(unsigned int *h_count);             // on the current device, since it was loaded
int launch_linear_wait_check(long long cycles, cudaStream_t st);

}  // namespace hikonv
