// hikonv_quantize_rows: rows of floats to codes with one scale per row.
//
// A row is read once: its values stay in registers between the maximum and the divisions.  The call is a stream (2 or 4 bytes in
// and one out per value), bound by HBM for many rows and by latency for one.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "hikonv_cuda.cuh"

namespace hikonv {

struct QuantizeParams {
    const void *x;
    long long x_row;                    // elements
    int8_t *codes;
    float *scale;
    int M, K, is_signed, lo, hi;
};

__device__ __forceinline__ float quantize_load(const float *p) { return load_ordered(p); }
__device__ __forceinline__ float quantize_load(const __half *p) { return __half2float(load_ordered(p)); }
__device__ __forceinline__ float quantize_load(const __nv_bfloat16 *p) { return __bfloat162float(load_ordered(p)); }

// The larger of two magnitudes; a NaN wins.
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// clamp(round(v / scale)); a NaN becomes 0.  The quotient is clamped before it is rounded, which gives the same code and keeps
// infinities inside the integer conversion.
__device__ __forceinline__ int quantize_value(float v, float scale, float lo, float hi) {
    const float q = __fdiv_rn(v, scale);
    return q != q ? 0 : __float2int_rn(fminf(fmaxf(q, lo), hi));
}

// Any row length and alignment: a CTA per row, which it reads twice.
template <typename T>
__global__ void __launch_bounds__(256) quantize_rows_kernel(const QuantizeParams p) {
    __shared__ float part[8];
    grid_dependency_release();
    grid_dependency_wait();
    for (int row = blockIdx.x; row < p.M; row += gridDim.x) {
        const T *x = (const T *)p.x + row * p.x_row;
        float top = 0.f;
        for (int k = threadIdx.x; k < p.K; k += 256) {
            const float v = quantize_load(x + k);
            top = max_nan(top, p.is_signed ? fabsf(v) : v);
        }
#pragma unroll
        for (int d = 16; d; d /= 2) top = max_nan(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
        if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = top;
        __syncthreads();
        top = part[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) top = max_nan(top, part[i]);
        const float scale = __fdiv_rn(top, (float)p.hi);
        if (threadIdx.x == 0) p.scale[row] = scale;
        for (int k = threadIdx.x; k < p.K; k += 256)
            p.codes[(size_t)row * p.K + k] = (int8_t)quantize_value(quantize_load(x + k), scale, (float)p.lo, (float)p.hi);
        __syncthreads();
    }
}

template <typename T>
static int launch_quantize(const QuantizeParams &p, cudaStream_t st) {
    return launch_dependent(quantize_rows_kernel<T>, dim3((unsigned)p.M), dim3(256), 0, st, p);
}

}  // namespace hikonv

using namespace hikonv;

extern "C" int hikonv_quantize_rows(const void *d_x, int x_type, long long x_row_stride, int M, int K, int bits, int is_signed,
                                    int8_t *d_codes, float *d_scale, void *stream) {
    if (x_type != HIKONV_OUT_F32 && x_type != HIKONV_OUT_F16 && x_type != HIKONV_OUT_BF16) return HIKONV_ERR_INVALID_ARG;
    if (M < 0 || K < 1 || bits < (is_signed ? 2 : 1) || bits > 8) return HIKONV_ERR_INVALID_ARG;
    if (M == 0) return HIKONV_OK;
    const size_t elem = x_type == HIKONV_OUT_F32 ? 4 : 2;
    if (M == 1) x_row_stride = K;
    // a stride of 0 (all rows are one) up to what keeps byte offsets in 64 bits
    if (!d_x || !d_codes || !d_scale || x_row_stride < 0 || x_row_stride > (1ll << 40)) return HIKONV_ERR_INVALID_ARG;
    if ((uintptr_t)d_x % elem || (uintptr_t)d_scale % 4) return HIKONV_ERR_INVALID_ARG;
    const uintptr_t x0 = (uintptr_t)d_x, x1 = x0 + ((size_t)(M - 1) * x_row_stride + K) * elem;
    const uintptr_t c0 = (uintptr_t)d_codes, c1 = c0 + (size_t)M * K, s0 = (uintptr_t)d_scale, s1 = s0 + (size_t)M * 4;
    if ((x0 < c1 && c0 < x1) || (x0 < s1 && s0 < x1) || (c0 < s1 && s0 < c1)) return HIKONV_ERR_INVALID_ARG;
    const QuantizeParams p{d_x, x_row_stride, d_codes, d_scale, M, K, is_signed != 0, is_signed ? -(1 << (bits - 1)) : 0,
                           is_signed ? (1 << (bits - 1)) - 1 : (1 << bits) - 1};
    cudaStream_t st = (cudaStream_t)stream;
    if (x_type == HIKONV_OUT_F32) return launch_quantize<float>(p, st);
    if (x_type == HIKONV_OUT_F16) return launch_quantize<__half>(p, st);
    return launch_quantize<__nv_bfloat16>(p, st);
}
