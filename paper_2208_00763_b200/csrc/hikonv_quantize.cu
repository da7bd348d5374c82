// hikonv_quantize_rows: rows of floats to codes with one scale per row.
//
// A row is read once: its values stay in registers between the maximum and the divisions.  The call is a stream (2 or 4 bytes in
// and one out per value), bound by HBM for many rows and by latency for one.
//
// The division is that of the definition, rounded to nearest in 32 bits, and a code is its rounded quotient; a multiply by the
// reciprocal differs next to the halves between two codes.  So a thread multiplies first, which is 2^-22.4 off at most, and divides only
// where that leaves the code open, in one value of some ten thousand: a division per value bound the kernel at 48 us where it now takes TODO.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "hikonv_cuda.cuh"
#include "hikonv_linear.h"

namespace hikonv {

struct QuantizeParams {
    const void *x;
    long long x_row;                    // elements
    int8_t *codes;
    float *scale;
    int M, K, lo, hi;
    int threads;                        // that share a row: 32, or all of a CTA
};

__device__ __forceinline__ float quantize_float(float v) { return v; }
__device__ __forceinline__ float quantize_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float quantize_float(__nv_bfloat16 v) { return __bfloat162float(v); }

// The larger of two magnitudes; a NaN wins.
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// clamp(round(v / scale)); a NaN becomes 0.  The quotient is clamped before it is rounded, which gives the same code and keeps
// infinities inside the integer conversion.
__device__ __forceinline__ uint32_t quantize_exactly(float v, float scale, float lo, float hi) {
    const float q = __fdiv_rn(v, scale);
    return q != q ? 0u : (uint32_t)__float2int_rn(fminf(fmaxf(q, lo), hi)) & 255u;
}
// The same by the rounded reciprocal of the scale, for a finite row and a normal scale; `distance`: of the product from the whole number
// next to it.  The reciprocal and the product are off by half a step each, so the product is within 2^-22.9 of
// the quotient, relative, and the quotient's own rounding adds 2^-24: below 256 the two differ by less than 2^-14.4.  Where
// the distance is below 1/2 - 2^-14, both round to the same code.  Adding 1.5 * 2^23 rounds to nearest, ties to even, and leaves the
// code in the low byte.  Bounds are needed below zero for unsigned codes alone: no product is above hi (1 + 2^-22) in magnitude.
template <bool SIGNED>
__device__ __forceinline__ uint32_t quantize_quickly(float v, float inverse, float *distance) {
    const float p = __fmul_rn(v, inverse), q = SIGNED ? p : fmaxf(p, 0.f), lifted = q + 12582912.f;
    *distance = fabsf(q - (lifted - 12582912.f));
    return __float_as_uint(lifted);
}
constexpr float kOpen = 0.5f - 0x1p-14f;

// A row's scale, and how its codes are found.
struct RowScale {
    float scale, inverse, lo, hi;
    bool quick;
    __device__ __forceinline__ RowScale(float top, const QuantizeParams &p) {
        scale = __fdiv_rn(top, (float)p.hi);
        inverse = __frcp_rn(scale);
        lo = (float)p.lo;
        hi = (float)p.hi;
        quick = scale >= 0x1p-120f && scale <= 0x1p120f;
    }
};

// The largest of a value over the threads that share a row.
__device__ __forceinline__ float row_max(float top, int threads, float *part) {
#pragma unroll
    for (int d = 16; d; d /= 2) top = max_nan(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
    if (threads > 32) {
        if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = top;
        __syncthreads();
        top = part[(threadIdx.x & 31) < threads / 32 ? threadIdx.x & 31 : 0];
#pragma unroll
        for (int d = 16; d; d /= 2) top = max_nan(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
    }
    return top;
}

// The largest magnitude (signed) or value of what a word holds and `top`, in the word's own type: exact, and two at a time for the short ones.
template <bool SIGNED>
__device__ __forceinline__ uint32_t word_max(uint32_t w, uint32_t top, float) {
    const float v = __uint_as_float(w);
    return __float_as_uint(max_nan(SIGNED ? fabsf(v) : v, __uint_as_float(top)));
}
template <bool SIGNED>
__device__ __forceinline__ uint32_t word_max(uint32_t w, uint32_t top, __half) {
    const __half2 v = *reinterpret_cast<__half2 *>(&w), m = __hmax2_nan(SIGNED ? __habs2(v) : v, *reinterpret_cast<__half2 *>(&top));
    return *reinterpret_cast<const uint32_t *>(&m);
}
template <bool SIGNED>
__device__ __forceinline__ uint32_t word_max(uint32_t w, uint32_t top, __nv_bfloat16) {
    const __nv_bfloat162 v = *reinterpret_cast<__nv_bfloat162 *>(&w), m = __hmax2_nan(SIGNED ? __habs2(v) : v, *reinterpret_cast<__nv_bfloat162 *>(&top));
    return *reinterpret_cast<const uint32_t *>(&m);
}

// Rows on 16-byte boundaries (codes on 8-byte ones): VECS pieces of eight values per thread, in registers.
template <typename T, int VECS, bool SIGNED>
__global__ void __launch_bounds__(512, VECS >= 4 && sizeof(T) == 4 ? 1 : 2) quantize_vectors_kernel(const QuantizeParams p) {
    constexpr int WORDS = sizeof(T) * 2;                // of eight values
    __shared__ float part[32];
    grid_dependency_release();
    grid_dependency_wait();
    const int at = p.threads == 32 ? threadIdx.x & 31 : threadIdx.x;
    const int row = p.threads == 32 ? blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32 : blockIdx.x;
    if (row >= p.M) return;                             // whole warps; rows of a whole CTA are all there
    const T *x = (const T *)p.x + row * p.x_row;
    const int pieces = p.K / 8;
    uint32_t v[VECS][WORDS];
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
        const int j = at + i * p.threads;
#pragma unroll
        for (int h = 0; h < WORDS / 4; ++h) {
            uint4 o = make_uint4(0, 0, 0, 0);
            if (j < pieces) o = load_ordered(reinterpret_cast<const uint4 *>(x + j * 8) + h);
            v[i][4 * h] = o.x; v[i][4 * h + 1] = o.y; v[i][4 * h + 2] = o.z; v[i][4 * h + 3] = o.w;
        }
    }
    auto value = [&](int i, int k) {
        if constexpr (sizeof(T) == 4) return __uint_as_float(v[i][k]);
        else {
            const unsigned short bits = (unsigned short)(v[i][k / 2] >> (16 * (k & 1)));
            return quantize_float(*reinterpret_cast<const T *>(&bits));
        }
    };
    uint32_t words = 0;
#pragma unroll
    for (int i = 0; i < VECS; ++i)
#pragma unroll
        for (int k = 0; k < WORDS; ++k) words = word_max<SIGNED>(v[i][k], words, T());
    float top;
    if constexpr (sizeof(T) == 4) {
        top = __uint_as_float(words);
    } else {
        const unsigned short low = (unsigned short)words, high = (unsigned short)(words >> 16);
        top = max_nan(quantize_float(*reinterpret_cast<const T *>(&low)), quantize_float(*reinterpret_cast<const T *>(&high)));
    }
    top = row_max(top, p.threads, part);
    const RowScale by(top, p);
    if (at == 0) p.scale[row] = by.scale;
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
        const int j = at + i * p.threads;
        if (j >= pieces) break;
        uint32_t o[8];
        float open = by.quick ? 0.f : 1.f;
#pragma unroll
        for (int k = 0; k < 8; k += 2) {
            float d0, d1;
            o[k] = quantize_quickly<SIGNED>(value(i, k), by.inverse, &d0);
            o[k + 1] = quantize_quickly<SIGNED>(value(i, k + 1), by.inverse, &d1);
            open = fmaxf(fmaxf(d0, d1), open);
        }
        if (open >= kOpen) {                            // rare, about one time in thirty for a warp
#pragma unroll
            for (int k = 0; k < 8; ++k) o[k] = quantize_exactly(value(i, k), by.scale, by.lo, by.hi);
        }
        auto four = [&](int k) { return byte_permute(byte_permute(o[k], o[k + 1], 0x0040), byte_permute(o[k + 2], o[k + 3], 0x0040), 0x5410); };
        *reinterpret_cast<uint2 *>(p.codes + (size_t)row * p.K + j * 8) = make_uint2(four(0), four(4));
    }
}

// Any alignment: VALUES single values per thread in registers, neighbours on neighbouring threads; longer rows (VALUES == 0) are
// read twice, the second time from the caches.
template <typename T, int VALUES, bool SIGNED>
__global__ void __launch_bounds__(1024, 1) quantize_values_kernel(const QuantizeParams p) {
    __shared__ float part[32];
    grid_dependency_release();
    grid_dependency_wait();
    const int row = blockIdx.x;
    const T *x = (const T *)p.x + row * p.x_row;
    int8_t *codes = p.codes + (size_t)row * p.K;
    float v[VALUES > 0 ? VALUES : 1], top = 0.f;
    if (VALUES > 0) {
#pragma unroll
        for (int i = 0; i < VALUES; ++i) {
            const int k = threadIdx.x + i * p.threads;
            v[i] = k < p.K ? quantize_float(load_ordered(x + k)) : 0.f;
        }
#pragma unroll
        for (int i = 0; i < VALUES; ++i) top = max_nan(top, SIGNED ? fabsf(v[i]) : v[i]);
    } else {
        for (int k = threadIdx.x; k < p.K; k += p.threads) {
            const float a = quantize_float(load_ordered(x + k));
            top = max_nan(top, SIGNED ? fabsf(a) : a);
        }
    }
    top = row_max(top, p.threads, part);
    const RowScale by(top, p);
    if (threadIdx.x == 0) p.scale[row] = by.scale;
    auto one = [&](float a) {
        float distance;
        uint32_t c = quantize_quickly<SIGNED>(a, by.inverse, &distance);
        if (!by.quick || distance >= kOpen) c = quantize_exactly(a, by.scale, by.lo, by.hi);
        return (int8_t)c;
    };
    if constexpr (VALUES > 0) {
        uint32_t c[VALUES];
        float open = by.quick ? 0.f : 1.f;
#pragma unroll
        for (int i = 0; i < VALUES; i += 2) {
            float d0, d1;
            c[i] = quantize_quickly<SIGNED>(v[i], by.inverse, &d0);
            c[i + 1] = quantize_quickly<SIGNED>(v[i + 1], by.inverse, &d1);
            open = fmaxf(fmaxf(d0, d1), open);
        }
        if (open >= kOpen) {                            // rare
#pragma unroll
            for (int i = 0; i < VALUES; ++i) c[i] = quantize_exactly(v[i], by.scale, by.lo, by.hi);
        }
#pragma unroll
        for (int i = 0; i < VALUES; ++i) {
            const int k = threadIdx.x + i * p.threads;
            if (k < p.K) codes[k] = (int8_t)c[i];
        }
    } else {
        for (int k = threadIdx.x; k < p.K; k += p.threads) codes[k] = one(quantize_float(load_ordered(x + k)));
    }
}

template <typename T, bool SIGNED>
static int launch_quantize(QuantizeParams p, cudaStream_t st) {
    const bool vectors = (uintptr_t)p.x % 16 == 0 && (p.M == 1 || p.x_row * sizeof(T) % 16 == 0) && (uintptr_t)p.codes % 8 == 0 && p.K % 8 == 0;
    if (vectors && p.K <= 8 * 8 * 512) {
        // a warp per row up to 512 values; then a CTA with two pieces per thread, four or eight where that makes more than 256 threads (so
        // that several CTAs share an SM, and one row's loads overlap another's arithmetic)
        const int pieces = p.K / 8;
        if (pieces <= 64) {
            p.threads = 32;
            const int warps = p.M >= sm_count_here() * 8 ? 8 : 1;
            const dim3 grid((unsigned)ceil_div(p.M, warps)), block((unsigned)(warps * 32));
            return pieces <= 32 ? launch_dependent(quantize_vectors_kernel<T, 1, SIGNED>, grid, block, 0, st, p)
                                : launch_dependent(quantize_vectors_kernel<T, 2, SIGNED>, grid, block, 0, st, p);
        }
        const int per = pieces <= 512 ? 2 : pieces <= 1024 ? 4 : 8;
        p.threads = ceil_div(ceil_div(pieces, per), 32) * 32;
        const dim3 grid((unsigned)p.M), block((unsigned)p.threads);
        return per == 2   ? launch_dependent(quantize_vectors_kernel<T, 2, SIGNED>, grid, block, 0, st, p)
               : per == 4 ? launch_dependent(quantize_vectors_kernel<T, 4, SIGNED>, grid, block, 0, st, p)
                          : launch_dependent(quantize_vectors_kernel<T, 8, SIGNED>, grid, block, 0, st, p);
    }
    // eight values per thread up to 256 threads, then 16, then 32
    const int per = p.K <= 8 * 256 ? 8 : p.K <= 16 * 1024 ? 16 : 32;
    p.threads = ceil_div(p.K, per) >= 1024 ? 1024 : ceil_div(ceil_div(p.K, per), 32) * 32;
    const dim3 grid((unsigned)p.M), block((unsigned)p.threads);
    if (per == 8) return launch_dependent(quantize_values_kernel<T, 8, SIGNED>, grid, block, 0, st, p);
    if (per == 16) return launch_dependent(quantize_values_kernel<T, 16, SIGNED>, grid, block, 0, st, p);
    if (p.K <= 32 * 1024) return launch_dependent(quantize_values_kernel<T, 32, SIGNED>, grid, block, 0, st, p);
    return launch_dependent(quantize_values_kernel<T, 0, SIGNED>, grid, block, 0, st, p);
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
    const QuantizeParams p{d_x, x_row_stride, d_codes, d_scale, M, K, is_signed ? -(1 << (bits - 1)) : 0,
                           is_signed ? (1 << (bits - 1)) - 1 : (1 << bits) - 1, 0};
    cudaStream_t st = (cudaStream_t)stream;
    if (x_type == HIKONV_OUT_F32) return is_signed ? launch_quantize<float, true>(p, st) : launch_quantize<float, false>(p, st);
    if (x_type == HIKONV_OUT_F16) return is_signed ? launch_quantize<__half, true>(p, st) : launch_quantize<__half, false>(p, st);
    return is_signed ? launch_quantize<__nv_bfloat16, true>(p, st) : launch_quantize<__nv_bfloat16, false>(p, st);
}
