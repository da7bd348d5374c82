// hikonv_quantize_rows: rows of floats to codes with one scale per row.
//
// A row is read once: its values stay in registers between the maximum and the divisions.  The call is a stream (2 or 4 bytes in
// and one out per value), bound by HBM for many rows and by latency for one.
//
// The division is that of the definition, rounded to nearest in 32 bits, and a code is its rounded quotient.  It is done by the scale's
// reciprocal and two corrections, by instructions that take two values, without a branch: between bf16 values exact halves are so frequent
// that a test for open codes found one in every second warp.  4096 x 16384 bf16 values: 85 us with a library division each and the row
// read twice, 60 with the row in registers, 44 by a rounded product and a division where that left a code open, 38 to 39 now (5.2 TB/s), about
// 11 instructions per value at 57 % of the issue rate; as fp32 53 us (6.3 TB/s, as fast as a copy).
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
// The same by the rounded reciprocal, two values at a time, for a finite row and a scale in the range that RowScale names.  Two steps
// after Markstein (Computation of elementary functions on the IBM RISC System/6000 processor, 1990): q' = q + (v - q s) / s, with the
// remainder by a fused multiply-add and 1 / s by its rounded value y.  The product v y is within 1.5 steps of v / s; after the first step
// q is off by at most 1/2 + 2^-22 steps u, its remainder is exact, and the second rounds v / s + e with |e| <= (1/2 + 2^-22) u s |1/s - y|.
// For s in [1, 2) that is below (1/2 + 2^-22) u s 2^-25, while v / s, a quotient of 24-bit numbers, lies at least u 2^-24 / s from any
// point between two floats: the same rounding for s^2 (1/2 + 2^-22) < 2, that is for all but the last few mantissas.
// Adding 1.5 * 2^23 rounds to the nearest whole number, ties to even, and leaves the code in the low byte.  Bounds are needed below zero
// for unsigned codes alone: the largest value's quotient rounds to hi or to a float next to it.
__device__ __forceinline__ uint64_t pair(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
template <bool SIGNED>
__device__ __forceinline__ void quantize_two(float v0, float v1, uint64_t minus_scale, uint64_t inverse, uint32_t &o0, uint32_t &o1) {
    const uint64_t v = SIGNED ? pair(v0, v1) : pair(fmaxf(v0, 0.f), fmaxf(v1, 0.f));
    uint64_t q, lifted;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(q) : "l"(v), "l"(inverse));
    q = fma_pair(fma_pair(q, minus_scale, v), inverse, q);
    q = fma_pair(fma_pair(q, minus_scale, v), inverse, q);
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(lifted) : "l"(q), "l"(pair(12582912.f, 12582912.f)));
    asm("mov.b64 {%0, %1}, %2;" : "=r"(o0), "=r"(o1) : "l"(lifted));
}

// A row's scale, and how its codes are found.
struct RowScale {
    float scale, inverse, lo, hi;
    bool quick;
    __device__ __forceinline__ RowScale(float top, const QuantizeParams &p) {
        scale = __fdiv_rn(top, (float)p.hi);
        inverse = __frcp_rn(scale);
        lo = (float)p.lo;
        hi = (float)p.hi;
        // remainders far from underflow, and a mantissa at least sixteen steps below 2
        quick = scale >= 0x1p-64f && scale <= 0x1p64f && (__float_as_uint(scale) & 0x7FFFF0u) != 0x7FFFF0u;
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

// VECS pieces of eight values per thread, in registers.  Pieces are taken from 16-byte boundaries.  Unless ALIGNED (every row starts on one,
// codes on an 8-byte one), a row begins `lead` values into its first piece, and what lies in front of it or behind its end is left out;
// its codes are moved into aligned words with the help of the lane before, which has the bytes that a word begins with.
template <typename T, int VECS, bool SIGNED, bool ALIGNED>
__global__ void __launch_bounds__(512, VECS >= 4 && sizeof(T) == 4 ? 1 : 2) quantize_pieces_kernel(const QuantizeParams p) {
    constexpr int WORDS = sizeof(T) * 2;                // of eight values
    __shared__ float part[32];
    grid_dependency_release();
    grid_dependency_wait();
    const int lane = threadIdx.x & 31, at = p.threads == 32 ? lane : threadIdx.x;
    const int row = p.threads == 32 ? blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32 : blockIdx.x;
    if (row >= p.M) return;                             // whole warps; rows of a whole CTA are all there
    const T *x = (const T *)p.x + row * p.x_row;
    const int lead = ALIGNED ? 0 : (int)((uintptr_t)x & 15) / (int)sizeof(T);
    auto whole = [&](int j) { return j * 8 - lead >= 0 && j * 8 - lead + 8 <= p.K; };
    uint32_t v[VECS][WORDS];
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
        const int j = at + i * p.threads, k0 = j * 8 - lead;
#pragma unroll
        for (int h = 0; h < WORDS; ++h) v[i][h] = 0;
        if (whole(j)) {
#pragma unroll
            for (int h = 0; h < WORDS / 4; ++h) {
                const uint4 o = load_ordered(reinterpret_cast<const uint4 *>(x + k0) + h);
                v[i][4 * h] = o.x; v[i][4 * h + 1] = o.y; v[i][4 * h + 2] = o.z; v[i][4 * h + 3] = o.w;
            }
        } else if (!ALIGNED) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k0 + k >= 0 && k0 + k < p.K) {
                    if constexpr (sizeof(T) == 4) v[i][k] = __float_as_uint(load_ordered((const float *)x + k0 + k));
                    else v[i][k / 2] |= (uint32_t)load_ordered((const unsigned short *)x + k0 + k) << (16 * (k & 1));
                }
        }
    }
    auto value = [&](int i, int k) {
        if constexpr (sizeof(T) == 4) return __uint_as_float(v[i][k]);
        else if constexpr (std::is_same<T, __nv_bfloat16>::value) return __uint_as_float(k & 1 ? v[i][k / 2] & 0xFFFF0000u : v[i][k / 2] << 16);
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
    const uint64_t minus_scale = pair(-by.scale, -by.scale), inverse = pair(by.inverse, by.inverse);
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
        const int j = at + i * p.threads, k0 = j * 8 - lead;
        uint32_t o[8];
        if (by.quick) {
#pragma unroll
            for (int k = 0; k < 8; k += 2) quantize_two<SIGNED>(value(i, k), value(i, k + 1), minus_scale, inverse, o[k], o[k + 1]);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) o[k] = quantize_exactly(value(i, k), by.scale, by.lo, by.hi);
        }
        auto four = [&](int k) { return byte_permute(byte_permute(o[k], o[k + 1], 0x0040), byte_permute(o[k + 2], o[k + 3], 0x0040), 0x5410); };
        const uint32_t low = four(0), high = four(4);
        int8_t *to = p.codes + (size_t)row * p.K + k0;
        if constexpr (ALIGNED) {
            if (whole(j)) *reinterpret_cast<uint2 *>(to) = make_uint2(low, high);
        } else {
            const uint32_t before = __shfl_up_sync(0xFFFFFFFFu, high, 1);
            const int off = (int)((uintptr_t)to & 3);
            if (whole(j)) {
                uint32_t *word = reinterpret_cast<uint32_t *>(to - off);
                const bool joined = off == 0 || (lane > 0 && whole(j - 1)), joins = off == 0 || (lane < 31 && whole(j + 1));
                if (joined) word[0] = __funnelshift_l(before, low, 8 * off);
                else
                    for (int b = 0; b < 4 - off; ++b) to[b] = (int8_t)(low >> (8 * b));
                word[1] = __funnelshift_l(low, high, 8 * off);
                if (!joins)
                    for (int b = 4 - off; b < 4; ++b) to[4 + b] = (int8_t)(high >> (8 * b));
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (k0 + k >= 0 && k0 + k < p.K) to[k] = (int8_t)o[k];
            }
        }
    }
}

// Longer rows, of any alignment: a CTA reads its row twice, the second time from the caches.
template <typename T, bool SIGNED>
__global__ void __launch_bounds__(1024) quantize_long_kernel(const QuantizeParams p) {
    __shared__ float part[32];
    grid_dependency_release();
    grid_dependency_wait();
    const int row = blockIdx.x;
    const uint32_t K = p.K;                             // unsigned: up to a CTA's threads beyond 2^31 - 1
    const T *x = (const T *)p.x + row * p.x_row;
    int8_t *codes = p.codes + (size_t)row * p.K;
    float top = 0.f;
    for (uint32_t k = threadIdx.x; k < K; k += p.threads) {
        const float a = quantize_float(load_ordered(x + k));
        top = max_nan(top, SIGNED ? fabsf(a) : a);
    }
    top = row_max(top, p.threads, part);
    const RowScale by(top, p);
    if (threadIdx.x == 0) p.scale[row] = by.scale;
    const uint64_t minus_scale = pair(-by.scale, -by.scale), inverse = pair(by.inverse, by.inverse);
    for (uint32_t k = threadIdx.x; k < K; k += p.threads) {
        const float a = quantize_float(load_ordered(x + k));
        uint32_t c, none;
        if (by.quick) quantize_two<SIGNED>(a, 0.f, minus_scale, inverse, c, none);
        else c = quantize_exactly(a, by.scale, by.lo, by.hi);
        codes[k] = (int8_t)c;
    }
}

template <typename T, bool SIGNED, bool ALIGNED>
static int launch_pieces(QuantizeParams p, cudaStream_t st) {
    // A warp per row up to 64 pieces; then a CTA with two pieces per thread, four or eight where that makes more than 256 threads (so that
    // several CTAs share an SM, and one row's loads overlap another's arithmetic).
    const int pieces = ALIGNED ? p.K / 8 : (p.K + 14) / 8;                  // a row may begin seven values into its first
    if (pieces <= 64) {
        p.threads = 32;
        const int warps = p.M >= sm_count_here() * 8 ? 8 : 1;
        const dim3 grid((unsigned)((p.M - 1) / warps + 1)), block((unsigned)(warps * 32));
        return pieces <= 32 ? launch_dependent(quantize_pieces_kernel<T, 1, SIGNED, ALIGNED>, grid, block, 0, st, p)
                            : launch_dependent(quantize_pieces_kernel<T, 2, SIGNED, ALIGNED>, grid, block, 0, st, p);
    }
    const int per = pieces <= 512 ? 2 : pieces <= 1024 ? 4 : 8;
    p.threads = ceil_div(ceil_div(pieces, per), 32) * 32;
    const dim3 grid((unsigned)p.M), block((unsigned)p.threads);
    return per == 2   ? launch_dependent(quantize_pieces_kernel<T, 2, SIGNED, ALIGNED>, grid, block, 0, st, p)
           : per == 4 ? launch_dependent(quantize_pieces_kernel<T, 4, SIGNED, ALIGNED>, grid, block, 0, st, p)
                      : launch_dependent(quantize_pieces_kernel<T, 8, SIGNED, ALIGNED>, grid, block, 0, st, p);
}

template <typename T, bool SIGNED>
static int launch_quantize(QuantizeParams p, cudaStream_t st) {
    constexpr int most = 8 * 8 * 512;                   // values that 512 threads hold
    const bool aligned = (uintptr_t)p.x % 16 == 0 && (p.M == 1 || p.x_row * sizeof(T) % 16 == 0) && (uintptr_t)p.codes % 8 == 0 && p.K % 8 == 0;
    if (aligned && p.K <= most) return launch_pieces<T, SIGNED, true>(p, st);
    if (p.K <= most - 16) return launch_pieces<T, SIGNED, false>(p, st);
    p.threads = 1024;
    return launch_dependent(quantize_long_kernel<T, SIGNED>, dim3((unsigned)p.M), dim3(1024), 0, st, p);
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
