// hikonv_quantize_blocks, hikonv_quantize_tiles: floats to 8-bit floating point numbers with a scale for each block of 128, or tile of
// 128 x 128.
//
// A row is read once: a block's values stay in the registers of eight lanes between its maximum and the divisions, and are stored once
// for each place that the row goes to.  Bound by the bytes: 2 or 4 read per value and 1 written per place.  8192 x 8192 bf16 values: 39 us
// (5.2 TB/s), 51 by a library division each; eight values a lane instead of sixteen 14 us more.  8192 x 4096 to eight places each: 65 us, of which ten are
// the scales, four bytes at a time into lines that other rows share.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <type_traits>

#include "hikonv_cuda.cuh"
#include "hikonv_linear.h"
#include "hikonv_pairs.cuh"

namespace hikonv {

constexpr int kF8Block = 128, kF8PerLane = 16, kF8Lanes = kF8Block / kF8PerLane;

struct BlocksParams {
    const void *x;
    long long x_row;                     // elements
    uint8_t *values;
    long long values_row;                // bytes
    float *scale;
    long long scale_row;                 // elements
    const int32_t *slots;                // null: rows stay where they are
    int M, K, blocks, k, R;
};

__device__ __forceinline__ float f8_float(float v) { return v; }
__device__ __forceinline__ float f8_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float f8_float(__nv_bfloat16 v) { return __bfloat162float(v); }
// The larger of two magnitudes; a NaN wins.
__device__ __forceinline__ float f8_max(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
template <bool E5M2> constexpr float kF8Most = E5M2 ? 57344.f : 448.f;

// Two quotients to two bytes, the first in the low one.  Quotients are at most the type's largest number and one step of 2^-24, which rounds to it; more
// where the scale is subnormal and was rounded down (the smallest bf16 number, 2^-133, to E5M2 has scale 2^-149 and quotient 65536), and then saturate.
template <bool E5M2>
__device__ __forceinline__ uint32_t f8_pair(float a, float b) {
    return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, E5M2 ? __NV_E5M2 : __NV_E4M3);
}
// Quotients of a block whose scale is `scale`; a block of zeros stays one.
__device__ __forceinline__ float f8_quotient(float v, float scale) { return scale == 0.f ? 0.f : __fdiv_rn(v, scale); }

// Sixteen values of a row from k on, as floats; zeros behind its end.
template <typename T, bool ALIGNED>
__device__ __forceinline__ void f8_read(const T *row, int k, int K, float (&v)[kF8PerLane]) {
    if (ALIGNED && k + kF8PerLane <= K) {
        constexpr int PER = 16 / sizeof(T);
        struct alignas(16) Pack { T v[PER]; };
#pragma unroll
        for (int i = 0; i < kF8PerLane / PER; ++i) {
            const Pack o = load_ordered(reinterpret_cast<const Pack *>(row + k) + i);
#pragma unroll
            for (int j = 0; j < PER; ++j) v[i * PER + j] = f8_float(o.v[j]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kF8PerLane; ++i) v[i] = k + i < K ? f8_float(load_ordered(row + k + i)) : 0.f;
    }
}
template <bool E5M2>
__device__ __forceinline__ uint4 f8_codes(const float (&v)[kF8PerLane], float scale) {
    uint32_t o[4];
    if (divides_quickly(scale)) {
        const float y = __frcp_rn(scale);
        const uint64_t minus = pair(-scale, -scale), inverse = pair(y, y);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float a, b, c, d;
            unpair(quotient_pair(pair(v[4 * i], v[4 * i + 1]), minus, inverse), a, b);
            unpair(quotient_pair(pair(v[4 * i + 2], v[4 * i + 3]), minus, inverse), c, d);
            o[i] = f8_pair<E5M2>(a, b) | f8_pair<E5M2>(c, d) << 16;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            o[i] = f8_pair<E5M2>(f8_quotient(v[4 * i], scale), f8_quotient(v[4 * i + 1], scale)) |
                   f8_pair<E5M2>(f8_quotient(v[4 * i + 2], scale), f8_quotient(v[4 * i + 3], scale)) << 16;
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
}
// Sixteen bytes of a row from k on (a multiple of 16), without those behind its end.
__device__ __forceinline__ void f8_write(uint8_t *row, int k, int K, const uint4 &o) {
    if (k + kF8PerLane <= K) {
        *reinterpret_cast<uint4 *>(row + k) = o;
    } else {
        const uint32_t w[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
        for (int i = 0; i < kF8PerLane; ++i)
            if (k + i < K) row[k + i] = (uint8_t)(w[i / 4] >> (8 * (i & 3)));
    }
}

// Block: (lanes along a row, rows).
template <typename T, bool E5M2, bool ALIGNED>
__global__ void __launch_bounds__(256) quantize_blocks_kernel(const BlocksParams p) {
    grid_dependency_release();
    grid_dependency_wait();
    const int m = blockIdx.x * blockDim.y + threadIdx.y, unit = blockIdx.y * blockDim.x + threadIdx.x;
    const bool inside = m < p.M && unit < p.blocks * kF8Lanes;          // the same for the lanes of a block
    const int k = unit * kF8PerLane;
    float v[kF8PerLane];
    float top = 0.f;
    if (inside) {
        f8_read<T, ALIGNED>((const T *)p.x + m * p.x_row, k, p.K, v);
#pragma unroll
        for (int i = 0; i < kF8PerLane; ++i) top = f8_max(top, fabsf(v[i]));
    }
#pragma unroll
    for (int d = kF8Lanes / 2; d; d /= 2) top = f8_max(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
    if (!inside) return;
    const float scale = __fdiv_rn(top, kF8Most<E5M2>);
    const uint4 o = f8_codes<E5M2>(v, scale);
    auto put = [&](long long row) {
        if (k < p.K) f8_write(p.values + row * p.values_row, k, p.K, o);
        if (unit % kF8Lanes == 0) p.scale[unit / kF8Lanes * p.scale_row + row] = scale;
    };
    if (!p.slots) {
        put(m);
        return;
    }
    const int32_t *slots = p.slots + (long long)m * p.k;
    for (int j = 0; j < p.k; ++j) {
        const int s = load_ordered(slots + j);
        if (s >= 0 && s < p.R) put(s);
    }
}

// A CTA per tile: the largest magnitude, then the quotients, from the caches.
struct TilesParams {
    const void *w;
    long long w_row, values_row;
    uint8_t *values;
    float *scale;
    int N, K, n_blocks, k_blocks;
};
template <typename T, bool E5M2>
__global__ void __launch_bounds__(256) quantize_tiles_kernel(const TilesParams p) {
    __shared__ float part[8];
    grid_dependency_release();
    grid_dependency_wait();
    const long long tile = blockIdx.x, e = tile / ((long long)p.n_blocks * p.k_blocks);
    const int kb = (int)(tile % p.k_blocks), nb = (int)(tile / p.k_blocks % p.n_blocks);
    const int k = kb * kF8Block + threadIdx.x % kF8Lanes * kF8PerLane;
    float v[kF8PerLane], top = 0.f;
    auto each = [&](auto f) {
        for (int r = threadIdx.x / kF8Lanes; r < kF8Block; r += 256 / kF8Lanes)
            if (nb * kF8Block + r < p.N) f(e * p.N + nb * kF8Block + r);
    };
    each([&](long long row) {
        f8_read<T, false>((const T *)p.w + row * p.w_row, k, p.K, v);
#pragma unroll
        for (int i = 0; i < kF8PerLane; ++i) top = f8_max(top, fabsf(v[i]));
    });
#pragma unroll
    for (int d = 16; d; d /= 2) top = f8_max(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
    if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = top;
    __syncthreads();
    for (int i = 0; i < 8; ++i) top = f8_max(top, part[i]);
    const float scale = __fdiv_rn(top, kF8Most<E5M2>);
    if (threadIdx.x == 0) p.scale[tile] = scale;
    each([&](long long row) {
        f8_read<T, false>((const T *)p.w + row * p.w_row, k, p.K, v);
        if (k < p.K) f8_write(p.values + row * p.values_row, k, p.K, f8_codes<E5M2>(v, scale));
    });
}

template <typename F>
static int with_f8_types(int x_type, int f8_type, F f) {
    auto second = [&](auto t) { return f8_type == HIKONV_F8_E5M2 ? f(t, std::true_type()) : f(t, std::false_type()); };
    return x_type == HIKONV_OUT_F32 ? second(float()) : x_type == HIKONV_OUT_F16 ? second(__half()) : second(__nv_bfloat16());
}
static bool f8_types_ok(int x_type, int f8_type) {
    return (x_type == HIKONV_OUT_F32 || x_type == HIKONV_OUT_F16 || x_type == HIKONV_OUT_BF16) && (f8_type == HIKONV_F8_E4M3 || f8_type == HIKONV_F8_E5M2);
}

}  // namespace hikonv

using namespace hikonv;

extern "C" int hikonv_quantize_blocks(const void *d_x, int x_type, long long x_row_stride, int M, int K, int f8_type, const int32_t *d_slots, int k, int R,
                                      uint8_t *d_values, long long values_row_stride, float *d_scale, long long scale_row_stride, void *stream) {
    if (!f8_types_ok(x_type, f8_type) || M < 0 || K < 1 || (d_slots ? k < 1 || R < 0 : k != 0 || R != 0)) return HIKONV_ERR_INVALID_ARG;
    if ((long long)M * (d_slots ? k : 1) > (1 << 30) || K > (1 << 26)) return HIKONV_ERR_UNSUPPORTED;
    const long long rows = d_slots ? R : M, size = x_type == HIKONV_OUT_F32 ? 4 : 2, blocks = (K - 1) / kF8Block + 1;
    if (M == 0 || rows == 0) return HIKONV_OK;
    if (M == 1) x_row_stride = K;
    if (rows == 1) values_row_stride = (long long)align_up(K, 16);
    if (blocks == 1) scale_row_stride = rows;
    // a stride of 0: all rows are one
    if (!d_x || !d_values || !d_scale || x_row_stride < 0 || x_row_stride > (1ll << 40) || values_row_stride < K || values_row_stride > (1ll << 40) ||
        scale_row_stride < rows || scale_row_stride > (1ll << 40))
        return HIKONV_ERR_INVALID_ARG;
    if ((uintptr_t)d_x % size || (uintptr_t)d_scale % 4 || (uintptr_t)d_slots % 4) return HIKONV_ERR_INVALID_ARG;
    if ((uintptr_t)d_values % 16 || values_row_stride % 16) return HIKONV_ERR_UNSUPPORTED;
    const size_t slot_bytes = d_slots ? (size_t)M * k * 4 : 0;
    if (rows_overlap(d_values, values_row_stride, K, rows, d_x, x_row_stride * size, K * size, M) ||
        rows_overlap(d_scale, scale_row_stride * 4, rows * 4, blocks, d_x, x_row_stride * size, K * size, M) ||
        rows_overlap(d_values, values_row_stride, K, rows, d_scale, scale_row_stride * 4, rows * 4, blocks) ||
        rows_overlap(d_values, values_row_stride, K, rows, d_slots, slot_bytes, slot_bytes, 1) ||
        rows_overlap(d_scale, scale_row_stride * 4, rows * 4, blocks, d_slots, slot_bytes, slot_bytes, 1))
        return HIKONV_ERR_INVALID_ARG;
    const BlocksParams p{d_x, x_row_stride, d_values, values_row_stride, d_scale, scale_row_stride, d_slots, M, K, (int)blocks, k, R};
    const bool aligned = (uintptr_t)d_x % 16 == 0 && x_row_stride * size % 16 == 0;
    int along = kF8Lanes;
    while (along < 256 && along < blocks * kF8Lanes) along *= 2;
    const dim3 block((unsigned)along, (unsigned)(256 / along));
    const dim3 grid((unsigned)((M - 1) / block.y + 1), (unsigned)((blocks * kF8Lanes + along - 1) / along));
    cudaStream_t st = (cudaStream_t)stream;
    return with_f8_types(x_type, f8_type, [&](auto t, auto e5m2) {
        using T = decltype(t);
        constexpr bool E5M2 = decltype(e5m2)::value;
        return aligned ? launch_dependent(quantize_blocks_kernel<T, E5M2, true>, grid, block, 0, st, p)
                       : launch_dependent(quantize_blocks_kernel<T, E5M2, false>, grid, block, 0, st, p);
    });
}

extern "C" int hikonv_quantize_tiles(const void *d_w, int w_type, long long w_row_stride, int E, int N, int K, int f8_type, uint8_t *d_values,
                                     long long values_row_stride, float *d_scale, void *stream) {
    if (!f8_types_ok(w_type, f8_type) || E < 1 || N < 1 || K < 1) return HIKONV_ERR_INVALID_ARG;
    const long long rows = (long long)E * N, size = w_type == HIKONV_OUT_F32 ? 4 : 2, n_blocks = (N - 1) / kF8Block + 1, k_blocks = (K - 1) / kF8Block + 1;
    if (rows > 0x7FFFFFFFll || K > (1 << 26) || E * n_blocks * k_blocks > 0x7FFFFFFFll) return HIKONV_ERR_UNSUPPORTED;
    if (rows == 1) w_row_stride = K, values_row_stride = (long long)align_up(K, 16);
    if (!d_w || !d_values || !d_scale || w_row_stride < 0 || w_row_stride > (1ll << 40) || values_row_stride < K || values_row_stride > (1ll << 40))
        return HIKONV_ERR_INVALID_ARG;
    if ((uintptr_t)d_w % size || (uintptr_t)d_scale % 4) return HIKONV_ERR_INVALID_ARG;
    if ((uintptr_t)d_values % 16 || values_row_stride % 16) return HIKONV_ERR_UNSUPPORTED;
    const size_t scales = (size_t)(E * n_blocks * k_blocks) * 4;
    if (rows_overlap(d_values, values_row_stride, K, rows, d_w, w_row_stride * size, K * size, rows) ||
        rows_overlap(d_scale, scales, scales, 1, d_w, w_row_stride * size, K * size, rows) || rows_overlap(d_scale, scales, scales, 1, d_values, values_row_stride, K, rows))
        return HIKONV_ERR_INVALID_ARG;
    const TilesParams p{d_w, w_row_stride, values_row_stride, d_values, d_scale, N, K, (int)n_blocks, (int)k_blocks};
    cudaStream_t st = (cudaStream_t)stream;
    return with_f8_types(w_type, f8_type, [&](auto t, auto e5m2) {
        return launch_dependent(quantize_tiles_kernel<decltype(t), decltype(e5m2)::value>, dim3((unsigned)(E * n_blocks * k_blocks)), dim3(256), 0, st, p);
    });
}
