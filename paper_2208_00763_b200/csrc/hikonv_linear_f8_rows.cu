// hikonv_linear_f8 on a few rows of x (one new token, or a handful): the weights stream by once, through registers, into the tensor instruction that
// takes its operands from there (mma.sync 16x8x32 on 8-bit floating point numbers, 32-bit sums).
//
// A warp takes 16 rows of w and up to eight rows of x.  A sum does not care for the order of its terms, so a thread's 16 bytes of a row are its
// operands for two steps, and x is read in the same order.  After the four steps of a block of 128 the sums, which began at zero, are added, times the
// block's scales, to the 32-bit sums of the whole depth.  The warps of a CTA share the depth of a tile and add their parts in shared memory, in order.
#include <cstring>

#include "hikonv_linear_f8.h"
#include "hikonv_linear_util.cuh"

namespace hikonv {

constexpr int kF8RowsWarps = 8, kF8RowsThreads = kF8RowsWarps * 32, kF8RowsAtOnce = 8;

struct F8RowsParams {
    LinearParams p;
    long long xs_row;
    int chunks, w_blocks;
    int ksplit;                          // warps that share a tile's depth: 1, 2, 4 or 8
};

template <bool X5, bool W5>
__device__ __forceinline__ void f8_mma_rows(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
#define HIKONV_MMA(ta, tb)                                                                                                      \
    asm volatile("mma.sync.aligned.m16n8k32.row.col.f32." ta "." tb ".f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};" \
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])                                                               \
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1))
    if constexpr (X5 && W5) HIKONV_MMA("e5m2", "e5m2");
    else if constexpr (X5) HIKONV_MMA("e4m3", "e5m2");
    else if constexpr (W5) HIKONV_MMA("e5m2", "e4m3");
    else HIKONV_MMA("e4m3", "e4m3");
#undef HIKONV_MMA
}

// Sixteen bytes of a row from k on (a multiple of 16); zeros behind its end, or for no row.
__device__ __forceinline__ uint4 f8_piece(const uint8_t *row, int k, int K) {
    if (!row || k >= K) return make_uint4(0, 0, 0, 0);
    uint4 v = load_ordered(reinterpret_cast<const uint4 *>(row + k));
    if (k + 16 > K) {
        uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int there = K - k - 4 * i;
            if (there < 4) w[i] = there <= 0 ? 0u : w[i] & ((1u << (8 * there)) - 1u);
        }
        v = make_uint4(w[0], w[1], w[2], w[3]);
    }
    return v;
}

template <bool X5, bool W5>
__global__ void __launch_bounds__(kF8RowsThreads, 2) linear_f8_rows_kernel(const __grid_constant__ F8RowsParams q) {
    __shared__ float part[kF8RowsWarps][16 * kF8RowsAtOnce];
    const LinearParams &p = q.p;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3, e = blockIdx.y;
    const int local = warp / q.ksplit, ks = warp % q.ksplit, n0 = (blockIdx.x * (kF8RowsWarps / q.ksplit) + local) * 16;
    const int b0 = (int)((long long)q.chunks * ks / q.ksplit), b1 = (int)((long long)q.chunks * (ks + 1) / q.ksplit);
    const uint8_t *w0 = p.w + (long long)e * p.N * p.w_row;
    const uint8_t *w[2] = {n0 + g < p.N ? w0 + (n0 + g) * p.w_row : nullptr, n0 + g + 8 < p.N ? w0 + (n0 + g + 8) * p.w_row : nullptr};
    grid_dependency_release();
    // This warp's share of its tile on its way to the second-level cache: a hint, so it need not wait for the kernel before, and it is not bounded by
    // registers as loads are.
    if (!p.offsets) {
        const int lines = min(b1 - b0, 16);
        for (int i = lane; i < 16 * lines; i += 32) {
            const int n = n0 + (i & 15);
            const long long k = (long long)(b0 + (i >> 4)) * 128;
            if (n < p.N && k < p.K) asm volatile("prefetch.global.L2 [%0];" ::"l"(w0 + n * p.w_row + k));
        }
    }
    grid_dependency_wait();
    const int2 range = group_rows(p, e);
    const float *ws = p.w_scale + ((long long)e * q.w_blocks + min(n0 / 128, q.w_blocks - 1)) * q.chunks;
    const int m0 = range.x, rows = min(kF8RowsAtOnce, range.y - m0);
    if (rows <= 0) return;
    const uint8_t *x = g < rows ? p.x + (m0 + g) * p.x_row : nullptr;
    float sum[4] = {};
    // blocks whose loads are on their way at once: 4096 x 4096 weights 6.2 us with four, 6.3 with two, 6.6 with one and three CTAs per SM
#pragma unroll 4
    for (int b = b0; b < b1; ++b) {
        const int k = b * 128 + t * 16;
        uint4 wv[2][2], xv[2];
        float s[2], c[4] = {};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            wv[h][0] = f8_piece(w[0], k + 64 * h, p.K);
            wv[h][1] = f8_piece(w[1], k + 64 * h, p.K);
            xv[h] = f8_piece(x, k + 64 * h, p.K);
        }
        const float sw = load_ordered(ws + b);
#pragma unroll
        for (int i = 0; i < 2; ++i) s[i] = 2 * t + i < rows ? load_ordered(p.x_scale + b * q.xs_row + m0 + 2 * t + i) * sw : 0.f;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            f8_mma_rows<X5, W5>(c, wv[h][0].x, wv[h][1].x, wv[h][0].y, wv[h][1].y, xv[h].x, xv[h].y);
            f8_mma_rows<X5, W5>(c, wv[h][0].z, wv[h][1].z, wv[h][0].w, wv[h][1].w, xv[h].z, xv[h].w);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] = fmaf(c[i], s[i & 1], sum[i]);
    }
    // rows g and g + 8 of the tile, rows 2 t and 2 t + 1 of x
#pragma unroll
    for (int i = 0; i < 4; ++i) part[warp][(2 * t + (i & 1)) * 16 + g + (i >> 1) * 8] = sum[i];
    __syncthreads();
    const int threads = q.ksplit * 32, who = tid % threads, n = n0 + (who & 15);
    for (int i = who; i < rows * 16 && n < p.N; i += threads) {
        float v = 0.f;
        for (int k = 0; k < q.ksplit; ++k) v += part[local * q.ksplit + k][i];
        const long long m = m0 + (i >> 4);
        if (p.bias) v += load_ordered((const float *)p.bias + (long long)e * p.N + n);
        v = activate(v, p.act);
        auto put = [&](auto zero) {
            using T = decltype(zero);
            if (p.residual) v += to_float(load_ordered((const T *)p.residual + m * p.res_row + n));
            from_float(v, (T *)p.out + m * p.out_row + n);
        };
        if (p.out_type == HIKONV_OUT_F32) put(float());
        else if (p.out_type == HIKONV_OUT_F16) put(__half());
        else put(__nv_bfloat16());
    }
}

// Where this kernel is the faster one, by what was measured on weights from memory.  Up to eight rows in all, so that a weight is read once however rows
// fall to groups (512 rows of 64 groups took 8 us here spread evenly and 248 in one group, 64 times eight of them; tiles take 9 and 6).  Plain, eight rows: 1024 x
// 1024 weights 2.2 us here, 4.7 by tiles; 2048 x 2048 3.5 and 6; 4096 x 4096 6.6 and 8.0; 4608 x 4096, whose CTAs are all that the GPU holds at once, 9.2 and
// 9.2; 5632 x 4096 10.0 and 9.7; 8192 x 8192 20 and 16.5, where the copies of the tiles keep more bytes on their way than the registers here.  Groups, eight
// rows: four of 2048 x 2048 6.7 and 8.7, five 10.9 and 9.1; 64 of 512 x 512 4.8 and 5.4; 16 of 1024 x 1024 6.1 and 6.8, 32 9.4 and 6.8.
bool linear_f8_rows_takes(const LinearParams &p) { return p.M <= kF8RowsAtOnce && (double)p.E * p.N * p.K <= 1 << 24; }

int launch_linear_f8_rows(const LinearParams &p, int x_f8, int w_f8, long long xs_row, cudaStream_t st) {
    F8RowsParams q;
    memset(&q, 0, sizeof(q));
    q.p = p;
    q.xs_row = xs_row;
    q.chunks = (p.K - 1) / 128 + 1;
    q.w_blocks = ceil_div(p.N, 128);
    const int tiles = ceil_div(p.N, 16);
    // All warps of a CTA on one tile, but no more CTAs than the GPU holds at once: each that comes later waits for its first weights anew.
    q.ksplit = kF8RowsWarps;
    while (q.ksplit > 1 && (long long)tiles * p.E * q.ksplit > (long long)sm_count_here() * 2 * kF8RowsWarps) q.ksplit /= 2;
    const dim3 grid((unsigned)ceil_div(tiles, kF8RowsWarps / q.ksplit), (unsigned)p.E);
    auto launch = [&](auto kernel) { return launch_dependent(kernel, grid, dim3(kF8RowsThreads), 0, st, q); };
    if (x_f8 == HIKONV_F8_E5M2) return w_f8 == HIKONV_F8_E5M2 ? launch(linear_f8_rows_kernel<true, true>) : launch(linear_f8_rows_kernel<true, false>);
    return w_f8 == HIKONV_F8_E5M2 ? launch(linear_f8_rows_kernel<false, true>) : launch(linear_f8_rows_kernel<false, false>);
}

}  // namespace hikonv
