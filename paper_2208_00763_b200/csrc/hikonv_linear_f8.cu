// hikonv_linear_f8, hikonv_grouped_linear_f8: matrix products of 8-bit floating point numbers with a scale for each block of 128 along the
// depth, on the tensor cores (tcgen05.mma kind::f8f6f4, 32-bit sums in tensor memory), operands staged in shared memory by TMA.
//
// A step is a block of 128: its products are summed by the tensor cores from zero, and warps of their own take the sums from tensor memory
// and add them, times x_scale[b][m] w_scale[n / 128][b], to 32-bit sums in registers while the next blocks are multiplied.
//
// The 128 lanes of tensor memory are rows of x on long inputs (TOKENS: a lane has one scale per step, and a thread's sums are
// neighbours in a row of the output) and output columns where rows are few (the number of rows is then that of the instruction's
// columns, any multiple of 16, and the CTAs of a cluster may share the depth of a tile).
//
// One CTA per SM walks over the tiles.  Warp 0 loads, warp 1 multiplies, warp 2 brings the scales, warps 4 to 11 add up and finish.
#include <atomic>
#include <cstddef>
#include <cstring>

#include "hikonv_linear_f8.h"
#include "hikonv_linear_tiles.cuh"

namespace hikonv {

constexpr int kF8Rows = 128, kF8Depth = 128;
constexpr int kF8MostStages = 12, kF8MostAccs = 4;
constexpr int kF8FirstAdder = 4, kF8Adders = 8, kF8Threads = (kF8FirstAdder + kF8Adders) * 32;
constexpr size_t kF8MostSmem = 226 * 1024;

struct F8Params {
    LinearParams p;
    long long xs_row;                    // elements from block to block of x_scale
    int nt, width;                       // rows of x and output columns per tile
    int m_tiles, n_blocks, tokens_first;
    int chunks, w_blocks;                // blocks of the depth; of the output columns, 128 each
    int splits, split_shift;
    int stages, stage_bytes, b_off;
    int acc_cols, accs, tmem_cols;
    uint32_t idesc;
    int feed_off, turn_off, held;        // behind the stages: the adders' scales; their buffers for turning outputs; the tables of the groups
    int whole_stores;                    // rows of out and residual on 32-byte boundaries
    long long wait_cycles;
};


static __device__ unsigned int linear_f8_timeouts;

__device__ __forceinline__ void f8_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a),
                 "l"(b), "r"(idesc), "r"(accumulate)
                 : "memory");
}
__device__ __forceinline__ void f8_load(uint32_t taddr, uint32_t (&v)[8]) { tc_load_columns(taddr, v); }
__device__ __forceinline__ void f8_load(uint32_t taddr, uint32_t (&v)[16]) { tc_load16(taddr, v); }
__device__ __forceinline__ void f8_load(uint32_t taddr, uint32_t (&v)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,"
                 "%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
                   "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]),
                   "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]),
                   "=r"(v[30]), "=r"(v[31])
                 : "r"(taddr));
}
// The wait for tcgen05.ld, which what it loaded goes through: no arithmetic on it can be moved in front.
template <int N>
__device__ __forceinline__ void f8_loaded(uint32_t (&v)[N]) {
    tc_wait_load();
#pragma unroll
    for (int i = 0; i < N; i += 8)
        asm volatile("" : "+r"(v[i]), "+r"(v[i + 1]), "+r"(v[i + 2]), "+r"(v[i + 3]), "+r"(v[i + 4]), "+r"(v[i + 5]), "+r"(v[i + 6]), "+r"(v[i + 7]));
}
__device__ __forceinline__ uint64_t f8_two(uint32_t a, uint32_t b) { return (uint64_t)b << 32 | a; }
__device__ __forceinline__ uint64_t f8_two(float a, float b) { return f8_two(__float_as_uint(a), __float_as_uint(b)); }
__device__ __forceinline__ uint64_t f8_fma(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t f8_mul(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float f8_low(uint64_t v) { return __uint_as_float((uint32_t)v); }
__device__ __forceinline__ float f8_high(uint64_t v) { return __uint_as_float((uint32_t)(v >> 32)); }
__device__ __forceinline__ void cp_async_4_at(uint32_t to, const float *from) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ float4 load_cluster_float4(uint32_t remote) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(remote));
    return v;
}
__device__ __forceinline__ void load_global32(const void *a, uint32_t (&v)[8]) {
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
                 : "l"(a)
                 : "memory");
}
__device__ __forceinline__ void store_global32(void *a, const uint32_t (&v)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(a), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]),
                 "r"(v[7])
                 : "memory");
}

__device__ __forceinline__ bool f8_wait(const F8Params &q, uint32_t bar, uint32_t parity) {
    if (__all_sync(0xFFFFFFFFu, mbarrier_try_wait(bar, parity))) return true;
    return __all_sync(0xFFFFFFFFu, mbarrier_wait(bar, parity, q.wait_cycles));
}

// Waits until every stage that the loads up to here, of which the ring holds the next, have filled is free again: all copies have landed and all
// multiplies of them have ended and arrived.  A stage that was never filled counts as free.
__device__ __forceinline__ bool f8_stages_free(const F8Params &q, Ring ring, uint32_t empty) {
    bool fine = true;
    for (int i = 0; fine && i < q.stages; ++i) {
        fine = f8_wait(q, empty + 8 * ring.stage, ring.phase ^ 1);
        ring.next(q.stages);
    }
    return fine;
}

// ---- scales
//
// The scales of x and w that a tile's steps need come to shared memory by asynchronous copies of four bytes (rows of scales begin anywhere), a few steps at
// a time, by a warp of their own, which runs ahead as far as the ring allows and waits for no copy: the copies themselves arrive at the slot's
// barrier.  Asked for by the warps that add up, a step's scales took them 150 cycles.
constexpr int kScaleBatch = 4, kScaleSlots = 4;         // steps of a slot; slots
constexpr int kScaleBytes = (kScaleBatch * kF8Rows + kScaleBatch) * 4;           // of a slot: [step][row of x], then [step] of w
struct ScaleBars {
    uint64_t full[kScaleSlots], empty[kScaleSlots];
};

// `rows` rows of x from row0 on; the scales of the tile's output columns at w.
__device__ __forceinline__ bool bring_scales(const F8Params &q, Ring &ring, uint32_t slots, uint32_t full, uint32_t empty, int row0, int rows, const float *w, int c0,
                                             int c1) {
    const int lane = threadIdx.x & 31;
    const float *xs = q.p.x_scale + c0 * q.xs_row + row0 + lane;
    for (int c = c0; c < c1; c += kScaleBatch) {
        if (!f8_wait(q, empty + 8 * ring.stage, ring.phase ^ 1)) return false;
        const uint32_t slot = slots + ring.stage * kScaleBytes;
#pragma unroll
        for (int b = 0; b < kScaleBatch; ++b) {
            if (c + b < c1) {
#pragma unroll
                for (int i = 0; i < kF8Rows; i += 32)
                    if (i + lane < rows) cp_async_4_at(slot + (b * kF8Rows + i + lane) * 4, xs + i);
            }
            xs += q.xs_row;
        }
        if (lane < kScaleBatch && c + lane < c1) cp_async_4_at(slot + (kScaleBatch * kF8Rows + lane) * 4, w + c + lane);
        asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(full + 8 * ring.stage) : "memory");
        ring.next(kScaleSlots);
    }
    return true;
}

// The reader's side, one warp: which slot and step is next.
struct ScaleRing {
    const F8Params &q;
    const uint32_t slots, full, empty;
    uint32_t beat = 0;                   // steps that slots were there for

    __device__ __forceinline__ ScaleRing(const F8Params &q_, uint32_t slots_, uint32_t full_, uint32_t empty_) : q(q_), slots(slots_), full(full_), empty(empty_) {}
    // The slot of the next step, once it has been brought; null when the wait for it ran out.
    __device__ __forceinline__ bool wait() {
        return beat % kScaleBatch != 0 || f8_wait(q, full + 8 * (beat / kScaleBatch % kScaleSlots), beat / (kScaleBatch * kScaleSlots) & 1);
    }
    __device__ __forceinline__ uint32_t xs() const { return slots + beat / kScaleBatch % kScaleSlots * kScaleBytes + beat % kScaleBatch * (kF8Rows * 4); }
    __device__ __forceinline__ uint32_t w() const {
        return slots + beat / kScaleBatch % kScaleSlots * kScaleBytes + (kScaleBatch * kF8Rows + beat % kScaleBatch) * 4;
    }
    // The step's scales have been read by this lane; `last`: of the tile.
    __device__ __forceinline__ void next(bool last) {
        const uint32_t slot = beat / kScaleBatch % kScaleSlots;
        ++beat;
        if (last) beat = (beat + kScaleBatch - 1) / kScaleBatch * kScaleBatch;
        if (beat % kScaleBatch == 0) {
            __syncwarp();
            if ((threadIdx.x & 31) == 0) mbarrier_arrive(empty + 8 * slot);
        }
    }
};
__device__ __forceinline__ float load_shared_float(uint32_t at) {
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
    return v;
}

struct F8Control {
    uint64_t full[kF8MostStages], empty[kF8MostStages], acc_full[kF8MostAccs], acc_empty[kF8MostAccs], drain;
    ScaleBars scales;
    uint32_t tmem;
    int whole;                           // no wait of this CTA has run out
};

// SiLU in front of outputs of 16 bits, as v / (1 + exp(-v)) for either sign.  -v log2(e) is rounded to z, a multiple of 2^-13 (by the sum with 1536);
// exp(-v) is 2^z (1 + e) with the rest e = -v - z ln 2, whose square is below 2^-29.  All of it is taken 2^-14 times, so that the divisor is finite and its
// reciprocal normal for every result that an output could hold, and |v| counts as 98 beyond that (the sign's and the minimum's instruction is one), which
// leaves infinite and NaN values to the last product.  Off by 2^-21.2 of the result at most over all values from -87 on (silu(): 2^-21.6), by 2^-17.4
// below, where the reciprocal times 2^-14 is subnormal (silu(): the same); measured on every one of them.  Eleven instructions a value against silu()'s
// 18, and one rounding of the whole exponent, two values to a reciprocal, has eleven, too, but is off by 2^-18 at -80: 32 groups of 16384 x 2048 x 4096 260 us
// (silu() 270, the coarse form 256).
__device__ __forceinline__ float silu_short(float v) {
    float a, t, r;
    asm("min.xorsign.abs.f32 %0, %1, %2;" : "=f"(a) : "f"(v), "f"(98.f));
    const float lifted = fmaf(a, -1.44269504f, 1536.f), e = fmaf(lifted - 1536.f, -0.693147182f, -a);
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(t) : "f"(lifted - 1550.f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(fmaf(t, e, t) + 0x1p-14f));
    return v * (r * 0x1p-14f);
}
// The activation of neighbouring values in front of an output of type T.
template <typename T, int COUNT>
__device__ __forceinline__ void activate_some(float (&v)[COUNT], int act) {
    switch (act) {
        case HIKONV_ACT_RELU:
#pragma unroll
            for (int i = 0; i < COUNT; ++i) v[i] = activate(v[i], HIKONV_ACT_RELU);
            break;
        case HIKONV_ACT_SILU:
#pragma unroll
            for (int i = 0; i < COUNT; ++i) v[i] = sizeof(T) == 2 ? silu_short(v[i]) : activate(v[i], HIKONV_ACT_SILU);
            break;
        case HIKONV_ACT_GELU:
#pragma unroll
            for (int i = 0; i < COUNT; ++i) v[i] = activate(v[i], HIKONV_ACT_GELU);
            break;
        default: break;
    }
}

// The sums of a thread, CPW neighbouring columns of its lane as pairs of floats, and what becomes of them: some at a time, after which the rest is
// moved down, so that the code for them is there once.
template <int CPW>
struct Sums {
    uint64_t sum[CPW / 2];

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < CPW / 2; ++i) sum[i] = 0;
    }
    __device__ __forceinline__ float at(int i) const { return i & 1 ? f8_high(sum[i / 2]) : f8_low(sum[i / 2]); }
    template <int COUNT>
    __device__ __forceinline__ void shift_out() {
#pragma unroll
        for (int i = 0; i + COUNT / 2 < CPW / 2; ++i) sum[i] = sum[i + COUNT / 2];
    }
    // Lanes are rows of x from row0 + quad 32 on, `rows` of them in all; columns from n on.  32 bytes of a row at once where rows begin on such a
    // boundary, else turned in shared memory, 16 columns at a time, so that neighbouring lanes write neighbouring columns.  A residual is asked for
    // before the columns in front of it are stored, or several rows at once (939 x 5002 x 3013 with bias and residual 50 us; a row at a time 76, without either
    // 36); whole rows' bias comes by a column a lane, through shared memory.
    template <typename T>
    __device__ __forceinline__ void finish_rows_as(const F8Params &q, int e, long long row0, int rows, int n, float *turn) {
        constexpr int PER = 32 / sizeof(T), SOME = CPW < 64 ? CPW : 64, ROWS = CPW < 128 ? 8 : 4;
        const LinearParams &p = q.p;
        const int lane = threadIdx.x & 31, quad = (threadIdx.x >> 5) & 3, row = quad * 32 + lane;
        const float *bias = (const float *)p.bias + (long long)e * p.N;
        if (q.whole_stores && n + CPW <= p.N) {
            T *o = (T *)p.out + (row0 + row) * p.out_row + n;
            const T *r = (const T *)p.residual + (row0 + row) * p.res_row + n;
            const bool there = row < rows;
            if (p.bias) {
                __syncwarp();
#pragma unroll
                for (int i = 0; i < CPW; i += 32) turn[i + lane] = load_ordered(bias + n + i + lane);
                __syncwarp();
            }
            union { uint32_t w[8]; T v[PER]; } x;
            const bool adds = p.residual && there;
            if (adds) load_global32(r, x.w);
#pragma unroll 1
            for (int i0 = 0; i0 < CPW; i0 += SOME) {
#pragma unroll
                for (int j = 0; j < SOME; j += PER) {
                    union { uint32_t w[8]; T v[PER]; } y;
                    float v[PER];
#pragma unroll
                    for (int i = 0; i < PER; ++i) v[i] = at(j + i);
                    if (p.bias) {
#pragma unroll
                        for (int i = 0; i < PER; ++i) v[i] += turn[i0 + j + i];
                    }
                    activate_some<T>(v, p.act);
                    if (p.residual) {
#pragma unroll
                        for (int i = 0; i < PER; ++i) v[i] += to_float(x.v[i]);
                        if (adds && i0 + j + PER < CPW) load_global32(r + i0 + j + PER, x.w);
                    }
#pragma unroll
                    for (int i = 0; i < PER; ++i) from_float(v[i], &y.v[i]);
                    if (there) store_global32(o + i0 + j, y.w);
                }
                shift_out<SOME>();
            }
            return;
        }
#pragma unroll 1
        for (int i0 = 0; i0 < CPW && n < p.N; i0 += 16, n += 16) {
            float v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = at(i);
            shift_out<16>();
            if (p.bias) {
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] += n + i < p.N ? load_ordered(bias + n + i) : 0.f;
            }
            activate_some<T>(v, p.act);
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 16; ++i) turn[lane * 17 + i] = v[i];
            __syncwarp();
            const int col = n + (lane & 15), first = quad * 32 + (lane >> 4), left = col < p.N ? rows - first : 0;      // this lane's rows: first, first + 2, ..
#pragma unroll 1
            for (int i = 0; 2 * i < left && i < 16; i += ROWS) {
                T res[ROWS];
                if (p.residual) {
                    const T *r = (const T *)p.residual + (row0 + first + 2 * i) * p.res_row + col;
#pragma unroll
                    for (int j = 0; j < ROWS; ++j)
                        if (2 * (i + j) < left) res[j] = load_ordered(r + 2 * j * p.res_row);
                }
                T *o = (T *)p.out + (row0 + first + 2 * i) * p.out_row + col;
                const float *mine = turn + (2 * i + (lane >> 4)) * 17 + (lane & 15);
#pragma unroll
                for (int j = 0; j < ROWS; ++j)
                    if (2 * (i + j) < left) from_float(p.residual ? mine[2 * j * 17] + to_float(res[j]) : mine[2 * j * 17], o + 2 * j * p.out_row);
            }
        }
    }
    __device__ __forceinline__ void finish_rows(const F8Params &q, int e, int row0, int rows, int n, float *turn) {
        switch (q.p.out_type) {
            case HIKONV_OUT_F32: finish_rows_as<float>(q, e, row0, rows, n, turn); break;
            case HIKONV_OUT_F16: finish_rows_as<__half>(q, e, row0, rows, n, turn); break;
            default: finish_rows_as<__nv_bfloat16>(q, e, row0, rows, n, turn); break;
        }
    }
    // Lanes are output columns from n0 + quad 32 on: each of `rows` rows of x from row0 on is written by neighbouring lanes, eight rows at a time.
    template <typename T>
    __device__ __forceinline__ void finish_columns_as(const F8Params &q, int e, long long row0, int rows, int n) {
        const LinearParams &p = q.p;
        const float b = p.bias ? load_ordered((const float *)p.bias + (long long)e * p.N + n) : 0.f;
        T *o = (T *)p.out + row0 * p.out_row + n;
        const T *r = (const T *)p.residual + row0 * p.res_row + n;
#pragma unroll 1
        for (int i0 = 0; i0 < CPW && rows > 0; i0 += 8, rows -= 8, o += 8 * p.out_row, r += 8 * p.res_row) {
            float v[8];
            T res[8];
            if (p.residual) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < rows) res[i] = load_ordered(r + i * p.res_row);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = p.bias ? at(i) + b : at(i);
            shift_out<8>();
            activate_some<T>(v, p.act);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < rows) from_float(p.residual ? v[i] + to_float(res[i]) : v[i], o + i * p.out_row);
        }
    }
    __device__ __forceinline__ void finish_columns(const F8Params &q, int e, int row0, int rows, int n0) {
        const int n = n0 + ((threadIdx.x >> 5) & 3) * 32 + (threadIdx.x & 31);
        if (n >= q.p.N) return;
        switch (q.p.out_type) {
            case HIKONV_OUT_F32: finish_columns_as<float>(q, e, row0, rows, n); break;
            case HIKONV_OUT_F16: finish_columns_as<__half>(q, e, row0, rows, n); break;
            default: finish_columns_as<__nv_bfloat16>(q, e, row0, rows, n); break;
        }
    }
};

// A warp that adds up: the 32 lanes of its quarter, CPW of the columns.
template <bool TOKENS, int CPW>
struct Adder {
    const F8Params &q;
    const uint32_t tmem, acc_full, acc_empty;
    int lane, quad, half;
    ScaleRing scales;
    Ring acc;
    Sums<CPW> sums;

    __device__ __forceinline__ Adder(const F8Params &q_, uint32_t tmem_, uint32_t full, uint32_t empty, const ScaleRing &s)
        : q(q_), tmem(tmem_), acc_full(full), acc_empty(empty), scales(s) {
        lane = threadIdx.x & 31;
        quad = (threadIdx.x >> 5) & 3;
        half = ((threadIdx.x >> 5) - kF8FirstAdder) >> 2;
    }
    __device__ __forceinline__ bool add(int steps) {
        constexpr int CH = CPW < 32 ? CPW : 32;
        sums.clear();
        for (int c = 0; c < steps; ++c) {
            if (!scales.wait()) return false;
            const float w = load_shared_float(scales.w());
            const uint32_t xs = scales.xs();
            float s = w;
            if (TOKENS) {
                s *= load_shared_float(xs + (quad * 32 + lane) * 4);
                scales.next(c == steps - 1);
            }
            const uint64_t ss = f8_two(s, s);
            if (!f8_wait(q, acc_full + 8 * acc.stage, acc.phase)) return false;
            tc_fence_after();
            const uint32_t d = tmem + acc.stage * q.acc_cols + ((uint32_t)(quad * 32) << 16) + half * CPW;
            uint32_t v[2][CH];
            f8_load(d, v[0]);
#pragma unroll
            for (int i = 0; i < CPW; i += CH) {
                uint32_t(&now)[CH] = v[(i / CH) & 1];
                f8_loaded(now);
                if (i + CH < CPW) {
                    f8_load(d + i + CH, v[(i / CH + 1) & 1]);
                } else {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbarrier_arrive(acc_empty + 8 * acc.stage);
                }
#pragma unroll
                for (int k = 0; k < CH; k += 4) {
                    uint64_t s01 = ss, s23 = ss;
                    if (!TOKENS) {
                        const uint4 x = load_shared16(xs + (half * CPW + i + k) * 4);
                        s01 = f8_mul(f8_two(x.x, x.y), ss);
                        s23 = f8_mul(f8_two(x.z, x.w), ss);
                    }
                    uint64_t *o = sums.sum + (i + k) / 2;
                    o[0] = f8_fma(f8_two(now[k], now[k + 1]), s01, o[0]);
                    o[1] = f8_fma(f8_two(now[k + 2], now[k + 3]), s23, o[1]);
                }
            }
            if (!TOKENS) scales.next(c == steps - 1);
            acc.next(q.accs);
        }
        return true;
    }
    __device__ __forceinline__ void finish(const Tile &t, float *turn) {
        if (TOKENS) sums.finish_rows(q, t.e, t.row0, t.rows, t.n0 + half * CPW, turn);
        else sums.finish_columns(q, t.e, t.row0 + half * CPW, t.rows - half * CPW, t.n0);
    }
};

// With a shared depth: this CTA's sums go to shared memory, [row of x][output column], over the stages (all that was loaded has been multiplied when
// the last sums are there); after the cluster's barrier the CTA finishes its share of the columns, four of a row per thread at a time, adding the
// parts in the order of the depth.
template <typename T>
__device__ __forceinline__ void finish_parts(const F8Params &q, const Tile &tile, int rank, uint32_t part) {
    const LinearParams &p = q.p;
    const int tid = threadIdx.x - kF8FirstAdder * 32;
    const int lanes = (kF8Rows / 4) >> q.split_shift, own = (rank * lanes + (tid & (lanes - 1))) * 4, step = kF8Adders * 32 / lanes;
    const int n = tile.n0 + own, inside = max(0, min(4, p.N - n));
    uint32_t from[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) from[r] = remote_address(part + own * 4, r < q.splits ? r : 0);
    float bias[4] = {};
    if (p.bias) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < inside) bias[k] = load_ordered((const float *)p.bias + (long long)tile.e * p.N + n + k);
    }
    for (int i = tid / lanes; i < tile.rows; i += step) {
        float res[4] = {};
        if (p.residual) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (k < inside) res[k] = to_float(load_ordered((const T *)p.residual + (tile.row0 + i) * p.res_row + n + k));
        }
        float4 v[8];
#pragma unroll
        for (int r = 0; r < 8; ++r)
            if (r < q.splits) v[r] = load_cluster_float4(from[r] + i * kF8Rows * 4);
        float s[4] = {};
#pragma unroll
        for (int r = 0; r < 8; ++r)
            if (r < q.splits) s[0] += v[r].x, s[1] += v[r].y, s[2] += v[r].z, s[3] += v[r].w;
        T *o = (T *)p.out + (tile.row0 + i) * p.out_row + n;
        T y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            s[k] = activate(s[k] + bias[k], p.act);
            from_float(p.residual ? s[k] + res[k] : s[k], &y[k]);
        }
        if (inside == 4 && (uintptr_t)o % (4 * sizeof(T)) == 0) {
            struct alignas(4 * sizeof(T)) Four { T v[4]; } four;
#pragma unroll
            for (int k = 0; k < 4; ++k) four.v[k] = y[k];
            *reinterpret_cast<Four *>(o) = four;
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (k < inside) o[k] = y[k];
        }
    }
}

template <bool TOKENS, int CPW>
__global__ void __launch_bounds__(kF8Threads, 1)
    linear_f8_kernel(const __grid_constant__ F8Params q, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b) {
    extern __shared__ __align__(16) uint8_t dynamic[];
    F8Control &ctl = *reinterpret_cast<F8Control *>(dynamic);
    const uint32_t control = smem_address(dynamic);
#define HIKONV_BAR(name, i) (control + (uint32_t)offsetof(F8Control, name) + 8u * (uint32_t)(i))
    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0);
    const LinearParams &p = q.p;
    const uint32_t stages = (control + (uint32_t)sizeof(F8Control) + 1023u) & ~1023u;
    uint8_t *const area = dynamic + (stages - control);
    int2 *group_row = reinterpret_cast<int2 *>(area + q.held);
    int *group_tiles = reinterpret_cast<int *>(group_row + p.E);
    const GroupTables tables{group_row, group_tiles};

    if (warp == 0) {
        if (lane < q.stages) {
            mbarrier_init(HIKONV_BAR(full, lane), 1);
            mbarrier_init(HIKONV_BAR(empty, lane), 1);
        }
        if (lane < q.accs) {
            mbarrier_init(HIKONV_BAR(acc_full, lane), 1);
            mbarrier_init(HIKONV_BAR(acc_empty, lane), kF8Adders);
        }
        if (lane < kScaleSlots) {
            mbarrier_init(HIKONV_BAR(scales.full, lane), 32);
            mbarrier_init(HIKONV_BAR(scales.empty, lane), kF8Adders);
        }
        if (lane == 0) {
            mbarrier_init(HIKONV_BAR(drain, 0), 1);
            ctl.whole = 1;
        }
        mbarrier_init_fence();
        if (lane == 3) {
            asm volatile("prefetch.tensormap [%0];" ::"l"(&map_a) : "memory");
            asm volatile("prefetch.tensormap [%0];" ::"l"(&map_b) : "memory");
        }
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_address(&ctl.tmem)), "r"(q.tmem_cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = ctl.tmem;
    // Not before this CTA has its tensor memory: a CTA of the kernel behind that came to this SM first could take it, and wait for this
    // one to end while this one waits for the memory.
    grid_dependency_release();
    grid_dependency_wait();
    int tiles = q.m_tiles * q.n_blocks;
    if (p.offsets) tiles = build_group_tables(q, group_row, group_tiles);
    const int rank = blockIdx.x & (q.splits - 1), t0 = blockIdx.x >> q.split_shift, step = gridDim.x >> q.split_shift;
    const int c0 = (int)(((long long)q.chunks * rank) >> q.split_shift), c1 = (int)(((long long)q.chunks * (rank + 1)) >> q.split_shift);

    bool fine = true;
    if (warp < kF8FirstAdder) {
        if (warp == 0) {
            Ring ring;
            int loads = 0;
            for (int t = t0; fine && t < tiles; t += step) {
                const Tile tile = find_tile(q, tables, t, q.width);
                const int w_row = tile.e * p.N + tile.n0;
                for (int c = c0; c < c1; ++c) {
                    fine = f8_wait(q, HIKONV_BAR(empty, ring.stage), ring.phase ^ 1);
                    if (!fine) break;
                    if (elect_one()) {
                        const uint32_t at = stages + ring.stage * q.stage_bytes, bar = HIKONV_BAR(full, ring.stage);
                        mbarrier_arrive_expect(bar, (uint32_t)(kF8Rows + (TOKENS ? q.width : q.nt)) * kF8Depth);
                        tma_load_2d(at, &map_a, c * kF8Depth, TOKENS ? tile.row0 : w_row, bar);
                        tma_load_2d(at + q.b_off, &map_b, c * kF8Depth, TOKENS ? w_row : tile.row0, bar);
                    }
                    ++loads;
                    ring.next(q.stages);
                }
            }
            // what is in flight has to land before the memory goes: the last load of every stage.  (The multiplies' last arrivals are at this CTA's own
            // barriers, committed in front of those that the adding warps wait for.)
            for (int i = 0; i < q.stages && i < loads; ++i) {
                ring.stage = ring.stage ? ring.stage - 1 : q.stages - 1;
                if (ring.stage == q.stages - 1) ring.phase ^= 1;
                fine &= f8_wait(q, HIKONV_BAR(full, ring.stage), ring.phase);
            }
        } else if (warp == 1) {
            Ring ring, acc;
            const uint64_t a0 = smem_descriptor(stages), b0 = smem_descriptor(stages + q.b_off);
            const uint32_t stage_units = (uint32_t)q.stage_bytes >> 4;
            for (int t = t0; fine && t < tiles; t += step) {
                const Tile tile = find_tile(q, tables, t, q.width);
                const int columns = TOKENS ? min(q.width, p.N - tile.n0) : tile.rows;
                const uint32_t idesc = q.idesc | ((uint32_t)((columns + 15) & ~15) >> 3 << 17);
                for (int c = c0; c < c1; ++c) {
                    fine = f8_wait(q, HIKONV_BAR(acc_empty, acc.stage), acc.phase ^ 1) && f8_wait(q, HIKONV_BAR(full, ring.stage), ring.phase);
                    if (!fine) break;
                    tc_fence_after();
                    if (elect_one()) {
                        const uint64_t a = a0 + ring.stage * stage_units, b = b0 + ring.stage * stage_units;
                        const uint32_t d = tmem + acc.stage * q.acc_cols;
#pragma unroll
                        for (int k = 0; k < kF8Depth / 32; ++k) f8_mma(d, a + k * 2, b + k * 2, idesc, k > 0);
                        tc_commit(HIKONV_BAR(empty, ring.stage));
                        tc_commit(HIKONV_BAR(acc_full, acc.stage));
                    }
                    ring.next(q.stages);
                    acc.next(q.accs);
                }
            }
            if (!fine) {                                // multiplies in flight read shared memory and write tensor memory
                if (elect_one()) tc_commit(HIKONV_BAR(drain, 0));
                f8_wait(q, HIKONV_BAR(drain, 0), 0);
            }
        }
        if (warp == 2) {
            Ring ring;
            for (int t = t0; fine && t < tiles; t += step) {
                const Tile tile = find_tile(q, tables, t, q.width);
                const float *w = p.w_scale + ((long long)tile.e * q.w_blocks + tile.n0 / kF8Depth) * q.chunks;
                fine = bring_scales(q, ring, stages + q.feed_off, HIKONV_BAR(scales.full, 0), HIKONV_BAR(scales.empty, 0), tile.row0, tile.rows, w, c0, c1);
            }
            asm volatile("cp.async.wait_all;" ::: "memory");        // these copies are in no group that is waited for
        }
        if (q.splits > 1) {
            if (!fine) ctl.whole = 0;
            __syncwarp();
            cluster_sync_all();
            cluster_sync_all();                         // the others may still read this CTA's part
        }
    } else {
        Adder<TOKENS, CPW> adder(q, tmem, HIKONV_BAR(acc_full, 0), HIKONV_BAR(acc_empty, 0),
                                   ScaleRing(q, stages + q.feed_off, HIKONV_BAR(scales.full, 0), HIKONV_BAR(scales.empty, 0)));
        float *turn = reinterpret_cast<float *>(area + q.turn_off) + (warp - kF8FirstAdder) * (32 * 17);
        if (!TOKENS && q.splits > 1) {
            Tile tile{0, 0, 0, 0};
            if (t0 < tiles) {
                tile = find_tile(q, tables, t0, q.width);
                fine = adder.add(c1 - c0);
            }
            if (t0 < tiles && fine) {
#pragma unroll
                for (int i = 0; i < CPW; ++i)
                    asm volatile("st.shared.f32 [%0], %1;" ::"r"(stages + ((adder.half * CPW + i) * kF8Rows + adder.quad * 32 + lane) * 4), "f"(adder.sums.at(i)) : "memory");
            }
            if (!fine) ctl.whole = 0;
            const uint32_t flag_at = remote_address(smem_address(&ctl.whole), lane & (q.splits - 1));
            __syncwarp();
            cluster_sync_all();
            const int flag = load_cluster_s32(flag_at);
            if (__all_sync(0xFFFFFFFFu, flag)) {
                if (p.out_type == HIKONV_OUT_F32) finish_parts<float>(q, tile, rank, stages);
                else if (p.out_type == HIKONV_OUT_F16) finish_parts<__half>(q, tile, rank, stages);
                else finish_parts<__nv_bfloat16>(q, tile, rank, stages);
            }
            cluster_sync_all();                         // the others may still read this CTA's part
        } else {
            for (int t = t0; t < tiles; t += step) {
                fine = adder.add(c1 - c0);
                if (!fine) break;
                adder.finish(find_tile(q, tables, t, q.width), turn);
            }
        }
    }
    if (!fine && lane == 0) atomicAdd(&linear_f8_timeouts, 1u);
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(q.tmem_cols));
#undef HIKONV_BAR
}

// ---- pairs of CTAs
//
// The two CTAs of a cluster take a tile of 256 rows of x by 256 output columns: each brings its 128 rows of x and half of the rows of w, and the
// first one's multiplies (cta_group::2) read both shared memories and write each CTA's 128 lanes in its own tensor memory.  That halves what an SM
// fetches of w and reads of it from shared memory: 32 KB per step of 128 instead of 48.
// A step is two multiplies of 128 columns each, which four warps each add up (every thread 128 sums): while one four load from tensor memory, the
// other four add.  4096 x 16384 x 4096: 250 us in a burst, 300 back to back (1.8 P operations per second at 1.4 GHz by the power limit; 249
// without reading tensor memory, 266 without additions).  A step takes 860 cycles, of which the tensor cores multiply for 512; a tile's begin and end 4900, with
// SiLU 8700.  The adding warps ask for their scales themselves: a warp that brings them, as below 256 rows a tile, made no difference (298 us).
constexpr int kPairRows = 256, kPairWidth = 256, kPairHalf = 128, kPairStages = 6, kPairStage = 2 * kF8Rows * kF8Depth;
constexpr int kPairAdders = 8, kPairThreads = (kF8FirstAdder + kPairAdders) * 32;
// The sums take more registers than an even share: those of a thread that adds up, and of one that does not.  Together no more than the launch's,
// which takes all that 384 threads can have.
constexpr int kPairAdderRegs = 232, kPairOtherRegs = 40, kPairLaunchRegs = 168;
static_assert(kPairAdderRegs * kPairAdders * 32 + kPairOtherRegs * kF8FirstAdder * 32 <= kPairLaunchRegs * kPairThreads, "registers of the launch");

constexpr int kPairAhead = 8;                           // steps whose scales of x are on their way

struct PairControl {
    uint64_t full[kPairStages], empty[kPairStages], acc_full[4], acc_empty[4], drain[2], peer;
    uint32_t tmem;
    int peer_loads;                      // of the second CTA, in the first one's memory, once that has arrived at peer
};

__device__ __forceinline__ void pair_load(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map),
                 "r"(x), "r"(y), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void pair_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a),
                 "l"(b), "r"(idesc), "r"(accumulate)
                 : "memory");
}
// Arrives at the barrier of this offset in both CTAs when the multiplies so far are done.
__device__ __forceinline__ void pair_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void arrive_at(uint32_t cluster_bar) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}

__device__ __forceinline__ void store_then_arrive_at(uint32_t cluster_address, int v, uint32_t cluster_bar) {
    asm volatile("st.shared::cluster.s32 [%0], %1;\n\tmbarrier.arrive.release.cluster.shared::cluster.b64 _, [%2];" ::"r"(cluster_address), "r"(v),
                 "r"(cluster_bar)
                 : "memory");
}

// A warp that adds up: a quarter of the lanes, 128 columns, 32 at a time.  Scales of x come by asynchronous copies, kPairAhead steps ahead, those of w
// 32 steps at a time.  A warp waits for 32 columns from tensor memory, then adds them; the other warp of its quarter of the SM, which has the other half
// of the columns, adds meanwhile.  The scale of the next step is made before the last columns of a step are added.
struct PairAdder {
    static constexpr int kChunk = 32;
    const F8Params &q;
    Sums<kPairHalf> sums;
    const float *xs, *ws;                // the next scale to ask for, of this lane's row; of this warp's columns
    const uint32_t feed;                 // kPairAhead slots of 32 scales of x
    float w_now, w_next;                 // scales of w, a lane each

    __device__ __forceinline__ PairAdder(const F8Params &q_, uint32_t feed_) : q(q_), feed(feed_) {}
    __device__ __forceinline__ void ask(int c) {
        if (c < q.chunks) asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(feed + c % kPairAhead * 128), "l"(xs) : "memory");
        xs += q.xs_row;
        cp_async_commit();
    }
    // A tile's first scales, asked for before the tile before is finished.  row: of this lane, or one that there is.
    __device__ __forceinline__ void begin(int e, int row, int block) {
        const int lane = threadIdx.x & 31;
        xs = q.p.x_scale + row;
        ws = q.p.w_scale + ((long long)e * q.w_blocks + block) * q.chunks + lane;
        w_next = lane < q.chunks ? load_ordered(ws) : 0.f;
#pragma unroll
        for (int i = 0; i < kPairAhead; ++i) ask(i);
    }
    // The scale of step c, and that of kPairAhead steps later asked for.
    __device__ __forceinline__ float scale(int c) {
        if ((c & 31) == 0) {
            w_now = w_next;
            w_next = c + 32 + (int)(threadIdx.x & 31) < q.chunks ? load_ordered(ws + c + 32) : 0.f;
        }
        asm volatile("cp.async.wait_group %0;" ::"n"(kPairAhead - 1) : "memory");
        float x;
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(feed + c % kPairAhead * 128) : "memory");
        const float s = x * __shfl_sync(0xFFFFFFFFu, w_now, c & 31);
        ask(c + kPairAhead);
        return s;
    }
    // taddr, bars: of the first of this warp's two accumulators, the second's 256 columns and two barriers on; empty: the cluster's address.
    __device__ __forceinline__ bool add(uint32_t taddr, uint32_t full, uint32_t empty, uint32_t &turn) {
        sums.clear();
        float s = scale(0);
#pragma unroll 1
        for (int c = 1; c <= q.chunks; ++c) {
            const uint64_t ss = f8_two(s, s);
            const uint32_t which = turn & 1, d = taddr + which * 2 * kPairHalf;
            if (!f8_wait(q, full + 16 * which, turn >> 1 & 1)) return false;
            tc_fence_after();
#pragma unroll
            for (int i = 0; i < kPairHalf; i += kChunk) {
                uint32_t v[kChunk];
                f8_load(d + i, v);
                f8_loaded(v);
                if (i + kChunk == kPairHalf) {
                    tc_fence_before();
                    __syncwarp();
                    if ((threadIdx.x & 31) == 0) arrive_at(empty + 16 * which);
                    if (c < q.chunks) s = scale(c);
                }
#pragma unroll
                for (int k = 0; k < kChunk; k += 2) sums.sum[(i + k) / 2] = f8_fma(f8_two(v[k], v[k + 1]), ss, sums.sum[(i + k) / 2]);
            }
            ++turn;
        }
        return true;
    }
};

__global__ void __launch_bounds__(kPairThreads, 1)
    linear_f8_pair_kernel(const __grid_constant__ F8Params q, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w) {
    extern __shared__ __align__(16) uint8_t dynamic[];
    PairControl &ctl = *reinterpret_cast<PairControl *>(dynamic);
    const uint32_t control = smem_address(dynamic);
#define HIKONV_BAR(name, i) (control + (uint32_t)offsetof(PairControl, name) + 8u * (uint32_t)(i))
    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0);
    const uint32_t rank = blockIdx.x & 1;
    const LinearParams &p = q.p;
    const uint32_t stages = (control + (uint32_t)sizeof(PairControl) + 1023u) & ~1023u;
    uint8_t *const area = dynamic + (stages - control);
    int2 *group_row = reinterpret_cast<int2 *>(area + q.held);
    int *group_tiles = reinterpret_cast<int *>(group_row + p.E);
    const GroupTables tables{group_row, group_tiles};

    if (warp == 0) {
        if (lane < q.stages) {
            mbarrier_init(HIKONV_BAR(full, lane), 1);
            mbarrier_init(HIKONV_BAR(empty, lane), 2);                     // a warp for each half of the columns
        }
        if (lane < 4) {
            mbarrier_init(HIKONV_BAR(acc_full, lane), 1);
            mbarrier_init(HIKONV_BAR(acc_empty, lane), kPairAdders);       // four warps of each CTA
        }
        if (lane < 2) mbarrier_init(HIKONV_BAR(drain, lane), 1);
        if (lane == 2) mbarrier_init(HIKONV_BAR(peer, 0), 1);
        mbarrier_init_fence();
        if (lane == 3) {
            asm volatile("prefetch.tensormap [%0];" ::"l"(&map_x) : "memory");
            asm volatile("prefetch.tensormap [%0];" ::"l"(&map_w) : "memory");
        }
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_address(&ctl.tmem)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();                                 // the other CTA's barriers are there
    tc_fence_after();
    const uint32_t tmem = ctl.tmem;
    // Not before this CTA has its tensor memory: a CTA of the kernel behind that came to this SM first could take it, and wait for this
    // one to end while this one waits for the memory.
    grid_dependency_release();
    grid_dependency_wait();
    int tiles = q.m_tiles * q.n_blocks;
    if (p.offsets) tiles = build_group_tables(q, group_row, group_tiles);
    const int t0 = blockIdx.x >> 1, step = gridDim.x >> 1;

    bool fine = true;
    if (warp < kF8FirstAdder) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kPairOtherRegs));
        if (warp == 0) {
            Ring ring;
            int loads = 0;
            for (int t = t0; fine && t < tiles; t += step) {
                const Tile tile = find_tile(q, tables, t, kPairWidth);
                const int x_row = tile.row0 + (int)rank * kF8Rows, w_row = tile.e * p.N + tile.n0 + (int)rank * (kPairHalf / 2);
                for (int c = 0; c < q.chunks; ++c) {
                    fine = f8_wait(q, HIKONV_BAR(empty, ring.stage), ring.phase ^ 1);
                    if (!fine) break;
                    if (elect_one()) {
                        const uint32_t at = stages + ring.stage * kPairStage, bar = remote_address(HIKONV_BAR(full, ring.stage), 0);
                        if (rank == 0) mbarrier_arrive_expect(HIKONV_BAR(full, ring.stage), 2 * kPairStage);
                        pair_load(at, &map_x, c * kF8Depth, x_row, bar);
                        pair_load(at + kF8Rows * kF8Depth, &map_w, c * kF8Depth, w_row, bar);
                        pair_load(at + (kF8Rows + kPairHalf / 2) * kF8Depth, &map_w, c * kF8Depth, w_row + kPairHalf, bar);
                    }
                    ++loads;
                    ring.next(q.stages);
                }
            }
            // both CTAs' copies and multiplies, and the multiplies' arrivals at this CTA's barriers
            fine = fine && f8_stages_free(q, ring, HIKONV_BAR(empty, 0));
            // Where a wait ran out, the two may have loaded different stages; both CTAs' copies end at the first one's barriers.
            if (rank == 1) {
                if (elect_one()) store_then_arrive_at(remote_address(control + (uint32_t)offsetof(PairControl, peer_loads), 0), loads, remote_address(HIKONV_BAR(peer, 0), 0));
            } else if (!fine) {
                // the second CTA's loading warp ends after one wait that runs out at most
                bool told = false;
                for (int i = 0; i < 4 && !told; ++i) told = f8_wait(q, HIKONV_BAR(peer, 0), 0);
                asm volatile("fence.acq_rel.cluster;" ::: "memory");
                const int theirs = told ? *(volatile int *)&ctl.peer_loads : loads, most = max(loads, theirs);
                // a step that one of them alone has loaded: the first counts the second's bytes, or brings as many in their place
                for (int u = min(loads, theirs); u < most; ++u) {
                    const uint32_t at = stages + u % q.stages * kPairStage, bar = HIKONV_BAR(full, u % q.stages);
                    if (elect_one()) {
                        if (u >= loads) {
                            mbarrier_arrive_expect(bar, kPairStage);
                        } else {
                            pair_load(at, &map_x, 0, 0, remote_address(bar, 0));
                            pair_load(at + kF8Rows * kF8Depth, &map_w, 0, 0, remote_address(bar, 0));
                            pair_load(at + (kF8Rows + kPairHalf / 2) * kF8Depth, &map_w, 0, 0, remote_address(bar, 0));
                        }
                    }
                }
                // what is in flight, of both CTAs, has to land before the memory goes: the last load of every stage
                for (int u = max(0, most - q.stages); u < most; ++u) f8_wait(q, HIKONV_BAR(full, u % q.stages), u / q.stages & 1);
            }
        } else if (warp <= 2 && rank == 0) {
            // a warp for each half of the columns
            const int h = warp - 1;
            Ring ring;
            uint32_t turn = 0;
            const uint64_t a0 = smem_descriptor(stages), b0 = smem_descriptor(stages + (kF8Rows + h * (kPairHalf / 2)) * kF8Depth);
            for (int t = t0; fine && t < tiles; t += step) {
                const bool there = p.N - find_tile(q, tables, t, kPairWidth).n0 > h * kPairHalf;
                for (int c = 0; c < q.chunks; ++c) {
                    const uint32_t acc = (turn & 1) * 2 + h;
                    fine = (!there || f8_wait(q, HIKONV_BAR(acc_empty, acc), turn >> 1 & 1 ^ 1)) && f8_wait(q, HIKONV_BAR(full, ring.stage), ring.phase);
                    if (!fine) break;
                    tc_fence_after();
                    if (elect_one()) {
                        if (there) {
                            const uint64_t a = a0 + ring.stage * (kPairStage >> 4), b = b0 + ring.stage * (kPairStage >> 4);
#pragma unroll
                            for (int k = 0; k < kF8Depth / 32; ++k) pair_mma(tmem + acc * kPairHalf, a + k * 2, b + k * 2, q.idesc, k > 0);
                            pair_commit(HIKONV_BAR(acc_full, acc));
                        }
                        pair_commit(HIKONV_BAR(empty, ring.stage));
                    }
                    turn += there;
                    ring.next(q.stages);
                }
            }
            if (!fine) {                                // multiplies in flight read shared memory and write tensor memory
                if (elect_one())
                    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(HIKONV_BAR(drain, h)) : "memory");
                f8_wait(q, HIKONV_BAR(drain, h), 0);
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kPairAdderRegs));
        PairAdder adder(q, stages + q.feed_off + (warp - kF8FirstAdder) * (kPairAhead * 128) + lane * 4);
        float *turn_area = reinterpret_cast<float *>(area + q.turn_off) + (warp - kF8FirstAdder) * (32 * 17);
        const int quad = warp & 3, half = (warp - kF8FirstAdder) >> 2;
        const uint32_t taddr = tmem + ((uint32_t)(quad * 32) << 16) + half * kPairHalf, full = HIKONV_BAR(acc_full, half);
        const uint32_t empty = remote_address(HIKONV_BAR(acc_empty, half), 0);
        uint32_t turn = 0;
        // tiles of which this warp has columns
        auto next_tile = [&](int t, Tile &tile) {
            for (; t < tiles; t += step) {
                tile = find_tile(q, tables, t, kPairWidth);
                if (tile.n0 + half * kPairHalf < p.N) break;
            }
            return t;
        };
        auto begin = [&](const Tile &tile) {
            const int row = min(tile.row0 + (int)rank * kF8Rows + quad * 32 + lane, p.M - 1);
            adder.begin(tile.e, row, tile.n0 / kF8Depth + half);
        };
        Tile tile{0, 0, 0, 0};
        int t = next_tile(t0, tile);
        if (t < tiles) begin(tile);
        while (t < tiles) {
            fine = adder.add(taddr, full, empty, turn);
            if (!fine) break;
            const Tile now = tile;
            t = next_tile(t + step, tile);
            if (t < tiles) begin(tile);
            adder.sums.finish_rows(q, now.e, now.row0 + (int)rank * kF8Rows, now.rows - (int)rank * kF8Rows, now.n0 + half * kPairHalf, turn_area);
        }
        cp_async_wait_all();
    }
    if (!fine && lane == 0) atomicAdd(&linear_f8_timeouts, 1u);
    __syncwarp();
    tc_fence_before();
    // The other CTA's copies, multiplies and arrivals are over: its own warps' by the barrier, the multiplies' arrivals by the waits for them in front
    // of it, of the adding warps for full accumulators and of each CTA's loading warp for free stages.
    cluster_sync_all();
    __syncthreads();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512));
#undef HIKONV_BAR
}

// A warp that waits as those above do, for a barrier that nothing completes, gives up and is counted.
__global__ void linear_f8_wait_check_kernel(const __grid_constant__ F8Params q) {
    __shared__ uint64_t bar;
    if (threadIdx.x == 0) {
        mbarrier_init(smem_address(&bar), 1);
        mbarrier_init_fence();
    }
    __syncwarp();
    if (!f8_wait(q, smem_address(&bar), 0) && threadIdx.x == 0) atomicAdd(&linear_f8_timeouts, 1u);
}

// ---- host

struct F8Shape {
    bool tokens, pair;
    int nt, width, splits;
};

// Whether the kernel of pairs was given the registers that its warps ask for: one that waits for registers which are not there waits for good.  Pairs are no
// choice where it was not, or where that cannot be asked.
static bool pair_has_registers() {
    static std::atomic<int> known{0};                    // 1: no, 2: yes
    int k = known.load(std::memory_order_relaxed);
    if (k == 0) {
        cudaFuncAttributes a;
        if (cudaFuncGetAttributes(&a, linear_f8_pair_kernel) != cudaSuccess) return false;
        k = (a.numRegs + 7) / 8 * 8 * kPairThreads >= kPairAdderRegs * kPairAdders * 32 + kPairOtherRegs * kF8FirstAdder * 32 ? 2 : 1;
        known.store(k, std::memory_order_relaxed);
    }
    return k == 2;
}

// The tile that a model of the time, in us, likes best: a set-up, and for each tile that a CTA or pair takes in turn its steps and its end, as measured
// on weights from memory at depths of 512 to 16384.  A step of a tile of few rows is the round of its sums from the multiplies to the adding warps
// and back, 0.265 us for 16 rows to 0.6 for 128; a shared depth has fewer steps and an exchange of sums.  4096 x 4096 weights: 16 rows 11.6 us,
// in two parts 9.6, in four 8.5; 128 rows by tiles of 64 rows in two parts 12.4, by 128 x 128 15.6, by pairs 21; 512 rows 27, 16.3 and 20; 1024 rows
// 50, 28.6 and 20.2; 4096 rows by 128 x 128 90, by pairs 70.
static F8Shape choose_f8_tile(const LinearParams &p, int sms) {
    const int chunks = ceil_div(p.K, kF8Depth), filled = p.E < p.M ? p.E : p.M;
    F8Shape best{false, false, 16, kF8Rows, 1};
    double least = 1e300;
    auto consider = [&](bool tokens, int nt, int width, int splits, double setup, double step, double end) {
        const double tiles = (p.offsets ? (double)p.M / nt + 0.5 * filled : (double)ceil_div(p.M, nt)) * ceil_div(p.N, width);
        // clusters of four and more do not fill every SM: their CTAs share one part of the GPU (16 clusters of eight took two turns)
        if (splits > 1 && (tiles * splits > (splits == 8 ? 96 : sms - 20) || splits > chunks)) return;
        const int units = nt == kPairRows ? sms / 2 : sms;
        const double turns = splits > 1 ? 1.0 : p.offsets ? (tiles > units ? tiles / units + 0.3 : 1.0) : (double)((long long)(tiles + units - 1) / units);
        const double time = setup + turns * (ceil_div(chunks, splits) * step + end) + (splits == 1 ? 0.0 : splits == 2 ? 2.3 : splits == 4 ? 2.6 : 2.9);
        if (time < least) {
            least = time;
            best = F8Shape{tokens, nt == kPairRows, nt, width, splits};
        }
    };
    for (int splits = 1; splits <= 8; splits *= 2) {
        consider(false, 16, kF8Rows, splits, 2.6, 0.265, 0.4);
        consider(false, 32, kF8Rows, splits, 2.6, 0.3, 0.5);
        consider(false, 64, kF8Rows, splits, 2.6, 0.385, 0.7);
        consider(false, 128, kF8Rows, splits, 2.6, 0.6, 1.1);
    }
    consider(true, kF8Rows, 128, 1, 3.0, 0.37, 0.9);
    const F8Shape single = best;
    consider(true, kPairRows, kPairWidth, 1, 4.5, 0.46, 1.3);
    return best.pair && !pair_has_registers() ? single : best;
}

static int launch_pair(F8Params q, int x_f8, int w_f8, cudaStream_t st) {
    const LinearParams &p = q.p;
    const size_t tables = p.offsets ? (size_t)p.E * 12 : 0;
    const int feeds = kPairAdders * kPairAhead * 32 * 4, turns = kPairAdders * 32 * 17 * 4;
    q.stages = (int)((kF8MostSmem - 2048 - tables - feeds - turns) / kPairStage);          // six; five beside the tables of 600 groups and more
    if (q.stages > kPairStages) q.stages = kPairStages;
    q.feed_off = q.stages * kPairStage;
    q.turn_off = q.feed_off + feeds;
    q.held = q.turn_off + turns;
    // sums in 32 bits (1), the operands' types, 128 columns, 256 rows
    q.idesc = (1u << 4) | ((uint32_t)x_f8 << 7) | ((uint32_t)w_f8 << 10) | ((uint32_t)(kPairHalf >> 3) << 17) | ((uint32_t)(kPairRows >> 4) << 24);
    CUtensorMap map_x, map_w;
    if (!encode_map(&map_x, p.x, (uint64_t)p.K, (uint64_t)p.M, (uint64_t)p.x_row, kF8Depth, kF8Rows) ||
        !encode_map(&map_w, p.w, (uint64_t)p.K, (uint64_t)p.E * p.N, (uint64_t)p.w_row, kF8Depth, kPairHalf / 2))
        return HIKONV_ERR_CUDA;
    const int pairs = sm_count_here() / 2;
    const long long tiles = (p.offsets ? p.M / q.nt + (p.E < p.M ? p.E : p.M) : (long long)q.m_tiles) * q.n_blocks;
    const size_t smem = (size_t)q.held + 2048 + tables;
    auto launch = [&](auto kernel) {
        return with_dynamic_smem((const void *)kernel, smem, [&] {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3((unsigned)(2 * (tiles < pairs ? tiles : pairs)));
            cfg.blockDim = dim3(kPairThreads);
            cfg.dynamicSmemBytes = smem;
            cfg.stream = st;
            cudaLaunchAttribute attr[2];
            attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
            attr[0].val.programmaticStreamSerializationAllowed = 1;
            attr[1].id = cudaLaunchAttributeClusterDimension;
            attr[1].val.clusterDim.x = 2;
            attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
            cfg.attrs = attr;
            cfg.numAttrs = 2;
            return cudaLaunchKernelEx(&cfg, kernel, q, map_x, map_w) == cudaSuccess ? HIKONV_OK : HIKONV_ERR_CUDA;
        });
    };
    return launch(linear_f8_pair_kernel);
}

static int launch_linear_f8(const LinearParams &p, int x_f8, int w_f8, long long xs_row, cudaStream_t st) {
    const int sms = sm_count_here();
    const F8Shape shape = choose_f8_tile(p, sms);
    F8Params q;
    memset(&q, 0, sizeof(q));
    q.p = p;
    q.xs_row = xs_row;
    q.nt = shape.nt;
    q.width = shape.width;
    q.splits = shape.splits;
    while ((1 << q.split_shift) < q.splits) ++q.split_shift;
    q.chunks = (p.K - 1) / kF8Depth + 1;
    q.w_blocks = ceil_div(p.N, kF8Depth);
    q.wait_cycles = kWaitCycles;
    q.n_blocks = ceil_div(p.N, q.width);
    q.m_tiles = ceil_div(p.M, q.nt);
    q.tokens_first = p.offsets || (long long)p.M <= (long long)p.N;
    const int elem = p.out_type == HIKONV_OUT_F32 ? 4 : 2;
    q.whole_stores = (uintptr_t)p.out % 32 == 0 && (uintptr_t)p.residual % 32 == 0 && p.out_row * elem % 32 == 0 && (!p.residual || p.res_row * elem % 32 == 0);
    if (shape.pair) return launch_pair(q, x_f8, w_f8, st);
    const int columns = shape.tokens ? q.width : q.nt;
    q.b_off = kF8Rows * kF8Depth;
    q.stage_bytes = q.b_off + columns * kF8Depth;
    q.acc_cols = columns < 32 ? 32 : columns;
    q.accs = 512 / q.acc_cols < kF8MostAccs ? 512 / q.acc_cols : kF8MostAccs;
    q.tmem_cols = q.accs * q.acc_cols;                   // a power of two
    const int feeds = kScaleSlots * kScaleBytes;
    const int turns = shape.tokens ? kF8Adders * 32 * 17 * 4 : 0;
    const size_t tables = p.offsets ? (size_t)p.E * 12 : 0;
    q.stages = (int)((kF8MostSmem - 2048 - tables - feeds - turns) / q.stage_bytes);
    if (q.stages > kF8MostStages) q.stages = kF8MostStages;
    const int parts = q.splits > 1 ? ceil_div(q.nt * kF8Rows * 4, q.stage_bytes) : 1;
    if (q.stages < parts || q.stages < 2) return HIKONV_ERR_UNSUPPORTED;
    const long long tiles = (p.offsets ? p.M / q.nt + (p.E < p.M ? p.E : p.M) : (long long)q.m_tiles) * q.n_blocks;
    const int own = ceil_div(q.chunks, q.splits);
    if (tiles * q.splits <= sms && q.stages > own) q.stages = own > parts ? own : parts;
    q.feed_off = q.stages * q.stage_bytes;
    q.turn_off = q.feed_off + feeds;
    q.held = q.turn_off + turns;
    // sums in 32 bits (1), the operands' types, 128 rows; the columns follow per tile
    const int a_type = shape.tokens ? x_f8 : w_f8, b_type = shape.tokens ? w_f8 : x_f8;
    q.idesc = (1u << 4) | ((uint32_t)a_type << 7) | ((uint32_t)b_type << 10) | ((uint32_t)(kF8Rows >> 4) << 24);
    // CTAs of a cluster wait for one another, and for tensor memory.  With two such kernels at once (two streams), each could hold the memory that the
    // other's CTA waits for.  Registers keep them apart: 384 threads with 113 of them and more, those of hikonv_linear's tiles 60000 in all, so that
    // no two CTAs with tensor memory are on one SM.  Should a compiler give them fewer, this much shared memory still keeps two with clusters apart; one
    // without waits for nobody once it has its memory, but for the kernels before its own, whose CTAs all have theirs.
    size_t smem = (size_t)q.held + 2048 + tables;
    if (q.splits > 1 && smem < 184 * 1024) smem = 184 * 1024;

    CUtensorMap map_x, map_w;
    if (!encode_map(&map_x, p.x, (uint64_t)p.K, (uint64_t)p.M, (uint64_t)p.x_row, kF8Depth, (uint32_t)q.nt) ||
        !encode_map(&map_w, p.w, (uint64_t)p.K, (uint64_t)p.E * p.N, (uint64_t)p.w_row, kF8Depth, (uint32_t)q.width))
        return HIKONV_ERR_CUDA;
    const unsigned grid = (unsigned)(q.splits > 1 ? tiles * q.splits : tiles < sms ? tiles : sms);
    auto launch = [&](auto kernel) {
        return with_dynamic_smem((const void *)kernel, smem > 49 * 1024 ? smem : 49 * 1024, [&] {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(grid);
            cfg.blockDim = dim3(kF8Threads);
            cfg.dynamicSmemBytes = smem;
            cfg.stream = st;
            cudaLaunchAttribute attr[2];
            attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
            attr[0].val.programmaticStreamSerializationAllowed = 1;
            attr[1].id = cudaLaunchAttributeClusterDimension;
            attr[1].val.clusterDim.x = (unsigned)q.splits;
            attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
            cfg.attrs = attr;
            cfg.numAttrs = q.splits > 1 ? 2 : 1;
            const CUtensorMap &a = shape.tokens ? map_x : map_w, &b = shape.tokens ? map_w : map_x;
            return cudaLaunchKernelEx(&cfg, kernel, q, a, b) == cudaSuccess ? HIKONV_OK : HIKONV_ERR_CUDA;
        });
    };
    if (shape.tokens) return launch(linear_f8_kernel<true, 64>);
    switch (q.nt) {
        case 16: return launch(linear_f8_kernel<false, 8>);
        case 32: return launch(linear_f8_kernel<false, 16>);
        case 64: return launch(linear_f8_kernel<false, 32>);
        default: return launch(linear_f8_kernel<false, 64>);
    }
}

int read_linear_f8_timeouts(unsigned int *h_count) {
    return cudaMemcpyFromSymbol(h_count, linear_f8_timeouts, sizeof(*h_count)) == cudaSuccess ? HIKONV_OK : HIKONV_ERR_CUDA;
}

int launch_linear_f8_wait_check(long long cycles, cudaStream_t st) {
    F8Params q;
    memset(&q, 0, sizeof(q));
    q.wait_cycles = cycles;
    return launch_plain(linear_f8_wait_check_kernel, dim3(1), dim3(32), 0, st, q);
}

static int linear_f8_run(const void *d_x, int x_f8, long long x_row, const void *d_w, int w_f8, long long w_row, const int32_t *d_offsets, bool grouped, int E,
                         int M, int N, int K, const float *d_x_scale, long long xs_row, const float *d_w_scale, void *d_out, long long out_row,
                         const hikonv_epilogue_t *ep, void *stream) {
    if (!ep || M < 0 || N < 1 || K < 1 || E < 1) return HIKONV_ERR_INVALID_ARG;
    if ((x_f8 != HIKONV_F8_E4M3 && x_f8 != HIKONV_F8_E5M2) || (w_f8 != HIKONV_F8_E4M3 && w_f8 != HIKONV_F8_E5M2)) return HIKONV_ERR_INVALID_ARG;
    const int type = ep->out_type;
    if (type != HIKONV_OUT_F32 && type != HIKONV_OUT_F16 && type != HIKONV_OUT_BF16) return HIKONV_ERR_INVALID_ARG;
    if (ep->activation < HIKONV_ACT_NONE || ep->activation > HIKONV_ACT_GELU) return HIKONV_ERR_INVALID_ARG;
    if (ep->d_x_scale || ep->d_w_scale || ep->shift || ep->lo || ep->hi) return HIKONV_ERR_INVALID_ARG;
    if (E > HIKONV_MAX_GROUPS || M > (1 << 30) || N > (1 << 30) || (long long)E * N > 0x7FFFFF00ll || K > (1 << 30)) return HIKONV_ERR_UNSUPPORTED;
    // few enough tiles for 32-bit counts
    if (((long long)M / 16 + (E < M ? E : M) + 1) * ceil_div(N, kF8Rows) >= 0x3FFFFFFFll) return HIKONV_ERR_UNSUPPORTED;
    if (M == 0) return HIKONV_OK;
    const int elem = type == HIKONV_OUT_F32 ? 4 : 2;
    const long long blocks = (K - 1) / kF8Depth + 1, n_blocks = (N - 1) / kF8Depth + 1, wide = (long long)align_up(K, 16);
    if (M == 1) x_row = wide, out_row = N;                       // there is no second row
    if ((long long)E * N == 1) w_row = wide;
    if (blocks == 1) xs_row = M;
    const long long res_row = M == 1 || !ep->d_residual ? N : ep->residual_row_stride;
    if (!d_x || !d_w || !d_out || !d_x_scale || !d_w_scale || (grouped && !d_offsets)) return HIKONV_ERR_INVALID_ARG;
    if (x_row < K || w_row < K || xs_row < M || out_row < N || res_row < N) return HIKONV_ERR_INVALID_ARG;
    constexpr long long most = 1ll << 39;                        // bytes from row to row: what a tensor map takes, and offsets stay in 64 bits
    if (x_row >= most || w_row >= most || xs_row >= most || out_row >= most || res_row >= most) return HIKONV_ERR_INVALID_ARG;
    if ((uintptr_t)d_out % elem || (uintptr_t)ep->d_residual % elem || (uintptr_t)ep->d_bias % 4 || (uintptr_t)d_x_scale % 4 || (uintptr_t)d_w_scale % 4 ||
        (uintptr_t)d_offsets % 4)
        return HIKONV_ERR_INVALID_ARG;
    if ((uintptr_t)d_x % 16 || x_row % 16 || (uintptr_t)d_w % 16 || w_row % 16) return HIKONV_ERR_UNSUPPORTED;
    const size_t columns = (size_t)E * N * 4, w_scales = (size_t)(E * n_blocks * blocks) * 4;
    if (rows_overlap(d_out, out_row * elem, N * elem, M, d_x, x_row, K, M) || rows_overlap(d_out, out_row * elem, N * elem, M, d_w, w_row, K, (size_t)E * N) ||
        rows_overlap(d_out, out_row * elem, N * elem, M, d_x_scale, xs_row * 4, (size_t)M * 4, blocks) ||
        rows_overlap(d_out, out_row * elem, N * elem, M, d_w_scale, w_scales, w_scales, 1) ||
        rows_overlap(d_out, out_row * elem, N * elem, M, ep->d_bias, columns, columns, 1) ||
        rows_overlap(d_out, out_row * elem, N * elem, M, d_offsets, (size_t)(E + 1) * 4, (size_t)(E + 1) * 4, 1))
        return HIKONV_ERR_INVALID_ARG;
    if (ep->d_residual && !(ep->d_residual == d_out && res_row == out_row) &&
        rows_overlap(d_out, out_row * elem, N * elem, M, ep->d_residual, res_row * elem, N * elem, M))
        return HIKONV_ERR_INVALID_ARG;
    LinearParams k;
    memset(&k, 0, sizeof(k));
    k.x = (const uint8_t *)d_x; k.w = (const uint8_t *)d_w; k.offsets = d_offsets;
    k.x_row = x_row; k.w_row = w_row;
    k.M = M; k.N = N; k.K = K; k.E = E;
    k.out_type = type; k.act = ep->activation;
    k.out = d_out; k.residual = ep->d_residual; k.bias = ep->d_bias;
    k.x_scale = d_x_scale; k.w_scale = d_w_scale;
    k.out_row = out_row; k.res_row = res_row;
    if (linear_f8_rows_takes(k)) return launch_linear_f8_rows(k, x_f8, w_f8, xs_row, (cudaStream_t)stream);
    return launch_linear_f8(k, x_f8, w_f8, xs_row, (cudaStream_t)stream);
}

}  // namespace hikonv

using namespace hikonv;

extern "C" int hikonv_linear_f8(const void *d_x, int x_f8, long long x_row_stride, const void *d_w, int w_f8, long long w_row_stride, int M, int N, int K,
                                const float *d_x_scale, long long x_scale_row_stride, const float *d_w_scale, void *d_out, long long out_row_stride,
                                const hikonv_epilogue_t *epilogue, void *stream) {
    return linear_f8_run(d_x, x_f8, x_row_stride, d_w, w_f8, w_row_stride, nullptr, false, 1, M, N, K, d_x_scale, x_scale_row_stride, d_w_scale, d_out,
                         out_row_stride, epilogue, stream);
}

extern "C" int hikonv_grouped_linear_f8(const void *d_x, int x_f8, long long x_row_stride, const void *d_w, int w_f8, long long w_row_stride,
                                        const int32_t *d_offsets, int E, int T, int N, int K, const float *d_x_scale, long long x_scale_row_stride,
                                        const float *d_w_scale, void *d_out, long long out_row_stride, const hikonv_epilogue_t *epilogue, void *stream) {
    return linear_f8_run(d_x, x_f8, x_row_stride, d_w, w_f8, w_row_stride, d_offsets, true, E, T, N, K, d_x_scale, x_scale_row_stride, d_w_scale, d_out,
                         out_row_stride, epilogue, stream);
}
