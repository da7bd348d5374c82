// hikonv_sort_by_expert, hikonv_rows_to_experts, hikonv_rows_from_experts and its gradient: a mixture of experts around the products of
// hikonv_grouped_linear and hikonv_grouped_linear_f8.
//
// Sorting is a stable counting sort: pairs of token and choice keep their order within an expert, so results do not depend on the order
// in which warps run.  Rows are moved by token: a token's row is read once however many experts it goes to, and what an expert's rows
// give back to a token is summed in registers, in the order of its choices.
//
// 512 pairs over 64 experts are sorted in 2.5 us, 262144 over 256 in 11 (two launches; the second's CTAs each read the counts of all).  Rows are bound by
// memory: 8192 tokens with eight rows of 4096 bf16 values each come back in 114 us (5.9 TB/s), and rows that start anywhere by the two or four
// bytes of a load or store (5003 x 3 rows of 1333 fp16 values go out in 12.3 us, 4.0 TB/s, by words of four bytes; 15.2 by elements, four a thread; by one 32.
// 8-bit ones 6.1 and 14).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <initializer_list>
#include <type_traits>

#include "hikonv_cuda.cuh"
#include "hikonv_linear.h"

namespace hikonv {

// ---- sorting

static_assert(HIKONV_MAX_GROUPS + 1 < 1 << 11, "bits of a key");

constexpr int kSortSteps = 8;            // pairs of a thread whose experts its registers hold
constexpr int kSortMostCtas = 128;

struct SortParams {
    const void *experts;
    int wide;                            // 8-byte indices
    long long row;                       // elements from token to token
    long long pairs;
    int k, E, ctas;
    long long per_cta;                   // pairs
    int32_t *offsets, *slots;
    uint32_t *counts;                    // [ctas][E + 1], null for one CTA
};

// The experts of a stretch of pairs that begins at `from`: step s of a warp are 32 neighbours, the steps of a warp follow one another.  E for none,
// -1 behind the end.
__device__ __forceinline__ void read_experts(const SortParams &p, long long from, long long end, int steps, int (&key)[kSortSteps]) {
    const long long first = from + (long long)((threadIdx.x >> 5) * steps) * 32 + (threadIdx.x & 31);
    long long e[kSortSteps];
#pragma unroll
    for (int s = 0; s < kSortSteps; ++s) {
        const long long i = first + s * 32;
        e[s] = -1;
        if (s >= steps || i >= end) continue;
        long long at = i;
        if (p.row != p.k) {
            const long long t = i <= 0x7FFFFFFF ? (long long)((uint32_t)i / (uint32_t)p.k) : i / p.k;
            at = t * p.row + (i - t * p.k);
        }
        e[s] = p.wide ? load_ordered((const long long *)p.experts + at) : (long long)load_ordered((const int32_t *)p.experts + at);
    }
#pragma unroll
    for (int s = 0; s < kSortSteps; ++s) key[s] = s >= steps || first + s * 32 >= end ? -1 : e[s] >= 0 && e[s] < p.E ? (int)e[s] : p.E;
}

// The lanes whose key is this lane's, bit by bit: the instruction that finds them at once (match.any) took a CTA of 32 warps 2000 cycles.
__device__ __forceinline__ uint32_t lanes_with(int key, int bits) {
    uint32_t same = 0xFFFFFFFFu;
#pragma unroll
    for (int b = 0; b < 11; ++b) {                      // keys are at most HIKONV_MAX_GROUPS + 1
        if (b >= bits) break;
        const bool set = key >> b & 1;
        const uint32_t those = __ballot_sync(0xFFFFFFFFu, set);
        same &= set ? those : ~those;
    }
    return same;
}

// How many pairs of each expert a CTA's stretch has.
template <int THREADS>
__global__ void __launch_bounds__(THREADS) sort_count_kernel(const SortParams p) {
    extern __shared__ uint32_t hist[];
    grid_dependency_release();
    for (int e = threadIdx.x; e <= p.E; e += THREADS) hist[e] = 0;
    grid_dependency_wait();
    __syncthreads();
    const long long begin = blockIdx.x * p.per_cta, end = min(begin + p.per_cta, p.pairs);
    for (long long from = begin; from < end; from += THREADS * kSortSteps) {
        int key[kSortSteps];
        read_experts(p, from, end, kSortSteps, key);
#pragma unroll
        for (int s = 0; s < kSortSteps; ++s)
            if (key[s] >= 0) atomicAdd(hist + key[s], 1u);
    }
    __syncthreads();
    for (int e = threadIdx.x; e <= p.E; e += THREADS) p.counts[(long long)blockIdx.x * (p.E + 1) + e] = hist[e];
}

// Places of a CTA's stretch.  Every warp takes neighbouring pairs, 32 at a time: the lanes of one expert find each other, and a place is the
// expert's next one, the pairs of warps before, of this warp so far, and of lanes before.
template <int THREADS>
__global__ void __launch_bounds__(THREADS) sort_place_kernel(const SortParams p) {
    constexpr int WARPS = THREADS / 32, AT_ONCE = WARPS < 16 ? WARPS : 16;
    extern __shared__ uint32_t shared[];
    const int E1 = p.E + 1, bits = 32 - __clz(E1), tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    // [warp][E1] pairs of each expert in each warp, then in the warps before; its next place; all its pairs; of this block; sums of warps
    uint32_t *hist = shared, *next = hist + WARPS * E1, *total = next + E1, *block = total + E1, *sums = block + E1;
    grid_dependency_release();
    for (int i = tid; i < (WARPS + 2) * E1; i += THREADS) shared[i] = 0;
    grid_dependency_wait();
    __syncthreads();
    const long long begin = blockIdx.x * p.per_cta, end = min(begin + p.per_cta, p.pairs);
    int key[kSortSteps];
    uint32_t same[kSortSteps];
    // The block's experts, in how many lanes of each step, and how many each warp has; then how many the warps before have.
    auto read = [&](long long from) {
        const int steps = (int)min((long long)kSortSteps, (end - from + THREADS - 1) / THREADS);
        read_experts(p, from, end, steps, key);
#pragma unroll
        for (int s = 0; s < kSortSteps; ++s) {
            if (s >= steps) break;
            same[s] = lanes_with(key[s] < 0 ? E1 : key[s], bits);
            if (key[s] >= 0 && lane == __ffs(same[s]) - 1) hist[warp * E1 + key[s]] += __popc(same[s]);
            __syncwarp();
        }
        __syncthreads();
        for (int e = tid; e < E1; e += THREADS) {
            uint32_t upto = 0;
#pragma unroll
            for (int w0 = 0; w0 < WARPS; w0 += AT_ONCE) {
                uint32_t of[AT_ONCE];
#pragma unroll
                for (int w = 0; w < AT_ONCE; ++w) of[w] = hist[(w0 + w) * E1 + e];
#pragma unroll
                for (int w = 0; w < AT_ONCE; ++w) {
                    hist[(w0 + w) * E1 + e] = upto;
                    upto += of[w];
                }
            }
            block[e] = upto;
        }
        return steps;
    };
    if (p.counts) {
        // columns of the counts, by several threads each: what lies in front of this CTA, and all
        constexpr int ROWS = 16;
        const int parts = (p.ctas + ROWS - 1) / ROWS;
        for (int i = tid; i < parts * E1; i += THREADS) {
            const int part = i / E1, e = i - part * E1;
            const uint32_t *at = p.counts + (part * ROWS * E1 + e);
            uint32_t v[ROWS], before = 0, all = 0;
#pragma unroll
            for (int j = 0; j < ROWS; ++j) v[j] = part * ROWS + j < p.ctas ? load_ordered(at + j * E1) : 0;
#pragma unroll
            for (int j = 0; j < ROWS; ++j) {
                all += v[j];
                if (part * ROWS + j < (int)blockIdx.x) before += v[j];
            }
            if (before) atomicAdd(next + e, before);
            if (all) atomicAdd(total + e, all);
        }
    }
    int steps = read(begin);
    __syncthreads();
    // where each expert begins
    const uint32_t *all = p.counts ? total : block;
    const int items = (E1 + THREADS - 1) / THREADS;
    uint32_t mine = 0;
    for (int i = 0; i < items; ++i) mine += tid * items + i < E1 ? all[tid * items + i] : 0;
    uint32_t upto = mine;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, upto, d);
        if (lane >= d) upto += v;
    }
    if (lane == 31) sums[warp] = upto;
    __syncthreads();
    uint32_t before = lane < warp ? sums[lane] : 0;
    before = __reduce_add_sync(0xFFFFFFFFu, before);
    uint32_t start = before + upto - mine;
    for (int i = 0; i < items; ++i) {
        const int e = tid * items + i;
        if (e >= E1) break;
        if (blockIdx.x == 0) p.offsets[e] = (int32_t)start;
        next[e] += start;
        start += all[e];
    }
    __syncthreads();
    for (long long from = begin; from < end;) {
#pragma unroll
        for (int s = 0; s < kSortSteps; ++s) {
            if (s >= steps) break;
            const long long i = from + (long long)(warp * steps + s) * 32 + lane;
            if (key[s] >= 0) {
                const int place = (int)(next[key[s]] + hist[warp * E1 + key[s]] + __popc(same[s] & ((1u << lane) - 1)));
                p.slots[i] = key[s] < p.E ? place : -2 - place;
            }
            __syncwarp();
            if (key[s] >= 0 && lane == __ffs(same[s]) - 1) hist[warp * E1 + key[s]] += __popc(same[s]);
            __syncwarp();
        }
        from += THREADS * kSortSteps;
        if (from >= end) break;
        __syncthreads();
        for (int e = tid; e < E1; e += THREADS) next[e] += block[e];
        for (int i = tid; i < WARPS * E1; i += THREADS) hist[i] = 0;
        __syncthreads();
        steps = read(from);
        __syncthreads();
    }
}

// CTAs for so many pairs, and the pairs of each.  One up to four steps (the launch that counts costs 2 us); then two steps each, since a CTA's matches
// take longer than its reading of the others' counts, until there are 128.
static int sort_ctas(long long pairs, long long *per_cta) {
    constexpr long long step = 1024;
    const long long steps = (pairs + step - 1) / step, per = (steps + kSortMostCtas - 1) / kSortMostCtas;
    *per_cta = (steps <= 4 ? 4 : per > 2 ? per : 2) * step;
    return pairs > 0 ? (int)((pairs + *per_cta - 1) / *per_cta) : 1;
}

// ---- rows

struct RowsParams {
    const void *x, *y, *residual;        // rows of tokens; rows of experts; added to a token's sum
    void *out, *out_y;
    float *out_weights;
    const int32_t *slots;
    const float *weights;
    long long x_row, y_row, res_row, out_row, out_y_row;    // elements
    int T, k, H, R;
};

template <typename T> __device__ __forceinline__ float rows_float(T v);
template <> __device__ __forceinline__ float rows_float(float v) { return v; }
template <> __device__ __forceinline__ float rows_float(__half v) { return __half2float(v); }
template <> __device__ __forceinline__ float rows_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T rows_round(float v);
template <> __device__ __forceinline__ float rows_round(float v) { return v; }
template <> __device__ __forceinline__ __half rows_round(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 rows_round(float v) { return __float2bfloat16_rn(v); }

// The V columns of a row that a thread takes: neighbours, loaded and stored as one, where rows begin on 16-byte boundaries (WIDE), else as far apart as
// there are threads, so that neighbouring threads load and store neighbours.
template <typename T, int V, bool WIDE>
struct Columns {
    struct alignas(WIDE ? sizeof(T) * V : sizeof(T)) Pack {
        T v[V];
    };
    static __device__ __forceinline__ int first(int thread) { return WIDE ? thread * V : thread; }
    static __device__ __forceinline__ Pack load(const T *row, int c, int apart, int H) {
        if constexpr (WIDE) {
            return load_ordered(reinterpret_cast<const Pack *>(row + c));
        } else {
            Pack o;
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (c + i * apart < H) o.v[i] = load_ordered(row + c + i * apart);
                else o.v[i] = T();
            return o;
        }
    }
    static __device__ __forceinline__ void store(T *row, int c, int apart, int H, const Pack &o) {
        if constexpr (WIDE) {
            *reinterpret_cast<Pack *>(row + c) = o;
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (c + i * apart < H) row[c + i * apart] = o.v[i];
        }
    }
};
// Block: (columns, tokens); a grid's second dimension goes on along the rows.
__device__ __forceinline__ int row_token() { return blockIdx.x * blockDim.y + threadIdx.y; }

// Copies: T stands for so many bytes.
template <typename T, int V>
__global__ void __launch_bounds__(256) rows_to_kernel(const RowsParams p) {
    using C = Columns<T, V, false>;
    grid_dependency_release();
    grid_dependency_wait();
    const int t = row_token(), c = blockIdx.y * blockDim.x * V + threadIdx.x;
    if (t >= p.T || c >= p.H) return;
    const typename C::Pack v = C::load((const T *)p.x + t * p.x_row, c, blockDim.x, p.H);
    const int32_t *slots = p.slots + (long long)t * p.k;
#pragma unroll 4
    for (int j = 0; j < p.k; ++j) {
        const int s = load_ordered(slots + j);
        if (s >= 0 && s < p.R) C::store((T *)p.out + s * p.out_row, c, blockDim.x, p.H, v);
    }
}

// Copies of rows that begin anywhere (p.x_row, p.out_row and p.H: bytes).  A thread's V words of four bytes of an output row come out of two neighbouring
// words of x's row each, moved by a funnel shift: unit q has the words q - 1 and q of x's row (words count from the one that its first byte lies in)
// and gives the output row's word q - 1, or q where the output row begins later in its first word than x's does.  The up to three bytes in front of
// an output row's first whole word and behind its last are a thread's each.
template <int V>
__global__ void __launch_bounds__(256) rows_to_bytes_kernel(const RowsParams p) {
    constexpr int BATCH = 4;
    grid_dependency_release();
    grid_dependency_wait();
    const int t = row_token(), apart = blockDim.x, first = blockIdx.y * blockDim.x * V + threadIdx.x;
    if (t >= p.T) return;
    const uint8_t *x = (const uint8_t *)p.x + t * p.x_row;
    const int32_t *slots = p.slots + (long long)t * p.k;
    const int m = (int)((uintptr_t)x & 3), words = (m + p.H + 3) / 4;
    const uint32_t *from = reinterpret_cast<const uint32_t *>(x - m);
    uint32_t low[V], high[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int q = first + i * apart;
        low[i] = q >= 1 && q <= words ? load_ordered(from + q - 1) : 0;
        high[i] = q < words ? load_ordered(from + q) : 0;
    }
    for (int j0 = 0; j0 < p.k; j0 += BATCH) {
        int s[BATCH];
#pragma unroll
        for (int j = 0; j < BATCH; ++j) s[j] = j0 + j < p.k ? load_ordered(slots + j0 + j) : -1;
#pragma unroll
        for (int j = 0; j < BATCH; ++j) {
            if (s[j] < 0 || s[j] >= p.R) continue;
            uint8_t *row = (uint8_t *)p.out + s[j] * p.out_row;
            const int a = (int)((uintptr_t)row & 3), later = m < a, shift = 8 * (m - a + 4 * later);
            const int b0 = (first - 1 + later) * 4 - a;                     // the row's byte that the first word begins with
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int b = b0 + i * apart * 4;
                if (b >= 0 && b + 4 <= p.H) *reinterpret_cast<uint32_t *>(row + b) = __funnelshift_r(low[i], high[i], shift);
            }
        }
    }
    if (blockIdx.y > 0) return;
    for (int i = threadIdx.x; i < 8 * p.k; i += apart) {
        const int s = load_ordered(slots + i / 8), n = i & 3;
        if (s < 0 || s >= p.R) continue;
        uint8_t *row = (uint8_t *)p.out + s * p.out_row;
        const int a = (int)((uintptr_t)row & 3), head = -a & 3, tail = ((a + p.H) & ~3) - a;
        const int b = i & 4 ? (tail >= head ? tail + n : p.H) : (n < head ? n : p.H);
        if (b < p.H) row[b] = load_ordered(x + b);
    }
}

template <typename T, int V, bool WIDE>
__global__ void __launch_bounds__(256) rows_from_kernel(const RowsParams p) {
    using C = Columns<T, V, WIDE>;
    constexpr int BATCH = 4;
    grid_dependency_release();
    grid_dependency_wait();
    const int t = row_token(), apart = blockDim.x, c = blockIdx.y * blockDim.x * V + C::first(threadIdx.x);
    if (t >= p.T || c >= p.H) return;
    const int32_t *slots = p.slots + (long long)t * p.k;
    const float *weights = p.weights ? p.weights + (long long)t * p.k : nullptr;
    float sum[V] = {};
    if (p.residual) {
        const typename C::Pack r = C::load((const T *)p.residual + t * p.res_row, c, apart, p.H);
#pragma unroll
        for (int i = 0; i < V; ++i) sum[i] = rows_float(r.v[i]);
    }
    for (int j0 = 0; j0 < p.k; j0 += BATCH) {
        int s[BATCH];
        float w[BATCH];
        typename C::Pack y[BATCH];
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            s[b] = j0 + b < p.k ? load_ordered(slots + j0 + b) : -1;
            if (s[b] >= p.R) s[b] = -1;
            w[b] = weights && s[b] >= 0 ? load_ordered(weights + j0 + b) : 1.f;
        }
#pragma unroll
        for (int b = 0; b < BATCH; ++b)
            if (s[b] >= 0) y[b] = C::load((const T *)p.y + s[b] * p.y_row, c, apart, p.H);
#pragma unroll
        for (int b = 0; b < BATCH; ++b)
            if (s[b] >= 0) {
#pragma unroll
                for (int i = 0; i < V; ++i) sum[i] = fmaf(w[b], rows_float(y[b].v[i]), sum[i]);
            }
    }
    typename C::Pack o;
#pragma unroll
    for (int i = 0; i < V; ++i) o.v[i] = rows_round<T>(sum[i]);
    C::store((T *)p.out + t * p.out_row, c, apart, p.H, o);
}

// The gradient: a token by blockDim.x threads, which walk along its row; dot products of eight choices in registers, the rows of LOADS of them on their
// way at a time.  Bound by the loads of all threads of an SM together: places and weights lie in shared memory, so that four CTAs fit one.  4096 tokens,
// eight rows of 4096 bf16 values each: 103 us (5.5 TB/s); with four rows on their way, 136 registers and one CTA 201, 80 and three 111.
constexpr int kGradBatch = 8;
template <typename T, int V, bool WIDE>
__global__ void __launch_bounds__(256, 4) rows_from_grad_kernel(const RowsParams p) {
    using C = Columns<T, V, WIDE>;
    constexpr int LOADS = WIDE ? 2 : 4;
    __shared__ float part[8][kGradBatch];
    __shared__ int slot[8][kGradBatch];
    __shared__ float weight[8][kGradBatch];
    grid_dependency_release();
    grid_dependency_wait();
    const int t = row_token(), apart = blockDim.x, y = threadIdx.y;
    const bool inside = t < p.T;
    const int lane = threadIdx.x & 31, warp = y * (blockDim.x / 32) + (threadIdx.x >> 5), warps = blockDim.x / 32;
    const T *g = (const T *)p.x + (inside ? t : 0) * p.x_row;
    for (int j0 = 0; j0 < p.k; j0 += kGradBatch) {
        const int some = min(kGradBatch, p.k - j0);
        const long long pair = (long long)(inside ? t : 0) * p.k + j0 + threadIdx.x;
        if (threadIdx.x < kGradBatch) {
            int s = -1;
            float w = 1.f;
            if (inside && (int)threadIdx.x < some) {
                s = load_ordered(p.slots + pair);
                if (p.weights) w = load_ordered(p.weights + pair);
            }
            slot[y][threadIdx.x] = s < p.R ? s : -1;
            weight[y][threadIdx.x] = w;
        }
        __syncthreads();
        float dot[kGradBatch] = {};
        for (int c = C::first(threadIdx.x); c < p.H && inside; c += apart * V) {
            const typename C::Pack gv = C::load(g, c, apart, p.H);
#pragma unroll
            for (int j1 = 0; j1 < kGradBatch; j1 += LOADS) {
                if (j1 >= some) break;
                typename C::Pack rows[LOADS];
                if (p.weights) {
#pragma unroll
                    for (int j = 0; j < LOADS; ++j) {
                        const int s = slot[y][j1 + j];
                        if (s >= 0) rows[j] = C::load((const T *)p.y + s * p.y_row, c, apart, p.H);
                    }
                }
#pragma unroll
                for (int j = 0; j < LOADS; ++j) {
                    const int s = slot[y][j1 + j], row = s >= 0 ? s : -2 - s;       // -1: nowhere
                    if (row < 0 || row >= p.R) continue;
                    const float w = weight[y][j1 + j];
                    typename C::Pack o;
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float v = rows_float(gv.v[i]);
                        o.v[i] = rows_round<T>(s >= 0 ? w * v : 0.f);
                        if (p.weights && s >= 0) dot[j1 + j] = fmaf(v, rows_float(rows[j].v[i]), dot[j1 + j]);
                    }
                    C::store((T *)p.out_y + row * p.out_y_row, c, apart, p.H, o);
                }
            }
        }
        if (p.weights) {
#pragma unroll
            for (int j = 0; j < kGradBatch; ++j) {
#pragma unroll
                for (int d = 16; d; d /= 2) dot[j] += __shfl_xor_sync(0xFFFFFFFFu, dot[j], d);
                if (lane == 0) part[warp][j] = dot[j];
            }
        }
        __syncthreads();
        if (p.weights && (int)threadIdx.x < some && inside) {
            float sum = 0.f;
            for (int i = 0; i < warps; ++i) sum += part[y * warps + i][threadIdx.x];
            p.out_weights[pair] = sum;
        }
    }
}

// Rows that no slot names: a byte per row, set by the pair that names it; then zeros to the rows whose byte is not set.  A warp looks at 32 rows at a
// time and writes whole rows.  32768 rows of 4096 bf16 values, all of them named: 5 us for the three launches, where zeros to all of them beforehand take 70.
struct OtherRowsParams {
    const int32_t *slots;
    uint8_t *named, *rows;
    long long pairs, row, bytes;         // bytes from row to row, of a row; both and the address multiples of two
    int R;
};
__global__ void __launch_bounds__(256) mark_rows_kernel(const OtherRowsParams p) {
    grid_dependency_release();
    grid_dependency_wait();
    for (long long i = blockIdx.x * 256ll + threadIdx.x; i < p.pairs; i += gridDim.x * 256ll) {
        const int s = load_ordered(p.slots + i), row = s >= 0 ? s : -2 - s;
        if (row >= 0 && row < p.R) p.named[row] = 1;
    }
}
__global__ void __launch_bounds__(256) zero_rows_kernel(const OtherRowsParams p) {
    grid_dependency_release();
    grid_dependency_wait();
    const int lane = threadIdx.x & 31;
    for (long long r0 = (blockIdx.x * 8ll + (threadIdx.x >> 5)) * 32; r0 < p.R; r0 += gridDim.x * 256ll) {
        uint32_t rest = __ballot_sync(0xFFFFFFFFu, r0 + lane < p.R && !load_ordered(p.named + r0 + lane));
        for (; rest; rest &= rest - 1) {
            uint8_t *at = p.rows + (r0 + __ffs(rest) - 1) * p.row, *const end = at + p.bytes;
            uint8_t *const first = (uint8_t *)(((uintptr_t)at + 15) & ~(uintptr_t)15), *const last = (uint8_t *)((uintptr_t)end & ~(uintptr_t)15);
            if (last <= first) {                        // less than two 16-byte boundaries inside
                for (at += 2 * lane; at < end; at += 64) *reinterpret_cast<uint16_t *>(at) = 0;
                continue;
            }
            if (at + 2 * lane < first) *reinterpret_cast<uint16_t *>(at + 2 * lane) = 0;
            if (last + 2 * lane < end) *reinterpret_cast<uint16_t *>(last + 2 * lane) = 0;
            for (uint8_t *a = first + 16 * lane; a < last; a += 512) *reinterpret_cast<uint4 *>(a) = make_uint4(0, 0, 0, 0);
        }
    }
}
// Threads along a row and tokens per block, of 256 threads at most; `columns`: threads that a row takes.  Along a row a power of two from `least` on, or
// whole warps, as many as share the row evenly between as few blocks as will do (168 columns: 192 threads, not 256 of which a third has nothing to do).
static dim3 row_block(long long columns, int least) {
    long long x = least;
    while (x < 32 && x < columns) x *= 2;
    if (columns > 32) {
        const long long blocks = (columns + 255) / 256;
        x = ((columns + blocks - 1) / blocks + 31) / 32 * 32;
    }
    return dim3((unsigned)x, (unsigned)(256 / x));
}
static dim3 row_grid(const dim3 &block, int T, long long columns) {
    return dim3((unsigned)((T - 1) / block.y + 1), (unsigned)((columns + block.x - 1) / block.x));
}
// The largest of 16, 8, .. `least` bytes that divides them all.
static int common_bytes(int least, std::initializer_list<long long> all) {
    int b = 16;
    for (const auto v : all)
        while (b > least && v % b) b /= 2;
    return b;
}

// A matrix in memory, as the checks of overlap see it.
struct Region {
    const void *at;
    long long row, bytes, rows;          // bytes from row to row, of a row; rows
};
static Region vector_region(const void *at, long long bytes) { return {at, bytes, bytes, 1}; }
// Whether the first overlaps any of the others.
static bool meets(const Region &a, std::initializer_list<Region> others) {
    for (const Region &b : others)
        if (rows_overlap(a.at, a.row, a.bytes, a.rows, b.at, b.row, b.bytes, b.rows)) return true;
    return false;
}
// Strides up to what keeps byte offsets in 64 bits.
static bool row_ok(long long row, long long H) { return row >= H && row <= (1ll << 40); }

template <typename T, int V>
static int launch_rows_to(const RowsParams &p, cudaStream_t st) {
    const int columns = ceil_div(p.H, V);
    const dim3 block = row_block(columns, 1);
    return launch_dependent(rows_to_kernel<T, V>, row_grid(block, p.T, columns), block, 0, st, p);
}
// Calls f with the type's Columns.
template <typename F>
static int with_columns(int type, int bytes, F f) {
    if (type == HIKONV_OUT_F32) return bytes == 16 ? f(float(), Columns<float, 4, true>()) : f(float(), Columns<float, 4, false>());
    if (type == HIKONV_OUT_F16) return bytes == 16 ? f(__half(), Columns<__half, 8, true>()) : f(__half(), Columns<__half, 4, false>());
    return bytes == 16 ? f(__nv_bfloat16(), Columns<__nv_bfloat16, 8, true>()) : f(__nv_bfloat16(), Columns<__nv_bfloat16, 4, false>());
}
template <typename T, int V, bool WIDE>
static int launch_rows_from(T, Columns<T, V, WIDE>, const RowsParams &p, cudaStream_t st) {
    const int columns = ceil_div(p.H, V);
    const dim3 block = row_block(columns, 1);
    return launch_dependent(rows_from_kernel<T, V, WIDE>, row_grid(block, p.T, columns), block, 0, st, p);
}
template <typename T, int V, bool WIDE>
static int launch_rows_from_grad(T, Columns<T, V, WIDE>, const RowsParams &p, cudaStream_t st) {
    const dim3 block = row_block(ceil_div(p.H, V), 32);
    return launch_dependent(rows_from_grad_kernel<T, V, WIDE>, dim3((unsigned)((p.T - 1) / block.y + 1)), block, 0, st, p);
}
static bool is_float_type(int type) { return type == HIKONV_OUT_F32 || type == HIKONV_OUT_F16 || type == HIKONV_OUT_BF16; }
static bool pairs_ok(int T, int k) { return T >= 0 && k >= 1 && (long long)T * k <= (1 << 30); }

}  // namespace hikonv

using namespace hikonv;

extern "C" size_t hikonv_sort_by_expert_workspace_bytes(int T, int k, int E) {
    if (!pairs_ok(T, k) || E < 1 || E > HIKONV_MAX_GROUPS) return 0;
    long long per;
    const int ctas = sort_ctas((long long)T * k, &per);
    return ctas > 1 ? (size_t)ctas * (E + 1) * 4 : 0;
}

extern "C" int hikonv_sort_by_expert(const void *d_experts, int index_bytes, long long experts_row_stride, int T, int k, int E, int32_t *d_offsets,
                                     int32_t *d_slots, void *d_workspace, size_t workspace_bytes, void *stream) {
    if ((index_bytes != 4 && index_bytes != 8) || T < 0 || k < 1 || E < 1) return HIKONV_ERR_INVALID_ARG;
    if (!pairs_ok(T, k) || E > HIKONV_MAX_GROUPS) return HIKONV_ERR_UNSUPPORTED;
    if (T <= 1) experts_row_stride = k;
    if (!d_offsets || (T > 0 && (!d_experts || !d_slots)) || experts_row_stride < 0 || experts_row_stride > (1ll << 40)) return HIKONV_ERR_INVALID_ARG;
    if ((uintptr_t)d_experts % index_bytes || (uintptr_t)d_offsets % 4 || (uintptr_t)d_slots % 4) return HIKONV_ERR_INVALID_ARG;
    const long long pairs = (long long)T * k;
    SortParams p{d_experts, index_bytes == 8, experts_row_stride, pairs, k, E, 1, 0, d_offsets, d_slots, nullptr};
    p.ctas = sort_ctas(pairs, &p.per_cta);
    const long long counts = p.ctas > 1 ? (long long)p.ctas * (E + 1) * 4 : 0;
    const Region experts{d_experts, experts_row_stride * index_bytes, (long long)k * index_bytes, T}, offsets = vector_region(d_offsets, (E + 1) * 4ll),
        slots = vector_region(d_slots, pairs * 4), space = vector_region(d_workspace, counts);
    if (T > 0 && (meets(experts, {offsets, slots}) || meets(offsets, {slots}))) return HIKONV_ERR_INVALID_ARG;
    if (counts) {
        if (!d_workspace || (uintptr_t)d_workspace % 4 || workspace_bytes < (size_t)counts) return HIKONV_ERR_WORKSPACE;
        if (meets(space, {experts, offsets, slots})) return HIKONV_ERR_INVALID_ARG;
        p.counts = (uint32_t *)d_workspace;
    }
    cudaStream_t st = (cudaStream_t)stream;
    // Threads of a CTA: each warp has a row of counts to clear and to add up, each step of a warp comes after the one before, and CTAs of 1024 threads begin
    // after those of the kernel before have left.  8 pairs of 64 experts take 1.9 us with 256 threads, 2.3 with 512, 3.6 with 1024; 512 pairs 2.4, 2.5 and
    // 3.7; 2048 pairs 4.8, 3.9 and 4.4; 4104 pairs 6.1 with 512 and 7.2 with 1024; 65536 of 256 experts 8.3 and 8.2, 262144 15.9 and 11.0.
    auto sort = [&](auto threads) {
        constexpr int THREADS = decltype(threads)::value;
        if (p.counts) {
            const int rc = launch_dependent(sort_count_kernel<THREADS>, dim3((unsigned)p.ctas), dim3(THREADS), (size_t)(E + 1) * 4, st, p);
            if (rc != HIKONV_OK) return rc;
        }
        const size_t smem = ((size_t)(THREADS / 32 + 3) * (E + 1) + THREADS / 32) * 4;
        return with_dynamic_smem((const void *)sort_place_kernel<THREADS>, smem,
                                 [&] { return launch_dependent(sort_place_kernel<THREADS>, dim3((unsigned)p.ctas), dim3(THREADS), smem, st, p); });
    };
    if (pairs <= 512) return sort(std::integral_constant<int, 256>());
    if (pairs <= 1 << 16) return sort(std::integral_constant<int, 512>());
    return sort(std::integral_constant<int, 1024>());
}

extern "C" int hikonv_rows_to_experts(const void *d_x, int element_bytes, long long x_row_stride, const int32_t *d_slots, int T, int k, int H, void *d_out,
                                      long long out_row_stride, int R, void *stream) {
    if ((element_bytes != 1 && element_bytes != 2 && element_bytes != 4) || T < 0 || k < 1 || H < 1 || R < 0) return HIKONV_ERR_INVALID_ARG;
    if (!pairs_ok(T, k) || H > (1 << 23)) return HIKONV_ERR_UNSUPPORTED;
    if (T == 0 || R == 0) return HIKONV_OK;
    if (T == 1) x_row_stride = H;
    if (R == 1) out_row_stride = H;
    // a stride of 0: all tokens' rows are one
    if (!d_x || !d_slots || !d_out || x_row_stride < 0 || x_row_stride > (1ll << 40) || !row_ok(out_row_stride, H)) return HIKONV_ERR_INVALID_ARG;
    if ((uintptr_t)d_x % element_bytes || (uintptr_t)d_out % element_bytes || (uintptr_t)d_slots % 4) return HIKONV_ERR_INVALID_ARG;
    const long long size = element_bytes;
    if (meets({d_out, out_row_stride * size, H * size, R}, {{d_x, x_row_stride * size, H * size, T}, vector_region(d_slots, (long long)T * k * 4)}))
        return HIKONV_ERR_INVALID_ARG;
    const int bytes = common_bytes(element_bytes, {(long long)(uintptr_t)d_x, (long long)(uintptr_t)d_out, x_row_stride * size, out_row_stride * size, H * size});
    const int per = bytes / element_bytes;
    RowsParams p{};
    p.x = d_x; p.out = d_out; p.slots = d_slots;
    p.x_row = x_row_stride / per; p.out_row = out_row_stride / per;
    p.T = T; p.k = k; p.H = H / per; p.R = R;
    cudaStream_t st = (cudaStream_t)stream;
    switch (bytes) {
        case 16: return launch_rows_to<uint4, 1>(p, st);
        case 8: return launch_rows_to<uint2, 2>(p, st);
        case 4: return launch_rows_to<uint32_t, 4>(p, st);
    }
    p.x_row = x_row_stride * size; p.out_row = out_row_stride * size; p.H = (int)(H * size);
    constexpr int V = 4;
    const int columns = ceil_div((p.H + 6) / 4 + 1, V);
    const dim3 block = row_block(columns, 1);
    return launch_dependent(rows_to_bytes_kernel<V>, row_grid(block, T, columns), block, 0, st, p);
}

extern "C" int hikonv_rows_from_experts(const void *d_y, int type, long long y_row_stride, int R, const int32_t *d_slots, const float *d_weights, int T, int k,
                                        int H, const void *d_residual, long long residual_row_stride, void *d_out, long long out_row_stride, void *stream) {
    if (!is_float_type(type) || T < 0 || k < 1 || H < 1 || R < 0) return HIKONV_ERR_INVALID_ARG;
    if (!pairs_ok(T, k) || H > (1 << 23)) return HIKONV_ERR_UNSUPPORTED;
    if (T == 0) return HIKONV_OK;
    const int size = type == HIKONV_OUT_F32 ? 4 : 2;
    if (T == 1) residual_row_stride = out_row_stride = H;
    if (R <= 1) y_row_stride = H;
    if (!d_residual) residual_row_stride = H;
    if ((!d_y && R > 0) || !d_slots || !d_out || y_row_stride < 0 || y_row_stride > (1ll << 40) || !row_ok(residual_row_stride, H) || !row_ok(out_row_stride, H))
        return HIKONV_ERR_INVALID_ARG;
    if ((uintptr_t)d_y % size || (uintptr_t)d_out % size || (uintptr_t)d_residual % size || (uintptr_t)d_slots % 4 || (uintptr_t)d_weights % 4)
        return HIKONV_ERR_INVALID_ARG;
    const Region y{d_y, y_row_stride * size, H * size, R}, out{d_out, out_row_stride * size, H * size, T}, residual{d_residual, residual_row_stride * size, H * size, T},
        slots = vector_region(d_slots, (long long)T * k * 4), weights = vector_region(d_weights, (long long)T * k * 4);
    if (meets(out, {y, slots, weights}) || (!(d_residual == d_out && residual_row_stride == out_row_stride) && meets(out, {residual})))
        return HIKONV_ERR_INVALID_ARG;
    RowsParams p{};
    p.y = d_y; p.residual = d_residual; p.out = d_out; p.slots = d_slots; p.weights = d_weights;
    p.y_row = y_row_stride; p.res_row = residual_row_stride; p.out_row = out_row_stride;
    p.T = T; p.k = k; p.H = H; p.R = R;
    const int bytes = common_bytes(size, {(long long)(uintptr_t)d_y, (long long)(uintptr_t)d_out, (long long)(uintptr_t)d_residual, y.row, residual.row, out.row, y.bytes});
    cudaStream_t st = (cudaStream_t)stream;
    return with_columns(type, bytes, [&](auto t, auto columns) { return launch_rows_from(t, columns, p, st); });
}

extern "C" int hikonv_rows_from_experts_grad(const void *d_grad, int type, long long grad_row_stride, const void *d_y, long long y_row_stride, int R,
                                             const int32_t *d_slots, const float *d_weights, int T, int k, int H, void *d_grad_y,
                                             long long grad_y_row_stride, float *d_grad_weights, void *stream) {
    if (!is_float_type(type) || T < 0 || k < 1 || H < 1 || R < 0) return HIKONV_ERR_INVALID_ARG;
    if (!pairs_ok(T, k) || H > (1 << 23)) return HIKONV_ERR_UNSUPPORTED;
    if ((d_weights != nullptr) != (d_grad_weights != nullptr)) return HIKONV_ERR_INVALID_ARG;
    if (T == 0) return HIKONV_OK;
    const int size = type == HIKONV_OUT_F32 ? 4 : 2;
    const long long pairs = (long long)T * k;
    if (T == 1) grad_row_stride = H;
    if (R <= 1) y_row_stride = grad_y_row_stride = H;
    if (!d_weights) y_row_stride = H;
    // strides of 0: one row for all
    if (!d_grad || !d_slots || (R > 0 && (!d_grad_y || (d_weights && !d_y)))) return HIKONV_ERR_INVALID_ARG;
    if (grad_row_stride < 0 || grad_row_stride > (1ll << 40) || y_row_stride < 0 || y_row_stride > (1ll << 40) || !row_ok(grad_y_row_stride, H))
        return HIKONV_ERR_INVALID_ARG;
    if ((uintptr_t)d_grad % size || (d_weights && (uintptr_t)d_y % size) || (uintptr_t)d_grad_y % size || (uintptr_t)d_slots % 4 ||
        (uintptr_t)d_weights % 4 || (uintptr_t)d_grad_weights % 4)
        return HIKONV_ERR_INVALID_ARG;
    const long long bytes_of_row = (long long)H * size;
    const Region grad{d_grad, grad_row_stride * size, bytes_of_row, T}, y{d_weights ? d_y : nullptr, y_row_stride * size, bytes_of_row, R},
        grad_y{d_grad_y, grad_y_row_stride * size, bytes_of_row, R}, slots = vector_region(d_slots, pairs * 4), weights = vector_region(d_weights, pairs * 4),
        grad_weights = vector_region(d_grad_weights, pairs * 4);
    if (meets(grad_y, {grad, y, slots, weights, grad_weights}) || meets(grad_weights, {grad, y, slots, weights})) return HIKONV_ERR_INVALID_ARG;
    RowsParams p{};
    p.x = d_grad; p.y = d_y; p.out_y = d_grad_y; p.out_weights = d_grad_weights; p.slots = d_slots; p.weights = d_weights;
    p.x_row = grad_row_stride; p.y_row = y_row_stride; p.out_y_row = grad_y_row_stride;
    p.T = T; p.k = k; p.H = H; p.R = R;
    const int bytes = common_bytes(size, {(long long)(uintptr_t)grad.at, (long long)(uintptr_t)y.at, (long long)(uintptr_t)grad_y.at, grad.row, y.row, grad_y.row,
                                          bytes_of_row});
    cudaStream_t st = (cudaStream_t)stream;
    return with_columns(type, bytes, [&](auto t, auto columns) { return launch_rows_from_grad(t, columns, p, st); });
}

extern "C" int hikonv_zero_other_rows(const int32_t *d_slots, int T, int k, void *d_rows, int element_bytes, long long row_stride, int R, int H, void *d_workspace,
                                      size_t workspace_bytes, void *stream) {
    if ((element_bytes != 2 && element_bytes != 4) || T < 0 || k < 1 || H < 1 || R < 0) return HIKONV_ERR_INVALID_ARG;
    if (!pairs_ok(T, k) || H > (1 << 23)) return HIKONV_ERR_UNSUPPORTED;
    if (R == 0) return HIKONV_OK;
    if (R == 1) row_stride = H;
    if (!d_rows || (T > 0 && !d_slots) || !row_ok(row_stride, H) || (uintptr_t)d_rows % element_bytes || (uintptr_t)d_slots % 4) return HIKONV_ERR_INVALID_ARG;
    const Region rows{d_rows, row_stride * element_bytes, (long long)H * element_bytes, R}, slots = vector_region(d_slots, (long long)T * k * 4),
        space = vector_region(d_workspace, R);
    if (meets(rows, {slots})) return HIKONV_ERR_INVALID_ARG;
    if (!d_workspace || workspace_bytes < (size_t)R) return HIKONV_ERR_WORKSPACE;
    if (meets(space, {rows, slots})) return HIKONV_ERR_INVALID_ARG;
    cudaStream_t st = (cudaStream_t)stream;
    if (cudaMemsetAsync(d_workspace, 0, (size_t)R, st) != cudaSuccess) return HIKONV_ERR_CUDA;
    const OtherRowsParams p{d_slots, (uint8_t *)d_workspace, (uint8_t *)d_rows, (long long)T * k, rows.row, rows.bytes, R};
    const long long most = 8ll * sm_count_here(), marks = (p.pairs + 255) / 256, zeros = ((long long)R + 255) / 256;
    if (p.pairs > 0) {
        const int rc = launch_dependent(mark_rows_kernel, dim3((unsigned)(marks < most ? marks : most)), dim3(256), 0, st, p);
        if (rc != HIKONV_OK) return rc;
    }
    return launch_dependent(zero_rows_kernel, dim3((unsigned)(zeros < most ? zeros : most)), dim3(256), 0, st, p);
}
