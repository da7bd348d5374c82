// hikonv_linear, hikonv_grouped_linear: argument checks, the choice of kernel, and the kernel for rows of any alignment and any
// pair of code types (linear_mma_kernel).
#include <cstring>
#include <mutex>

#include "hikonv_linear_util.cuh"

namespace hikonv {

template <bool AU, bool BU>
__device__ __forceinline__ void mma_16x8x32(int32_t (&c)[4], const uint32_t (&a)[4], const uint32_t (&b)[2]) {
#define HIKONV_MMA(ta, tb)                                                                                                     \
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32." ta "." tb ".s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};" \
                 : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])                                                              \
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]))
    if constexpr (AU && BU) HIKONV_MMA("u8", "u8");
    else if constexpr (AU) HIKONV_MMA("u8", "s8");
    else if constexpr (BU) HIKONV_MMA("s8", "u8");
    else HIKONV_MMA("s8", "s8");
#undef HIKONV_MMA
}

// The group and row tile that block x of a grid over all groups' row tiles works on; one warp looks.  Returns first row and end.
template <int BM>
__device__ __forceinline__ void find_tile(const LinearParams &p, int want, int *e_out, int *row0, int *row_end) {
    const int lane = threadIdx.x & 31;
    int before = 0;
    for (int e0 = 0; e0 < p.E; e0 += 32) {
        int2 r = make_int2(0, 0);
        if (e0 + lane < p.E) r = group_rows(p, e0 + lane);
        const int tiles = (r.y - r.x + BM - 1) / BM;
        int upto = tiles;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int v = __shfl_up_sync(0xFFFFFFFFu, upto, d);
            if (lane >= d) upto += v;
        }
        const unsigned over = __ballot_sync(0xFFFFFFFFu, before + upto > want);
        if (over) {
            const int l = __ffs(over) - 1;
            const int first = __shfl_sync(0xFFFFFFFFu, before + upto - tiles, l);
            const int a = __shfl_sync(0xFFFFFFFFu, r.x, l), b = __shfl_sync(0xFFFFFFFFu, r.y, l);
            if (lane == 0) {
                *e_out = e0 + l;
                *row0 = a + (want - first) * BM;
                *row_end = b;
            }
            return;
        }
        before += __shfl_sync(0xFFFFFFFFu, upto, 31);
    }
    if (lane == 0) *e_out = -1;
}

// Tensor-core tiles fed through registers: every 16 codes are read from whatever byte they start at (aligned words and a funnel
// shift), dense ones unpacked, and stored to shared memory, where the next 64 of the depth are prepared while these are multiplied.
// A tile is BM rows of x by 128 rows of w; 8 warps, WM of them along the rows of x.  The pitch of 80 bytes keeps the fragments'
// 4-byte reads free of bank conflicts (row g, word t: bank 20 g + t).
constexpr int kMmaN = 128, kMmaK = 64, kMmaPitch = 80;
template <int BM, int WM, bool XU, bool WU>
__global__ void __launch_bounds__(256) linear_mma_kernel(const __grid_constant__ LinearParams p) {
    constexpr int WN = 8 / WM, TM = BM / WM / 16, TN = kMmaN / WN / 8, PIECES = kMmaK / 16;
    constexpr int XP = (BM * PIECES + 255) / 256, WP = kMmaN * PIECES / 256;
    __shared__ __align__(16) uint8_t sx[2][BM * kMmaPitch], sw[2][kMmaN * kMmaPitch];
    __shared__ int tile[3];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, wm = warp % WM, wn = warp / WM;
    grid_dependency_release();
    grid_dependency_wait();
    if (warp == 0) find_tile<BM>(p, blockIdx.x, &tile[0], &tile[1], &tile[2]);
    __syncthreads();
    const int e = tile[0], m0 = tile[1], m_end = tile[2], n0 = blockIdx.y * kMmaN;
    if (e < 0) return;
    const uint8_t *w = p.w + ((size_t)e * p.N) * p.w_row;
    const bool up = p.down > 0;

    uint32_t rx[XP][4], rw[WP][4];
    auto load = [&](int k0) {
#pragma unroll
        for (int i = 0; i < XP; ++i) {
            const int at = tid + i * 256, row = at / PIECES, k = k0 + (at % PIECES) * 16;
            const int valid = (XP * 256 == BM * PIECES || row < BM) && m0 + row < m_end ? min(max(p.K - k, 0), 16) : 0;
            load_bytes<4>(p.x + (m0 + row) * p.x_row + k, valid, rx[i]);
            keep_bytes(rx[i], valid);                  // nothing behind the row: its products would count
        }
#pragma unroll
        for (int i = 0; i < WP; ++i) {
            const int at = tid + i * 256, row = at / PIECES, k = k0 + (at % PIECES) * 16;
            const int valid = n0 + row < p.N ? min(max(p.K - k, 0), 16) : 0;
            load_weights16(w + (n0 + row) * p.w_row + ((size_t)k * p.w_bits >> 3), valid, p.w_bits, up, rw[i]);
        }
    };
    auto store = [&](int b) {
#pragma unroll
        for (int i = 0; i < XP; ++i) {
            const int at = tid + i * 256, row = at / PIECES;
            if (XP * 256 == BM * PIECES || row < BM)
                *reinterpret_cast<uint4 *>(&sx[b][row * kMmaPitch + (at % PIECES) * 16]) = make_uint4(rx[i][0], rx[i][1], rx[i][2], rx[i][3]);
        }
#pragma unroll
        for (int i = 0; i < WP; ++i) {
            const int at = tid + i * 256;
            *reinterpret_cast<uint4 *>(&sw[b][(at / PIECES) * kMmaPitch + (at % PIECES) * 16]) = make_uint4(rw[i][0], rw[i][1], rw[i][2], rw[i][3]);
        }
    };

    int32_t acc[TM][TN][4] = {};
    const int g = lane >> 2, t = lane & 3;
    load(0);
    store(0);
    __syncthreads();
    for (int k0 = 0, b = 0; k0 < p.K; k0 += kMmaK, b ^= 1) {
        const bool more = k0 + kMmaK < p.K;
        if (more) load(k0 + kMmaK);
#pragma unroll
        for (int kk = 0; kk < kMmaK; kk += 32) {
            uint32_t fb[TN][2];
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const uint8_t *at = &sw[b][(wn * TN * 8 + j * 8 + g) * kMmaPitch + kk + t * 4];
                fb[j][0] = *reinterpret_cast<const uint32_t *>(at);
                fb[j][1] = *reinterpret_cast<const uint32_t *>(at + 16);
            }
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const uint8_t *at = &sx[b][(wm * TM * 16 + i * 16 + g) * kMmaPitch + kk + t * 4];
                const uint32_t fa[4] = {*reinterpret_cast<const uint32_t *>(at), *reinterpret_cast<const uint32_t *>(at + 8 * kMmaPitch),
                                        *reinterpret_cast<const uint32_t *>(at + 16), *reinterpret_cast<const uint32_t *>(at + 8 * kMmaPitch + 16)};
#pragma unroll
                for (int j = 0; j < TN; ++j) mma_16x8x32<XU, WU>(acc[i][j], fa, fb[j]);
            }
        }
        if (more) store(b ^ 1);                        // the other buffer: its readers passed the barrier of the step before
        __syncthreads();
    }

    with_out_type(p.out_type, [&](auto kind) {
        constexpr int OUT = decltype(kind)::value;
        using T = typename OutElem<OUT>::type;
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int n = n0 + wn * TN * 8 + j * 8 + t * 2 + c;
                if (n >= p.N) continue;
                const ColumnTerms terms = column_terms<OUT>(p, e, n);
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const int m = m0 + wm * TM * 16 + i * 16 + g + r * 8;
                        if (m >= m_end) continue;
                        const float xs = p.x_scale ? load_ordered(p.x_scale + m) : 1.f;
                        ((T *)p.out)[m * p.out_row + n] =
                            finish<OUT>(p, acc[i][j][r * 2 + c] >> p.down, xs, terms, residual_at<T>(p, m, n));
                    }
            }
    });
}

template <int BM, int WM>
static int launch_mma_tile(const LinearParams &p, cudaStream_t st) {
    const long long tiles = p.offsets ? p.M / BM + (p.E < p.M ? p.E : p.M) : ((long long)p.M + BM - 1) / BM;
    const int nt = ceil_div(p.N, kMmaN);
    if (tiles > 0x7FFFFFFFll || nt > 65535) return HIKONV_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)tiles, (unsigned)nt);
    if (p.x_u8 && p.w_u8) return launch_dependent(linear_mma_kernel<BM, WM, true, true>, grid, dim3(256), 0, st, p);
    if (p.x_u8) return launch_dependent(linear_mma_kernel<BM, WM, true, false>, grid, dim3(256), 0, st, p);
    if (p.w_u8) return launch_dependent(linear_mma_kernel<BM, WM, false, true>, grid, dim3(256), 0, st, p);
    return launch_dependent(linear_mma_kernel<BM, WM, false, false>, grid, dim3(256), 0, st, p);
}

int launch_linear_mma(const LinearParams &p, cudaStream_t st) {
    const int rows = p.offsets ? ceil_div(p.M, p.E) : p.M;       // of a group, on average
    return rows <= 16 ? launch_mma_tile<16, 1>(p, st) : launch_mma_tile<128, 2>(p, st);
}

static size_t element_bytes(int out_type) {
    return out_type == HIKONV_OUT_CODES ? 1 : out_type == HIKONV_OUT_SUMS || out_type == HIKONV_OUT_F32 ? 4 : 2;
}
// Whether two memory ranges have a byte in common.
static bool overlap(const void *a, size_t an, const void *b, size_t bn) {
    return a && b && an && bn && (uintptr_t)a < (uintptr_t)b + bn && (uintptr_t)b < (uintptr_t)a + an;
}

static int linear_run(const void *d_x, long long x_row, const void *d_w, int w_bits, const int32_t *d_offsets, int grouped, int E, int M,
                      int N, int K, int p, int q, int xs, int ws, void *d_out, long long out_row, const hikonv_epilogue_t *ep, void *stream) {
    const int rc = validate_codes(p, q);
    if (rc != HIKONV_OK) return rc;
    if (!ep || M < 0 || N < 1 || K < 1 || E < 1) return HIKONV_ERR_INVALID_ARG;
    if (E > HIKONV_MAX_GROUPS) return HIKONV_ERR_UNSUPPORTED;
    const int type = ep->out_type, real = type >= HIKONV_OUT_F32;
    if (type < HIKONV_OUT_SUMS || type > HIKONV_OUT_BF16) return HIKONV_ERR_INVALID_ARG;
    if (ep->activation < HIKONV_ACT_NONE || ep->activation > HIKONV_ACT_GELU) return HIKONV_ERR_INVALID_ARG;
    if (!real && (ep->activation || ep->d_x_scale || ep->d_w_scale || ep->d_residual)) return HIKONV_ERR_INVALID_ARG;
    if (type == HIKONV_OUT_SUMS && ep->d_bias) return HIKONV_ERR_INVALID_ARG;
    if (type == HIKONV_OUT_CODES) {
        if (ep->shift < 0 || ep->shift > 31 || ep->lo < -128 || ep->hi > 255 || ep->lo > ep->hi) return HIKONV_ERR_INVALID_ARG;
    } else if (ep->shift || ep->lo || ep->hi) {
        return HIKONV_ERR_INVALID_ARG;
    }
    if (w_bits != 8 && (w_bits != q || (q != 1 && q != 2 && q != 4))) return HIKONV_ERR_INVALID_ARG;
    if (((long long)K * w_bits) % 8 != 0) return HIKONV_ERR_UNSUPPORTED;
    const long long xmax = xs ? 1ll << (p - 1) : (1ll << p) - 1, wmax = ws ? 128 : (1ll << q) - 1;
    if (K * xmax * wmax > 0x7FFFFFFFll) return HIKONV_ERR_NO_FIT;
    if (M == 0) return HIKONV_OK;
    if (M == 1) x_row = K, out_row = N;                          // there is no second row
    const long long res_row = M == 1 ? N : ep->residual_row_stride;
    if (!d_x || !d_w || !d_out || (grouped && !d_offsets)) return HIKONV_ERR_INVALID_ARG;
    if (x_row < K || out_row < N || (ep->d_residual && res_row < N)) return HIKONV_ERR_INVALID_ARG;
    if (x_row > (1ll << 40) || out_row > (1ll << 40) || res_row > (1ll << 40)) return HIKONV_ERR_INVALID_ARG;   // byte offsets stay in 64 bits
    const size_t elem = element_bytes(type);
    if ((uintptr_t)d_out % elem || (uintptr_t)ep->d_residual % elem || (uintptr_t)ep->d_bias % 4 || (uintptr_t)ep->d_x_scale % 4 ||
        (uintptr_t)ep->d_w_scale % 4 || (uintptr_t)d_offsets % 4)
        return HIKONV_ERR_INVALID_ARG;
    const long long w_row = (long long)K * w_bits / 8;
    const size_t out_bytes = ((size_t)(M - 1) * out_row + N) * elem, columns = (size_t)E * N * 4;
    if (overlap(d_out, out_bytes, d_x, (size_t)(M - 1) * x_row + K) || overlap(d_out, out_bytes, d_w, (size_t)E * N * w_row) ||
        overlap(d_out, out_bytes, d_offsets, ((size_t)E + 1) * 4) || overlap(d_out, out_bytes, ep->d_x_scale, (size_t)M * 4) ||
        overlap(d_out, out_bytes, ep->d_w_scale, columns) || overlap(d_out, out_bytes, ep->d_bias, columns))
        return HIKONV_ERR_INVALID_ARG;
    if (ep->d_residual && !(ep->d_residual == d_out && res_row == out_row) &&
        overlap(d_out, out_bytes, ep->d_residual, ((size_t)(M - 1) * res_row + N) * elem))
        return HIKONV_ERR_INVALID_ARG;

    LinearParams k;
    memset(&k, 0, sizeof(k));
    k.x = (const uint8_t *)d_x; k.w = (const uint8_t *)d_w; k.offsets = d_offsets;
    k.x_row = x_row; k.w_row = w_row;
    k.M = M; k.N = N; k.K = K; k.E = E;
    k.x_signed = xs; k.w_signed = ws;
    k.x_u8 = !xs && p == 8; k.w_u8 = !ws && q == 8;
    k.w_bits = w_bits;
    k.down = w_bits < 8 && ws ? 8 - w_bits : 0;
    k.out_type = type; k.act = ep->activation;
    k.out = d_out; k.residual = ep->d_residual; k.bias = ep->d_bias;
    k.x_scale = ep->d_x_scale; k.w_scale = ep->d_w_scale;
    k.out_row = out_row; k.res_row = res_row;
    k.shift = ep->shift; k.lo = ep->lo; k.hi = ep->hi;
    const int rows = grouped ? ceil_div(M, E) : M;               // of a group, on average
    if (linear_rows_takes(k, rows)) return launch_linear_rows(k, (cudaStream_t)stream);
    return linear_tc_takes(k) ? launch_linear_tc(k, (cudaStream_t)stream) : launch_linear_mma(k, (cudaStream_t)stream);
}

}  // namespace hikonv

using namespace hikonv;

extern "C" int hikonv_linear(const void *d_x, long long x_row_stride, const void *d_w, int w_store_bits, int M, int N, int K, int p, int q,
                             int x_signed, int w_signed, void *d_out, long long out_row_stride, const hikonv_epilogue_t *epilogue,
                             void *stream) {
    return linear_run(d_x, x_row_stride, d_w, w_store_bits, nullptr, 0, 1, M, N, K, p, q, x_signed != 0, w_signed != 0, d_out, out_row_stride,
                      epilogue, stream);
}

extern "C" int hikonv_grouped_linear(const void *d_x, long long x_row_stride, const void *d_w, int w_store_bits, const int32_t *d_offsets,
                                     int E, int T, int N, int K, int p, int q, int x_signed, int w_signed, void *d_out,
                                     long long out_row_stride, const hikonv_epilogue_t *epilogue, void *stream) {
    return linear_run(d_x, x_row_stride, d_w, w_store_bits, d_offsets, 1, E, T, N, K, p, q, x_signed != 0, w_signed != 0, d_out,
                      out_row_stride, epilogue, stream);
}

extern "C" int hikonv_linear_wait_timeouts(unsigned int *h_count) {
    if (!h_count) return HIKONV_ERR_INVALID_ARG;
    constexpr int kDevices = 64;
    static std::mutex mutex;
    static unsigned int told[kDevices];                              // what earlier calls have reported
    *h_count = 0;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kDevices || cudaDeviceSynchronize() != cudaSuccess) return HIKONV_ERR_CUDA;
    std::lock_guard<std::mutex> lock(mutex);
    unsigned int total = 0;
    const int rc = read_linear_timeouts(&total);
    if (rc != HIKONV_OK) return rc;
    *h_count = total - told[dev];
    told[dev] = total;
    return HIKONV_OK;
}

extern "C" int hikonv_linear_wait_check(long long cycles, void *stream) {
    if (cycles < 0 || cycles > kWaitCycles) return HIKONV_ERR_INVALID_ARG;
    return launch_linear_wait_check(cycles, (cudaStream_t)stream);
}
