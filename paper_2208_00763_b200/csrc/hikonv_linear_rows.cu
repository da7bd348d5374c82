// Linear layers on a few rows of x (one new token, or a handful): the weights stream by once.
//
// Each weight is used once per row of x, so the call reads N K q / 8 bytes for 2 M N K operations and is bound by that stream, or, when
// small, by latency: no accumulators to set up, no staging of the weights.  A warp takes 16 rows of w and up to 8 rows of x through the
// register-fed tensor instruction (mma.sync 16x8x32).  Byte dot products would need M N K / 4 of an instruction that measured about
// five per cycle and SM here (one row of x against 4096 x 4096: 9 us of them); this instruction does 420 products per cycle and SM.
//
// A sum does not care for the order of its terms, so the codes are not brought into the instruction's order: a thread's 16 bytes of a
// row are its operands for two steps (dense weights: 2 * 8 / b steps), and x is read, or staged, in the same order.
// The warps of a CTA share the depth of a tile and add their parts in shared memory.
//
// Rows of w may start on any byte.  All rows of a tile start on the same byte of a 16-byte piece (rows r, r + D, r + 2 D, ... with
// D = 16 / gcd(16, row bytes)) and are read in aligned pieces; x is then staged in shared memory, moved by that many bytes and with
// zeros around it, which is what the pieces' stray bytes at both ends of a row meet.  Where all rows start on 16-byte boundaries x is
// read as it is, without staging or a barrier.
// From memory: 1 x 4096 x 4096 in 4.7 us (8-bit weights, 3.6 TB/s) and 3.9 us (4-bit), 8 x 4096 x 8192 8-bit in 7.7 us (4.4 TB/s), 128 rows
// over 64 groups of 2048 x 2048 4-bit weights in 31 us (3.7 TB/s).  Sixteen warps per SM, by their registers, hold too few loads to
// fill the memory's pipe; a ring of asynchronous copies in shared memory in their place was slower (1 x 4096 x 4096: 5.8 us, for the staging
// of x that it needs), and so were 24 warps with spilled registers.
#include <cstring>

#include "hikonv_linear_util.cuh"

namespace hikonv {

constexpr int kRowsWarps = 8, kRowsThreads = kRowsWarps * 32;
// 64-byte parts of a tile's rows in flight per warp: what the registers hold of them and of the x that they meet.
template <int BITS, int TOK> constexpr int kRowsUnroll = BITS == 8 ? (TOK == 8 ? 4 : 3) : BITS == 4 ? (TOK == 8 ? 4 : 2) : BITS == 2 ? (TOK == 8 ? 2 : 1) : 1;
constexpr int kRowsMostSmem = 39 * 1024;    // with the parts, what needs no raised limit

struct RowsParams {
    LinearParams p;
    int ksplit;                         // warps that share a tile's depth: 1, 2, 4 or 8
    int classes;                        // D
    int class_tiles;                    // tiles of 16 rows per class
    int x_pieces, x_pitch;              // staged x: pieces per row, words from row to row
};

template <bool XU, bool WU>
__device__ __forceinline__ void mma_rows(int32_t (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
#define HIKONV_MMA(ta, tb)                                                                                                      \
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32." ta "." tb ".s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};" \
                 : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])                                                               \
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1))
    if constexpr (XU && WU) HIKONV_MMA("u8", "u8");
    else if constexpr (XU) HIKONV_MMA("s8", "u8");
    else if constexpr (WU) HIKONV_MMA("u8", "s8");
    else HIKONV_MMA("s8", "s8");
#undef HIKONV_MMA
}

// 16 codes (1-bit weights: 32) of x to the order in which the masked words of w ask for them.
template <int PER_BYTE>
__device__ __forceinline__ void reorder(uint32_t (&v)[PER_BYTE == 8 ? 8 : 4]) {
    auto transpose = [](uint32_t &a, uint32_t &b, uint32_t &c, uint32_t &d) {      // byte i of word j to byte j of word i
        const uint32_t ab0 = byte_permute(a, b, 0x5140), ab1 = byte_permute(a, b, 0x7362);
        const uint32_t cd0 = byte_permute(c, d, 0x5140), cd1 = byte_permute(c, d, 0x7362);
        a = byte_permute(ab0, cd0, 0x5410);
        b = byte_permute(ab0, cd0, 0x7632);
        c = byte_permute(ab1, cd1, 0x5410);
        d = byte_permute(ab1, cd1, 0x7632);
    };
    if constexpr (PER_BYTE == 2) {                      // even codes, then odd ones, of eight
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            const uint32_t even = byte_permute(v[i], v[i + 1], 0x6420), odd = byte_permute(v[i], v[i + 1], 0x7531);
            v[i] = even;
            v[i + 1] = odd;
        }
    } else if constexpr (PER_BYTE == 4) {
        transpose(v[0], v[1], v[2], v[3]);
    } else if constexpr (PER_BYTE == 8) {               // code j + 8 b is byte j % 4 of word 2 b + j / 4
        uint32_t t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = v[i];
        transpose(t[0], t[2], t[4], t[6]);
        transpose(t[1], t[3], t[5], t[7]);
        v[0] = t[0]; v[1] = t[2]; v[2] = t[4]; v[3] = t[6];
        v[4] = t[1]; v[5] = t[3]; v[6] = t[5]; v[7] = t[7];
    }
}

__device__ __forceinline__ void split16(const uint4 &o, uint32_t *v) {
    v[0] = o.x; v[1] = o.y; v[2] = o.z; v[3] = o.w;
}

// The masked word of w that holds the codes at position `pos` of its bytes.
template <int BITS>
__device__ __forceinline__ uint32_t codes_at(uint32_t w, int pos, int down) {
    if constexpr (BITS == 8) return w;
    constexpr uint32_t LOW = ((1u << BITS) - 1u) * 0x01010101u, HIGH = LOW << (8 - BITS);
    return down ? (w << (8 - BITS - pos * BITS)) & HIGH : (w >> (pos * BITS)) & LOW;
}

template <int BITS, int TOK, bool STAGED, bool XU, bool WU>
__global__ void __launch_bounds__(kRowsThreads, 2) linear_rows_kernel(const __grid_constant__ RowsParams q) {
    constexpr int PER_BYTE = 8 / BITS;                  // codes per byte of w; words of x per word of w
    constexpr int XW = 4 * PER_BYTE;                    // words of x per piece of w
    constexpr int GROUP = PER_BYTE == 8 ? 8 : 4;        // words that reorder() takes
    constexpr int UNROLL = kRowsUnroll<BITS, TOK>;
    extern __shared__ __align__(16) uint32_t sx[];      // [TOK][x_pitch]: per row [PER_BYTE][x_pieces] of 16 bytes
    __shared__ int32_t part[kRowsWarps][16 * TOK];
    __shared__ float x_scales[TOK];
    const LinearParams &p = q.p;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int tiles_per_cta = kRowsWarps / q.ksplit, ways = (q.class_tiles + tiles_per_cta - 1) / tiles_per_cta;
    const int cls = blockIdx.x / ways, e = blockIdx.y;
    const int local = warp / q.ksplit, ks = warp % q.ksplit;
    const int tile0 = ((int)blockIdx.x % ways) * tiles_per_cta;
    const uint8_t *w0 = p.w + (long long)e * p.N * p.w_row;
    const int off = STAGED ? (int)((uintptr_t)(w0 + cls * p.w_row) & 15) : 0;
    const int pieces = (int)((off + p.w_row + 15) >> 4), parts = (pieces + 3) >> 2;
    const int part0 = (int)((long long)parts * ks / q.ksplit), part1 = (int)((long long)parts * (ks + 1) / q.ksplit);
    auto row_of = [&](int tile, int r) { return cls + (tile * 16 + r) * q.classes; };
    // this thread's rows of w: their pieces from aligned addresses, nothing (null) where there is no such row
    const uint8_t *src[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int n = row_of(tile0 + local, g + 8 * h);
        src[h] = n < p.N ? w0 + n * p.w_row - off : nullptr;
    }
    auto load_w = [&](int h, int j) -> uint4 {
        if (!src[h] || j >= pieces) return make_uint4(0, 0, 0, 0);
        const uint8_t *a = src[h] + j * 16;
        if (!STAGED) return load_ordered(reinterpret_cast<const uint4 *>(a));
        const uint8_t *begin = src[h] + off, *end = begin + p.w_row;
        if (a >= begin && a + 16 <= end) return load_ordered(reinterpret_cast<const uint4 *>(a));
        uint32_t o[4];                                  // the ends of the row: only words that hold some of it
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = a + k * 4 + 4 > begin && a + k * 4 < end ? load_ordered(reinterpret_cast<const uint32_t *>(a) + k) : 0u;
        return make_uint4(o[0], o[1], o[2], o[3]);
    };

    grid_dependency_release();
    // This warp's share of its tile on its way to the second-level cache: a hint, so it need not wait for the kernel before, and it is
    // not bounded by registers as loads are.  From memory, 1 x 4096 x 4096 8-bit weights 5.4 -> 4.6 us.
    if (!p.offsets) {
        const long long b0 = (long long)part0 * 64, share = min((long long)(part1 - part0) * 64, p.w_row - b0);
        const int lines = (int)((min(share, 2048ll) + 127) >> 7);
        for (int i = lane; i < 16 * lines; i += 32) {
            const int n = row_of(tile0 + local, i & 15);
            if (n < p.N && b0 + (i >> 4) * 128 < p.w_row) asm volatile("prefetch.global.L2 [%0];" ::"l"(w0 + n * p.w_row + b0 + (i >> 4) * 128));
        }
    }
    grid_dependency_wait();
    const int2 range = group_rows(p, e);
    // the output that this thread writes: 128 of them per tile, dealt out over the tile's warps
    const int threads = q.ksplit * 32, who = tid % threads;
    const int own_n = row_of(tile0 + local, who & 15);
    ColumnTerms terms{1.f, 0.f, 0};
    if (own_n < p.N && range.x < range.y) {
        const size_t column = (size_t)e * p.N + own_n;
        if (p.w_scale) terms.scale = load_ordered(p.w_scale + column);
        if (p.bias) terms.ibias = load_ordered((const int32_t *)p.bias + column);
        if (p.out_type != HIKONV_OUT_CODES) terms.bias = __int_as_float(terms.ibias);
    }
    for (int m0 = range.x; m0 < range.y; m0 += TOK) {
        const int rows = min(TOK, range.y - m0);
        if (STAGED) {
            if (m0 > range.x) __syncthreads();
            const int units = (pieces * XW + GROUP - 1) / GROUP;
            for (int at = tid; at < rows * units; at += kRowsThreads) {
                const int r = at / units, u = at - r * units;
                const uint8_t *x = p.x + (m0 + r) * p.x_row;
                uint32_t v[GROUP];
                const int k0 = u * GROUP * 4 - off * PER_BYTE;
                if (k0 >= 0 && k0 + GROUP * 4 <= p.K) {
                    load_bytes<GROUP>(x + k0, GROUP * 4, v);
                } else {
#pragma unroll
                    for (int i = 0; i < GROUP; ++i) {
                        v[i] = 0;
#pragma unroll
                        for (int b = 0; b < 4; ++b) {
                            const int k = k0 + i * 4 + b;
                            if (k >= 0 && k < p.K) v[i] |= (uint32_t)load_ordered(x + k) << (8 * b);
                        }
                    }
                }
                reorder<PER_BYTE>(v);
#pragma unroll
                for (int i = 0; i < GROUP; i += 4) {
                    const int h = (u * GROUP + i) / 4 % PER_BYTE, j = (u * GROUP + i) / XW;
                    *reinterpret_cast<uint4 *>(sx + r * q.x_pitch + (h * q.x_pieces + j) * 4) = make_uint4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                }
            }
            __syncthreads();
        }
        const uint8_t *x[TOK / 8];
#pragma unroll
        for (int b = 0; b < TOK / 8; ++b) x[b] = g + 8 * b < rows ? p.x + (m0 + g + 8 * b) * p.x_row : nullptr;
        int32_t acc[TOK / 8][4] = {};
        float own_scale = 1.f;                          // on its way to shared memory while the weights stream
        if (tid < rows && p.x_scale) own_scale = load_ordered(p.x_scale + m0 + tid);
        for (int c = part0; c < part1; c += UNROLL) {
            uint4 w[UNROLL][2];
            uint32_t xv[UNROLL][TOK / 8][XW];
#pragma unroll
            for (int i = 0; i < UNROLL; ++i) {
                const int j = (c + i) * 4 + t;
                const bool mine = c + i < part1 && j < pieces;
#pragma unroll
                for (int h = 0; h < 2; ++h) w[i][h] = mine ? load_w(h, j) : make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int b = 0; b < TOK / 8; ++b)
#pragma unroll
                    for (int h = 0; h < PER_BYTE; ++h) {
                        uint4 o = make_uint4(0, 0, 0, 0);
                        if (x[b] && mine) {
                            if (STAGED) o = *reinterpret_cast<const uint4 *>(sx + (g + 8 * b) * q.x_pitch + (h * q.x_pieces + j) * 4);
                            else o = load_ordered(reinterpret_cast<const uint4 *>(x[b]) + j * PER_BYTE + h);
                        }
                        split16(o, &xv[i][b][h * 4]);
                    }
            }
#pragma unroll
            for (int i = 0; i < UNROLL; ++i) {
                if (!STAGED && PER_BYTE > 1) {
#pragma unroll
                    for (int b = 0; b < TOK / 8; ++b)
#pragma unroll
                        for (int k = 0; k < XW; k += GROUP) reorder<PER_BYTE>(*reinterpret_cast<uint32_t(*)[GROUP]>(&xv[i][b][k]));
                }
                uint32_t wa[4], wb[4];
                split16(w[i][0], wa);
                split16(w[i][1], wb);
#pragma unroll
                for (int k = 0; k < XW; k += 2) {
                    // words k and k + 1 of the order in which x lies: word k / PER_BYTE of w, position k % PER_BYTE
                    const uint32_t a0 = codes_at<BITS>(wa[k / PER_BYTE], k % PER_BYTE, p.down), a1 = codes_at<BITS>(wb[k / PER_BYTE], k % PER_BYTE, p.down);
                    const uint32_t a2 = codes_at<BITS>(wa[(k + 1) / PER_BYTE], (k + 1) % PER_BYTE, p.down);
                    const uint32_t a3 = codes_at<BITS>(wb[(k + 1) / PER_BYTE], (k + 1) % PER_BYTE, p.down);
#pragma unroll
                    for (int b = 0; b < TOK / 8; ++b) mma_rows<XU, WU>(acc[b], a0, a1, a2, a3, xv[i][b][k], xv[i][b][k + 1]);
                }
            }
        }
        if (m0 > range.x) __syncthreads();              // the parts of the rows before have been read
        // rows g and g + 8 of the tile, rows 2 t and 2 t + 1 of each eight of x
#pragma unroll
        for (int b = 0; b < TOK / 8; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) part[warp][(8 * b + 2 * t + (i & 1)) * 16 + g + (i >> 1) * 8] = acc[b][i];
        if (tid < rows) x_scales[tid] = own_scale;
        __syncthreads();
        for (int i = who; i < rows * 16; i += threads) {
            int32_t sum = 0;
            for (int s = 0; s < q.ksplit; ++s) sum += part[local * q.ksplit + s][i];
            if (own_n >= p.N) break;
            const long long m = m0 + (i >> 4);
            with_out_type(p.out_type, [&](auto kind) {
                constexpr int OUT = decltype(kind)::value;
                using T = typename OutElem<OUT>::type;
                ((T *)p.out)[m * p.out_row + own_n] = finish<OUT>(p, sum >> p.down, x_scales[i >> 4], terms, residual_at<T>(p, m, own_n));
            });
        }
    }
}

static int gcd16(long long v) {
    int g = 16;
    while (v % g) g /= 2;
    return g;
}
// Whether x need not be moved: every row of x and w on a 16-byte boundary.
static bool rows_as_they_are(const LinearParams &p) {
    return (uintptr_t)p.w % 16 == 0 && p.w_row % 16 == 0 && (uintptr_t)p.x % 16 == 0 && (p.M == 1 || p.x_row % 16 == 0);
}
// Pieces of a row of w that starts in the middle of one, and the words from one staged row of x to the next: 64 bytes off a multiple of
// 128, so that the eight threads of a 16-byte access that read two rows meet in no bank.
static long long staged_pieces(const LinearParams &p) { return (15 + p.w_row + 15) / 16; }
static long long staged_pitch(const LinearParams &p) { return (staged_pieces(p) * 4 * (8 / p.w_bits) + 31) / 32 * 32 + 16; }

// Rows of x at a time.
static int rows_at_a_time(const LinearParams &p) { return p.offsets || p.M <= 8 ? 8 : 16; }

// Where this kernel is the faster one.  Both are a set-up and a time per weight, in us, measured on weights from memory, for x = N K E /
// 2^24 weights and R rows, at x from 1/64 to 32.  Here: 8-bit 2.0 + 3.1 x, or 2.0 + 3.6 x beyond 8 rows; 4-bit 2.0 + 2.0 x or
// 2.0 + 2.65 x; 2-bit 2.2 + (1.65 + R / 15) x; 1-bit 2.5 + (1.5 + R / 5) x; and 4.2 us per 2^20 outputs.  On tcgen05 tiles, whose set-up
// has more CTAs to join where there is depth to share: 8-bit 3.0 + 1.3 d + 2.4 x for d = min(1, K / 2048); fewer bits
// 3.2 + 2.8 d + 1.35 x, in groups 5.6 + 1.85 x (4-bit) or 5.6 + 1.6 x.  Rows that do not start on 16-byte boundaries: 1 us and 0.9 us per
// 4096 staged codes of x more here, a launch and a copy of the weights more there.
bool linear_rows_takes(const LinearParams &p, int rows) {
    if (rows > (p.offsets ? 8 : kLinearFewRows) || p.E > 65535) return false;
    const bool stays = rows_as_they_are(p);
    if (!stays && staged_pitch(p) * 4 * (p.offsets ? 8 : p.M) > kRowsMostSmem) return false;
    const double x = (double)p.N * p.K * p.E / (1 << 24), depth = p.K < 2048 ? p.K / 2048.0 : 1.0;
    const bool eight = rows_at_a_time(p) == 8;
    double here, tiles;
    switch (p.w_bits) {
        case 8: here = 2.0 + (eight ? 3.1 : 3.6) * x; break;
        case 4: here = 2.0 + (eight ? 2.0 : 2.65) * x; break;
        case 2: here = 2.2 + (1.65 + rows / 15.0) * x; break;
        default: here = 2.5 + (1.5 + rows / 5.0) * x;
    }
    here += 4.2 * p.M * p.N / (1 << 20);
    if (p.w_bits == 8) tiles = 3.0 + 1.3 * depth + 2.4 * x;
    else if (!p.offsets) tiles = 3.2 + 2.8 * depth + 1.35 * x;
    else tiles = 5.6 + (p.w_bits == 4 ? 1.85 : 1.6) * x;
    if (!stays) {
        here += 1.0 + 0.9 / 4096 * rows * p.K;
        tiles += 0.9 + 4.8 * x * p.w_bits / 8;
    }
    return here <= tiles;
}

template <int BITS, int TOK, bool STAGED>
static int launch_rows(const RowsParams &q, dim3 grid, size_t smem, cudaStream_t st) {
    auto launch = [&](auto kernel) { return launch_dependent(kernel, grid, dim3(kRowsThreads), smem, st, q); };
    if constexpr (BITS == 8) {
        if (q.p.w_u8)
            return q.p.x_u8 ? launch(linear_rows_kernel<8, TOK, STAGED, true, true>) : launch(linear_rows_kernel<8, TOK, STAGED, false, true>);
    }
    return q.p.x_u8 ? launch(linear_rows_kernel<BITS, TOK, STAGED, true, false>) : launch(linear_rows_kernel<BITS, TOK, STAGED, false, false>);
}
template <int TOK, bool STAGED>
static int launch_rows_bits(const RowsParams &q, dim3 grid, size_t smem, cudaStream_t st) {
    switch (q.p.w_bits) {
        case 8: return launch_rows<8, TOK, STAGED>(q, grid, smem, st);
        case 4: return launch_rows<4, TOK, STAGED>(q, grid, smem, st);
        case 2: return launch_rows<2, TOK, STAGED>(q, grid, smem, st);
        default: return launch_rows<1, TOK, STAGED>(q, grid, smem, st);
    }
}

int launch_linear_rows(const LinearParams &p, cudaStream_t st) {
    RowsParams q;
    memset(&q, 0, sizeof(q));
    q.p = p;
    const int sms = sm_count_here();
    const bool staged = !rows_as_they_are(p);
    q.classes = 16 / gcd16(p.w_row);
    q.class_tiles = ceil_div(ceil_div(p.N, q.classes), 16);
    if (staged) {
        q.x_pieces = (int)staged_pieces(p);
        q.x_pitch = (int)staged_pitch(p);
    }
    // All warps of a CTA on one tile, however short its rows: they share the tile's outputs, too (16 x 1024 x 1024 1-bit: 9.5 us by one
    // warp per tile, 3.4 by eight).  But no more CTAs than the GPU holds at once: each that comes later waits for its first weights anew
    // (eight groups of 2048 x 2048 4-bit weights, 8 rows: 13.3 us in 1024 CTAs, 8.5 in 512, 6.4 in 256; 1 x 4096 x 16384 8-bit: 16.7,
    // 15.3, 13.9).
    q.ksplit = kRowsWarps;
    while (q.ksplit > 1 && (long long)q.class_tiles * q.classes * p.E * q.ksplit > (long long)sms * 2 * kRowsWarps) q.ksplit /= 2;
    const int ways = ceil_div(q.class_tiles, kRowsWarps / q.ksplit);
    const dim3 grid((unsigned)(ways * q.classes), (unsigned)p.E);
    const size_t smem = (size_t)q.x_pitch * 4 * (p.offsets ? 8 : p.M);
    if (rows_at_a_time(p) == 8) return staged ? launch_rows_bits<8, true>(q, grid, smem, st) : launch_rows_bits<8, false>(q, grid, smem, st);
    return staged ? launch_rows_bits<16, true>(q, grid, smem, st) : launch_rows_bits<16, false>(q, grid, smem, st);
}

}  // namespace hikonv
