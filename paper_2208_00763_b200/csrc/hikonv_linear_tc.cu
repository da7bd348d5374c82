// Linear layers on the tensor cores: tcgen05.mma on byte codes (kind::i8, int32 sums in tensor memory), operands staged in shared
// memory by TMA.
//
// The WEIGHTS are the matrix of 128 rows and the rows of x the matrix of up to 256 columns: D[n][m] = sum_k w[n][k] x[m][k].  The
// number of columns can be any multiple of 16, so one token costs 16 columns instead of 128 rows, a group's last tile costs what it
// has, and the columns of a tile can be chosen so that the tiles fill the SMs evenly.  A lane of tensor memory is an output column of
// the layer: its scale and bias are one register each, and a warp writes 32 neighbours of an output row at a time.
//
// One CTA per SM walks over the tiles.  Warp 0 loads, warp 1 multiplies, warps 4 to 11 take finished sums through the epilogue while the
// next tile is multiplied (two accumulators), and, where the operands are not yet bytes of one sign, warps 12 to 23 change them between
// the two: dense weights are unpacked into tensor memory, and unsigned 8-bit activations of signed weights get 128 subtracted (their top bit flipped; the instruction takes either two signed or two unsigned operands here).  What that takes
// off, 128 sum_k w[n][k], comes from the multiply itself: a row of ones behind the rows of x makes a column of those sums.  Unsigned 8-bit
// weights of signed activations, the rare case, are flipped too, and 128 sum_k x[m][k] is added by multiplying x twice by a tile of 64s:
// 4096^3 in 143 us, where signed codes take 66 and unsigned activations of signed weights 102.
// TMA wants rows on 16-byte boundaries.  Operands whose rows start anywhere are copied to rows that do in a launch of their own
// (align_rows_kernel): read by helper warps word by word instead, 433 x 9100 x 4352 took 103 us and 333 x 1001 x 1501 13.3.
//
// Small layers have fewer tiles than there are SMs: there the CTAs of a cluster share a tile's depth, and the cluster adds their sums
// through distributed shared memory, each CTA finishing its part of the tile's output columns.
//
// 4096 x 4096 x 16384 with GELU: 196 us without the activation in a short burst, 232 with it, 252 back to back for seconds (2.2 P
// operations per second; the 1000 W limit then holds the clock near 1.2 GHz).  A step of 128 codes on a 256-row tile takes 650 cycles
// where its multiplies take 512: 148 SMs fetch 70 bytes per cycle each from the second-level cache, and 48 KB a step.
#include <cstddef>
#include <cstring>

#include "hikonv_linear_tiles.cuh"

namespace hikonv {

constexpr int kTcRows = 128;             // output columns of the layer per tile: rows of the instruction
constexpr int kTcDepth = 128;            // codes of the depth per step: one 128-byte swizzled row
constexpr int kTcMostStages = 12;
constexpr int kFirstEpilogueWarp = 4;
// How operands come to the multiplies: by TMA alone, or by TMA and changed by warps of their own.
enum TcMode { kTma = 0, kTransform = 1 };
constexpr int kEpilogueWarps = 8;
template <int MODE> constexpr int kHelperWarps = MODE == kTma ? 0 : 12;
template <int MODE> constexpr int kTcThreads = (kFirstEpilogueWarp + kEpilogueWarps + kHelperWarps<MODE>) * 32;
template <int MODE> constexpr int kEpilogueBatch = MODE == kTma ? 16 : 8;       // rows of x at a time: what the registers hold
constexpr int kUnitRows = 32;            // operand rows that a helper warp works on at a time
constexpr size_t kTcMostSmem = 226 * 1024;

struct TcParams {
    LinearParams p;
    int nt;                              // rows of x per tile, a multiple of 16
    int acc_cols;                        // tensor-memory columns per accumulator
    int stages, stage_bytes;             // a stage: `atoms` steps of kTcDepth codes, atom_bytes apart
    int atoms, atom_bytes, x_off, raw_off;
    int teams;                           // of helper warps: each takes every so manieth stage
    int a_slots, a_column;               // unpacked weights: slots of `atoms` steps, 32 columns each, of tensor memory from this column on (0: none)
    int tmem_cols;
    int splits, chunks;                  // CTAs that share a tile's depth (log2 in split_shift); steps of the depth in all
    int split_shift;
    int n_blocks, m_tiles, tokens_first;
    uint32_t idesc;
    int units;                           // of helper work per step
    int flip, ones;                      // x has its top bits flipped; so many rows (16) with ones lie behind it
    int flip_w, halves_off;              // w has; a tile of 64s lies there, behind the first stage
    int held;                            // bytes of all stages and slots: the tables of the groups lie behind them
    long long wait_cycles;
};

// The front of a CTA's (dynamic) shared memory; the stages follow on the next multiple of 1024 bytes, then the tables of the groups.
struct TcControl {
    uint64_t full[kTcMostStages], ready[kTcMostStages], empty[kTcMostStages], unpacked_empty[kTcMostStages], acc_full[2], acc_empty[2], drain;
    uint32_t tmem;
    int whole;                           // no wait of this CTA has run out
};

static __device__ unsigned int linear_timeouts;

__device__ __forceinline__ void tc_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a),
                 "l"(b), "r"(idesc), "r"(accumulate)
                 : "memory");
}
// ... with the first operand in tensor memory: a lane per row, four codes per column.
__device__ __forceinline__ void tc_mma_from_tmem(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::i8 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a),
                 "l"(b), "r"(idesc), "r"(accumulate)
                 : "memory");
}
__device__ __forceinline__ void tc_store32(uint32_t taddr, const uint32_t (&v)[32]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,"
                 "%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
                 "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]),
                 "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]),
                 "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31])
                 : "memory");
}
__device__ __forceinline__ void tc_wait_store() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ Tile find_tc_tile(const TcParams &q, const GroupTables &g, int t) { return find_tile(q, g, t, kTcRows); }

__device__ __forceinline__ bool wait_all_of(const TcParams &q, uint32_t bar, uint32_t parity) {
    return __all_sync(0xFFFFFFFFu, mbarrier_wait(bar, parity, q.wait_cycles));
}

// One unit (32 rows, a quarter of the lanes) of dense weights, from the bytes as TMA left them (swizzled, so that a lane can read its row
// without bank conflicts) to tensor memory: 128 codes of a lane's row are 32 columns.  That spares shared memory a write and a read of
// 16 KB per step of 128 codes.  The step takes 300 cycles with 48 rows of x (8192 x 8192 4-bit weights: 13.8 us, 2.6 TB/s), which is what
// three teams of helpers and the issuing warps need; eight helpers and one step per stage took 560 and 16.5 us.
template <int BITS, bool UP>
__device__ __forceinline__ void unpack_unit(uint32_t raw, uint32_t to, int row0) {
    constexpr int PIECES = BITS;                       // of 16 bytes
    const int row = row0 + (threadIdx.x & 31);
    const uint32_t turn = BITS == 4 ? (row >> 1) & 3 : BITS == 2 ? (row >> 2) & 1 : 0;
    uint32_t o[32];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const uint4 v = load_shared16(raw + row * PIECES * 16 + ((i ^ turn) << 4));
        const uint32_t in[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t *at = &o[(i * 4 + j) * (8 / BITS)];
            if constexpr (BITS == 4) {
                unpack4<UP>(in[j], *reinterpret_cast<uint32_t(*)[2]>(at));
            } else if constexpr (BITS == 2) {
                unpack2<UP>(in[j], *reinterpret_cast<uint32_t(*)[4]>(at));
            } else {
                unpack1<UP>(in[j], *reinterpret_cast<uint32_t(*)[4]>(at));
                unpack1<UP>(in[j] >> 16, *reinterpret_cast<uint32_t(*)[4]>(at + 4));
            }
        }
    }
    tc_store32(to + ((uint32_t)row0 << 16), o);
}

// The helper warps: the units of a stage dealt out over a team of them, on from where its stage before left off.  A stage costs a warp
// some 400 cycles beside its units (waits, fences, the report), so there are several teams where a stage has few units.
__device__ __forceinline__ bool help(const TcParams &q, const GroupTables &tables, int t0, int tiles, int step, int c0, int c1, uint32_t stages,
                                     uint32_t tmem, TcControl &ctl) {
    const LinearParams &p = q.p;
    const int lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) - kFirstEpilogueWarp - kEpilogueWarps;
    const int w_units = p.w_bits < 8 || q.flip_w ? kTcRows / kUnitRows : 0;
    Ring ring, unpacked;                               // stages, and slots of unpacked weights
    const int team_warps = kHelperWarps<kTransform> / q.teams, team = warp / team_warps;
    int turn = warp % team_warps, due = team;          // the unit that falls to this warp first, and the stages until this team's next
    for (int t = t0; t < tiles; t += step) {
        for (int c = c0; c < c1; c += q.atoms) {
            if (due-- > 0) {
                ring.next(q.stages);
                unpacked.next(q.a_slots);
                continue;
            }
            due = q.teams - 1;
            const int total = min(q.atoms, c1 - c) * q.units;
            const uint32_t stage = stages + ring.stage * q.stage_bytes, slot = tmem + q.a_column + unpacked.stage * q.atoms * 32;
            if (q.a_column) {
                if (!wait_all_of(q, smem_address(&ctl.unpacked_empty[unpacked.stage]), unpacked.phase ^ 1)) return false;
                tc_fence_after();
            }
            if (!wait_all_of(q, smem_address(&ctl.full[ring.stage]), ring.phase)) return false;
            int i = turn, atom = 0, unit = turn;
            for (; i < total; i += team_warps, unit += team_warps) {
                while (unit >= q.units) unit -= q.units, ++atom;
                const uint32_t at = stage + atom * q.atom_bytes, to = slot + atom * 32;
                const bool of_w = unit < w_units;
                const int row0 = (of_w ? unit : unit - w_units) * kUnitRows;
                if (of_w && p.w_bits < 8) {
                    const uint32_t raw = at + q.raw_off;
                    if (p.w_bits == 4) p.down ? unpack_unit<4, true>(raw, to, row0) : unpack_unit<4, false>(raw, to, row0);
                    else if (p.w_bits == 2) p.down ? unpack_unit<2, true>(raw, to, row0) : unpack_unit<2, false>(raw, to, row0);
                    else p.down ? unpack_unit<1, true>(raw, to, row0) : unpack_unit<1, false>(raw, to, row0);
                } else if (of_w || q.flip) {
                    const int pieces = (of_w ? kTcRows : q.nt) * 8;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int k = row0 * 8 + j * 32 + lane;
                        if (k < pieces) {
                            const uint32_t a = at + (of_w ? 0 : q.x_off) + k * 16;
                            const uint4 v = load_shared16(a);
                            store_shared16(a, v.x ^ 0x80808080u, v.y ^ 0x80808080u, v.z ^ 0x80808080u, v.w ^ 0x80808080u);
                        }
                    }
                }
            }
            turn = i - total;
            if (q.a_column) {
                tc_wait_store();
                tc_fence_before();
            }
            if (q.flip || q.flip_w) proxy_fence();
            __syncwarp();
            if (lane == 0) mbarrier_arrive(smem_address(&ctl.ready[unpacked.stage]));
            ring.next(q.stages);
            unpacked.next(q.a_slots);
        }
    }
    return true;
}

// The epilogue of a warp: the 32 output columns of its quarter of the lanes, every so manieth batch of B rows of x.  Each output costs about
// ten instructions here, and with eight warps they have to overlap: output type and activation are constants, a batch's sums and
// residuals are in flight together, and what belongs to a column is loaded before its sums are there.
template <int WARPS, int B, int OUT, int ACT>
__device__ __forceinline__ bool finish_tiles(const TcParams &q, const GroupTables &tables, int t0, int tiles, int step, uint32_t tmem,
                                             uint32_t acc_full, uint32_t acc_empty) {
    using T = typename OutElem<OUT>::type;
    constexpr bool REAL = OUT >= HIKONV_OUT_F32;
    const LinearParams &p = q.p;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, quad = warp & 3, half = (warp - kFirstEpilogueWarp) >> 2;
    Ring acc;
    for (int t = t0; t < tiles; t += step) {
        const Tile tile = find_tc_tile(q, tables, t);
        const int n = tile.n0 + quad * 32 + lane;
        const bool inside = n < p.N;
        ColumnTerms terms{1.f, 0.f, 0};
        if (inside) terms = column_terms<OUT>(p, tile.e, n);
        // scales of the rows of a batch, a lane each, asked for a batch ahead: a load here and now would take as long as all of a batch
        auto row_scales = [&](int col) {
            const int i = col + (lane & (B - 1));
            return REAL && p.x_scale && i < tile.rows ? load_ordered(p.x_scale + tile.row0 + i) : 1.f;
        };
        float xs_next = row_scales(half * B);
        // ... and the residuals of a batch: loads that depend on nothing, converted when they are used
        T res_next[B];
        auto row_residuals = [&](int col) {
            if (!REAL || !p.residual || !inside || col >= tile.rows) return;
            const T *r = (const T *)p.residual + (long long)(tile.row0 + col) * p.res_row + n;
            if (tile.rows - col >= B) {
#pragma unroll
                for (int i = 0; i < B; ++i) res_next[i] = load_ordered(r + i * p.res_row);
            } else {
#pragma unroll
                for (int i = 0; i < B; ++i)
                    if (col + i < tile.rows) res_next[i] = load_ordered(r + i * p.res_row);
            }
        };
        row_residuals(half * B);
        if (!wait_all_of(q, acc_full + 8 * acc.stage, acc.phase)) return false;
        tc_fence_after();
        const uint32_t d = tmem + acc.stage * q.acc_cols + ((uint32_t)(quad * 32) << 16);
        int32_t correction = 0;
        if (q.ones) {
            correction = (int32_t)tc_load1(d + q.nt) * 128;
            tc_wait_load();
        }
        for (int col = half * B; col < tile.rows; col += WARPS / 4 * B) {
            uint32_t v[B];
            float scale[B];
            T res[B];
            tc_load_columns(d + col, v);
            const long long m = tile.row0 + col;
            const int left = tile.rows - col;
            if (REAL) {
                const float xs = xs_next;
                xs_next = row_scales(col + WARPS / 4 * B);
                if (p.residual) {
#pragma unroll
                    for (int i = 0; i < B; ++i) res[i] = res_next[i];
                    row_residuals(col + WARPS / 4 * B);
                }
#pragma unroll
                for (int i = 0; i < B; ++i) scale[i] = __shfl_sync(0xFFFFFFFFu, xs, i);
            }
            tc_wait_load();
            if (inside) {
                T *o = (T *)p.out + m * p.out_row + n;
                auto one = [&](int i) {
                    float r = 0.f;
                    if constexpr (REAL)
                        if (p.residual) r = to_float(res[i]);
                    *o = finish<OUT, ACT>(p, ((int32_t)v[i] + correction) >> p.down, REAL ? scale[i] : 1.f, terms, r);
                    o += p.out_row;
                };
                if (left >= B) {
#pragma unroll
                    for (int i = 0; i < B; ++i) one(i);
                } else {
#pragma unroll
                    for (int i = 0; i < B; ++i)
                        if (i < left) one(i);
                }
            }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbarrier_arrive(acc_empty + 8 * acc.stage);
        acc.next(2);
    }
    return true;
}

// With a shared depth: this CTA's part of the sums goes to shared memory, [row of x][output column], over the stages (all loads have been
// multiplied when the sums are there); after the cluster's barrier the CTA takes the sums of all parts through the epilogue for its share
// of the output columns, four columns of two rows per thread at a time.  What else that needs is loaded before the barrier: a fetch from
// another SM takes several hundred cycles, as one from the second-level cache does.
template <int WARPS, int OUT, int ACT>
__device__ __forceinline__ bool finish_shared_tile(const TcParams &q, const GroupTables &tables, int t, int tiles, int rank, uint32_t tmem,
                                                   uint32_t part, TcControl &ctl) {
    using T = typename OutElem<OUT>::type;
    constexpr bool REAL = OUT >= HIKONV_OUT_F32;
    constexpr int BATCH = 2;
    const LinearParams &p = q.p;
    const int tid = threadIdx.x - kFirstEpilogueWarp * 32, lane = tid & 31, quad = (tid >> 5) & 3, half = tid >> 7;
    const int lanes = (kTcRows / 4) >> q.split_shift;      // threads that share a row
    const int own = (rank * lanes + (tid & (lanes - 1))) * 4, step = WARPS * 32 / lanes;
    const int first = tid / lanes;
    Tile tile{0, 0, 0, 0};
    if (t < tiles) tile = find_tc_tile(q, tables, t);
    const int n = tile.n0 + own, inside = max(0, min(4, p.N - n));       // columns that there are
    ColumnTerms terms[4];
    float xs[BATCH], res[BATCH][4];
    auto fetch = [&](int i0) {
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const int i = i0 + b * step;
            xs[b] = 1.f;
#pragma unroll
            for (int k = 0; k < 4; ++k) res[b][k] = 0.f;
            if (REAL && i < tile.rows) {
                if (p.x_scale) xs[b] = load_ordered(p.x_scale + tile.row0 + i);
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (k < inside) res[b][k] = residual_at<T>(p, tile.row0 + i, n + k);
            }
        }
    };
#pragma unroll
    for (int k = 0; k < 4; ++k) terms[k] = t < tiles && k < inside ? column_terms<OUT>(p, tile.e, n + k) : ColumnTerms{1.f, 0.f, 0};
    fetch(first);
    bool fine = true;
    if (t < tiles) {
        fine = wait_all_of(q, smem_address(&ctl.acc_full[0]), 0);
        if (fine) {
            tc_fence_after();
            const uint32_t d = tmem + ((uint32_t)(quad * 32) << 16);
            uint32_t correction = 0;
            if (q.ones) {
                correction = tc_load1(d + q.nt) * 128u;
                tc_wait_load();
            }
            for (int col = half * 16; col < tile.rows; col += WARPS * 4) {
                uint32_t v[16];
                tc_load16(d + col, v);
                tc_wait_load();
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    asm volatile("st.shared.u32 [%0], %1;" ::"r"(part + ((col + i) * kTcRows + quad * 32 + lane) * 4), "r"(v[i] + correction) : "memory");
            }
            tc_fence_before();
        }
    }
    if (!fine) ctl.whole = 0;
    uint32_t from[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) from[r] = remote_address(part + own * 4, r < q.splits ? r : 0);
    const uint32_t flag_at = remote_address(smem_address(&ctl.whole), lane & (q.splits - 1));
    cluster_sync_all();
    const int flag = load_cluster_s32(flag_at);
    for (int i0 = first; i0 - first < tile.rows; i0 += BATCH * step) {
        if (i0 != first) fetch(i0);
        int32_t sum[BATCH][4] = {};
#pragma unroll
        for (int r0 = 0; r0 < 8; r0 += 4) {
            if (r0 >= q.splits) break;
            int4 v[4][BATCH];
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int b = 0; b < BATCH; ++b)
                    v[r][b] = r0 + r < q.splits && i0 + b * step < tile.rows ? load_cluster_int4(from[r0 + r] + (i0 + b * step) * kTcRows * 4)
                                                                             : make_int4(0, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int b = 0; b < BATCH; ++b) sum[b][0] += v[r][b].x, sum[b][1] += v[r][b].y, sum[b][2] += v[r][b].z, sum[b][3] += v[r][b].w;
        }
        if (i0 == first && !__all_sync(0xFFFFFFFFu, flag)) break;
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const int i = i0 + b * step;
            if (i < tile.rows) {
                T *o = (T *)p.out + (tile.row0 + i) * p.out_row + n;
                T y[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) y[k] = finish<OUT, ACT>(p, sum[b][k] >> p.down, xs[b], terms[k], res[b][k]);
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
    }
    cluster_sync_all();                                // the others may still read this CTA's part
    return fine;
}

template <int MODE>
__global__ void __launch_bounds__(kTcThreads<MODE>, 1)
    linear_tc_kernel(const __grid_constant__ TcParams q, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w) {
    extern __shared__ __align__(16) uint8_t dynamic[];
    TcControl &ctl = *reinterpret_cast<TcControl *>(dynamic);
    const uint32_t control = smem_address(dynamic);
    auto barrier = [&](size_t offset, int i) { return control + (uint32_t)offset + 8u * (uint32_t)i; };
#define HIKONV_BAR(name, i) barrier(offsetof(TcControl, name), i)
    constexpr int EPI = kEpilogueWarps, FIRST_HELPER = kFirstEpilogueWarp + EPI;
    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(0xFFFFFFFFu, tid >> 5, 0);       // the same in all lanes, which the compiler does not see from tid
    const LinearParams &p = q.p;
    const uint32_t stages = (smem_address(dynamic) + (uint32_t)sizeof(TcControl) + 1023u) & ~1023u;
    uint8_t *behind = dynamic + (stages - smem_address(dynamic)) + q.held;
    int2 *group_row = reinterpret_cast<int2 *>(behind);
    int *group_tiles = reinterpret_cast<int *>(group_row + p.E);
    const GroupTables tables{group_row, group_tiles};

    if (warp == 0) {
        if (lane < q.stages) {
            mbarrier_init(HIKONV_BAR(full, lane), 1);
            mbarrier_init(HIKONV_BAR(ready, lane), MODE == kTma ? 1 : kHelperWarps<MODE> / q.teams);
            mbarrier_init(HIKONV_BAR(empty, lane), 1);
            mbarrier_init(HIKONV_BAR(unpacked_empty, lane), 1);
        }
        if (lane < 2) {
            mbarrier_init(HIKONV_BAR(acc_full, lane), 1);
            mbarrier_init(HIKONV_BAR(acc_empty, lane), EPI);
        }
        if (lane == 2) {
            mbarrier_init(HIKONV_BAR(drain, 0), 1);
            ctl.whole = 1;
        }
        mbarrier_init_fence();
        if (lane == 3) {
            asm volatile("prefetch.tensormap [%0];" ::"l"(&map_x) : "memory");
            asm volatile("prefetch.tensormap [%0];" ::"l"(&map_w) : "memory");
        }
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_address(&ctl.tmem)), "r"(q.tmem_cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    if (MODE != kTma && q.ones) {
        // sixteen rows behind the rows of x, the first of them ones; nothing writes there again
        for (int i = tid; i < q.stages * q.atoms * 128; i += blockDim.x) {
            const uint32_t v = (i & 127) < 8 ? 0x01010101u : 0u;
            store_shared16(stages + (i >> 7) * q.atom_bytes + q.x_off + q.nt * 128 + (i & 127) * 16, v, v, v, v);
        }
        proxy_fence();
    }
    if (MODE != kTma && q.flip_w) {
        for (int i = tid; i < kTcRows * kTcDepth / 16; i += blockDim.x)
            store_shared16(stages + q.halves_off + i * 16, 0x40404040u, 0x40404040u, 0x40404040u, 0x40404040u);
        proxy_fence();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = ctl.tmem;
    // Not before this CTA has its tensor memory: a CTA of the kernel behind that came to this SM first could take it, and wait for this
    // one to end while this one waits for the memory.
    grid_dependency_release();

    // Each role waits for the kernel before where it first touches global memory, or waits, with a bound, for what others bring from there.
    int tiles = q.m_tiles * q.n_blocks;
    if (p.offsets) {
        grid_dependency_wait();
        tiles = build_group_tables(q, group_row, group_tiles);
    }
    const int rank = blockIdx.x & (q.splits - 1), t0 = blockIdx.x >> q.split_shift, step = gridDim.x >> q.split_shift;
    const int c0 = (q.chunks * rank) >> q.split_shift, c1 = (q.chunks * (rank + 1)) >> q.split_shift;

    auto wait = [&](uint32_t bar, uint32_t parity) { return wait_all_of(q, bar, parity); };
    bool fine = true;
    if (warp == 0) {
        Ring ring;
        const int depth_bytes = kTcDepth * p.w_bits / 8;
        const uint32_t bytes = (uint32_t)(q.nt * kTcDepth + kTcRows * depth_bytes);
        const uint32_t w_off = p.w_bits == 8 ? 0u : (uint32_t)q.raw_off;
        int loads = 0;
        for (int t = t0; fine && t < tiles; t += step) {
            const Tile tile = find_tc_tile(q, tables, t);
            const int w_row0 = tile.e * p.N + tile.n0;
            if (loads == 0) grid_dependency_wait();
            for (int c = c0; c < c1; c += q.atoms) {
                fine = wait(HIKONV_BAR(empty, ring.stage), ring.phase ^ 1);
                if (!fine) break;
                const uint32_t bar = HIKONV_BAR(full, ring.stage);
                const int some = min(q.atoms, c1 - c);
                if (elect_one()) {
                    uint32_t at = stages + ring.stage * q.stage_bytes;
                    mbarrier_arrive_expect(bar, bytes * some);
                    for (int i = 0; i < some; ++i, at += q.atom_bytes) {
                        tma_load_2d(at + w_off, &map_w, (c + i) * depth_bytes, w_row0, bar);
                        tma_load_2d(at + q.x_off, &map_x, (c + i) * kTcDepth, tile.row0, bar);
                    }
                }
                ++loads;
                ring.next(q.stages);
            }
        }
        // what is in flight has to land before the memory goes: the last load of every stage
        for (int i = 0; i < q.stages && i < loads; ++i) {
            ring.stage = ring.stage ? ring.stage - 1 : q.stages - 1;
            if (ring.stage == q.stages - 1) ring.phase ^= 1;
            fine &= wait(HIKONV_BAR(full, ring.stage), ring.phase);
        }
    } else if (warp == 1) {
        grid_dependency_wait();
        Ring ring, unpacked, acc;
        const uint64_t halves = smem_descriptor(stages + q.halves_off);
        const uint64_t a0 = smem_descriptor(stages), b0 = smem_descriptor(stages + q.x_off);
        const uint32_t stage_units = (uint32_t)q.stage_bytes >> 4, atom_units = (uint32_t)q.atom_bytes >> 4;
        for (int t = t0; fine && t < tiles; t += step) {
            const Tile tile = find_tc_tile(q, tables, t);
            const uint32_t cols = q.ones ? (uint32_t)(q.nt + q.ones) : (uint32_t)((tile.rows + 15) & ~15);
            const uint32_t idesc = q.idesc | ((cols >> 3) << 17);
            const uint32_t d = tmem + acc.stage * q.acc_cols;
            fine = wait(HIKONV_BAR(acc_empty, acc.stage), acc.phase ^ 1);
            if (!fine) break;
            uint32_t accumulate = 0;
            for (int c = c0; c < c1; c += q.atoms) {
                // where helpers have a hand in the operands, their waits have seen the copies land
                fine = MODE == kTma ? wait(HIKONV_BAR(full, ring.stage), ring.phase) : wait(HIKONV_BAR(ready, unpacked.stage), unpacked.phase);
                if (!fine) break;
                tc_fence_after();
                const int some = min(q.atoms, c1 - c);
                if (elect_one()) {
                    uint64_t b = b0 + ring.stage * stage_units;
                    if (MODE == kTransform && q.a_column) {
                        uint32_t a = tmem + q.a_column + unpacked.stage * q.atoms * 32;
                        for (int i = 0; i < some; ++i, a += 32, b += atom_units) {
#pragma unroll
                            for (int k = 0; k < kTcDepth / 32; ++k) {
                                tc_mma_from_tmem(d, a + k * 8, b + k * 2, idesc, accumulate);
                                accumulate = 1;
                            }
                        }
                    } else {
                        uint64_t a = a0 + ring.stage * stage_units;
                        for (int i = 0; i < some; ++i, a += atom_units, b += atom_units) {
#pragma unroll
                            for (int k = 0; k < kTcDepth / 32; ++k) {
                                tc_mma(d, a + k * 2, b + k * 2, idesc, accumulate);
                                accumulate = 1;
                                if (MODE != kTma && q.flip_w) {
                                    tc_mma(d, halves, b + k * 2, idesc, 1);
                                    tc_mma(d, halves, b + k * 2, idesc, 1);
                                }
                            }
                        }
                    }
                    tc_commit(HIKONV_BAR(empty, ring.stage));
                    if (MODE == kTransform && q.a_column) tc_commit(HIKONV_BAR(unpacked_empty, unpacked.stage));
                }
                accumulate = 1;
                ring.next(q.stages);
                unpacked.next(q.a_slots);
            }
            if (!fine) break;
            if (elect_one()) tc_commit(HIKONV_BAR(acc_full, acc.stage));
            acc.next(2);
        }
        if (!fine) {                                   // multiplies in flight read shared memory and write tensor memory
            if (elect_one()) tc_commit(HIKONV_BAR(drain, 0));
            wait(HIKONV_BAR(drain, 0), 0);
        }
    } else if (MODE != kTma && warp >= FIRST_HELPER) {
        grid_dependency_wait();
        if constexpr (MODE != kTma) fine = help(q, tables, t0, tiles, step, c0, c1, stages, tmem, ctl);
    } else if (warp >= kFirstEpilogueWarp && warp < FIRST_HELPER) {
        grid_dependency_wait();
        with_epilogue(p, [&](auto kind, auto act) {
            constexpr int OUT = decltype(kind)::value, ACT = decltype(act)::value;
            if (q.splits > 1) fine = finish_shared_tile<EPI, OUT, ACT>(q, tables, t0, tiles, rank, tmem, stages, ctl);
            else fine = finish_tiles<EPI, kEpilogueBatch<MODE>, OUT, ACT>(q, tables, t0, tiles, step, tmem, HIKONV_BAR(acc_full, 0), HIKONV_BAR(acc_empty, 0));
        });
    }
    if (!fine && lane == 0) atomicAdd(&linear_timeouts, 1u);
    __syncwarp();
    if (q.splits > 1 && (warp < kFirstEpilogueWarp || warp >= FIRST_HELPER)) {
        if (!fine) ctl.whole = 0;
        cluster_sync_all();
        cluster_sync_all();                            // the others may still read this CTA's part
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(q.tmem_cols));
}

#undef HIKONV_BAR

// Rows of bytes from any address and pitch to rows on 16-byte boundaries, two matrices in one launch; a thread per 16 bytes.  What lies
// behind a row in its last piece is anything.
struct AlignRows {
    const uint8_t *src;
    uint8_t *dst;
    long long src_row;
    int bytes, pieces;                   // of a row
    long long total;                     // pieces of the matrix
};
__global__ void __launch_bounds__(256) align_rows_kernel(const AlignRows a, const AlignRows b, int a_blocks) {
    grid_dependency_release();
    grid_dependency_wait();
    const AlignRows &m = (int)blockIdx.x < a_blocks ? a : b;
    const long long i = ((long long)blockIdx.x - ((int)blockIdx.x < a_blocks ? 0 : a_blocks)) * 256 + threadIdx.x;
    if (i >= m.total) return;
    const long long row = m.total <= 0xFFFFFFFFll ? (long long)((uint32_t)i / (uint32_t)m.pieces) : i / m.pieces;
    const int at = (int)(i - row * m.pieces) * 16;
    uint32_t v[4];
    load_bytes<4>(m.src + row * m.src_row + at, min(16, m.bytes - at), v);
    *reinterpret_cast<uint4 *>(m.dst + i * 16) = make_uint4(v[0], v[1], v[2], v[3]);
}

__global__ void linear_wait_check_kernel(long long cycles) {
    __shared__ uint64_t bar;
    mbarrier_init(smem_address(&bar), 1);
    mbarrier_init_fence();
    if (!mbarrier_wait(smem_address(&bar), 0, cycles)) atomicAdd(&linear_timeouts, 1u);
}

// ---- host

int sm_count_here() {
    static thread_local int known_dev = -1, sms = 148;
    int dev = 0;
    if (cudaGetDevice(&dev) == cudaSuccess && dev != known_dev) {
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
        known_dev = dev;
    }
    return sms;
}

// Whether the layer has few enough tiles and rows of weights for 32-bit counts.
static bool fits(const LinearParams &p) {
    if ((long long)p.E * p.N > 0x7FFFFFFFll || p.M > (1 << 30)) return false;
    return ((long long)p.M / 16 + (p.E < p.M ? p.E : p.M) + 1) * ceil_div(p.N, kTcRows) < 0x3FFFFFFFll;
}
// Whether TMA reads the rows of x, and of w, as they are: all on 16-byte boundaries.
static bool x_aligned(const LinearParams &p) { return (uintptr_t)p.x % 16 == 0 && (p.M == 1 || p.x_row % 16 == 0); }
static bool w_aligned(const LinearParams &p) { return (uintptr_t)p.w % 16 == 0 && p.w_row % 16 == 0; }

size_t linear_tc_workspace(const LinearParams &p) {
    return (x_aligned(p) ? 0 : (size_t)p.M * align_up(p.K, 16)) + (w_aligned(p) ? 0 : (size_t)p.E * p.N * align_up(p.w_row, 16));
}

// Copies what is not aligned into the workspace and points the layer there.
static int align_operands(LinearParams *p, void *workspace, cudaStream_t st) {
    uint8_t *to = (uint8_t *)workspace;
    AlignRows m[2] = {};
    int n = 0;
    auto add = [&](const uint8_t **base, long long *row, long long rows, long long bytes) {
        AlignRows &a = m[n++];
        a.src = *base; a.src_row = *row; a.dst = to;
        a.bytes = (int)bytes; a.pieces = (int)((bytes + 15) / 16); a.total = rows * a.pieces;
        *base = to;
        *row = (long long)a.pieces * 16;
        to += a.total * 16;
    };
    const bool x_stays = x_aligned(*p), w_stays = w_aligned(*p);
    if (!x_stays) add(&p->x, &p->x_row, p->M, p->K);
    if (!w_stays) add(&p->w, &p->w_row, (long long)p->E * p->N, p->w_row);
    const long long a_blocks = (m[0].total + 255) / 256, b_blocks = (m[1].total + 255) / 256;
    if (a_blocks + b_blocks > 0x7FFFFFFFll) return HIKONV_ERR_UNSUPPORTED;
    return launch_dependent(align_rows_kernel, dim3((unsigned)(a_blocks + b_blocks)), dim3(256), 0, st, m[0], m[1], (int)a_blocks);
}

// Steps per stage where weights are unpacked: as many as leave three slots of tensor memory and three stages.  The loops around a stage
// cost the issuing warps and the helpers as much as a step of it.
static int unpacked_atoms(int nt, int ones, int w_bits) {
    const int acc = (int)align_up(nt + ones, 32), bytes = (nt + ones) * kTcDepth + kTcRows * kTcDepth * w_bits / 8;
    for (int atoms = 4; atoms > 1; atoms /= 2)
        if ((512 - 2 * acc) / (32 * atoms) >= 3 && 3 * atoms * (int)align_up(bytes, 1024) <= (int)kTcMostSmem - 16 * 1024) return atoms;
    return 1;
}
// Steps of a depth, which may be anything up to 2^31 - 1.
static int depth_steps(int K) { return (K - 1) / kTcDepth + 1; }
// Rows of x per tile and CTAs per tile that a model of the time, in cycles, likes best.  A step of 128 codes costs the longest of its
// multiplies (2 per row), its way from the second-level cache (70 bytes per cycle and SM) and the helpers' work on it; a tile alone on its
// SM costs 3000 for the set-up and the end of its epilogue; one with a shared depth two barriers of the cluster, which are dearer the
// larger it is, and the fetches of all parts.
// It ranks shapes of one layer and leaves out the launch and the way from memory: 8-bit 4096 x 4096 with 64 and 256 rows and 8192 x 8192 with
// 48 are 11.8, 16.3 and 18.7 thousand cycles of it and take 7.0, 8.6 and 15.5 us with weights from memory.  2048^3 is 19.4 thousand with 240
// rows per tile (144 tiles, one wave), 20.2 with 256, and takes 10.2 us.
static void choose_tile(const LinearParams &p, int mode, bool ones, int sms, int *nt_out, int *splits_out) {
    const int n_blocks = ceil_div(p.N, kTcRows), chunks = depth_steps(p.K);
    // unpacked weights take tensor memory from the accumulators
    const int most = mode == kTransform && p.w_bits < 8 ? 192 : ones ? 240 : 256;
    double best = 1e300;
    for (int nt = 16; nt <= most; nt += 16) {
        // groups: on average half a tile of each is left empty
        const int filled = p.E < p.M ? p.E : p.M;
        const double tiles = (p.offsets ? (double)p.M / nt + 0.5 * filled : (double)ceil_div(p.M, nt)) * n_blocks;
        const double bytes = kTcRows * kTcDepth * p.w_bits / 8.0 + nt * (double)kTcDepth;
        double step = 2.0 * nt > bytes / 70.0 ? 2.0 * nt : bytes / 70.0;
        const int atoms = mode == kTransform && p.w_bits < 8 ? unpacked_atoms(nt, ones ? 16 : 0, p.w_bits) : 0;
        const double help = mode != kTransform ? 200.0 : atoms == 4 ? 300.0 : atoms == 2 ? 400.0 : atoms == 1 ? 460.0 : 370.0;
        if (step < help) step = help;
        for (int splits = 1; splits <= 8 && splits <= chunks; splits *= 2) {
            // clusters of four and more do not fill every SM: their CTAs share one part of the GPU
            if (splits > 1 && (tiles * splits > sms - 20 || nt > 128)) break;
            const double waves = splits > 1 ? 1.0 : p.offsets ? (tiles > sms ? tiles / sms + 0.3 : 1.0) : (double)((long long)(tiles + sms - 1) / sms);
            const double time = waves * ceil_div(chunks, splits) * step + 3000.0 +
                                (splits > 1 ? 2500.0 + 500.0 * splits + 62.0 * nt / splits + 8.0 * nt : 800.0 + 20.0 * nt);
            if (time < best) {
                best = time;
                *nt_out = nt;
                *splits_out = splits;
            }
        }
        if (nt >= p.M) break;
    }
}

int launch_linear_tc(LinearParams p, void *workspace, size_t workspace_bytes, cudaStream_t st) {
    if (!fits(p)) return HIKONV_ERR_UNSUPPORTED;
    if (const size_t need = linear_tc_workspace(p)) {
        if (!workspace || (uintptr_t)workspace % 16 || workspace_bytes < need) return HIKONV_ERR_WORKSPACE;
        const int rc = align_operands(&p, workspace, st);
        if (rc != HIKONV_OK) return rc;
    }
    TcParams q;
    memset(&q, 0, sizeof(q));
    q.p = p;
    const int sms = sm_count_here();
    const bool as_unsigned = (p.x_u8 || p.w_u8) && !p.x_signed && !p.w_signed;
    q.flip = p.x_u8 && !as_unsigned;
    q.ones = q.flip ? 16 : 0;
    q.flip_w = p.w_u8 && !as_unsigned;
    const int mode = p.w_bits < 8 || q.flip || q.flip_w ? kTransform : kTma;
    choose_tile(p, mode, q.flip, sms, &q.nt, &q.splits);
    // units that unpack weights fall to the warps of their lanes: their number per step is a multiple of four
    q.units = (p.w_bits < 8 || q.flip_w ? kTcRows / kUnitRows : 0) + (q.flip ? ceil_div(q.nt, kUnitRows) : 0);
    if (mode == kTransform && p.w_bits < 8) q.units = (int)align_up(q.units, 4);
    q.chunks = depth_steps(p.K);
    q.n_blocks = ceil_div(p.N, kTcRows);
    q.m_tiles = ceil_div(p.M, q.nt);
    q.tokens_first = p.offsets || (long long)p.M * p.K <= (long long)p.N * p.w_row;
    q.acc_cols = (int)align_up(q.nt + q.ones, 32);
    // Dense weights arrive as they are stored and are unpacked into tensor memory.
    const bool apart = mode == kTransform && p.w_bits < 8;
    const int operand_bytes = kTcRows * kTcDepth;
    q.x_off = apart ? 0 : operand_bytes;
    q.raw_off = q.x_off + (q.nt + q.ones) * kTcDepth;
    q.atom_bytes = (int)align_up(q.raw_off + (apart ? operand_bytes * p.w_bits / 8 : 0), 1024);
    while ((1 << q.split_shift) < q.splits) ++q.split_shift;
    // a step of a narrow tile is shorter than the loop around it: several to a stage
    q.atoms = apart ? unpacked_atoms(q.nt, q.ones, p.w_bits) : q.nt <= 32 ? 4 : q.nt <= 96 ? 2 : 1;
    const size_t tables = p.offsets ? (size_t)p.E * 12 : 0, all = kTcMostSmem - 2048 - tables - (q.flip_w ? operand_bytes : 0);
    while (q.atoms > 1 && all / (q.atoms * q.atom_bytes) < (apart ? 3u : 4u)) q.atoms /= 2;
    q.stage_bytes = q.atoms * q.atom_bytes;
    q.stages = (int)(all / q.stage_bytes);
    if (q.stages > kTcMostStages) q.stages = kTcMostStages;
    const int own = ceil_div(ceil_div(q.chunks, q.splits), q.atoms);                  // stages that a CTA fills for a tile
    const int parts = q.splits > 1 ? ceil_div(q.nt * kTcRows * 4, q.stage_bytes) : 1; // the sums that are exchanged lie over the stages
    if (q.stages < parts) return HIKONV_ERR_UNSUPPORTED;
    const long long tiles = (p.offsets ? p.M / q.nt + (p.E < p.M ? p.E : p.M) : (long long)q.m_tiles) * q.n_blocks;
    if (tiles * q.splits <= sms && q.stages > own) q.stages = own > parts ? own : parts;
    q.a_slots = q.stages;
    if (apart) {
        q.a_column = 2 * q.acc_cols;
        q.a_slots = (512 - q.a_column) / (32 * q.atoms);
        if (q.a_slots > 6) q.a_slots = 6;
        if (q.a_slots > q.stages) q.a_slots = q.stages;      // as many of their barriers are there as of the stages'
        if (q.a_slots < 1) return HIKONV_ERR_UNSUPPORTED;
    }
    q.tmem_cols = 32;
    while (q.tmem_cols < 2 * q.acc_cols + (apart ? q.a_slots * 32 * q.atoms : 0)) q.tmem_cols *= 2;
    q.halves_off = q.stages * q.stage_bytes;
    q.held = q.halves_off + (q.flip_w ? operand_bytes : 0);
    // Teams of at least four warps, since a warp reaches a quarter of the lanes of tensor memory only.  A team that waits for the parity of
    // a barrier must know that the use before the last is over, or it takes an older use for its own.  Of slot s for stage n: the team saw
    // the multiplies of stage n - 3 - a_slots end, which are not before those of n - 2 a_slots if there are three slots.  Of stage n's
    // copies, after that: all multiplies up to stage n - a_slots are over, so the copies of n - stages have landed, since there are no
    // fewer stages than slots.
    q.teams = 1;
    if (apart && q.units == 4 && q.stages >= 3 && q.a_slots >= 3) q.teams = 3;
    // accumulators of signed operands: format 2 (int32), types 1 (signed) or 0 (unsigned) of both, 128 rows; the columns follow per tile
    q.idesc = (2u << 4) | ((as_unsigned ? 0u : 1u) << 7) | ((as_unsigned ? 0u : 1u) << 10) | ((uint32_t)(kTcRows >> 4) << 24);
    q.wait_cycles = kWaitCycles;
    const size_t smem = (size_t)q.held + 2048 + tables;

    CUtensorMap map_x, map_w;
    if (!encode_map(&map_x, p.x, (uint64_t)p.K, (uint64_t)p.M, p.M > 1 ? (uint64_t)p.x_row : (uint64_t)align_up(p.K, 16), kTcDepth, (uint32_t)q.nt) ||
        !encode_map(&map_w, p.w, (uint64_t)p.K * p.w_bits / 8, (uint64_t)p.E * p.N, (uint64_t)p.w_row, (uint32_t)(kTcDepth * p.w_bits / 8), kTcRows))
        return HIKONV_ERR_CUDA;
    const unsigned grid = (unsigned)(q.splits > 1 ? tiles * q.splits : tiles < sms ? tiles : sms);
    auto launch = [&](auto kernel, int threads) {
        return with_dynamic_smem((const void *)kernel, smem > 49 * 1024 ? smem : 49 * 1024, [&] {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(grid);
            cfg.blockDim = dim3((unsigned)threads);
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
            return cudaLaunchKernelEx(&cfg, kernel, q, map_x, map_w) == cudaSuccess ? HIKONV_OK : HIKONV_ERR_CUDA;
        });
    };
    return mode == kTma ? launch(linear_tc_kernel<kTma>, kTcThreads<kTma>) : launch(linear_tc_kernel<kTransform>, kTcThreads<kTransform>);
}

int read_linear_timeouts(unsigned int *h_count) {
    return cudaMemcpyFromSymbol(h_count, linear_timeouts, sizeof(*h_count)) == cudaSuccess ? HIKONV_OK : HIKONV_ERR_CUDA;
}
int launch_linear_wait_check(long long cycles, cudaStream_t st) { return launch_plain(linear_wait_check_kernel, dim3(1), dim3(1), 0, st, cycles); }

}  // namespace hikonv
