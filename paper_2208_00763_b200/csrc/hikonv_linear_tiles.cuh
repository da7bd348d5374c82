// What the tiled kernels of the linear layers share: tcgen05 and TMA instructions, rings of stages, tiles of groups of rows, tensor maps.
#pragma once

#include <cuda.h>

#include "hikonv_cluster.cuh"
#include "hikonv_linear_util.cuh"

namespace hikonv {

// ---- tensor cores and tensor memory

__device__ __forceinline__ uint64_t smem_descriptor(uint32_t address) {
    // rows of 128 bytes with the 128-byte swizzle, eight of them 1024 bytes after one another
    return (uint64_t)((address & 0x3FFFFu) >> 4) | ((uint64_t)1 << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_load16(uint32_t taddr, uint32_t (&v)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
                   "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
                 : "r"(taddr));
}
__device__ __forceinline__ void tc_load_columns(uint32_t taddr, uint32_t (&v)[16]) { tc_load16(taddr, v); }
__device__ __forceinline__ void tc_load_columns(uint32_t taddr, uint32_t (&v)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7])
                 : "r"(taddr));
}
__device__ __forceinline__ uint32_t tc_load1(uint32_t taddr) {
    uint32_t v;
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(v) : "r"(taddr));
    return v;
}
__device__ __forceinline__ void tc_wait_load() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map),
                 "r"(x), "r"(y), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void mbarrier_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void cluster_sync_all() {
    cluster_arrive();
    cluster_wait();
}
__device__ __forceinline__ uint32_t remote_address(uint32_t smem_addr, uint32_t rank) {
    uint32_t remote;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(smem_addr), "r"(rank));
    return remote;
}
// Without a clobber of memory, so that several are in flight; volatile, so that they stay between the two cluster barriers.
__device__ __forceinline__ int32_t load_cluster_s32(uint32_t remote) {
    int32_t v;
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(remote));
    return v;
}
__device__ __forceinline__ int4 load_cluster_int4(uint32_t remote) {
    int4 v;
    asm volatile("ld.shared::cluster.v4.s32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(remote));
    return v;
}
__device__ __forceinline__ uint4 load_shared16(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void store_shared16(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}

// One lane of a converged warp.  The warps that issue TMA copies and multiplies run their loops as a whole and issue under this: with one
// thread in the loop, its values are not known to be uniform and a step of 128 codes took 590 cycles instead of 130.
__device__ __forceinline__ bool elect_one() {
    uint32_t yes;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
    return yes != 0;
}

// A ring of stages: which one is next and in which of its phases it is.
struct Ring {
    int stage = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void next(int stages) {
        if (++stage == stages) {
            stage = 0;
            phase ^= 1;
        }
    }
};

struct Tile {
    int e, row0, rows, n0;
};

// Tables of the groups in shared memory: row ranges, and the number of tiles up to the end of each.
struct GroupTables {
    const int2 *rows;
    const int *tile_end;
};

// Tile t of a layer: `width` output columns by q.nt rows of x.  Q: p (LinearParams), nt, m_tiles, n_blocks, tokens_first.
template <typename Q>
__device__ __forceinline__ Tile find_tile(const Q &q, const GroupTables &g, int t, int width) {
    Tile r;
    int local = t, m_tiles = q.m_tiles, first = 0, end = q.p.M;
    r.e = 0;
    if (q.p.offsets) {
        int lo = 0, hi = q.p.E - 1;                    // the first group whose tiles end behind t
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (g.tile_end[mid] > t) hi = mid;
            else lo = mid + 1;
        }
        r.e = lo;
        if (lo > 0) local -= g.tile_end[lo - 1];
        first = g.rows[lo].x;
        end = g.rows[lo].y;
        m_tiles = (end - first + q.nt - 1) / q.nt;
    }
    const int i = q.tokens_first ? local % m_tiles : local / q.n_blocks;
    const int j = q.tokens_first ? local / m_tiles : local % q.n_blocks;
    r.row0 = first + i * q.nt;
    r.rows = min(q.nt, end - r.row0);
    r.n0 = j * width;
    return r;
}

// Row ranges that overlap, which only offsets that decrease somewhere make, to ranges that do not, by one warp.  The grid, the stages
// and the shared depth (one tile per cluster) count on no more tiles than disjoint ranges of M rows have.  From the front, the rows go
// to the group that holds the next one and reaches furthest, up to its end: each group has one stretch at most, a row that any group
// claims has one group, and a row that just one claims has that one.
__device__ __forceinline__ void separate_groups(int2 *rows, int E) {
    const int lane = threadIdx.x & 31;
    for (int at = 0;;) {
        int reach = at, best = 0x7FFFFFFF, next = 0x7FFFFFFF;
        for (int e = lane; e < E; e += 32) {
            const int2 r = rows[e];
            if (r.x == r.y || r.y <= at) continue;
            if (r.x > at) {
                next = min(next, r.x);
            } else if (r.y > reach) {
                reach = r.y;
                best = e;
            }
        }
        __syncwarp();
        const int to = __reduce_max_sync(0xFFFFFFFFu, reach);
        if (to > at) {
            best = __reduce_min_sync(0xFFFFFFFFu, reach == to ? best : 0x7FFFFFFF);
            if (lane == 0) rows[best].x = ~at;         // taken: below zero until all are
            __syncwarp();
            at = to;
        } else {
            at = __reduce_min_sync(0xFFFFFFFFu, next);
            if (at == 0x7FFFFFFF) break;
        }
    }
    for (int e = lane; e < E; e += 32) {
        int2 r = rows[e];
        if (r.x < 0) r.x = ~r.x;
        else r.y = r.x;
        rows[e] = r;
    }
    __syncwarp();
}

// The tables of the groups, by a whole CTA: row ranges, tiles up to the end of each group.  Returns the tiles in all.
template <typename Q>
__device__ __forceinline__ int build_group_tables(const Q &q, int2 *group_row, int *group_tiles) {
    const LinearParams &p = q.p;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int decreasing = 0;
    for (int e = tid; e < p.E; e += blockDim.x) {
        const int2 r = group_rows(p, e);
        group_row[e] = r;
        decreasing |= load_ordered(p.offsets + e + 1) < load_ordered(p.offsets + e);
        group_tiles[e] = ((r.y - r.x + q.nt - 1) / q.nt) * q.n_blocks;
    }
    if (__syncthreads_or(decreasing)) {
        if (warp == 0) separate_groups(group_row, p.E);
        __syncthreads();
        for (int e = tid; e < p.E; e += blockDim.x) group_tiles[e] = ((group_row[e].y - group_row[e].x + q.nt - 1) / q.nt) * q.n_blocks;
        __syncthreads();
    }
    if (warp == 0) {
        // no more in all than the host counted; as 32-bit sums they cost the kernel a spilled register
        long long before = 0;
        for (int e0 = 0; e0 < p.E; e0 += 32) {
            long long upto = e0 + lane < p.E ? group_tiles[e0 + lane] : 0;
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const long long v = __shfl_up_sync(0xFFFFFFFFu, upto, d);
                if (lane >= d) upto += v;
            }
            if (e0 + lane < p.E) group_tiles[e0 + lane] = (int)(before + upto);
            before += __shfl_sync(0xFFFFFFFFu, upto, 31);
        }
    }
    __syncthreads();
    return group_tiles[p.E - 1];
}

// ---- host

using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                 const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline EncodeTiled encode_tiled() {
    static const EncodeTiled f = [] {
        void *ptr = nullptr;
        cudaDriverEntryPointQueryResult found;
        const bool ok = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &ptr, 12000, cudaEnableDefault, &found) == cudaSuccess &&
                        found == cudaDriverEntryPointSuccess;
        return ok ? (EncodeTiled)ptr : (EncodeTiled) nullptr;
    }();
    return f;
}
// Byte matrix [rows][row_bytes], rows `stride` bytes apart, in boxes of box_rows x box_bytes, swizzled over a box row.
inline bool encode_map(CUtensorMap *map, const void *base, uint64_t row_bytes, uint64_t rows, uint64_t stride, uint32_t box_bytes, uint32_t box_rows) {
    const cuuint64_t dims[2] = {row_bytes, rows}, strides[1] = {stride};
    const cuuint32_t box[2] = {box_bytes, box_rows}, one[2] = {1, 1};
    const EncodeTiled f = encode_tiled();
    return f && f(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  box_bytes == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : box_bytes == 64 ? CU_TENSOR_MAP_SWIZZLE_64B
                  : box_bytes == 32 ? CU_TENSOR_MAP_SWIZZLE_32B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace hikonv
