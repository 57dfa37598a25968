// A persistent tensor-core product for sm_100a, the base of the softmax operators (softmax.cu): C = A B^T with both
// operands in 16 bits and fp32 accumulators in tensor memory.
//
// One CTA (CG = 1: tiles of 128 x BN) or a pair of CTAs on two SMs (CG = 2: tiles of 256 x BN, each CTA holds half of
// either operand) walks tiles in a fixed order. Warp 0 fetches 64-wide slices of both operands with tiled bulk copies
// into a ring of stages, one thread of warp 1 issues the products (the pair's leader for both CTAs), eight warps read
// the accumulators back and finish the tile while the next tile's products run into the other half of tensor memory.
//
// Either operand may have the summed index contiguous ("K-major", rows of 64 elements) or the other one
// ("MN-major", boxes of 64 x 64 elements); both in the 128-byte swizzle.
//
// Single precision goes through the same kernel: an fp32 matrix is held as three bf16 planes whose sum has all 24 bits,
// and the six products of planes that matter (2+0, 0+2, 1+1, 1+0, 0+1, 0+0; what is left is below 2^-24) are summed into
// one accumulator. `pairs` is 1 or 6.
//
// Every wait is bounded in time; a wait that runs out sets a status bit, the CTA's copies and products in flight are
// waited for and tensor memory is given back before it returns.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "chicle_internal.cuh"

namespace chicle {
namespace tc {

constexpr int kBK = 64;              // summed elements per stage: 128 bytes, one swizzle span
constexpr int kThreads = 320;        // copy warp, product warp, 8 epilogue warps
constexpr int kEpiWarps = 8;
constexpr uint64_t kWaitNs = 4000000000ull;

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// Arrives at a barrier of any CTA of the cluster (a shared::cluster address).
__device__ __forceinline__ void bar_arrive_cluster(uint32_t bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ uint64_t now_ns()
{
    uint64_t t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}
// False once the wait has run out, here or in another role of the CTA.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile uint32_t *stopped)
{
    if (bar_try(bar, parity)) return true;
    const uint64_t t0 = now_ns();
    for (;;) {
        for (int i = 0; i < 64; ++i)
            if (bar_try(bar, parity)) return true;
        if (*stopped) return false;
        if (now_ns() - t0 > kWaitNs) {
            *stopped = 1;
            return false;
        }
    }
}
// The same address in CTA `rank` of the cluster.
__device__ __forceinline__ uint32_t map_rank(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

template <int CG>
__device__ __forceinline__ void fetch(uint32_t dst, const CUtensorMap *map, int32_t x, int32_t y, int32_t z, uint32_t bar)
{
    if constexpr (CG == 2)
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4}], [%5];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}

// Shared-memory descriptor, 128-byte swizzle. K-major: 8 rows of 128 bytes per group, groups 1024 bytes apart.
// MN-major: 64 x 8 elements per group, groups along K 1024 bytes apart, along MN `lead` bytes apart.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, uint32_t lead)
{
    return (uint64_t)((addr & 0x3FFFF) >> 4) | ((uint64_t)(lead >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) |
           ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}

template <int CG>
__device__ __forceinline__ void product(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add)
{
    if constexpr (CG == 2)
        asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
    else
        asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
// The barrier (of both CTAs of a pair) is arrived at when all products issued before are done.
template <int CG> __device__ __forceinline__ void commit(uint32_t bar)
{
    if constexpr (CG == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(bar), "h"((uint16_t)3) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void wait_loads() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// 32 columns of this warp's 32 rows: register j of a lane is column j of the lane's row. Asynchronous until wait_loads.
__device__ __forceinline__ void load32(uint32_t addr, uint32_t (&r)[32])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
                   "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
                   "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(addr));
}

// Which operand elements and which tiles. All counts in int32; products of them in int64.
struct Shape {
    int32_t m, n;           // rows and columns of C
    int32_t m_tiles, n_tiles;
    int32_t k_steps;        // slices of kBK of the summed index (per pair of planes)
    int32_t pairs;          // 1, or 6 for single precision
    int32_t splits;         // the summed index is cut into so many pieces, each a tile of its own
    int32_t group;          // m tiles walked together before the next column of tiles
    int32_t half;           // operands fp16 (else bf16)
    uint32_t *status;       // may be null
};

struct Tile {
    int32_t m, n, split;
    int32_t first, last; // slices of the flattened (k step, pair of planes) order
};

// Tile t of the walk: groups of `group` m tiles; within a group, splits outermost, then n, then m.
__device__ __forceinline__ Tile tile_of(const Shape &s, int64_t t)
{
    Tile r;
    const int64_t per_group = (int64_t)s.group * s.n_tiles * s.splits;
    const int32_t g = (int32_t)(t / per_group);
    int64_t in = t - (int64_t)g * per_group;
    const int32_t gm = min(s.group, s.m_tiles - g * s.group);
    const int64_t per_split = (int64_t)gm * s.n_tiles;
    r.split = (int32_t)(in / per_split);
    in -= (int64_t)r.split * per_split;
    r.n = (int32_t)(in / gm);
    r.m = g * s.group + (int32_t)(in - (int64_t)r.n * gm);
    const int64_t all = (int64_t)s.k_steps * s.pairs;
    r.first = (int32_t)(all * r.split / s.splits);
    r.last = (int32_t)(all * (r.split + 1) / s.splits);
    return r;
}

// Planes of the six products, smallest first.
__device__ __forceinline__ int plane_a(int pairs, int q) { return pairs == 1 ? 0 : (0x001102 >> (4 * q)) & 3; }
__device__ __forceinline__ int plane_b(int pairs, int q) { return pairs == 1 ? 0 : (0x010120 >> (4 * q)) & 3; }

template <int CG, int BN> struct Layout {
    static constexpr int kBM = 128;                // rows of A per CTA
    static constexpr int kBNc = BN / CG;           // rows of B per CTA
    static constexpr uint32_t kABytes = kBM * kBK * 2;
    static constexpr uint32_t kBBytes = kBNc * kBK * 2;
    static constexpr uint32_t kStageBytes = kABytes + kBBytes;
    static constexpr int kStages = (int)((200u * 1024u) / kStageBytes) > 8 ? 8 : (int)((200u * 1024u) / kStageBytes);
    static constexpr uint32_t kSmem = kStages * kStageBytes + 1024; // room to start on 1024 bytes
};

// Epi has `template <int BN> __device__ void tile(const Shape &, const Tile &, int row0, int col0, uint32_t tmem, int quarter,
// int half, int lane) const`: called by each of the eight epilogue warps, it finishes rows row0 + 32 quarter .. and the
// columns col0 + half BN / 2 .. of the tile. It has read tensor memory when it returns.
template <int CG, int BN, bool AMN, bool BMN, class Epi>
__global__ void __launch_bounds__(kThreads, 1)
k_product(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const Shape s, const Epi epi)
{
    using L = Layout<CG, BN>;
    constexpr uint32_t kCols = 2 * BN; // tensor memory columns: two accumulators
    static_assert(kCols == 512 || kCols == 256 || kCols == 128, "a power of two");
    extern __shared__ uint8_t smem_raw[];
    __shared__ alignas(8) uint64_t s_full[L::kStages], s_empty[L::kStages], s_done[2], s_free[2], s_drain;
    __shared__ uint32_t s_tmem;
    __shared__ volatile uint32_t s_stop;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CG == 2 ? cluster_rank() : 0;
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
    if (threadIdx.x == 0) {
        for (int i = 0; i < L::kStages; ++i) {
            bar_init(smem_u32(&s_full[i]), 1);
            bar_init(smem_u32(&s_empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(smem_u32(&s_done[i]), 1);
            bar_init(smem_u32(&s_free[i]), CG * kEpiWarps);
        }
        bar_init(smem_u32(&s_drain), 1);
        s_stop = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_a) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_b) : "memory");
    }
    if (warp == 1) {
        if constexpr (CG == 2) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(kCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(kCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
        fence_before();
    }
    __syncthreads();
    if constexpr (CG == 2) cluster_sync();
    fence_after();
    const uint32_t tmem = s_tmem;

    const int64_t tiles = (int64_t)s.m_tiles * s.n_tiles * s.splits;
    const int64_t first_tile = blockIdx.x / CG, stride = gridDim.x / CG;

    if (warp == 0) {
        if (lane == 0) {
            uint32_t it = 0; // slices fetched so far
            bool ok = true;
            // a copy of either CTA of a pair completes at the leader's barrier
            for (int64_t t = first_tile; ok && t < tiles; t += stride) {
                const Tile tl = tile_of(s, t);
                const int row = (tl.m * CG + (int)rank) * L::kBM, col = tl.n * BN + (int)rank * L::kBNc;
                int k = tl.first / s.pairs, q = tl.first - k * s.pairs;
                for (int i = tl.first; i < tl.last; ++i, ++it) {
                    const uint32_t st = it % L::kStages, ph = (it / L::kStages) & 1;
                    if (!bar_wait(smem_u32(&s_empty[st]), ph ^ 1, &s_stop)) {
                        ok = false;
                        break;
                    }
                    uint32_t full = smem_u32(&s_full[st]);
                    if (rank == 0) bar_expect(full, CG * L::kStageBytes);
                    if constexpr (CG == 2) full = map_rank(full, 0);
                    const uint32_t a = ring + st * L::kStageBytes, b = a + L::kABytes;
                    const int za = plane_a(s.pairs, q), zb = plane_b(s.pairs, q);
                    if constexpr (AMN) {
#pragma unroll
                        for (int j = 0; j < L::kBM / 64; ++j) fetch<CG>(a + j * 8192, &map_a, row + j * 64, k * kBK, za, full);
                    } else {
                        fetch<CG>(a, &map_a, k * kBK, row, za, full);
                    }
                    if constexpr (BMN) {
#pragma unroll
                        for (int j = 0; j < L::kBNc / 64; ++j) fetch<CG>(b + j * 8192, &map_b, col + j * 64, k * kBK, zb, full);
                    } else {
                        fetch<CG>(b, &map_b, k * kBK, col, zb, full);
                    }
                    if (++q == s.pairs) {
                        q = 0;
                        ++k;
                    }
                }
            }
            if (!ok && rank == 0) // what is in flight still lands in this CTA's shared memory
                for (uint32_t j = it > (uint32_t)L::kStages ? it - L::kStages : 0; j < it; ++j) {
                    const uint64_t t0 = now_ns();
                    while (!bar_try(smem_u32(&s_full[j % L::kStages]), (j / L::kStages) & 1) && now_ns() - t0 < kWaitNs) {}
                }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            const uint32_t type = s.half ? 0u : 1u;
            const uint32_t idesc = (1u << 4) | (type << 7) | (type << 10) | ((AMN ? 1u : 0u) << 15) | ((BMN ? 1u : 0u) << 16) |
                                   ((uint32_t)(BN >> 3) << 17) | ((uint32_t)((CG * 128) >> 4) << 24);
            uint32_t it = 0, n_tile = 0;
            bool ok = true;
            for (int64_t t = first_tile; ok && t < tiles; t += stride, ++n_tile) {
                const Tile tl = tile_of(s, t);
                const uint32_t acc = n_tile & 1, ph = (n_tile >> 1) & 1;
                if (!bar_wait(smem_u32(&s_free[acc]), ph ^ 1, &s_stop)) break;
                fence_after();
                const uint32_t d = tmem + acc * BN;
                for (int i = tl.first; i < tl.last; ++i, ++it) {
                    const uint32_t st = it % L::kStages;
                    if (!bar_wait(smem_u32(&s_full[st]), (it / L::kStages) & 1, &s_stop)) {
                        ok = false;
                        break;
                    }
                    fence_after();
                    const uint32_t a = ring + st * L::kStageBytes;
                    const uint64_t da = operand_desc(a, AMN ? 8192 : 16), db = operand_desc(a + L::kABytes, BMN ? 8192 : 16);
#pragma unroll
                    for (int kk = 0; kk < kBK / 16; ++kk) // 16 summed elements: 32 bytes on (K-major) or two groups of 8 rows
                        product<CG>(d, da + kk * (AMN ? 128 : 2), db + kk * (BMN ? 128 : 2), idesc, i > tl.first || kk > 0);
                    commit<CG>(smem_u32(&s_empty[st]));
                }
                if (ok) commit<CG>(smem_u32(&s_done[acc]));
            }
            if (s_stop) { // products in flight are waited for before tensor memory is given back
                commit<CG>(smem_u32(&s_drain));
                const uint64_t t0 = now_ns();
                while (!bar_try(smem_u32(&s_drain), 0) && now_ns() - t0 < kWaitNs) {}
            }
        }
    } else {
        const int w = warp - 2;
        uint32_t n_tile = 0;
        for (int64_t t = first_tile; t < tiles; t += stride, ++n_tile) {
            const Tile tl = tile_of(s, t);
            const uint32_t acc = n_tile & 1, ph = (n_tile >> 1) & 1;
            // (one lane's verdict for the warp: the loads from tensor memory are the whole warp's)
            bool ok = true;
            if (lane == 0) ok = bar_wait(smem_u32(&s_done[acc]), ph, &s_stop);
            if (!__shfl_sync(0xffffffffu, (int)ok, 0)) break;
            fence_after();
            // (the lanes of tensor memory that a warp may read are 32 (its number in the CTA % 4) ..)
            epi.template tile<BN>(s, tl, (tl.m * CG + (int)rank) * L::kBM, tl.n * BN, tmem + acc * BN, warp & 3, w >> 2, lane);
            fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive_cluster(CG == 2 ? map_rank(smem_u32(&s_free[acc]), 0) : smem_u32(&s_free[acc]));
        }
    }
    __syncwarp();
    fence_before();
    __syncthreads();
    if constexpr (CG == 2) cluster_sync();
    fence_after();
    if (warp == 1) {
        if constexpr (CG == 2)
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCols) : "memory");
        else
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCols) : "memory");
    }
    if (threadIdx.x == 0 && s_stop && s.status) atomicOr(s.status, (uint32_t)ST_WAIT_TIMEOUT);
}

} // namespace tc
} // namespace chicle
