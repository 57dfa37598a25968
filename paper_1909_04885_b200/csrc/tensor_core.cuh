// A persistent tensor-core product for sm_100a, the base of the softmax operators (softmax.cu): C = A B^T with both
// operands in 16 bits and fp32 accumulators in tensor memory.
//
// One CTA (CG = 1: tiles of 128 x BN) or a pair of CTAs on two SMs (CG = 2: tiles of 256 x BN, each CTA holds half of
// either operand) walks tiles in a fixed order. Warp 0 fetches 64-wide slices of both operands with tiled bulk copies
// into a ring of stages, one thread of warp 1 issues the products (the pair's leader for both CTAs), the other warps read
// the accumulators back and finish the tile while the next tile's products run into the other half of tensor memory.
//
// Either operand may have the summed index contiguous ("K-major", rows of 64 elements) or the other one
// ("MN-major", boxes of 64 x 64 elements); both in the 128-byte swizzle.
//
// Single precision goes through the same kernel: an fp32 matrix, scaled by a power of two so that its largest element
// lies in [2^14, 2^15), is held as two fp16 planes. Their sum is off by 2^-22 of an element at most (1e-7 on average, what a sum
// in fp32 is off by, too), and of elements below 2^-17 of the largest by 2^-39 of that. Three products of planes (1+0, 0+1,
// 0+0) are summed into one accumulator; the fourth is below 2^-22 of a term. `pairs` is 1, 3, or 2: A alone in two planes.
//
// The tensor cores cut an accumulator's low bits off at every step of 16 terms, and the terms' below them: 1.6e-7 to 1.9e-7 of the
// accumulator per step, always with the same sign (measured: sums of 131072 terms of one sign came out 5e-4 too small, of both signs
// with 12 000 steps 1.3e-5). So a sum that has to keep fp32's accuracy is cut into chunks of `chunk` slices, each with an
// accumulator of its own in tensor memory, and the epilogue's warps add the chunks in registers; inside a chunk the small products
// of planes come first.
//
// Every wait is bounded in time; a wait that runs out sets a status bit, the CTA's tiles that are not finished come out NaN, its
// copies and products in flight are waited for (within the same limit, all of them together) and tensor memory is given back
// before it returns.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "operators.cuh"

namespace chicle {
namespace tc {

constexpr int kBK = 64;              // summed elements per stage: 128 bytes, one swizzle span
constexpr int kEpiWarps = 8;                 // (sixteen with half the columns each: products of 4096 terms 6 % slower, of 64 the same)
constexpr int kThreads = 64 + 32 * kEpiWarps; // and a copy warp, a product warp
constexpr uint32_t kPatchBytes = 2048;  // shared memory of an epilogue warp: 32 rows of 64 bytes
constexpr long long kWaitClocks = 6000000000ll; // some seconds: Shape::limit, but for tests

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
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// False once the wait has run out, here or in another role of the CTA.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile uint32_t *stopped, long long limit)
{
    if (bar_try(bar, parity)) return true;
    const long long t0 = clock64();
    for (;;) {
#pragma unroll 1
        for (int i = 0; i < 16; ++i)
            if (bar_try(bar, parity)) return true;
        if (*stopped) return false;
        if (clock64() - t0 > limit) {
            *stopped = 1;
            return false;
        }
    }
}
// The epilogue's warps wait for an accumulator: one of their threads looks, the others sleep at a barrier (threads that all
// look take power and issue slots from the products: dX of 2048 rows, 32768 classes and 4096 columns took 410 us, 396 so). All of
// them get the same answer.
__device__ __forceinline__ bool epilogue_wait(uint32_t bar, uint32_t parity, volatile uint32_t *stopped, long long limit, volatile uint32_t *answer,
                                              bool looks)
{
    if (looks) *answer = bar_wait(bar, parity, stopped, limit);
    __syncwarp();
    asm volatile("bar.sync 1, %0;" ::"n"(32 * kEpiWarps) : "memory");
    return *answer != 0;
}
// For what is in flight when a CTA stops. t0: when its drains began; they share one limit.
__device__ __forceinline__ void bar_drain(uint32_t bar, uint32_t parity, long long t0, long long limit)
{
    while (!bar_try(bar, parity) && clock64() - t0 <= limit) {}
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
// The barrier (of both CTAs of a pair, or of those in `ctas`) is arrived at when all products issued before are done.
template <int CG> __device__ __forceinline__ void commit(uint32_t bar, uint32_t ctas = 3)
{
    if constexpr (CG == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(bar), "h"((uint16_t)ctas) : "memory");
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
    int32_t a_rows;         // rows of A that a copy brings: 128, or fewer where C has no more (K-major A, CG = 1 only)
    int32_t cols;           // columns per tile: BN, or fewer (a multiple of 16, CG = 1 only; every epilogue warp keeps some)
    int32_t k_steps;        // slices of kBK of the summed index (per pair of planes)
    int32_t pairs;          // products of planes: 1, 3 (single precision) or 2 (A in two planes)
    int32_t parts;          // epilogue warps that share a tile's columns
    int32_t chunk;          // slices whose products of planes come one behind the other; kChunked: summed in one accumulator
    int32_t splits;         // the summed index is cut into so many pieces, each a tile of its own
    int32_t group;          // m tiles walked together before the next column of tiles
    int32_t half;           // operands fp16 (else bf16)
    int64_t fetched;        // tiles whose operands are fetched: all of them, but for a test of what happens where a copy never comes
    int64_t limit;          // of a wait, in clocks
    uint32_t *status;       // may be null
};

struct Tile {
    int32_t m, n, split;
    int32_t first, last; // slices
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
    r.first = (int32_t)((int64_t)s.k_steps * r.split / s.splits);
    r.last = (int32_t)((int64_t)s.k_steps * (r.split + 1) / s.splits);
    return r;
}

// Planes of the products, smallest first.
__device__ __forceinline__ int plane_a(int pairs, int q) { return pairs > 1 && q == 0; }
__device__ __forceinline__ int plane_b(int pairs, int q) { return pairs == 3 && q == 1; }

template <int CG, int BN> struct Layout {
    static constexpr int kBM = 128;                // rows of A per CTA
    static constexpr int kBNc = BN / CG;           // rows of B per CTA (at most)
    static constexpr uint32_t kABytes = kBM * kBK * 2;
    static constexpr uint32_t kBBytes = kBNc * kBK * 2;
    static constexpr uint32_t kStageBytes = kABytes + kBBytes;
    static constexpr int kStages = (int)((192u * 1024u) / kStageBytes) > 8 ? 8 : (int)((192u * 1024u) / kStageBytes);
    static constexpr uint32_t kSmem = kStages * kStageBytes + kEpiWarps * kPatchBytes + 1024; // room to start on 1024 bytes
    static_assert(kSmem <= 227u * 1024u - 512u, "shared memory of an SM");
};

// 16-byte piece `c` of row `r` of a warp's patch: rows of 64 bytes whose pieces are exchanged so that both a piece of all rows and
// whole rows are free of bank conflicts. Results go through it so that a warp's store covers 8 rows of 64 bytes, not 32 of 16.
__device__ __forceinline__ uint4 *patch_at(uint8_t *patch, int r, int c) { return reinterpret_cast<uint4 *>(patch + r * 64 + ((c ^ ((r >> 1) & 3)) << 4)); }

// Epi has `template <int N> __device__ void finish(const Shape &, const Tile &, int row0, int lane, int col, int end, bool ok,
// uint32_t (&acc)[N], uint8_t *patch) const`: called by the epilogue warps, lane by lane with N columns col .. of row
// row0 + lane of C (rows behind the last and columns from `end` on are not C's: what acc holds there is undefined). Not ok: the
// CTA has stopped, acc holds nothing, and the tile's results are to be NaN. All lanes call. kChunked: every chunk has an
// accumulator, and finish gets the sums of all columns of the warp (128 sums, and 32 more on their way: 168 registers, the most
// that 320 threads can have, and about 100 bytes of spills with tiles of 256); else a tile has one, and finish gets Epi::kStep
// columns at a time (0: all).
template <int CG, int BN, bool AMN, bool BMN, bool kChunked, class Epi>
__global__ void __launch_bounds__(kThreads, 1)
k_product(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const Shape s, const Epi epi)
{
    using L = Layout<CG, BN>;
    constexpr uint32_t kCols = 2 * BN; // tensor memory columns: two accumulators
    static_assert(kCols == 512 || kCols == 256 || kCols == 128, "a power of two");
    extern __shared__ uint8_t smem_raw[];
    __shared__ alignas(8) uint64_t s_full[L::kStages], s_empty[L::kStages], s_done[2], s_free[2], s_drain;
    __shared__ uint32_t s_tmem;
    __shared__ volatile uint32_t s_stop, s_answer[2]; // (two answers: the thread that looks is less than two ahead)

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
            const uint32_t bytes = CG * (uint32_t)(s.a_rows + s.cols / CG) * (kBK * 2);
            for (int64_t t = first_tile; ok && t < s.fetched; t += stride) {
                const Tile tl = tile_of(s, t);
                const int row = (tl.m * CG + (int)rank) * L::kBM, col = tl.n * s.cols + (int)rank * L::kBNc;
                for (int c0 = tl.first; ok && c0 < tl.last; c0 += s.chunk) {
                    const int c1 = min(c0 + s.chunk, tl.last);
                    for (int q = 0; ok && q < s.pairs; ++q) {
                        const int za = plane_a(s.pairs, q), zb = plane_b(s.pairs, q);
                        for (int k = c0; k < c1; ++k, ++it) {
                            const uint32_t st = it % L::kStages, ph = (it / L::kStages) & 1;
                            if (!bar_wait(smem_u32(&s_empty[st]), ph ^ 1, &s_stop, s.limit)) {
                                ok = false;
                                break;
                            }
                            uint32_t full = smem_u32(&s_full[st]);
                            if (rank == 0) bar_expect(full, bytes);
                            if constexpr (CG == 2) full = map_rank(full, 0);
                            const uint32_t a = ring + st * L::kStageBytes, b = a + L::kABytes;
                            if constexpr (AMN) {
#pragma unroll
                                for (int j = 0; j < L::kBM / 64; ++j) fetch<CG>(a + j * 8192, &map_a, row + j * 64, k * kBK, za, full);
                            } else {
                                fetch<CG>(a, &map_a, k * kBK, row, za, full);
                            }
                            if constexpr (BMN) {
#pragma unroll
                                for (int j = 0; j < L::kBNc / 64; ++j) // (only whole tiles: cols == BN)
                                    fetch<CG>(b + j * 8192, &map_b, col + j * 64, k * kBK, zb, full);
                            } else {
                                fetch<CG>(b, &map_b, k * kBK, col, zb, full);
                            }
                        }
                    }
                }
            }
            // The products' arrivals at this CTA's barriers have to be there before it ends: its shared memory belongs to the next
            // CTA on the SM then, and an arrival that comes late would count at that one's barrier. So the last use of every
            // stage is waited for. (Stopped: the copies in flight, which complete at the leader's barriers.)
            const uint32_t used = it < (uint32_t)L::kStages ? it : L::kStages;
            const long long t0 = clock64();
            for (uint32_t j = it - used; j < it; ++j) {
                if (ok) ok = bar_wait(smem_u32(&s_empty[j % L::kStages]), (j / L::kStages) & 1, &s_stop, s.limit);
                if (!ok && rank == 0) bar_drain(smem_u32(&s_full[j % L::kStages]), (j / L::kStages) & 1, t0, s.limit);
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            const uint32_t type = s.half ? 0u : 1u;
            const uint32_t idesc = (1u << 4) | (type << 7) | (type << 10) | ((AMN ? 1u : 0u) << 15) | ((BMN ? 1u : 0u) << 16) |
                                   ((uint32_t)(s.cols >> 3) << 17) | ((uint32_t)((CG * 128) >> 4) << 24);
            uint32_t it = 0, n_chunk = 0;
            bool ok = true;
            for (int64_t t = first_tile; ok && t < tiles; t += stride) {
                const Tile tl = tile_of(s, t);
                const int step = kChunked ? s.chunk : tl.last - tl.first;
                for (int c0 = tl.first; c0 < tl.last; c0 += step, ++n_chunk) {
                    const int slices = (min(c0 + step, tl.last) - c0) * s.pairs;
                    const uint32_t acc = n_chunk & 1;
                    ok = bar_wait(smem_u32(&s_free[acc]), ((n_chunk >> 1) & 1) ^ 1, &s_stop, s.limit);
                    if (!ok) break;
                    fence_after();
                    const uint32_t d = tmem + acc * BN;
                    for (int i = 0; i < slices; ++i, ++it) {
                        const uint32_t st = it % L::kStages;
                        ok = bar_wait(smem_u32(&s_full[st]), (it / L::kStages) & 1, &s_stop, s.limit);
                        if (!ok) break;
                        fence_after();
                        const uint32_t a = ring + st * L::kStageBytes;
                        const uint64_t da = operand_desc(a, AMN ? 8192 : 16), db = operand_desc(a + L::kABytes, BMN ? 8192 : 16);
#pragma unroll
                        for (int kk = 0; kk < kBK / 16; ++kk) // 16 summed elements: 32 bytes on (K-major) or two groups of 8 rows
                            product<CG>(d, da + kk * (AMN ? 128 : 2), db + kk * (BMN ? 128 : 2), idesc, i > 0 || kk > 0);
                        commit<CG>(smem_u32(&s_empty[st]));
                    }
                    if (!ok) break;
                    commit<CG>(smem_u32(&s_done[acc]));
                }
            }
            // (and the epilogues' last arrivals, the other CTA's among them)
            for (uint32_t j = n_chunk < 2 ? 0 : n_chunk - 2; ok && j < n_chunk; ++j) ok = bar_wait(smem_u32(&s_free[j & 1]), (j >> 1) & 1, &s_stop, s.limit);
            if (s_stop) { // products in flight are waited for before tensor memory is given back
                commit<CG>(smem_u32(&s_drain), 1); // (this CTA's barrier alone: the other one waits for nothing there)
                bar_drain(smem_u32(&s_drain), 0, clock64(), s.limit);
            }
        }
    } else {
        constexpr int kN = BN * 4 / kEpiWarps; // columns of a warp
        // the lanes of tensor memory that a warp may read: 32 (its number in the CTA % 4) ..
        const int quarter = warp & 3, part = (warp - 2) >> 2;
        const uint32_t at = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(part * kN);
        uint8_t *patch = smem_raw + (ring - smem_u32(smem_raw)) + L::kStages * L::kStageBytes + (warp - 2) * kPatchBytes;
        uint32_t n_chunk = 0;
        bool ok = true;
        for (int64_t t = first_tile; t < tiles; t += stride) { // (stopped: the tiles that are left come out NaN)
            const Tile tl = tile_of(s, t);
            const int row0 = (tl.m * CG + (int)rank) * L::kBM + quarter * 32, col = tl.n * s.cols + part * kN;
            const int end = min(s.n, (tl.n + 1) * s.cols); // the tile's columns end here
            static_assert(Epi::kStep % 32 == 0, "loads are of 32 columns");
            if constexpr (!kChunked) {
                constexpr int kStep = Epi::kStep ? Epi::kStep : kN;
                const uint32_t a = n_chunk & 1;
                if (ok) ok = epilogue_wait(smem_u32(&s_done[a]), (n_chunk >> 1) & 1, &s_stop, s.limit, &s_answer[a], threadIdx.x == 64);
                ++n_chunk;
                fence_after();
#pragma unroll 1
                for (int c = 0; c < kN && col + c < end; c += kStep) {
                    uint32_t r[kStep];
                    // (stopped: loaded all the same, a branch around the loads costs the full-width epilogues 800 bytes of spills)
#pragma unroll
                    for (int j = 0; j < kStep; j += 32)
                        if (j == 0 || col + c + j < end) load32(at + a * BN + c + j, *reinterpret_cast<uint32_t(*)[32]>(&r[j]));
                    wait_loads();
                    epi.template finish<kStep>(s, tl, row0, lane, col + c, end, ok, r, patch);
                }
                fence_before();
                __syncwarp();
                if (ok && lane == 0) bar_arrive_cluster(CG == 2 ? map_rank(smem_u32(&s_free[a]), 0) : smem_u32(&s_free[a]));
            } else {
            uint32_t acc[kN];
            for (int c0 = tl.first; ok && c0 < tl.last; c0 += s.chunk, ++n_chunk) {
                const uint32_t a = n_chunk & 1;
                ok = epilogue_wait(smem_u32(&s_done[a]), (n_chunk >> 1) & 1, &s_stop, s.limit, &s_answer[a], threadIdx.x == 64);
                if (!ok) break;
                fence_after();
                if (c0 == tl.first) {
#pragma unroll
                    for (int c = 0; c < kN; c += 32)
                        if (col + c < end) load32(at + a * BN + c, *reinterpret_cast<uint32_t(*)[32]>(&acc[c]));
                    wait_loads();
                } else {
#pragma unroll
                    for (int c = 0; c < kN; c += 32)
                        if (col + c < end) {
                            uint32_t r[32];
                            load32(at + a * BN + c, r);
                            wait_loads();
#pragma unroll
                            for (int j = 0; j < 32; ++j) acc[c + j] = __float_as_uint(__uint_as_float(acc[c + j]) + __uint_as_float(r[j]));
                        }
                }
                fence_before();
                __syncwarp();
                if (lane == 0) bar_arrive_cluster(CG == 2 ? map_rank(smem_u32(&s_free[a]), 0) : smem_u32(&s_free[a]));
            }
            epi.template finish<kN>(s, tl, row0, lane, col, end, ok, acc, patch);
            }
            __syncwarp();
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
