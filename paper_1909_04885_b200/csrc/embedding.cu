// Embedding lookup with scaling, and its gradient by sorted ids (chicle_embedding, chicle_embedding_grad): the product of
// a row of ids with a model that has a vector per id, and the sum of the rows' gradients per id.
//
//   out_i = s T[id_i]                dT_v = s sum_{i: id_i = v} G_i
//
// Both are bound by memory. The gradient sorts (id, position) pairs, stably, so that the terms of an id are added in one
// order whatever the timing: up to 4096 ids each position counts the ones in front of it (n^2 comparisons, one launch),
// above that by radix passes of up to 10 bits. The sorted entries are cut into windows of equal length; a window sums
// its runs of equal ids, writes those that lie inside it and leaves the ones that cross its ends as partial sums in fp32, which
// a last kernel adds in order. So an id with most of the entries takes no longer than many ids with a few.
// Rows without an id are zeroed by further CTAs of the same launches: the sort leaves the memory idle.
#include <algorithm>
#include <cmath>

#include "operators.cuh"

namespace chicle {
namespace {

constexpr int kMaxRankN = 4096;   // ids sorted by counting (8192 ids of 1000 rows of 256: 46 us in all, with one radix pass 34)
constexpr int kTile = 2048;       // entries per CTA of a radix pass
constexpr int kTileThreads = 512;
constexpr int kDigits = 1024;
constexpr int kGroupTiles = 16;   // tiles whose digit counts are added up in advance
constexpr int64_t kTargetThreads = 148 * 1024;
constexpr int64_t kZeroBytes = 64 * 1024; // of dtable per zeroing CTA
// What a launch of the sort zeroes beside it: what memory writes in the 8 to 12 us that it takes up to 10^5 entries, and in
// the time that more take.
constexpr int64_t kZeroShare = 48 << 20, kZeroPerEntry = 64;

template <typename T> __device__ __forceinline__ float to_float(T v) { return (float)v; }
template <typename T> __device__ __forceinline__ T of_float(float v);
template <> __device__ __forceinline__ float of_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 of_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half of_float<__half>(float v) { return __float2half_rn(v); }

template <typename T, int E> struct alignas(sizeof(T) * E > 16 ? 16 : sizeof(T) * E) Vec {
    T v[E];
};

// ---- lookup ------------------------------------------------------------------------------------------------

// A thread takes one vector of R rows: R independent row reads are in flight.
template <typename T, int E, int R>
__global__ void __launch_bounds__(256)
k_lookup(const T *__restrict__ table, int64_t ld, int32_t rows, const int32_t *__restrict__ ids, int64_t n, int32_t vecs, int tpr_log,
         float scale, T *__restrict__ out, int64_t ld_out, uint32_t *status)
{
    const int tpr = 1 << tpr_log;
    const int c = blockIdx.y * tpr + (threadIdx.x & (tpr - 1));
    const int64_t i0 = ((int64_t)blockIdx.x * (256 >> tpr_log) + (threadIdx.x >> tpr_log)) * R;
    if (c >= vecs) return;
    Vec<T, E> q[R];
    bool has[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int32_t id = i0 + r < n ? ids[i0 + r] : -1;
        has[r] = (uint32_t)id < (uint32_t)rows;
        if (id >= rows && c == 0 && status) atomicOr(status, (uint32_t)ST_BAD_INDEX);
        if (has[r]) q[r] = *reinterpret_cast<const Vec<T, E> *>(table + (int64_t)id * ld + (int64_t)c * E);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (i0 + r >= n) break;
        Vec<T, E> o;
#pragma unroll
        for (int j = 0; j < E; ++j) o.v[j] = has[r] ? of_float<T>(to_float(q[r].v[j]) * scale) : of_float<T>(0.f);
        *reinterpret_cast<Vec<T, E> *>(out + (i0 + r) * ld_out + (int64_t)c * E) = o;
    }
}

// ---- sorting ids -------------------------------------------------------------------------------------------

__device__ __forceinline__ int32_t key_of(int32_t id, int32_t rows, uint32_t *status)
{
    if (id >= rows && status) atomicOr(status, (uint32_t)ST_BAD_INDEX);
    return (uint32_t)id < (uint32_t)rows ? id : rows; // no id: behind all others
}

// Rows [v0, v1) of dtable to be zeroed, `per` of them by a CTA, in accesses of `width` bytes. `present`: a bit per row; rows
// with an id are left out (null: none are).
struct ZeroJob {
    uint8_t *base;
    int64_t pitch; // bytes
    int32_t row_bytes, width, per;
    int64_t v0, v1;
    const uint32_t *present;
    __host__ __device__ int64_t blocks() const { return v1 > v0 ? (v1 - v0 + per - 1) / per : 0; }
};

template <typename W> __device__ __forceinline__ void zero_rows(const ZeroJob &z, int64_t block)
{
    const int pieces = z.row_bytes / (int)sizeof(W);
    int log = 0;
    while ((1 << log) < pieces && (2 << log) <= (int)blockDim.x) ++log; // threads per row
    const int64_t v0 = z.v0 + block * z.per, v1 = min(v0 + z.per, z.v1);
    for (int64_t v = v0 + (threadIdx.x >> log); v < v1; v += blockDim.x >> log) {
        if (z.present && ((z.present[v >> 5] >> (v & 31)) & 1u)) continue;
        W *row = reinterpret_cast<W *>(z.base + v * z.pitch);
#pragma unroll 4
        for (int c = threadIdx.x & ((1 << log) - 1); c < pieces; c += 1 << log) row[c] = W{};
    }
}

__device__ __forceinline__ void zero_block(const ZeroJob &z, int64_t block)
{
    if (z.width == 16) zero_rows<uint4>(z, block);
    else if (z.width == 8) zero_rows<uint2>(z, block);
    else if (z.width == 4) zero_rows<uint32_t>(z, block);
    else zero_rows<uint16_t>(z, block);
}

// Place of every id in the sorted order: the number of smaller ones, and of equal ones in front of it. 32 ids per CTA,
// eight threads each count an eighth.
__global__ void __launch_bounds__(256) k_rank_ids(const int32_t *__restrict__ ids, int32_t n, int32_t rows, int32_t *__restrict__ keys,
                                                  int32_t *__restrict__ order, uint32_t *status, const ZeroJob zero)
{
    if ((int64_t)blockIdx.x * 32 >= n) return zero_block(zero, (int64_t)blockIdx.x - (n + 31) / 32);
    __shared__ __align__(16) int32_t s_key[kMaxRankN];
    __shared__ int s_part[8][32];
    const int padded = (n + 31) & ~31;
    for (int j = threadIdx.x; j < padded; j += 256) s_key[j] = j < n ? key_of(ids[j], rows, blockIdx.x == 0 ? status : nullptr) : INT32_MAX;
    __syncthreads();
    const int i = blockIdx.x * 32 + (threadIdx.x & 31), part = threadIdx.x >> 5;
    const int32_t mine = i < n ? s_key[i] : -1;
    const int quads = padded / 4;
    const int q0 = quads * part / 8, q1 = quads * (part + 1) / 8;
    int count = 0;
    for (int q = q0; q < q1; ++q) {
        const int4 k = reinterpret_cast<const int4 *>(s_key)[q];
        // in front of i: equal ones count too
        count += (k.x < mine + (4 * q < i)) + (k.y < mine + (4 * q + 1 < i)) + (k.z < mine + (4 * q + 2 < i)) + (k.w < mine + (4 * q + 3 < i));
    }
    s_part[part][threadIdx.x & 31] = count;
    __syncthreads();
    if (part == 0 && i < n) {
        int at = 0;
#pragma unroll
        for (int p = 0; p < 8; ++p) at += s_part[p][threadIdx.x];
        keys[at] = mine;
        order[at] = i;
    }
}

// Digit counts of a tile: its own row of `hist`, and added to its group's row and to the total.
__global__ void __launch_bounds__(kTileThreads) k_id_hist(const int32_t *__restrict__ in, int64_t n, int32_t rows, bool raw, int shift, int digits,
                                                          uint32_t *__restrict__ hist, uint32_t *__restrict__ group,
                                                          uint32_t *__restrict__ total, uint32_t *present, uint32_t *status,
                                                          const ZeroJob zero)
{
    __shared__ uint32_t h[kDigits];
    if ((int64_t)blockIdx.x * kTile >= n) return zero_block(zero, (int64_t)blockIdx.x - (n + kTile - 1) / kTile);
    for (int j = threadIdx.x; j < digits; j += kTileThreads) h[j] = 0;
    __syncthreads();
    const int64_t base = (int64_t)blockIdx.x * kTile;
#pragma unroll
    for (int it = 0; it < kTile / kTileThreads; ++it) {
        const int64_t i = base + it * kTileThreads + threadIdx.x;
        const bool live = i < n;
        const int32_t k = live ? (raw ? key_of(in[i], rows, status) : in[i]) : 0;
        if (live && present && k < rows) { // (looked at first: a frequent id's word would queue up its atomics)
            const uint32_t bit = 1u << (k & 31);
            if (!(__ldcg(&present[k >> 5]) & bit)) atomicOr(&present[k >> 5], bit);
        }
        const int dg = live ? (k >> shift) & (digits - 1) : -1;
        // one atomic per digit of a warp: a frequent id would queue up
        const uint32_t peers = __match_any_sync(0xffffffffu, dg);
        if (live && (threadIdx.x & 31) == __ffs(peers) - 1) atomicAdd(&h[dg], (uint32_t)__popc(peers));
    }
    __syncthreads();
    for (int j = threadIdx.x; j < digits; j += kTileThreads) {
        const uint32_t c = h[j];
        hist[(int64_t)blockIdx.x * digits + j] = c;
        if (c) {
            atomicAdd(&group[(int64_t)(blockIdx.x / kGroupTiles) * digits + j], c);
            atomicAdd(&total[j], c);
        }
    }
}

// Stable scatter of a tile by one digit.
__global__ void __launch_bounds__(kTileThreads) k_id_scatter(const int32_t *__restrict__ in, const int32_t *__restrict__ order_in, int64_t n,
                                                             int32_t rows, bool raw, int shift, int digits, const uint32_t *__restrict__ hist,
                                                             const uint32_t *__restrict__ group, const uint32_t *__restrict__ total,
                                                             int32_t *__restrict__ keys, int32_t *__restrict__ order, const ZeroJob zero)
{
    if ((int64_t)blockIdx.x * kTile >= n) return zero_block(zero, (int64_t)blockIdx.x - (n + kTile - 1) / kTile);
    constexpr int kWarps = kTileThreads / 32, kItems = kTile / kTileThreads;
    extern __shared__ __align__(16) uint32_t smem[];
    uint32_t(*cnt)[kDigits] = reinterpret_cast<uint32_t(*)[kDigits]>(smem); // [warp][digit]
    __shared__ uint32_t s_scan[kWarps];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t base = (int64_t)blockIdx.x * kTile + (int64_t)warp * (kItems * 32);
    const uint32_t below = (1u << lane) - 1u;
    int32_t key[kItems], dig[kItems];
    uint32_t rank[kItems];
#pragma unroll
    for (int it = 0; it < kItems; ++it) {
        const int64_t i = base + it * 32 + lane;
        key[it] = i < n ? (raw ? key_of(in[i], rows, nullptr) : in[i]) : 0;
        dig[it] = i < n ? (key[it] >> shift) & (digits - 1) : -1;
    }
    // where a digit's entries of this tile begin: digits in front (scan of the totals), groups and tiles in front. Two digits
    // per thread, fetched before the ranking so that its loads are on their way meanwhile.
    static_assert(kDigits <= 2 * kTileThreads, "two digits per thread");
    const int g = blockIdx.x / kGroupTiles, d0 = threadIdx.x * 2;
    uint32_t tot[2] = {0, 0}, own[2] = {0, 0};
    if (d0 < digits) { // (digits: an even number)
        const uint2 t2 = *reinterpret_cast<const uint2 *>(total + d0);
        tot[0] = t2.x, tot[1] = t2.y;
#pragma unroll 8
        for (int j = 0; j < g; ++j) {
            const uint2 x = *reinterpret_cast<const uint2 *>(group + (int64_t)j * digits + d0);
            own[0] += x.x, own[1] += x.y;
        }
#pragma unroll 8
        for (int j = g * kGroupTiles; j < (int)blockIdx.x; ++j) {
            const uint2 x = *reinterpret_cast<const uint2 *>(hist + (int64_t)j * digits + d0);
            own[0] += x.x, own[1] += x.y;
        }
    }
    for (int j = threadIdx.x; j < kWarps * kDigits / 4; j += kTileThreads) reinterpret_cast<uint4 *>(smem)[j] = make_uint4(0, 0, 0, 0);
    __syncthreads();
#pragma unroll
    for (int it = 0; it < kItems; ++it) {
        const int d = dig[it];
        const uint32_t peers = __match_any_sync(0xffffffffu, d);
        const uint32_t before = d >= 0 ? cnt[warp][d] : 0u;
        __syncwarp();
        if (d >= 0 && (peers & below) == 0u) cnt[warp][d] = before + __popc(peers);
        __syncwarp();
        rank[it] = before + __popc(peers & below);
    }
    uint32_t inc = tot[0] + tot[1];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
    }
    if (lane == 31) s_scan[warp] = inc;
    __syncthreads(); // (the warps' counters are complete, too)
    uint32_t start = inc - tot[0] - tot[1];
    for (int w = 0; w < warp; ++w) start += s_scan[w];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int d = d0 + k;
        if (d < digits) {
            uint32_t run = start + own[k];
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const uint32_t c = cnt[w][d];
                cnt[w][d] = run;
                run += c;
            }
        }
        start += tot[k];
    }
    __syncthreads();
#pragma unroll
    for (int it = 0; it < kItems; ++it) {
        const int64_t i = base + it * 32 + lane;
        if (i < n) {
            const uint32_t at = cnt[warp][dig[it]] + rank[it];
            keys[at] = key[it];
            order[at] = raw ? (int32_t)i : order_in[i];
        }
    }
}

// ---- sums by id --------------------------------------------------------------------------------------------

// First entry of keys[0, n) that is >= v; a whole warp.
__device__ __forceinline__ int32_t first_not_below(const int32_t *__restrict__ keys, int32_t n, int32_t v)
{
    const int lane = threadIdx.x & 31;
    int32_t lo = 0, len = n; // the answer lies in [lo, lo + len]
    while (len > 0) {
        const int32_t step = (len + 31) / 32;
        const int32_t at = lo + lane * step;
        const uint32_t below = __ballot_sync(0xffffffffu, at < lo + len && keys[at] < v);
        const int32_t k = __popc(below); // the first k probes are below v
        if (k == 0) break;
        const int32_t end = lo + len;
        lo += (k - 1) * step + 1;
        len = min(step - 1, end - lo);
    }
    return lo;
}

struct Sums {
    const int32_t *keys, *order;
    int64_t n;
    int32_t rows, d, vecs;
    int tpr_log, slabs;   // threads per row and slabs of a row
    int64_t window, windows;
    float scale;
    int accumulate;
    float *partial;       // [window][2][d]: of the run that came in, of the run that goes out
    int64_t sum_blocks;   // CTAs that sum; the others zero
    int join_windows;     // windows per CTA of the joining kernel
};

template <typename T, int E>
__device__ __forceinline__ void put_row(const Sums &s, T *table, int64_t ld, int32_t v, int c, const float (&acc)[E])
{
    T *at = table + (int64_t)v * ld + (int64_t)c * E;
    Vec<T, E> o;
    if (s.accumulate) {
        o = *reinterpret_cast<const Vec<T, E> *>(at);
#pragma unroll
        for (int j = 0; j < E; ++j) o.v[j] = of_float<T>(to_float(o.v[j]) + acc[j] * s.scale);
    } else {
#pragma unroll
        for (int j = 0; j < E; ++j) o.v[j] = of_float<T>(acc[j] * s.scale);
    }
    *reinterpret_cast<Vec<T, E> *>(at) = o;
}

template <int E> __device__ __forceinline__ void put_partial(const Sums &s, int64_t at, int c, const float (&acc)[E])
{
    Vec<float, E> o;
#pragma unroll
    for (int j = 0; j < E; ++j) o.v[j] = acc[j];
    *reinterpret_cast<Vec<float, E> *>(s.partial + at * s.d + (int64_t)c * E) = o;
}

// Rows are fetched several at a time (16 bytes each), and enough CTAs have to fit on an SM for the zeroing ones to keep memory
// busy: eight rows of 8 elements take 137 registers and leave room for one (16384 entries of 4096 bf16: 280 us, four rows and four
// CTAs: 215; 131072 entries: 170 with three CTAs, 153 with four; 319488 entries of 64 fp32 the other way round, 132 with four and 116).
template <typename T, int E>
__global__ void __launch_bounds__(256, E == 8 ? 4 : 3) k_sum_by_id(const Sums s, const T *__restrict__ grad, int64_t ld, T *__restrict__ table, int64_t ld_t,
                                                   const ZeroJob zero)
{
    if (blockIdx.x >= s.sum_blocks) return zero_block(zero, (int64_t)blockIdx.x - s.sum_blocks);
    const int tpr = 1 << s.tpr_log, per = 256 >> s.tpr_log;
    const int64_t slab = blockIdx.x % s.slabs, wb = blockIdx.x / s.slabs;
    const int c = (int)slab * tpr + (threadIdx.x & (tpr - 1));
    const int64_t w = wb * per + (threadIdx.x >> s.tpr_log);
    if (c >= s.vecs || w >= s.windows) return;
    const int64_t e0 = w * s.window, e1 = min(e0 + s.window, s.n);
    float acc[E];
    int32_t cur = s.keys[e0];
    bool from_before = e0 > 0 && s.keys[e0 - 1] == cur;
#pragma unroll
    for (int j = 0; j < E; ++j) acc[j] = 0.f;
    constexpr int kAhead = E == 8 ? 4 : 8;
    for (int64_t e = e0; e < e1; e += kAhead) {
        // (windows begin at multiples of 8; the arrays have room behind the last entry)
        const Vec<int32_t, kAhead> at = *reinterpret_cast<const Vec<int32_t, kAhead> *>(s.order + e);
        Vec<int32_t, kAhead> keys = *reinterpret_cast<const Vec<int32_t, kAhead> *>(s.keys + e);
        int32_t(&key)[kAhead] = keys.v;
        Vec<T, E> q[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            if (e + a >= e1) key[a] = s.rows;
            if (key[a] < s.rows) q[a] = *reinterpret_cast<const Vec<T, E> *>(grad + (int64_t)at.v[a] * ld + (int64_t)c * E);
        }
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            if (e + a >= e1) break;
            if (key[a] != cur) {
                if (from_before) {
                    put_partial<E>(s, w * 2, c, acc);
                    from_before = false;
                } else {
                    put_row<T, E>(s, table, ld_t, cur, c, acc);
                }
#pragma unroll
                for (int j = 0; j < E; ++j) acc[j] = 0.f;
                cur = key[a];
            }
            if (cur >= s.rows) return; // from here on entries without an id
#pragma unroll
            for (int j = 0; j < E; ++j) acc[j] += to_float(q[a].v[j]);
        }
    }
    const bool goes_on = e1 < s.n && s.keys[e1] == cur;
    if (!from_before && !goes_on) {
        put_row<T, E>(s, table, ld_t, cur, c, acc);
    } else {
        put_partial<E>(s, w * 2 + (from_before ? 0 : 1), c, acc);
    }
}

// Adds the partial sums of the runs that cross windows, in order. A warp looks at the window where a run may begin; it adds
// a few partial sums itself, many are left to the CTA: its groups of threads take consecutive windows each, and their
// sums are added in order.
constexpr int kWarpJoin = 32; // vectors per lane that a warp takes (16384 entries of 4096 bf16: 44 us with 32 partial sums of any length)

template <typename T, int E>
__global__ void __launch_bounds__(256) k_join_windows(const Sums s, T *__restrict__ table, int64_t ld_t)
{
    __shared__ float s_sum[256][E];
    __shared__ int64_t s_count[8];
    __shared__ int32_t s_key[8];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int tpr = 1 << s.tpr_log;
    const int c_end = min(s.vecs, ((int)blockIdx.y + 1) * tpr), c_begin = (int)blockIdx.y * tpr;
    const int64_t w0 = (int64_t)blockIdx.x * s.join_windows;
    int64_t count = 0;
    {
        const int64_t w = w0 + warp;
        const int64_t e0 = w * s.window, e1 = e0 + s.window;
        if (warp < s.join_windows && e1 < s.n) {
            const int32_t k = s.keys[e1], last = s.keys[e1 - 1], first = s.keys[e0], before = e0 > 0 ? s.keys[e0 - 1] : -1;
            if (last == k && k < s.rows && !(first == k && before == k)) {
                // windows w + 1 .. the one with the run's last entry hold the rest
                const int64_t end = first_not_below(s.keys + e1, (int32_t)(s.n - e1), k + 1) + e1;
                count = (end - 1) / s.window - w + 1;
                if (count * ((c_end - c_begin + 31) / 32) <= kWarpJoin) {
                    for (int c = c_begin + lane; c < c_end; c += 32) {
                        float acc[E];
#pragma unroll
                        for (int j = 0; j < E; ++j) acc[j] = 0.f;
#pragma unroll 4
                        for (int64_t i = 0; i < count; ++i) {
                            const Vec<float, E> p = *reinterpret_cast<const Vec<float, E> *>(s.partial + ((w + i) * 2 + (i == 0 ? 1 : 0)) * s.d + (int64_t)c * E);
#pragma unroll
                            for (int j = 0; j < E; ++j) acc[j] += p.v[j];
                        }
                        put_row<T, E>(s, table, ld_t, k, c, acc);
                    }
                    count = 0;
                }
                if (lane == 0) s_key[warp] = k;
            }
        }
    }
    if (lane == 0) s_count[warp] = count;
    __syncthreads();
    const int groups = 256 >> s.tpr_log, g = threadIdx.x >> s.tpr_log, c = c_begin + (threadIdx.x & (tpr - 1));
    for (int i = 0; i < s.join_windows; ++i) {
        count = s_count[i];
        if (count == 0) continue; // (the same for all threads)
        const int64_t w = w0 + i;
        float acc[E];
#pragma unroll
        for (int j = 0; j < E; ++j) acc[j] = 0.f;
        if (c < c_end) {
            const int64_t a = count * g / groups, b = count * (g + 1) / groups;
#pragma unroll 8
            for (int64_t q = a; q < b; ++q) {
                const Vec<float, E> p = *reinterpret_cast<const Vec<float, E> *>(s.partial + ((w + q) * 2 + (q == 0 ? 1 : 0)) * s.d + (int64_t)c * E);
#pragma unroll
                for (int j = 0; j < E; ++j) acc[j] += p.v[j];
            }
        }
#pragma unroll
        for (int j = 0; j < E; ++j) s_sum[threadIdx.x][j] = acc[j];
        __syncthreads();
        if (g == 0 && c < c_end) {
            for (int o = 1; o < groups; ++o)
#pragma unroll
                for (int j = 0; j < E; ++j) acc[j] += s_sum[threadIdx.x + (o << s.tpr_log)][j];
            put_row<T, E>(s, table, ld_t, s_key[i], c, acc);
        }
        __syncthreads();
    }
}

// ---- host --------------------------------------------------------------------------------------------------

int log2_up(int64_t v)
{
    int l = 0;
    while (((int64_t)1 << l) < v) ++l;
    return l;
}

struct IdPlan {
    int passes = 0, digit_bits = 0;
    int64_t tiles = 0, groups = 0;
    int64_t window = 0, windows = 0;
    size_t keys[2], order[2], hist, group, total, present, partial, bytes; // offsets; what has to begin at zero lies together
    size_t zero_at, zero_bytes;
};

// Windows: long enough that about kTargetThreads threads share the work, eight entries at least.
IdPlan make_plan(int64_t n, int64_t rows, int64_t cols)
{
    IdPlan p;
    size_t at = 0;
    auto take = [&](size_t b) {
        const size_t here = at;
        at += (b + 255) / 256 * 256;
        return here;
    };
    const int64_t threads_per_row = std::max<int64_t>(1, cols / 8);
    const int64_t want = std::max<int64_t>(1, kTargetThreads / threads_per_row);
    p.window = 8;
    while (p.window < 4096 && ceil_div(n, p.window) > want) p.window *= 2;
    p.windows = ceil_div(n, p.window);
    for (int k = 0; k < 2; ++k) {
        p.keys[k] = take((size_t)n * 4 + 32); // (read in eights)
        p.order[k] = take((size_t)n * 4 + 32);
    }
    if (n > kMaxRankN) {
        const int bits = log2_up(rows + 1);
        p.passes = (int)std::max<int64_t>(1, ceil_div(bits, 10));
        p.digit_bits = (int)std::max<int64_t>(1, ceil_div(bits, p.passes)); // (rows + 1 keys: two at least)
        p.tiles = ceil_div(n, kTile);
        p.groups = ceil_div(p.tiles, kGroupTiles);
        const size_t digits = (size_t)1 << p.digit_bits;
        p.hist = take((size_t)p.tiles * digits * 4);
        p.zero_at = at;
        p.group = take((size_t)p.passes * p.groups * digits * 4);
        p.total = take((size_t)p.passes * digits * 4);
        p.present = take((size_t)ceil_div(rows, 32) * 4);
        p.zero_bytes = at - p.zero_at;
    }
    p.partial = take((size_t)p.windows * 2 * cols * 4);
    p.bytes = at;
    return p;
}

// Sorted keys and order are in buffer `which` afterwards. Takes its share of the rows to be zeroed off `zero`.
cudaError_t sort_ids(const IdPlan &p, const int32_t *ids, int64_t n, int32_t rows, uint8_t *ws, uint32_t *status, cudaStream_t s, int *which,
                     ZeroJob *zero)
{
    int32_t *keys[2] = {reinterpret_cast<int32_t *>(ws + p.keys[0]), reinterpret_cast<int32_t *>(ws + p.keys[1])};
    int32_t *order[2] = {reinterpret_cast<int32_t *>(ws + p.order[0]), reinterpret_cast<int32_t *>(ws + p.order[1])};
    *which = 0;
    if (n <= kMaxRankN) {
        // (a few thousand rows at most are written twice)
        const int64_t blocks = ceil_div(n, 32) + zero->blocks();
        k_rank_ids<<<(unsigned)blocks, 256, 0, s>>>(ids, (int32_t)n, rows, keys[0], order[0], status, *zero);
        zero->v0 = zero->v1;
        return cudaGetLastError();
    }
    constexpr int kSmem = kTileThreads / 32 * kDigits * 4;
    cudaError_t e = cudaFuncSetAttribute(k_id_scatter, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e == cudaSuccess) e = cudaMemsetAsync(ws + p.zero_at, 0, p.zero_bytes, s);
    const int digits = 1 << p.digit_bits;
    const int64_t share = std::max<int64_t>(1, (kZeroShare + kZeroPerEntry * n) / zero->row_bytes);
    auto part = [&] { // the next launch's share, in whole words of `present`
        ZeroJob z = *zero;
        z.v1 = std::min(z.v1, (z.v0 + share + 31) / 32 * 32);
        zero->v0 = z.v1;
        return z;
    };
    uint32_t *present = zero->blocks() ? reinterpret_cast<uint32_t *>(ws + p.present) : nullptr;
    for (int k = 0; e == cudaSuccess && k < p.passes; ++k) {
        const bool raw = k == 0;
        const int32_t *in = raw ? ids : keys[(k + 1) & 1];
        uint32_t *hist = reinterpret_cast<uint32_t *>(ws + p.hist);
        uint32_t *group = reinterpret_cast<uint32_t *>(ws + p.group) + (size_t)k * p.groups * digits;
        uint32_t *total = reinterpret_cast<uint32_t *>(ws + p.total) + (size_t)k * digits;
        ZeroJob z = part();
        k_id_hist<<<(unsigned)(p.tiles + z.blocks()), kTileThreads, 0, s>>>(in, n, rows, raw, k * p.digit_bits, digits, hist, group, total,
                                                                            raw ? present : nullptr, status, z);
        if (raw) zero->present = present; // known from here on
        z = part();
        k_id_scatter<<<(unsigned)(p.tiles + z.blocks()), kTileThreads, kSmem, s>>>(in, order[(k + 1) & 1], n, rows, raw, k * p.digit_bits, digits, hist,
                                                                                   group, total, keys[k & 1], order[k & 1], z);
        e = cudaGetLastError();
        *which = k & 1;
    }
    return e;
}

// Elements per access: the largest power of two up to 16 bytes that divides addresses, row pitches and the row length.
int vector_elements(const chicle_dense_t &a, const chicle_dense_t &b)
{
    const int es = element_size(a.type);
    uint64_t bits = 16u | reinterpret_cast<uintptr_t>(a.data) | reinterpret_cast<uintptr_t>(b.data) | (uint64_t)a.cols * es;
    if (a.rows > 1) bits |= (uint64_t)a.ld * es;
    if (b.rows > 1) bits |= (uint64_t)b.ld * es;
    const uint64_t low = bits & (~bits + 1);
    return (int)std::max<uint64_t>(1, low / es);
}

template <typename T, int E>
cudaError_t lookup(const chicle_dense_t &t, const int32_t *ids, float scale, const chicle_dense_t &o, uint32_t *status, cudaStream_t s)
{
    const int vecs = (int)(t.cols / E);
    const int tpr_log = std::min(8, log2_up(vecs));
    const unsigned slabs = (unsigned)ceil_div(vecs, 1 << tpr_log);
    const int64_t per = 256 >> tpr_log;
    // four rows per thread where that leaves every SM its CTAs
    if (ceil_div(o.rows, per * 4) * slabs >= kSms * 8)
        k_lookup<T, E, 4><<<dim3((unsigned)ceil_div(o.rows, per * 4), slabs), 256, 0, s>>>((const T *)t.data, t.ld, (int32_t)t.rows, ids, o.rows, vecs, tpr_log, scale, (T *)o.data, o.ld, status);
    else
        k_lookup<T, E, 1><<<dim3((unsigned)ceil_div(o.rows, per), slabs), 256, 0, s>>>((const T *)t.data, t.ld, (int32_t)t.rows, ids, o.rows, vecs, tpr_log, scale, (T *)o.data, o.ld, status);
    return cudaGetLastError();
}

template <typename T, int E>
cudaError_t sum_by_id(Sums sm, const chicle_dense_t &g, const chicle_dense_t &t, const ZeroJob &zero, cudaStream_t s)
{
    sm.vecs = (int)(g.cols / E);
    sm.tpr_log = std::min(8, log2_up(sm.vecs));
    sm.slabs = (int)ceil_div(sm.vecs, 1 << sm.tpr_log);
    sm.sum_blocks = ceil_div(sm.windows, 256 >> sm.tpr_log) * sm.slabs;
    k_sum_by_id<T, E><<<(unsigned)(sm.sum_blocks + zero.blocks()), 256, 0, s>>>(sm, (const T *)g.data, g.ld, (T *)t.data, t.ld, zero);
    // (wide rows: a run's sums are the work of a CTA, and one CTA does them one behind the other)
    sm.join_windows = sm.tpr_log == 8 ? 1 : 8;
    cudaError_t e = cudaGetLastError();
    if (e == cudaSuccess && sm.windows > 1) {
        k_join_windows<T, E><<<dim3((unsigned)ceil_div(sm.windows, sm.join_windows), (unsigned)sm.slabs), 256, 0, s>>>(sm, (T *)t.data, t.ld);
        e = cudaGetLastError();
    }
    return e;
}

// Calls f(type's tag, elements per access) for the access width.
template <typename T, typename F> cudaError_t by_width(int e, F f)
{
    constexpr int kMost = 16 / (int)sizeof(T);
    if constexpr (kMost == 8)
        if (e >= 8) return f(T{}, std::integral_constant<int, 8>{});
    if (e >= 4) return f(T{}, std::integral_constant<int, 4>{});
    if (e >= 2) return f(T{}, std::integral_constant<int, 2>{});
    return f(T{}, std::integral_constant<int, 1>{});
}
template <typename F> cudaError_t by_type(chicle_dtype_t t, int e, F f)
{
    if (t == CHICLE_F32) return by_width<float>(e, f);
    if (t == CHICLE_BF16) return by_width<__nv_bfloat16>(e, f);
    return by_width<__half>(e, f);
}

const char *check_pair(const chicle_dense_t *a, const chicle_dense_t *b, float scale)
{
    if (const char *m = check_dense(a)) return m;
    if (const char *m = check_dense(b)) return m;
    if (a->type != b->type) return "both matrices must have one element type";
    if (a->cols != b->cols) return "both matrices must have the same number of columns";
    if (overlapping(*a, *b)) return "the matrices must not overlap";
    if (!std::isfinite(scale)) return "scale must be finite";
    return nullptr;
}

} // namespace
} // namespace chicle

using namespace chicle;

extern "C" chicle_status_t chicle_embedding(int device, void *cuda_stream, const chicle_dense_t *table, const int32_t *dev_ids, float scale,
                                            const chicle_dense_t *out, uint32_t *dev_status, char *host_errbuf, size_t errbuf_len)
{
    const CallError err{host_errbuf, errbuf_len};
    if (const char *m = check_pair(table, out, scale)) return err(CHICLE_ERR_INVALID_ARG, m);
    if (out->rows == 0) return CHICLE_OK;
    if (!dev_ids) return err(CHICLE_ERR_INVALID_ARG, "ids must be a non-NULL device pointer");
    const DeviceGuard guard(device);
    if (!guard.ok()) return err(CHICLE_ERR_CUDA, guard.message());
    const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    const cudaError_t e = by_type(table->type, vector_elements(*table, *out), [&](auto tag, auto width) {
        return lookup<decltype(tag), decltype(width)::value>(*table, dev_ids, scale, *out, dev_status, s);
    });
    return e == cudaSuccess ? CHICLE_OK : err.cuda(e);
}

extern "C" chicle_status_t chicle_embedding_grad_workspace(int64_t n, int64_t rows, int64_t cols, size_t *host_bytes)
{
    if (!host_bytes || n < 0 || rows < 0 || cols < 1 || n > INT32_MAX - 4096 || rows > INT32_MAX - 4096 || cols > 65536)
        return CHICLE_ERR_INVALID_ARG;
    *host_bytes = n ? make_plan(n, rows, cols).bytes : 0;
    return CHICLE_OK;
}

extern "C" chicle_status_t chicle_embedding_grad(int device, void *cuda_stream, const int32_t *dev_ids, const chicle_dense_t *grad, float scale,
                                                 int accumulate, const chicle_dense_t *dtable, void *dev_workspace, size_t workspace_bytes,
                                                 uint32_t *dev_status, char *host_errbuf, size_t errbuf_len)
{
    const CallError err{host_errbuf, errbuf_len};
    if (const char *m = check_pair(grad, dtable, scale)) return err(CHICLE_ERR_INVALID_ARG, m);
    const int64_t n = grad->rows;
    if (n > 0 && !dev_ids) return err(CHICLE_ERR_INVALID_ARG, "ids must be a non-NULL device pointer");
    const IdPlan p = n ? make_plan(n, dtable->rows, grad->cols) : IdPlan{};
    if (n > 0)
        if (const char *m = check_workspace(dev_workspace, workspace_bytes, p.bytes)) return err(CHICLE_ERR_INVALID_ARG, m);
    const DeviceGuard guard(device);
    if (!guard.ok()) return err(CHICLE_ERR_CUDA, guard.message());
    const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t e = cudaSuccess;
    if (n == 0) {
        const size_t es = (size_t)element_size(dtable->type);
        if (!accumulate && dtable->rows > 0)
            e = cudaMemset2DAsync(dtable->data, (size_t)dtable->ld * es, 0, (size_t)dtable->cols * es, (size_t)dtable->rows, s);
        return e == cudaSuccess ? CHICLE_OK : err.cuda(e);
    }
    uint8_t *ws = static_cast<uint8_t *>(dev_workspace);
    int which = 0;
    ZeroJob zero{};
    zero.base = static_cast<uint8_t *>(dtable->data);
    zero.row_bytes = (int32_t)(dtable->cols * element_size(dtable->type));
    zero.pitch = dtable->ld * element_size(dtable->type);
    zero.width = vector_elements(*dtable, *dtable) * element_size(dtable->type);
    zero.per = (int32_t)std::max<int64_t>(1, kZeroBytes / zero.row_bytes);
    zero.v1 = accumulate ? 0 : dtable->rows;
    e = sort_ids(p, dev_ids, n, (int32_t)dtable->rows, ws, dev_status, s, &which, &zero);
    if (e == cudaSuccess) {
        Sums sm{};
        sm.keys = reinterpret_cast<int32_t *>(ws + p.keys[which]);
        sm.order = reinterpret_cast<int32_t *>(ws + p.order[which]);
        sm.n = n, sm.rows = (int32_t)dtable->rows, sm.d = (int32_t)grad->cols;
        sm.window = p.window, sm.windows = p.windows;
        sm.scale = scale, sm.accumulate = accumulate;
        sm.partial = reinterpret_cast<float *>(ws + p.partial);
        e = by_type(grad->type, vector_elements(*grad, *dtable), [&](auto tag, auto width) {
            return sum_by_id<decltype(tag), decltype(width)::value>(sm, *grad, *dtable, zero, s);
        });
    }
    return e == cudaSuccess ? CHICLE_OK : err.cuda(e);
}
