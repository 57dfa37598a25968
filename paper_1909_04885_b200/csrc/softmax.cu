// Softmax cross entropy of a linear map to many classes, and its gradients (chicle_softmax_loss,
// chicle_softmax_loss_grad): the multi-class sibling of the logistic loss.
//
//   l_iv = x_i . w_v        lse_i = log sum_v exp(l_iv)        loss_i = lse_i - l_{i, y_i}
//   p_iv = g_i (exp(l_iv - lse_i) - [v = y_i])                 dX = P W,  dW = P^T X
//
// The logits are never held as a whole. The loss alone keeps, per row and block of classes (a warp's columns of a tile), the
// largest logit and the sum of exponentials relative to it; a second kernel joins them. For the gradients the rows are
// taken in pieces of about two gigabytes of 16-bit values: the product's epilogue writes exp(l - m) of its tile (m: the
// largest of the row in the block) as fp16, an elementwise pass turns the piece into P in place, and two products
// take dX and the piece's share of dW from it. So the logits are computed once: 6 n V d operations, against 8 where they
// are computed again for the gradient, for 6 bytes of traffic per logit (at d = 4096 a third of the products' time against a
// twentieth).
//
// Rounding: logits, sums and gradients in fp32. The exponentials are held times 2^15, so that 2^-29 of the block's
// largest still has all its bits (single precision: in fp32). P is rounded once to the operands' type (fp16: scaled so that the
// largest weight comes to 2^14 and more; single precision: to two fp16 planes, tensor_core.cuh), and the entry of the label
// comes from expm1(-loss), not from a difference. That entry's rounding is most of what a gradient is off by beside the
// rounding of the result: together 1.41 times the result's alone, more where one row decides. (Exponentials in 16 bits with half
// of fp16's step, no sign bit, changed nothing.)
#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdlib>

#include "operators.cuh"
#include "tensor_core.cuh"

namespace chicle {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kStoreScale = 32768.f; // fp16 exponentials are held times 2^15

// Two floats in one register pair: sm_100 adds and multiplies them in one instruction.
__device__ __forceinline__ uint64_t pair_of(float lo, float hi) { return (uint64_t)__float_as_uint(lo) | ((uint64_t)__float_as_uint(hi) << 32); }
__device__ __forceinline__ float low_of(uint64_t p) { return __uint_as_float((uint32_t)p); }
__device__ __forceinline__ float high_of(uint64_t p) { return __uint_as_float((uint32_t)(p >> 32)); }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// 2^x, off by 2^-22 of itself; what would be subnormal is 0.
__device__ __forceinline__ float exp2_of(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Powers of two in device memory: of P (its largest weight comes to [2^14, 2^15)), X and W (their largest elements do), and their
// inverses. P is scaled wherever it is held in fp16, X and W in single precision.
enum { kLift, kInvLift, kLiftX, kInvX, kLiftW, kInvW, kScales };

// v times both powers of two, one after the other, the smaller one first: their product may leave fp32's range where the result
// does not (operands of 1e-20 each, or rows of zeros beside rows of 1e25).
struct TwoScales {
    float small, large;
    __device__ __forceinline__ TwoScales(float a, float b) : small(fminf(a, b)), large(fmaxf(a, b)) {}
    __device__ __forceinline__ float operator()(float v) const { return (v * small) * large; }
};

// ---- epilogues ---------------------------------------------------------------------------------------------

// Reduces a tile of logits to (largest, sum of exponentials) per row and N classes, keeps the label's logit, and
// writes the exponentials for the gradients: StoreT NoStore (loss alone), half, or float (single precision).
template <typename StoreT> struct LogitsEpilogue {
    static constexpr int kStep = 0;
    const int32_t *labels; // rows of this piece
    float2 *stats;         // [block of N classes][rows]
    float *label_logit;    // [rows]
    StoreT *store;         // [rows][ld]
    int64_t ld;
    const float *scales;   // single precision: the operands' scales (Scales); else null

    template <int N>
    __device__ __forceinline__ void finish(const tc::Shape &s, const tc::Tile &tl, int row0, int lane, int c0, int end, bool ok,
                                           uint32_t (&r)[N], uint8_t *patch) const
    {
        const int row = row0 + lane;
        const bool live = row < s.m;
        const TwoScales logit(scales ? scales[kInvX] : 1.f, scales ? scales[kInvW] : 1.f); // of an accumulator
        const int lab = live ? labels[row] - c0 : -1; // (a negative label is in front of every block)
        if (c0 + N > end) {
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (c0 + j >= end) r[j] = 0xff800000u; // -inf
        }
        float t[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int j = 0; j < N; ++j) t[j & 3] = fmaxf(t[j & 3], __uint_as_float(r[j]));
        const float top = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
#pragma unroll
        for (int g = 0; g < N; g += 32)
            if ((uint32_t)(lab - g) < 32u && c0 + lab < end) { // one of 32 registers by the bits of its number
                uint32_t q[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) q[j] = (lab & 16) ? r[g + 16 + j] : r[g + j];
#pragma unroll
                for (int w = 8; w > 0; w >>= 1)
#pragma unroll
                    for (int j = 0; j < w; ++j) q[j] = (lab & w) ? q[w + j] : q[j];
                label_logit[row] = logit(__uint_as_float(q[0]));
            }
        // (a block without a logit above -inf: relative to 0, so that its exponentials are 0 and not NaN)
        const float ref = !ok ? NAN : top == -INFINITY ? 0.f : top;
        uint64_t sum[2] = {0, 0}; // pairs of floats
        // (differences are -inf, 0 or of 2^-48 to 2^48: kept within fp32's range, the factor leaves of them what the true one
        // does, and 0 and -inf as they are)
        const float factor = fminf(fmaxf(logit(kLog2e), 0x1p-126f), 0x1p126f);
        const uint64_t back = pair_of(-ref, -ref), to_log2 = pair_of(factor, factor);
        constexpr int kWidth = sizeof(StoreT) >= 2 ? 64 / (int)sizeof(StoreT) : N; // columns of a patch
        constexpr int kPer = sizeof(StoreT) >= 2 ? 16 / (int)sizeof(StoreT) : 8;    // and of a piece
#pragma unroll
        for (int g = 0; g < N; g += kWidth) {
            __syncwarp();
#pragma unroll
            for (int c = 0; c < kWidth; c += kPer) {
                float e[kPer];
#pragma unroll
                for (int j = 0; j < kPer; j += 2) {
                    // (the difference first: it is exact where it matters, the logarithm's product is not)
                    const uint64_t z = mul2(add2(pair_of(__uint_as_float(r[g + c + j]), __uint_as_float(r[g + c + j + 1])), back), to_log2);
                    e[j] = exp2_of(low_of(z));
                    e[j + 1] = exp2_of(high_of(z));
                    sum[(j >> 1) & 1] = add2(sum[(j >> 1) & 1], pair_of(e[j], e[j + 1]));
                }
                if constexpr (sizeof(StoreT) == 2) {
                    uint4 q;
                    __half2 *h = reinterpret_cast<__half2 *>(&q);
#pragma unroll
                    for (int i = 0; i < 4; ++i) h[i] = __floats2half2_rn(e[2 * i] * kStoreScale, e[2 * i + 1] * kStoreScale);
                    *tc::patch_at(patch, lane, c / kPer) = q;
                } else if constexpr (sizeof(StoreT) == 4) {
                    *reinterpret_cast<float4 *>(tc::patch_at(patch, lane, c / kPer)) = make_float4(e[0], e[1], e[2], e[3]);
                }
            }
            if constexpr (sizeof(StoreT) >= 2) {
                __syncwarp();
                const int piece = lane & 3, col = c0 + g + piece * kPer;
                StoreT *dst = store + (int64_t)(row0 + (lane >> 2)) * ld + col;
#pragma unroll
                for (int i = 0; i < 4; ++i) { // (ld: a multiple of 64, what lies behind the last class is not read)
                    const int rr = 8 * i + (lane >> 2);
                    if (row0 + rr < s.m && col < end) *reinterpret_cast<uint4 *>(dst + (int64_t)(8 * i) * ld) = *tc::patch_at(patch, rr, piece);
                }
            }
        }
        // NaN: fmaxf passes over it, the sum does not
        if (live && c0 < end) stats[(int64_t)(tl.n * s.parts + (c0 - tl.n * s.cols) / N) * s.m + row] = make_float2(logit(top), (low_of(sum[0]) + low_of(sum[1])) + (high_of(sum[0]) + high_of(sum[1])));
    }
};

struct NoStore {
    char c;
};

__device__ __forceinline__ TwoScales scales_of(const float *a, const float *b) { return TwoScales(a ? *a : 1.f, b ? *b : 1.f); }

template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// Where a tile of a gradient goes. With splits: to `partial`, one plane per split. Else sum = (add ? *add : 0) + tile; to
// `keep` (fp32, for the pieces that follow) or to `out`.
template <typename OutT> struct GradEpilogue {
    static constexpr int kStep = 32; // (not used where sums come in chunks)
    OutT *out;
    int64_t ld;
    float *partial;          // [split][m][n]
    const float *add;        // [m][n], or null
    float *keep;             // [m][n], or null
    const float *scale, *scale_b; // device factors of the result, or null
    const int32_t *labels;   // rows without a label come out 0 whatever the other operand holds; or null
    int32_t classes;

    template <int N>
    __device__ __forceinline__ void finish(const tc::Shape &s, const tc::Tile &tl, int row0, int lane, int c0, int end, bool ok,
                                           uint32_t (&r)[N], uint8_t *patch) const
    {
        if (!ok) {
#pragma unroll
            for (int j = 0; j < N; ++j) r[j] = 0x7fffffffu;
        }
        const bool whole = partial || keep;
        const TwoScales f = whole ? TwoScales(1.f, 1.f) : scales_of(scale, scale_b);
        const uint32_t zeros = __ballot_sync(0xffffffffu, labels && row0 + lane < s.m && (uint32_t)labels[row0 + lane] >= (uint32_t)classes);
        float *dst32 = partial ? partial + (int64_t)tl.split * s.m * s.n : keep;
        const float *src = partial ? nullptr : add;
        if constexpr (sizeof(OutT) == 2 && N == 32) {
            // straight to the result: rounded first, so that a warp's store covers 8 rows of 64 bytes
            if (!whole && !src && ((reinterpret_cast<uintptr_t>(out) | (uintptr_t)(ld * 2)) & 15) == 0) {
                const bool zero = (zeros >> lane) & 1u;
                __syncwarp();
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    alignas(16) OutT q[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) q[j] = from_float<OutT>(zero ? 0.f : f(__uint_as_float(r[8 * c + j])));
                    *tc::patch_at(patch, lane, c) = *reinterpret_cast<const uint4 *>(q);
                }
                __syncwarp();
                const int col = c0 + 8 * (lane & 3);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int rr = 8 * i + (lane >> 2), row = row0 + rr;
                    if (row >= s.m || col >= end) continue;
                    alignas(16) OutT q[8];
                    *reinterpret_cast<uint4 *>(q) = *tc::patch_at(patch, rr, lane & 3);
                    OutT *dst = out + (int64_t)row * ld + col;
                    if (col + 8 <= end) {
                        *reinterpret_cast<uint4 *>(dst) = *reinterpret_cast<const uint4 *>(q);
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            if (col + j < end) dst[j] = q[j];
                    }
                }
                return;
            }
        }
        const bool quads = (s.n & 3) == 0; // fp32 rows of n: 16-byte pieces
        const bool quads_out = ((reinterpret_cast<uintptr_t>(out) | (uintptr_t)(ld * sizeof(OutT))) & (4 * sizeof(OutT) - 1)) == 0;
#pragma unroll
        for (int g = 0; g < N; g += 16) {
            if (c0 + g >= end) break;
            __syncwarp();
#pragma unroll
            for (int c = 0; c < 4; ++c) *tc::patch_at(patch, lane, c) = make_uint4(r[g + 4 * c], r[g + 4 * c + 1], r[g + 4 * c + 2], r[g + 4 * c + 3]);
            __syncwarp();
            const int col = c0 + g + 4 * (lane & 3);
#pragma unroll 2
            for (int i = 0; i < 4; ++i) {
                const int rr = 8 * i + (lane >> 2), row = row0 + rr;
                if (row >= s.m || col >= end) continue;
                float4 v = *reinterpret_cast<const float4 *>(tc::patch_at(patch, rr, lane & 3));
                if ((zeros >> rr) & 1u) v = make_float4(0.f, 0.f, 0.f, 0.f);
                const int64_t at = (int64_t)row * s.n + col;
                if (col + 4 <= s.n && (whole ? quads : quads_out) && (!src || quads)) {
                    if (src) {
                        const float4 o = *reinterpret_cast<const float4 *>(src + at);
                        v.x += o.x, v.y += o.y, v.z += o.z, v.w += o.w;
                    }
                    if (whole) {
                        *reinterpret_cast<float4 *>(dst32 + at) = v;
                    } else {
                        struct alignas(4 * sizeof(OutT)) {
                            OutT v[4];
                        } q{{from_float<OutT>(f(v.x)), from_float<OutT>(f(v.y)), from_float<OutT>(f(v.z)), from_float<OutT>(f(v.w))}};
                        *reinterpret_cast<decltype(q) *>(out + (int64_t)row * ld + col) = q;
                    }
                } else {
                    const float w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (col + j < s.n) {
                            const float x = w[j] + (src ? src[at + j] : 0.f);
                            if (whole) dst32[at + j] = x;
                            else out[(int64_t)row * ld + col + j] = from_float<OutT>(f(x));
                        }
                }
            }
        }
    }
};

// Joins the splits' planes in ascending order, V elements per thread; add, keep, out as above.
template <typename OutT, int V>
__global__ void __launch_bounds__(256) k_join_splits(const float *__restrict__ partial, int splits, int64_t m, int32_t n,
                                                     const float *add, float *keep, OutT *out, int64_t ld, const float *scale,
                                                     const float *scale_b, const int32_t *labels, int32_t classes)
{
    struct alignas(4 * V) Quad {
        float v[V];
    };
    const int64_t all = m * n / V;
    const TwoScales f = scales_of(scale, scale_b);
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < all; i += (int64_t)gridDim.x * blockDim.x) {
        Quad v{};
#pragma unroll 8
        for (int k = 0; k < splits; ++k) {
            const Quad o = reinterpret_cast<const Quad *>(partial)[(int64_t)k * all + i];
#pragma unroll
            for (int j = 0; j < V; ++j) v.v[j] += o.v[j];
        }
        const int64_t row = i * V / n;
        if (labels && (uint32_t)labels[row] >= (uint32_t)classes) v = Quad{};
        if (add) {
            const Quad o = reinterpret_cast<const Quad *>(add)[i];
#pragma unroll
            for (int j = 0; j < V; ++j) v.v[j] += o.v[j];
        }
        if (keep) {
            reinterpret_cast<Quad *>(keep)[i] = v;
        } else {
            OutT *dst = out + row * ld + (i * V - row * n);
#pragma unroll
            for (int j = 0; j < V; ++j) dst[j] = from_float<OutT>(f(v.v[j]));
        }
    }
}

// ---- small kernels -----------------------------------------------------------------------------------------

// (top, sum) of one more block. Equal ones, infinite ones too, without a difference.
__device__ __forceinline__ void join_into(float &top, float &sum, float2 o)
{
    const float m = fmaxf(top, o.x);
    sum = (top == m ? sum : sum * exp2f((top - m) * kLog2e)) + (o.x == m ? o.y : o.y * exp2f((o.x - m) * kLog2e));
    top = m;
}

// loss and lse of a row, relative to the largest logit: lse and the label's logit would lose the bits that they share.
__device__ __forceinline__ float2 loss_of(float top, float sum, bool has, float label_logit)
{
    return has ? make_float2((top - label_logit) + logf(sum), top + logf(sum)) : make_float2(0.f, 0.f);
}

// Joins the blocks of classes of R rows per CTA; threads of one row run down its blocks, fixed order.
template <int R>
__global__ void __launch_bounds__(512) k_join_blocks(const float2 *__restrict__ stats, int blocks, int32_t n,
                                                     const int32_t *__restrict__ labels, int32_t classes,
                                                     const float *__restrict__ label_logit, float *__restrict__ loss,
                                                     float *__restrict__ lse, float2 *__restrict__ norm, uint32_t *status)
{
    constexpr int kT = 512 / R;
    __shared__ float s_top[kT][R], s_sum[kT][R];
    const int r = threadIdx.x % R, t = threadIdx.x / R;
    const int row = blockIdx.x * R + r;
    float top = -INFINITY, sum = 0.f;
    if (row < n) {
#pragma unroll 4
        for (int b = t; b < blocks; b += kT) join_into(top, sum, stats[(int64_t)b * n + row]);
    }
    s_top[t][r] = top;
    s_sum[t][r] = sum;
    __syncthreads();
    for (int w = kT / 2; w > 0; w >>= 1) {
        if (t < w) {
            join_into(top, sum, make_float2(s_top[t + w][r], s_sum[t + w][r]));
            s_top[t][r] = top;
            s_sum[t][r] = sum;
        }
        __syncthreads();
    }
    if (t == 0 && row < n) {
        const int32_t y = labels[row];
        const bool has = (uint32_t)y < (uint32_t)classes;
        const float2 l = loss_of(top, sum, has, has ? label_logit[row] : 0.f);
        loss[row] = l.x;
        lse[row] = l.y;
        if (norm) norm[row] = make_float2(top, 1.f / sum);
        if (y >= classes && status) atomicOr(status, (uint32_t)ST_BAD_INDEX);
    }
}

// Exponentials to P, kSteps times 8 classes of a row per thread: in place for 16-bit operands, from fp32 to two fp16 planes for
// single precision. Bound by memory: 8192 x 131072 in 640 us, 6.7 TB/s (with one step 850; 10000 x 1000: one step 13 us, four
// 26, most of whose threads have nothing to do).
// kJoin: a CTA has a whole row, and joins its blocks of classes itself (k_join_blocks): one launch less where launches count.
// kPlanes: of P.
template <typename PT, bool kWide, int kPlanes, int kSteps, bool kJoin>
__global__ void __launch_bounds__(256)
k_probabilities(const void *store, PT *p, int64_t ld, int64_t plane, int32_t n, int32_t classes, const float2 *__restrict__ stats,
                float2 *norm, float *loss, const int32_t *__restrict__ labels, const float *__restrict__ weights, float scale,
                const float *__restrict__ lift, int block_log, int blocks, const float *__restrict__ label_logit, float *lse, uint32_t *status)
{
    const int row = blockIdx.y;
    const int c0 = (blockIdx.x * kSteps * 256 + threadIdx.x) * 8;
    const int32_t y = labels[row];
    const bool has = (uint32_t)y < (uint32_t)classes;
    uint4 in[kSteps][kWide ? 2 : 1];
    float ref[kSteps];
    if (has) {
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const int c = c0 + k * 2048;
            if (c >= classes) break;
            if constexpr (kWide) {
                const uint4 *src = reinterpret_cast<const uint4 *>(static_cast<const float *>(store) + (int64_t)row * ld + c);
                in[k][0] = src[0], in[k][1] = src[1];
            } else {
                in[k][0] = *reinterpret_cast<const uint4 *>(static_cast<const __half *>(store) + (int64_t)row * ld + c);
            }
            ref[k] = stats[(int64_t)(c >> block_log) * n + row].x;
        }
    }
    float g = weights ? weights[row] * scale : scale;
    if (lift) g *= *lift;
    float2 of;   // relative to the largest logit: lse has lost the bits that the two share
    float of_label;
    if constexpr (kJoin) {
        // every warp joins the row's blocks for itself, 32 at a time
        float top = -INFINITY, sum = 0.f;
        for (int b = threadIdx.x & 31; b < blocks; b += 32) join_into(top, sum, stats[(int64_t)b * n + row]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
            join_into(top, sum, make_float2(__shfl_xor_sync(0xffffffffu, top, o), __shfl_xor_sync(0xffffffffu, sum, o)));
        top = __shfl_sync(0xffffffffu, top, 0); // (the lanes' sums may differ in the last bit)
        sum = __shfl_sync(0xffffffffu, sum, 0);
        of = make_float2(top, 1.f / sum);
        const float2 l = loss_of(top, sum, has, has ? label_logit[row] : 0.f);
        of_label = l.x;
        if (threadIdx.x == 0) {
            loss[row] = l.x;
            lse[row] = l.y;
            if (y >= classes && status) atomicOr(status, (uint32_t)ST_BAD_INDEX);
        }
    } else {
        of = norm[row];
        of_label = loss[row];
    }
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
        const int c = c0 + k * 2048;
        if (c >= classes) break;
        float v[8];
        if (has) {
            const float f = exp2f((ref[k] - of.x) * kLog2e) * of.y * (kWide ? 1.f : 1.f / kStoreScale) * g;
            if constexpr (kWide) {
                const float *e = reinterpret_cast<const float *>(in[k]);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = e[j] * f;
            } else {
                const __half2 *h = reinterpret_cast<const __half2 *>(in[k]);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 t = __half22float2(h[j]);
                    v[2 * j] = t.x * f;
                    v[2 * j + 1] = t.y * f;
                }
            }
            if (y >= c && y < c + 8) {
                const float at = g * expm1f(-of_label);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (y - c == j) v[j] = at;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = 0.f;
        }
        alignas(16) PT q[8];
#pragma unroll
        for (int w = 0; w < kPlanes; ++w) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                q[j] = from_float<PT>(v[j]);
                v[j] -= (float)q[j];
            }
            *reinterpret_cast<uint4 *>(p + w * plane + (int64_t)row * ld + c) = *reinterpret_cast<const uint4 *>(q);
        }
    }
}

// The power of two that takes a largest magnitude to [2^14, 2^15), and its inverse.
__device__ __forceinline__ float2 scale_of(float top)
{
    int e = 15;
    if (top > 0.f) frexpf(top, &e); // top in [2^(e-1), 2^e)
    e = max(-120, min(120, 15 - e));
    return make_float2(ldexpf(1.f, e), ldexpf(1.f, -e));
}

// The largest of the CTA's 256 values.
__device__ __forceinline__ float block_largest(float top)
{
    __shared__ float s[8];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, s[i]);
    return top;
}

// Largest finite magnitudes, one word per CTA: kMaxBlocks CTAs for X (rows with a label), as many for W and for the weights
// times the scale (of rows with a label), of these groups the ones from `first` on.
constexpr int kMaxBlocks = 148 * 4;

__global__ void __launch_bounds__(256) k_largest(const float *__restrict__ x, int64_t ld_x, int64_t n, const int32_t *__restrict__ labels,
                                                 int32_t classes, const float *__restrict__ w, int64_t ld_w, int32_t d,
                                                 const float *__restrict__ weights, float scale, int first_group, float *__restrict__ largest)
{
    const int group = first_group + (int)blockIdx.x / kMaxBlocks, block = (int)blockIdx.x % kMaxBlocks;
    const int64_t first = (int64_t)block * 256 + threadIdx.x, step = (int64_t)kMaxBlocks * 256;
    float top = 0.f;
    auto take = [&](float v) {
        v = fabsf(v);
        if (v < INFINITY) top = fmaxf(top, v);
    };
    const bool of_x = group == 0;
    const float *src = of_x ? x : w;
    const int64_t ld = of_x ? ld_x : ld_w, rows = of_x ? n : classes;
    const bool quads = (reinterpret_cast<uintptr_t>(src) & 15) == 0 && (ld & 3) == 0 && (d & 3) == 0;
    if (group == 2) {
#pragma unroll 4
        for (int64_t i = first; i < n; i += step)
            if ((uint32_t)labels[i] < (uint32_t)classes) take(weights[i] * scale);
    } else if (!of_x && quads && ld == d) { // no rows to be told apart: 134 MB in 24 us instead of 47
        const float4 *flat = reinterpret_cast<const float4 *>(src);
        const int64_t all = rows * (d / 4);
#pragma unroll 8
        for (int64_t i = first; i < all; i += step) {
            const float4 v = flat[i];
            take(v.x), take(v.y), take(v.z), take(v.w);
        }
    } else {
        const int per = quads ? d / 4 : d;
        const int64_t all = rows * per;
#pragma unroll 4
        for (int64_t i = first; i < all; i += step) {
            const int64_t row = i / per;
            const int c = (int)(i - row * per);
            if (of_x && (uint32_t)labels[row] >= (uint32_t)classes) continue;
            if (quads) {
                const float4 v = *reinterpret_cast<const float4 *>(src + row * ld + 4 * c);
                take(v.x), take(v.y), take(v.z), take(v.w);
            } else {
                take(src[row * ld + c]);
            }
        }
    }
    top = block_largest(top);
    if (threadIdx.x == 0) largest[group * kMaxBlocks + block] = top;
}

// One of the matrices that k_pack lays out. `lift`: words of Scales that its scale goes to (single precision).
struct Packed {
    const void *src;
    int64_t ld, rows, plane;
    void *dst;
    const int32_t *labels; // rows without a label become zeros; or null
    unsigned blocks;       // CTAs for it (0: it is used as it is)
    int lift;
};

// Rows in a layout that the bulk copies take (whole lines), single precision scaled and as two fp16 planes. The first CTA of
// a launch also finds the scale of P where there is one: from the weights themselves (of X's rows with a label) while they are
// few.
constexpr int64_t kFewWeights = 4096;

template <typename T, typename P>
__global__ void __launch_bounds__(256) k_pack(const Packed x, const Packed w, int32_t d, int64_t pitch, int32_t classes,
                                              const float *__restrict__ largest, const float *__restrict__ weights, int64_t n, float scale,
                                              float *__restrict__ scales)
{
    const bool of_x = blockIdx.x < x.blocks;
    const Packed &m = of_x ? x : w;
    const unsigned block = of_x ? blockIdx.x : blockIdx.x - x.blocks;
    if (scales && blockIdx.x == 0) {
        float top = 0.f;
        if (weights && n > kFewWeights) {
            for (int i = threadIdx.x; i < kMaxBlocks; i += 256) top = fmaxf(top, largest[2 * kMaxBlocks + i]);
        } else if (weights) {
#pragma unroll 16
            for (int64_t i = threadIdx.x; i < n; i += 256) {
                const float v = fabsf(weights[i] * scale);
                if ((uint32_t)x.labels[i] < (uint32_t)classes && v < INFINITY) top = fmaxf(top, v);
            }
        } else {
            top = fabsf(scale);
        }
        const float2 f = scale_of(block_largest(top));
        if (threadIdx.x == 0) scales[kLift] = f.x, scales[kInvLift] = f.y;
    }
    float up = 1.f;
    if constexpr (sizeof(T) == 4) {
        float top = 0.f;
        for (int i = threadIdx.x; i < kMaxBlocks; i += 256) top = fmaxf(top, largest[(of_x ? 0 : kMaxBlocks) + i]);
        const float2 f = scale_of(block_largest(top));
        up = f.x;
        if (block == 0 && threadIdx.x == 0) scales[m.lift] = f.x, scales[m.lift + 1] = f.y;
    }
    const int per = (int)(pitch / 8);
    const int64_t all = m.rows * per;
    for (int64_t i = (int64_t)block * 256 + threadIdx.x; i < all; i += (int64_t)m.blocks * 256) {
        const int64_t row = i / per;
        const int c = (int)(i - row * per) * 8;
        const bool has = !m.labels || (uint32_t)m.labels[row] < (uint32_t)classes;
        const T *from = static_cast<const T *>(m.src) + row * m.ld + c;
        P *to = static_cast<P *>(m.dst) + row * pitch + c;
        alignas(16) T in[8];
        if (has && c + 8 <= d && (reinterpret_cast<uintptr_t>(from) & 15) == 0) {
#pragma unroll
            for (int j = 0; j < (int)(8 * sizeof(T) / 16); ++j)
                reinterpret_cast<uint4 *>(in)[j] = reinterpret_cast<const uint4 *>(from)[j];
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) in[j] = has && c + j < d ? from[j] : from_float<T>(0.f);
        }
        if constexpr (sizeof(T) == 4) {
            alignas(16) P hi[8], lo[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float v = in[j] * up;
                hi[j] = from_float<P>(v);
                lo[j] = from_float<P>(v - (float)hi[j]);
            }
            *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(hi);
            *reinterpret_cast<uint4 *>(to + m.plane) = *reinterpret_cast<const uint4 *>(lo);
        } else {
            *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(in);
        }
    }
}

// ---- host --------------------------------------------------------------------------------------------------

using EncodeFn = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                              const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeFn encode_fn()
{
    static const EncodeFn fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q{};
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) {
            (void)cudaGetLastError();
            p = nullptr;
        }
        return reinterpret_cast<EncodeFn>(p);
    }();
    return fn;
}

// A 16-bit matrix on the device: `planes` of rows x cols, rows `pitch` elements apart (a multiple of 8).
struct Operand {
    const void *data = nullptr;
    int64_t rows = 0, cols = 0, pitch = 0, plane = 0;
    int planes = 1;
};

bool make_map(CUtensorMap *map, const Operand &o, bool half, int box_cols, int box_rows)
{
    const EncodeFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)o.cols, (cuuint64_t)o.rows, (cuuint64_t)o.planes};
    const cuuint64_t strides[2] = {(cuuint64_t)o.pitch * 2, (cuuint64_t)(o.planes > 1 ? o.plane : o.pitch) * 2};
    const cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1}, step[3] = {1, 1, 1};
    return fn(map, half ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(o.data), dims,
              strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Test aid (read once per process): from this tile on the operands of the products are not fetched, and waits are short. -1: none.
int64_t dropped_copies()
{
    static const int64_t drop = [] {
        const char *env = getenv("CHICLE_TEST_DROP_COPIES");
        return env ? std::max<int64_t>(0, atoll(env)) : -1;
    }();
    return drop;
}
constexpr int64_t kTestClocks = 20000000; // 10 to 20 ms

template <int CG, int BN, bool AMN, bool BMN, bool kChunked, class Epi>
cudaError_t launch_product(const Operand &a, const Operand &b, tc::Shape s, int cols, const Epi &epi, cudaStream_t stream)
{
    using L = tc::Layout<CG, BN>;
    CUtensorMap ma, mb;
    s.a_rows = AMN || s.m >= L::kBM ? L::kBM : (s.m + 7) / 8 * 8; // (what lies behind them in shared memory is not of C)
    if (!make_map(&ma, a, s.half, 64, AMN ? 64 : s.a_rows) || !make_map(&mb, b, s.half, 64, BMN ? 64 : cols / CG)) return cudaErrorInvalidValue;
    s.m_tiles = (int32_t)ceil_div(s.m, CG * L::kBM);
    s.n_tiles = (int32_t)ceil_div(s.n, cols);
    s.cols = cols;
    auto *kernel = tc::k_product<CG, BN, AMN, BMN, kChunked, Epi>;
    s.parts = tc::kEpiWarps / 4;
    // (once per device and process: 0.5 us a call)
    static std::atomic<uint64_t> allowed{0};
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    const uint64_t bit = (uint64_t)1 << (device & 63);
    if (e == cudaSuccess && !(allowed.load(std::memory_order_relaxed) & bit)) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)L::kSmem);
        if (e == cudaSuccess) allowed.fetch_or(bit, std::memory_order_relaxed);
    }
    if (e != cudaSuccess) return e;
    const int64_t tiles = (int64_t)s.m_tiles * s.n_tiles * s.splits;
    const int64_t drop = dropped_copies();
    s.fetched = drop < 0 ? tiles : std::min(tiles, drop);
    s.limit = drop < 0 ? tc::kWaitClocks : kTestClocks;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(CG * (tiles < kSms / CG ? tiles : kSms / CG)));
    cfg.blockDim = dim3(tc::kThreads);
    cfg.dynamicSmemBytes = L::kSmem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {CG, 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, ma, mb, s, epi);
}

// Which tiles. Pairs of CTAs (256 rows) wherever C has more rows than one CTA takes: each fetches half of B (single CTAs: 23.8 ms for
// 8192 x 131072 x 4096 with gradients, pairs 23.5; 1777 x 50001 x 1000: 823 and 670 us).
bool pairs_of_ctas(int64_t m) { return m > 128; }
// Columns per tile: 128 where C has no more, else 256.
int tile_columns(int64_t n) { return n <= 128 ? 128 : 256; }
int tile_rows(int64_t m) { return pairs_of_ctas(m) ? 256 : 128; }

// The loss of few rows is bound by the stream of W: there the tile has as many columns as share the classes out most evenly
// (131072 classes on 148 SMs: four turns of 224 instead of 256, and nothing left to do in the fifth).
int logit_columns(int64_t rows, int64_t classes, int parts, bool grad)
{
    const int most = tile_columns(classes);
    if (grad || most == 128 || pairs_of_ctas(rows)) return most;
    int best = most;
    for (int c = most - 16; c > most / parts * (parts - 1); c -= 16)
        if (ceil_div(ceil_div(classes, c), kSms) * (c + 8) < ceil_div(ceil_div(classes, best), kSms) * (best + 8)) best = c;
    return best;
}

// Pairs of (largest, sum) per row: one for each part of a tile that has columns.
int64_t blocks_of(int64_t classes, int cols, int parts)
{
    const int64_t tiles = ceil_div(classes, cols), last = classes - (tiles - 1) * cols;
    return parts * (tiles - 1) + ceil_div(last, tile_columns(classes) / parts);
}

template <bool AMN, bool BMN, bool kChunked, class Epi>
cudaError_t run_product(const Operand &a, const Operand &b, const tc::Shape &s, int cols, const Epi &epi, cudaStream_t stream)
{
    if (tile_columns(s.n) == 128)
        return pairs_of_ctas(s.m) ? launch_product<2, 128, AMN, BMN, kChunked>(a, b, s, cols, epi, stream)
                                  : launch_product<1, 128, AMN, BMN, kChunked>(a, b, s, cols, epi, stream);
    return pairs_of_ctas(s.m) ? launch_product<2, 256, AMN, BMN, kChunked>(a, b, s, cols, epi, stream)
                              : launch_product<1, 256, AMN, BMN, kChunked>(a, b, s, cols, epi, stream);
}

template <class Epi>
cudaError_t run_logits(const Operand &a, const Operand &b, const tc::Shape &s, int cols, const Epi &epi, cudaStream_t stream)
{
    return s.k_steps > s.chunk ? run_product<false, false, true>(a, b, s, cols, epi, stream) : run_product<false, false, false>(a, b, s, cols, epi, stream);
}

// Bytes per logit of a piece of rows: 16-bit values in place, or 16-bit or fp32 values and two planes.
int64_t logit_bytes(bool wide, int p_planes) { return wide ? 8 : p_planes == 2 ? 6 : 2; }

bool takes_bulk(const chicle_dense_t &x)
{
    return x.type != CHICLE_F32 && (reinterpret_cast<uintptr_t>(x.data) & 15) == 0 && (x.ld & 7) == 0;
}

// The summed index of a gradient is cut where its tiles alone would leave SMs idle: time of the waves plus that of
// writing and joining the planes.
int plan_splits(int64_t m, int64_t n, int64_t steps, int pairs)
{
    const int rows = tile_rows(m), cols = tile_columns(n);
    const int64_t tiles = ceil_div(m, rows) * ceil_div(n, cols), slots = kSms / (rows / 128);
    const double slice = cols == 256 ? 0.28e-6 : 0.25e-6; // (narrow tiles wait for their copies: three quarters of the bytes)
    int best = 1;
    double best_t = 0;
    for (int s = 1; s <= 64 && s <= steps; ++s) {
        const double waves = (double)ceil_div(tiles * s, slots);
        const double t = waves * ((double)(ceil_div(steps, s) * pairs) * slice + 1.0e-6) + (s > 1 ? 6e-6 + (double)s * m * n * 8.0 / 5e12 : 0.0);
        if (s == 1 || t < best_t * 0.95) {
            best = s;
            best_t = t;
        }
    }
    return best;
}

// Slices that an accumulator of a 16-bit gradient takes. What it cuts off, 1.6e-7 of itself per step of 16 terms where the terms have
// one sign (tensor_core.cuh), comes to half of that times the steps, of the terms' magnitudes, and stays below an eighth of half a step
// of the result: 768 steps in fp16, 6144 in bf16. (One accumulator for 131072 classes: 2.5e-4 off, half of fp16's half step; for
// 800000: 1.7e-3.) Longer sums are added chunk by chunk in registers.
constexpr int64_t kLongestF16 = 768 * 16 / tc::kBK, kLongestBf16 = 6144 * 16 / tc::kBK;
// Logits of a piece. Nothing hangs on where a piece ends: 8192 rows of 131072 classes and 4096 columns in bf16 take 23.7 ms in one
// piece, 8193 in two 23.7 to 24.0; with 2^30 instead 23.0 and 24.2, 16384 rows 46.3 and 48.0 with 2^31, of 1024 columns 13.4 and 13.1
// (one GPU's power limit moves these by 4 %).
constexpr int64_t kPieceBytes = (int64_t)1 << 31;
constexpr int64_t kFewRows = 32;
constexpr int64_t kStatBytes = (int64_t)1 << 30; // the loss alone: pairs of (largest, sum), for so many bytes of rows at a time

struct Plan {
    bool wide, half; // single precision; operands in fp16 (else bf16)
    int planes, pairs;                  // of the operands
    int p_planes, grad_pairs;           // of P, and products of planes of the gradients
    int64_t n, v, d;
    bool pack_x, pack_w;
    int64_t pitch_d, ld_v;
    int64_t piece;     // rows per piece
    int logit_chunk, grad_chunk; // slices per accumulator
    int longest;                 // and of a gradient of 16 bits, where its sum has more
    int cols, parts;   // of the logits' tiles
    int splits_x, splits_w;
    // offsets into the workspace
    size_t x, w, stats, label_logit, norm, store, p, acc, partial, scales, largest, total;
};

Plan make_plan(const chicle_dense_t &X, const chicle_dense_t &W, bool grad)
{
    Plan p{};
    p.wide = X.type == CHICLE_F32;
    p.half = X.type != CHICLE_BF16;
    p.planes = p.wide ? 2 : 1;
    p.pairs = p.wide ? 3 : 1;
    // Few rows: P in two planes. One row's gradients hang on the rounding of one or a few entries of P (n = 1: twice what the
    // rounding of the result costs), and the products of few rows wait for W and dW anyway.
    p.p_planes = p.wide || X.rows <= kFewRows ? 2 : 1;
    p.grad_pairs = p.wide ? 3 : p.p_planes;
    p.n = X.rows, p.v = W.rows, p.d = X.cols;
    p.pack_x = grad || !takes_bulk(X);
    p.pack_w = !takes_bulk(W);
    // rows of whole 128-byte lines: a row of a bulk copy that straddles two takes two requests
    p.pitch_d = (p.d + 63) / 64 * 64;
    p.ld_v = (p.v + 63) / 64 * 64;
    // Slices per accumulator (why: tensor_core.cuh): 512 elements of a logit, whose errors its exponential takes on whole (16 bits, terms
    // of one sign: 1024 are off by 6e-6 of the logit, 512 by 3e-6; of both signs loss off by 3e-7 and 1.5e-7; 4096 x 100000 x 2048 takes
    // 1355 us with 1024, 1403 with 512, 1527 with 256), and of a gradient in single precision (2048: off by 2.5e-6, 512: 7e-7, 256:
    // 4e-7). A gradient that is rounded to 16 bits in the end has one accumulator for `longest` of them.
    p.logit_chunk = 512 / tc::kBK;
    p.grad_chunk = (p.wide ? 512 : 1024) / tc::kBK; // (16 bits, P in two planes: what is fetched again is still in L2)
    p.longest = (int)((p.half ? kLongestF16 : kLongestBf16) / p.grad_pairs);
    p.parts = tc::kEpiWarps / 4;
    p.cols = logit_columns(p.n, p.v, p.parts, grad);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    p.piece = p.n;
    if (grad) {
        const int64_t row_bytes = p.ld_v * logit_bytes(p.wide, p.p_planes);
        const int64_t most = std::max<int64_t>(1, 4 * kPieceBytes / row_bytes);
        // fewer than 2048 rows: the fp32 sums of dW would be read and written too often beside the products of a piece
        const int64_t rows = std::max(kPieceBytes / row_bytes / 256 * 256, std::min<int64_t>(2048, most));
        if (rows < p.n) {
            p.piece = ceil_div(p.n, ceil_div(p.n, rows));
            const int64_t whole = ceil_div(p.piece, 256) * 256; // (whole tiles, where there is room for them)
            if (whole <= most) p.piece = whole;
        }
    } else {
        const int64_t rows = std::max<int64_t>(4096, kStatBytes / (blocks_of(p.v, p.cols, p.parts) * (int64_t)sizeof(float2)) / 256 * 256);
        p.piece = std::min(p.n, rows);
    }
    if (p.pack_x) p.x = take((size_t)p.planes * p.n * p.pitch_d * 2);
    if (p.pack_w) p.w = take((size_t)p.planes * p.v * p.pitch_d * 2);
    p.stats = take((size_t)(blocks_of(p.v, p.cols, p.parts) * p.piece) * sizeof(float2));
    p.label_logit = take((size_t)p.piece * 4);
    if (grad) p.norm = take((size_t)p.piece * sizeof(float2));
    if (grad) {
        if (p.wide) {
            p.store = take((size_t)p.piece * p.ld_v * 4);
            p.p = take((size_t)2 * p.piece * p.ld_v * 2);
        } else if (p.p_planes == 2) {
            p.store = take((size_t)p.piece * p.ld_v * 2);
            p.p = take((size_t)2 * p.piece * p.ld_v * 2);
        } else {
            p.store = p.p = take((size_t)p.piece * p.ld_v * 2);
        }
        if (p.piece < p.n) p.acc = take((size_t)p.v * p.d * 4);
        p.splits_x = plan_splits(p.piece, p.d, ceil_div(p.v, tc::kBK), p.grad_pairs);
        p.splits_w = plan_splits(p.v, p.d, ceil_div(p.piece, tc::kBK), p.grad_pairs);
        size_t part = 0;
        if (p.splits_x > 1) part = (size_t)p.splits_x * p.piece * p.d * 4;
        if (p.splits_w > 1) part = std::max(part, (size_t)p.splits_w * p.v * p.d * 4);
        if (part) p.partial = take(part);
    }
    p.scales = take(kScales * sizeof(float));
    if (p.half) p.largest = take(3 * kMaxBlocks * sizeof(float));
    p.total = at;
    return p;
}

// Lays out what has to be, and finds the scales that these operands take (*scales: null where they take none).
template <typename T, typename P>
cudaError_t pack(const chicle_dense_t &X, const chicle_dense_t &W, const Plan &p, const int32_t *labels, const float *weights, float scale,
                 uint8_t *ws, cudaStream_t s, bool grad, float **scales)
{
    *scales = p.wide || (p.half && grad) ? reinterpret_cast<float *>(ws + p.scales) : nullptr;
    float *largest = nullptr;
    const bool many = *scales && weights && p.n > kFewWeights;
    if (p.wide || many) {
        largest = reinterpret_cast<float *>(ws + p.largest);
        const int first = p.wide ? 0 : 2, groups = (many ? 3 : 2) - first;
        k_largest<<<(unsigned)(groups * kMaxBlocks), 256, 0, s>>>((const float *)X.data, X.ld, p.n, labels, (int32_t)p.v, (const float *)W.data, W.ld,
                                                                  (int32_t)p.d, weights, scale, first, largest);
    }
    auto part = [&](const chicle_dense_t &m, bool is_packed, size_t at, const int32_t *rows_with, int lift) {
        const int64_t blocks = is_packed ? std::min<int64_t>(ceil_div(m.rows * (p.pitch_d / 8), 256), kSms * 16) : 0;
        return Packed{m.data, m.ld, m.rows, m.rows * p.pitch_d, ws + at, rows_with, (unsigned)blocks, lift};
    };
    const Packed x = part(X, p.pack_x, p.x, labels, kLiftX), w = part(W, p.pack_w, p.w, nullptr, kLiftW);
    if (x.blocks + w.blocks)
        k_pack<T, P><<<x.blocks + w.blocks, 256, 0, s>>>(x, w, (int32_t)p.d, p.pitch_d, (int32_t)p.v, largest, weights, p.n, scale, *scales);
    return cudaGetLastError();
}

Operand operand_of(const chicle_dense_t &src, const void *packed, bool is_packed, const Plan &p)
{
    Operand o;
    o.rows = src.rows;
    o.cols = p.d;
    o.data = is_packed ? packed : src.data;
    o.pitch = is_packed ? p.pitch_d : src.ld;
    o.planes = p.planes;
    o.plane = src.rows * o.pitch;
    return o;
}

tc::Shape shape_of(const Plan &p, int64_t m, int64_t n, int64_t k, int pairs, int chunk, int splits, int group, uint32_t *status)
{
    tc::Shape s{};
    s.m = (int32_t)m, s.n = (int32_t)n;
    s.k_steps = (int32_t)ceil_div(k, tc::kBK);
    s.pairs = pairs;
    s.chunk = chunk;
    s.splits = splits;
    s.group = group;
    s.half = p.half;
    s.status = status;
    return s;
}

cudaError_t join_blocks(const Plan &p, const float2 *stats, int64_t rows, const int32_t *labels, const float *label_logit, float *loss,
                        float *lse, float2 *norm, uint32_t *status, cudaStream_t s)
{
    const int blocks = (int)blocks_of(p.v, p.cols, p.parts);
    if (rows >= 32 * 64)
        k_join_blocks<32><<<(unsigned)ceil_div(rows, 32), 512, 0, s>>>(stats, blocks, (int32_t)rows, labels, (int32_t)p.v, label_logit, loss, lse, norm, status);
    else if (rows >= 8)
        k_join_blocks<8><<<(unsigned)ceil_div(rows, 8), 512, 0, s>>>(stats, blocks, (int32_t)rows, labels, (int32_t)p.v, label_logit, loss, lse, norm, status);
    else
        k_join_blocks<1><<<(unsigned)rows, 512, 0, s>>>(stats, blocks, (int32_t)rows, labels, (int32_t)p.v, label_logit, loss, lse, norm, status);
    return cudaGetLastError();
}

// m tiles walked together: as many as their rows of A (all of the summed index) stay in a quarter of L2 beside the stream of B.
int group_of(int64_t k, int planes, int rows_per_tile)
{
    const int64_t bytes = k * 2 * planes * rows_per_tile;
    return (int)std::max<int64_t>(1, std::min<int64_t>(64, ((int64_t)32 << 20) / std::max<int64_t>(1, bytes)));
}

template <typename OutT>
cudaError_t gradient(const Plan &p, const Operand &a, const Operand &b, bool of_x, tc::Shape s, GradEpilogue<OutT> epi, cudaStream_t stream)
{
    const int cols = tile_columns(s.n);
    bool chunked = true;
    if constexpr (sizeof(OutT) == 2) {
        chunked = ceil_div(s.k_steps, s.splits) > p.longest;
        if (chunked) s.chunk = p.longest;
    }
    cudaError_t e;
    if (chunked) {
        e = of_x ? run_product<false, true, true>(a, b, s, cols, epi, stream) : run_product<true, true, true>(a, b, s, cols, epi, stream);
    } else if constexpr (sizeof(OutT) == 2) {
        e = of_x ? run_product<false, true, false>(a, b, s, cols, epi, stream) : run_product<true, true, false>(a, b, s, cols, epi, stream);
    }
    if (e == cudaSuccess && s.splits > 1) {
        const int64_t all = (int64_t)s.m * s.n;
        auto *join = (s.n & 3) == 0 ? k_join_splits<OutT, 4> : k_join_splits<OutT, 1>;
        join<<<(unsigned)std::min<int64_t>(ceil_div(all, 1024), kSms * 8), 256, 0, stream>>>(epi.partial, s.splits, s.m, s.n, epi.add, epi.keep, epi.out, epi.ld, epi.scale, epi.scale_b, epi.labels, epi.classes);
        e = cudaGetLastError();
    }
    return e;
}

template <typename T, typename PT, typename StoreT>
cudaError_t run_grad(const Plan &p, const chicle_dense_t &X, const chicle_dense_t &W, const int32_t *labels, const float *weights,
                     float scale, float *loss, float *lse, const chicle_dense_t &dX, const chicle_dense_t &dW, uint8_t *ws,
                     uint32_t *status, cudaStream_t stream)
{
    constexpr bool kWide = sizeof(T) == 4;
    float *scales;
    cudaError_t e = pack<T, PT>(X, W, p, labels, weights, scale, ws, stream, true, &scales);
    const Operand w = operand_of(W, ws + p.w, p.pack_w, p);
    for (int64_t r0 = 0; e == cudaSuccess && r0 < p.n; r0 += p.piece) {
        const int64_t rows = std::min(p.piece, p.n - r0);
        Operand x = operand_of(X, ws + p.x, true, p);
        x.data = static_cast<const uint16_t *>(x.data) + r0 * p.pitch_d;
        x.rows = rows;
        float2 *stats = reinterpret_cast<float2 *>(ws + p.stats);
        float *label_logit = reinterpret_cast<float *>(ws + p.label_logit);
        float2 *norm = reinterpret_cast<float2 *>(ws + p.norm);
        StoreT *store = reinterpret_cast<StoreT *>(ws + p.store);
        PT *prob = reinterpret_cast<PT *>(ws + p.p);
        const LogitsEpilogue<StoreT> le{labels + r0, stats, label_logit, store, p.ld_v, kWide ? scales : nullptr};
        e = run_logits(x, w, shape_of(p, rows, p.v, p.d, p.pairs, p.logit_chunk, 1, group_of(p.d, p.planes, tile_rows(p.n)), status), p.cols, le, stream);
        // a CTA of the elementwise pass has a whole row; it takes longer so, which shows where the rows take several turns (10000
        // rows: 4 us more than the launch)
        const bool joins = p.v <= 2048 && rows <= 8 * kSms;
        if (e == cudaSuccess && !joins) e = join_blocks(p, stats, rows, labels + r0, label_logit, loss + r0, lse + r0, norm, status, stream);
        if (e != cudaSuccess) break;
        Operand q;
        q.data = prob;
        q.rows = rows, q.cols = p.v, q.pitch = p.ld_v, q.plane = p.piece * p.ld_v, q.planes = p.p_planes;
        const int steps = p.v >= 8192 ? 4 : 1;
        constexpr int kMany = kWide ? 2 : 1; // planes of P where rows are many
        const unsigned threads = p.v <= 1024 ? 128 : 256; // (one CTA for the row, then: the other threads would have nothing to do)
        auto *probabilities = p.p_planes != kMany ? (steps == 4 ? k_probabilities<PT, kWide, 2, 4, false>
                                                     : joins    ? k_probabilities<PT, kWide, 2, 1, true>
                                                                : k_probabilities<PT, kWide, 2, 1, false>)
                              : steps == 4        ? k_probabilities<PT, kWide, kMany, 4, false>
                              : joins             ? k_probabilities<PT, kWide, kMany, 1, true>
                                                  : k_probabilities<PT, kWide, kMany, 1, false>;
        for (int64_t y = 0; y < rows; y += 65535)
            probabilities<<<dim3((unsigned)ceil_div(p.v, 2048 * steps), (unsigned)std::min<int64_t>(65535, rows - y)), threads, 0, stream>>>(store + y * p.ld_v, prob + y * p.ld_v, p.ld_v, q.plane, (int32_t)rows, (int32_t)p.v, stats + y, norm + y, loss + r0 + y,
                labels + r0 + y, weights ? weights + r0 + y : nullptr, scale, scales ? scales + kLift : nullptr,
                __builtin_ctz(tile_columns(p.v) / p.parts), (int)blocks_of(p.v, p.cols, p.parts), label_logit + y, lse + r0 + y, status);
        if ((e = cudaGetLastError()) != cudaSuccess) break;
        const float *back = scales ? scales + kInvLift : nullptr;
        float *partial = reinterpret_cast<float *>(ws + p.partial);
        GradEpilogue<T> ex{static_cast<T *>(dX.data) + r0 * dX.ld, dX.ld, p.splits_x > 1 ? partial : nullptr, nullptr, nullptr, back,
                           kWide ? scales + kInvW : nullptr, labels + r0, (int32_t)p.v};
        e = gradient<T>(p, q, w, true, shape_of(p, rows, p.d, p.v, p.grad_pairs, p.grad_chunk, p.splits_x, 8, status), ex, stream);
        if (e != cudaSuccess) break;
        // dW over the pieces: the sums stay in fp32 until the last
        const bool first = r0 == 0, last = r0 + rows >= p.n;
        GradEpilogue<T> ew{static_cast<T *>(dW.data), dW.ld, nullptr, nullptr, nullptr, back, kWide ? scales + kInvX : nullptr, nullptr, 0};
        float *acc = reinterpret_cast<float *>(ws + p.acc);
        if (!first) ew.add = acc;
        if (!last) ew.keep = acc;
        const int splits = (int)std::min<int64_t>(p.splits_w, ceil_div(rows, tc::kBK));
        if (splits > 1) ew.partial = partial;
        e = gradient<T>(p, q, x, false, shape_of(p, p.v, p.d, rows, p.grad_pairs, p.grad_chunk, splits, 8, status), ew, stream);
    }
    return e;
}

} // namespace

// ---- checks ------------------------------------------------------------------------------------------------

const char *check_dense(const chicle_dense_t *x)
{
    if (!x) return "a matrix is NULL";
    if ((int)x->type < 0 || (int)x->type > 2) return "unknown element type";
    if (x->rows < 0 || x->cols < 1) return "rows must be >= 0 and cols >= 1";
    if (x->ld < x->cols) return "ld < cols";
    if (x->rows > INT32_MAX - 4096 || x->cols > 65536) return "more than 2^31 - 4097 rows or 65536 columns";
    if (x->rows > 0 && !x->data) return "data is NULL";
    if (reinterpret_cast<uintptr_t>(x->data) % (x->type == CHICLE_F32 ? 4 : 2)) return "data is not aligned to its element type";
    if (x->ld > ((int64_t)1 << 38)) return "ld too large";
    return nullptr;
}

} // namespace chicle

using namespace chicle;

namespace {

const char *check_softmax(const chicle_dense_t *X, const chicle_dense_t *W, chicle_status_t *st)
{
    *st = CHICLE_ERR_INVALID_ARG;
    if (const char *m = check_dense(X)) return m;
    if (const char *m = check_dense(W)) return m;
    if (X->type != W->type) return "X and W must have one element type";
    if (X->cols != W->cols) return "X and W must have the same number of columns";
    if (W->rows < 1) return "W needs at least one class";
    return nullptr;
}

} // namespace

extern "C" chicle_status_t chicle_softmax_workspace(const chicle_dense_t *X, const chicle_dense_t *W, int gradients, size_t *host_bytes)
{
    chicle_status_t st;
    if (!host_bytes || check_softmax(X, W, &st)) return CHICLE_ERR_INVALID_ARG;
    *host_bytes = make_plan(*X, *W, gradients != 0).total;
    return CHICLE_OK;
}

extern "C" chicle_status_t chicle_softmax_loss(int device, void *cuda_stream, const chicle_dense_t *X, const chicle_dense_t *W,
                                               const int32_t *dev_labels, float *dev_loss, float *dev_lse, void *dev_workspace,
                                               size_t workspace_bytes, uint32_t *dev_status, char *host_errbuf, size_t errbuf_len)
{
    const CallError err{host_errbuf, errbuf_len};
    chicle_status_t st;
    if (const char *m = check_softmax(X, W, &st)) return err(st, m);
    if (X->rows == 0) return CHICLE_OK;
    if (!dev_labels || !dev_loss || !dev_lse) return err(CHICLE_ERR_INVALID_ARG, "labels, loss and lse must be non-NULL device pointers");
    const Plan p = make_plan(*X, *W, false);
    if (const char *m = check_workspace(dev_workspace, workspace_bytes, p.total)) return err(CHICLE_ERR_INVALID_ARG, m);
    const DeviceGuard guard(device);
    if (!guard.ok()) return err(CHICLE_ERR_CUDA, guard.message());
    if (!encode_fn()) return err(CHICLE_ERR_CUDA, "the driver has no cuTensorMapEncodeTiled");
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    uint8_t *ws = static_cast<uint8_t *>(dev_workspace);
    float *scales = nullptr;
    // (rows without a label are left out of the scale, so they have to be zeros)
    cudaError_t e = p.wide ? pack<float, __half>(*X, *W, p, dev_labels, nullptr, 1.f, ws, s, false, &scales)
                    : p.half ? pack<__half, __half>(*X, *W, p, dev_labels, nullptr, 1.f, ws, s, false, &scales)
                             : pack<__nv_bfloat16, __nv_bfloat16>(*X, *W, p, dev_labels, nullptr, 1.f, ws, s, false, &scales);
    float2 *stats = reinterpret_cast<float2 *>(ws + p.stats);
    float *label_logit = reinterpret_cast<float *>(ws + p.label_logit);
    const Operand w = operand_of(*W, ws + p.w, p.pack_w, p);
    for (int64_t r0 = 0; e == cudaSuccess && r0 < p.n; r0 += p.piece) {
        const int64_t rows = std::min(p.piece, p.n - r0);
        Operand x = operand_of(*X, ws + p.x, p.pack_x, p);
        x.data = static_cast<const uint16_t *>(x.data) + r0 * x.pitch; // (16-bit elements, planes too)
        x.rows = rows;
        const LogitsEpilogue<NoStore> le{dev_labels + r0, stats, label_logit, nullptr, 0, scales};
        e = run_logits(x, w, shape_of(p, rows, p.v, p.d, p.pairs, p.logit_chunk, 1, group_of(p.d, p.planes, tile_rows(rows)), dev_status), p.cols, le, s);
        if (e == cudaSuccess) e = join_blocks(p, stats, rows, dev_labels + r0, label_logit, dev_loss + r0, dev_lse + r0, nullptr, dev_status, s);
    }
    return e == cudaSuccess ? CHICLE_OK : err.cuda(e);
}

extern "C" chicle_status_t chicle_softmax_loss_grad(int device, void *cuda_stream, const chicle_dense_t *X, const chicle_dense_t *W,
                                                    const int32_t *dev_labels, const float *dev_weights, float scale, float *dev_loss,
                                                    float *dev_lse, const chicle_dense_t *dX, const chicle_dense_t *dW,
                                                    void *dev_workspace, size_t workspace_bytes, uint32_t *dev_status, char *host_errbuf,
                                                    size_t errbuf_len)
{
    const CallError err{host_errbuf, errbuf_len};
    chicle_status_t st;
    if (const char *m = check_softmax(X, W, &st)) return err(st, m);
    if (const char *m = check_dense(dX)) return err(CHICLE_ERR_INVALID_ARG, m);
    if (const char *m = check_dense(dW)) return err(CHICLE_ERR_INVALID_ARG, m);
    if (dX->type != X->type || dX->rows != X->rows || dX->cols != X->cols) return err(CHICLE_ERR_INVALID_ARG, "dX must have X's type and shape");
    if (dW->type != W->type || dW->rows != W->rows || dW->cols != W->cols) return err(CHICLE_ERR_INVALID_ARG, "dW must have W's type and shape");
    if (overlapping(*dX, *W) || overlapping(*dW, *X) || overlapping(*dW, *W) || overlapping(*dX, *X) || overlapping(*dX, *dW))
        return err(CHICLE_ERR_INVALID_ARG, "dX and dW must not overlap X, W or each other");
    if (!std::isfinite(scale)) return err(CHICLE_ERR_INVALID_ARG, "scale must be finite");
    if (X->rows > 0 && (!dev_labels || !dev_loss || !dev_lse))
        return err(CHICLE_ERR_INVALID_ARG, "labels, loss and lse must be non-NULL device pointers");
    const Plan p = make_plan(*X, *W, true);
    if (X->rows > 0)
        if (const char *m = check_workspace(dev_workspace, workspace_bytes, p.total)) return err(CHICLE_ERR_INVALID_ARG, m);
    const DeviceGuard guard(device);
    if (!guard.ok()) return err(CHICLE_ERR_CUDA, guard.message());
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    if (X->rows == 0) {
        const size_t es = (size_t)element_size(dW->type);
        const cudaError_t e = cudaMemset2DAsync(dW->data, (size_t)dW->ld * es, 0, (size_t)dW->cols * es, (size_t)dW->rows, s);
        return e == cudaSuccess ? CHICLE_OK : err.cuda(e);
    }
    if (!encode_fn()) return err(CHICLE_ERR_CUDA, "the driver has no cuTensorMapEncodeTiled");
    uint8_t *ws = static_cast<uint8_t *>(dev_workspace);
    cudaError_t e;
    if (X->type == CHICLE_F32)
        e = run_grad<float, __half, float>(p, *X, *W, dev_labels, dev_weights, scale, dev_loss, dev_lse, *dX, *dW, ws, dev_status, s);
    else if (X->type == CHICLE_BF16)
        e = run_grad<__nv_bfloat16, __nv_bfloat16, __half>(p, *X, *W, dev_labels, dev_weights, scale, dev_loss, dev_lse, *dX, *dW, ws, dev_status, s);
    else
        e = run_grad<__half, __half, __half>(p, *X, *W, dev_labels, dev_weights, scale, dev_loss, dev_lse, *dX, *dW, ws, dev_status, s);
    return e == cudaSuccess ? CHICLE_OK : err.cuda(e);
}
