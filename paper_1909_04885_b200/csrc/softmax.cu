// Softmax cross entropy of a linear map to many classes, and its gradients (chicle_softmax_loss,
// chicle_softmax_loss_grad): the multi-class sibling of the logistic loss.
//
//   l_iv = x_i . w_v        lse_i = log sum_v exp(l_iv)        loss_i = lse_i - l_{i, y_i}
//   p_iv = g_i (exp(l_iv - lse_i) - [v = y_i])                 dX = P W,  dW = P^T X
//
// The logits are never held as a whole. The loss alone keeps, per row and 128 classes, the largest logit and the sum of
// exponentials relative to it; a second kernel joins them. For the gradients the rows are taken in pieces of about a
// gigabyte of 16-bit values: the product's epilogue writes exp(l - m) of its tile (m: the largest of the row in 128
// classes) as fp16, scaled by 2^15 so that what is 2^-29 of the tile's largest still has all its bits; an elementwise
// pass turns the piece into P in place, and two products take dX and the piece's share of dW from it. So the
// logits are computed once: 6 n V d operations, against 8 where they are computed again for the gradient, for 6 bytes of traffic
// per logit (at d = 4096 a third of the products' time against a twentieth).
//
// Rounding: logits, sums and gradients in fp32; P is rounded once to the operands' type (fp16: scaled so that the
// largest weight comes to 2^14), and the entry of the label comes from expm1(-loss), not from a difference.
#include <algorithm>
#include <cmath>

#include "operators.cuh"
#include "tensor_core.cuh"

namespace chicle {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kStoreScale = 32768.f; // fp16 exponentials are held times 2^15
constexpr int kHalfTile = 128;         // classes per pair of (largest, sum)

// ---- epilogues ---------------------------------------------------------------------------------------------

// Reduces a tile of logits to (largest, sum of exponentials) per row and 128 classes, keeps the label's logit, and
// writes the exponentials for the gradients: StoreT void (loss alone), half, or float (single precision).
template <typename StoreT> struct LogitsEpilogue {
    const int32_t *labels; // rows of this piece
    float2 *stats;         // [128-class block][rows]
    float *label_logit;    // [rows]
    StoreT *store;         // [rows][ld]
    int64_t ld;

    template <int BN>
    __device__ __forceinline__ void tile(const tc::Shape &s, const tc::Tile &, int row0, int col0, uint32_t tmem, int quarter,
                                         int half, int lane) const
    {
        static_assert(BN == 2 * kHalfTile, "a warp takes 128 classes");
        const int row = row0 + quarter * 32 + lane;
        const int c0 = col0 + half * kHalfTile;
        const uint32_t at = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(half * kHalfTile);
        const bool live = row < s.m;
        const int lab = live ? labels[row] - c0 : -1; // (a negative label is in front of every block)
        uint32_t r[32];
        float top = -INFINITY;
#pragma unroll 1
        for (int c = 0; c < kHalfTile; c += 32) {
            if (c0 + c >= s.n) break;
            tc::load32(at + c, r);
            tc::wait_loads();
            if (c0 + c + 32 > s.n) {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (c0 + c + j >= s.n) r[j] = 0xff800000u;
            }
            float t[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int j = 0; j < 32; ++j) t[j & 3] = fmaxf(t[j & 3], __uint_as_float(r[j]));
            top = fmaxf(top, fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3])));
            if (lab >= c && lab < c + 32) {
                float v = 0.f;
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (lab - c == j) v = __uint_as_float(r[j]);
                label_logit[row] = v;
            }
            __syncwarp();
        }
        // (a block without a logit above -inf: relative to 0, so that its exponentials are 0 and not NaN)
        const float ref = top == -INFINITY ? 0.f : top;
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
        for (int c = 0; c < kHalfTile; c += 32) {
            if (c0 + c >= s.n) break;
            tc::load32(at + c, r);
            tc::wait_loads();
            if (c0 + c + 32 > s.n) {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (c0 + c + j >= s.n) r[j] = 0xff800000u;
            }
            float e[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                e[j] = exp2f((__uint_as_float(r[j]) - ref) * kLog2e);
                sum[j & 3] += e[j];
            }
            if constexpr (sizeof(StoreT) == 2) {
                if (live) {
                    uint4 *dst = reinterpret_cast<uint4 *>(store + (int64_t)row * ld + c0 + c);
#pragma unroll
                    for (int j = 0; j < 32; j += 8) {
                        if (c0 + c + j < s.n) { // (ld: a multiple of 8, what lies behind the last class is not read)
                            uint4 q;
                            __half2 *h = reinterpret_cast<__half2 *>(&q);
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                h[i] = __floats2half2_rn(e[j + 2 * i] * kStoreScale, e[j + 2 * i + 1] * kStoreScale);
                            dst[j / 8] = q;
                        }
                    }
                }
            } else if constexpr (sizeof(StoreT) == 4) {
                if (live) {
                    float4 *dst = reinterpret_cast<float4 *>(store + (int64_t)row * ld + c0 + c);
#pragma unroll
                    for (int j = 0; j < 32; j += 4)
                        if (c0 + c + j < s.n) dst[j / 4] = make_float4(e[j], e[j + 1], e[j + 2], e[j + 3]);
                }
            }
            __syncwarp();
        }
        // NaN: fmaxf passes over it, the sum does not
        if (live && c0 < s.n) stats[(int64_t)(c0 / kHalfTile) * s.m + row] = make_float2(top, (sum[0] + sum[1]) + (sum[2] + sum[3]));
    }
};

struct NoStore {
    char c;
};

template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// Where a tile of a gradient goes. With splits: to `partial`, one plane per split. Else sum = (add ? *add : 0) + tile; to
// `keep` (fp32, for the pieces that follow) or to `out`.
template <typename OutT> struct GradEpilogue {
    OutT *out;
    int64_t ld;
    float *partial;          // [split][m][n]
    const float *add;        // [m][n], or null
    float *keep;             // [m][n], or null
    const float *scale;      // device factor of the result, or null
    const int32_t *labels;   // rows without a label come out 0 whatever the other operand holds; or null
    int32_t classes;

    template <int BN>
    __device__ __forceinline__ void tile(const tc::Shape &s, const tc::Tile &tl, int row0, int col0, uint32_t tmem, int quarter,
                                         int half, int lane) const
    {
        const int row = row0 + quarter * 32 + lane;
        const int c0 = col0 + half * (BN / 2);
        const uint32_t at = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(half * (BN / 2));
        const bool live = row < s.m;
        const bool whole = partial || keep;
        const float f = whole || !scale ? 1.f : *scale;
        const bool zero = live && labels && ((uint32_t)labels[row] >= (uint32_t)classes);
        float *dst32 = partial ? partial + ((int64_t)tl.split * s.m + row) * s.n : keep + (int64_t)row * s.n;
        const bool quads = (s.n & 3) == 0; // fp32 rows of n: 16-byte pieces
        uint32_t r[32];
#pragma unroll 1
        for (int c = 0; c < BN / 2; c += 32) {
            const int col = c0 + c;
            if (col >= s.n) break;
            tc::load32(at + c, r);
            tc::wait_loads();
            if (live) finish(s, row, col, r, zero, whole, f, quads, dst32);
            __syncwarp();
        }
    }

    __device__ __forceinline__ void finish(const tc::Shape &s, int row, int col, const uint32_t (&r)[32], bool zero, bool whole, float f,
                                           bool quads, float *dst32) const
    {
        float v[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = zero ? 0.f : __uint_as_float(r[j]);
        const bool full = col + 32 <= s.n;
        if (add && !partial) {
            const float *src = add + (int64_t)row * s.n + col;
            if (full && quads) {
#pragma unroll
                for (int j = 0; j < 32; j += 4) {
                    const float4 o = *reinterpret_cast<const float4 *>(src + j);
                    v[j] += o.x, v[j + 1] += o.y, v[j + 2] += o.z, v[j + 3] += o.w;
                }
            } else {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (col + j < s.n) v[j] += src[j];
            }
        }
        if (whole) {
            if (full && quads) {
#pragma unroll
                for (int j = 0; j < 32; j += 4)
                    *reinterpret_cast<float4 *>(dst32 + col + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
            } else {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (col + j < s.n) dst32[col + j] = v[j];
            }
            return;
        }
        OutT *dst = out + (int64_t)row * ld + col;
        constexpr int kPer = 16 / (int)sizeof(OutT);
        if (full && (reinterpret_cast<uintptr_t>(dst) & 15) == 0) {
#pragma unroll
            for (int j = 0; j < 32; j += kPer) {
                alignas(16) OutT q[kPer];
#pragma unroll
                for (int i = 0; i < kPer; ++i) q[i] = from_float<OutT>(v[j + i] * f);
                *reinterpret_cast<uint4 *>(dst + j) = *reinterpret_cast<const uint4 *>(q);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if (col + j < s.n) dst[j] = from_float<OutT>(v[j] * f);
        }
    }
};

// Joins the splits' planes in ascending order; add, keep, out as above.
template <typename OutT>
__global__ void __launch_bounds__(256) k_join_splits(const float *__restrict__ partial, int splits, int64_t m, int64_t n,
                                                     const float *add, float *keep, OutT *out, int64_t ld, const float *scale,
                                                     const int32_t *labels, int32_t classes)
{
    const int64_t all = m * n;
    const float f = scale ? *scale : 1.f;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < all; i += (int64_t)gridDim.x * blockDim.x) {
        float v = 0.f;
        for (int k = 0; k < splits; ++k) v += partial[(int64_t)k * all + i];
        const int64_t row = i / n;
        if (labels && (uint32_t)labels[row] >= (uint32_t)classes) v = 0.f;
        if (add) v += add[i];
        if (keep) keep[i] = v;
        else out[row * ld + (i - row * n)] = from_float<OutT>(v * f);
    }
}

// ---- small kernels -----------------------------------------------------------------------------------------

// Joins the blocks of 128 classes of R rows per CTA; threads of one row run down its blocks, fixed order.
template <int R>
__global__ void __launch_bounds__(512) k_join_blocks(const float2 *__restrict__ stats, int blocks, int32_t n,
                                                     const int32_t *__restrict__ labels, int32_t classes,
                                                     const float *__restrict__ label_logit, float *__restrict__ loss,
                                                     float *__restrict__ lse, uint32_t *status)
{
    constexpr int kT = 512 / R;
    __shared__ float s_top[kT][R], s_sum[kT][R];
    const int r = threadIdx.x % R, t = threadIdx.x / R;
    const int row = blockIdx.x * R + r;
    float top = -INFINITY, sum = 0.f;
    if (row < n) {
#pragma unroll 4
        for (int b = t; b < blocks; b += kT) {
            const float2 o = stats[(int64_t)b * n + row];
            const float m = fmaxf(top, o.x);
            // (equal ones, infinite ones too, without a difference)
            sum = (top == m ? sum : sum * exp2f((top - m) * kLog2e)) + (o.x == m ? o.y : o.y * exp2f((o.x - m) * kLog2e));
            top = m;
        }
    }
    s_top[t][r] = top;
    s_sum[t][r] = sum;
    __syncthreads();
    for (int w = kT / 2; w > 0; w >>= 1) {
        if (t < w) {
            const float b = s_top[t + w][r], m = fmaxf(top, b), bs = s_sum[t + w][r];
            sum = (top == m ? sum : sum * exp2f((top - m) * kLog2e)) + (b == m ? bs : bs * exp2f((b - m) * kLog2e));
            top = m;
            s_top[t][r] = top;
            s_sum[t][r] = sum;
        }
        __syncthreads();
    }
    if (t == 0 && row < n) {
        const int32_t y = labels[row];
        const bool has = (uint32_t)y < (uint32_t)classes;
        const float total = top + logf(sum);
        lse[row] = has ? total : 0.f;
        // relative to the largest logit: lse and the label's logit would lose the bits that they share
        loss[row] = has ? (top - label_logit[row]) + logf(sum) : 0.f;
        if (y >= classes && status) atomicOr(status, (uint32_t)ST_BAD_INDEX);
    }
}

// Exponentials to P, 8 classes per thread. Bits: 16-bit operands, in place; else three bf16 planes.
template <typename PT, bool kWide>
__global__ void __launch_bounds__(256)
k_probabilities(const void *store, PT *p, int64_t ld, int64_t plane, int32_t n, int32_t classes, const float2 *__restrict__ stats,
                const float *__restrict__ lse, const float *__restrict__ loss, const int32_t *__restrict__ labels,
                const float *__restrict__ weights, float scale, const float *__restrict__ lift)
{
    const int row = blockIdx.y;
    const int c = (blockIdx.x * 256 + threadIdx.x) * 8;
    if (c >= classes) return;
    const int32_t y = labels[row];
    const bool has = (uint32_t)y < (uint32_t)classes;
    float v[8];
    if (has) {
        float g = weights ? weights[row] * scale : scale;
        if (lift) g *= *lift;
        const float f = exp2f((stats[(int64_t)(c / kHalfTile) * n + row].x - lse[row]) * kLog2e) * (kWide ? 1.f : 1.f / kStoreScale) * g;
        if constexpr (kWide) {
            const float4 *src = reinterpret_cast<const float4 *>(static_cast<const float *>(store) + (int64_t)row * ld + c);
            const float4 a = src[0], b = src[1];
            v[0] = a.x * f, v[1] = a.y * f, v[2] = a.z * f, v[3] = a.w * f;
            v[4] = b.x * f, v[5] = b.y * f, v[6] = b.z * f, v[7] = b.w * f;
        } else {
            const uint4 q = *reinterpret_cast<const uint4 *>(static_cast<const __half *>(store) + (int64_t)row * ld + c);
            const __half2 *h = reinterpret_cast<const __half2 *>(&q);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 t = __half22float2(h[j]);
                v[2 * j] = t.x * f;
                v[2 * j + 1] = t.y * f;
            }
        }
        if (y >= c && y < c + 8) {
            const float at = g * expm1f(-loss[row]);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (y - c == j) v[j] = at;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 0.f;
    }
    alignas(16) PT q[8];
    if constexpr (kWide) {
#pragma unroll
        for (int k = 0; k < 3; ++k) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                q[j] = from_float<PT>(v[j]);
                v[j] -= (float)q[j];
            }
            *reinterpret_cast<uint4 *>(p + k * plane + (int64_t)row * ld + c) = *reinterpret_cast<const uint4 *>(q);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) q[j] = from_float<PT>(v[j]);
        *reinterpret_cast<uint4 *>(p + (int64_t)row * ld + c) = *reinterpret_cast<const uint4 *>(q);
    }
}

// Rows in a layout that the bulk copies take (16-byte pitch), single precision as three bf16 planes; rows without a
// label become zeros where labels are given.
template <typename T, typename P>
__global__ void __launch_bounds__(256) k_pack(const T *__restrict__ src, int64_t ld, int64_t rows, int32_t d, P *__restrict__ dst,
                                              int64_t pitch, int64_t plane, const int32_t *__restrict__ labels, int32_t classes)
{
    const int per = (int)((pitch + 7) / 8);
    const int64_t all = rows * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / per;
        const int c = (int)(i - row * per) * 8;
        const bool has = !labels || (uint32_t)labels[row] < (uint32_t)classes;
        const T *from = src + row * ld + c;
        alignas(16) T in[8];
        if (has && c + 8 <= d && (reinterpret_cast<uintptr_t>(from) & 15) == 0) {
#pragma unroll
            for (int j = 0; j < (int)(8 * sizeof(T) / 16); ++j)
                reinterpret_cast<uint4 *>(in)[j] = reinterpret_cast<const uint4 *>(from)[j];
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) in[j] = has && c + j < d ? from[j] : from_float<T>(0.f);
        }
        alignas(16) P q[8];
        if constexpr (sizeof(T) == 4) {
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = in[j];
#pragma unroll
            for (int k = 0; k < 3; ++k) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    q[j] = from_float<P>(v[j]);
                    // (infinite: the planes behind it are 0, not inf - inf)
                    v[j] = isinf((float)q[j]) ? 0.f : v[j] - (float)q[j];
                }
                *reinterpret_cast<uint4 *>(dst + k * plane + row * pitch + c) = *reinterpret_cast<const uint4 *>(q);
            }
        } else {
            *reinterpret_cast<uint4 *>(dst + row * pitch + c) = *reinterpret_cast<const uint4 *>(in);
        }
    }
}

// fp16: the power of two that takes the largest weight to [2^13, 2^14), and its inverse.
__global__ void __launch_bounds__(1024) k_lift(const float *__restrict__ weights, int64_t n, float scale, float *__restrict__ lift)
{
    __shared__ float s[32];
    float top = 0.f;
    if (weights)
        for (int64_t i = threadIdx.x; i < n; i += 1024) {
            const float v = fabsf(weights[i] * scale);
            if (v < INFINITY) top = fmaxf(top, v);
        }
    else
        top = fabsf(scale);
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = top;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 32; ++i) top = fmaxf(top, s[i]);
        int e = 0;
        if (top > 0.f) frexpf(top, &e); // top in [2^(e-1), 2^e)
        e = max(-100, min(100, 14 - e));
        lift[0] = ldexpf(1.f, e);
        lift[1] = ldexpf(1.f, -e);
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

template <int CG, int BN, bool AMN, bool BMN, class Epi>
cudaError_t launch_product(const Operand &a, const Operand &b, tc::Shape s, const Epi &epi, cudaStream_t stream)
{
    using L = tc::Layout<CG, BN>;
    CUtensorMap ma, mb;
    if (!make_map(&ma, a, s.half, 64, AMN ? 64 : L::kBM) || !make_map(&mb, b, s.half, 64, BMN ? 64 : L::kBNc)) return cudaErrorInvalidValue;
    s.m_tiles = (int32_t)ceil_div(s.m, CG * L::kBM);
    s.n_tiles = (int32_t)ceil_div(s.n, BN);
    auto *kernel = tc::k_product<CG, BN, AMN, BMN, Epi>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)L::kSmem);
    if (e != cudaSuccess) return e;
    const int64_t tiles = (int64_t)s.m_tiles * s.n_tiles * s.splits;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(CG * (tiles < kSms / CG ? tiles : kSms / CG)));
    cfg.blockDim = dim3(tc::kThreads);
    cfg.dynamicSmemBytes = L::kSmem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    if (CG == 2) {
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim = {2, 1, 1};
        cfg.attrs = attr;
        cfg.numAttrs = 1;
    }
    return cudaLaunchKernelEx(&cfg, kernel, ma, mb, s, epi);
}

int element_size(chicle_dtype_t t) { return t == CHICLE_F32 ? 4 : 2; }

// Bytes per logit of a piece of rows: 16-bit values in place, or fp32 values and three planes.
int64_t logit_bytes(bool wide) { return wide ? 10 : 2; }

bool takes_bulk(const chicle_dense_t &x)
{
    return x.type != CHICLE_F32 && (reinterpret_cast<uintptr_t>(x.data) & 15) == 0 && (x.ld & 7) == 0;
}

// The summed index of a gradient is cut where its tiles alone would leave SMs idle: time of the waves plus that of
// writing and joining the planes.
int plan_splits(int64_t m_tiles, int64_t n_tiles, int64_t steps, int64_t m, int64_t n, int slots)
{
    const int64_t tiles = m_tiles * n_tiles;
    int best = 1;
    double best_t = 0;
    for (int s = 1; s <= 64 && s <= steps; ++s) {
        const double waves = (double)ceil_div(tiles * s, slots);
        const double t = waves * ((double)ceil_div(steps, s) * 0.30e-6 + 1.0e-6) + (s > 1 ? 4e-6 + (double)s * m * n * 8.0 / 5e12 : 0.0);
        if (s == 1 || t < best_t * 0.97) {
            best = s;
            best_t = t;
        }
    }
    return best;
}

constexpr int64_t kPieceBytes = (int64_t)1 << 30;
constexpr int kBN = 256;

struct Plan {
    bool wide, half;
    int planes;
    int64_t n, v, d;
    bool pack_x, pack_w;
    int64_t pitch_d, ld_v;
    int64_t piece;     // rows per piece
    int splits_x, splits_w;
    // offsets into the workspace
    size_t x, w, stats, label_logit, store, p, acc, partial, lift, total;
};

Plan make_plan(const chicle_dense_t &X, const chicle_dense_t &W, bool grad)
{
    Plan p{};
    p.wide = X.type == CHICLE_F32;
    p.half = X.type == CHICLE_F16;
    p.planes = p.wide ? 3 : 1;
    p.n = X.rows, p.v = W.rows, p.d = X.cols;
    p.pack_x = grad || !takes_bulk(X);
    p.pack_w = !takes_bulk(W);
    p.pitch_d = (p.d + 7) / 8 * 8;
    p.ld_v = (p.v + 7) / 8 * 8;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    p.piece = p.n;
    if (grad) {
        int64_t rows = kPieceBytes / (p.ld_v * logit_bytes(p.wide)) / 256 * 256;
        // fewer than 2048 rows: the fp32 sums of dW would be read and written too often beside the products of a piece
        rows = std::max(rows, std::min<int64_t>(2048, 8 * kPieceBytes / (p.ld_v * logit_bytes(p.wide))));
        rows = std::max<int64_t>(rows, 256);
        if (rows < p.n) p.piece = ceil_div(ceil_div(p.n, ceil_div(p.n, rows)), 256) * 256;
    }
    if (p.pack_x) p.x = take((size_t)p.planes * p.n * p.pitch_d * 2);
    if (p.pack_w) p.w = take((size_t)p.planes * p.v * p.pitch_d * 2);
    p.stats = take((size_t)ceil_div(p.v, kHalfTile) * p.piece * sizeof(float2));
    p.label_logit = take((size_t)p.piece * 4);
    if (grad) {
        if (p.wide) {
            p.store = take((size_t)p.piece * p.ld_v * 4);
            p.p = take((size_t)3 * p.piece * p.ld_v * 2);
        } else {
            p.store = p.p = take((size_t)p.piece * p.ld_v * 2);
        }
        if (p.piece < p.n) p.acc = take((size_t)p.v * p.d * 4);
        const int pairs = p.wide ? 6 : 1;
        p.splits_x = plan_splits(ceil_div(p.piece, 128), ceil_div(p.d, kBN), ceil_div(p.v, tc::kBK) * pairs, p.piece, p.d, kSms);
        p.splits_w = plan_splits(ceil_div(p.v, 128), ceil_div(p.d, kBN), ceil_div(p.piece, tc::kBK) * pairs, p.v, p.d, kSms);
        size_t part = 0;
        if (p.splits_x > 1) part = (size_t)p.splits_x * p.piece * p.d * 4;
        if (p.splits_w > 1) part = std::max(part, (size_t)p.splits_w * p.v * p.d * 4);
        if (part) p.partial = take(part);
        p.lift = take(8);
    }
    p.total = at;
    return p;
}

cudaError_t pack(const chicle_dense_t &src, void *dst, const Plan &p, const int32_t *labels, int32_t classes, cudaStream_t s)
{
    const int64_t all = src.rows * (p.pitch_d / 8);
    const unsigned grid = (unsigned)std::min<int64_t>(ceil_div(all, 256), kSms * 16);
    const int64_t plane = src.rows * p.pitch_d;
    if (src.type == CHICLE_F32)
        k_pack<float, __nv_bfloat16><<<grid, 256, 0, s>>>((const float *)src.data, src.ld, src.rows, (int32_t)p.d, (__nv_bfloat16 *)dst, p.pitch_d, plane, labels, classes);
    else if (src.type == CHICLE_BF16)
        k_pack<__nv_bfloat16, __nv_bfloat16><<<grid, 256, 0, s>>>((const __nv_bfloat16 *)src.data, src.ld, src.rows, (int32_t)p.d, (__nv_bfloat16 *)dst, p.pitch_d, plane, labels, classes);
    else
        k_pack<__half, __half><<<grid, 256, 0, s>>>((const __half *)src.data, src.ld, src.rows, (int32_t)p.d, (__half *)dst, p.pitch_d, plane, labels, classes);
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

tc::Shape shape_of(const Plan &p, int64_t m, int64_t n, int64_t k, int splits, int group, uint32_t *status)
{
    tc::Shape s{};
    s.m = (int32_t)m, s.n = (int32_t)n;
    s.k_steps = (int32_t)ceil_div(k, tc::kBK);
    s.pairs = p.wide ? 6 : 1;
    s.splits = splits;
    s.group = group;
    s.half = p.half;
    s.status = status;
    return s;
}

cudaError_t join_blocks(const Plan &p, const float2 *stats, int64_t rows, const int32_t *labels, const float *label_logit, float *loss,
                        float *lse, uint32_t *status, cudaStream_t s)
{
    const int blocks = (int)ceil_div(p.v, kHalfTile);
    if (rows >= 32 * 64)
        k_join_blocks<32><<<(unsigned)ceil_div(rows, 32), 512, 0, s>>>(stats, blocks, (int32_t)rows, labels, (int32_t)p.v, label_logit, loss, lse, status);
    else if (rows >= 8)
        k_join_blocks<8><<<(unsigned)ceil_div(rows, 8), 512, 0, s>>>(stats, blocks, (int32_t)rows, labels, (int32_t)p.v, label_logit, loss, lse, status);
    else
        k_join_blocks<1><<<(unsigned)rows, 512, 0, s>>>(stats, blocks, (int32_t)rows, labels, (int32_t)p.v, label_logit, loss, lse, status);
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
    cudaError_t e = of_x ? launch_product<1, kBN, false, true>(a, b, s, epi, stream) : launch_product<1, kBN, true, true>(a, b, s, epi, stream);
    if (e == cudaSuccess && s.splits > 1) {
        const int64_t all = (int64_t)s.m * s.n;
        k_join_splits<OutT><<<(unsigned)std::min<int64_t>(ceil_div(all, 256), kSms * 8), 256, 0, stream>>>(
            epi.partial, s.splits, s.m, s.n, epi.add, epi.keep, epi.out, epi.ld, epi.scale, epi.labels, epi.classes);
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
    cudaError_t e = pack(X, ws + p.x, p, labels, (int32_t)p.v, stream);
    if (e == cudaSuccess && p.pack_w) e = pack(W, ws + p.w, p, nullptr, 0, stream);
    float *lift = nullptr;
    if (e == cudaSuccess && p.half) {
        lift = reinterpret_cast<float *>(ws + p.lift);
        k_lift<<<1, 1024, 0, stream>>>(weights, p.n, scale, lift);
        e = cudaGetLastError();
    }
    const Operand w = operand_of(W, ws + p.w, p.pack_w, p);
    for (int64_t r0 = 0; e == cudaSuccess && r0 < p.n; r0 += p.piece) {
        const int64_t rows = std::min(p.piece, p.n - r0);
        Operand x = operand_of(X, ws + p.x, true, p);
        x.data = static_cast<const uint16_t *>(x.data) + r0 * p.pitch_d;
        x.rows = rows;
        float2 *stats = reinterpret_cast<float2 *>(ws + p.stats);
        float *label_logit = reinterpret_cast<float *>(ws + p.label_logit);
        StoreT *store = reinterpret_cast<StoreT *>(ws + p.store);
        PT *prob = reinterpret_cast<PT *>(ws + p.p);
        const LogitsEpilogue<StoreT> le{labels + r0, stats, label_logit, store, p.ld_v};
        e = launch_product<1, kBN, false, false>(x, w, shape_of(p, rows, p.v, p.d, 1, group_of(p.d, p.planes, 128), status), le, stream);
        if (e == cudaSuccess) e = join_blocks(p, stats, rows, labels + r0, label_logit, loss + r0, lse + r0, status, stream);
        if (e != cudaSuccess) break;
        Operand q;
        q.data = prob;
        q.rows = rows, q.cols = p.v, q.pitch = p.ld_v, q.plane = p.piece * p.ld_v, q.planes = p.planes;
        for (int64_t y = 0; y < rows; y += 65535)
            k_probabilities<PT, kWide><<<dim3((unsigned)ceil_div(p.v, 2048), (unsigned)std::min<int64_t>(65535, rows - y)), 256, 0, stream>>>(
                store + y * p.ld_v, prob + y * p.ld_v, p.ld_v, q.plane, (int32_t)rows, (int32_t)p.v, stats + y, lse + r0 + y, loss + r0 + y,
                labels + r0 + y, weights ? weights + r0 + y : nullptr, scale, lift);
        if ((e = cudaGetLastError()) != cudaSuccess) break;
        const float *back = lift ? lift + 1 : nullptr;
        float *partial = reinterpret_cast<float *>(ws + p.partial);
        GradEpilogue<T> ex{static_cast<T *>(dX.data) + r0 * dX.ld, dX.ld, p.splits_x > 1 ? partial : nullptr, nullptr, nullptr, back, labels + r0, (int32_t)p.v};
        e = gradient<T>(p, q, w, true, shape_of(p, rows, p.d, p.v, p.splits_x, 8, status), ex, stream);
        if (e != cudaSuccess) break;
        // dW over the pieces: the sums stay in fp32 until the last
        const bool first = r0 == 0, last = r0 + rows >= p.n;
        GradEpilogue<T> ew{static_cast<T *>(dW.data), dW.ld, nullptr, nullptr, nullptr, back, nullptr, 0};
        float *acc = reinterpret_cast<float *>(ws + p.acc);
        if (!first) ew.add = acc;
        if (!last) ew.keep = acc;
        const int splits = (int)std::min<int64_t>(p.splits_w, ceil_div(rows, tc::kBK) * (kWide ? 6 : 1));
        if (splits > 1) ew.partial = partial;
        e = gradient<T>(p, q, x, false, shape_of(p, p.v, p.d, rows, splits, 8, status), ew, stream);
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

bool overlap(const chicle_dense_t &a, const chicle_dense_t &b)
{
    if (a.rows == 0 || b.rows == 0) return false;
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a.data), b0 = reinterpret_cast<uintptr_t>(b.data);
    const uintptr_t an = (uintptr_t)((a.rows - 1) * a.ld + a.cols) * (uintptr_t)element_size(a.type);
    const uintptr_t bn = (uintptr_t)((b.rows - 1) * b.ld + b.cols) * (uintptr_t)element_size(b.type);
    return a0 < b0 + bn && b0 < a0 + an;
}

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
    cudaError_t e = cudaSuccess;
    if (p.pack_x) e = pack(*X, ws + p.x, p, nullptr, 0, s);
    if (e == cudaSuccess && p.pack_w) e = pack(*W, ws + p.w, p, nullptr, 0, s);
    float2 *stats = reinterpret_cast<float2 *>(ws + p.stats);
    float *label_logit = reinterpret_cast<float *>(ws + p.label_logit);
    const LogitsEpilogue<NoStore> le{dev_labels, stats, label_logit, nullptr, 0};
    if (e == cudaSuccess)
        e = launch_product<1, kBN, false, false>(operand_of(*X, ws + p.x, p.pack_x, p), operand_of(*W, ws + p.w, p.pack_w, p),
                                                 shape_of(p, p.n, p.v, p.d, 1, group_of(p.d, p.planes, 128), dev_status), le, s);
    if (e == cudaSuccess) e = join_blocks(p, stats, p.n, dev_labels, label_logit, dev_loss, dev_lse, dev_status, s);
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
    if (overlap(*dX, *W) || overlap(*dW, *X) || overlap(*dW, *W) || overlap(*dX, *X) || overlap(*dX, *dW))
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
        e = run_grad<float, __nv_bfloat16, float>(p, *X, *W, dev_labels, dev_weights, scale, dev_loss, dev_lse, *dX, *dW, ws, dev_status, s);
    else if (X->type == CHICLE_BF16)
        e = run_grad<__nv_bfloat16, __nv_bfloat16, __half>(p, *X, *W, dev_labels, dev_weights, scale, dev_loss, dev_lse, *dX, *dW, ws, dev_status, s);
    else
        e = run_grad<__half, __half, __half>(p, *X, *W, dev_labels, dev_weights, scale, dev_loss, dev_lse, *dX, *dW, ws, dev_status, s);
    return e == cudaSuccess ? CHICLE_OK : err.cuda(e);
}
