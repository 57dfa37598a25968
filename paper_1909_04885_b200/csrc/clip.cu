// The common norm of many tensors, and clipping by it (chicle_clip_gradients).
//
//   N = sqrt(sum g^2),  g' = g min(1, max_norm / (N + 1e-6))
//
// Two launches whatever the number of tensors (up to 512): their table travels as a kernel argument. The first adds the
// squares, CTA by CTA in a fixed order; in the second every CTA joins the CTAs' sums and scales its share, in the
// opposite order, so that what the first launch read last is still in L2. Bound by memory: two reads and one write.
//
// Squares are added in fp32 eight at a time and then in fp64, unless the largest of the eight would leave fp32's range
// when squared: those are squared in fp64.
#include <algorithm>
#include <cmath>
#include <vector>

#include "operators.cuh"

namespace chicle {
namespace {

constexpr int kMost = 512;            // tensors per launch
constexpr int kFew = 96;              // up to so many, a launch with a smaller argument
constexpr int kChunk = 16384;         // elements that a CTA takes at a time
constexpr int kBlocks = 148 * 8;      // CTAs, and words of workspace
static_assert(kBlocks * sizeof(double) <= CHICLE_CLIP_WORKSPACE, "workspace");

template <int M> struct Table {
    const void *in[M];
    void *out[M];
    int64_t n[M];
    uint32_t end[M]; // chunks up to and with this tensor
    uint8_t type[M];
    int32_t count;
};

template <typename T> __device__ __forceinline__ T rounded(float v);
template <> __device__ __forceinline__ float rounded<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 rounded<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half rounded<__half>(float v) { return __float2half_rn(v); }

// Tensor of a chunk, and its place in it.
template <int M> __device__ __forceinline__ int tensor_of(const Table<M> &t, uint32_t chunk, int64_t &first)
{
    int lo = 0, hi = t.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (chunk < t.end[mid]) hi = mid;
        else lo = mid + 1;
    }
    first = (int64_t)(chunk - (lo ? t.end[lo - 1] : 0u)) * kChunk;
    return lo;
}

// Elements in front of the first 16-byte boundary.
template <typename T> __device__ __forceinline__ int head_of(const T *p, int len)
{
    return min(len, (int)(((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / sizeof(T)));
}

template <int E> __device__ __forceinline__ double squares(const float (&v)[E])
{
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < E; ++j) top = fmaxf(top, fabsf(v[j]));
    if (top < 1e18f && top > 1e-14f) { // (a NaN passes fmaxf: the sum has it)
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < E; ++j) s[j & 1] = fmaf(v[j], v[j], s[j & 1]);
        return (double)(s[0] + s[1]);
    }
    double s = 0.0;
#pragma unroll
    for (int j = 0; j < E; ++j) s = fma((double)v[j], (double)v[j], s);
    return s;
}

template <typename T> __device__ __forceinline__ double chunk_squares(const T *p, int len)
{
    constexpr int kPer = 16 / (int)sizeof(T);
    const int head = head_of(p, len), vecs = (len - head) / kPer;
    const uint4 *q = reinterpret_cast<const uint4 *>(p + head);
    double s = 0.0;
#pragma unroll 4
    for (int j = threadIdx.x; j < vecs; j += 256) {
        const uint4 x = q[j];
        const T *e = reinterpret_cast<const T *>(&x);
        float v[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i) v[i] = (float)e[i];
        s += squares<kPer>(v);
    }
    const int rest = len - vecs * kPer; // in front and behind
    if ((int)threadIdx.x < rest) {
        const int i = (int)threadIdx.x < head ? threadIdx.x : threadIdx.x + vecs * kPer;
        const double v = (double)(float)p[i];
        s += v * v;
    }
    return s;
}

__device__ __forceinline__ double block_sum(double s)
{
    __shared__ double part[8];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int w = 0; w < 8; ++w) s += part[w];
    __syncthreads();
    return s;
}

template <int M>
__global__ void __launch_bounds__(256) k_squares(const __grid_constant__ Table<M> t, uint32_t chunks, double *__restrict__ sums, bool first)
{
    double s = 0.0;
    for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
        int64_t at;
        const int k = tensor_of(t, c, at);
        const int len = (int)min((int64_t)kChunk, t.n[k] - at);
        if (t.type[k] == CHICLE_F32) s += chunk_squares(static_cast<const float *>(t.in[k]) + at, len);
        else if (t.type[k] == CHICLE_BF16) s += chunk_squares(static_cast<const __nv_bfloat16 *>(t.in[k]) + at, len);
        else s += chunk_squares(static_cast<const __half *>(t.in[k]) + at, len);
    }
    s = block_sum(s);
    if (threadIdx.x == 0) sums[blockIdx.x] = first ? s : sums[blockIdx.x] + s;
}

// The factor as two: below fp32's normal range it would lose its bits, a power of two in front of it takes them back.
struct Factor {
    float power, rest;
    __device__ __forceinline__ explicit Factor(double f) : power(f < 0x1p-100 ? 0x1p-64f : 1.f), rest((float)(f < 0x1p-100 ? f * 0x1p64 : f)) {}
    __device__ __forceinline__ float operator()(float v) const { return (v * power) * rest; }
};

template <typename T> __device__ __forceinline__ void chunk_scale(const T *p, T *o, int len, const Factor &f)
{
    constexpr int kPer = 16 / (int)sizeof(T);
    // (in and out at different places within 16 bytes: element by element)
    const bool alike = ((reinterpret_cast<uintptr_t>(p) ^ reinterpret_cast<uintptr_t>(o)) & 15) == 0;
    const int head = alike ? head_of(p, len) : len, vecs = (len - head) / kPer;
    const uint4 *q = reinterpret_cast<const uint4 *>(p + head);
    uint4 *r = reinterpret_cast<uint4 *>(o + head);
#pragma unroll 4
    for (int j = threadIdx.x; j < vecs; j += 256) {
        uint4 x = q[j];
        T *e = reinterpret_cast<T *>(&x);
#pragma unroll
        for (int i = 0; i < kPer; ++i) e[i] = rounded<T>(f((float)e[i]));
        r[j] = x;
    }
    const int rest = len - vecs * kPer;
    for (int j = threadIdx.x; j < rest; j += 256) {
        const int i = j < head ? j : j + vecs * kPer;
        o[i] = rounded<T>(f((float)p[i]));
    }
}

template <int M>
__global__ void __launch_bounds__(256) k_scale(const __grid_constant__ Table<M> t, uint32_t chunks, const double *__restrict__ sums, int n_sums,
                                               float max_norm, float *norm)
{
    double s = 0.0;
    for (int i = threadIdx.x; i < n_sums; i += 256) s += sums[i];
    const double total = sqrt(block_sum(s));
    // (what the caller sees decides: a norm beyond fp32 is shown as infinity, and the elements stay)
    const float shown = (float)total;
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm = shown;
    const double f64 = (double)max_norm / (total + 1e-6);
    const Factor f(f64 < 1.0 && shown < INFINITY ? f64 : 1.0); // (a NaN fails both)
    for (uint32_t i = blockIdx.x; i < chunks; i += gridDim.x) {
        const uint32_t c = chunks - 1 - i;
        int64_t at;
        const int k = tensor_of(t, c, at);
        if (!t.out[k] || (f.power * f.rest == 1.f && t.out[k] == t.in[k])) continue;
        const int len = (int)min((int64_t)kChunk, t.n[k] - at);
        if (t.type[k] == CHICLE_F32) chunk_scale(static_cast<const float *>(t.in[k]) + at, static_cast<float *>(t.out[k]) + at, len, f);
        else if (t.type[k] == CHICLE_BF16)
            chunk_scale(static_cast<const __nv_bfloat16 *>(t.in[k]) + at, static_cast<__nv_bfloat16 *>(t.out[k]) + at, len, f);
        else chunk_scale(static_cast<const __half *>(t.in[k]) + at, static_cast<__half *>(t.out[k]) + at, len, f);
    }
}

// Whether elements that one tensor's result goes to are read or written for another one too (the same tensor listed twice, say):
// CTAs would race on them.
bool results_overlap(const chicle_tensor_t *x, int64_t count)
{
    struct Span {
        uintptr_t from, to;
        bool written;
    };
    std::vector<Span> spans;
    spans.reserve((size_t)count * 2);
    for (int64_t i = 0; i < count; ++i) {
        if (x[i].n == 0) continue;
        const uintptr_t bytes = (uintptr_t)x[i].n * (x[i].type == CHICLE_F32 ? 4 : 2);
        const uintptr_t a = reinterpret_cast<uintptr_t>(x[i].in), b = reinterpret_cast<uintptr_t>(x[i].out);
        if (b) spans.push_back({b, b + bytes, true});
        if (a != b) spans.push_back({a, a + bytes, false});
    }
    const auto before = [](const Span &p, const Span &q) { return p.from < q.from; };
    if (!std::is_sorted(spans.begin(), spans.end(), before)) std::sort(spans.begin(), spans.end(), before);
    uintptr_t any = 0, written = 0; // where the spans so far end
    for (const Span &s : spans) {
        if (s.from < (s.written ? any : written)) return true;
        any = std::max(any, s.to);
        if (s.written) written = std::max(written, s.to);
    }
    return false;
}

struct Call {
    const chicle_tensor_t *tensors;
    int64_t count;
    float max_norm;
    float *norm;
    double *sums;
    cudaStream_t stream;
};

// Launches take up to M tensors and 2^31 chunks. Their CTAs' sums are added to the same words.
template <int M> cudaError_t run(const Call &c)
{
    cudaError_t e = cudaSuccess;
    int n_sums = 1;
    for (int phase = 0; phase < 2 && e == cudaSuccess; ++phase) {
        int64_t i = 0;
        bool first = true;
        do {
            Table<M> t;
            t.count = 0;
            uint64_t chunks = 0;
            bool any_out = false;
            for (; i < c.count && t.count < M; ++i) {
                const chicle_tensor_t &x = c.tensors[i];
                if (x.n == 0) continue;
                const uint64_t more = (uint64_t)ceil_div(x.n, kChunk);
                if (t.count && chunks + more > 0x7fffffffu) break;
                chunks += more;
                t.in[t.count] = x.in;
                t.out[t.count] = x.out;
                t.n[t.count] = x.n;
                t.type[t.count] = (uint8_t)x.type;
                t.end[t.count++] = (uint32_t)chunks;
                any_out |= x.out != nullptr;
            }
            const unsigned grid = (unsigned)std::max<uint64_t>(1, std::min<uint64_t>(chunks, kBlocks));
            if (phase == 0) {
                if (first) n_sums = (int)grid;
                // (the launches behind the first keep to its words)
                k_squares<M><<<first ? grid : std::min<unsigned>(grid, (unsigned)n_sums), 256, 0, c.stream>>>(t, (uint32_t)chunks, c.sums, first);
                e = cudaGetLastError();
            } else if (first || any_out) {
                k_scale<M><<<any_out ? grid : 1, 256, 0, c.stream>>>(t, any_out ? (uint32_t)chunks : 0u, c.sums, n_sums, c.max_norm, c.norm);
                e = cudaGetLastError();
            }
            first = false;
        } while (i < c.count && e == cudaSuccess);
    }
    return e;
}

} // namespace
} // namespace chicle

using namespace chicle;

extern "C" chicle_status_t chicle_clip_gradients(int device, void *cuda_stream, int64_t count, const chicle_tensor_t *host_tensors, float max_norm,
                                                 float *dev_norm, void *dev_workspace, size_t workspace_bytes, char *host_errbuf,
                                                 size_t errbuf_len)
{
    const CallError err{host_errbuf, errbuf_len};
    if (count < 0 || (count > 0 && !host_tensors)) return err(CHICLE_ERR_INVALID_ARG, "count < 0 or the tensors are NULL");
    if (!(max_norm >= 0.f)) return err(CHICLE_ERR_INVALID_ARG, "max_norm must be >= 0");
    if (!dev_norm) return err(CHICLE_ERR_INVALID_ARG, "norm must be a non-NULL device pointer");
    if (const char *m = check_workspace(dev_workspace, workspace_bytes, CHICLE_CLIP_WORKSPACE)) return err(CHICLE_ERR_INVALID_ARG, m);
    for (int64_t i = 0; i < count; ++i) {
        const chicle_tensor_t &x = host_tensors[i];
        if ((int)x.type < 0 || (int)x.type > 2) return err(CHICLE_ERR_INVALID_ARG, "unknown element type");
        if (x.n < 0 || x.n > ((int64_t)1 << 40)) return err(CHICLE_ERR_INVALID_ARG, "a tensor's length is negative or above 2^40");
        if (x.n > 0 && !x.in) return err(CHICLE_ERR_INVALID_ARG, "a tensor's data is NULL");
        const uintptr_t es = x.type == CHICLE_F32 ? 4 : 2, a = reinterpret_cast<uintptr_t>(x.in), b = reinterpret_cast<uintptr_t>(x.out);
        if (a % es || b % es) return err(CHICLE_ERR_INVALID_ARG, "data is not aligned to its element type");
    }
    try {
        if (results_overlap(host_tensors, count))
            return err(CHICLE_ERR_INVALID_ARG, "a tensor's out must be its in, or overlap neither an in nor another out (is a tensor listed twice?)");
    } catch (...) {
        return err(CHICLE_ERR_OOM, "host allocation failed");
    }
    const DeviceGuard guard(device);
    if (!guard.ok()) return err(CHICLE_ERR_CUDA, guard.message());
    const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    const Call call{host_tensors, count, max_norm, dev_norm, static_cast<double *>(dev_workspace), s};
    const cudaError_t e = count <= kFew ? run<kFew>(call) : run<kMost>(call);
    return e == cudaSuccess ? CHICLE_OK : err.cuda(e);
}
