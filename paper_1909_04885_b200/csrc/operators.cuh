// What the operators without a handle share (softmax.cu, embedding.cu, clip.cu): argument checks, error text, the device.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cstdio>

#include "chicle_internal.cuh"

namespace chicle {

constexpr int kSms = 148; // B200: grids and workspaces are planned for it, so that a workspace's size needs no device

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

inline int element_size(chicle_dtype_t t) { return t == CHICLE_F32 ? 4 : 2; }

// Whether two matrices have a byte in common. Exact where their rows are equally far apart (or one has a single row), so that
// they may lie side by side in one buffer; of rows at different distances the extents are compared.
inline bool overlapping(const chicle_dense_t &a, const chicle_dense_t &b)
{
    if (a.rows == 0 || b.rows == 0) return false;
    using Wide = __int128; // (rows times pitch may leave 64 bits)
    const Wide a0 = reinterpret_cast<uintptr_t>(a.data), b0 = reinterpret_cast<uintptr_t>(b.data);
    const Wide wa = a.cols * element_size(a.type), wb = b.cols * element_size(b.type); // bytes of a row
    const Wide pa = (Wide)a.ld * element_size(a.type), pb = (Wide)b.ld * element_size(b.type);
    if (a0 >= b0 + (b.rows - 1) * pb + wb || b0 >= a0 + (a.rows - 1) * pa + wa) return false;
    if ((a.rows == 1 && b.rows == 1) || (a.rows > 1 && b.rows > 1 && pa != pb)) return true;
    // b's row j and a's row i meet where -wb < b0 - a0 + k pitch < wa with k = j - i: the smallest k to the right of -wb decides
    const Wide pitch = a.rows > 1 ? pa : pb, from = a0 - b0 - wb;
    const Wide below = from >= 0 ? from / pitch : -((-from + pitch - 1) / pitch); // rounded down
    const Wide k = std::max<Wide>(below + 1, 1 - a.rows);
    return k < b.rows && b0 - a0 + k * pitch < wa;
}

// nullptr, or what is wrong with the description.
const char *check_dense(const chicle_dense_t *x);

inline const char *check_workspace(const void *ws, size_t have, size_t need)
{
    if (have < need || (need > 0 && !ws)) return "the workspace is smaller than the size query says";
    if (reinterpret_cast<uintptr_t>(ws) & 255) return "the workspace is not aligned to 256 bytes";
    return nullptr;
}

// Error text for a caller without a handle.
struct CallError {
    char *buf;
    size_t len;
    chicle_status_t operator()(chicle_status_t st, const char *text) const
    {
        if (buf && len) snprintf(buf, len, "%s", text);
        return st;
    }
    chicle_status_t cuda(cudaError_t e) const
    {
        (void)cudaGetLastError();
        return (*this)(e == cudaErrorMemoryAllocation ? CHICLE_ERR_OOM : CHICLE_ERR_CUDA, cudaGetErrorString(e));
    }
};

// Makes `device` current for the length of a call.
class DeviceGuard {
  public:
    explicit DeviceGuard(int device)
    {
        e_ = cudaGetDevice(&before_);
        if (e_ == cudaSuccess && before_ != device) {
            e_ = cudaSetDevice(device);
            changed_ = e_ == cudaSuccess;
        }
        if (e_ != cudaSuccess) (void)cudaGetLastError();
    }
    ~DeviceGuard()
    {
        if (changed_) (void)cudaSetDevice(before_);
    }
    DeviceGuard(const DeviceGuard &) = delete;
    DeviceGuard &operator=(const DeviceGuard &) = delete;
    bool ok() const { return e_ == cudaSuccess; }
    const char *message() const { return cudaGetErrorString(e_); }

  private:
    int before_ = 0;
    bool changed_ = false;
    cudaError_t e_ = cudaSuccess;
};

} // namespace chicle
