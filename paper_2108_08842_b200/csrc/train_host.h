// What the host side of the training step's entry points shares: checks of arguments, scratch from
// the context's workspace, launches.
#pragma once

#include <algorithm>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "context.h"
#include "kernels_checkpoint.cuh"

namespace eden {
namespace {

constexpr uint64_t kStatusBytes = 256;          // start of the workspace: the status word
constexpr uint64_t kMaxCount = (1ull << 31) - 1;

uint64_t align_to(uint64_t v, uint64_t a) { return (v + a - 1) / a * a; }
uint64_t groups_of(uint64_t n) { return (n + kGroup - 1) / kGroup; }
uint64_t padded(uint64_t n) { return align_to(n, 16); }          // 32-byte rows of a 16-bit matrix

// The caller's current device stays what it was.
struct DeviceGuard {
    int before = -1;
    bool ok;
    explicit DeviceGuard(int device)
    {
        ok = cudaGetDevice(&before) == cudaSuccess && (before == device || cudaSetDevice(device) == cudaSuccess);
        if (before == device) before = -1;
    }
    ~DeviceGuard() { if (before >= 0) cudaSetDevice(before); }
};

// Scratch of one call, carved from the context's workspace behind the status word.
struct Scratch {
    char* base;
    uint64_t used, size;
    explicit Scratch(const eden_ctx* ctx) : base(ctx->ws), used(kStatusBytes), size(ctx->ws_bytes) {}
    template <typename U> U* take(uint64_t count)
    {
        const uint64_t at = used, end = at + align_to(count * sizeof(U), 256);
        if (end > size) return nullptr;
        used = end;
        return (U*)(base + at);
    }
};

bool aligned(const void* p, size_t size) { return ((uintptr_t)p & (size - 1)) == 0; }

bool wide_rows(const void* p, uint64_t stride, size_t size) { return aligned(p, 32) && stride * size % 32 == 0; }

bool half_type(int type) { return type == EDEN_TYPE_BF16 || type == EDEN_TYPE_FP16; }
bool known_act(int act) { return act >= EDEN_ACT_NONE && act <= EDEN_ACT_SILU; }

// a matrix of `size`-byte elements with rows of n
bool matrix_ok(const void* p, uint64_t stride, uint64_t n, size_t size) { return p && aligned(p, size) && stride >= n; }
bool optional_ok(const void* p, uint64_t stride, uint64_t n, size_t size) { return !p || matrix_ok(p, stride, n, size); }
bool checkpoint_ok(const int8_t* codes, uint64_t cs, const uint8_t* exps, uint64_t es, uint64_t n)
{
    return codes && exps && cs >= n && es >= groups_of(n);
}

int counts_ok(uint64_t m, uint64_t n, uint64_t k)
{
    if (n == 0 || k == 0) return EDEN_ERR_INVALID_ARG;
    return std::max(m, std::max(n, k)) > kMaxCount ? EDEN_ERR_TOO_LARGE : EDEN_OK;
}

// f(T{}) with the type behind an EDEN_TYPE_* of 16 bits
#define EDEN_DISPATCH_HALF(type, CALL)                                      \
    if ((type) == EDEN_TYPE_BF16) { using T_ = __nv_bfloat16; CALL; }        \
    else { using T_ = __half; CALL; }

#define EDEN_DISPATCH_TYPE(type, CALL)                                      \
    if ((type) == EDEN_TYPE_BF16) { using T_ = __nv_bfloat16; CALL; }        \
    else if ((type) == EDEN_TYPE_FP16) { using T_ = __half; CALL; }          \
    else { using T_ = float; CALL; }

size_t type_size(int type) { return type == EDEN_TYPE_FP32 ? 4 : 2; }

CheckpointView view(const int8_t* codes, uint64_t cs, const uint8_t* exps, uint64_t es)
{
    return {const_cast<int8_t*>(codes), cs, const_cast<uint8_t*>(exps), es};
}

// A launch that may begin before the stream's previous kernel has ended: kernels launched so
// wait for it themselves (dependency_wait).  cluster = blocks per cluster, along x, or along
// y where the grid is that high.
template <typename... KArgs, typename... Args>
int launch(eden_ctx* ctx, const char* name, double bytes, void (*kernel)(KArgs...), dim3 grid, uint32_t block, uint32_t shared,
           uint32_t cluster, Args&&... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = shared;
    cfg.stream = ctx->stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim = {grid.y == cluster ? 1 : cluster, grid.y == cluster ? cluster : 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    profile_begin(ctx, name, bytes);
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, KArgs(args)...);
    profile_end(ctx);
    ++ctx->launches;
    CUDA_OK(e);
    return EDEN_OK;
}

// partial [rows][n] -> out [n]
int sum_columns(eden_ctx* ctx, const float* partial, uint64_t rows, uint64_t n, float* out, int accumulate)
{
    return launch(ctx, "t_column_sum", 4.0 * (double)(rows + 1) * n, k_column_sum, dim3((uint32_t)((n + 31) / 32)), kCkptThreads, 0, 1,
                  partial, rows, n, out, accumulate);
}

// Nothing throws across the C boundary: the launch records grow a vector while profiling.
template <typename F>
int guarded(eden_ctx* ctx, F&& f)
{
    DeviceGuard device(ctx->device);
    CUDA_OK(device.ok ? cudaSuccess : cudaErrorInvalidDevice);
    ctx->order.clear();                          // the workspace no longer holds a call's client figures
    try {
        return f();
    } catch (...) {
        return EDEN_ERR_INVALID_ARG;
    }
}

}  // namespace
}  // namespace eden
