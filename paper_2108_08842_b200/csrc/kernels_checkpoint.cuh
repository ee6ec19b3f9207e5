// 8-bit checkpoints of activations: save, restore, and the gradient of an activation whose
// argument is a checkpoint.
#pragma once

#include "train_device.cuh"

namespace eden {

struct CheckpointView {
    int8_t* codes;
    uint64_t codes_stride;
    uint8_t* exps;
    uint64_t exps_stride;
};

constexpr int kCkptThreads = 256;

// One warp per group, one value per lane: any alignment, any row length.
template <typename T>
__global__ void __launch_bounds__(kCkptThreads) k_checkpoint_save(const T* __restrict__ x, uint64_t x_stride,
                                                                 CheckpointView c, uint64_t n, uint64_t groups, uint64_t total)
{
    const uint64_t warp = (uint64_t)blockIdx.x * (kCkptThreads / 32) + threadIdx.x / 32;
    if (warp >= total) return;
    const uint64_t row = warp / groups, group = warp % groups, col = group * kGroup + threadIdx.x % 32;
    const float v = col < n ? to_float(x[row * x_stride + col]) : 0.f;
    const uint32_t e = group_exponent(__reduce_max_sync(0xFFFFFFFFu, magnitude_bits(v)));
    if (col < n) c.codes[row * c.codes_stride + col] = (int8_t)group_code(v, group_inverse(e));
    if (threadIdx.x % 32 == 0) c.exps[row * c.exps_stride + group] = (uint8_t)e;
}

template <typename T>
__global__ void __launch_bounds__(kCkptThreads) k_checkpoint_restore(T* __restrict__ x, uint64_t x_stride,
                                                                    CheckpointView c, uint64_t n, uint64_t groups, uint64_t total)
{
    const uint64_t warp = (uint64_t)blockIdx.x * (kCkptThreads / 32) + threadIdx.x / 32;
    if (warp >= total) return;
    const uint64_t row = warp / groups, group = warp % groups, col = group * kGroup + threadIdx.x % 32;
    if (col >= n) return;
    x[row * x_stride + col] = restored<T>(code_value(c.codes[row * c.codes_stride + col], group_scale(c.exps[row * c.exps_stride + group])));
}

// dz = dy * act'(z), one lane per column: a block takes 32 columns of a run of rows and
// leaves the run's column sums in partial[run][n].
template <typename T>
__global__ void __launch_bounds__(kCkptThreads) k_act_backward(const T* dy, uint64_t dy_stride, CheckpointView pre, T* dz,
                                                              uint64_t dz_stride, float* __restrict__ partial, uint64_t m,
                                                              uint64_t n, uint64_t rows_per_run, int act)
{
    const uint64_t group = blockIdx.x, col = group * kGroup + threadIdx.x % 32;
    const uint64_t begin = (uint64_t)blockIdx.y * rows_per_run, end = begin + rows_per_run < m ? begin + rows_per_run : m;
    float sum = 0.f;
    if (col < n) {
        with_act(act, [&](auto a) {
            for (uint64_t row = begin + threadIdx.x / 32; row < end; row += kCkptThreads / 32) {
                float v = to_float(dy[row * dy_stride + col]);
                if constexpr (decltype(a)::value != EDEN_ACT_NONE)
                    v *= act_slope<decltype(a)::value>(code_value(pre.codes[row * pre.codes_stride + col],
                                                                  group_scale(pre.exps[row * pre.exps_stride + group])));
                sum += v;
                if (dz) dz[row * dz_stride + col] = from_float<T>(v);
            }
        });
    }
    if (!partial) return;
    __shared__ float sums[kCkptThreads / 32][32];
    sums[threadIdx.x / 32][threadIdx.x % 32] = sum;
    __syncthreads();
    if (threadIdx.x < 32 && col < n) {
        float total = 0.f;
        for (int w = 0; w < kCkptThreads / 32; ++w) total += sums[w][threadIdx.x];
        partial[(uint64_t)blockIdx.y * n + col] = total;
    }
}

// out[n] (+)= the sum of partial's rows, in their order
__global__ void __launch_bounds__(kCkptThreads) k_column_sum(const float* __restrict__ partial, uint64_t rows, uint64_t n,
                                                            float* __restrict__ out, int accumulate)
{
    const uint64_t col = (uint64_t)blockIdx.x * kCkptThreads + threadIdx.x;
    if (col >= n) return;
    float sum = 0.f;
    for (uint64_t r = 0; r < rows; ++r) sum += partial[r * n + col];
    out[col] = accumulate ? out[col] + sum : sum;
}

}  // namespace eden
