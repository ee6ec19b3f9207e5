// The three products of a linear layer and what follows them in the same kernel.
//   forward       y  = act(x W^T + b) + r       rows = tokens,  columns = n, sum over k
//   input grad    dx = (dz W + r) * act'(z)     rows = tokens,  columns = k, sum over n
//   weight grad   dW = dz^T x                   rows = n,       columns = k, sum over tokens
#pragma once

#include "kernels_checkpoint.cuh"

namespace eden {

enum { kForward = 0, kInputGrad = 1, kWeightGrad = 2 };

struct LinearEpilogue {
    const void* bias;                  // forward
    const void* residual;              // forward, input grad
    uint64_t residual_stride;
    void* out;
    uint64_t out_stride;
    CheckpointView ckpt;               // forward: what is saved; input grad: the pre-activation
    float* column_sums;                // input grad: [ceil(rows / 32)][cols] sums of 32 rows, or null
    uint64_t rows, cols;
    int act, save, accumulate;
};

// v[32]: fp32 sums of one row's columns col0 .. col0 + 31, held by the lane that owns the
// row.  All 32 lanes of the warp call this together, for rows row0 + lane (row0 % 32 == 0)
// and the same col0 (col0 % 32 == 0), also where the row is past the last one.
template <int OP, typename T>
__device__ __forceinline__ void linear_epilogue(float (&v)[32], uint64_t row, uint64_t col0, const LinearEpilogue& p)
{
    const bool live = row < p.rows;
    const int count = (int)(p.cols - col0 < 32 ? p.cols - col0 : 32);
    if constexpr (OP == kWeightGrad) {
        if (!live) return;
        float* out = (float*)p.out + row * p.out_stride + col0;
#pragma unroll
        for (int j = 0; j < 32; ++j)
            if (j < count) out[j] = p.accumulate ? out[j] + v[j] : v[j];
        return;
    }
    const T* residual = p.residual && live ? (const T*)p.residual + row * p.residual_stride + col0 : nullptr;
    if constexpr (OP == kForward) {
        if (p.bias) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if (j < count) v[j] += to_float(((const T*)p.bias)[col0 + j]);
        }
        auto save = [&]() {
            if (!live) return;
            uint32_t most = 0;
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if (j < count) most = max(most, magnitude_bits(v[j]));
            const uint32_t e = group_exponent(most);
            const float inverse = group_inverse(e);
            p.ckpt.exps[row * p.ckpt.exps_stride + col0 / kGroup] = (uint8_t)e;
            int8_t* codes = p.ckpt.codes + row * p.ckpt.codes_stride + col0;
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if (j < count) codes[j] = (int8_t)group_code(v[j], inverse);
        };
        if (p.save == EDEN_SAVE_PRE) save();
        with_act(p.act, [&](auto a) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = act_value<decltype(a)::value>(v[j]);
        });
        if (residual) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if (j < count) v[j] += to_float(residual[j]);
        }
        if (p.save == EDEN_SAVE_OUT) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = to_float(from_float<T>(v[j]));
            save();
        }
    } else {
        if (residual) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if (j < count) v[j] += to_float(residual[j]);
        }
        if (p.act != EDEN_ACT_NONE) {
            const int8_t* codes = p.ckpt.codes + row * p.ckpt.codes_stride + col0;
            const float scale = live ? group_scale(p.ckpt.exps[row * p.ckpt.exps_stride + col0 / kGroup]) : 0.f;
            with_act(p.act, [&](auto a) {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (live && j < count) v[j] *= act_slope<decltype(a)::value>(code_value(codes[j], scale));
            });
        }
        if (p.column_sums) {
            // lane j ends with the sum of column j: halves are exchanged and added five times
            float s[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) s[j] = live ? v[j] : 0.f;
            const int lane = threadIdx.x % 32;
#pragma unroll
            for (int half = 16; half >= 1; half /= 2) {
                const bool upper = lane & half;
#pragma unroll
                for (int j = 0; j < half; ++j) {
                    const float keep = upper ? s[j + half] : s[j], give = upper ? s[j] : s[j + half];
                    s[j] = keep + __shfl_xor_sync(0xFFFFFFFFu, give, half);
                }
            }
            if (lane < count) p.column_sums[row / 32 * p.cols + col0 + lane] = s[0];
        }
    }
    if (live) {
        T* out = (T*)p.out + row * p.out_stride + col0;
#pragma unroll
        for (int j = 0; j < 32; ++j)
            if (j < count) out[j] = from_float<T>(v[j]);
    }
}

struct LinearOperands {
    const void *a, *b;
    uint64_t a_stride, b_stride;
    uint64_t depth;                    // length of the sum
};

// A block of 128 threads takes 128 rows x 32 columns, one row per thread.
template <int OP, typename T>
__global__ void __launch_bounds__(128) k_linear_simple(LinearOperands g, LinearEpilogue p)
{
    __shared__ float sa[32][129], sb[32][32];
    const uint64_t col_tiles = (p.cols + 31) / 32;
    const uint64_t row0 = blockIdx.x / col_tiles * 128, col0 = blockIdx.x % col_tiles * 32;
    const T *a = (const T*)g.a, *b = (const T*)g.b;
    const int t = threadIdx.x;
    float v[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = 0.f;
    for (uint64_t d0 = 0; d0 < g.depth; d0 += 32) {
        for (int i = t; i < 32 * 128; i += 128) {
            const int d = OP == kWeightGrad ? i / 128 : i % 32, r = OP == kWeightGrad ? i % 128 : i / 32;
            const uint64_t row = row0 + r, dep = d0 + d;
            sa[d][r] = row < p.rows && dep < g.depth ? to_float(a[OP == kWeightGrad ? dep * g.a_stride + row : row * g.a_stride + dep]) : 0.f;
        }
        for (int i = t; i < 32 * 32; i += 128) {
            const int d = OP == kForward ? i % 32 : i / 32, c = OP == kForward ? i / 32 : i % 32;
            const uint64_t col = col0 + c, dep = d0 + d;
            sb[d][c] = col < p.cols && dep < g.depth ? to_float(b[OP == kForward ? col * g.b_stride + dep : dep * g.b_stride + col]) : 0.f;
        }
        __syncthreads();
        for (int d = 0; d < 32; ++d) {
            const float x = sa[d][t];
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] += x * sb[d][j];
        }
        __syncthreads();
    }
    linear_epilogue<OP, T>(v, row0 + t, col0, p);
}

}  // namespace eden
