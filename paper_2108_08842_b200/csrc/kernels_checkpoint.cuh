// 8-bit checkpoints of activations: save, restore, and the gradient of an activation whose
// argument is a checkpoint.  All three move a few bytes per value and compute little: HBM
// bounds them, so what counts is enough bytes in flight (32 bytes per thread and load).
#pragma once

#include "train_device.cuh"

namespace eden {

constexpr int kCkptThreads = 256;

// A thread takes half a group: 16 values, 32 bytes of a 16-bit type (fp32: 64) and 16 codes.
// `halves` = 2 * groups of a row, so that the halves of a group sit in neighbouring lanes.
// WIDE: rows of values start on 32 bytes and rows of codes on 16, and full half groups move in
// one access each; else loads are put together from the aligned chunks that they touch.
// A value per lane, the simple form for any alignment, took 41 us to save and restore
// 5368 x 1116 fp16, against 12 us.
template <bool WIDE, typename T>
__device__ __forceinline__ void load_values(const T* p, int count, uint32_t (&w)[4 * sizeof(T)])
{
    if (WIDE && count >= 16) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) load_32b((const char*)p + 32 * i, *(uint32_t(*)[8])(w + 8 * i));
    } else if constexpr (!WIDE) {
        load_shifted(p, count * (int)sizeof(T), w);
    } else {                                                 // the end of a row
#pragma unroll
        for (int j = 0; j < 4 * (int)sizeof(T); ++j) {
            if constexpr (sizeof(T) == 4) {
                w[j] = j < count ? ((const uint32_t*)p)[j] : 0;
            } else {
                const uint32_t lo = 2 * j < count ? ((const uint16_t*)p)[2 * j] : 0, hi = 2 * j + 1 < count ? ((const uint16_t*)p)[2 * j + 1] : 0;
                w[j] = lo | hi << 16;
            }
        }
    }
}

template <typename T>
__device__ __forceinline__ void store_values(T* p, int count, const float (&v)[16])
{
    if (count >= 16) {
        uint32_t w[4 * sizeof(T)];
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int j = 0; j < 16; ++j) w[j] = __float_as_uint(v[j]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = pack<T>(v[2 * j], v[2 * j + 1]);
        }
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) store_32b((char*)p + 32 * i, *(const uint32_t(*)[8])(w + 8 * i));
    } else {
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (j < count) p[j] = from_float<T>(v[j]);
    }
}

template <typename T>
__device__ __forceinline__ void widen(const uint32_t (&w)[4 * sizeof(T)], float (&v)[16])
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j] = __uint_as_float(w[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) unpack<T>(w[j], v[2 * j], v[2 * j + 1]);
    }
}

template <bool WIDE>
__device__ __forceinline__ void load_codes(const int8_t* p, int count, uint32_t (&w)[4])
{
    if (WIDE && count >= 16) {
        *(uint4*)w = *(const uint4*)p;
    } else if constexpr (!WIDE) {
        load_shifted(p, count, w);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = 0;
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (j < count) w[j / 4] |= (uint32_t)(uint8_t)p[j] << 8 * (j % 4);
    }
}

template <typename T, bool WIDE>
__global__ void __launch_bounds__(kCkptThreads) k_checkpoint_save(const T* x, uint64_t x_stride, CheckpointView c, uint32_t n,
                                                                 uint32_t halves, uint64_t total)
{
    dependency_wait();
    dependency_release();
    const uint64_t i = (uint64_t)blockIdx.x * kCkptThreads + threadIdx.x;
    const uint64_t row = total <= 0xFFFFFFFFull ? (uint32_t)i / halves : i / halves;
    const uint32_t half = (uint32_t)(i - row * halves), col = half * 16;
    const bool live = i < total;
    const int count = live && col < n ? (int)min(n - col, 16u) : 0;
    uint32_t raw[4 * sizeof(T)];
    float v[16];
    load_values<WIDE>(x + (live ? row * x_stride + col : 0), count, raw);
    widen<T>(raw, v);
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < 16; j += 2) top = max_magnitude(top, v[j], v[j + 1]);
    uint32_t most = magnitude_bits(top);
    most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
    const uint32_t e = group_exponent(most);
    const float inverse = group_inverse(e);
    if (!live) return;
    if ((half & 1) == 0) c.exps[row * c.exps_stride + half / 2] = (uint8_t)e;
    int8_t* codes = c.codes + row * c.codes_stride + col;
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = group_codes(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3], inverse);
    if (WIDE && count == 16) *(uint4*)codes = make_uint4(w[0], w[1], w[2], w[3]);
    else store_shifted(codes, count, w);
}

// Without WIDE the warp hands its 32 x 16 values round in shared memory and stores them one
// after the other, a lane each: words put together by every thread for its own half group lie 32
// bytes apart across the lanes, and took 206 us for 16384 x 4096 bf16 against 54 us.
template <typename T, bool WIDE>
__global__ void __launch_bounds__(kCkptThreads) k_checkpoint_restore(T* x, uint64_t x_stride, CheckpointView c, uint32_t n,
                                                                    uint32_t halves, uint64_t total)
{
    dependency_wait();
    dependency_release();
    const uint64_t i = (uint64_t)blockIdx.x * kCkptThreads + threadIdx.x;
    const uint64_t row = total <= 0xFFFFFFFFull ? (uint32_t)i / halves : i / halves;
    const uint32_t half = (uint32_t)(i - row * halves), col = half * 16;
    const int count = i < total && col < n ? (int)min(n - col, 16u) : 0;
    if (WIDE && count == 0) return;
    float v[16];
    if (count > 0) {
        const uint32_t e = c.exps[row * c.exps_stride + half / 2];
        uint32_t w[4];
        load_codes<WIDE>(c.codes + row * c.codes_stride + col, count, w);
        const Pair scale(group_scale(e));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            Pair v01, v23;
            code_values(w[j], scale, v01, v23);
            v01.get(v[4 * j], v[4 * j + 1]);
            v23.get(v[4 * j + 2], v[4 * j + 3]);
        }
        if (e >= kSaturates<T>) {
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = saturated<T>(v[j]);
        }
    }
    T* to = x + row * x_stride + col;
    if constexpr (WIDE) {
        store_values(to, count, v);
    } else {
        __shared__ T values[kCkptThreads / 32][32][16 + 2];            // rows of an odd number of words for 16 bits
        const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
        if (count > 0) {
#pragma unroll
            for (int j = 0; j < 16; ++j) values[warp][lane][j] = from_float<T>(v[j]);
        }
        __syncwarp();
#pragma unroll 4
        for (int k = 0; k < 16; ++k) {
            const int owner = 2 * k + lane / 16;
            T* at = (T*)__shfl_sync(0xFFFFFFFFu, (unsigned long long)to, owner) + lane % 16;
            if (lane % 16 < __shfl_sync(0xFFFFFFFFu, count, owner)) *at = values[warp][owner][lane % 16];
        }
    }
}

// dz = dy * act'(z).  A warp spans 32 half groups (512 columns) and walks down a run of rows,
// eight warps to a block, each keeping the sums of its own rows; the block adds the eight up
// and leaves the run's column sums in partial[run][n].  The next row waits in registers as it
// lies in memory, so that four blocks fit on an SM: 8192 x 16384 bf16 with gelu takes 131 us on the
// device (138 to 144 a call with three states in turn), HBM's floor being 103; with two blocks and a shorter polynomial in
// gelu's tail it took 180, with four 123.  Without WIDE the row goes round the warp to be
// stored, as in the restore.
template <typename T, int ACT, bool WIDE>
__global__ void __launch_bounds__(kCkptThreads, WIDE ? 4 : 3) k_act_backward(const T* dy, uint64_t dy_stride, CheckpointView pre, T* dz,
                                                                            uint64_t dz_stride, float* partial, uint32_t m, uint32_t n,
                                                                            uint32_t rows_per_run)
{
    dependency_wait();
    dependency_release();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t half = blockIdx.x * 32 + lane, col = half * 16;
    const uint32_t begin = blockIdx.y * rows_per_run, end = min(m, begin + rows_per_run);
    const int count = col < n ? (int)min(n - col, 16u) : 0;
    Pair sum[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] = Pair(0.f);
    uint32_t next[8], next_codes[4] = {0, 0, 0, 0}, next_exp = 0;
    auto fetch = [&](uint32_t row) {
        if (row >= end || count == 0) return;
        load_values<WIDE>(dy + (uint64_t)row * dy_stride + col, count, next);
        if constexpr (ACT != EDEN_ACT_NONE) {
            next_exp = pre.exps[(uint64_t)row * pre.exps_stride + half / 2];
            load_codes<WIDE>(pre.codes + (uint64_t)row * pre.codes_stride + col, count, next_codes);
        }
    };
    fetch(begin + warp);
    for (uint32_t row = begin + warp; row < end; row += kCkptThreads / 32) {
        if (WIDE && count == 0) break;
        float v[16];
        widen<T>(next, v);
        const uint32_t w[4] = {next_codes[0], next_codes[1], next_codes[2], next_codes[3]};
        const float scale = slope_scale(next_exp);
        fetch(row + kCkptThreads / 32);
        if constexpr (ACT != EDEN_ACT_NONE) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                Pair z01, z23;
                code_values(w[j], Pair(scale), z01, z23);
                (Pair(v[4 * j], v[4 * j + 1]) * act_slope<ACT>(z01)).get(v[4 * j], v[4 * j + 1]);
                (Pair(v[4 * j + 2], v[4 * j + 3]) * act_slope<ACT>(z23)).get(v[4 * j + 2], v[4 * j + 3]);
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] = sum[j] + Pair(v[2 * j], v[2 * j + 1]);
        if (!dz) continue;
        if constexpr (WIDE) {
            store_values(dz + (uint64_t)row * dz_stride + col, count, v);
        } else {
            __shared__ uint32_t values[kCkptThreads / 32][32][9];
#pragma unroll
            for (int j = 0; j < 8; ++j) values[warp][lane][j] = pack<T>(v[2 * j], v[2 * j + 1]);
            __syncwarp();
            const uint32_t first = blockIdx.x * 512 + lane;
            T* to = dz + (uint64_t)row * dz_stride + first;
#pragma unroll
            for (int k = 0; k < 16; ++k)
                if (first + 32 * k < n) to[32 * k] = ((const T*)values[warp][2 * k + lane / 16])[lane % 16];
            __syncwarp();
        }
    }
    if (!partial) return;
    __shared__ float sums[kCkptThreads / 32][16][33];
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j].get(sums[warp][2 * j][lane], sums[warp][2 * j + 1][lane]);
    __syncthreads();
    for (int i = threadIdx.x; i < 512; i += kCkptThreads) {
        const uint32_t at = blockIdx.x * 512 + i;
        float total = 0.f;
#pragma unroll
        for (int w = 0; w < kCkptThreads / 32; ++w) total += sums[w][i % 16][i / 16];
        if (at < n) partial[(uint64_t)blockIdx.y * n + at] = total;
    }
}

// out[n] (+)= the sum of partial's rows: 32 columns per block, each warp every eighth row,
// the eight added in order
static __global__ void __launch_bounds__(kCkptThreads) k_column_sum(const float* partial, uint64_t rows, uint64_t n,
                                                            float* out, int accumulate)
{
    dependency_wait();
    dependency_release();
    const uint64_t col = (uint64_t)blockIdx.x * 32 + threadIdx.x % 32;
    const int warp = threadIdx.x / 32;
    float sum = 0.f;
    if (col < n) {
#pragma unroll 8
        for (uint64_t r = warp; r < rows; r += kCkptThreads / 32) sum += partial[r * n + col];
    }
    __shared__ float sums[kCkptThreads / 32][32];
    sums[warp][threadIdx.x % 32] = sum;
    __syncthreads();
    if (warp == 0 && col < n) {
        float total = 0.f;
        for (int w = 0; w < kCkptThreads / 32; ++w) total += sums[w][threadIdx.x];
        out[col] = accumulate ? out[col] + total : total;
    }
}

}  // namespace eden
