// What joins a block to the residual stream, forward and backward in one pass each:
//     u = after(h)    x = scale * residual + gate * dropout(u)    y = before(x)
// Norms are v' = (v - mean) * rate, u = v' * weight + bias, with mean = 0 for "rms".
//   backward of a norm   dv = rate * (g - mean(g) - v' mean(g v'))   g = du * weight; "rms" without mean(g)
//   dropout              Philox4x32-10, stream 3, counter (column / 8, row), key the seed: eight
//                        16-bit numbers a call, a value is kept where its number is below `keep`;
//                        the mask is made again wherever it is needed
// All of it reads and writes a few bytes a value and computes little: HBM bounds it.
#pragma once

#include "eden_device.cuh"
#include "tensor_core.cuh"
#include "train_device.cuh"

namespace eden {

// A thread takes 8 columns (one Philox call) of its team's rows; a team is the warps that hold a row,
// 256 columns each.  A block has as many teams as fit into 16 warps.  Rows of more than 4096 columns
// are shared by the blocks of a cluster (their sums go through distributed shared memory), or, where
// no norm needs a row's sums, by independent blocks.
constexpr int kBlockThreads = 512, kBlockWarps = kBlockThreads / 32, kBlockColumns = 8 * kBlockThreads, kBlockCluster = 8;

struct NormView {
    const void* weight;                // or null: 1
    const void* bias;                  // or null: 0
    float* stats;                      // [m][2] mean, rate; forward: written, or null
    float eps;
    int kind;                          // EDEN_NORM_*
};

struct BlockShape {
    uint32_t m, n;
    uint32_t warps, teams;             // of a team, of a block
    uint32_t span;                     // columns of a block
    uint32_t blocks;                   // of a cluster
};

struct DropView {
    uint64_t seed;
    const uint64_t* seed_at;           // or null: seed
    uint32_t keep, first_row;          // of 65536; row of the first row of the matrices
    float factor;                      // 65536 / keep, 0 for 0
};

__device__ __forceinline__ float warp_sum_f(float v)
{
#pragma unroll
    for (int i = 16; i > 0; i /= 2) v += __shfl_xor_sync(0xFFFFFFFFu, v, i);
    return v;
}

// Where a thread stands: its team, its columns.
struct Place {
    uint32_t team, warp, lane, rank, first, col;
    int count;                         // of its 8 columns exist
    __device__ __forceinline__ explicit Place(const BlockShape& s)
    {
        const uint32_t w = threadIdx.x / 32;
        lane = threadIdx.x % 32;
        team = w / s.warps;
        warp = w - team * s.warps;
        rank = s.blocks > 1 ? cluster_rank() : 0;
        first = (s.blocks > 1 ? rank : blockIdx.y) * s.span;
        col = first + warp * 256 + lane * 8;
        count = col < s.n ? (int)min(s.n - col, 8u) : 0;
    }
};

// Sums over a row.  Each warp leaves a pair of its own; `take(i, pair)` then gets warp i's, every
// lane some of them, alike in all warps.  Two places in turn: a place is written again after the
// next exchange, which nobody passes before all have read this one.
struct Exchange {
    float2 places[2][kBlockWarps * kBlockCluster];
};

template <typename F>
__device__ __forceinline__ void exchange(Exchange& e, uint32_t& turn, const BlockShape& s, const Place& at, float2 mine, F&& take)
{
    if (s.blocks == 1 && s.warps == 1) {
        if (at.lane == 0) take(0u, mine);
        return;
    }
    float2* const place = e.places[turn];
    turn ^= 1;
    if (s.blocks == 1) {
        float2* const team = place + at.team * s.warps;
        if (at.lane == 0) team[at.warp] = mine;
        __syncwarp();
        asm volatile("barrier.sync %0, %1;" ::"r"(at.team + 1), "r"(s.warps * 32) : "memory");
        if (at.lane < s.warps) take(at.lane, team[at.lane]);
        return;
    }
    if (at.lane < s.blocks) {
        const uint32_t to = address_in(shared_address(place + at.rank * kBlockWarps + at.warp), at.lane);
        asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(mine.x), "f"(mine.y) : "memory");
    }
    cluster_arrive_wait();
    for (uint32_t i = at.lane; i < s.blocks * kBlockWarps; i += 32) {
        const uint32_t w = i % kBlockWarps;
        if (w < s.warps) take(i / kBlockWarps * s.warps + w, place[i]);
    }
}

// columns of warp i (in the order of `exchange`)
__device__ __forceinline__ float columns_of(const BlockShape& s, uint32_t i)
{
    const uint32_t begin = i / s.warps * s.span + i % s.warps * 256;
    return begin < s.n ? (float)min(s.n - begin, 256u) : 0.f;
}

// Mean and rate of a row.  "layer": each warp's mean and the sum of squares around it, put together
// around the row's mean, so that no difference of large squares makes a small one.
__device__ __forceinline__ float2 row_statistics(Exchange& e, uint32_t& turn, const BlockShape& s, const Place& at, const NormView& norm, const float (&v)[8])
{
    const float n = (float)s.n;
    if (norm.kind == EDEN_NORM_RMS) {
        float q = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) q = fmaf(v[j], v[j], q);               // columns that do not exist hold 0
        float total = 0.f;
        exchange(e, turn, s, at, make_float2(warp_sum_f(q), 0.f), [&](uint32_t, float2 w) { total += w.x; });
        return make_float2(0.f, rsqrtf(warp_sum_f(total) / n + norm.eps));
    }
    float sum = 0.f, q = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += v[j];
    sum = warp_sum_f(sum);
    const float own = columns_of(s, (s.blocks > 1 ? at.rank : 0) * s.warps + at.warp), middle = own > 0.f ? sum / own : 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j)
        if (j < at.count) q = fmaf(v[j] - middle, v[j] - middle, q);
    float2 held[kBlockCluster * kBlockWarps / 32];
    float columns[kBlockCluster * kBlockWarps / 32];
#pragma unroll
    for (int i = 0; i < kBlockCluster * kBlockWarps / 32; ++i) held[i] = make_float2(0.f, 0.f), columns[i] = 0.f;
    int got = 0;
    float total = 0.f;
    exchange(e, turn, s, at, make_float2(sum, warp_sum_f(q)), [&](uint32_t i, float2 w) {
#pragma unroll
        for (int k = 0; k < kBlockCluster * kBlockWarps / 32; ++k)
            if (k == got) held[k] = w, columns[k] = columns_of(s, i);
        ++got;
        total += w.x;
    });
    const float mean = warp_sum_f(total) / n;
    q = 0.f;
#pragma unroll
    for (int k = 0; k < kBlockCluster * kBlockWarps / 32; ++k)
        if (columns[k] > 0.f) {
            const float off = held[k].x / columns[k] - mean;
            q += fmaf(columns[k] * off, off, held[k].y);
        }
    return make_float2(mean, rsqrtf(warp_sum_f(q) / n + norm.eps));
}

// both sums over the row
__device__ __forceinline__ float2 row_sums(Exchange& e, uint32_t& turn, const BlockShape& s, const Place& at, float a, float b)
{
    float2 total = make_float2(0.f, 0.f);
    exchange(e, turn, s, at, make_float2(warp_sum_f(a), warp_sum_f(b)), [&](uint32_t, float2 w) { total.x += w.x; total.y += w.y; });
    return make_float2(warp_sum_f(total.x), warp_sum_f(total.y));
}

template <typename T>
__device__ __forceinline__ void widen_8(const uint4& w, float (&v)[8])
{
    unpack<T>(w.x, v[0], v[1]);
    unpack<T>(w.y, v[2], v[3]);
    unpack<T>(w.z, v[4], v[5]);
    unpack<T>(w.w, v[6], v[7]);
}

// 8 values at p, of which `count` exist (zeros after them); WIDE: on 16 bytes
template <bool WIDE, typename T>
__device__ __forceinline__ uint4 load_row_8(const T* p, int count)
{
    if (WIDE && count == 8) return *(const uint4*)p;
    return load_shifted_8(p, count);
}

// The lane's 8 values to p, of which `count` exist.  Without WIDE the warp hands them round in shared
// memory (`buffer`, its own 128 words) and stores them side by side.
template <bool WIDE, typename T>
__device__ __forceinline__ void store_row_8(T* p, int count, const float (&v)[8], uint4* buffer, uint32_t lane)
{
    const uint4 w = make_uint4(pack<T>(v[0], v[1]), pack<T>(v[2], v[3]), pack<T>(v[4], v[5]), pack<T>(v[6], v[7]));
    if constexpr (WIDE) {
        if (count == 8) {
            *(uint4*)p = w;
            return;
        }
        const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < count) ((uint16_t*)p)[j] = (uint16_t)(words[j / 2] >> 16 * (j % 2));
        return;
    }
    __syncwarp();
    buffer[lane] = w;
    __syncwarp();
    const int in_warp = __reduce_add_sync(0xFFFFFFFFu, count);             // lanes' columns follow one another
    uint16_t* const row = (uint16_t*)p - lane * 8;
    if (((uintptr_t)row & 3) == 0) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = j * 32 + (int)lane;
            if (2 * i + 1 < in_warp) ((uint32_t*)row)[i] = ((const uint32_t*)buffer)[i];
            else if (2 * i < in_warp) row[2 * i] = ((const uint16_t*)buffer)[2 * i];
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = j * 32 + (int)lane;
            if (i < in_warp) row[i] = ((const uint16_t*)buffer)[i];
        }
    }
}

// factors of the 8 values: 0 or 65536 / keep
__device__ __forceinline__ uint32_t kept_bits(const DropView& d, uint64_t seed, uint32_t row, uint32_t col)
{
    const uint4 r = philox_stream(seed, 3u, (uint64_t)(d.first_row + row) << 32 | col / 8);
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
    uint32_t bits = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        bits |= (w[j] & 0xFFFFu) < d.keep ? 1u << 2 * j : 0u;
        bits |= w[j] >> 16 < d.keep ? 2u << 2 * j : 0u;
    }
    return bits;
}

struct JoinView {
    const void* h;         uint64_t h_stride;
    const void* residual;  uint64_t residual_stride;       // or null
    const void* gate;      uint64_t gate_stride;           // or null; stride 0: a vector
    void* x;               uint64_t x_stride;              // or null
    void* y;               uint64_t y_stride;              // before.kind != none
    NormView after, before;
    DropView drop;
    float scale;
    int has_drop;
};

template <typename T, bool WIDE, bool AFTER, bool BEFORE>
__global__ void __launch_bounds__(kBlockThreads, 2) k_join(JoinView p, BlockShape s)
{
    __shared__ Exchange sums;
    __shared__ uint4 buffers[WIDE ? 1 : kBlockWarps][32];
    dependency_wait();
    dependency_release();
    const Place at(s);
    uint4* const buffer = buffers[WIDE ? 0 : threadIdx.x / 32];
    const uint64_t seed = p.drop.seed_at ? *p.drop.seed_at : p.drop.seed;
    const uint32_t step = gridDim.x / s.blocks * s.teams;
    uint32_t turn = 0, row = blockIdx.x / s.blocks * s.teams + at.team;
    auto vector = [&](const void* v) { return load_shifted_8((const T*)v + at.col, v ? at.count : 0); };
    uint4 after_weight, after_bias, before_weight, before_bias, gate = vector(p.gate_stride ? nullptr : p.gate);
    if (AFTER) after_weight = vector(p.after.weight), after_bias = vector(p.after.bias);
    if (BEFORE) before_weight = vector(p.before.weight), before_bias = vector(p.before.bias);
    auto affine = [&](float (&v)[8], const NormView& norm, const uint4& weight, const uint4& bias) {
        float w[8];
        if (norm.weight) {
            widen_8<T>(weight, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= w[j];
        }
        if (norm.bias) {
            widen_8<T>(bias, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += w[j];
        }
    };
    // the next row waits as it lies in memory
    uint4 next_h, next_residual, next_gate;
    auto fetch = [&](uint32_t r) {
        const int count = r < s.m ? at.count : 0;
        next_h = load_row_8<WIDE>((const T*)p.h + (uint64_t)r * p.h_stride + at.col, count);
        if (p.residual) next_residual = load_row_8<WIDE>((const T*)p.residual + (uint64_t)r * p.residual_stride + at.col, count);
        if (p.gate_stride) next_gate = load_row_8<WIDE>((const T*)p.gate + (uint64_t)r * p.gate_stride + at.col, count);
    };
    fetch(row);
    for (; row < s.m; row += step) {
        float v[8], residual[8], g[8];
        widen_8<T>(next_h, v);
        if (p.residual) widen_8<T>(next_residual, residual);
        if (p.gate) widen_8<T>(p.gate_stride ? next_gate : gate, g);
        fetch(row + step);
        if constexpr (AFTER) {
            const float2 st = row_statistics(sums, turn, s, at, p.after, v);
            if (p.after.stats && at.col == 0) *(float2*)(p.after.stats + 2 * (uint64_t)row) = st;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = (v[j] - st.x) * st.y;
            affine(v, p.after, after_weight, after_bias);
        }
        if (p.has_drop) {
            const uint32_t bits = kept_bits(p.drop, seed, row, at.col);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = bits >> j & 1 ? v[j] * p.drop.factor : 0.f;
        }
        if (p.gate) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= g[j];
        }
        if (p.residual) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = fmaf(p.scale, residual[j], v[j]);
        }
        if (p.x) store_row_8<WIDE>((T*)p.x + (uint64_t)row * p.x_stride + at.col, at.count, v, buffer, at.lane);
        if constexpr (BEFORE) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = j < at.count ? v[j] : 0.f;
            const float2 st = row_statistics(sums, turn, s, at, p.before, v);
            if (p.before.stats && at.col == 0) *(float2*)(p.before.stats + 2 * (uint64_t)row) = st;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = (v[j] - st.x) * st.y;
            affine(v, p.before, before_weight, before_bias);
            store_row_8<WIDE>((T*)p.y + (uint64_t)row * p.y_stride + at.col, at.count, v, buffer, at.lane);
        }
    }
    // a block's places are written by the others of its cluster as long as they run
    if (s.blocks > 1) cluster_arrive_wait();
}

// ---- backward -----------------------------------------------------------------------
// An activation that was kept: a matrix of 16-bit values, or a checkpoint.
struct KeptView {
    const void* data;      uint64_t stride;                // null: the checkpoint
    CheckpointView held;
};

struct KeptRaw {
    uint4 w;                           // 16-bit values; or two words of codes
    uint32_t exp;
};

// 8 bytes at any address, of which `count` exist
__device__ __forceinline__ uint2 load_bytes_8(const int8_t* p, int count)
{
    const uint32_t off = (uint32_t)((uintptr_t)p & 3u);
    const uint32_t* const word = (const uint32_t*)(p - off);
    const int end = count > 0 ? (int)off + count : 0;
    const uint32_t a = end > 0 ? word[0] : 0u, b = end > 4 ? word[1] : 0u, c = end > 8 ? word[2] : 0u;
    uint2 v = make_uint2(__funnelshift_r(a, b, 8 * off), __funnelshift_r(b, c, 8 * off));
    if (count < 8) {
        v.x &= count >= 4 ? 0xFFFFFFFFu : count > 0 ? 0xFFFFFFFFu >> (32 - 8 * count) : 0u;
        v.y &= count > 4 ? 0xFFFFFFFFu >> (64 - 8 * count) : 0u;
    }
    return v;
}

template <bool WIDE, typename T>
__device__ __forceinline__ KeptRaw load_kept(const KeptView& k, uint32_t row, uint32_t col, int count)
{
    KeptRaw raw;
    if (k.data) {
        raw.w = load_row_8<WIDE>((const T*)k.data + (uint64_t)row * k.stride + col, count);
        raw.exp = 0;
    } else {
        const int8_t* const codes = k.held.codes + (uint64_t)row * k.held.codes_stride + col;
        const uint2 w = WIDE && count == 8 ? *(const uint2*)codes : load_bytes_8(codes, count);
        raw.w = make_uint4(w.x, w.y, 0, 0);
        raw.exp = count > 0 ? k.held.exps[(uint64_t)row * k.held.exps_stride + col / kGroup] : 1u;
    }
    return raw;
}

template <typename T>
__device__ __forceinline__ void kept_values(const KeptView& k, const KeptRaw& raw, float (&v)[8])
{
    if (k.data) {
        widen_8<T>(raw.w, v);
        return;
    }
    const Pair scale(group_scale(raw.exp));
    Pair a, b;
    code_values(raw.w.x, scale, a, b);
    a.get(v[0], v[1]);
    b.get(v[2], v[3]);
    code_values(raw.w.y, scale, a, b);
    a.get(v[4], v[5]);
    b.get(v[6], v[7]);
}

enum { kBeforeWeight = 0, kBeforeBias = 1, kAfterWeight = 2, kAfterBias = 3, kGateSum = 4, kJoinSums = 5 };

struct JoinBackwardView {
    const void* dx;        uint64_t dx_stride;             // or null: 0
    const void* dy;        uint64_t dy_stride;             // before.kind != none
    KeptView h, x;                                         // h: after.kind != none or a gate
    const void* gate;      uint64_t gate_stride;
    void* d_residual;      uint64_t d_residual_stride;     // or null
    void* dh;              uint64_t dh_stride;             // or null
    void* d_gate;          uint64_t d_gate_stride;         // a matrix gate's gradient, or null
    float* partial;        uint32_t wanted;                // sums over rows that are wanted: [part][number of them][n]
    NormView after, before;
    DropView drop;
    float scale;
    int has_drop;
};

// Each team keeps the sums of its rows over the columns in registers and leaves them in its part of
// `partial`, which k_join_sums adds up.
template <typename T, bool WIDE, bool AFTER, bool BEFORE>
__global__ void __launch_bounds__(kBlockThreads, 1) k_join_backward(JoinBackwardView p, BlockShape s)
{
    __shared__ Exchange sums;
    __shared__ uint4 buffers[WIDE ? 1 : kBlockWarps][32];
    dependency_wait();
    dependency_release();
    const Place at(s);
    uint4* const buffer = buffers[WIDE ? 0 : threadIdx.x / 32];
    const uint64_t seed = p.drop.seed_at ? *p.drop.seed_at : p.drop.seed;
    const uint32_t group = blockIdx.x / s.blocks, step = gridDim.x / s.blocks * s.teams;
    uint32_t turn = 0, row = group * s.teams + at.team;
    const float n = (float)s.n;
    auto vector = [&](const void* v) { return load_shifted_8((const T*)v + at.col, v ? at.count : 0); };
    uint4 after_weight, after_bias, before_weight, gate = vector(p.gate_stride ? nullptr : p.gate);
    if (AFTER) after_weight = vector(p.after.weight), after_bias = vector(p.after.bias);
    if (BEFORE) before_weight = vector(p.before.weight);
    const bool needs_h = AFTER || p.gate;
    float total[kJoinSums][8];
#pragma unroll
    for (int i = 0; i < kJoinSums; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) total[i][j] = 0.f;

    uint4 next_dx = make_uint4(0, 0, 0, 0), next_dy, next_gate;
    KeptRaw next_x, next_h;
    float2 next_before, next_after;
    auto fetch = [&](uint32_t r) {
        const int count = r < s.m ? at.count : 0;
        if (p.dx) next_dx = load_row_8<WIDE>((const T*)p.dx + (uint64_t)r * p.dx_stride + at.col, count);
        if (BEFORE) {
            next_dy = load_row_8<WIDE>((const T*)p.dy + (uint64_t)r * p.dy_stride + at.col, count);
            next_x = load_kept<WIDE, T>(p.x, r, at.col, count);
            next_before = r < s.m ? *(const float2*)(p.before.stats + 2 * (uint64_t)r) : make_float2(0.f, 0.f);
        }
        if (needs_h) next_h = load_kept<WIDE, T>(p.h, r, at.col, count);
        if (AFTER) next_after = r < s.m ? *(const float2*)(p.after.stats + 2 * (uint64_t)r) : make_float2(0.f, 0.f);
        if (p.gate_stride) next_gate = load_row_8<WIDE>((const T*)p.gate + (uint64_t)r * p.gate_stride + at.col, count);
    };
    fetch(row);
    for (; row < s.m; row += step) {
        float d[8], h[8], g[8], dy[8], x[8];
        widen_8<T>(next_dx, d);
        if (needs_h) kept_values<T>(p.h, next_h, h);
        if (p.gate) widen_8<T>(p.gate_stride ? next_gate : gate, g);
        if (BEFORE) widen_8<T>(next_dy, dy), kept_values<T>(p.x, next_x, x);
        const float2 before = next_before, after = next_after;
        fetch(row + step);
        if constexpr (BEFORE) {
            float w[8], sum = 0.f, dot = 0.f;
            widen_8<T>(before_weight, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x[j] = (x[j] - before.x) * before.y;
                total[kBeforeWeight][j] = fmaf(dy[j], x[j], total[kBeforeWeight][j]);
                total[kBeforeBias][j] += dy[j];
                if (p.before.weight) dy[j] *= w[j];
                if (j < at.count) {
                    sum += dy[j];
                    dot = fmaf(dy[j], x[j], dot);
                }
            }
            float2 mean = row_sums(sums, turn, s, at, sum, dot);
            mean.x = p.before.kind == EDEN_NORM_LAYER ? mean.x / n : 0.f;
            mean.y /= n;
#pragma unroll
            for (int j = 0; j < 8; ++j) d[j] = fmaf(before.y, dy[j] - mean.x - x[j] * mean.y, d[j]);
        }
        if (p.d_residual) {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = p.scale * d[j];
            store_row_8<WIDE>((T*)p.d_residual + (uint64_t)row * p.d_residual_stride + at.col, at.count, x, buffer, at.lane);
        }
        if constexpr (AFTER) {
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] = (h[j] - after.x) * after.y;
        }
        const uint32_t bits = p.has_drop ? kept_bits(p.drop, seed, row, at.col) : 0xFFu;
        if (p.gate) {
            float u[8], w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) u[j] = h[j];
            if (AFTER && p.after.weight) {
                widen_8<T>(after_weight, w);
#pragma unroll
                for (int j = 0; j < 8; ++j) u[j] *= w[j];
            }
            if (AFTER && p.after.bias) {
                widen_8<T>(after_bias, w);
#pragma unroll
                for (int j = 0; j < 8; ++j) u[j] += w[j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) u[j] = bits >> j & 1 ? u[j] * p.drop.factor * d[j] : 0.f;
            if (p.gate_stride) {
                if (p.d_gate) store_row_8<WIDE>((T*)p.d_gate + (uint64_t)row * p.d_gate_stride + at.col, at.count, u, buffer, at.lane);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) total[kGateSum][j] += u[j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) d[j] *= g[j];
        }
        if (p.has_drop) {
#pragma unroll
            for (int j = 0; j < 8; ++j) d[j] = bits >> j & 1 ? d[j] * p.drop.factor : 0.f;
        }
        if constexpr (AFTER) {
            float w[8], sum = 0.f, dot = 0.f;
            widen_8<T>(after_weight, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                total[kAfterWeight][j] = fmaf(d[j], h[j], total[kAfterWeight][j]);
                total[kAfterBias][j] += d[j];
                if (p.after.weight) d[j] *= w[j];
                if (j < at.count) {
                    sum += d[j];
                    dot = fmaf(d[j], h[j], dot);
                }
            }
            float2 mean = row_sums(sums, turn, s, at, sum, dot);
            mean.x = p.after.kind == EDEN_NORM_LAYER ? mean.x / n : 0.f;
            mean.y /= n;
#pragma unroll
            for (int j = 0; j < 8; ++j) d[j] = after.y * (d[j] - mean.x - h[j] * mean.y);
        }
        if (p.dh) store_row_8<WIDE>((T*)p.dh + (uint64_t)row * p.dh_stride + at.col, at.count, d, buffer, at.lane);
    }
    if (p.wanted) {
        float* to = p.partial + (uint64_t)(group * s.teams + at.team) * __popc(p.wanted) * s.n + at.col;
#pragma unroll
        for (int i = 0; i < kJoinSums; ++i) {
            if (!(p.wanted >> i & 1)) continue;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < at.count) to[j] = total[i][j];
            to += s.n;
        }
    }
    if (s.blocks > 1) cluster_arrive_wait();
}

struct JoinSumsView {
    const float* partial;
    float* out[kJoinSums];             // in the order of the sums that are wanted
    uint32_t parts, n, sums;
    int accumulate;
};

// out[i][col] (+)= the sum of the parts' sums i: 32 columns per block, each warp every eighth
// part, the eight added in order
__global__ void __launch_bounds__(256) k_join_sums(JoinSumsView p)
{
    dependency_wait();
    dependency_release();
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32, i = blockIdx.y;
    const uint64_t col = (uint64_t)blockIdx.x * 32 + lane;
    float sum = 0.f;
    if (col < p.n) {
#pragma unroll 8
        for (uint32_t r = warp; r < p.parts; r += 8) sum += p.partial[((uint64_t)r * p.sums + i) * p.n + col];
    }
    __shared__ float sums[8][32];
    sums[warp][lane] = sum;
    __syncthreads();
    if (warp == 0 && col < p.n) {
        float total = 0.f;
        for (int w = 0; w < 8; ++w) total += sums[w][lane];
        float* const out = p.out[i];
        out[col] = p.accumulate ? out[col] + total : total;
    }
}

}  // namespace eden
