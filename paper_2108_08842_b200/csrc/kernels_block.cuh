// What joins a block to the residual stream, forward and backward in one pass each:
//     u = after(h)    x = scale * residual + gate * dropout(u)    y = before(x)
// Norms are v' = (v - mean) * rate, u = v' * weight + bias, with mean = 0 for "rms".
//   backward of a norm   dv = rate * (g - mean(g) - v' mean(g v'))   g = du * weight; "rms" without mean(g)
//   dropout              Philox4x32-10, stream 3, counter (column / 8, row), key the seed: eight
//                        16-bit numbers a call, a value is kept where its number is below `keep`;
//                        the mask is made again wherever it is needed
// All of it reads and writes a few bytes a value, but the mask's numbers, the sums over rows and the columns'
// sums take instructions too: 16384 x 4096 with norms, gate and dropout is bound by issue slots (57 % busy forward,
// 52 % backward) next to HBM, 112 and 188 us; without norms by HBM.
#pragma once

#include "eden_device.cuh"
#include "tensor_core.cuh"
#include "train_device.cuh"

namespace eden {

// A thread takes K pieces of 8 columns (a Philox call each) of its team's rows, 256 columns apart; a
// team is the warps, up to 16, that hold a row.  Rows that 16 warps do not hold are shared by the blocks
// of a cluster (their sums go through distributed shared memory).  K = 2 halves the shuffles and waits per
// value and leaves another team to run while one waits; K = 1 spreads a few rows over more warps.
//
// What a row needs is brought to shared memory by bulk copies, the next rows of the team while this
// one is worked on.  Copies start on 16 bytes: a row's first and last chunks may hold bytes of its
// neighbours, which are not used.
//
// FULL: a mean is taken off, biases are added, or a gate is a matrix.  WIDE: every row starts on 16
// bytes and has a multiple of 8 columns; a thread then has all 8 columns of a piece or none, and reads
// zeros where there are none.  A kernel that asked for both at run time took 1230 instructions for 256
// values of a row's gradients, and its loop for four rows did not fit the instruction cache: 780 us for the
// gradients of 16384 x 4096; 364 a row at a time with FULL as a template; 188 now, 884 instructions for 512 values.
//
// The vectors over the columns (weights, biases, a gate) lie in shared memory as well: in registers,
// they made the gradients' kernel spill, and left the forward one 16 warps on an SM.  Forward 24 warps of
// 80 registers, backward 16 of 128, which hold the column sums.
constexpr int kTeamWarps = 16, kJoinThreads = 768, kJoinBackwardThreads = 512, kBlockCluster = 8;
constexpr int kMaxSources = 9, kMaxStages = 4, kMaxTeams = 24;

struct NormView {
    const void* weight;                // or null: 1
    const void* bias;                  // or null: 0
    float* stats;                      // [m][2] mean, rate; forward: written, or null
    float eps;
    int kind;                          // EDEN_NORM_*
};

// What a row needs of a matrix: `number` bytes for 2^shift columns; or, `fixed`, those bytes.
struct Source {
    const char* base;                  // or null: not wanted
    uint64_t stride;                   // bytes from row to row
    uint32_t number, shift, fixed;
    uint32_t at;                       // in a row's place in shared memory
    uint32_t aligned;                  // all rows start on 16 bytes
    __host__ __device__ __forceinline__ uint32_t begin(uint32_t first) const { return fixed ? 0 : (first >> shift) * number; }
    __host__ __device__ __forceinline__ uint32_t bytes_of(uint32_t cols) const { return fixed ? number : ((cols + (1u << shift) - 1) >> shift) * number; }
    // what a row's place begins with that is not the row's
    __device__ __forceinline__ uint32_t skew(uint32_t r, uint32_t first) const
    {
        return aligned ? 0 : ((uint32_t)(uintptr_t)base + r * (uint32_t)stride + begin(first)) & 15u;
    }
};

struct BlockShape {
    uint32_t m, n;
    uint32_t warps, teams;             // of a team, of a block
    uint32_t span;                     // columns of a block
    uint32_t blocks;                   // of a cluster
    uint32_t stages, row_bytes;
    uint32_t vectors;                  // where those begin in shared memory, behind the rows
    Source source[kMaxSources];
};

struct DropView {
    uint64_t seed;
    const uint64_t* seed_at;           // or null: seed
    uint32_t keep, first_row;          // of 65536; row of the first row of the matrices
    float factor;                      // 65536 / keep, 0 for 0
};

// Where a thread stands: its team, its columns.
template <int K>
struct Place {
    uint32_t team, warp, lane, rank, first, col, width;
    int count[K];                      // of its 8 columns at col + 256 * i exist
    __device__ __forceinline__ explicit Place(const BlockShape& s)
    {
        const uint32_t w = threadIdx.x / 32;
        lane = threadIdx.x % 32;
        team = w / s.warps;
        warp = w - team * s.warps;
        rank = s.blocks > 1 ? cluster_rank() : 0;
        first = rank * s.span;
        width = first < s.n ? min(s.n - first, s.span) : 0;
        col = first + warp * (256 * K) + lane * 8;
#pragma unroll
        for (int i = 0; i < K; ++i) count[i] = col + 256 * i < s.n ? (int)min(s.n - col - 256 * i, 8u) : 0;
        columns = s.n;
        const uint32_t begin = first + warp * (256 * K);
        over_own = begin < s.n ? 1.f / (float)min(s.n - begin, 256u * K) : 0.f;
    }
    uint32_t columns;
    float over_own;                    // one over the number of the warp's columns that exist
    // columns of the warp's piece that exist
    __device__ __forceinline__ int in_warp(int i) const { return min(max((int)columns - (int)(col - lane * 8 + 256 * i), 0), 256); }
};

template <int K>
using Values = Pair[K][4];

// ---- sums over rows -----------------------------------------------------------------
__device__ __forceinline__ float warp_total(float a)
{
#pragma unroll
    for (int i = 16; i > 0; i /= 2) a += __shfl_xor_sync(0xFFFFFFFFu, a, i);
    return a;
}

// Each warp leaves a pair; `take(i, pair)` then gets warp i's, each lane some of them (without a
// cluster one, alike in both halves of the warp), alike in all warps.  Two places in turn: a place is
// written again after the next exchange, which nobody passes before all have read this one.
struct Exchange {
    float2 places[2][kTeamWarps * kBlockCluster];
};

template <int K, typename F>
__device__ __forceinline__ void exchange(Exchange& e, uint32_t& turn, const BlockShape& s, const Place<K>& at, float2 mine, F&& take)
{
    float2* const place = e.places[turn];
    turn ^= 1;
    if (s.blocks == 1) {
        float2* const team = place + at.team * s.warps;
        if (at.lane == 0) team[at.warp] = mine;
        __syncwarp();
        if (s.warps > 1) asm volatile("barrier.sync %0, %1;" ::"r"(at.team + 1), "r"(s.warps * 32) : "memory");
        const uint32_t i = at.lane % kTeamWarps;
        if (i < s.warps) take(i, team[i]);
        __syncwarp();
        return;
    }
    if (at.lane < s.blocks) {
        const uint32_t to = address_in(shared_address(place + at.rank * kTeamWarps + at.warp), at.lane);
        asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(mine.x), "f"(mine.y) : "memory");
    }
    cluster_arrive_wait();
    for (uint32_t i = at.lane; i < s.blocks * kTeamWarps; i += 32) {
        const uint32_t w = i % kTeamWarps;
        if (w < s.warps) take(i / kTeamWarps * s.warps + w, place[i]);
    }
    __syncwarp();
}

// what the lanes hold after an exchange, added up
__device__ __forceinline__ float lanes_total(const BlockShape& s, float a)
{
#pragma unroll
    for (int i = kTeamWarps / 2; i > 0; i /= 2) a += __shfl_xor_sync(0xFFFFFFFFu, a, i);
    if (s.blocks > 1) a += __shfl_xor_sync(0xFFFFFFFFu, a, 16);
    return a;
}

// columns of warp i (in the order of `exchange`)
template <int K>
__device__ __forceinline__ float columns_of(const BlockShape& s, uint32_t i)
{
    const uint32_t begin = s.blocks == 1 ? i * (256 * K) : i / s.warps * s.span + i % s.warps * (256 * K);
    return begin < s.n ? (float)min(s.n - begin, 256u * K) : 0.f;
}

__device__ __forceinline__ float both(Pair a)
{
    float x, y;
    a.get(x, y);
    return x + y;
}

// Sums over a row's columns: of b, and (FULL) of a.
template <bool FULL, int K>
__device__ __forceinline__ float2 row_sums(Exchange& e, uint32_t& turn, const BlockShape& s, const Place<K>& at, Pair a, Pair b)
{
    float2 total = make_float2(0.f, 0.f);
    exchange<K>(e, turn, s, at, make_float2(FULL ? warp_total(both(a)) : 0.f, warp_total(both(b))), [&](uint32_t, float2 w) {
        if (FULL) total.x += w.x;
        total.y += w.y;
    });
    return make_float2(FULL ? lanes_total(s, total.x) : 0.f, lanes_total(s, total.y));
}

// Mean and rate of a row.  "layer": each warp's mean and the sum of squares around it, put together
// around the row's mean, so that no difference of large squares makes a small one.  Sums that pass
// fp32's largest number (bf16 values beyond 10^17) are made again of smaller values: all threads of a row
// hold the same sum, and take the second way together.
template <bool FULL, bool WIDE, int K>
__device__ __forceinline__ float2 row_statistics(Exchange& e, uint32_t& turn, const BlockShape& s, const Place<K>& at, const NormView& norm, const Values<K>& v)
{
    const float over_n = 1.f / (float)s.n;
    constexpr float kSmaller = 8.271806125530277e-25f;     // 2^-80
    float mean = 0.f, square = 0.f;
    auto sums = [&](auto scaled) {
        const Pair by(decltype(scaled)::value ? kSmaller : 1.f);
        auto times = [&](Pair a) { return decltype(scaled)::value ? a * by : a; };
        if (!FULL || norm.kind == EDEN_NORM_RMS) {
            Pair q(0.f);
#pragma unroll
            for (int i = 0; i < K; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) q = fma(times(v[i][j]), times(v[i][j]), q);      // columns that do not exist hold 0
            square = row_sums<false, K>(e, turn, s, at, q, q).y * over_n;
        } else {
            Pair t(0.f);
#pragma unroll
            for (int i = 0; i < K; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) t = t + times(v[i][j]);
            const float sum = warp_total(both(t)), middle = sum * at.over_own;
            float q = 0.f;
#pragma unroll
            for (int i = 0; i < K; ++i) {
                Pair part(0.f);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    Pair off = times(v[i][j]) + Pair(-middle);
                    if (!WIDE && at.count[i] < 8) {
                        float x, y;
                        off.get(x, y);
                        off = Pair(2 * j < at.count[i] ? x : 0.f, 2 * j + 1 < at.count[i] ? y : 0.f);
                    }
                    part = fma(off, off, part);
                }
                q += at.count[i] > 0 ? both(part) : 0.f;
            }
            // the lane's warps (one, without a cluster) as one: columns, their mean, the squares around it
            float columns = 0.f, mid = 0.f, squares = 0.f, total = 0.f;
            exchange<K>(e, turn, s, at, make_float2(sum, warp_total(q)), [&](uint32_t i, float2 w) {
                const float c = columns_of<K>(s, i);
                if (c == 0.f) return;
                const float m = w.x / c;
                total += w.x;
                if (columns == 0.f) {
                    columns = c, mid = m, squares = w.y;
                    return;
                }
                const float off = m - mid, part = c / (columns + c);
                squares += fmaf(off * off * columns, part, w.y);
                mid = fmaf(off, part, mid);
                columns += c;
            });
            mean = lanes_total(s, total) * over_n;
            const float off = mid - mean;
            square = lanes_total(s, columns > 0.f ? fmaf(columns * off, off, squares) : 0.f) * over_n;
        }
    };
    sums(std::false_type());
    if (square < 3.0e38f) return make_float2(mean, rsqrtf(square + norm.eps));
    sums(std::true_type());
    // eps is nothing beside such squares, but all there is where only the sum of the values was too large
    return make_float2(mean / kSmaller, square == 0.f ? rsqrtf(norm.eps) : rsqrtf(fmaf(norm.eps * kSmaller, kSmaller, square)) * kSmaller);
}

// The 16 bytes that begin `skew` bytes, an even number, into two chunks.  One branch where the skew is
// the same for all lanes, as it is for a row.
__device__ __forceinline__ void shift_words(uint32_t (&w)[4], const uint4& lo, const uint4& hi, uint32_t skew)
{
    const uint32_t c[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w}, bits = (skew & 2u) * 8;
    auto from = [&](auto first) {
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = __funnelshift_r(c[decltype(first)::value + j], c[decltype(first)::value + j + 1], bits);
    };
    switch (skew >> 2) {
        case 0: from(std::integral_constant<int, 0>()); break;
        case 1: from(std::integral_constant<int, 1>()); break;
        case 2: from(std::integral_constant<int, 2>()); break;
        default: from(std::integral_constant<int, 3>()); break;
    }
}

// ---- rows in shared memory ----------------------------------------------------------
// A row of every source, `stages` times for each team: a row's copies are counted by its stage's barrier.
template <int K>
struct Stages {
    const BlockShape& s;
    const Place<K>& at;
    char* buffers;
    const char* row;                   // the place of the row that is worked on
    uint32_t bars;                     // this team's
    const char* from;                  // a lane's source: its first row's bytes for this block, how many, and their place
    uint64_t stride;
    uint32_t bytes, to;
    __device__ __forceinline__ Stages(const BlockShape& s, const Place<K>& at, char* block, uint32_t bars)
        : s(s), at(at), buffers(block + at.team * s.stages * s.row_bytes), row(buffers), bars(bars + at.team * kMaxStages * 8), from(nullptr), stride(0), bytes(0), to(0)
    {
        if (at.lane >= kMaxSources) return;
        const Source& source = s.source[at.lane];
        if (!source.base || (!at.width && !source.fixed)) return;          // a cluster's block without columns reads a row's statistics too
        from = source.base + source.begin(at.first);
        stride = source.stride;
        bytes = source.bytes_of(at.width);
        to = shared_address(buffers) + source.at;
    }

    // the team's first warp, a source per lane
    __device__ __forceinline__ void fetch(uint32_t stage, uint32_t r) const
    {
        const uint32_t bar = bars + 8 * stage;
        const char* const begin = from + r * stride;
        const uint32_t skew = (uint32_t)(uintptr_t)begin & 15u, size = bytes ? (skew + bytes + 15) & ~15u : 0;
        const uint32_t all = __reduce_add_sync(0xFFFFFFFFu, size);
        if (at.lane == 0) barrier_expect(bar, all);
        __syncwarp();
        if (size)
            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                         ::"r"(to + stage * s.row_bytes), "l"(begin - skew), "r"(size), "r"(bar) : "memory");
        __syncwarp();
    }

    __device__ __forceinline__ void go_to(uint32_t stage) { row = buffers + stage * s.row_bytes; }
    __device__ __forceinline__ const char* place(const Source& source) const { return row + source.at; }

    // The thread's values of 16 bits, zeros where there is no column.
    template <typename T, bool WIDE>
    __device__ __forceinline__ void values(Values<K>& v, uint32_t r, const Source& source) const
    {
        const char* const begin = place(source) + (at.col - at.first) * 2;
        const uint32_t skew = WIDE ? 0 : source.skew(r, at.first);
#pragma unroll
        for (int i = 0; i < K; ++i) {
            uint32_t w[4] = {0, 0, 0, 0};
            const char* const from = begin + 512 * i;
            if constexpr (WIDE) {
                const uint4 q = *(const uint4*)from;
                w[0] = q.x, w[1] = q.y, w[2] = q.z, w[3] = q.w;
            } else if (at.count[i] > 0) {
                // The chunks that hold them, shifted by the row's skew, the same for all lanes.  Five words a
                // lane, 16 bytes apart across the lanes, would meet four times in a bank.
                shift_words(w, *(const uint4*)from, *(const uint4*)(from + 16), skew);
                if (at.count[i] < 8) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] &= at.count[i] >= 2 * j + 2 ? 0xFFFFFFFFu : at.count[i] == 2 * j + 1 ? 0xFFFFu : 0u;
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float x, y;
                unpack<T>(w[j], x, y);
                v[i][j] = Pair(x, y);
            }
        }
    }

    // The same from a checkpoint, times `factor`.
    template <bool WIDE>
    __device__ __forceinline__ void coded(Values<K>& v, uint32_t r, const Source& codes, const Source& exps, float factor) const
    {
        const char* const begin = place(codes) + (at.col - at.first);
        const uint32_t skew = WIDE ? 0 : codes.skew(r, at.first);
        const uint8_t* const exp = (const uint8_t*)place(exps) + exps.skew(r, at.first) + (at.col - at.first) / kGroup;
#pragma unroll
        for (int i = 0; i < K; ++i) {
            uint32_t a = 0, b = 0, e = 1;
            const char* const from = begin + 256 * i;
            if constexpr (WIDE) {
                const uint2 q = *(const uint2*)from;
                const bool there = at.count[i] > 0;
                e = exp[256 / kGroup * i];
                a = there ? q.x : 0u, b = there ? q.y : 0u, e = there ? e : 1u;
            } else if (at.count[i] > 0) {
                const uint2 lo = *(const uint2*)(from + (skew & 8u)), hi = *(const uint2*)(from + (skew & 8u) + 8);
                const uint32_t c0 = skew & 4u ? lo.y : lo.x, c1 = skew & 4u ? hi.x : lo.y, c2 = skew & 4u ? hi.y : hi.x;
                a = __funnelshift_r(c0, c1, (skew & 3u) * 8);
                b = __funnelshift_r(c1, c2, (skew & 3u) * 8);
                e = exp[256 / kGroup * i];
                if (at.count[i] < 8) {
                    a &= at.count[i] >= 4 ? 0xFFFFFFFFu : 0xFFFFFFFFu >> (32 - 8 * at.count[i]);
                    b &= at.count[i] > 4 ? 0xFFFFFFFFu >> (64 - 8 * at.count[i]) : 0u;
                }
            }
            const Pair scale(group_scale(e) * factor);
            code_values(a, scale, v[i][0], v[i][1]);
            code_values(b, scale, v[i][2], v[i][3]);
        }
    }

    // Zeros behind the last value of every row's place of 16-bit values, up to the team's last column: no
    // copy reaches there, as their rows start on 16 bytes (a checkpoint's exponents may lie up to 15 bytes
    // further back, where a copy would meet these stores; what is not there is left out as it is read).
    // The whole block.
    __device__ __forceinline__ void clear(char* block) const
    {
        for (int i = 0; i < kMaxSources; ++i) {
            const Source& source = s.source[i];
            if (!source.base || source.fixed || source.number != 2) continue;
            const uint32_t begin = (source.bytes_of(at.width) + 15) & ~15u, end = source.bytes_of(s.span);
            if (begin >= end) continue;
            for (uint32_t row = 0; row < s.teams * s.stages; ++row)
                for (uint32_t to = begin + threadIdx.x * 4; to < end; to += blockDim.x * 4) *(uint32_t*)(block + row * s.row_bytes + source.at + to) = 0;
        }
    }

    // A vector over the columns is vector `which` of the block, in 32 bits; ones where there is none.
    // The whole block.
    template <typename T>
    __device__ __forceinline__ void keep_vector(char* block, int which, const void* v) const
    {
        for (uint32_t c = threadIdx.x * 8; c < s.span; c += blockDim.x * 8) {
            const uint32_t col = at.first + c;
            const uint4 q = load_shifted_8((const T*)v + col, v && col < s.n ? (int)min(s.n - col, 8u) : 0);
            const uint32_t w[4] = {q.x, q.y, q.z, q.w};
            float x[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) unpack<T>(w[j], x[2 * j], x[2 * j + 1]);
            // the halves of a thread's 8 apart: its lanes meet all banks once
            float4* const to = (float4*)(block + s.vectors + (which * s.span + (c & ~255u)) * 4) + c % 256 / 8;
            to[0] = v ? make_float4(x[0], x[1], x[2], x[3]) : make_float4(1.f, 1.f, 1.f, 1.f);
            to[32] = v ? make_float4(x[4], x[5], x[6], x[7]) : make_float4(1.f, 1.f, 1.f, 1.f);
        }
    }

    __device__ __forceinline__ void vector(Values<K>& v, const char* block, int which) const
    {
        const ulonglong2* const from = (const ulonglong2*)(block + s.vectors + (which * s.span + at.warp * 256 * K) * 4) + at.lane;
#pragma unroll
        for (int i = 0; i < K; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const ulonglong2 q = from[64 * i + 32 * j];
                v[i][2 * j].bits = q.x;
                v[i][2 * j + 1].bits = q.y;
            }
    }

    // A row's statistics.
    __device__ __forceinline__ float2 pair(uint32_t r, const Source& source) const
    {
        return *(const float2*)(place(source) + source.skew(r, 0));
    }

    // After a wait that ran out: the copies still on their way land before the block ends.
    __device__ __forceinline__ void drain(uint32_t first, uint32_t step) const
    {
        const uint32_t rows = first < s.m ? (s.m - first + step - 1) / step : 0;
        for (uint32_t i = 0; i < s.stages && i < rows; ++i) barrier_wait(bars + 8 * i, (rows - 1 - i) / s.stages & 1);
    }
};

// The lane's 8 values to p, of which `count` exist.  Without WIDE they go round the warp in shared
// memory (`buffer`, its own 132 words) and are stored side by side, whole words wherever the matrix
// has them; `in_warp` of the warp's 256 columns exist.  With it the row's length is a multiple of 8: all
// 8 exist or none.
template <typename T, bool WIDE>
__device__ __forceinline__ void store_row_8(T* p, int count, int in_warp, const Pair (&v)[4], uint32_t* buffer, uint32_t lane)
{
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float x, y;
        v[j].get(x, y);
        w[j] = pack<T>(x, y);
    }
    if constexpr (WIDE) {
        if (count > 0) *(uint4*)p = make_uint4(w[0], w[1], w[2], w[3]);
        return;
    }
    __syncwarp();
    *(uint4*)(buffer + 4 * lane) = make_uint4(w[0], w[1], w[2], w[3]);
    __syncwarp();
    uint16_t* const row = (uint16_t*)p - lane * 8;
    const int skew = ((uintptr_t)row & 3) != 0;                            // the first value is a word's second half
    uint32_t* const words = (uint32_t*)(row - skew);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int i = j * 32 + (int)lane, first = 2 * i - skew;            // the word holds values first and first + 1
        uint32_t word = buffer[i];
        if (skew) word = __funnelshift_r(buffer[i > 0 ? i - 1 : 0], word, 16);
        if ((j > 0 || first >= 0) && (in_warp == 256 || first + 1 < in_warp)) words[i] = word;
    }
    // a first and a last value that share their words with others
    const int last = in_warp - 1;
    if (lane == 0 && skew && in_warp > 0) row[0] = (uint16_t)buffer[0];
    if (lane == 1 && last >= skew && ((last + skew) & 1) == 0) row[last] = ((const uint16_t*)buffer)[last];
}

// The eight numbers that decide on 8 values.
__device__ __forceinline__ uint4 drop_numbers(const DropView& d, uint64_t seed, uint32_t row, uint32_t col)
{
    return philox_stream(seed, 3u, (uint64_t)(d.first_row + row) << 32 | col / 8);
}

// Dropped values are 0, whatever they were; the others are multiplied by `factor`.  A number's half of a
// word is compared at the word's top (keep is below 65536 where anything is dropped).
__device__ __forceinline__ void drop_values(Pair (&v)[4], const uint4& numbers, uint32_t keep, float factor)
{
    const uint32_t w[4] = {numbers.x, numbers.y, numbers.z, numbers.w}, below = keep << 16;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float x, y;
        (v[j] * Pair(factor)).get(x, y);
        v[j] = Pair(w[j] << 16 < below ? x : 0.f, w[j] < below ? y : 0.f);
    }
}

// columns that do not exist are 0
template <bool WIDE>
__device__ __forceinline__ void mask_values(Pair (&v)[4], int count)
{
    if (count == 8) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float x, y;
        v[j].get(x, y);
        v[j] = WIDE ? Pair(0.f) : Pair(2 * j < count ? x : 0.f, 2 * j + 1 < count ? y : 0.f);
    }
}

// A row's pieces to p, the first one's place.
template <typename T, bool WIDE, int K>
__device__ __forceinline__ void store_row(T* p, const Place<K>& at, const Values<K>& v, uint32_t* buffer)
{
#pragma unroll
    for (int i = 0; i < K; ++i) store_row_8<T, WIDE>(p + 256 * i, at.count[i], at.in_warp(i), v[i], buffer, at.lane);
}

// Vectors of a block.
enum { kAfterWeights = 0, kBeforeWeights = 1, kGateVector = 2, kAfterBiases = 3, kBeforeBiases = 4 };
template <bool FULL> constexpr int kVectors = FULL ? 5 : 3;

// f(i, j) for a thread's K x 4 pairs
template <int K, typename F>
__device__ __forceinline__ void each(F&& f)
{
#pragma unroll
    for (int i = 0; i < K; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) f(i, j);
}

enum { kSourceH = 0, kSourceResidual = 1, kSourceGate = 2 };

struct JoinView {
    const void* gate;                  // a vector, or null
    void* x;               uint64_t x_stride;              // or null
    void* y;               uint64_t y_stride;              // before.kind != none
    NormView after, before;
    DropView drop;
    float scale;
    int has_drop;
};

__device__ __forceinline__ void stages_init(uint32_t bars, uint32_t teams)
{
    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < teams * kMaxStages; ++i) barrier_init(bars + 8 * i, 1);
        barrier_init_done();
    }
    __syncthreads();
}

// The block's vectors lie in shared memory; in a cluster, all of its blocks have started, whose shared
// memory the others write to from their first sums on.
__device__ __forceinline__ void block_ready(uint32_t blocks)
{
    if (blocks > 1) cluster_arrive_wait(); else __syncthreads();
}

template <typename T, bool AFTER, bool BEFORE, bool FULL, bool WIDE, int K>
__global__ void __launch_bounds__(kJoinThreads, 1) k_join(JoinView p, const __grid_constant__ BlockShape s, uint32_t* status)
{
    __shared__ Exchange sums;
    __shared__ uint32_t buffers[WIDE ? 1 : kMaxTeams][132];
    __shared__ __align__(8) uint64_t bars[kMaxTeams * kMaxStages];
    extern __shared__ __align__(16) char rows_of_block[];
    const Place<K> at(s);
    Stages<K> stages(s, at, rows_of_block, shared_address(bars));
    if constexpr (WIDE) stages.clear(rows_of_block);
    stages_init(shared_address(bars), s.teams);
    dependency_wait();
    dependency_release();
    uint32_t* const buffer = buffers[WIDE ? 0 : threadIdx.x / 32];
    const uint64_t seed = p.drop.seed_at ? *p.drop.seed_at : p.drop.seed;
    const uint32_t step = gridDim.x / s.blocks * s.teams, first = blockIdx.x / s.blocks * s.teams + at.team;
    if (at.warp == 0)
        for (uint32_t i = 0; i < s.stages; ++i)
            if (first + i * (uint64_t)step < s.m) stages.fetch(i, first + i * step);
    stages.template keep_vector<T>(rows_of_block, kGateVector, p.gate);
    if (AFTER) stages.template keep_vector<T>(rows_of_block, kAfterWeights, p.after.weight);
    if (BEFORE) stages.template keep_vector<T>(rows_of_block, kBeforeWeights, p.before.weight);
    if (FULL && AFTER && p.after.bias) stages.template keep_vector<T>(rows_of_block, kAfterBiases, p.after.bias);
    if (FULL && BEFORE && p.before.bias) stages.template keep_vector<T>(rows_of_block, kBeforeBiases, p.before.bias);
    block_ready(s.blocks);
    auto vector = [&](Values<K>& v, int which) { stages.vector(v, rows_of_block, which); };
    uint32_t turn = 0, stage = 0, phase = 0;
    bool ok = true;
    for (uint32_t row = first; row < s.m; row += step) {
        // a wait that ran out: the row is worked on all the same, so that every warp and every block of
        // the cluster meets at the same barriers; the status says that the results are not to be used
        ok = barrier_wait(stages.bars + 8 * stage, phase) && ok;
        stages.go_to(stage);
        // everybody has done the row before this one: its stage is free
        auto refill = [&] {
            const uint64_t next = row + (uint64_t)step * (s.stages - 1);
            if (at.warp == 0 && row != first && next < s.m) stages.fetch(stage == 0 ? s.stages - 1 : stage - 1, (uint32_t)next);
        };
        Values<K> v, w;
        stages.template values<T, WIDE>(v, row, s.source[kSourceH]);
        if constexpr (AFTER) {
            const float2 st = row_statistics<FULL, WIDE, K>(sums, turn, s, at, p.after, v);
            refill();
            if (p.after.stats && at.col == 0) *(float2*)(p.after.stats + 2 * (uint64_t)row) = st;
            vector(w, kAfterWeights);
            each<K>([&](int i, int j) {
                if (FULL) v[i][j] = v[i][j] + Pair(-st.x);
                v[i][j] = v[i][j] * Pair(st.y) * w[i][j];
            });
            if (FULL && p.after.bias) {
                vector(w, kAfterBiases);
                each<K>([&](int i, int j) { v[i][j] = v[i][j] + w[i][j]; });
            }
        }
        if (p.has_drop) {
#pragma unroll
            for (int i = 0; i < K; ++i) drop_values(v[i], drop_numbers(p.drop, seed, row, at.col + 256 * i), p.drop.keep, p.drop.factor);
        }
        if (FULL && s.source[kSourceGate].base) {
            stages.template values<T, WIDE>(w, row, s.source[kSourceGate]);
            each<K>([&](int i, int j) { v[i][j] = v[i][j] * w[i][j]; });
        } else if (p.gate) {
            vector(w, kGateVector);
            each<K>([&](int i, int j) { v[i][j] = v[i][j] * w[i][j]; });
        }
        if (s.source[kSourceResidual].base) {
            stages.template values<T, WIDE>(w, row, s.source[kSourceResidual]);
            each<K>([&](int i, int j) { v[i][j] = fma(w[i][j], Pair(p.scale), v[i][j]); });
        }
        if (p.x) store_row<T, WIDE, K>((T*)p.x + (uint64_t)row * p.x_stride + at.col, at, v, buffer);
        if constexpr (BEFORE) {
            // (without a mean, columns that do not exist are 0 but for a row whose norm after is NaN)
            if (FULL || AFTER) {
#pragma unroll
                for (int i = 0; i < K; ++i) mask_values<WIDE>(v[i], at.count[i]);
            }
            const float2 st = row_statistics<FULL, WIDE, K>(sums, turn, s, at, p.before, v);
            if (!AFTER) refill();
            if (p.before.stats && at.col == 0) *(float2*)(p.before.stats + 2 * (uint64_t)row) = st;
            vector(w, kBeforeWeights);
            each<K>([&](int i, int j) {
                if (FULL) v[i][j] = v[i][j] + Pair(-st.x);
                v[i][j] = v[i][j] * Pair(st.y) * w[i][j];
            });
            if (FULL && p.before.bias) {
                vector(w, kBeforeBiases);
                each<K>([&](int i, int j) { v[i][j] = v[i][j] + w[i][j]; });
            }
            store_row<T, WIDE, K>((T*)p.y + (uint64_t)row * p.y_stride + at.col, at, v, buffer);
        }
        // a team of one warp has no barrier: its lanes meet before the stage is filled again
        __syncwarp();
        if (++stage == s.stages) stage = 0, phase ^= 1;
    }
    if (!ok) {
        stages.drain(first, step);
        if (at.lane == 0) atomicOr(status, EDEN_STATUS_TIMEOUT);
    }
    // a block's places are written by the others of its cluster as long as they run
    if (s.blocks > 1) cluster_arrive_wait();
}

// ---- backward -----------------------------------------------------------------------
enum { kBeforeWeight = 0, kBeforeBias = 1, kAfterWeight = 2, kAfterBias = 3, kGateSum = 4, kJoinSums = 5 };
enum { kSourceDx = 0, kSourceDy = 1, kSourceX = 2, kSourceXExps = 3, kSourceBefore = 4, kSourceKeptH = 5, kSourceHExps = 6, kSourceAfter = 7, kSourceGateMatrix = 8 };

struct JoinBackwardView {
    const void* gate;                  // a vector, or null
    void* d_residual;      uint64_t d_residual_stride;     // or null
    void* dh;              uint64_t dh_stride;             // or null
    void* d_gate;          uint64_t d_gate_stride;         // a matrix gate's gradient, or null
    float* partial;                    // sums over rows that are wanted: [part][number of them][n]
    uint32_t wanted;
    NormView after, before;
    DropView drop;
    float scale;
    int has_drop;
};

// Each team keeps the sums of its rows over the columns in registers; a block leaves them in its part
// of `partial`, which k_join_sums adds up.  LEVEL: 1 FULL but for biases, 2 with their sums as well.
template <typename T, bool AFTER, bool BEFORE, int LEVEL, bool WIDE, int K>
__global__ void __launch_bounds__(kJoinBackwardThreads, 1) k_join_backward(JoinBackwardView p, const __grid_constant__ BlockShape s, uint32_t* status)
{
    constexpr bool FULL = LEVEL > 0, BIASES = LEVEL > 1;
    __shared__ Exchange sums;
    __shared__ uint32_t buffers[WIDE ? 1 : kMaxTeams][132];
    __shared__ __align__(8) uint64_t bars[kMaxTeams * kMaxStages];
    extern __shared__ __align__(16) char rows_of_block[];
    const Place<K> at(s);
    Stages<K> stages(s, at, rows_of_block, shared_address(bars));
    if constexpr (WIDE) stages.clear(rows_of_block);
    stages_init(shared_address(bars), s.teams);
    dependency_wait();
    dependency_release();
    uint32_t* const buffer = buffers[WIDE ? 0 : threadIdx.x / 32];
    const uint64_t seed = p.drop.seed_at ? *p.drop.seed_at : p.drop.seed;
    const uint32_t group = blockIdx.x / s.blocks, step = gridDim.x / s.blocks * s.teams, first = group * s.teams + at.team;
    if (at.warp == 0)
        for (uint32_t i = 0; i < s.stages; ++i)
            if (first + i * (uint64_t)step < s.m) stages.fetch(i, first + i * step);
    const float over_n = 1.f / (float)s.n;
    stages.template keep_vector<T>(rows_of_block, kGateVector, p.gate);
    if (AFTER) stages.template keep_vector<T>(rows_of_block, kAfterWeights, p.after.weight);
    if (BEFORE) stages.template keep_vector<T>(rows_of_block, kBeforeWeights, p.before.weight);
    if (BIASES && AFTER && p.after.bias) stages.template keep_vector<T>(rows_of_block, kAfterBiases, p.after.bias);
    block_ready(s.blocks);
    auto vector = [&](Values<K>& v, int which) { stages.vector(v, rows_of_block, which); };
    const bool matrix_gate = FULL && s.source[kSourceGateMatrix].base, gated = p.gate || matrix_gate;
    Values<K> total[kJoinSums];
#pragma unroll
    for (int k = 0; k < kJoinSums; ++k) each<K>([&](int i, int j) { total[k][i][j] = Pair(0.f); });
    // the normalised row of an activation that was kept
    auto unit = [&](Values<K>& v, int which, uint32_t row, float2 st) {
        const bool coded = s.source[which + 1].base;
        if (coded) stages.template coded<WIDE>(v, row, s.source[which], s.source[which + 1], FULL ? 1.f : st.y);
        else stages.template values<T, WIDE>(v, row, s.source[which]);
        if (FULL) {
#pragma unroll
            for (int i = 0; i < K; ++i) {
                const Pair rate(at.count[i] > 0 ? st.y : 0.f);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[i][j] = (v[i][j] + Pair(-st.x)) * rate;
                if (!WIDE) mask_values<false>(v[i], at.count[i]);
            }
        } else if (!coded) {
            each<K>([&](int i, int j) { v[i][j] = v[i][j] * Pair(st.y); });
        }
    };
    uint32_t turn = 0, stage = 0, phase = 0;
    bool ok = true;
    for (uint32_t row = first; row < s.m; row += step) {
        ok = barrier_wait(stages.bars + 8 * stage, phase) && ok;
        stages.go_to(stage);
        auto refill = [&] {
            const uint64_t next = row + (uint64_t)step * (s.stages - 1);
            if (at.warp == 0 && row != first && next < s.m) stages.fetch(stage == 0 ? s.stages - 1 : stage - 1, (uint32_t)next);
        };
        Values<K> d, g, u;
        if constexpr (BEFORE) {
            const float2 st = stages.pair(row, s.source[kSourceBefore]);
            stages.template values<T, WIDE>(g, row, s.source[kSourceDy]);
            unit(u, kSourceX, row, st);
            Pair a(0.f), b(0.f);
            vector(d, kBeforeWeights);
            each<K>([&](int i, int j) {
                total[kBeforeWeight][i][j] = fma(g[i][j], u[i][j], total[kBeforeWeight][i][j]);
                if (BIASES) total[kBeforeBias][i][j] = total[kBeforeBias][i][j] + g[i][j];
                g[i][j] = g[i][j] * d[i][j];
                if (FULL) a = a + g[i][j];
                b = fma(g[i][j], u[i][j], b);
            });
            const float2 mean = row_sums<FULL, K>(sums, turn, s, at, a, b);
            refill();
            const Pair off(p.before.kind == EDEN_NORM_LAYER ? -mean.x * over_n : 0.f), inner(-mean.y * over_n), rate(st.y);
            if (s.source[kSourceDx].base) stages.template values<T, WIDE>(d, row, s.source[kSourceDx]);
            else each<K>([&](int i, int j) { d[i][j] = Pair(0.f); });
            each<K>([&](int i, int j) {
                if (FULL) g[i][j] = g[i][j] + off;
                d[i][j] = fma(fma(u[i][j], inner, g[i][j]), rate, d[i][j]);
            });
        } else {
            stages.template values<T, WIDE>(d, row, s.source[kSourceDx]);
        }
        if (p.d_residual) {
            each<K>([&](int i, int j) { g[i][j] = d[i][j] * Pair(p.scale); });
            store_row<T, WIDE, K>((T*)p.d_residual + (uint64_t)row * p.d_residual_stride + at.col, at, g, buffer);
        }
        uint4 numbers[K];
        if (p.has_drop) {
#pragma unroll
            for (int i = 0; i < K; ++i) {
                numbers[i] = drop_numbers(p.drop, seed, row, at.col + 256 * i);
                drop_values(d[i], numbers[i], p.drop.keep, p.drop.factor);
            }
        }
        const float2 st = AFTER ? stages.pair(row, s.source[kSourceAfter]) : make_float2(0.f, 1.f);
        if (AFTER || gated) unit(u, kSourceKeptH, row, st);
        if (gated) {
            if (AFTER) {
                vector(g, kAfterWeights);
                each<K>([&](int i, int j) { g[i][j] = g[i][j] * u[i][j]; });
            } else {
                each<K>([&](int i, int j) { g[i][j] = u[i][j]; });
            }
            if (BIASES && AFTER && p.after.bias) {
                Values<K> bias;
                vector(bias, kAfterBiases);
                each<K>([&](int i, int j) { g[i][j] = g[i][j] + bias[i][j]; });
            }
            each<K>([&](int i, int j) { g[i][j] = g[i][j] * d[i][j]; });
            // A value of h that was dropped, whatever it is.  A NaN that a norm made (of a row with an infinity or a NaN) is
            // NaN in the gradient of the norm's weight as well, and stays: to leave it out took 188 us to 252 for 16384 x 4096.
            if (!AFTER && p.has_drop) {
#pragma unroll
                for (int i = 0; i < K; ++i) drop_values(g[i], numbers[i], p.drop.keep, 1.f);
            }
            if (matrix_gate) {
                if (p.d_gate) store_row<T, WIDE, K>((T*)p.d_gate + (uint64_t)row * p.d_gate_stride + at.col, at, g, buffer);
                stages.template values<T, WIDE>(g, row, s.source[kSourceGateMatrix]);
                each<K>([&](int i, int j) { d[i][j] = d[i][j] * g[i][j]; });
            } else {
                each<K>([&](int i, int j) { total[kGateSum][i][j] = total[kGateSum][i][j] + g[i][j]; });
                vector(g, kGateVector);
                each<K>([&](int i, int j) { d[i][j] = d[i][j] * g[i][j]; });
            }
        }
        if constexpr (AFTER) {
            Pair a(0.f), b(0.f);
            if (FULL || BEFORE) {
#pragma unroll
                for (int i = 0; i < K; ++i) mask_values<WIDE>(d[i], at.count[i]);
            }
            vector(g, kAfterWeights);
            each<K>([&](int i, int j) {
                total[kAfterWeight][i][j] = fma(d[i][j], u[i][j], total[kAfterWeight][i][j]);
                if (BIASES) total[kAfterBias][i][j] = total[kAfterBias][i][j] + d[i][j];
                d[i][j] = d[i][j] * g[i][j];
                if (FULL) a = a + d[i][j];
                b = fma(d[i][j], u[i][j], b);
            });
            const float2 mean = row_sums<FULL, K>(sums, turn, s, at, a, b);
            if (!BEFORE) refill();
            const Pair off(p.after.kind == EDEN_NORM_LAYER ? -mean.x * over_n : 0.f), inner(-mean.y * over_n), rate(st.y);
            each<K>([&](int i, int j) {
                if (FULL) d[i][j] = d[i][j] + off;
                d[i][j] = fma(u[i][j], inner, d[i][j]) * rate;
            });
        }
        if (p.dh) store_row<T, WIDE, K>((T*)p.dh + (uint64_t)row * p.dh_stride + at.col, at, d, buffer);
        __syncwarp();
        if (++stage == s.stages) stage = 0, phase ^= 1;
    }
    if (!ok) {
        stages.drain(first, step);
        if (at.lane == 0) atomicOr(status, EDEN_STATUS_TIMEOUT);
    }
    if (p.wanted) {
        // the teams' sums meet in the rows' place, and are added up in the teams' order
        const uint32_t sums_wanted = __popc(p.wanted);
        __syncthreads();
        float* to = (float*)rows_of_block + at.team * sums_wanted * s.span + at.col - at.first;
#pragma unroll
        for (int k = 0; k < kJoinSums; ++k) {
            if (!(p.wanted >> k & 1)) continue;
#pragma unroll
            for (int i = 0; i < K; ++i) {
                float x[8];
#pragma unroll
                for (int j = 0; j < 4; ++j) total[k][i][j].get(x[2 * j], x[2 * j + 1]);
                *(float4*)(to + 256 * i) = make_float4(x[0], x[1], x[2], x[3]);
                *(float4*)(to + 256 * i + 4) = make_float4(x[4], x[5], x[6], x[7]);
            }
            to += s.span;
        }
        __syncthreads();
        float* const part = p.partial + (uint64_t)group * sums_wanted * s.n + at.first;
        const float* const held = (const float*)rows_of_block;
        for (uint32_t k = 0; k < sums_wanted; ++k)
            for (uint32_t c = threadIdx.x; c < at.width; c += blockDim.x) {
                float sum = 0.f;
                for (uint32_t team = 0; team < s.teams; ++team) sum += held[(team * sums_wanted + k) * s.span + c];
                part[(uint64_t)k * s.n + c] = sum;
            }
    }
    if (s.blocks > 1) cluster_arrive_wait();
}

// ---- without norms -------------------------------------------------------------------
// Nothing is summed over a row, so a block takes 256 columns a warp of its own choice and any rows:
// kPlainRows of them at a time, all of their loads on their way together (twice as many a row where rows
// do not start on 16 bytes).
constexpr int kPlainThreads = 256;
template <bool WIDE> constexpr int kPlainRows = WIDE ? 4 : 2;

struct PlainView {
    const void* h;         uint64_t h_stride;
    const void* residual;  uint64_t residual_stride;       // or null
    const void* gate;      uint64_t gate_stride;           // or null; stride 0: a vector
    void* x;               uint64_t x_stride;
    DropView drop;
    float scale;
    int has_drop;
    uint32_t m, n, warps_across;       // warps that cover a row
};

// 8 values of 16 bits as they lie in memory: a chunk, or the two that hold them.
template <bool WIDE>
struct Raw8 {
    uint4 lo, hi;
    uint32_t skew;
    int count;
    template <typename T>
    __device__ __forceinline__ void load(const T* p, int n)
    {
        count = n;
        lo = hi = make_uint4(0, 0, 0, 0);
        skew = WIDE ? 0 : (uint32_t)(uintptr_t)p & 15u;
        const uint4* const chunk = (const uint4*)((uintptr_t)p - skew);
        if (n > 0) lo = chunk[0];
        if (!WIDE && (int)skew + 2 * n > 16) hi = chunk[1];
    }
    // zeros after those that exist
    __device__ __forceinline__ uint4 get() const
    {
        uint32_t w[4] = {lo.x, lo.y, lo.z, lo.w};
        if (!WIDE) shift_words(w, lo, hi, skew);
        if (count < 8) {
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] &= count >= 2 * j + 2 ? 0xFFFFFFFFu : count == 2 * j + 1 ? 0xFFFFu : 0u;
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

template <bool WIDE, typename T>
__device__ __forceinline__ uint4 load_row_8(const T* p, int count)
{
    Raw8<WIDE> raw;
    raw.load(p, count);
    return raw.get();
}

template <typename T>
__device__ __forceinline__ void widen_8(const uint4& q, Pair (&v)[4])
{
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float x, y;
        unpack<T>(w[j], x, y);
        v[j] = Pair(x, y);
    }
}

template <typename T, bool WIDE>
__global__ void __launch_bounds__(kPlainThreads, 3) k_join_plain(PlainView p)
{
    constexpr int kRows = kPlainRows<WIDE>;
    __shared__ uint32_t buffers[WIDE ? 1 : kPlainThreads / 32][132];
    dependency_wait();
    dependency_release();
    const uint32_t lane = threadIdx.x % 32;
    uint32_t* const buffer = buffers[WIDE ? 0 : threadIdx.x / 32];
    const uint64_t unit = (uint64_t)blockIdx.x * (kPlainThreads / 32) + threadIdx.x / 32, row0 = unit / p.warps_across * kRows;
    if (row0 >= p.m) return;
    const uint32_t col = (uint32_t)(unit % p.warps_across) * 256 + lane * 8;
    const int in_warp = min(max((int)p.n - (int)(col - lane * 8), 0), 256), count = col < p.n ? (int)min(p.n - col, 8u) : 0, rows = (int)min((uint64_t)p.m - row0, (uint64_t)kRows);
    const uint64_t seed = p.drop.seed_at ? *p.drop.seed_at : p.drop.seed;
    Raw8<WIDE> h[kRows], residual[kRows];
    uint4 gate[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const int here = r < rows ? count : 0;
        h[r].load((const T*)p.h + (row0 + r) * p.h_stride + col, here);
        if (p.residual) residual[r].load((const T*)p.residual + (row0 + r) * p.residual_stride + col, here);
        if (p.gate) gate[r] = p.gate_stride ? load_row_8<WIDE>((const T*)p.gate + (row0 + r) * p.gate_stride + col, here) : load_shifted_8((const T*)p.gate + col, here);
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        if (r >= rows) break;
        Pair v[4], w[4];
        widen_8<T>(h[r].get(), v);
        if (p.has_drop) drop_values(v, drop_numbers(p.drop, seed, (uint32_t)row0 + r, col), p.drop.keep, p.drop.factor);
        if (p.gate) {
            widen_8<T>(gate[r], w);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = v[j] * w[j];
        }
        if (p.residual) {
            widen_8<T>(residual[r].get(), w);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = fma(w[j], Pair(p.scale), v[j]);
        }
        store_row_8<T, WIDE>((T*)p.x + (row0 + r) * p.x_stride + col, count, in_warp, v, buffer, lane);
    }
}

// An activation that was kept: a matrix of 16-bit values, or a checkpoint.
struct KeptView {
    const void* data;      uint64_t stride;                // null: the checkpoint
    CheckpointView held;
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
__device__ __forceinline__ void load_kept(const KeptView& k, uint64_t row, uint32_t col, int count, Pair (&v)[4])
{
    if (k.data) {
        widen_8<T>(load_row_8<WIDE>((const T*)k.data + row * k.stride + col, count), v);
        return;
    }
    const uint2 w = load_bytes_8(k.held.codes + row * k.held.codes_stride + col, count);
    const Pair scale(group_scale(count > 0 ? k.held.exps[row * k.held.exps_stride + col / kGroup] : 1u));
    code_values(w.x, scale, v[0], v[1]);
    code_values(w.y, scale, v[2], v[3]);
}

struct PlainBackwardView {
    const void* dx;        uint64_t dx_stride;
    KeptView h;                        // with a gate
    const void* gate;      uint64_t gate_stride;
    void* d_residual;      uint64_t d_residual_stride;
    void* dh;              uint64_t dh_stride;
    void* d_gate;          uint64_t d_gate_stride;
    float* partial;                    // a vector gate's sums: [run][n], or null
    DropView drop;
    float scale;
    int has_drop;
    uint32_t m, n, rows_per_run;
};

// Eight warps side by side along the columns walk down a run of rows, one at a time: two at a time spill
// (16384 x 4096 with dropout and a vector gate 201 us in place of 174, with a matrix gate 280 in place of 224).
template <typename T, bool WIDE>
__global__ void __launch_bounds__(kPlainThreads, 3) k_join_plain_backward(PlainBackwardView p)
{
    __shared__ uint32_t buffers[WIDE ? 1 : kPlainThreads / 32][132];
    dependency_wait();
    dependency_release();
    const uint32_t lane = threadIdx.x % 32, col = blockIdx.x * (kPlainThreads * 8) + threadIdx.x * 8;
    uint32_t* const buffer = buffers[WIDE ? 0 : threadIdx.x / 32];
    const int in_warp = min(max((int)p.n - (int)(col - lane * 8), 0), 256), count = col < p.n ? (int)min(p.n - col, 8u) : 0;
    const uint64_t begin = (uint64_t)blockIdx.y * p.rows_per_run, end = min((uint64_t)p.m, begin + p.rows_per_run);
    const uint64_t seed = p.drop.seed_at ? *p.drop.seed_at : p.drop.seed;
    Pair total[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) total[j] = Pair(0.f);
    uint4 vector = make_uint4(0, 0, 0, 0);
    if (p.gate && !p.gate_stride) vector = load_shifted_8((const T*)p.gate + col, count);
#pragma unroll 1
    for (uint64_t row = begin; row < end; ++row) {
        // all of a row's loads before its stores: a result may lie over any of the inputs
        Pair v[4], w[4], h[4];
        uint4 gate = vector;
        widen_8<T>(load_row_8<WIDE>((const T*)p.dx + row * p.dx_stride + col, count), v);
        if (p.gate) load_kept<WIDE, T>(p.h, row, col, count, h);
        if (p.gate && p.gate_stride) gate = load_row_8<WIDE>((const T*)p.gate + row * p.gate_stride + col, count);
        if (p.d_residual) {
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = v[j] * Pair(p.scale);
            store_row_8<T, WIDE>((T*)p.d_residual + row * p.d_residual_stride + col, count, in_warp, w, buffer, lane);
        }
        uint4 numbers;
        if (p.has_drop) {
            numbers = drop_numbers(p.drop, seed, (uint32_t)row, col);
            drop_values(v, numbers, p.drop.keep, p.drop.factor);
        }
        if (p.gate) {
#pragma unroll
            for (int j = 0; j < 4; ++j) h[j] = h[j] * v[j];
            if (p.has_drop) drop_values(h, numbers, p.drop.keep, 1.f);
            widen_8<T>(gate, w);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[j] = v[j] * w[j];
                total[j] = total[j] + h[j];
            }
            if (p.d_gate) store_row_8<T, WIDE>((T*)p.d_gate + row * p.d_gate_stride + col, count, in_warp, h, buffer, lane);
        }
        if (p.dh) store_row_8<T, WIDE>((T*)p.dh + row * p.dh_stride + col, count, in_warp, v, buffer, lane);
    }
    if (!p.partial) return;
    float* const to = p.partial + (uint64_t)blockIdx.y * p.n + col;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float x, y;
        total[j].get(x, y);
        if (2 * j < count) to[2 * j] = x;
        if (2 * j + 1 < count) to[2 * j + 1] = y;
    }
}

struct JoinSumsView {
    const float* partial;
    float* out[kJoinSums];             // in the order of the sums that are wanted
    uint32_t parts, n, sums;
    int accumulate;
};

// out[i][col] (+)= the sum of the parts' sums i: 32 columns per block, each warp every eighth
// part, the eight added in order
static __global__ void __launch_bounds__(256) k_join_sums(JoinSumsView p)
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
