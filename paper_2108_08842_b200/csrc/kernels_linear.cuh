// The three products of a linear layer and what follows them in the same kernel.
//   forward       y  = act(x W^T + b) + r       rows = tokens,  columns = n, sum over k
//   input grad    dx = (dz W + r) * act'(z)     rows = tokens,  columns = k, sum over n
//   weight grad   dW = dz^T x                   rows = n,       columns = k, sum over tokens
#pragma once

#include "kernels_checkpoint.cuh"
#include "tensor_core.cuh"

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
    int grain_out, grain_residual, grain_codes, grain_bias;      // bytes that all rows start on, at most 32
};

// ---- epilogue -----------------------------------------------------------------------
// A warp finishes 32 rows x 32 columns at a time, a row per lane.  How it reaches a matrix
// depends on the largest power of two that all its rows start on (its grain):
//   32 bytes   the lane reads or writes its own row, whole 32-byte sectors
//   16 bytes   through a buffer in shared memory, so that the lanes of an access take
//              consecutive 16-byte pieces of a few rows
//   less       likewise: reads take whole 4-byte words and undo each row's own misalignment by
//              a funnel shift between buffer and registers; stores take words where all rows
//              start on one, else single elements (words with partial ends branched, and took
//              3750 cycles a piece)
// A lane per row with less than a sector each took 451 us for 7376 x 6088 x 376 results that
// start on 16 bytes, against 48 us.
constexpr int kOutWords = 32 * 20, kStageWords = kOutWords + 32 * 12;       // a warp's buffer: 16-bit rows, codes

__device__ __forceinline__ void copy_async_16(uint32_t to, const void* from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}

__device__ __forceinline__ void copy_async_4(uint32_t to, const void* from)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(from) : "memory");
}

__device__ __forceinline__ void copy_async_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Rows of 32 elements of 1 or 2 bytes.  In the buffer a row of 16-byte pieces has 4 words of
// padding (128-bit accesses of eight lanes' rows then meet all banks once), a row of words one
// (an odd pitch), the word that only shifted rows touch.
template <int ELEM>
struct Rows {
    static constexpr int kWords = 8 * ELEM, kPiecePitch = kWords + 4, kPitch = kWords + 1;

    // f(row, piece) for the lane's share of 32 rows of PER_ROW pieces, a power of two
    template <int PER_ROW, typename F>
    static __device__ __forceinline__ void share(F&& f)
    {
        const int lane = threadIdx.x % 32;
#pragma unroll 4
        for (int i = 0; i < PER_ROW; ++i) f(i * (32 / PER_ROW) + lane / PER_ROW, lane % PER_ROW);
    }

    // matrix -> buffer, on its way; `rows` rows and `count` elements of the piece at `from` exist
    static __device__ __forceinline__ void fetch(uint32_t* buffer, const char* from, uint64_t stride, int rows, int count, int grain)
    {
        const uint32_t to = shared_address(buffer);
        if (grain >= 16 && count == 32) {
            share<kWords / 4>([&](int r, int piece) {
                if (r < rows) copy_async_16(to + (r * kPiecePitch + 4 * piece) * 4, from + r * stride + 16 * piece);
            });
        } else {
            auto word = [&](int r, int at) {
                const char* row = from + r * stride;
                const int off = (int)((uintptr_t)row & 3);
                if (r < rows && 4 * at < off + count * ELEM) copy_async_4(to + (r * kPitch + at) * 4, row - off + 4 * at);
            };
            share<kWords>(word);
            word(threadIdx.x % 32, kWords);
        }
    }

    // buffer -> the lane's row, once the fetch is in
    static __device__ __forceinline__ void take(uint32_t (&w)[kWords], const uint32_t* buffer, const char* from, uint64_t stride, int count,
                                                int grain)
    {
        const int lane = threadIdx.x % 32;
        copy_async_wait();
        __syncwarp();
        if (grain >= 16 && count == 32) {
#pragma unroll
            for (int j = 0; j < kWords / 4; ++j) *(uint4*)(w + 4 * j) = *(const uint4*)(buffer + lane * kPiecePitch + 4 * j);
        } else {
            const uint32_t shift = 8 * (uint32_t)((uintptr_t)(from + lane * stride) & 3);
#pragma unroll
            for (int j = 0; j < kWords; ++j) w[j] = __funnelshift_r(buffer[lane * kPitch + j], buffer[lane * kPitch + j + 1], shift);
        }
        __syncwarp();
    }

    // matrix -> the lane's row
    static __device__ __forceinline__ void get(uint32_t (&w)[kWords], const char* from, uint64_t stride, int rows, int count, int grain,
                                               uint32_t* buffer)
    {
        const int lane = threadIdx.x % 32;
        if (grain == 32 && count == 32) {
            if (lane < rows) {
#pragma unroll
                for (int i = 0; i < ELEM; ++i) load_32b(from + lane * stride + 32 * i, *(uint32_t(*)[8])(w + 8 * i));
            }
            return;
        }
        fetch(buffer, from, stride, rows, count, grain);
        take(w, buffer, from, stride, count, grain);
    }

    // the lane's row -> matrix
    static __device__ __forceinline__ void put(const uint32_t (&w)[kWords], char* to, uint64_t stride, int rows, int count, int grain,
                                               uint32_t* buffer)
    {
        const int lane = threadIdx.x % 32;
        if (grain == 32 && count == 32) {
            if (lane >= rows) return;
#pragma unroll
            for (int i = 0; i < ELEM; ++i) store_32b(to + lane * stride + 32 * i, *(const uint32_t(*)[8])(w + 8 * i));
            return;
        }
        if (grain >= 16 && count == 32) {
#pragma unroll
            for (int j = 0; j < kWords / 4; ++j) *(uint4*)(buffer + lane * kPiecePitch + 4 * j) = *(const uint4*)(w + 4 * j);
            __syncwarp();
            share<kWords / 4>([&](int r, int piece) {
                if (r < rows) *(uint4*)(to + r * stride + 16 * piece) = *(const uint4*)(buffer + r * kPiecePitch + 4 * piece);
            });
        } else {
            // no branches: every store is predicated, so that several are on their way
#pragma unroll
            for (int j = 0; j < kWords; ++j) buffer[lane * kPitch + j] = w[j];
            __syncwarp();
            if (grain >= 4 && (count * ELEM & 3) == 0) {
                constexpr int at_once = 32 / kWords;
                const int word = lane % kWords;
                char* row = to + (lane / kWords) * stride + 4 * word;
                const uint32_t* from = buffer + (lane / kWords) * kPitch + word;
                const int mine = 4 * word < count * ELEM ? rows - lane / kWords : 0;
#pragma unroll 8
                for (int r = 0; r < 32; r += at_once) {
                    if (r < mine) *(uint32_t*)row = *from;
                    row += at_once * stride;
                    from += at_once * kPitch;
                }
            } else {
                using U = std::conditional_t<ELEM == 1, uint8_t, uint16_t>;
                char* row = to + lane * ELEM;
                const U* from = (const U*)buffer + lane;
                const int mine = lane < count ? rows : 0;
#pragma unroll 8
                for (int r = 0; r < 32; ++r) {
                    if (r < mine) *(U*)row = *from;
                    row += stride;
                    from += kPitch * 4 / ELEM;
                }
            }
        }
        __syncwarp();
    }
};

// Rows of 32 fp32 values, whole 128-byte lines where they are aligned, always through the buffer:
// eight lanes to a row touch each line once, where a lane per row with 32 bytes a store touches
// it four times (6656 x 1984 gradients of 64 tokens took 20 us so, 13.9 like this).  16-byte chunk c of row r
// lies in place c ^ (r % 8) of its row: no two lanes of an access meet in a bank.
struct WideRows {
    static __device__ __forceinline__ float4* place(uint32_t* buffer, int row, int chunk) { return (float4*)buffer + row * 8 + (chunk ^ (row & 7)); }

    // v[j] += the lane's row of the piece at `from`
    static __device__ __forceinline__ void add(float (&v)[32], const char* from, uint64_t stride, int rows, int count, int grain, uint32_t* buffer)
    {
        const int lane = threadIdx.x % 32;
        __syncwarp();
        if (grain >= 16 && count == 32) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int r = 4 * i + lane / 8;
                if (r < rows) copy_async_16(shared_address(place(buffer, r, lane % 8)), from + r * stride + 16 * (lane % 8));
            }
        } else {
#pragma unroll 8
            for (int r = 0; r < 32; ++r)
                if (r < rows && lane < count) copy_async_4(shared_address((float*)place(buffer, r, lane / 4) + lane % 4), from + r * stride + 4 * lane);
        }
        copy_async_wait();
        __syncwarp();
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const float4 f = *place(buffer, lane, c);
            v[4 * c] += f.x;
            v[4 * c + 1] += f.y;
            v[4 * c + 2] += f.z;
            v[4 * c + 3] += f.w;
        }
        __syncwarp();
    }

    static __device__ __forceinline__ void put(const float (&v)[32], char* to, uint64_t stride, int rows, int count, int grain, uint32_t* buffer)
    {
        const int lane = threadIdx.x % 32;
#pragma unroll
        for (int c = 0; c < 8; ++c) *place(buffer, lane, c) = make_float4(v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
        __syncwarp();
        if (grain >= 16 && count == 32) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int r = 4 * i + lane / 8;
                if (r < rows) *(float4*)(to + r * stride + 16 * (lane % 8)) = *place(buffer, r, lane % 8);
            }
        } else if (grain >= 8 && count == 32) {
            const int q = lane % 16;
#pragma unroll 8
            for (int r = lane / 16; r < 32; r += 2)
                if (r < rows) *(float2*)(to + r * stride + 8 * q) = ((const float2*)place(buffer, r, q / 2))[q % 2];
        } else {
            const int mine = lane < count ? rows : 0;
#pragma unroll 8
            for (int r = 0; r < 32; ++r)
                if (r < mine) *(float*)(to + r * stride + 4 * lane) = ((const float*)place(buffer, r, lane / 4))[lane % 4];
        }
        __syncwarp();
    }
};

// The piece at (row0, col0): rows and columns that exist.
struct Piece {
    uint64_t row0, col0;
    int rows, count;
    __device__ __forceinline__ Piece(const LinearEpilogue& p, uint64_t row, uint64_t col)
        : row0(row), col0(col), rows((int)(p.rows - row < 32 ? p.rows - row : 32)), count((int)(p.cols - col < 32 ? p.cols - col : 32)) {}
    __device__ __forceinline__ char* in(const void* matrix, uint64_t stride, int size) const { return (char*)matrix + (row0 * stride + col0) * size; }
};

// The codes and exponents of a piece's pre-activation, set on their way while the piece before it
// is finished.
__device__ __forceinline__ void fetch_codes(const Piece& at, const LinearEpilogue& p, uint32_t* buffer, uint32_t& exp)
{
    const int lane = threadIdx.x % 32;
    if (p.act == EDEN_ACT_NONE) return;
    Rows<1>::fetch(buffer + kOutWords, at.in(p.ckpt.codes, p.ckpt.codes_stride, 1), p.ckpt.codes_stride, at.rows, at.count, p.grain_codes);
    exp = lane < at.rows ? p.ckpt.exps[(at.row0 + lane) * p.ckpt.exps_stride + at.col0 / kGroup] : 0;
}

// v[32]: fp32 sums of the lane's row of a piece.  All 32 lanes of the warp call this together;
// `buffer` is the warp's own.  Input grad: the piece's codes were fetched, with their `exp`, and
// `next`'s are, if there is a piece after it.
template <int OP, typename T>
__device__ __forceinline__ void linear_epilogue(float (&v)[32], const Piece& at, const LinearEpilogue& p, uint32_t* buffer, uint32_t& exp,
                                                const Piece* next)
{
    const int lane = threadIdx.x % 32;
    const bool live = lane < at.rows;
    if constexpr (OP == kWeightGrad) {
        char* out = at.in(p.out, p.out_stride, 4);
        if (p.accumulate) WideRows::add(v, out, p.out_stride * 4, at.rows, at.count, p.grain_out, buffer);
        WideRows::put(v, out, p.out_stride * 4, at.rows, at.count, p.grain_out, buffer);
        return;
    }
    auto add_halves = [&](const uint32_t (&w)[16]) {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            float lo, hi;
            unpack<T>(w[j], lo, hi);
            (Pair(v[2 * j], v[2 * j + 1]) + Pair(lo, hi)).get(v[2 * j], v[2 * j + 1]);
        }
    };
    auto add_residual = [&]() {
        if (!p.residual) return;
        uint32_t w[16];
        Rows<2>::get(w, at.in(p.residual, p.residual_stride, 2), p.residual_stride * 2, at.rows, at.count, p.grain_residual, buffer);
        add_halves(w);
    };
    if constexpr (OP == kForward) {
        if (p.bias) {
            const T* bias = (const T*)p.bias + at.col0;
            if (at.count == 32 && p.grain_bias == 32) {
                uint32_t w[16];
                load_32b(bias, *(uint32_t(*)[8])w);
                load_32b(bias + 16, *(uint32_t(*)[8])(w + 8));
                add_halves(w);
            } else {
                const float mine = lane < at.count ? to_float(bias[lane]) : 0.f;
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] += __shfl_sync(0xFFFFFFFFu, mine, j);
            }
        }
        // the 8-bit form of the row's group
        auto save = [&]() {
            float most = 0.f;
            if (at.count == 32) {
#pragma unroll
                for (int j = 0; j < 32; j += 2) most = max_magnitude(most, v[j], v[j + 1]);
            } else {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (j < at.count) most = max_magnitude(most, v[j], v[j]);
            }
            const uint32_t e = group_exponent(magnitude_bits(most));
            const float inverse = group_inverse(e);
            if (live) p.ckpt.exps[(at.row0 + lane) * p.ckpt.exps_stride + at.col0 / kGroup] = (uint8_t)e;
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = group_codes(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3], inverse);
            Rows<1>::put(w, at.in(p.ckpt.codes, p.ckpt.codes_stride, 1), p.ckpt.codes_stride, at.rows, at.count, p.grain_codes, buffer);
        };
        if (p.save == EDEN_SAVE_PRE) save();
        with_act(p.act, [&](auto a) {
#pragma unroll
            for (int j = 0; j < 32; j += 2) act_value<decltype(a)::value>(Pair(v[j], v[j + 1])).get(v[j], v[j + 1]);
        });
        add_residual();
        if (p.save == EDEN_SAVE_OUT) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = to_float(from_float<T>(v[j]));
            save();
        }
    } else {
        add_residual();
        if (p.act != EDEN_ACT_NONE) {
            uint32_t w[8];
            Rows<1>::take(w, buffer + kOutWords, at.in(p.ckpt.codes, p.ckpt.codes_stride, 1), p.ckpt.codes_stride, at.count, p.grain_codes);
            const float scale = live ? slope_scale(exp) : 0.f;
            if (next) fetch_codes(*next, p, buffer, exp);
            with_act(p.act, [&](auto a) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    Pair z01, z23;
                    code_values(w[i], Pair(scale), z01, z23);
                    (Pair(v[4 * i], v[4 * i + 1]) * act_slope<decltype(a)::value>(z01)).get(v[4 * i], v[4 * i + 1]);
                    (Pair(v[4 * i + 2], v[4 * i + 3]) * act_slope<decltype(a)::value>(z23)).get(v[4 * i + 2], v[4 * i + 3]);
                }
            });
        }
        if (p.column_sums) {
            // lane j ends with the sum of column j: halves are exchanged and added five times
            float s[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) s[j] = live ? v[j] : 0.f;
#pragma unroll
            for (int half = 16; half >= 1; half /= 2) {
                const bool upper = lane & half;
#pragma unroll
                for (int j = 0; j < half; ++j) {
                    const float keep = upper ? s[j + half] : s[j], give = upper ? s[j] : s[j + half];
                    s[j] = keep + __shfl_xor_sync(0xFFFFFFFFu, give, half);
                }
            }
            if (lane < at.count) p.column_sums[at.row0 / 32 * p.cols + at.col0 + lane] = s[0];
        }
    }
    uint32_t w[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) w[j] = pack<T>(v[2 * j], v[2 * j + 1]);
    Rows<2>::put(w, at.in(p.out, p.out_stride, 2), p.out_stride * 2, at.rows, at.count, p.grain_out, buffer);
}

// Tiles of the result, in the order in which they are handed out: bands of kBand tile rows,
// column by column, so that the tiles in flight share few rows of A and of B in the L2 cache.
struct TileGrid {
    uint32_t rows, cols;               // tiles
    uint32_t begin, end;               // those of this launch, in their order
    uint32_t depth_steps;              // steps of the shape's kDepth along the sum
    uint32_t splits;                   // parts of the sum, one block (pair) of a cluster each
};

constexpr uint32_t kBand = 8;

__device__ __forceinline__ void tile_at(const TileGrid& g, uint32_t t, uint32_t& row, uint32_t& col)
{
    const uint32_t per_band = kBand * g.cols, first = t / per_band * kBand;
    const uint32_t height = min(kBand, g.rows - first), in_band = t % per_band;
    row = first + in_band % height;
    col = in_band / height;
}

// Shape of a block's share of a tile: 128 rows of A and BN / CG rows of B per step along the sum.
// Each of the four quarters of its 128 rows of sums has SIDES epilogue warps side by side.  A
// step is one box of 64 for pairs, whose four products outlast their issue (512 cycles), and two
// for single blocks: waiting for a stage, releasing it and issuing four products takes 410 to 440
// cycles whatever their size, of which 180 are the stage's.
template <int CG, int BN, int SIDES>
struct LinearShape {
    static constexpr int kRowsB = BN / CG, kBoxes = CG == 1 ? 2 : 1, kDepth = 64 * kBoxes;
    static constexpr uint32_t kBoxA = 128 * 128, kBoxB = kRowsB * 128;
    static constexpr uint32_t kBytesA = kBoxes * kBoxA, kStageBytes = kBoxes * (kBoxA + kBoxB);
    static constexpr int kStages = CG == 2 ? (SIDES == 2 ? 6 : 5) : BN == 128 ? 3 : 4;
    static constexpr int kPieces = BN / SIDES / 32;      // pieces of 32 columns per warp
    static constexpr int kWarps = 4 * SIDES, kThreads = 128 + 32 * kWarps;
    static constexpr uint32_t kBuffers = kStages * kStageBytes, kBarriers = kBuffers + kWarps * kStageWords * 4;
    static constexpr uint32_t kSharedBytes = kBarriers + (2 * kStages + 5) * 8 + 16;
    static constexpr uint32_t kColumns = 2 * BN;       // tensor memory: two tiles' sums
    static_assert(kSharedBytes <= 227 * 1024, "a block's shared memory");
};

// The tensor cores cut off what their fp32 sums cannot hold, always towards zero, so long sums
// drift: 512 products of 16 left fp32 weight gradients 4e-6 off.  Where a result of 32 bits comes
// of them (weight gradients, the column sums of input gradients) or codes do (a value between two
// of them shows the smallest difference: of 16384 steps 6.5e-4 of the codes' values were off,
// 1.5e-4 in fp32), they are taken out of tensor memory every kPromote products of 64 and added up,
// rounded to nearest.  Whatever the length, weight gradients are 1.4e-7 off then in bf16 and 4.3e-7
// in fp16, whose products have bits to cut off too (2.9e-7 and 8e-7 in runs of 1024; plain fp32 over
// 4096 steps 2.5e-7 and 6.2e-7), column sums 6.5e-7 (1.3e-6 of 1024 steps in one run), codes 1e-4.
// Results of 16 bits alone do not show the drift: 1.66e-3 either way.
//   Two runs: each has its half of the tensor memory; they are added up in the second one's place, and
// the next tile's first run takes the other.  Linear 4096 x 4096 x 1024 with gelu and codes 45 -> 47 us.
//   More: added up in registers while the next run is summed.  8192 x 4096 x 4096 with codes 198 -> 216
// us, weight gradients 4096 x 4096 over 8191 tokens 209 -> 211 against runs of 1024.
// RUNS: a kernel of its own, since its registers cost the others' epilogue time.
constexpr uint32_t kPromote = 8;

// D = A B^T for tiles of 128 * CG x BN, persistent: block (pair) c takes tiles c, c + blocks, ...
//   warp 0   fills the stages with tensor copies, kStages ahead of the products
//   warp 1   (of the pair's first block) issues the products
//   warp 2   owns the tensor memory
//   warps 4+ read finished sums from tensor memory and run the epilogue, while the products
//            of the next tile (or of the next kPromote steps) fill its other half.  Eight warps
//            (SIDES = 2), or sixteen with 104 registers each and a stage less where an epilogue
//            that is more than a store may outlast the products: 36 against 40 us for bias, gelu
//            and 8-bit codes on 4096 x 4096 x 1024 in one run, but 176 against 171 us for
//            8192 x 4096 x 4096
// CG = 2: the blocks of a pair hold 128 rows of A and half of the rows of B each; the first
// one's barriers count both blocks' bytes, and its products write both blocks' sums.
// SPLIT: one tile per cluster.  Its blocks (pairs) take a part of the sum each, leave their
// sums in shared memory, and then every block joins and finishes a share of the tile's 32 x 32
// pieces, adding the parts in their order.
template <int OP, typename T, int CG, int BN, bool SPLIT, bool RUNS, int SIDES>
__global__ void __launch_bounds__(LinearShape<CG, BN, SIDES>::kThreads, 1)
k_linear(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, LinearEpilogue p, TileGrid grid,
         uint32_t* status)
{
    using S = LinearShape<CG, BN, SIDES>;
    constexpr bool a_mn = OP == kWeightGrad, b_mn = OP != kForward;
    constexpr uint32_t descriptor = product_descriptor(std::is_same_v<T, __nv_bfloat16>, a_mn, b_mn, 128 * CG, BN);

    extern __shared__ __align__(1024) char raw[];          // tiles of 128-byte rows swizzle by address bits 7 to 9
    const uint32_t base = shared_address(raw);
    const uint32_t full = base + S::kBarriers, empty = full + 8 * S::kStages;
    const uint32_t sums_full = empty + 8 * S::kStages, sums_empty = sums_full + 16, drained = sums_empty + 16, slot = drained + 8;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    uint32_t* const buffer = (uint32_t*)(raw + S::kBuffers) + (warp >= 4 ? warp - 4 : 0) * kStageWords;
    const uint32_t in_cluster = CG == 2 || SPLIT ? cluster_rank() : 0, rank = in_cluster % CG, leader = in_cluster - rank;
    const uint32_t splits = SPLIT ? grid.splits : 1, part = in_cluster / CG;
    const uint32_t first = grid.begin + blockIdx.x / (CG * splits), step = gridDim.x / (CG * splits);
    const uint32_t depth_begin = (uint32_t)((uint64_t)grid.depth_steps * part / splits);
    const uint32_t depth_end = (uint32_t)((uint64_t)grid.depth_steps * (part + 1) / splits);
    constexpr uint32_t run = RUNS ? kPromote / S::kBoxes : 1u << 30;        // steps summed in tensor memory

    if (threadIdx.x == 0) {
        for (int i = 0; i < S::kStages; ++i) {
            barrier_init(full + 8 * i, 1);
            barrier_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            barrier_init(sums_full + 8 * i, 1);
            barrier_init(sums_empty + 8 * i, S::kWarps * CG);
        }
        barrier_init(drained, 1);
        barrier_init_done();
        prefetch_map(&map_a);
        prefetch_map(&map_b);
    }
    if (warp == 2) tmem_alloc<CG>(slot, S::kColumns);
    tmem_fence_before();
    if constexpr (CG == 2 || SPLIT) cluster_arrive_wait(); else __syncthreads();
    tmem_fence_after();
    dependency_wait();
    dependency_release();
    uint32_t sums;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(sums) : "r"(slot));

    bool ok = true;
    if (warp < 4) {
        registers_down<SIDES>();         // the block's registers move to the epilogue's warps
        if (warp == 0) {
            uint32_t s = 0, phase = 0, issued = 0;
            for (uint32_t t = first; t < grid.end && ok; t += step) {
                uint32_t tile_row, tile_col;
                tile_at(grid, t, tile_row, tile_col);
                const int row = (int)(tile_row * 128 * CG + rank * 128), col = (int)(tile_col * BN + rank * S::kRowsB);
                for (uint32_t d = depth_begin; d < depth_end; ++d) {
                    if (!(ok = barrier_wait(empty + 8 * s, phase ^ 1))) break;
                    if (elected()) {
                        const uint32_t bar = CG == 2 ? address_in(full + 8 * s, leader) : full + 8 * s;
                        if (rank == 0) barrier_expect(full + 8 * s, CG * S::kStageBytes);
                        const uint32_t a = base + s * S::kStageBytes, b = a + S::kBytesA;
#pragma unroll
                        for (int box = 0; box < S::kBoxes; ++box) {
                            const int depth = (int)d * S::kDepth + 64 * box;
                            if constexpr (a_mn) {
                                copy_box<CG>(a + box * S::kBoxA, &map_a, row, depth, bar);
                                copy_box<CG>(a + box * S::kBoxA + 8192, &map_a, row + 64, depth, bar);
                            } else {
                                copy_box<CG>(a + box * S::kBoxA, &map_a, depth, row, bar);
                            }
                            if constexpr (b_mn) {
#pragma unroll
                                for (int i = 0; i < S::kRowsB / 64; ++i)
                                    copy_box<CG>(b + box * S::kBoxB + 8192 * i, &map_b, col + 64 * i, depth, bar);
                            } else {
                                copy_box<CG>(b + box * S::kBoxB, &map_b, depth, col, bar);
                            }
                        }
                    }
                    __syncwarp();
                    issued = min(issued + 1, (uint32_t)S::kStages);
                    if (++s == S::kStages) { s = 0; phase ^= 1; }
                }
            }
            // the products' last arrivals on this block's barriers land before the block ends
            uint32_t drain = s, drain_phase = phase;
            for (int i = 0; i < S::kStages && ok; ++i) {
                ok = barrier_wait(empty + 8 * drain, drain_phase ^ 1);
                if (++drain == S::kStages) { drain = 0; drain_phase ^= 1; }
            }
            // gave up: the copies still on their way (counted by the pair's first block) land as well;
            // s is the stage after the last one that was filled
            if (!ok && rank == 0)
                for (; issued > 0; --issued) {
                    if (s-- == 0) { s = S::kStages - 1; phase ^= 1; }
                    barrier_wait(full + 8 * s, phase);
                }
        } else if (warp == 1) {
            if (rank == 0) {
                uint32_t s = 0, phase = 0, half = 0, half_phase = 1;
                const uint32_t low_a = descriptor_low(base), low_b = descriptor_low(base + S::kBytesA);
                uint32_t a = low_a, b = low_b;
                for (uint32_t t = first; t < grid.end && ok; t += step) {
                    for (uint32_t part_begin = depth_begin; part_begin < depth_end && ok; part_begin += run) {
                        const uint32_t d_address = sums + half * BN, part_end = depth_end - part_begin < run ? depth_end : part_begin + run;
                        if (!(ok = barrier_wait(sums_empty + 8 * half, half_phase))) break;
                        tmem_fence_after();
                        for (uint32_t d = part_begin; d < part_end; ++d) {
                            if (!(ok = barrier_wait(full + 8 * s, phase))) break;
                            tmem_fence_after();
                            if (elected()) {
#pragma unroll
                                for (int k = 0; k < 4 * S::kBoxes; ++k)
                                    tile_product<CG>(d_address, tile_descriptor(a + k / 4 * (S::kBoxA / 16) + k % 4 * (a_mn ? 2048 / 16 : 32 / 16)),
                                                     tile_descriptor(b + k / 4 * (S::kBoxB / 16) + k % 4 * (b_mn ? 2048 / 16 : 32 / 16)),
                                                     descriptor, k > 0 || d > part_begin);
                                tile_commit<CG>(empty + 8 * s, leader);
                                if (d + 1 == part_end) tile_commit<CG>(sums_full + 8 * half, leader);
                            }
                            __syncwarp();
                            a += S::kStageBytes / 16;
                            b += S::kStageBytes / 16;
                            if (++s == S::kStages) { s = 0; phase ^= 1; a = low_a; b = low_b; }
                        }
                        half ^= 1;
                        half_phase ^= half ^ 1;
                    }
                }
                if (!ok) {
                    if (elected()) tile_commit<CG>(drained, leader);
                    __syncwarp();
                    barrier_wait(drained, 0);
                }
            }
        }
        __syncwarp();
        if constexpr (SPLIT) cluster_arrive_wait();
    } else {
        registers_up<SIDES>();
        const int quarter = warp % 4, side = (warp - 4) / 4;
        const uint32_t my_sums = sums + ((uint32_t)quarter * 32 << 16) + side * S::kPieces * 32;
        uint32_t half = 0, phase = 0;
        const bool both = RUNS && depth_end - depth_begin > run && depth_end - depth_begin <= 2 * run;
        auto release = [&]() {
            tmem_fence_before();
            __syncwarp();
            if (lane == 0) barrier_arrive_remote(CG == 2 ? address_in(sums_empty + 8 * half, leader) : sums_empty + 8 * half);
        };
        for (uint32_t t = first; t < grid.end && ok; t += step) {
            uint32_t tile_row, tile_col;
            tile_at(grid, t, tile_row, tile_col);
            const uint64_t row0 = (uint64_t)tile_row * 128 * CG + rank * 128 + quarter * 32;
            const uint32_t in_tile = side * S::kPieces * 32;
            uint32_t exp = 0;
            if (OP == kInputGrad && !SPLIT && row0 < p.rows && (uint64_t)tile_col * BN + in_tile < p.cols)
                fetch_codes(Piece(p, row0, (uint64_t)tile_col * BN + in_tile), p, buffer, exp);
            auto finish = [&](float (&v)[32], int c) {
                if constexpr (SPLIT) {
                    // [column][row], over the stages: every product that read them is done
#pragma unroll
                    for (int j = 0; j < 32; ++j) shared_store(base + ((in_tile + 32 * c + j) * 128 + quarter * 32 + lane) * 4, v[j]);
                } else {
                    const uint64_t col0 = (uint64_t)tile_col * BN + in_tile + 32 * c;
                    if (row0 < p.rows && col0 < p.cols) {
                        const Piece next(p, row0, col0 + 32);
                        linear_epilogue<OP, T>(v, Piece(p, row0, col0), p, buffer, exp, c + 1 < S::kPieces && col0 + 32 < p.cols ? &next : nullptr);
                    }
                }
            };
            if (RUNS && SIDES == 2 && depth_end - depth_begin > 2 * run) {
                // the runs added up, and the total put back in the last one's place
                float total[S::kPieces][32];
                for (uint32_t part_begin = depth_begin;; part_begin += run) {
                    if (!(ok = barrier_wait(sums_full + 8 * half, phase))) break;
                    tmem_fence_after();
                    const bool last = depth_end - part_begin <= run;
#pragma unroll
                    for (int c = 0; c < S::kPieces; ++c) {
                        float v[32];
                        tmem_load(my_sums + half * BN + 32 * c, v);
#pragma unroll
                        for (int j = 0; j < 32; j += 2) {
                            const Pair sum = part_begin == depth_begin ? Pair(v[j], v[j + 1]) : Pair(total[c][j], total[c][j + 1]) + Pair(v[j], v[j + 1]);
                            sum.get(total[c][j], total[c][j + 1]);
                        }
                        if (last) tmem_store(my_sums + half * BN + 32 * c, total[c]);
                    }
                    if (last) break;
                    release();
                    half ^= 1;
                    phase ^= half ^ 1;
                }
            } else {
                ok = barrier_wait(sums_full + 8 * half, phase);
                if (both && ok && (ok = barrier_wait(sums_full + 8, phase))) {   // half is 0 for every tile
                    // the two runs added up in the second one's place
                    tmem_fence_after();
#pragma unroll 1
                    for (int c = 0; c < S::kPieces; ++c) {
                        float v[32], w[32];
                        tmem_load(my_sums + 32 * c, v);
                        tmem_load(my_sums + BN + 32 * c, w);
#pragma unroll
                        for (int j = 0; j < 32; j += 2) (Pair(v[j], v[j + 1]) + Pair(w[j], w[j + 1])).get(v[j], v[j + 1]);
                        tmem_store(my_sums + BN + 32 * c, v);
                    }
                    release();
                    half = 1;
                }
            }
            if (!ok) break;
            tmem_fence_after();
#pragma unroll 1
            for (int c = 0; c < S::kPieces; ++c) {
                float v[32];
                __syncwarp();
                tmem_load(my_sums + half * BN + 32 * c, v);
                if (c == S::kPieces - 1) release();
                finish(v, c);
            }
            half ^= 1;
            phase ^= half ^ 1;
        }
        __syncwarp();
        if constexpr (SPLIT) {
            cluster_arrive_wait();
            uint32_t tile_row, tile_col;
            tile_at(grid, first, tile_row, tile_col);
            for (uint32_t unit = part + splits * (warp - 4); unit < BN / 8; unit += splits * S::kWarps) {
                const uint32_t quarter = unit % 4, in_tile = unit / 4 * 32;
                const uint64_t row0 = (uint64_t)tile_row * 128 * CG + rank * 128 + quarter * 32, col0 = (uint64_t)tile_col * BN + in_tile;
                // A piece without a row or column of the result is not read: its values would not be
                // waited for, and the block that holds them could end before they are fetched.
                if (col0 >= p.cols || row0 >= p.rows) continue;
                const Piece at(p, row0, col0);
                uint32_t exp = 0;
                if (OP == kInputGrad) fetch_codes(at, p, buffer, exp);
                float v[32];
                for (uint32_t i = 0; i < splits; ++i) {
                    const uint32_t from = address_in(base, i * CG + rank) + (in_tile * 128 + quarter * 32 + lane) * 4;
                    float w[32];
#pragma unroll
                    for (int j = 0; j < 32; ++j) w[j] = cluster_load(from + j * 512);
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] = i == 0 ? w[j] : v[j] + w[j];
                }
                linear_epilogue<OP, T>(v, at, p, buffer, exp, nullptr);
            }
        }
    }
    if (!ok) {
        copy_async_wait();
        atomicOr(status, EDEN_STATUS_TIMEOUT);
    }
    __syncwarp();
    tmem_fence_before();
    if constexpr (CG == 2 || SPLIT) cluster_arrive_wait(); else __syncthreads();
    tmem_fence_after();
    if (warp == 2) tmem_free<CG>(sums, S::kColumns);
}

// ---- few tokens ---------------------------------------------------------------------
// y [m, n] for m <= 8 * NT: every weight is read once and used m times, so reading W is all
// that takes time.  A block takes 16 * R rows of W; its 16 warps take steps of 64 along the sum
// in turn, all loads of one or two steps on their way together, straight to registers in the
// layout of the 16 x 8 x 16 product: the sum's index may be permuted alike in W and in x, so
// each lane loads 16 consecutive bytes and feeds them as the fragments of two products.  The
// 16 warps' sums are added in their order.  R = 2 where groups of 32 results are saved.  Where
// few rows of W meet a long sum, a cluster of blocks shares it: each block adds up its warps, and
// the first one adds the blocks' sums, out of their shared memory, in their order (SHARED; the
// same code with a cluster of one block took 7.4 us where this takes 4.8).
// Two blocks on an SM hide each other's ends: one with twice the loads on their way took 5.8 us
// against 4.1 for 13 x 2731 x 1000 and 7.7 against 4.0 for 1 x 2731 x 1001.  1 x 4096 x 4096 bf16
// takes 8.2 us with weights from HBM, whose floor is 5.1 (4.9 with the weights in the L2 cache, hot),
// 1 x 16384 x 4096 25.7 us (21).
constexpr int kFewThreads = 512;

// 8 values at p, of which the first `count` exist; VEC: 16-byte aligned, count 8 or 0
template <bool VEC, typename T>
__device__ __forceinline__ uint4 load_8(const T* p, int count)
{
    if constexpr (VEC) return count > 0 ? *(const uint4*)p : make_uint4(0, 0, 0, 0);
    return load_shifted_8(p, count);
}

template <typename T>
__device__ __forceinline__ void few_product(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    if constexpr (std::is_same_v<T, __nv_bfloat16>)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <typename T, int NT, int R, bool VEC, bool SHARED>
__global__ void __launch_bounds__(kFewThreads, NT <= 2 ? 2 : 1) k_linear_few(const T* x, uint64_t x_stride, const T* w, uint64_t w_stride, uint32_t k,
                                                           LinearEpilogue p)
{
    constexpr int kWarps = kFewThreads / 32, kAhead = NT == 1 && R == 1 && VEC ? 2 : 1;
    dependency_wait();
    dependency_release();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
    const uint64_t n0 = (uint64_t)blockIdx.x * (16 * R);
    const T* row[2 * R];                                   // past the end: any row, its sums are dropped
#pragma unroll
    for (int i = 0; i < 2 * R; ++i) row[i] = w + min(n0 + g + 8 * i, p.cols - 1) * w_stride;
    float c[R][NT][4];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < NT; ++i) c[r][i][0] = c[r][i][1] = c[r][i][2] = c[r][i][3] = 0.f;

    uint32_t blocks = 1, part = 0, first_step = 0;                          // of the cluster: 2, 4 or 8
    if constexpr (SHARED) {
        blocks = gridDim.y;
        part = blockIdx.y;
        const uint32_t steps = (k + 63) / 64, shift = 31 - __clz(blocks);
        first_step = steps * part >> shift;
        k = min(k, (steps * (part + 1) >> shift) * 64);
    }
    for (uint32_t k0 = (first_step + warp) * 64; k0 < k; k0 += kWarps * 64 * kAhead) {
        uint4 a[kAhead][2][2 * R], b[kAhead][NT][2];
#pragma unroll
        for (int s = 0; s < kAhead; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t at = k0 + s * kWarps * 64 + h * 32 + t * 8;
                const int count = at < k ? (int)min(k - at, 8u) : 0;
#pragma unroll
                for (int i = 0; i < 2 * R; ++i) a[s][h][i] = load_8<VEC>(row[i] + at, count);
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                    const uint32_t token = i * 8 + g;
                    b[s][i][h] = token < p.rows ? load_8<VEC>(x + token * x_stride + at, count) : make_uint4(0, 0, 0, 0);
                }
            }
#pragma unroll
        for (int s = 0; s < kAhead; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int i = 0; i < NT; ++i) {
                        const uint4 u = a[s][h][2 * r], v = a[s][h][2 * r + 1], z = b[s][i][h];
                        few_product<T>(c[r][i], u.x, v.x, u.y, v.y, z.x, z.y);
                        few_product<T>(c[r][i], u.z, v.z, u.w, v.w, z.z, z.w);
                    }
    }
    // eight tokens at a time, [warp][token][row of W]; warp 0's place then takes the block's sums
    __shared__ float sums[kWarps][8][16 * R + 1];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        if (8 * i >= p.rows) break;                        // alike in all blocks of a cluster
        if (i > 0) __syncthreads();
#pragma unroll
        for (int r = 0; r < R; ++r) {
            sums[warp][2 * t][16 * r + g] = c[r][i][0];
            sums[warp][2 * t + 1][16 * r + g] = c[r][i][1];
            sums[warp][2 * t][16 * r + g + 8] = c[r][i][2];
            sums[warp][2 * t + 1][16 * r + g + 8] = c[r][i][3];
        }
        __syncthreads();
        const bool mine = threadIdx.x < 128 * R;
        const uint32_t in_tile = threadIdx.x / (16 * R), in = threadIdx.x % (16 * R), token = 8 * i + in_tile;
        float v = 0.f;
        if (mine) {
#pragma unroll
            for (int j = 0; j < kWarps; ++j) v += sums[j][in_tile][in];
        }
        if constexpr (SHARED) {
            if (mine) sums[0][in_tile][in] = v;            // its own reader's value: no other thread's
            cluster_arrive_wait();
            if (mine && part == 0 && token < p.rows) {     // what is fetched is stored, and so waited for
                for (uint32_t j = 1; j < blocks; ++j) v += cluster_load(address_in(shared_address(&sums[0][in_tile][in]), j));
            }
        }
        if (mine && part == 0) {
            const uint64_t col = n0 + in;
            const bool live = token < p.rows && col < p.cols;
            if (p.bias && live) v += to_float(((const T*)p.bias)[col]);
            auto save = [&]() {                            // R = 2: the warp holds a token's group
                const uint32_t e = group_exponent(__reduce_max_sync(0xFFFFFFFFu, live ? magnitude_bits(v) : 0u));
                if (!live) return;
                p.ckpt.codes[token * p.ckpt.codes_stride + col] = (int8_t)group_code(v, group_inverse(e));
                if (in == 0) p.ckpt.exps[token * p.ckpt.exps_stride + n0 / kGroup] = (uint8_t)e;
            };
            if (R == 2 && p.save == EDEN_SAVE_PRE) save();
            with_act(p.act, [&](auto act) { v = act_value<decltype(act)::value>(v); });
            if (p.residual && live) v += to_float(((const T*)p.residual)[token * p.residual_stride + col]);
            const T y = from_float<T>(v);
            if (R == 2 && p.save == EDEN_SAVE_OUT) {
                v = to_float(y);
                save();
            }
            if (live) ((T*)p.out)[token * p.out_stride + col] = y;
        }
        // the sums were used (also where nothing was stored) before their blocks go on
        if constexpr (SHARED) cluster_arrive_wait();
    }
}

// ---- operands -----------------------------------------------------------------------
// What the tile kernel's tensor copies cannot read is laid out anew, both operands in one launch:
// rows that do not start on 16 bytes are copied to such rows, checkpoints are restored to them.
struct Layout {
    const void* from;                  // 16-bit values, or null: a checkpoint
    CheckpointView held;
    uint64_t from_stride;
    uint16_t* to;                      // rows of `stride` values, a multiple of 16, on 32 bytes
    uint64_t stride, n, total;         // chunks of 16 values
    bool wide;                         // codes on 16-byte boundaries
};

template <typename T>
__global__ void __launch_bounds__(256) k_lay_out(Layout first, Layout second, uint32_t first_blocks)
{
    dependency_wait();
    dependency_release();
    const bool is_second = blockIdx.x >= first_blocks;
    const Layout& l = is_second ? second : first;
    const uint64_t chunk = (uint64_t)(blockIdx.x - (is_second ? first_blocks : 0)) * 256 + threadIdx.x;
    if (chunk >= l.total) return;
    const uint32_t per_row = (uint32_t)(l.stride / 16);
    const uint64_t row = l.total <= 0xFFFFFFFFull ? (uint32_t)chunk / per_row : chunk / per_row;
    const uint64_t col = (chunk - row * per_row) * 16;
    const int count = (int)min((uint64_t)16, l.n - col);
    uint32_t out[8];
    if (l.from) {
        load_shifted((const uint16_t*)l.from + row * l.from_stride + col, 2 * count, out);
    } else {
        const int8_t* codes = l.held.codes + row * l.held.codes_stride + col;
        const uint32_t e = l.held.exps[row * l.held.exps_stride + col / kGroup];
        uint32_t w[4];
        if (l.wide && count == 16) *(uint4*)w = *(const uint4*)codes;
        else load_shifted(codes, count, w);
        const Pair scale(group_scale(e));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            Pair p[2];
            code_values(w[j], scale, p[0], p[1]);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float x, y;
                p[i].get(x, y);
                if (e >= kSaturates<T>) {
                    x = saturated<T>(x);
                    y = saturated<T>(y);
                }
                out[2 * j + i] = pack<T>(x, y);
            }
        }
    }
    store_32b(l.to + row * l.stride + col, out);
}

}  // namespace eden
