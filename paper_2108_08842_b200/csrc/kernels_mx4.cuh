// Microscaled 4-bit floating point: quantising, restoring, and products on the tensor cores.
//   group   32 values along the sum, 2^e with e the smallest that holds max|v| <= 6 * 2^e, and sign
//           and magnitude (0, 0.5, 1, 1.5, 2, 3, 4, 6) of each v / 2^e, rounded to nearest even
//   product D = A B^T, both operands with their groups along the sum: the tensor cores multiply the
//           values exactly, scale them by both powers of two and add up in fp32
#pragma once

#include "kernels_linear.cuh"

namespace eden {

// Codes: 16 bytes for each group of a row, two values a byte, the low half first; values past the
// row's end are 0.  Exponent bytes (e + 127): tiles of 128 rows x 256 values, 1024 bytes, in the
// order in which the tensor cores want them beside a tile of codes.
constexpr uint32_t kMx4TileRows = 128, kMx4TileDepth = 256, kMx4TileBytes = 1024;

struct Mx4View {
    uint8_t* codes;                    // or null: this form is not wanted
    uint64_t stride;                   // bytes, a multiple of 16
    uint8_t* exps;
    uint64_t tiles;                    // of exponents along the sum
};

__host__ __device__ __forceinline__ uint64_t mx4_exponent_at(uint64_t tiles, uint64_t row, uint64_t group)
{
    return (row / 128 * tiles + group / 8) * kMx4TileBytes + group / 4 % 2 * 512 + row % 32 * 16 + row / 32 % 4 * 4 + group % 4;
}

// Exponent byte of a group from its largest magnitude's bits: max = 1.f * 2^E, and 6 * 2^(E - 2) is
// 1.5 * 2^E, so e = E - 2, or E - 1 where the fraction is above 0x400000.
__device__ __forceinline__ uint32_t mx4_exponent(uint32_t max_bits)
{
    if (max_bits >= 0x7F800000u) return 255u;
    const int e = (int)((max_bits + 0x3FFFFFu) >> 23) - 2;
    return (uint32_t)(e < 1 ? 1 : e);
}

// 8 values times `inverse`, as codes
__device__ __forceinline__ uint32_t mx4_codes(const float* v, float inverse)
{
    float s[8];
#pragma unroll
    for (int j = 0; j < 8; j += 2) (Pair(v[j], v[j + 1]) * Pair(inverse)).get(s[j], s[j + 1]);
    uint32_t w;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(w) : "f"(s[0]), "f"(s[1]), "f"(s[2]), "f"(s[3]), "f"(s[4]), "f"(s[5]), "f"(s[6]), "f"(s[7]));
    return inverse == 0.f ? 0u : w;
}

// fp16 values of eight codes, exact: h[j] holds 2 j and 2 j + 1
__device__ __forceinline__ void mx4_halves(uint32_t w, uint32_t (&h)[4])
{
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "mov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
}

// The largest magnitudes of 16-bit values, two a word, of the low and the high halves: as whole numbers
// without their signs, which NaN tops.
__device__ __forceinline__ uint32_t halves_max(uint32_t most, uint32_t a, uint32_t b) { return __vimax3_u16x2(most, a & 0x7FFF7FFFu, b & 0x7FFF7FFFu); }

template <typename T>
__device__ __forceinline__ uint32_t half_magnitude_bits(uint32_t half)
{
    float lo, hi;
    unpack<T>(half & 0xFFFFu, lo, hi);
    return __float_as_uint(lo);
}

// 32 values as 16 bytes of codes; value(j) is value j
template <typename F>
__device__ __forceinline__ uint4 mx4_group(float inverse, F&& value)
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = value(8 * i + j);
        w[i] = mx4_codes(v, inverse);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// 32 values at p, of which `count` exist, zeros after them; WIDE: on 32 bytes
template <bool WIDE, typename T>
__device__ __forceinline__ void load_group(const T* p, int count, uint32_t (&w)[8 * sizeof(T)])
{
    if (WIDE && count == 32) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T); ++i) load_32b((const char*)p + 32 * i, *(uint32_t(*)[8])(w + 8 * i));
    } else if (count == 32 && ((uintptr_t)p & 15) == 0) {
#pragma unroll
        for (int i = 0; i < 2 * (int)sizeof(T); ++i) *(uint4*)(w + 4 * i) = ((const uint4*)p)[i];
    } else {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T); ++i) load_shifted((const char*)p + 32 * i, min(max(count * (int)sizeof(T) - 32 * i, 0), 32), *(uint32_t(*)[8])(w + 8 * i));
    }
}

// x [m][n] -> its rows' form and its columns' form (of x^T), from one read.  A block takes 128 x 128
// values: a thread quantises two groups of the rows straight from its registers; for the columns the
// block passes the values through shared memory, in chunks of 16 bytes whose places are exchanged so
// that neither the rows' side, eight lanes of which hold two rows' groups, nor the columns', a warp of
// which takes a row's words side by side, meets in a bank (rows of an odd number of words, stored word
// by word, took 53 us for 8192 x 8192 bf16 both ways, the shared memory 80 % busy).
constexpr int kMx4Threads = 256;
template <typename T, bool COLUMNS> constexpr uint32_t kMx4Shared = COLUMNS ? 128 * 128 * sizeof(T) + 128 * 64 : 0;

// place of chunk c of a row of the tile
template <typename T>
__device__ __forceinline__ uint32_t mx4_chunk(uint32_t row, uint32_t c)
{
    constexpr uint32_t kChunks = 8 * sizeof(T);
    return row * kChunks + (sizeof(T) == 2 ? c ^ (c >> 3 & 1) ^ (row & 1) << 1 : c ^ (c >> 3 & 3) ^ (row & 1) << 2);
}

// place of group g of column c of the result
__device__ __forceinline__ uint32_t mx4_result(uint32_t c, uint32_t g) { return (c * 4 + g) ^ (c >> 1 & 3) ^ (c >> 3 & 1) << 2; }

template <typename T, bool WIDE, bool COLUMNS>
__global__ void __launch_bounds__(kMx4Threads, sizeof(T) == 2 ? 4 : 2) k_mx4_quantize(const T* x, uint64_t x_stride, Mx4View rows, Mx4View columns, uint32_t m, uint32_t n,
                                                             uint32_t blocks_x)
{
    __shared__ __align__(16) uint8_t exps[2][512];
    extern __shared__ __align__(16) uint32_t tile[];
    dependency_wait();
    dependency_release();
    const uint32_t block_y = blockIdx.x / blocks_x, block_x = blockIdx.x - block_y * blocks_x, row0 = block_y * 128, col0 = block_x * 128;
    const uint32_t g = threadIdx.x % 4, col = col0 + 32 * g;
    auto count_of = [&](uint32_t row) { return row < m && col < n ? (int)min(n - col, 32u) : 0; };
    uint32_t raw[2][8 * sizeof(T)];                        // both groups on their way together
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t row = row0 + i * 64 + threadIdx.x / 4;
        load_group<WIDE>(x + (count_of(row) ? (uint64_t)row * x_stride + col : 0), count_of(row), raw[i]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t r = i * 64 + threadIdx.x / 4, row = row0 + r;
        if constexpr (COLUMNS) {
#pragma unroll
            for (int j = 0; j < 2 * (int)sizeof(T); ++j)
                ((uint4*)tile)[mx4_chunk<T>(r, g * 2 * sizeof(T) + j)] = make_uint4(raw[i][4 * j], raw[i][4 * j + 1], raw[i][4 * j + 2], raw[i][4 * j + 3]);
        }
        if (rows.codes) {
            uint32_t most = 0;
            if constexpr (sizeof(T) == 4) {
                float top = 0.f;
#pragma unroll
                for (int j = 0; j < 32; j += 2) top = max_magnitude(top, __uint_as_float(raw[i][j]), __uint_as_float(raw[i][j + 1]));
                most = magnitude_bits(top);
            } else {
#pragma unroll
                for (int j = 0; j < 16; j += 2) most = halves_max(most, raw[i][j], raw[i][j + 1]);
                most = half_magnitude_bits<T>(max(most & 0xFFFFu, most >> 16));
            }
            const uint32_t e = mx4_exponent(most);
            const float inverse = group_inverse(e);
            exps[0][r % 32 * 16 + r / 32 * 4 + g] = (uint8_t)e;
            if (count_of(row))
                *(uint4*)(rows.codes + (uint64_t)row * rows.stride + col / 2) = mx4_group(inverse, [&](int j) {
                    if constexpr (sizeof(T) == 4) return __uint_as_float(raw[i][j]);
                    float pair[2];
                    unpack<T>(raw[i][j / 2], pair[0], pair[1]);
                    return pair[j % 2];
                });
        }
    }
    __syncthreads();
    if constexpr (COLUMNS) {
        uint4* const out = (uint4*)tile + 128 * 8 * sizeof(T);
        constexpr int kTogether = 4 / sizeof(T);                               // columns in a word
#pragma unroll
        for (int i = 0; i < 2 / kTogether; ++i) {
            const uint32_t word = i * 64 + threadIdx.x % 64, g = threadIdx.x / 64;
            uint32_t raw[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) raw[j] = tile[mx4_chunk<T>(32 * g + j, word / 4) * 4 + word % 4];
            uint32_t most[2] = {0, 0};
            if constexpr (sizeof(T) == 4) {
                float top = 0.f;
#pragma unroll
                for (int j = 0; j < 32; j += 2) top = max_magnitude(top, __uint_as_float(raw[j]), __uint_as_float(raw[j + 1]));
                most[0] = magnitude_bits(top);
            } else {
                uint32_t both = 0;
#pragma unroll
                for (int j = 0; j < 32; j += 2) both = halves_max(both, raw[j], raw[j + 1]);
                most[0] = half_magnitude_bits<T>(both & 0xFFFFu);
                most[1] = half_magnitude_bits<T>(both >> 16);
            }
#pragma unroll
            for (int h = 0; h < kTogether; ++h) {
                const uint32_t c = word * kTogether + h, e = mx4_exponent(most[h]);
                exps[1][c % 32 * 16 + c / 32 * 4 + g] = (uint8_t)e;
                out[mx4_result(c, g)] = mx4_group(group_inverse(e), [&](int j) {
                    if constexpr (sizeof(T) == 4) return __uint_as_float(raw[j]);
                    float pair[2];
                    unpack<T>(raw[j], pair[0], pair[1]);
                    return pair[h];
                });
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t c = i * 64 + threadIdx.x / 4, g = threadIdx.x % 4;
            if (col0 + c < n && row0 + 32 * g < m)
                *(uint4*)(columns.codes + (uint64_t)(col0 + c) * columns.stride + row0 / 2 + 16 * g) = out[mx4_result(c, g)];
        }
    }
    if (threadIdx.x < 64) {
        const bool second = threadIdx.x >= 32;
        const Mx4View& form = second ? columns : rows;
        const uint32_t along = second ? block_y : block_x, across = second ? block_x : block_y, i = threadIdx.x % 32;
        if (form.codes && across * 128 < (second ? n : m))
            *(uint4*)(form.exps + (across * form.tiles + along / 2) * kMx4TileBytes + along % 2 * 512 + i * 16) = *(const uint4*)&exps[second][i * 16];
    }
}

// groups whose exponent byte is below this cannot pass the largest number: 6 * 2^e
template <typename T> constexpr uint32_t kMx4Saturates = std::is_same_v<T, __half> ? 127 + 14 : 127 + 126;

// codes -> x [m][n]; four lanes to 128 values of a row.  Without WIDE a warp hands its 8 x 128 values
// round in shared memory and stores each row's side by side.
template <typename T, bool WIDE>
__global__ void __launch_bounds__(kMx4Threads) k_mx4_restore(T* x, uint64_t x_stride, Mx4View q, uint32_t m, uint32_t n, uint32_t blocks_x)
{
    __shared__ T values[WIDE ? 1 : kMx4Threads / 32][8][128 + 8 / sizeof(T)];
    dependency_wait();
    dependency_release();
    const uint32_t block_y = blockIdx.x / blocks_x, col0 = (blockIdx.x - block_y * blocks_x) * 128, group = col0 / 32 + threadIdx.x % 4;
    const uint32_t row = block_y * 64 + threadIdx.x / 4, col = group * 32;
    const int count = row < m && col < n ? (int)min(n - col, 32u) : 0, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    if (count > 0) {
        const uint4 w = *(const uint4*)(q.codes + (uint64_t)row * q.stride + group * 16);
        const uint32_t e = q.exps[mx4_exponent_at(q.tiles, row, group)], words[4] = {w.x, w.y, w.z, w.w};
        const float scale = group_scale(e);
        T* const to = x + (uint64_t)row * x_stride + col;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float v[16];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                uint32_t halves[4];
                mx4_halves(words[2 * h + i], halves);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float lo, hi;
                    unpack<__half>(halves[j], lo, hi);
                    (Pair(lo, hi) * Pair(scale)).get(v[8 * i + 2 * j], v[8 * i + 2 * j + 1]);
                }
            }
            if (e >= kMx4Saturates<T>) {
#pragma unroll
                for (int j = 0; j < 16; ++j) v[j] = saturated<T>(v[j]);
            }
            if constexpr (WIDE) {
                if (count >= 16 * h + 1) store_values(to + 16 * h, min(count - 16 * h, 16), v);
            } else {
#pragma unroll
                for (int j = 0; j < 16; ++j) values[warp][lane / 4][32 * (lane % 4) + 16 * h + j] = from_float<T>(v[j]);
            }
        }
    }
    if constexpr (!WIDE) {
        __syncwarp();
        const uint32_t row0 = block_y * 64 + warp * 8;
#pragma unroll
        for (int r = 0; r < 8; ++r)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (row0 + r < m && col0 + 32 * j + lane < n) x[(uint64_t)(row0 + r) * x_stride + col0 + 32 * j + lane] = values[warp][r][32 * j + lane];
    }
}

// ---- products -----------------------------------------------------------------------
// kind::mxf4, 64 values a step of the sum: both operands are packed codes along the sum, and each row
// has two exponent bytes a step, the first or the last two (`half`) of a word in tensor memory.
__host__ __device__ constexpr uint32_t mx4_descriptor(int m, int n, int half)
{
    return (uint32_t)half << 5 | 1u << 7 | 1u << 10 | (uint32_t)(n / 8) << 17 | 1u << 23 | (uint32_t)(m / 16) << 24 | (uint32_t)half << 30;
}

template <int CG>
__device__ __forceinline__ void mx4_product(uint32_t d, uint64_t a, uint64_t b, uint32_t descriptor, uint32_t scale_a, uint32_t scale_b, bool add)
{
    if constexpr (CG == 2)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%5], [%6], p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(descriptor), "r"((uint32_t)add), "r"(scale_a), "r"(scale_b) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%5], [%6], p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(descriptor), "r"((uint32_t)add), "r"(scale_a), "r"(scale_b) : "memory");
}

// 32 x 16 bytes, in order, from shared memory to four columns of tensor memory, alike in each quarter
// of its lanes.  Descriptor: no swizzle, groups of 8 x 16 bytes every 128 bytes.  Copies and products
// that one thread issues run in their order.
template <int CG>
__device__ __forceinline__ void copy_scales(uint32_t to, uint32_t from)
{
    const uint64_t descriptor = (uint64_t)(128 >> 4 | 1u << 14) << 32 | (from >> 4 & 0x3FFFu);
    if constexpr (CG == 2) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(to), "l"(descriptor) : "memory");
    else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(to), "l"(descriptor) : "memory");
}

// A step along the sum: 256 values, 128 bytes, of 128 rows of A and BN / CG rows of B, and the
// exponents of 128 rows of A and of all rows of B, which both blocks of a pair hold.
template <int CG, int BN, int SIDES>
struct Mx4Shape {
    static constexpr int kRowsB = BN / CG, kTilesB = (BN + 127) / 128;
    static constexpr uint32_t kBytesA = 128 * 128, kBytesB = kRowsB * 128;
    static constexpr uint32_t kScaleA = kBytesA + kBytesB, kScaleB = kScaleA + kMx4TileBytes, kStageBytes = kScaleB + kTilesB * kMx4TileBytes;
    static constexpr int kPieces = BN / SIDES / 32, kWarps = 4 * SIDES, kThreads = 128 + 32 * kWarps;
    static constexpr uint32_t kAfter = kWarps * kStageWords * 4 + 256;
    static constexpr int kStages = (int)((227 * 1024 - kAfter) / kStageBytes) > 8 ? 8 : (int)((227 * 1024 - kAfter) / kStageBytes);
    static constexpr uint32_t kBuffers = kStages * kStageBytes, kBarriers = kBuffers + kWarps * kStageWords * 4;
    static constexpr uint32_t kSharedBytes = kBarriers + (2 * kStages + 5) * 8 + 16;
    // Tensor memory: two tiles' sums and a step's exponents.  Two tiles of 256 columns would leave no
    // place for those, so the second one begins in the last 32 columns of the first: a tile's epilogue
    // takes the columns that the next tile shares first, and gives them free.
    static constexpr bool kShared = BN == 256;
    static constexpr uint32_t kSecond = kShared ? 224 : BN, kSums = kSecond + BN, kScalesA = kSums, kScalesB = kSums + 8;
    static constexpr uint32_t kColumns = BN == 64 ? 256 : 512;
    static_assert(kScalesB + 8 * kTilesB <= kColumns, "tensor memory");
    static_assert(kStageBytes % 1024 == 0 && kSharedBytes <= 227 * 1024 && kStages >= 3, "a block's shared memory");
};

struct Mx4Exponents {
    uint32_t tiles_a, tiles_b;         // along the sum
};

// As k_linear: warp 0 fills the stages, warp 1 of a pair's first block copies exponents and issues
// products, warp 2 owns the tensor memory, the others finish tiles.  RUNS: sums of `run` steps each
// are added up in registers, rounded to nearest.
template <int OP, typename T, int CG, int BN, bool RUNS, int SIDES>
__global__ void __launch_bounds__(Mx4Shape<CG, BN, SIDES>::kThreads, 1)
k_mx4_linear(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_exp_a,
             const __grid_constant__ CUtensorMap map_exp_b, LinearEpilogue p, TileGrid grid, Mx4Exponents tiles, uint32_t* status)
{
    using S = Mx4Shape<CG, BN, SIDES>;
    constexpr uint32_t kRun = RUNS ? 8 : 1u << 30;         // steps summed in tensor memory
    extern __shared__ __align__(1024) char raw[];
    const uint32_t base = shared_address(raw);
    const uint32_t full = base + S::kBarriers, empty = full + 8 * S::kStages;
    const uint32_t sums_full = empty + 8 * S::kStages, sums_empty = sums_full + 16, drained = sums_empty + 16, slot = drained + 8;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    uint32_t* const buffer = (uint32_t*)(raw + S::kBuffers) + (warp >= 4 ? warp - 4 : 0) * kStageWords;
    const uint32_t rank = CG == 2 ? cluster_rank() : 0;
    const uint32_t first = grid.begin + blockIdx.x / CG, step = gridDim.x / CG;

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
        prefetch_map(&map_exp_a);
        prefetch_map(&map_exp_b);
    }
    if (warp == 2) tmem_alloc<CG>(slot, S::kColumns);
    tmem_fence_before();
    if constexpr (CG == 2) cluster_arrive_wait(); else __syncthreads();
    tmem_fence_after();
    dependency_wait();
    dependency_release();
    uint32_t sums;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(sums) : "r"(slot));

    bool ok = true;
    if (warp < 4) {
        registers_down<SIDES>();
        if (warp == 0) {
            uint32_t s = 0, phase = 0, issued = 0;
            for (uint32_t t = first; t < grid.end && ok; t += step) {
                uint32_t tile_row, tile_col;
                tile_at(grid, t, tile_row, tile_col);
                const int row = (int)(tile_row * 128 * CG + rank * 128), col = (int)(tile_col * BN);
                const int exp_a = (int)(tile_row * CG + rank), exp_b = col / 128;
                for (uint32_t d = 0; d < grid.depth_steps; ++d) {
                    if (!(ok = barrier_wait(empty + 8 * s, phase ^ 1))) break;
                    if (elected()) {
                        const uint32_t bar = CG == 2 ? address_in(full + 8 * s, 0) : full + 8 * s;
                        if (rank == 0) barrier_expect(full + 8 * s, CG * S::kStageBytes);
                        const uint32_t to = base + s * S::kStageBytes;
                        copy_box<CG>(to, &map_a, (int)d * 128, row, bar);
                        copy_box<CG>(to + S::kBytesA, &map_b, (int)d * 128, col + (int)(rank * S::kRowsB), bar);
                        copy_box<CG>(to + S::kScaleA, &map_exp_a, 0, exp_a * (int)tiles.tiles_a + (int)d, bar);
#pragma unroll
                        for (int i = 0; i < S::kTilesB; ++i)
                            copy_box<CG>(to + S::kScaleB + i * kMx4TileBytes, &map_exp_b, 0, (exp_b + i) * (int)tiles.tiles_b + (int)d, bar);
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
            // gave up: the copies still on their way (counted by the pair's first block) land as well
            if (!ok && rank == 0)
                for (; issued > 0; --issued) {
                    if (s-- == 0) { s = S::kStages - 1; phase ^= 1; }
                    barrier_wait(full + 8 * s, phase);
                }
        } else if (warp == 1) {
            if (rank == 0) {
                uint32_t s = 0, phase = 0, half = 0, done = 0;
                const uint32_t low_a = descriptor_low(base), low_b = descriptor_low(base + S::kBytesA);
                for (uint32_t t = first; t < grid.end && ok; t += step) {
                    // a tile of 64 columns starts in the middle of every other tile of exponents
                    uint32_t tile_row, tile_col;
                    tile_at(grid, t, tile_row, tile_col);
                    const uint32_t scale_b = sums + S::kScalesB + (BN == 64 ? tile_col % 2 * 2 : 0);
                    for (uint32_t begin = 0; begin < grid.depth_steps && ok; begin += kRun) {
                        const uint32_t d_address = sums + half * S::kSecond, end = grid.depth_steps - begin < kRun ? grid.depth_steps : begin + kRun;
                        // The sums before the last ones are read; where these share columns with the last
                        // ones, so are those: the release of sums number `done - kBehind`.
                        constexpr uint32_t kBehind = S::kShared ? 1 : 2;
                        if (done >= kBehind && !(ok = barrier_wait(sums_empty + 8 * ((done - kBehind) & 1), (done - kBehind) >> 1 & 1))) break;
                        ++done;
                        tmem_fence_after();
                        for (uint32_t d = begin; d < end; ++d) {
                            if (!(ok = barrier_wait(full + 8 * s, phase))) break;
                            tmem_fence_after();
                            if (elected()) {
                                const uint32_t from = base + s * S::kStageBytes, at = s * (S::kStageBytes / 16);
#pragma unroll
                                for (int k = 0; k < 2; ++k) {
                                    copy_scales<CG>(sums + S::kScalesA + 4 * k, from + S::kScaleA + 512 * k);
#pragma unroll
                                    for (int i = 0; i < S::kTilesB; ++i)
                                        copy_scales<CG>(sums + S::kScalesB + 4 * S::kTilesB * k + 4 * i, from + S::kScaleB + i * kMx4TileBytes + 512 * k);
                                }
#pragma unroll
                                for (int k = 0; k < 4; ++k)
                                    mx4_product<CG>(d_address, tile_descriptor(low_a + at + 2 * k), tile_descriptor(low_b + at + 2 * k),
                                                    mx4_descriptor(128 * CG, BN, k % 2), sums + S::kScalesA + 4 * (k / 2),
                                                    scale_b + 4 * S::kTilesB * (k / 2), k > 0 || d > begin);
                                tile_commit<CG>(empty + 8 * s, 0);
                                if (d + 1 == end) tile_commit<CG>(sums_full + 8 * half, 0);
                            }
                            __syncwarp();
                            if (++s == S::kStages) { s = 0; phase ^= 1; }
                        }
                        half ^= 1;
                    }
                }
                if (!ok) {
                    if (elected()) tile_commit<CG>(drained, 0);
                    __syncwarp();
                    barrier_wait(drained, 0);
                }
            }
        }
    } else {
        registers_up<SIDES>();
        const int quarter = warp % 4, side = (warp - 4) / 4;
        const uint32_t my_sums = sums + ((uint32_t)quarter * 32 << 16) + side * S::kPieces * 32;
        uint32_t half = 0, phase = 0;
        // Once for each finished part.  With shared columns: what came before it is read (this warp is
        // behind it), and so are the columns that the next one shares with it, which the side that
        // holds them takes first.  Else when it is read.
        auto release = [&]() {
            tmem_fence_before();
            __syncwarp();
            if (lane == 0) barrier_arrive_remote(CG == 2 ? address_in(sums_empty + 8 * half, 0) : sums_empty + 8 * half);
        };
        for (uint32_t t = first; t < grid.end && ok; t += step) {
            uint32_t tile_row, tile_col;
            tile_at(grid, t, tile_row, tile_col);
            const uint64_t row0 = (uint64_t)tile_row * 128 * CG + rank * 128 + quarter * 32;
            const uint64_t tile_col0 = (uint64_t)tile_col * BN + side * S::kPieces * 32;
            if (RUNS && SIDES == 2 && grid.depth_steps > kRun) {
                // the runs added up, and the total put back in the last one's place
                float total[S::kPieces][32];
                for (uint32_t begin = 0;; begin += kRun) {
                    if (!(ok = barrier_wait(sums_full + 8 * half, phase))) break;
                    tmem_fence_after();
                    const bool last = grid.depth_steps - begin <= kRun;
#pragma unroll
                    for (int c = 0; c < S::kPieces; ++c) {
                        float v[32];
                        tmem_load(my_sums + half * S::kSecond + 32 * c, v);
#pragma unroll
                        for (int j = 0; j < 32; j += 2) {
                            const Pair sum = begin == 0 ? Pair(v[j], v[j + 1]) : Pair(total[c][j], total[c][j + 1]) + Pair(v[j], v[j + 1]);
                            sum.get(total[c][j], total[c][j + 1]);
                        }
                        if (last) tmem_store(my_sums + half * S::kSecond + 32 * c, total[c]);
                    }
                    if (last) break;
                    release();
                    half ^= 1;
                    phase ^= half ^ 1;
                }
            } else {
                ok = barrier_wait(sums_full + 8 * half, phase);
            }
            if (!ok) break;
            tmem_fence_after();
            const bool descending = half == 0;                  // the shared columns are the first tile's last, the second's first
            const int shared_side = descending ? SIDES - 1 : 0;
            if (S::kShared && side != shared_side) release();
            auto column_of = [&](int i) { return tile_col0 + 32 * (descending ? S::kPieces - 1 - i : i); };
            // a piece without rows or columns of the result has nothing to fetch or finish
            auto exists = [&](int i) { return i < S::kPieces && row0 < p.rows && column_of(i) < p.cols; };
            uint32_t exp = 0;
            bool fetched = false;
#pragma unroll 1
            for (int i = 0; i < S::kPieces; ++i) {
                float v[32];
                __syncwarp();
                tmem_load(my_sums + half * S::kSecond + (descending ? S::kPieces - 1 - i : i) * 32, v);
                if (S::kShared ? i == 0 && side == shared_side : i == S::kPieces - 1) release();
                if (!exists(i)) continue;
                const Piece at(p, row0, column_of(i));
                if (OP == kInputGrad && !fetched) fetch_codes(at, p, buffer, exp);
                fetched = exists(i + 1);
                const Piece next(p, row0, fetched ? column_of(i + 1) : column_of(i));
                linear_epilogue<OP, T>(v, at, p, buffer, exp, fetched ? &next : nullptr);
            }
            half ^= 1;
            phase ^= half ^ 1;
        }
    }
    if (!ok) {
        copy_async_wait();
        atomicOr(status, EDEN_STATUS_TIMEOUT);
    }
    __syncwarp();
    tmem_fence_before();
    if constexpr (CG == 2) cluster_arrive_wait(); else __syncthreads();
    tmem_fence_after();
    if (warp == 2) tmem_free<CG>(sums, S::kColumns);
}

// ---- few tokens ---------------------------------------------------------------------
// y [m, n] for m <= 8: as k_linear_few, every weight is read once, straight to registers.  A lane
// reads 8 codes of a group (its row's group lies with the four lanes of the row); their values are fed
// as fp16 to two products of 16 x 8 x 16, in the same order of the sum's index for W and x.  The
// products of a group are exact and added up in fp32 by themselves, then times both powers of two.
//   FROM_MATRIX   x is a matrix of 16-bit values, which the block quantises into its shared memory
//                 first, while its weights are on their way; else x is in 4 bits.
// Instructions bound it: values by shifts and masks of fp16 numbers with an exponent 14 too low, with
// the powers of two checked for 0 and NaN, took 9.1 us for 1 x 4096 x 4096.  16 tokens took 28 us, more than
// the tiles' 16.
// 2^e of byte `group`; infinity for 255, whose group's products are 0: their product is NaN
__device__ __forceinline__ float mx4_scale(uint32_t word, int group)
{
    return __uint_as_float((group < 3 ? word << (23 - 8 * group) : word >> 1) & 0x7F800000u);
}

struct Mx4Few {
    const void* x;         uint64_t x_stride;              // FROM_MATRIX
    Mx4View held;                                          // else
    Mx4View weight;
    uint32_t k;
};

// a row of x's codes in shared memory is 16 bytes longer than it is: eight rows meet all banks once
__host__ __device__ __forceinline__ uint32_t mx4_few_pitch(uint32_t k) { return (k + 127) / 128 * 64 + 16; }
__host__ __device__ __forceinline__ uint32_t mx4_few_shared(uint32_t m, uint32_t k) { return m * (mx4_few_pitch(k) + (k + 127) / 128 * 4); }

template <typename T, int R, bool FROM_MATRIX, bool SHARED>
__global__ void __launch_bounds__(kFewThreads, R == 1 ? 2 : 1) k_mx4_few(Mx4Few q, LinearEpilogue p)
{
    constexpr int kWarps = kFewThreads / 32;
    extern __shared__ __align__(16) uint8_t held[];
    dependency_wait();
    dependency_release();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
    const uint64_t n0 = (uint64_t)blockIdx.x * (16 * R);
    const uint32_t groups = (q.k + 31) / 32, steps = (q.k + 127) / 128, tokens = (uint32_t)p.rows;
    uint32_t blocks = 1, part = 0, first_step = 0, last_step = steps;       // of the cluster: 2, 4 or 8
    if constexpr (SHARED) {
        blocks = gridDim.y;
        part = blockIdx.y;
        const uint32_t shift = 31 - __clz(blocks);
        first_step = steps * part >> shift;
        last_step = steps * (part + 1) >> shift;
    }
    // A warp's steps are kWarps apart, an even number: the bytes from one to the next are the same for all.
    constexpr uint32_t kCodesOn = 64 * kWarps, kExpsOn = kMx4TileBytes * kWarps / 2;
    const uint32_t mine = first_step + warp;
    const uint8_t *codes[2 * R], *exps[2 * R];             // of the next step to fetch; past the end: any row, its sums are dropped
#pragma unroll
    for (int i = 0; i < 2 * R; ++i) {
        const uint64_t row = min(n0 + g + 8 * i, p.cols - 1);
        codes[i] = q.weight.codes + row * q.weight.stride + 64 * mine + 4 * t;
        exps[i] = q.weight.exps + mx4_exponent_at(q.weight.tiles, row, 4 * mine);
    }
    // four words of a row, of which the last step may have fewer
    auto load_words = [&](uint32_t (&to)[4], const uint8_t* from, uint32_t step) {
        if (4 * step + 4 <= groups) {
#pragma unroll
            for (int j = 0; j < 4; ++j) to[j] = *(const uint32_t*)(from + 16 * j);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) to[j] = 4 * step + j < groups ? *(const uint32_t*)(from + 16 * j) : 0u;
        }
    };
    constexpr int kAhead = 1;                              // steps of 128 on their way: with two, registers spill (8 us for 6.5)
    uint32_t w[kAhead][2 * R][4], we[kAhead][2 * R];
    auto fetch = [&](uint32_t step, int s) {
        if (step >= last_step) return;
#pragma unroll
        for (int i = 0; i < 2 * R; ++i) {
            load_words(w[s][i], codes[i], step);
            we[s][i] = *(const uint32_t*)exps[i];
            codes[i] += kCodesOn;
            exps[i] += kExpsOn;
        }
    };
#pragma unroll
    for (int s = 0; s < kAhead; ++s) fetch(mine + s * kWarps, s);
    // what the end reads comes nearer meanwhile
    if (threadIdx.x < tokens) {
        if (p.residual) asm volatile("prefetch.global.L2 [%0];" ::"l"((const T*)p.residual + threadIdx.x * p.residual_stride + n0));
        if (p.bias) asm volatile("prefetch.global.L2 [%0];" ::"l"((const T*)p.bias + n0));
    }
    const uint32_t pitch = mx4_few_pitch(q.k);
    if constexpr (FROM_MATRIX) {
        uint8_t* const held_exps = held + tokens * pitch;
        const uint32_t begin = first_step * 16, per_row = last_step * 16 - begin;        // units of 8 values, four to a group
        const uint32_t units = tokens * per_row;
        for (uint32_t u0 = threadIdx.x; u0 < (units + 31) / 32 * 32; u0 += 4 * kFewThreads) {
            uint4 raw[4];                                  // on their way together
            auto place = [&](int i, uint32_t& token, uint32_t& unit) {
                const uint32_t u = u0 + i * kFewThreads;
                token = u / per_row;
                unit = begin + u - token * per_row;
                return u < units;
            };
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (u0 - lane + i * kFewThreads >= units) break;                  // all lanes together
                uint32_t token, unit;
                const bool live = place(i, token, unit);
                const int count = live && unit * 8 < q.k ? (int)min(q.k - unit * 8, 8u) : 0;
                raw[i] = load_shifted_8((const T*)q.x + (count ? token * q.x_stride + unit * 8 : 0), count);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (u0 - lane + i * kFewThreads >= units) break;
                uint32_t token, unit;
                const bool live = place(i, token, unit);
                float v[8];
                unpack<T>(raw[i].x, v[0], v[1]);
                unpack<T>(raw[i].y, v[2], v[3]);
                unpack<T>(raw[i].z, v[4], v[5]);
                unpack<T>(raw[i].w, v[6], v[7]);
                float top = 0.f;
#pragma unroll
                for (int j = 0; j < 8; j += 2) top = max_magnitude(top, v[j], v[j + 1]);
                uint32_t most = magnitude_bits(top);
                most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
                most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 2));
                const uint32_t e = mx4_exponent(most);
                if (!live) continue;
                *(uint32_t*)(held + token * pitch + unit * 4) = mx4_codes(v, group_inverse(e));
                if (unit % 4 == 0) held_exps[token * (steps * 4) + unit / 4] = (uint8_t)e;
            }
        }
        __syncthreads();
    }
    float c[R][1][4];
#pragma unroll
    for (int r = 0; r < R; ++r) c[r][0][0] = c[r][0][1] = c[r][0][2] = c[r][0][3] = 0.f;
    // This lane's codes are token g's; its sums belong to tokens 2 t and 2 t + 1.  Tokens that do not
    // exist multiply another one's codes: their sums are dropped.
    const uint8_t *x_codes, *x_exps[2];
    if constexpr (FROM_MATRIX) {
        x_codes = held + min((uint32_t)g, tokens - 1) * pitch + 64 * mine + 4 * t;
#pragma unroll
        for (int s = 0; s < 2; ++s) x_exps[s] = held + tokens * pitch + min((uint32_t)(2 * t + s), tokens - 1) * (steps * 4) + 4 * mine;
    } else {
        x_codes = q.held.codes + min((uint32_t)g, tokens - 1) * q.held.stride + 64 * mine + 4 * t;
#pragma unroll
        for (int s = 0; s < 2; ++s) x_exps[s] = q.held.exps + mx4_exponent_at(q.held.tiles, min((uint32_t)(2 * t + s), tokens - 1), 4 * mine);
    }
    for (uint32_t step0 = mine; step0 < last_step; step0 += kWarps * kAhead) {
#pragma unroll
        for (int ahead = 0; ahead < kAhead; ++ahead) {
            const uint32_t step = step0 + ahead * kWarps;
            if (step >= last_step) break;
            uint32_t a[2 * R][4], ae[2 * R], b[4], be[2];
#pragma unroll
            for (int i = 0; i < 2 * R; ++i) {
#pragma unroll
                for (int j = 0; j < 4; ++j) a[i][j] = w[ahead][i][j];
                ae[i] = we[ahead][i];
            }
            fetch(step + kWarps * kAhead, ahead);
            if constexpr (FROM_MATRIX) {                   // zeros behind the last value
#pragma unroll
                for (int j = 0; j < 4; ++j) b[j] = *(const uint32_t*)(x_codes + 16 * j);
            } else {
                load_words(b, x_codes, step);
            }
            x_codes += kCodesOn;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                be[s] = *(const uint32_t*)x_exps[s];
                x_exps[s] += FROM_MATRIX ? 4 * kWarps : kExpsOn;
            }
            // d * sx is exact down to 2^-126; with one of x's powers from 2^65 on it could pass the range though the
            // result does not, and the smaller of the two powers comes first
            const bool large = ((be[0] & be[0] << 1 | be[1] & be[1] << 1) & 0x80808080u) != 0;
            // the products of two groups, then what they are scaled by
#pragma unroll
            for (int j0 = 0; j0 < 4; j0 += 2) {
                float d[2][R][4];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t z[4];
                    mx4_halves(b[j0 + h], z);
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        uint32_t u[4], v[4];
                        mx4_halves(a[2 * r][j0 + h], u);
                        mx4_halves(a[2 * r + 1][j0 + h], v);
                        d[h][r][0] = d[h][r][1] = d[h][r][2] = d[h][r][3] = 0.f;
                        few_product<__half>(d[h][r], u[0], v[0], u[1], v[1], z[0], z[1]);
                        few_product<__half>(d[h][r], u[2], v[2], u[3], v[3], z[2], z[3]);
                    }
                }
                auto add = [&](auto ordered) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float sx[2] = {mx4_scale(be[0], j0 + h), mx4_scale(be[1], j0 + h)};
#pragma unroll
                        for (int r = 0; r < R; ++r)
#pragma unroll
                            for (int s = 0; s < 4; s += 2) {
                                const float sw = mx4_scale(ae[2 * r + s / 2], j0 + h);
                                float(&sum)[4] = c[r][0];
                                const Pair first = decltype(ordered)::value ? Pair(fminf(sx[0], sw), fminf(sx[1], sw)) : Pair(sx[0], sx[1]);
                                const Pair second = decltype(ordered)::value ? Pair(fmaxf(sx[0], sw), fmaxf(sx[1], sw)) : Pair(sw);
                                fma(Pair(d[h][r][s], d[h][r][s + 1]) * first, second, Pair(sum[s], sum[s + 1])).get(sum[s], sum[s + 1]);
                            }
                    }
                };
                if (__builtin_expect(large, 0)) add(std::true_type());
                else add(std::false_type());
            }
        }
    }
    few_finish<T, 1, R, SHARED>(c, p, n0, blocks, part);
}

}  // namespace eden
