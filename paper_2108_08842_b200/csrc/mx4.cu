// C ABI of microscaled 4-bit floating point (declared in include/eden.h): argument checks,
// workspace carving and launches.
#include <algorithm>
#include <atomic>

#include "kernels_mx4.cuh"
#include "tensor_map.h"
#include "train_host.h"

using namespace eden;

namespace {

constexpr uint64_t kFewFused = 16384;           // values of x that every block of a product with few tokens quantises

uint64_t tiles_along(uint64_t features) { return (features + kMx4TileDepth - 1) / kMx4TileDepth; }
uint64_t tiles_across(uint64_t rows) { return (rows + kMx4TileRows - 1) / kMx4TileRows; }
uint64_t exponent_bytes(uint64_t rows, uint64_t features) { return tiles_across(rows) * tiles_along(features) * kMx4TileBytes; }
uint64_t code_bytes_of(uint64_t features) { return groups_of(features) * 16; }

bool mx4_ok(const eden_mx4& q, uint64_t features)
{
    return q.codes && q.exps && aligned(q.codes, 16) && aligned(q.exps, 16) && q.codes_stride % 16 == 0 && q.codes_stride >= code_bytes_of(features);
}

Mx4View mx4_view(const eden_mx4& q, uint64_t features) { return {q.codes, q.codes_stride, q.exps, tiles_along(features)}; }

template <typename T>
int quantize(eden_ctx* ctx, const void* x, uint64_t x_stride, const Mx4View& rows, const Mx4View& columns, uint64_t m, uint64_t n)
{
    // exponents of both halves of a tile are written, also where the second holds no values
    const uint64_t bx = rows.codes ? 2 * tiles_along(n) : tiles_across(n), by = columns.codes ? 2 * tiles_along(m) : tiles_across(m);
    if (bx * by > kMaxCount) return EDEN_ERR_TOO_LARGE;
    const bool wide = wide_rows(x, x_stride, sizeof(T));
    const double bytes = (double)m * n * sizeof(T) + (rows.codes ? 17.0 * m * groups_of(n) : 0.0) + (columns.codes ? 17.0 * n * groups_of(m) : 0.0);
    const auto kernel = columns.codes ? (wide ? k_mx4_quantize<T, true, true> : k_mx4_quantize<T, false, true>)
                                      : (wide ? k_mx4_quantize<T, true, false> : k_mx4_quantize<T, false, false>);
    const uint32_t shared = columns.codes ? kMx4Shared<T, true> : 0;
    if (shared > 48 * 1024) CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)shared));
    return launch(ctx, "t_mx4_quantize", bytes, kernel, dim3((uint32_t)(bx * by)), kMx4Threads, shared, 1, (const T*)x, x_stride, rows, columns, m, n, bx);
}

template <typename T>
int restore(eden_ctx* ctx, const Mx4View& q, void* x, uint64_t x_stride, uint64_t m, uint64_t n)
{
    const uint64_t bx = (n + 127) / 128, by = (m + 63) / 64;
    if (bx * by > kMaxCount) return EDEN_ERR_TOO_LARGE;
    return launch(ctx, "t_mx4_restore", (double)m * n * sizeof(T) + 17.0 * m * groups_of(n), wide_rows(x, x_stride, sizeof(T)) ? k_mx4_restore<T, true> : k_mx4_restore<T, false>,
                  dim3((uint32_t)(bx * by)), kMx4Threads, 0, 1, (T*)x, x_stride, q, m, n, bx);
}

// An operand of a product: `rows` rows of `features` values along the sum.
struct Mx4Operand {
    const uint8_t* codes;
    uint64_t stride;
    const uint8_t* exps;
    uint64_t rows, features;
};

// boxes of 128 bytes (256 values) x box_rows rows of codes, 128-byte swizzle, zeros outside
int map_of_codes(CUtensorMap* map, const Mx4Operand& o, uint32_t box_rows)
{
    const cuuint64_t dims[2] = {code_bytes_of(o.features), o.rows}, strides[1] = {o.stride};
    const cuuint32_t box[2] = {128, box_rows};
    return encode_tiles(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, o.codes, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}

// boxes of one tile of exponents
int map_of_exponents(CUtensorMap* map, const Mx4Operand& o)
{
    const cuuint64_t dims[2] = {kMx4TileBytes / 4, tiles_across(o.rows) * tiles_along(o.features)}, strides[1] = {kMx4TileBytes};
    const cuuint32_t box[2] = {kMx4TileBytes / 4, 1};
    return encode_tiles(map, CU_TENSOR_MAP_DATA_TYPE_INT32, o.exps, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_NONE);
}

struct Mx4Product {
    const char* name;
    int type;
    Mx4Operand a, b;                   // rows of the result, columns of it
    LinearEpilogue p;
    double bytes;
};

template <int OP, typename T, int CG, int BN, bool RUNS, int SIDES>
int launch_mx4(eden_ctx* ctx, const Mx4Product& q)
{
    using S = Mx4Shape<CG, BN, SIDES>;
    CUtensorMap map_a, map_b, map_exp_a, map_exp_b;
    if (int rc = map_of_codes(&map_a, q.a, 128)) return rc;
    if (int rc = map_of_codes(&map_b, q.b, S::kRowsB)) return rc;
    if (int rc = map_of_exponents(&map_exp_a, q.a)) return rc;
    if (int rc = map_of_exponents(&map_exp_b, q.b)) return rc;
    const uint64_t rows = (q.p.rows + 128 * CG - 1) / (128 * CG), cols = (q.p.cols + BN - 1) / BN, tiles = tiles_along(q.a.features);
    // a box past the last tile of exponents is named by its number too
    if (rows * cols * CG > kMaxCount || (tiles_across(q.a.rows) + 2) * tiles > kMaxCount || (tiles_across(q.b.rows) + 2) * tiles > kMaxCount) return EDEN_ERR_TOO_LARGE;
    const TileGrid grid{(uint32_t)rows, (uint32_t)cols, 0, (uint32_t)(rows * cols), (uint32_t)tiles, 1};
    const Mx4Exponents exps{(uint32_t)tiles, (uint32_t)tiles};
    const auto kernel = k_mx4_linear<OP, T, CG, BN, RUNS, SIDES>;
    static std::atomic<uint64_t> asked{0};       // devices on which this kernel may use its shared memory
    const uint64_t device = 1ull << (ctx->device & 63);
    if (!(asked.load(std::memory_order_relaxed) & device) || ctx->device > 63) {
        // a kernel compiled to fewer registers than its warps redistribute would wait for them for good
        cudaFuncAttributes attributes;
        CUDA_OK(cudaFuncGetAttributes(&attributes, kernel));
        if ((attributes.numRegs + 7) / 8 * 8 < kLaunchRegisters[SIDES == 4]) return EDEN_ERR_CUDA;
        CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSharedBytes));
        asked.fetch_or(device, std::memory_order_relaxed);
    }
    const uint32_t groups = std::min<uint32_t>(grid.end, ctx->sm_count / CG);
    return launch(ctx, q.name, q.bytes, kernel, dim3(groups * CG), S::kThreads, S::kSharedBytes, CG, map_a, map_b, map_exp_a, map_exp_b, q.p, grid, exps,
                  (uint32_t*)ctx->ws);
}

// The cheapest form by a model of its time in microseconds, fitted to sums of 256 to 4096 on 16 to 8192
// tiles: a launch's fixed part, and for each wave of tiles a step of 256 along the sum (and the gap
// between two tiles' products) or the epilogue, whichever is longer.  8192 x 8192 results over 4096: 96 us
// in pairs, 139 and 246 in the others; 128 x 4096 over 4096: 11.3, 9.1 and 7.8.
template <int OP>
int choose_form(const eden_ctx* ctx, const Mx4Product& q)
{
    const int form = ctx->linear_form;
    if (form == EDEN_LINEAR_PAIR || form == EDEN_LINEAR_SINGLE || form == EDEN_LINEAR_NARROW) return form;
    // epilogues: a store of 16 bits, an activation or a residual, a slope with its sums, a store of 32 bits
    const int kind = OP == kWeightGrad ? 3 : OP == kInputGrad && (q.p.act || q.p.column_sums) ? 2 : q.p.act || q.p.residual || q.p.save ? 1 : 0;
    static const struct { int form; uint64_t rows, cols, blocks; double fixed, gap, step, finish[4]; } forms[] = {
        {EDEN_LINEAR_PAIR, 256, 256, 2, 4.5, 1.7, 0.32, {3.2, 4.0, 8.6, 3.8}},
        {EDEN_LINEAR_SINGLE, 128, 128, 1, 3.8, 0.8, 0.26, {1.8, 2.9, 5.5, 1.7}},
        {EDEN_LINEAR_NARROW, 128, 64, 1, 3.1, 0.45, 0.246, {0.8, 1.4, 2.9, 0.9}}};
    const double steps = (double)tiles_along(q.a.features);
    int best = EDEN_LINEAR_PAIR;
    double least = 1e300;
    for (const auto& f : forms) {
        const uint64_t tiles = ((q.p.rows + f.rows - 1) / f.rows) * ((q.p.cols + f.cols - 1) / f.cols), slots = ctx->sm_count / f.blocks;
        const double waves = (double)((tiles + slots - 1) / slots);
        const double cost = f.fixed + f.finish[kind] - f.finish[0] + waves * std::max(f.gap + f.step * steps, f.finish[kind]);
        if (cost < least) least = cost, best = f.form;
    }
    return best;
}

template <int OP, typename T>
int product(eden_ctx* ctx, Mx4Product q)
{
    LinearEpilogue& p = q.p;
    p.grain_out = row_grain(p.out, p.out_stride, OP == kWeightGrad ? 4 : 2);
    p.grain_residual = row_grain(p.residual, p.residual_stride, 2);
    p.grain_codes = row_grain(p.ckpt.codes, p.ckpt.codes_stride, 1);
    p.grain_bias = row_grain(p.bias, 0, 2);
    // Weight gradients, of 32 bits, are added up in runs.  Column sums are not: sums of 4-bit products are
    // mostly exact in fp32 as they come (no error at all over 16384 normal or Laplace values), and the runs'
    // registers cost an epilogue half its warps: 8192 x 4096 over 4096 with gelu's slope 76 us, 128 in runs.
    constexpr bool runs = OP == kWeightGrad;
    switch (choose_form<OP>(ctx, q)) {
        case EDEN_LINEAR_SINGLE: return launch_mx4<OP, T, 1, 128, runs, 2>(ctx, q);
        case EDEN_LINEAR_NARROW: return launch_mx4<OP, T, 1, 64, runs, 2>(ctx, q);
        default: break;
    }
    // sixteen epilogue warps wherever it is more than a store
    if constexpr (!runs) {
        if (p.act || p.residual || p.save || p.column_sums) return launch_mx4<OP, T, 2, 256, false, 4>(ctx, q);
    }
    return launch_mx4<OP, T, 2, 256, runs, 2>(ctx, q);
}

// A block for each SM where there are fewer rows of W than that, as long as its warps have a step each.
uint32_t few_parts(const eden_ctx* ctx, uint64_t blocks, uint64_t steps)
{
    uint32_t parts = 1;
    while (parts < 8 && blocks * parts * 2 <= (uint64_t)ctx->sm_count && steps >= 16 * 2 * parts) parts *= 2;
    return parts;
}

template <typename T, int R>
int launch_few(eden_ctx* ctx, const Mx4Few& q, const LinearEpilogue& p, double bytes)
{
    const uint64_t blocks = (p.cols + 16 * R - 1) / (16 * R);
    const uint32_t parts = few_parts(ctx, blocks, (q.k + 127) / 128), shared = q.x ? mx4_few_shared((uint32_t)p.rows, q.k) : 0;
    const auto kernel = q.x ? (parts > 1 ? k_mx4_few<T, R, true, true> : k_mx4_few<T, R, true, false>)
                            : (parts > 1 ? k_mx4_few<T, R, false, true> : k_mx4_few<T, R, false, false>);
    return launch(ctx, "t_mx4_linear", bytes, kernel, dim3((uint32_t)blocks, parts), kFewThreads, shared, parts, q, p);
}

// A matrix of 16-bit values as an operand: quantised into the workspace.
int quantized(eden_ctx* ctx, Scratch& scratch, int type, const void* x, uint64_t x_stride, uint64_t m, uint64_t n, Mx4Operand* o)
{
    const uint64_t stride = code_bytes_of(n);
    uint8_t* const codes = scratch.take<uint8_t>(m * stride);
    uint8_t* const exps = scratch.take<uint8_t>(exponent_bytes(m, n));
    if (!codes || !exps) return EDEN_ERR_WORKSPACE;
    *o = {codes, stride, exps, m, n};
    EDEN_DISPATCH_HALF(type, return quantize<T_>(ctx, x, x_stride, Mx4View{codes, stride, exps, tiles_along(n)}, Mx4View{}, m, n));
}

Mx4Operand operand_of(const eden_mx4& q, uint64_t rows, uint64_t features) { return {q.codes, q.codes_stride, q.exps, rows, features}; }

}  // namespace

extern "C" uint64_t eden_mx4_code_bytes(uint64_t features) { return code_bytes_of(features); }
extern "C" uint64_t eden_mx4_exponent_bytes(uint64_t rows, uint64_t features) { return exponent_bytes(rows, features); }

extern "C" uint64_t eden_mx4_workspace_bytes(uint64_t m, uint64_t n, uint64_t k)
{
    // a matrix operand in 4 bits, and the partial column sums
    const uint64_t x = std::max(m * code_bytes_of(k) + exponent_bytes(m, k), m * code_bytes_of(n) + exponent_bytes(m, n));
    return std::max(least_workspace(), kStatusBytes + x + std::max<uint64_t>((m + 31) / 32, 1) * k * 4 + 4 * 256);
}

extern "C" int eden_mx4_quantize(eden_ctx* ctx, const eden_mx4_quantize_args* a)
{
    if (!ctx || !a || a->type < EDEN_TYPE_BF16 || a->type > EDEN_TYPE_FP32) return EDEN_ERR_INVALID_ARG;
    if (int rc = counts_ok(a->m, a->n, 1)) return rc;
    if (!a->rows.codes && !a->columns.codes) return EDEN_ERR_INVALID_ARG;
    if (a->m == 0) return EDEN_OK;
    if (!matrix_ok(a->x, a->x_stride, a->n, type_size(a->type)) || (a->rows.codes && !mx4_ok(a->rows, a->n)) || (a->columns.codes && !mx4_ok(a->columns, a->m)))
        return EDEN_ERR_INVALID_ARG;
    return guarded(ctx, [&]() -> int {
        EDEN_DISPATCH_TYPE(a->type, return quantize<T_>(ctx, a->x, a->x_stride, mx4_view(a->rows, a->n), mx4_view(a->columns, a->m), a->m, a->n));
    });
}

extern "C" int eden_mx4_restore(eden_ctx* ctx, const eden_mx4_restore_args* a)
{
    if (!ctx || !a || a->type < EDEN_TYPE_BF16 || a->type > EDEN_TYPE_FP32) return EDEN_ERR_INVALID_ARG;
    if (int rc = counts_ok(a->m, a->n, 1)) return rc;
    if (a->m == 0) return EDEN_OK;
    if (!matrix_ok(a->x, a->x_stride, a->n, type_size(a->type)) || !mx4_ok(a->q, a->n)) return EDEN_ERR_INVALID_ARG;
    return guarded(ctx, [&]() -> int {
        EDEN_DISPATCH_TYPE(a->type, return restore<T_>(ctx, mx4_view(a->q, a->n), a->x, a->x_stride, a->m, a->n));
    });
}

extern "C" int eden_mx4_linear(eden_ctx* ctx, const eden_mx4_linear_args* a)
{
    if (!ctx || !a) return EDEN_ERR_INVALID_ARG;
    if (int rc = counts_ok(a->m, a->n, a->k)) return rc;
    if (!half_type(a->type) || !known_act(a->act) || a->save < EDEN_SAVE_NONE || a->save > EDEN_SAVE_OUT) return EDEN_ERR_INVALID_ARG;
    if (!mx4_ok(a->weight, a->k) || !optional_ok(a->bias, a->n, a->n, 2)) return EDEN_ERR_INVALID_ARG;
    if (a->m == 0) return EDEN_OK;
    if ((a->x ? !matrix_ok(a->x, a->x_stride, a->k, 2) || a->held.codes : !mx4_ok(a->held, a->k)) || !optional_ok(a->residual, a->residual_stride, a->n, 2) ||
        !matrix_ok(a->y, a->y_stride, a->n, 2))
        return EDEN_ERR_INVALID_ARG;
    if (a->save != EDEN_SAVE_NONE && !checkpoint_ok(a->saved, a->saved_stride, a->saved_exp, a->saved_exp_stride, a->n)) return EDEN_ERR_INVALID_ARG;
    return guarded(ctx, [&]() -> int {
        Scratch scratch(ctx);
        LinearEpilogue p{a->bias, a->residual, a->residual_stride, a->y, a->y_stride, view(a->saved, a->saved_stride, a->saved_exp, a->saved_exp_stride),
                         nullptr, a->m, a->n, a->act, a->save, 0};
        const double bytes = 17.0 * groups_of(a->k) * ((double)a->m + a->n) + 2.0 * (a->n + (double)a->m * a->n * (a->residual ? 2 : 1)) +
                             (a->save ? (double)a->m * (a->n + groups_of(a->n)) : 0.0);
        const bool few = a->m <= 8 && (ctx->linear_form == EDEN_LINEAR_AUTO || ctx->linear_form == EDEN_LINEAR_FEW);
        // A token's values are quantised by the blocks that use them (1 x 4096 x 4096 in 7.0 us, as a launch of
        // its own 8.9; 3 tokens 9.2 and 9.4); of many, each block would do too much (8 tokens 13.9 and 9.4).
        const bool fused = few && a->x && a->m * a->k <= kFewFused;
        Mx4Operand x = operand_of(a->held, a->m, a->k);
        if (a->x && !fused) {
            if (int rc = quantized(ctx, scratch, a->type, a->x, a->x_stride, a->m, a->k, &x)) return rc;
        }
        if (few) {
            const Mx4Few q{fused ? a->x : nullptr, a->x_stride, {const_cast<uint8_t*>(x.codes), x.stride, const_cast<uint8_t*>(x.exps), tiles_along(a->k)},
                           mx4_view(a->weight, a->k), (uint32_t)a->k};
            // groups of 32 results are saved by a warp that holds them: two times 16 rows of W
            EDEN_DISPATCH_HALF(a->type, return (a->save ? launch_few<T_, 2>(ctx, q, p, bytes) : launch_few<T_, 1>(ctx, q, p, bytes)));
        }
        const Mx4Product q{"t_mx4_linear", a->type, x, operand_of(a->weight, a->n, a->k), p, bytes};
        EDEN_DISPATCH_HALF(a->type, return (product<kForward, T_>(ctx, q)));
    });
}

extern "C" int eden_mx4_linear_input_grad(eden_ctx* ctx, const eden_mx4_linear_input_grad_args* a)
{
    if (!ctx || !a) return EDEN_ERR_INVALID_ARG;
    if (int rc = counts_ok(a->m, a->n, a->k)) return rc;
    if (!half_type(a->type) || !known_act(a->act)) return EDEN_ERR_INVALID_ARG;
    if (!mx4_ok(a->weight_t, a->n) || !optional_ok(a->bias_grad, a->k, a->k, 4)) return EDEN_ERR_INVALID_ARG;
    if (a->m > 0) {
        if ((a->dz ? !matrix_ok(a->dz, a->dz_stride, a->n, 2) || a->held.codes : !mx4_ok(a->held, a->n)) || !optional_ok(a->residual, a->residual_stride, a->k, 2) ||
            !matrix_ok(a->dx, a->dx_stride, a->k, 2))
            return EDEN_ERR_INVALID_ARG;
        if (a->act != EDEN_ACT_NONE && !checkpoint_ok(a->pre, a->pre_stride, a->pre_exp, a->pre_exp_stride, a->k)) return EDEN_ERR_INVALID_ARG;
    }
    return guarded(ctx, [&]() -> int {
        const uint64_t runs = (a->m + 31) / 32;
        float* partial = nullptr;
        if (a->m > 0) {
            Scratch scratch(ctx);
            if (a->bias_grad && (runs > 1 || a->accumulate)) {
                partial = scratch.take<float>(runs * a->k);
                if (!partial) return EDEN_ERR_WORKSPACE;
            } else {
                partial = a->bias_grad;              // 32 rows' sums are the result
            }
            Mx4Operand dz = operand_of(a->held, a->m, a->n);
            if (a->dz) {
                if (int rc = quantized(ctx, scratch, a->type, a->dz, a->dz_stride, a->m, a->n, &dz)) return rc;
            }
            LinearEpilogue p{nullptr, a->residual, a->residual_stride, a->dx, a->dx_stride, view(a->pre, a->pre_stride, a->pre_exp, a->pre_exp_stride), partial,
                             a->m, a->k, a->act, 0, 0};
            const double bytes = 17.0 * groups_of(a->n) * ((double)a->m + a->k) + 2.0 * (double)a->m * a->k * (a->residual ? 2 : 1) +
                                 (a->act ? (double)a->m * (a->k + groups_of(a->k)) : 0.0);
            const Mx4Product q{"t_mx4_input_grad", a->type, dz, operand_of(a->weight_t, a->k, a->n), p, bytes};
            int rc = EDEN_OK;
            EDEN_DISPATCH_HALF(a->type, rc = (product<kInputGrad, T_>(ctx, q)));
            if (rc) return rc;
        }
        return partial != a->bias_grad ? sum_columns(ctx, partial, runs, a->k, a->bias_grad, a->accumulate) : EDEN_OK;
    });
}

extern "C" int eden_mx4_linear_weight_grad(eden_ctx* ctx, const eden_mx4_linear_weight_grad_args* a)
{
    if (!ctx || !a) return EDEN_ERR_INVALID_ARG;
    if (int rc = counts_ok(a->m, a->n, a->k)) return rc;
    if (!matrix_ok(a->weight_grad, a->weight_grad_stride, a->k, 4)) return EDEN_ERR_INVALID_ARG;
    if (a->m > 0 && (!mx4_ok(a->dz_t, a->m) || !mx4_ok(a->x_t, a->m))) return EDEN_ERR_INVALID_ARG;
    if (a->m == 0 && a->accumulate) return EDEN_OK;
    return guarded(ctx, [&]() -> int {
        if (a->m == 0) {
            CUDA_OK(cudaMemset2DAsync(a->weight_grad, a->weight_grad_stride * 4, 0, a->k * 4, a->n, ctx->stream));
            return EDEN_OK;
        }
        LinearEpilogue p{nullptr, nullptr, 0, a->weight_grad, a->weight_grad_stride, {}, nullptr, a->n, a->k, 0, 0, a->accumulate};
        const double bytes = 17.0 * groups_of(a->m) * ((double)a->n + a->k) + 4.0 * a->n * a->k * (a->accumulate ? 2 : 1);
        return product<kWeightGrad, __nv_bfloat16>(ctx, {"t_mx4_weight_grad", EDEN_TYPE_BF16, operand_of(a->dz_t, a->n, a->m), operand_of(a->x_t, a->k, a->m), p, bytes});
    });
}
