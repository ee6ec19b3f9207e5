// C ABI of the client's training step (declared in include/eden.h): argument checks,
// workspace carving and launches.
#include <algorithm>
#include <atomic>
#include <cmath>

#include "kernels_checkpoint.cuh"
#include "kernels_linear.cuh"
#include "tensor_map.h"
#include "train_host.h"

using namespace eden;

namespace {

constexpr uint64_t kMaxRuns = 512;              // runs of rows that leave partial column sums

// The kernels' WIDE forms: rows of values on 32-byte boundaries, rows of codes on 16-byte ones.
// 16384 x 4096 bf16 is saved and restored in 64 to 67 us a call by them, in 98 us by the others.
bool wide_codes(const CheckpointView& c) { return aligned(c.codes, 16) && c.codes_stride % 16 == 0; }

template <typename T>
int save(eden_ctx* ctx, const T* x, uint64_t x_stride, CheckpointView c, uint64_t m, uint64_t n)
{
    const uint64_t groups = groups_of(n), total = m * groups * 2, blocks = (total + kCkptThreads - 1) / kCkptThreads;
    if (blocks > kMaxCount) return EDEN_ERR_TOO_LARGE;
    const bool wide = wide_rows(x, x_stride, sizeof(T)) && wide_codes(c);
    return launch(ctx, "t_save", (double)m * (n * (1.0 + sizeof(T)) + groups), wide ? k_checkpoint_save<T, true> : k_checkpoint_save<T, false>,
                  dim3((uint32_t)blocks), kCkptThreads, 0, 1, x, x_stride, c, n, groups * 2, total);
}

template <typename T>
int restore(eden_ctx* ctx, CheckpointView c, T* x, uint64_t x_stride, uint64_t m, uint64_t n)
{
    const uint64_t groups = groups_of(n), total = m * groups * 2, blocks = (total + kCkptThreads - 1) / kCkptThreads;
    if (blocks > kMaxCount) return EDEN_ERR_TOO_LARGE;
    const bool wide = wide_rows(x, x_stride, sizeof(T)) && wide_codes(c);
    return launch(ctx, "t_restore", (double)m * (n * (1.0 + sizeof(T)) + groups),
                  wide ? k_checkpoint_restore<T, true> : k_checkpoint_restore<T, false>, dim3((uint32_t)blocks), kCkptThreads, 0, 1, x, x_stride, c,
                  n, groups * 2, total);
}

template <typename T, int ACT>
int act_backward(eden_ctx* ctx, const eden_act_backward_args* a, float* partial, uint64_t strips, uint64_t runs, uint64_t rows_per_run)
{
    const bool wide = wide_rows(a->dy, a->dy_stride, 2) && (!a->dz || wide_rows(a->dz, a->dz_stride, 2)) &&
                      (ACT == EDEN_ACT_NONE || wide_codes(view(a->pre, a->pre_stride, a->pre_exp, a->pre_exp_stride)));
    const double bytes = (double)a->m * a->n * (2.0 + (a->dz ? 2.0 : 0.0) + (ACT ? 1.0 : 0.0));
    return launch(ctx, "t_act_backward", bytes, wide ? k_act_backward<T, ACT, true> : k_act_backward<T, ACT, false>,
                  dim3((uint32_t)strips, (uint32_t)runs), kCkptThreads, 0, 1, (const T*)a->dy, a->dy_stride,
                  view(a->pre, a->pre_stride, a->pre_exp, a->pre_exp_stride), (T*)a->dz, a->dz_stride, partial, a->m, a->n, rows_per_run);
}

#define EDEN_DISPATCH_ACT(act, CALL)                                                            \
    switch (act) {                                                                              \
        case EDEN_ACT_RELU: { constexpr int ACT_ = EDEN_ACT_RELU; CALL; } break;                \
        case EDEN_ACT_GELU: { constexpr int ACT_ = EDEN_ACT_GELU; CALL; } break;                \
        case EDEN_ACT_GELU_TANH: { constexpr int ACT_ = EDEN_ACT_GELU_TANH; CALL; } break;      \
        case EDEN_ACT_SILU: { constexpr int ACT_ = EDEN_ACT_SILU; CALL; } break;                \
        default: { constexpr int ACT_ = EDEN_ACT_NONE; CALL; } break;                           \
    }

// An operand of a product: `rows` rows of `n` 16-bit values, or (data null) a checkpoint of them.
struct Operand {
    const void* data;
    uint64_t stride, rows, n;
    CheckpointView held;
};

// Tensor copies want 16-byte aligned rows of values: other operands are laid out so in the
// workspace first, both in one launch.
template <typename T>
int lay_out(eden_ctx* ctx, Scratch& scratch, Operand& a, Operand& b)
{
    Layout job[2] = {};
    uint64_t blocks[2] = {0, 0};
    double bytes = 0;
    int n = 0;
    for (Operand* o : {&a, &b}) {
        if (o->data && o->rows == 1) o->stride = padded(o->n);
        if (o->data && aligned(o->data, 16) && o->stride % 8 == 0) continue;
        const uint64_t stride = padded(o->n), total = o->rows * (stride / 16);
        uint16_t* to = scratch.take<uint16_t>(o->rows * stride);
        if (!to) return EDEN_ERR_WORKSPACE;
        job[n] = {o->data, o->held, o->stride, to, stride, o->n, total, aligned(o->held.codes, 16) && o->held.codes_stride % 16 == 0};
        blocks[n] = (total + 255) / 256;
        bytes += (double)o->rows * o->n * (o->data ? 4 : 3);
        o->data = to;
        o->stride = stride;
        ++n;
    }
    if (n == 0) return EDEN_OK;
    if (blocks[0] + blocks[1] > kMaxCount) return EDEN_ERR_TOO_LARGE;
    return launch(ctx, "t_lay_out", bytes, k_lay_out<T>, dim3((uint32_t)(blocks[0] + blocks[1])), 256, 0, 1, job[0], job[1], (uint32_t)blocks[0]);
}

// boxes of 64 values x box_rows rows, 128-byte swizzle, zeros outside
int make_map(CUtensorMap* map, int type, const Operand& o, uint32_t box_rows)
{
    const cuuint64_t dims[2] = {o.n, o.rows}, strides[1] = {o.stride * 2};
    const cuuint32_t box[2] = {64, box_rows};
    return encode_tiles(map, type == EDEN_TYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, o.data, dims, strides, box,
                        CU_TENSOR_MAP_SWIZZLE_128B);
}

struct Product {
    const char* name;
    int type;
    Operand a, b;                      // rows of the result (weight grad: steps of the sum), columns likewise
    uint64_t depth;                    // length of the sum
    LinearEpilogue p;
    double bytes;
};

template <int OP, typename T, int CG, int BN, bool SPLIT, bool RUNS, int SIDES = 2>
int launch_linear(eden_ctx* ctx, const Product& q, uint32_t splits, uint32_t begin, uint32_t end)
{
    using S = LinearShape<CG, BN, SIDES>;
    CUtensorMap map_a, map_b;
    if (int rc = make_map(&map_a, q.type, q.a, OP == kWeightGrad ? 64 : 128)) return rc;
    if (int rc = make_map(&map_b, q.type, q.b, OP == kForward ? S::kRowsB : 64)) return rc;
    const uint64_t rows = (q.p.rows + 128 * CG - 1) / (128 * CG), cols = (q.p.cols + BN - 1) / BN;
    if (rows * cols * CG * splits > kMaxCount) return EDEN_ERR_TOO_LARGE;
    if (end == 0) end = (uint32_t)(rows * cols);
    const TileGrid grid{(uint32_t)rows, (uint32_t)cols, begin, end, (uint32_t)((q.depth + S::kDepth - 1) / S::kDepth), splits};
    const auto kernel = k_linear<OP, T, CG, BN, SPLIT, RUNS, SIDES>;
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
    const uint32_t groups = SPLIT ? end - begin : std::min<uint32_t>(end - begin, ctx->sm_count / CG);
    return launch(ctx, q.name, q.bytes, kernel, dim3(groups * CG * splits), S::kThreads, S::kSharedBytes, CG * splits, map_a, map_b, q.p,
                  grid, (uint32_t*)ctx->ws);
}

template <int OP, typename T, int CG, int BN, bool SPLIT>
int launch_runs(eden_ctx* ctx, const Product& q, uint32_t splits, uint32_t begin = 0, uint32_t end = 0)
{
    // codes and column sums are not left with the drift of long sums (kPromote)
    const bool exact = OP == kInputGrad ? q.p.column_sums != nullptr : q.p.save != EDEN_SAVE_NONE;
    const bool runs = exact && (q.depth + 63) / 64 > (uint64_t)kPromote * splits;
    if constexpr (OP != kWeightGrad && CG == 2 && !SPLIT) {
        // sums of up to 2048 do not hide such an epilogue behind their products (8200 cycles for 1024);
        // more than two runs do not fit the registers of sixteen epilogue warps
        if ((q.p.act || q.p.residual || exact) && q.depth <= (runs ? 128 * kPromote : 2048)) {
            if (runs) return launch_linear<OP, T, CG, BN, SPLIT, true, 4>(ctx, q, 1, begin, end);
            return launch_linear<OP, T, CG, BN, SPLIT, false, 4>(ctx, q, 1, begin, end);
        }
    }
    if constexpr (OP != kWeightGrad) {
        if (!runs) return launch_linear<OP, T, CG, BN, SPLIT, false>(ctx, q, splits, begin, end);
    }
    return launch_linear<OP, T, CG, BN, SPLIT, true>(ctx, q, splits, begin, end);
}

// How a product is cut up: a form (EDEN_LINEAR_*) and the parts of each tile's sum; and, where the
// last wave of whole tiles would leave many SMs without one, the first of the tiles that a second
// launch takes in `tail_splits` parts each.
struct Cut {
    int form;
    uint32_t splits, tail, tail_splits;
};

template <int OP, int CG, int BN>
int launch_tiles(eden_ctx* ctx, const Product& q, const Cut& cut)
{
    int rc = EDEN_OK;
    if (cut.splits > 1) {
        EDEN_DISPATCH_HALF(q.type, rc = (launch_runs<OP, T_, CG, BN, true>(ctx, q, cut.splits)));
        return rc;
    }
    EDEN_DISPATCH_HALF(q.type, rc = (launch_runs<OP, T_, CG, BN, false>(ctx, q, 1, 0, cut.tail)));
    if (rc || cut.tail == 0) return rc;
    EDEN_DISPATCH_HALF(q.type, rc = (launch_runs<OP, T_, CG, BN, true>(ctx, q, cut.tail_splits, cut.tail)));
    return rc;
}

// A block for each SM where there are fewer rows of W than that, as long as its warps have a step each.
uint32_t few_parts(const eden_ctx* ctx, uint64_t blocks, uint64_t depth)
{
    uint32_t parts = 1;
    while (parts < 8 && blocks * parts * 2 <= (uint64_t)ctx->sm_count && (depth + 63) / 64 >= 16 * 2 * parts) parts *= 2;
    return parts;
}

template <typename T, int NT, int R>
int launch_few(eden_ctx* ctx, const Product& q)
{
    const bool vec = aligned(q.a.data, 16) && aligned(q.b.data, 16) && q.depth % 8 == 0 && (q.a.stride % 8 == 0 || q.a.rows == 1) &&
                     (q.b.stride % 8 == 0 || q.b.rows == 1);
    const uint64_t blocks = (q.p.cols + 16 * R - 1) / (16 * R);
    const uint32_t parts = few_parts(ctx, blocks, q.depth);
    const auto kernel = parts > 1 ? (vec ? k_linear_few<T, NT, R, true, true> : k_linear_few<T, NT, R, false, true>)
                                  : (vec ? k_linear_few<T, NT, R, true, false> : k_linear_few<T, NT, R, false, false>);
    return launch(ctx, q.name, q.bytes, kernel, dim3((uint32_t)blocks, parts), kFewThreads, 0, parts, (const T*)q.a.data, q.a.stride,
                  (const T*)q.b.data, q.b.stride, q.depth, q.p);
}

template <typename T>
int launch_few(eden_ctx* ctx, const Product& q)
{
    if (q.p.save) return q.p.rows <= 8 ? launch_few<T, 1, 2>(ctx, q) : q.p.rows <= 16 ? launch_few<T, 2, 2>(ctx, q) : launch_few<T, 4, 2>(ctx, q);
    return q.p.rows <= 8 ? launch_few<T, 1, 1>(ctx, q) : q.p.rows <= 16 ? launch_few<T, 2, 1>(ctx, q) : launch_few<T, 4, 1>(ctx, q);
}

// Clusters of 1, 2, 4 or 8 blocks with a tile's stages that the device runs at once: clusters do
// not span the GPU's processing clusters, so fewer blocks fit than there are SMs.
int cluster_slots(eden_ctx* ctx, uint32_t cluster)
{
    int& known = ctx->cluster_slots[cluster];
    if (known > 0) return known;
    const auto kernel = k_linear<kForward, __nv_bfloat16, 1, 128, true, false, 2>;
    using S = LinearShape<1, 128, 2>;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(cluster * ctx->sm_count);
    cfg.blockDim = dim3(S::kThreads);
    cfg.dynamicSmemBytes = S::kSharedBytes;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim = {cluster, 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSharedBytes) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n <= 0) {
        cudaGetLastError();
        n = std::max(1, ctx->sm_count / (int)cluster * 3 / 4);
    }
    return known = n;
}

// The cheapest form by a model of its time in microseconds, fitted to sums of 1024 and 4096 on
// one to 512 tiles: a launch's fixed part, a step of 64 along the sum (the pair's is its
// products' time, the others' the issue of their products and barriers), the epilogue of a tile
// where it outlasts the tile's steps, and the join of a split tile.
template <int OP>
Cut choose_cut(eden_ctx* ctx, const Product& q)
{
    const uint64_t steps = (q.depth + 63) / 64;
    const int form = ctx->linear_form;
    if (OP == kForward && q.p.rows <= 32 && (form == EDEN_LINEAR_FEW || (form == EDEN_LINEAR_AUTO && q.p.rows <= 16))) return {EDEN_LINEAR_FEW, 1, 0, 0};
    static const struct { int form; uint64_t rows, cols, depth; uint32_t blocks; double fixed, step, finish, split, join; } tiles[] = {
        {EDEN_LINEAR_PAIR, 256, 256, 64, 2, 6.0, 0.265, OP == kWeightGrad ? 3.4 : 2.2, 0.0, 0.5},
        {EDEN_LINEAR_SINGLE, 128, 128, 128, 1, 4.9, 0.185, OP == kWeightGrad ? 1.6 : 1.3, 1.0, 0.5},
        {EDEN_LINEAR_NARROW, 128, 64, 128, 1, 3.6, 0.159, OP == kWeightGrad ? 0.95 : 0.9, 1.2, 0.4}};
    // fp32 rows that start on 16, 8 or 4 bytes leave in more and smaller stores
    const int grain = OP == kWeightGrad ? row_grain(q.p.out, q.p.out_stride, 4) : 32;
    const double slower = grain >= 32 ? 1.0 : grain >= 16 ? 1.4 : grain >= 8 ? 1.75 : 2.7;
    Cut best{EDEN_LINEAR_PAIR, 1, 0, 0};
    double least = 1e300;
    for (const auto& t : tiles) {
        if (form != EDEN_LINEAR_AUTO && form != EDEN_LINEAR_FEW && form != t.form) continue;
        const uint64_t count = (q.p.rows + t.rows - 1) / t.rows * ((q.p.cols + t.cols - 1) / t.cols);
        uint32_t most = 1;
        while (2 * most * t.blocks <= 8 && 2 * most <= (steps * 64 + t.depth - 1) / t.depth) most *= 2;
        for (uint32_t splits = 1; splits <= most; splits *= 2) {
            if (ctx->linear_splits && splits != std::min(most, (uint32_t)ctx->linear_splits)) continue;
            const uint64_t slots = cluster_slots(ctx, splits * t.blocks), waves = (count + slots - 1) / slots;
            const double sum = (double)((steps + splits - 1) / splits) * t.step;
            const double cost = splits > 1 ? waves * (t.fixed + t.split + t.join * splits + sum) : t.fixed + waves * std::max(sum, t.finish * slower);
            if (cost < least) {
                least = cost;
                best = {t.form, splits, 0, 0};
            }
            // whole waves, and the rest in parts: 256 tiles on 74 pairs are 3 waves and 34 tiles
            const uint64_t pairs = cluster_slots(ctx, t.blocks), whole = count / pairs * pairs;
            if (splits == 1 || ctx->linear_splits || whole == 0 || whole == count) continue;
            const uint64_t tail_waves = (count - whole + slots - 1) / slots;
            const double with_tail = t.fixed + (double)(whole / pairs) * std::max((double)steps * t.step, t.finish * slower) +
                                     tail_waves * (t.fixed + t.split + t.join * splits + sum);
            if (with_tail < least) {
                least = with_tail;
                best = {t.form, 1, (uint32_t)whole, splits};
            }
        }
    }
    // 17 to 32 tokens: the form for few takes W at HBM's rate, but its blocks (a wave of 148 costs 2 us)
    // each read all of x, at about 20 TB/s from the caches.  Up to 16 it was never behind by more than a tenth.
    if (OP == kForward && form == EDEN_LINEAR_AUTO && q.p.rows <= 32) {
        const double blocks = (double)((q.p.cols + 15) / 16), waves = std::ceil(blocks / ctx->sm_count);
        const double few = 1.5 + waves * 2.0 + (double)q.p.cols * q.depth * 2 / 6e6 + blocks * q.p.rows * q.depth * 2 / 20e6 +
                           (double)steps / (16 * few_parts(ctx, (uint64_t)blocks, q.depth)) * 0.8;
        if (few < least) best = {EDEN_LINEAR_FEW, 1, 0, 0};
    }
    return best;
}

template <int OP>
int product(eden_ctx* ctx, Scratch& scratch, Product q)
{
    const Cut cut = choose_cut<OP>(ctx, q);
    if constexpr (OP == kForward) {
        if (cut.form == EDEN_LINEAR_FEW) { EDEN_DISPATCH_HALF(q.type, return launch_few<T_>(ctx, q)); }
    }
    int rc = EDEN_OK;
    EDEN_DISPATCH_HALF(q.type, rc = lay_out<T_>(ctx, scratch, q.a, q.b));
    if (rc) return rc;
    LinearEpilogue& p = q.p;
    p.grain_out = row_grain(p.out, p.out_stride, OP == kWeightGrad ? 4 : 2);
    p.grain_residual = row_grain(p.residual, p.residual_stride, 2);
    p.grain_codes = row_grain(p.ckpt.codes, p.ckpt.codes_stride, 1);
    p.grain_bias = row_grain(p.bias, 0, 2);
    switch (cut.form) {
        case EDEN_LINEAR_PAIR: return launch_tiles<OP, 2, 256>(ctx, q, cut);
        case EDEN_LINEAR_SINGLE: return launch_tiles<OP, 1, 128>(ctx, q, cut);
        default: return launch_tiles<OP, 1, 64>(ctx, q, cut);
    }
}

}  // namespace

extern "C" uint64_t eden_checkpoint_groups(uint64_t features) { return groups_of(features); }

extern "C" uint64_t eden_linear_workspace_bytes(uint64_t m, uint64_t n, uint64_t k)
{
    // 16-bit copies of operands whose rows are not 16-byte aligned (or are restored from
    // codes), and the partial column sums
    const uint64_t mn = m * padded(n) * 2, mk = m * padded(k) * 2, nk = n * padded(k) * 2;
    const uint64_t sums = std::max(std::max<uint64_t>((m + 31) / 32, 1) * k, kMaxRuns * n) * 4;
    return std::max(least_workspace(), kStatusBytes + std::max(mk + nk, std::max(mn + nk, mn + mk)) + sums + 4 * 256);
}

extern "C" int eden_linear(eden_ctx* ctx, const eden_linear_args* a)
{
    if (!ctx || !a) return EDEN_ERR_INVALID_ARG;
    if (int rc = counts_ok(a->m, a->n, a->k)) return rc;
    if (!half_type(a->type) || !known_act(a->act) || a->save < EDEN_SAVE_NONE || a->save > EDEN_SAVE_OUT) return EDEN_ERR_INVALID_ARG;
    if (!matrix_ok(a->weight, a->weight_stride, a->k, 2) || !optional_ok(a->bias, a->n, a->n, 2)) return EDEN_ERR_INVALID_ARG;
    if (a->m == 0) return EDEN_OK;
    if (!matrix_ok(a->x, a->x_stride, a->k, 2) || !optional_ok(a->residual, a->residual_stride, a->n, 2) ||
        !matrix_ok(a->y, a->y_stride, a->n, 2))
        return EDEN_ERR_INVALID_ARG;
    if (a->save != EDEN_SAVE_NONE && !checkpoint_ok(a->saved, a->saved_stride, a->saved_exp, a->saved_exp_stride, a->n))
        return EDEN_ERR_INVALID_ARG;
    return guarded(ctx, [&]() -> int {
        Scratch scratch(ctx);
        LinearEpilogue p{a->bias, a->residual, a->residual_stride, a->y, a->y_stride,
                         view(a->saved, a->saved_stride, a->saved_exp, a->saved_exp_stride), nullptr, a->m, a->n, a->act, a->save, 0};
        const double bytes = 2.0 * ((double)a->m * a->k + (double)a->n * a->k + a->n + (double)a->m * a->n * (a->residual ? 2 : 1)) +
                             (a->save ? (double)a->m * (a->n + groups_of(a->n)) : 0.0);
        return product<kForward>(ctx, scratch, {"t_linear", a->type, {a->x, a->x_stride, a->m, a->k, {}}, {a->weight, a->weight_stride, a->n, a->k, {}},
                                                a->k, p, bytes});
    });
}

extern "C" int eden_checkpoint_save(eden_ctx* ctx, const eden_checkpoint_args* a)
{
    if (!ctx || !a || a->n == 0 || a->type < EDEN_TYPE_BF16 || a->type > EDEN_TYPE_FP32) return EDEN_ERR_INVALID_ARG;
    if (std::max(a->m, a->n) > kMaxCount) return EDEN_ERR_TOO_LARGE;
    if (a->m == 0) return EDEN_OK;
    if (!matrix_ok(a->x, a->x_stride, a->n, type_size(a->type)) ||
        !checkpoint_ok(a->codes, a->codes_stride, a->exps, a->exps_stride, a->n))
        return EDEN_ERR_INVALID_ARG;
    return guarded(ctx, [&]() -> int {
        const CheckpointView c = view(a->codes, a->codes_stride, a->exps, a->exps_stride);
        EDEN_DISPATCH_TYPE(a->type, return save(ctx, (const T_*)a->x, a->x_stride, c, a->m, a->n));
    });
}

extern "C" int eden_checkpoint_restore(eden_ctx* ctx, const eden_checkpoint_args* a)
{
    if (!ctx || !a || a->n == 0 || a->type < EDEN_TYPE_BF16 || a->type > EDEN_TYPE_FP32) return EDEN_ERR_INVALID_ARG;
    if (std::max(a->m, a->n) > kMaxCount) return EDEN_ERR_TOO_LARGE;
    if (a->m == 0) return EDEN_OK;
    if (!matrix_ok(a->x, a->x_stride, a->n, type_size(a->type)) ||
        !checkpoint_ok(a->codes, a->codes_stride, a->exps, a->exps_stride, a->n))
        return EDEN_ERR_INVALID_ARG;
    return guarded(ctx, [&]() -> int {
        const CheckpointView c = view(a->codes, a->codes_stride, a->exps, a->exps_stride);
        EDEN_DISPATCH_TYPE(a->type, return restore(ctx, c, (T_*)a->x, a->x_stride, a->m, a->n));
    });
}

extern "C" int eden_act_backward(eden_ctx* ctx, const eden_act_backward_args* a)
{
    if (!ctx || !a || a->n == 0 || !half_type(a->type) || !known_act(a->act)) return EDEN_ERR_INVALID_ARG;
    if (std::max(a->m, a->n) > kMaxCount) return EDEN_ERR_TOO_LARGE;
    if (!optional_ok(a->bias_grad, a->n, a->n, 4)) return EDEN_ERR_INVALID_ARG;
    if (a->m > 0) {
        if (!matrix_ok(a->dy, a->dy_stride, a->n, 2) || !optional_ok(a->dz, a->dz_stride, a->n, 2)) return EDEN_ERR_INVALID_ARG;
        if (a->act != EDEN_ACT_NONE && !checkpoint_ok(a->pre, a->pre_stride, a->pre_exp, a->pre_exp_stride, a->n)) return EDEN_ERR_INVALID_ARG;
    }
    return guarded(ctx, [&]() -> int {
        uint64_t runs = 0;
        float* partial = nullptr;
        if (a->m > 0 && (a->dz || a->bias_grad)) {
            // about six blocks of eight warps for each SM, at least 8 rows (one per warp) to a run
            const uint64_t strips = (a->n + 511) / 512;
            const uint64_t want = std::min<uint64_t>(kMaxRuns, std::max<uint64_t>(1, 6ull * ctx->sm_count / strips));
            const uint64_t rows_per_run = std::max<uint64_t>(a->m <= 32 ? 32 : 8, (a->m + want - 1) / want);
            runs = (a->m + rows_per_run - 1) / rows_per_run;
            if (a->bias_grad && (runs > 1 || a->accumulate)) {
                partial = Scratch(ctx).take<float>(runs * a->n);
                if (!partial) return EDEN_ERR_WORKSPACE;
            } else {
                partial = a->bias_grad;              // one run's sums are the result
            }
            int rc = EDEN_OK;
            EDEN_DISPATCH_HALF(a->type, EDEN_DISPATCH_ACT(a->act, rc = (act_backward<T_, ACT_>(ctx, a, partial, strips, runs, rows_per_run))));
            if (rc) return rc;
        }
        return partial != a->bias_grad ? sum_columns(ctx, partial, runs, a->n, a->bias_grad, a->accumulate) : EDEN_OK;
    });
}

extern "C" int eden_linear_input_grad(eden_ctx* ctx, const eden_linear_input_grad_args* a)
{
    if (!ctx || !a) return EDEN_ERR_INVALID_ARG;
    if (int rc = counts_ok(a->m, a->n, a->k)) return rc;
    if (!half_type(a->type) || !known_act(a->act)) return EDEN_ERR_INVALID_ARG;
    if (!matrix_ok(a->weight, a->weight_stride, a->k, 2) || !optional_ok(a->bias_grad, a->k, a->k, 4)) return EDEN_ERR_INVALID_ARG;
    if (a->m > 0) {
        if (!matrix_ok(a->dz, a->dz_stride, a->n, 2) || !optional_ok(a->residual, a->residual_stride, a->k, 2) ||
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
            LinearEpilogue p{nullptr, a->residual, a->residual_stride, a->dx, a->dx_stride,
                             view(a->pre, a->pre_stride, a->pre_exp, a->pre_exp_stride), partial, a->m, a->k, a->act, 0, 0};
            const double bytes = 2.0 * ((double)a->m * a->n + (double)a->n * a->k + (double)a->m * a->k * (a->residual ? 2 : 1)) +
                                 (a->act ? (double)a->m * (a->k + groups_of(a->k)) : 0.0);
            if (int rc = product<kInputGrad>(ctx, scratch, {"t_input_grad", a->type, {a->dz, a->dz_stride, a->m, a->n, {}},
                                                            {a->weight, a->weight_stride, a->n, a->k, {}}, a->n, p, bytes}))
                return rc;
        }
        return partial != a->bias_grad ? sum_columns(ctx, partial, runs, a->k, a->bias_grad, a->accumulate) : EDEN_OK;
    });
}

extern "C" int eden_linear_weight_grad(eden_ctx* ctx, const eden_linear_weight_grad_args* a)
{
    if (!ctx || !a) return EDEN_ERR_INVALID_ARG;
    if (int rc = counts_ok(a->m, a->n, a->k)) return rc;
    if (!half_type(a->type) || !matrix_ok(a->weight_grad, a->weight_grad_stride, a->k, 4)) return EDEN_ERR_INVALID_ARG;
    if (a->m > 0) {
        if (!matrix_ok(a->dz, a->dz_stride, a->n, 2) || !!a->x == !!a->codes) return EDEN_ERR_INVALID_ARG;
        if (a->x ? !matrix_ok(a->x, a->x_stride, a->k, 2) : !checkpoint_ok(a->codes, a->codes_stride, a->exps, a->exps_stride, a->k))
            return EDEN_ERR_INVALID_ARG;
    }
    if (a->m == 0 && a->accumulate) return EDEN_OK;
    return guarded(ctx, [&]() -> int {
        if (a->m == 0) {
            CUDA_OK(cudaMemset2DAsync(a->weight_grad, a->weight_grad_stride * 4, 0, a->k * 4, a->n, ctx->stream));
            return EDEN_OK;
        }
        Scratch scratch(ctx);
        const Operand x{a->x, a->x_stride, a->m, a->k, view(a->codes, a->codes_stride, a->exps, a->exps_stride)};
        LinearEpilogue p{nullptr, nullptr, 0, a->weight_grad, a->weight_grad_stride, {}, nullptr, a->n, a->k, 0, 0, a->accumulate};
        const double bytes = 2.0 * a->m * a->n + (double)a->m * (a->codes ? a->k + groups_of(a->k) : 2 * a->k) +
                             4.0 * a->n * a->k * (a->accumulate ? 2 : 1);
        return product<kWeightGrad>(ctx, scratch, {"t_weight_grad", a->type, {a->dz, a->dz_stride, a->m, a->n, {}}, x, a->m, p, bytes});
    });
}
