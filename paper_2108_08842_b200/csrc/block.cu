// C ABI of what joins a client's blocks (declared in include/eden.h): argument checks, workspace
// carving and launches.
#include <atomic>
#include <cmath>

#include "kernels_block.cuh"
#include "train_host.h"

using namespace eden;

namespace {

constexpr uint64_t kMaxSlots = 192;             // blocks of a launch with norms, whatever the device
constexpr uint64_t kMaxRuns = 512;              // runs of rows of a backward launch without norms
constexpr uint64_t kMaxNormColumns = 512ull * kTeamWarps * kBlockCluster / 2;   // whatever a row needs fits a cluster
static_assert(kMaxNormColumns == EDEN_NORM_MAX_FEATURES, "as documented");

bool rows_on_16(const void* p, uint64_t stride) { return !p || (aligned(p, 16) && stride % 8 == 0); }

bool known_norm(const eden_norm& n)
{
    if (n.kind < EDEN_NORM_NONE || n.kind > EDEN_NORM_LAYER) return false;
    return n.kind == EDEN_NORM_NONE || (aligned(n.weight, 2) && aligned(n.bias, 2) && n.eps >= 0.f && std::isfinite(n.eps));
}

bool drop_ok(const eden_drop& d, uint64_t m)
{
    return d.rate >= 0.0 && d.rate <= 1.0 && aligned(d.seed_at, 8) && d.first_row <= kMaxCount && d.first_row + m <= 1ull << 32;
}

DropView drop_view(const eden_drop& d, int* has)
{
    DropView v{d.seed, d.seed_at, (uint32_t)(65536.0 * (1.0 - d.rate) + 0.5), (uint32_t)d.first_row, 0.f};
    v.factor = v.keep ? 65536.f / (float)v.keep : 0.f;
    *has = v.keep != 65536;
    return v;
}

// stride 0 where one vector serves all rows
uint64_t gate_stride(const void* gate, int per_value, uint64_t stride) { return gate && per_value ? stride : 0; }

Source matrix_source(const void* p, uint64_t stride) { return {(const char*)p, stride * 2, 2, 0, 0, 0, rows_on_16(p, stride)}; }
Source stats_source(const float* p) { return {(const char*)p, 8, 8, 0, 1, 0, 0}; }

// Rows over teams, blocks and clusters: see kernels_block.cuh.
struct Grid {
    BlockShape s;
    uint32_t blocks, threads, shared, pieces, parts;
    bool wide;                         // of the sources; the outputs' rows count as well
};

// What a block has beside its rows and vectors: places for sums, store buffers and barriers.
constexpr uint32_t kRowsShared = (227 - 17) * 1024;

Grid grid_of(const eden_ctx* ctx, uint64_t m, uint64_t n, const Source (&source)[kMaxSources], uint32_t warps, bool full, uint32_t sums)
{
    Grid g{};
    BlockShape& s = g.s;
    s.m = (uint32_t)m;
    s.n = (uint32_t)n;
    const uint64_t sms = std::min<uint64_t>(ctx->sm_count, kMaxSlots);
    // Two pieces a thread where that leaves a row for every SM, or where one would need a cluster.
    // (gradients with everything do not fit the registers with two: 200 to 600 bytes of spills)
    g.pieces = n > 256 * kTeamWarps || (n > 256 && m >= sms && !(full && sums)) ? 2 : 1;
    const uint64_t columns = 256ull * kTeamWarps * g.pieces;
    uint32_t vectors = 0;
    for (s.blocks = 1;; s.blocks *= 2) {
        s.warps = (uint32_t)(((n + s.blocks - 1) / s.blocks + 256 * g.pieces - 1) / (256 * g.pieces));
        s.span = s.warps * 256 * g.pieces;
        vectors = (full ? kVectors<true> : kVectors<false>) * s.span * 4;
        const uint32_t width = (uint32_t)std::min<uint64_t>(n, s.span);
        s.row_bytes = 0;
        g.wide = n % 8 == 0;
        for (int i = 0; i < kMaxSources; ++i) {
            s.source[i] = source[i];
            if (!source[i].base) continue;
            s.source[i].at = s.row_bytes;
            // up to 15 bytes of a neighbour, and whole words behind the last value; all of the team's columns
            s.row_bytes += (uint32_t)align_to(std::max(source[i].bytes_of(width) + 48, source[i].bytes_of(s.span)), 16);
            if (!source[i].fixed && !source[i].shift) g.wide = g.wide && source[i].aligned;
        }
        if (s.blocks * columns >= n && 2 * s.row_bytes + vectors <= kRowsShared) break;
        if (s.blocks == kBlockCluster) return g;                  // not reached: rows of that many columns are refused
    }
    s.teams = s.blocks > 1 ? 1 : warps / s.warps;                  // a cluster's blocks work on one row
    // few rows: a team of each block has one before a block has two
    while (s.teams > 1 && (2 * s.row_bytes * s.teams + vectors > kRowsShared || (uint64_t)s.teams * (sms / s.blocks) >= 2 * m)) s.teams = (s.teams + 1) / 2;
    s.stages = std::min<uint32_t>(kMaxStages, (kRowsShared - vectors) / (s.row_bytes * s.teams));
    s.vectors = s.teams * s.stages * s.row_bytes;
    const uint64_t groups = std::min<uint64_t>((m + s.teams - 1) / s.teams, std::max<uint64_t>(1, sms / s.blocks));
    g.blocks = (uint32_t)groups * s.blocks;
    g.threads = s.teams * s.warps * 32;
    g.shared = std::max(s.vectors + vectors, s.teams * sums * s.span * 4);     // the teams' sums, at most 160 KB
    g.parts = (uint32_t)groups;
    return g;
}

template <auto kernel, typename View>
int launch_rows(eden_ctx* ctx, const char* name, double bytes, const View& p, const Grid& g)
{
    static std::atomic<uint64_t> asked{0};       // devices on which this kernel may use its shared memory
    const uint64_t device = 1ull << (ctx->device & 63);
    if (!(asked.load(std::memory_order_relaxed) & device) || ctx->device > 63) {
        CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kRowsShared));
        asked.fetch_or(device, std::memory_order_relaxed);
    }
    return launch(ctx, name, bytes, kernel, dim3(g.blocks), g.threads, g.shared, g.s.blocks, p, g.s, (uint32_t*)ctx->ws);
}

bool full(const eden_norm& n) { return n.kind == EDEN_NORM_LAYER || (n.kind != EDEN_NORM_NONE && n.bias); }

// The launch of the kernel for everything or less, aligned rows or any, and one or two pieces a thread.
#define EDEN_JOIN_PIECES(kernel, f, w, pieces, ...) \
    ((pieces) == 2 ? launch_rows<kernel<T, AFTER, BEFORE, f, w, 2>>(__VA_ARGS__) : launch_rows<kernel<T, AFTER, BEFORE, f, w, 1>>(__VA_ARGS__))
#define EDEN_JOIN_KERNEL(kernel, f, w, pieces, ...)                                                                                             \
    ((f) ? ((w) ? EDEN_JOIN_PIECES(kernel, true, true, pieces, __VA_ARGS__) : EDEN_JOIN_PIECES(kernel, true, false, pieces, __VA_ARGS__))       \
         : ((w) ? EDEN_JOIN_PIECES(kernel, false, true, pieces, __VA_ARGS__) : EDEN_JOIN_PIECES(kernel, false, false, pieces, __VA_ARGS__)))

template <typename T, bool AFTER, bool BEFORE>
int join(eden_ctx* ctx, const JoinView& p, const Grid& g, bool f, double bytes)
{
    const bool wide = g.wide && rows_on_16(p.x, p.x_stride) && rows_on_16(p.y, p.y_stride);
    return EDEN_JOIN_KERNEL(k_join, f, wide, g.pieces, ctx, "t_join", bytes, p, g);
}

template <typename T, bool AFTER, bool BEFORE>
int join_backward(eden_ctx* ctx, const JoinBackwardView& p, const Grid& g, bool f, double bytes)
{
    const bool wide = g.wide && rows_on_16(p.d_residual, p.d_residual_stride) && rows_on_16(p.dh, p.dh_stride) && rows_on_16(p.d_gate, p.d_gate_stride);
    return EDEN_JOIN_KERNEL(k_join_backward, f, wide, g.pieces, ctx, "t_join_backward", bytes, p, g);
}

#define EDEN_DISPATCH_NORMS(after, before, CALL)                                                   \
    if (after) {                                                                                  \
        if (before) { constexpr bool AFTER_ = true, BEFORE_ = true; CALL; }                       \
        else { constexpr bool AFTER_ = true, BEFORE_ = false; CALL; }                             \
    } else { constexpr bool AFTER_ = false, BEFORE_ = true; CALL; }

int sizes_ok(uint64_t m, uint64_t n, bool sums)
{
    if (int rc = counts_ok(m, n, 1)) return rc;
    return sums && n > kMaxNormColumns ? EDEN_ERR_TOO_LARGE : EDEN_OK;
}

bool kept_ok(const eden_kept& k, uint64_t n)
{
    return k.data ? matrix_ok(k.data, k.stride, n, 2) : checkpoint_ok(k.codes, k.codes_stride, k.exps, k.exps_stride, n);
}

KeptView kept_view(const eden_kept& k) { return {k.data, k.stride, view(k.codes, k.codes_stride, k.exps, k.exps_stride)}; }

}  // namespace

extern "C" uint64_t eden_block_workspace_bytes(uint64_t n)
{
    return std::max(least_workspace(), kStatusBytes + 4 * std::max<uint64_t>(kJoinSums * kMaxSlots * 512 * kTeamWarps, kMaxRuns * n) + 256);
}

extern "C" int eden_block_join(eden_ctx* ctx, const eden_block_join_args* a)
{
    if (!ctx || !a || !half_type(a->type) || !known_norm(a->after) || !known_norm(a->before)) return EDEN_ERR_INVALID_ARG;
    const bool after = a->after.kind != EDEN_NORM_NONE, before = a->before.kind != EDEN_NORM_NONE;
    if (int rc = sizes_ok(a->m, a->n, after || before)) return rc;
    if (!drop_ok(a->drop, a->m) || !std::isfinite(a->scale) || (!a->x && !before)) return EDEN_ERR_INVALID_ARG;
    if (a->m == 0) return EDEN_OK;
    if (!matrix_ok(a->h, a->h_stride, a->n, 2) || !optional_ok(a->residual, a->residual_stride, a->n, 2) || !optional_ok(a->x, a->x_stride, a->n, 2) ||
        (before && !matrix_ok(a->y, a->y_stride, a->n, 2)) || !optional_ok(a->gate, a->gate_per_value ? a->gate_stride : a->n, a->n, 2) ||
        !aligned(a->after_stats, 8) || !aligned(a->before_stats, 8))
        return EDEN_ERR_INVALID_ARG;
    return guarded(ctx, [&]() -> int {
        const uint64_t per_value = gate_stride(a->gate, a->gate_per_value, a->gate_stride);
        const double bytes = 2.0 * a->m * a->n * (1 + (a->residual ? 1 : 0) + (per_value ? 1 : 0) + (a->x ? 1 : 0) + (before ? 1 : 0));
        if (!after && !before) {
            PlainView p{a->h, a->h_stride, a->residual, a->residual_stride, a->gate, per_value, a->x, a->x_stride, {}, a->scale, 0,
                        (uint32_t)a->m, (uint32_t)a->n, (uint32_t)((a->n + 255) / 256)};
            p.drop = drop_view(a->drop, &p.has_drop);
            const bool wide = rows_on_16(p.h, p.h_stride) && rows_on_16(p.residual, p.residual_stride) && (!per_value || rows_on_16(p.gate, per_value)) &&
                              rows_on_16(p.x, p.x_stride);
            const uint64_t rows = wide ? kPlainRows<true> : kPlainRows<false>, blocks = ((a->m + rows - 1) / rows * p.warps_across + kPlainThreads / 32 - 1) / (kPlainThreads / 32);
            if (blocks > kMaxCount) return EDEN_ERR_TOO_LARGE;
            EDEN_DISPATCH_HALF(a->type, return launch(ctx, "t_join_plain", bytes, wide ? k_join_plain<T_, true> : k_join_plain<T_, false>, dim3((uint32_t)blocks),
                                                      kPlainThreads, 0, 1, p));
        }
        JoinView p{per_value ? nullptr : a->gate, a->x, a->x_stride, before ? a->y : nullptr, a->y_stride,
                   {a->after.weight, a->after.bias, a->after_stats, a->after.eps, a->after.kind},
                   {a->before.weight, a->before.bias, a->before_stats, a->before.eps, a->before.kind}, {}, a->scale, 0};
        p.drop = drop_view(a->drop, &p.has_drop);
        Source source[kMaxSources] = {};
        source[kSourceH] = matrix_source(a->h, a->h_stride);
        if (a->residual) source[kSourceResidual] = matrix_source(a->residual, a->residual_stride);
        if (per_value) source[kSourceGate] = matrix_source(a->gate, per_value);
        const bool f = full(a->after) || full(a->before) || per_value;
        const Grid g = grid_of(ctx, a->m, a->n, source, kJoinThreads / 32, f, 0);
        EDEN_DISPATCH_HALF(a->type, EDEN_DISPATCH_NORMS(after, before, return (join<T_, AFTER_, BEFORE_>(ctx, p, g, f, bytes))));
    });
}

extern "C" int eden_block_join_backward(eden_ctx* ctx, const eden_block_join_backward_args* a)
{
    if (!ctx || !a || !half_type(a->type) || !known_norm(a->after) || !known_norm(a->before)) return EDEN_ERR_INVALID_ARG;
    const bool after = a->after.kind != EDEN_NORM_NONE, before = a->before.kind != EDEN_NORM_NONE, vector_gate = a->gate && !a->gate_per_value;
    if (int rc = sizes_ok(a->m, a->n, after || before)) return rc;
    if (!drop_ok(a->drop, a->m) || !std::isfinite(a->scale) || (!a->dx && !before)) return EDEN_ERR_INVALID_ARG;
    float* const sums[kJoinSums] = {a->before_weight_grad, a->before_bias_grad, a->after_weight_grad, a->after_bias_grad, a->gate_sum};
    const bool there[kJoinSums] = {before, before, after, after, vector_gate};
    JoinSumsView out{};
    uint32_t wanted = 0;
    for (int i = 0; i < kJoinSums; ++i)
        if (sums[i]) {
            if (!there[i] || !aligned(sums[i], 4)) return EDEN_ERR_INVALID_ARG;
            out.out[out.sums++] = sums[i];
            wanted |= 1u << i;
        }
    if (a->m > 0) {
        if (!optional_ok(a->dx, a->dx_stride, a->n, 2) || (before && !matrix_ok(a->dy, a->dy_stride, a->n, 2)) || (before && !kept_ok(a->x, a->n)) ||
            ((after || a->gate) && !kept_ok(a->h, a->n)) || !optional_ok(a->gate, a->gate_per_value ? a->gate_stride : a->n, a->n, 2) ||
            !optional_ok(a->d_residual, a->d_residual_stride, a->n, 2) || !optional_ok(a->dh, a->dh_stride, a->n, 2) ||
            !optional_ok(a->d_gate, a->d_gate_stride, a->n, 2) || (a->d_gate && (!a->gate || vector_gate)))
            return EDEN_ERR_INVALID_ARG;
        if ((after && !(a->after_stats && aligned(a->after_stats, 8))) || (before && !(a->before_stats && aligned(a->before_stats, 8)))) return EDEN_ERR_INVALID_ARG;
    }
    return guarded(ctx, [&]() -> int {
        out.n = (uint32_t)a->n;
        out.accumulate = a->accumulate;
        if (a->m > 0 && (wanted || a->d_residual || a->dh || a->d_gate)) {
            const uint64_t per_value = gate_stride(a->gate, a->gate_per_value, a->gate_stride);
            const double bytes = (double)a->m * a->n * (2.0 * (!!a->dx + before + !!per_value + !!a->d_residual + !!a->dh + !!a->d_gate) +
                                                        (before ? (a->x.data ? 2 : 1) : 0) + (after || a->gate ? (a->h.data ? 2 : 1) : 0));
            int has_drop;
            const DropView drop = drop_view(a->drop, &has_drop);
            auto partial = [&](uint64_t parts) {
                out.parts = (uint32_t)parts;
                float* const to = wanted ? Scratch(ctx).take<float>(parts * out.sums * a->n) : nullptr;
                out.partial = to;
                return to;
            };
            int rc = EDEN_OK;
            if (!after && !before) {
                const uint64_t strips = (a->n + 8 * kPlainThreads - 1) / (8 * kPlainThreads);
                const uint64_t want = std::min<uint64_t>(kMaxRuns, std::max<uint64_t>(1, 8ull * ctx->sm_count / strips));
                const uint64_t rows_per_run = std::max<uint64_t>(4, (a->m + want - 1) / want), runs = (a->m + rows_per_run - 1) / rows_per_run;
                PlainBackwardView p{a->dx, a->dx_stride, a->gate ? kept_view(a->h) : KeptView{}, a->gate, per_value, a->d_residual, a->d_residual_stride, a->dh, a->dh_stride,
                                    a->d_gate, a->d_gate_stride, partial(runs), drop, a->scale, has_drop, (uint32_t)a->m, (uint32_t)a->n, (uint32_t)rows_per_run};
                if (wanted && !p.partial) return EDEN_ERR_WORKSPACE;
                const bool wide = rows_on_16(p.dx, p.dx_stride) && rows_on_16(p.h.data, p.h.stride) && (!per_value || rows_on_16(p.gate, per_value)) &&
                                  rows_on_16(p.d_residual, p.d_residual_stride) && rows_on_16(p.dh, p.dh_stride) && rows_on_16(p.d_gate, p.d_gate_stride);
                EDEN_DISPATCH_HALF(a->type, rc = launch(ctx, "t_join_plain_backward", bytes, wide ? k_join_plain_backward<T_, true> : k_join_plain_backward<T_, false>,
                                                        dim3((uint32_t)strips, (uint32_t)runs), kPlainThreads, 0, 1, p));
            } else {
                Source source[kMaxSources] = {};
                auto kept = [&](int at, const eden_kept& k) {
                    if (k.data) {
                        source[at] = matrix_source(k.data, k.stride);
                    } else {
                        source[at] = {(const char*)k.codes, k.codes_stride, 1, 0, 0, 0, aligned(k.codes, 16) && k.codes_stride % 16 == 0};
                        source[at + 1] = {(const char*)k.exps, k.exps_stride, 1, 5, 0, 0, 0};
                        static_assert(kGroup == 1 << 5, "a byte for 2^shift columns");
                    }
                };
                if (a->dx) source[kSourceDx] = matrix_source(a->dx, a->dx_stride);
                if (before) {
                    source[kSourceDy] = matrix_source(a->dy, a->dy_stride);
                    kept(kSourceX, a->x);
                    source[kSourceBefore] = stats_source(a->before_stats);
                }
                if (after || a->gate) kept(kSourceKeptH, a->h);
                if (after) source[kSourceAfter] = stats_source(a->after_stats);
                if (per_value) source[kSourceGateMatrix] = matrix_source(a->gate, per_value);
                const bool f = full(a->after) || full(a->before) || per_value || (wanted & (1u << kBeforeBias | 1u << kAfterBias));
                const Grid g = grid_of(ctx, a->m, a->n, source, kJoinBackwardThreads / 32, f, kJoinSums);
                JoinBackwardView p{per_value ? nullptr : a->gate, a->d_residual, a->d_residual_stride, a->dh, a->dh_stride, a->d_gate, a->d_gate_stride,
                                   partial(g.parts), wanted, {a->after.weight, a->after.bias, nullptr, a->after.eps, a->after.kind},
                                   {a->before.weight, a->before.bias, nullptr, a->before.eps, a->before.kind}, drop, a->scale, has_drop};
                if (wanted && !p.partial) return EDEN_ERR_WORKSPACE;
                EDEN_DISPATCH_HALF(a->type, EDEN_DISPATCH_NORMS(after, before, rc = (join_backward<T_, AFTER_, BEFORE_>(ctx, p, g, f, bytes))));
            }
            if (rc) return rc;
        }
        if (!wanted) return EDEN_OK;
        return launch(ctx, "t_join_sums", 4.0 * (out.parts + 1) * out.sums * (double)a->n, k_join_sums, dim3((uint32_t)((a->n + 31) / 32), out.sums), 256, 0, 1, out);
    });
}
