// C ABI of what joins a client's blocks (declared in include/eden.h): argument checks and launches.
// The backward pass is a file of its own, so that both compile side by side.
#include "block_host.h"

using namespace eden;

namespace {

template <typename T, bool AFTER, bool BEFORE>
int join(eden_ctx* ctx, const JoinView& p, const Grid& g, int level, double bytes)
{
    const bool wide = g.wide && rows_on_16(p.x, p.x_stride) && rows_on_16(p.y, p.y_stride);
    return level ? EDEN_JOIN_KERNEL(k_join, true, wide, g.pieces, ctx, "t_join", bytes, p, g) : EDEN_JOIN_KERNEL(k_join, false, wide, g.pieces, ctx, "t_join", bytes, p, g);
}

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
            // (rows that end inside a chunk are not stored in chunks: what lies behind them is not the call's)
            const bool wide = a->n % 8 == 0 && rows_on_16(p.h, p.h_stride) && rows_on_16(p.residual, p.residual_stride) && (!per_value || rows_on_16(p.gate, per_value)) &&
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
        const int level = std::max({level_of(a->after), level_of(a->before), per_value ? 1 : 0});
        const Grid g = grid_of(ctx, a->m, a->n, source, kJoinThreads / 32, level, 0);
        EDEN_DISPATCH_HALF(a->type, EDEN_DISPATCH_NORMS(after, before, return (join<T_, AFTER_, BEFORE_>(ctx, p, g, level, bytes))));
    });
}
