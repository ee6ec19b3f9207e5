// The backward pass of what joins a client's blocks: argument checks, workspace carving and launches.
#include "block_host.h"

using namespace eden;

namespace {

template <typename T, bool AFTER, bool BEFORE>
int join_backward(eden_ctx* ctx, const JoinBackwardView& p, const Grid& g, int level, double bytes)
{
    const bool wide = g.wide && rows_on_16(p.d_residual, p.d_residual_stride) && rows_on_16(p.dh, p.dh_stride) && rows_on_16(p.d_gate, p.d_gate_stride);
    switch (level) {
        case 0: return EDEN_JOIN_KERNEL(k_join_backward, 0, wide, g.pieces, ctx, "t_join_backward", bytes, p, g);
        case 1: return EDEN_JOIN_KERNEL(k_join_backward, 1, wide, g.pieces, ctx, "t_join_backward", bytes, p, g);
        default: return EDEN_JOIN_KERNEL(k_join_backward, 2, wide, g.pieces, ctx, "t_join_backward", bytes, p, g);
    }
}

bool kept_ok(const eden_kept& k, uint64_t n)
{
    return k.data ? matrix_ok(k.data, k.stride, n, 2) : checkpoint_ok(k.codes, k.codes_stride, k.exps, k.exps_stride, n);
}

KeptView kept_view(const eden_kept& k) { return {k.data, k.stride, view(k.codes, k.codes_stride, k.exps, k.exps_stride)}; }

}  // namespace

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
                const bool wide = a->n % 8 == 0 && rows_on_16(p.dx, p.dx_stride) && rows_on_16(p.h.data, p.h.stride) && (!per_value || rows_on_16(p.gate, per_value)) &&
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
                const int level = std::max({level_of(a->after), level_of(a->before), per_value ? 1 : 0, wanted & (1u << kBeforeBias | 1u << kAfterBias) ? 2 : 0});
                const Grid g = grid_of(ctx, a->m, a->n, source, kJoinBackwardThreads / 32, level, kJoinSums);
                JoinBackwardView p{per_value ? nullptr : a->gate, a->d_residual, a->d_residual_stride, a->dh, a->dh_stride, a->d_gate, a->d_gate_stride,
                                   partial(g.parts), wanted, {a->after.weight, a->after.bias, nullptr, a->after.eps, a->after.kind},
                                   {a->before.weight, a->before.bias, nullptr, a->before.eps, a->before.kind}, drop, a->scale, has_drop};
                if (wanted && !p.partial) return EDEN_ERR_WORKSPACE;
                EDEN_DISPATCH_HALF(a->type, EDEN_DISPATCH_NORMS(after, before, rc = (join_backward<T_, AFTER_, BEFORE_>(ctx, p, g, level, bytes))));
            }
            if (rc) return rc;
        }
        if (!wanted) return EDEN_OK;
        return launch(ctx, "t_join_sums", 4.0 * (out.parts + 1) * out.sums * (double)a->n, k_join_sums, dim3((uint32_t)((a->n + 31) / 32), out.sums), 256, 0, 1, out);
    });
}
