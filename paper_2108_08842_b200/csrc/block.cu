// C ABI of what joins a client's blocks (declared in include/eden.h): argument checks, workspace
// carving and launches.
#include <cmath>

#include "kernels_block.cuh"
#include "train_host.h"

using namespace eden;

namespace {

constexpr uint64_t kMaxSlots = 192;             // blocks of a backward launch, whatever the device
constexpr uint64_t kMaxNormColumns = (uint64_t)kBlockColumns * kBlockCluster;
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

// Rows over teams, blocks and clusters: see kernels_block.cuh.
struct Grid {
    BlockShape s;
    dim3 grid;
    uint32_t threads, cluster, parts;
};

Grid grid_of(uint64_t m, uint64_t n, bool sums, uint64_t slots)
{
    Grid g;
    uint32_t blocks = 1;
    while ((uint64_t)blocks * kBlockColumns < n && blocks < (sums ? (uint32_t)kBlockCluster : 1u << 30)) blocks *= 2;
    if (!sums) blocks = (uint32_t)((n + kBlockColumns - 1) / kBlockColumns);
    g.s.m = (uint32_t)m;
    g.s.n = (uint32_t)n;
    g.s.warps = (uint32_t)(((n + blocks - 1) / blocks + 255) / 256);
    g.s.teams = kBlockWarps / g.s.warps;
    g.s.span = g.s.warps * 256;
    g.s.blocks = sums ? blocks : 1;
    const uint32_t strips = sums ? 1 : (uint32_t)((n + g.s.span - 1) / g.s.span);
    const uint64_t want = (m + g.s.teams - 1) / g.s.teams, most = std::max<uint64_t>(1, slots / blocks);
    const uint32_t groups = (uint32_t)std::min(want, most);
    g.grid = dim3(groups * g.s.blocks, strips);
    g.threads = g.s.teams * g.s.warps * 32;
    g.cluster = g.s.blocks;
    g.parts = groups * g.s.teams;
    return g;
}

uint64_t slots_of(const eden_ctx* ctx) { return std::min<uint64_t>(ctx->sm_count, kMaxSlots); }

template <typename T, bool AFTER, bool BEFORE>
int join(eden_ctx* ctx, const JoinView& p, const Grid& g, double bytes)
{
    const bool wide = rows_on_16(p.h, p.h_stride) && rows_on_16(p.residual, p.residual_stride) && rows_on_16(p.gate_stride ? p.gate : nullptr, p.gate_stride) &&
                      rows_on_16(p.x, p.x_stride) && rows_on_16(p.y, p.y_stride);
    return launch(ctx, "t_join", bytes, wide ? k_join<T, true, AFTER, BEFORE> : k_join<T, false, AFTER, BEFORE>, g.grid, g.threads, 0, g.cluster, p, g.s);
}

bool kept_wide(const KeptView& k)
{
    return k.data ? rows_on_16(k.data, k.stride) : aligned(k.held.codes, 8) && k.held.codes_stride % 8 == 0;
}

template <typename T, bool AFTER, bool BEFORE>
int join_backward(eden_ctx* ctx, const JoinBackwardView& p, const Grid& g, double bytes)
{
    const bool wide = rows_on_16(p.dx, p.dx_stride) && rows_on_16(p.dy, p.dy_stride) && rows_on_16(p.gate_stride ? p.gate : nullptr, p.gate_stride) &&
                      rows_on_16(p.d_residual, p.d_residual_stride) && rows_on_16(p.dh, p.dh_stride) && rows_on_16(p.d_gate, p.d_gate_stride) &&
                      kept_wide(p.h) && kept_wide(p.x);
    return launch(ctx, "t_join_backward", bytes, wide ? k_join_backward<T, true, AFTER, BEFORE> : k_join_backward<T, false, AFTER, BEFORE>, g.grid, g.threads,
                  0, g.cluster, p, g.s);
}

#define EDEN_DISPATCH_NORMS(after, before, CALL)                                                   \
    if (after) {                                                                                  \
        if (before) { constexpr bool AFTER_ = true, BEFORE_ = true; CALL; }                       \
        else { constexpr bool AFTER_ = true, BEFORE_ = false; CALL; }                             \
    } else {                                                                                      \
        if (before) { constexpr bool AFTER_ = false, BEFORE_ = true; CALL; }                      \
        else { constexpr bool AFTER_ = false, BEFORE_ = false; CALL; }                            \
    }

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
    return std::max(least_workspace(), kStatusBytes + kJoinSums * 4 * std::max<uint64_t>(kMaxSlots * kBlockColumns, n) + 256);
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
        JoinView p{a->h, a->h_stride, a->residual, a->residual_stride, a->gate, gate_stride(a->gate, a->gate_per_value, a->gate_stride), a->x, a->x_stride,
                   before ? a->y : nullptr, a->y_stride, {a->after.weight, a->after.bias, a->after_stats, a->after.eps, a->after.kind},
                   {a->before.weight, a->before.bias, a->before_stats, a->before.eps, a->before.kind}, {}, a->scale, 0};
        p.drop = drop_view(a->drop, &p.has_drop);
        const Grid g = grid_of(a->m, a->n, after || before, 2 * (uint64_t)ctx->sm_count);
        const double bytes = 2.0 * a->m * a->n * (1 + (a->residual ? 1 : 0) + (p.gate_stride ? 1 : 0) + (a->x ? 1 : 0) + (before ? 1 : 0));
        EDEN_DISPATCH_HALF(a->type, EDEN_DISPATCH_NORMS(after, before, return (join<T_, AFTER_, BEFORE_>(ctx, p, g, bytes))));
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
            JoinBackwardView p{};
            p.dx = a->dx; p.dx_stride = a->dx_stride;
            if (before) p.dy = a->dy, p.dy_stride = a->dy_stride, p.x = kept_view(a->x);
            if (after || a->gate) p.h = kept_view(a->h);
            p.gate = a->gate; p.gate_stride = gate_stride(a->gate, a->gate_per_value, a->gate_stride);
            p.d_residual = a->d_residual; p.d_residual_stride = a->d_residual_stride;
            p.dh = a->dh; p.dh_stride = a->dh_stride;
            p.d_gate = a->d_gate; p.d_gate_stride = a->d_gate_stride;
            p.after = {a->after.weight, a->after.bias, const_cast<float*>(a->after_stats), a->after.eps, a->after.kind};
            p.before = {a->before.weight, a->before.bias, const_cast<float*>(a->before_stats), a->before.eps, a->before.kind};
            p.drop = drop_view(a->drop, &p.has_drop);
            p.scale = a->scale;
            p.wanted = wanted;
            const Grid g = grid_of(a->m, a->n, after || before, slots_of(ctx));
            if (wanted) {
                out.parts = g.parts;
                p.partial = Scratch(ctx).take<float>((uint64_t)g.parts * out.sums * a->n);
                if (!p.partial) return EDEN_ERR_WORKSPACE;
                out.partial = p.partial;
            }
            const double each = (double)a->m * a->n;
            const double bytes = each * (2.0 * (!!a->dx + before + !!p.gate_stride + !!a->d_residual + !!a->dh + !!a->d_gate) +
                                         (before ? (a->x.data ? 2 : 1) : 0) + (after || a->gate ? (a->h.data ? 2 : 1) : 0));
            int rc = EDEN_OK;
            EDEN_DISPATCH_HALF(a->type, EDEN_DISPATCH_NORMS(after, before, rc = (join_backward<T_, AFTER_, BEFORE_>(ctx, p, g, bytes))));
            if (rc) return rc;
        }
        if (!wanted) return EDEN_OK;
        return launch(ctx, "t_join_sums", 4.0 * (out.parts + 1) * out.sums * (double)a->n, k_join_sums, dim3((uint32_t)((a->n + 31) / 32), out.sums), 256, 0, 1, out);
    });
}
