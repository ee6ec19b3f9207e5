// What the host side of the joins' two directions shares: checks of arguments, the shape of a launch.
#pragma once

#include <atomic>
#include <cmath>

#include "kernels_block.cuh"
#include "train_host.h"

namespace eden {
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

Grid grid_of(const eden_ctx* ctx, uint64_t m, uint64_t n, const Source (&source)[kMaxSources], uint32_t warps, int level, uint32_t sums)
{
    Grid g{};
    BlockShape& s = g.s;
    s.m = (uint32_t)m;
    s.n = (uint32_t)n;
    const uint64_t sms = std::min<uint64_t>(ctx->sm_count, kMaxSlots);
    // Two pieces a thread where that leaves a row for every SM, or where one would need a cluster.
    // (Gradients with the sums of biases do not fit the registers with two: 200 to 600 bytes of spills; with a
    // matrix gate two teams leave room for two rows each: 387 us for 16384 x 4096, against 288.)
    const bool alone = sums && (level == 2 || source[kSourceGateMatrix].base);
    g.pieces = n > 256 * kTeamWarps || (n > 256 && m >= sms && !alone) ? 2 : 1;
    const uint64_t columns = 256ull * kTeamWarps * g.pieces;
    uint32_t vectors = 0;
    for (s.blocks = 1;; s.blocks *= 2) {
        s.warps = (uint32_t)(((n + s.blocks - 1) / s.blocks + 256 * g.pieces - 1) / (256 * g.pieces));
        s.span = s.warps * 256 * g.pieces;
        vectors = (level ? kVectors<true> : kVectors<false>) * s.span * 4;
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

// what a norm asks of the kernels: nothing more, its mean, its bias
int level_of(const eden_norm& n) { return n.kind != EDEN_NORM_NONE && n.bias ? 2 : n.kind == EDEN_NORM_LAYER ? 1 : 0; }

// The launch of the kernel for that level, aligned rows or any, and one or two pieces a thread.
#define EDEN_JOIN_PIECES(kernel, level, w, pieces, ...) \
    ((pieces) == 2 ? launch_rows<kernel<T, AFTER, BEFORE, level, w, 2>>(__VA_ARGS__) : launch_rows<kernel<T, AFTER, BEFORE, level, w, 1>>(__VA_ARGS__))
#define EDEN_JOIN_KERNEL(kernel, level, w, pieces, ...) \
    ((w) ? EDEN_JOIN_PIECES(kernel, level, true, pieces, __VA_ARGS__) : EDEN_JOIN_PIECES(kernel, level, false, pieces, __VA_ARGS__))

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

}  // namespace
}  // namespace eden
