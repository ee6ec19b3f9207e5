// The context behind every entry point of include/eden.h, and the launch macro that counts
// launches and (when profiling is on) brackets them with events.
#pragma once

#include <cstdint>
#include <utility>
#include <vector>

#include <cuda_runtime.h>

#include "../../include/eden.h"

// the smallest workspace that eden_create takes
uint64_t least_workspace();

struct ProfileRecord {
    const char* name;
    double bytes;                    // algorithmic bytes of this launch
    cudaEvent_t start, stop;
};

struct ProfileSummary {
    const char* name;
    uint64_t launches;
    double ms, bytes;
};

struct eden_ctx {
    int device;
    cudaStream_t stream;
    char* ws;
    uint64_t ws_bytes;
    uint64_t launches;
    std::vector<uint32_t> order;     // processing order of the last call: order[j] = client
    uint64_t states_off;             // where the last call put its ClientState array
    bool profiling;
    bool profile_open;               // profile_begin recorded a start event that profile_end must close
    bool force_generic;
    int plan_variant;
    int row_staging;                 // 1: the sender's row pass runs in its persistent, bulk-copy-staged form
    int sel_rounds;                  // 3: the b < 1 mask threshold is found in three histogram rounds at every size
    int sel_band;                    // half-width of the predicted band of the one-pass selection, tenths of a standard deviation
    int sel_ahead;                   // 1: the masks of a call's b < 1 clients are selected on a side stream while the b >= 1 groups run
    cudaStream_t sel_stream;         // that side stream (created on first use)
    std::vector<cudaEvent_t> sel_events;   // fork (0), join (1) and one per b < 1 group (2 + ...)
    int slab_mib;                    // > 0: middle and row pass are launched slab by slab (MiB of intermediate per slab)
    int slab_streams;                // slabs are dealt round-robin to this many streams (1 = the context's own)
    int slab_sides;                  // bit 0: the sender uses the slab order, bit 1: the receiver
    std::vector<cudaStream_t> side;  // side streams of the slab order
    std::vector<cudaEvent_t> slab_events;   // fork (0) and join (1 + stream) events of the slab order
    int linear_form;                 // EDEN_OPT_LINEAR_FORM
    int linear_splits;               // EDEN_OPT_LINEAR_SPLITS
    int cluster_slots[9];            // clusters of 1, 2, 4, 8 blocks that run at once; 0: not asked yet
    int sm_count;
    std::vector<ProfileRecord> records;
    std::vector<std::pair<cudaEvent_t, cudaEvent_t>> event_pool;
    std::vector<ProfileSummary> summary;
    // host-buffer entry points: side streams and events for overlapping copies with kernels
    cudaStream_t copy_in, copy_out;
    std::vector<cudaEvent_t> sync_events;
};

inline void profile_begin(eden_ctx* ctx, const char* name, double bytes)
{
    ctx->profile_open = false;
    if (!ctx->profiling) return;
    ProfileRecord r;
    r.name = name;
    r.bytes = bytes;
    if (ctx->records.size() < ctx->event_pool.size()) {
        r.start = ctx->event_pool[ctx->records.size()].first;
        r.stop = ctx->event_pool[ctx->records.size()].second;
    } else {
        if (cudaEventCreate(&r.start) != cudaSuccess) return;
        if (cudaEventCreate(&r.stop) != cudaSuccess) {
            cudaEventDestroy(r.start);
            return;
        }
        ctx->event_pool.push_back({r.start, r.stop});
    }
    cudaEventRecord(r.start, ctx->stream);
    ctx->records.push_back(r);
    ctx->profile_open = true;
}

inline void profile_end(eden_ctx* ctx)
{
    if (!ctx->profile_open) return;
    cudaEventRecord(ctx->records.back().stop, ctx->stream);
    ctx->profile_open = false;
}

// An error that is returned is taken off the runtime's record, or the next call's launch would
// report it again.
#define CUDA_OK(expr)              \
    do {                           \
        if ((expr) != cudaSuccess) { \
            cudaGetLastError();    \
            return EDEN_ERR_CUDA;  \
        }                          \
    } while (0)

// name and algorithmic bytes feed the optional per-kernel event timing (eden_profile_*)
#define LAUNCH(ctx, name, bytes, kernel, grid, block, smem, ...)             \
    do {                                                                     \
        profile_begin(ctx, name, (double)(bytes));                           \
        kernel<<<grid, block, smem, (ctx)->stream>>>(__VA_ARGS__);           \
        profile_end(ctx);                                                    \
        ++(ctx)->launches;                                                   \
        if (cudaGetLastError() != cudaSuccess) return EDEN_ERR_CUDA;         \
    } while (0)
