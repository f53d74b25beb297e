// Launchers of the routing kernels (include/nimble_moe.h).  Every launcher only enqueues.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace nimble::moe {

// Rows are cut into chunks of equal length, a workgroup each; a chunk is cut further where a
// segment ends inside it.  The part of segment s inside chunk c has number c + s: from one part
// to the next (in row order) either the chunk or the segment goes up, so numbers are distinct,
// and the parts of a segment are neighbours.  Sums are made per part, into scratch memory, and
// added up per segment in the order of the parts.
struct Rows {
    int32_t tokens;
    int32_t chunk;               // rows of a chunk
    int32_t chunks;
    int32_t segments;
    const int32_t *seg_ptr;      // null: one segment of all rows
};

struct RouteArgs {
    Rows rows;
    int32_t experts, top_k;
    uint32_t flags;
    const void *logits;
    int64_t stride;              // in elements
    const float *bias;
    bool bias_runs;              // it is made of runs of four, aligned to their size
    const uint8_t *keep;
    float scale;
    int32_t *index;
    float *weight;
    int32_t *counts, *routed;    // null: no sums
    float *prob_sum;
    float *part_prob;            // [chunks + segments][experts]
    int32_t *part_count;         // [chunks + segments][experts]
    int32_t *part_routed;        // [chunks + segments]
};

struct BackwardArgs {
    Rows rows;
    int32_t experts, top_k;
    uint32_t flags;
    const void *logits;
    int64_t stride;
    const uint8_t *keep;
    float scale;
    const int32_t *index;
    const float *weight, *grad_weight;
    float alpha;
    const int32_t *counts, *routed;
    bool count_runs;             // counts are made of runs of four, aligned to their size
    const float *grad_loss;
    void *grad;
    int64_t grad_stride;
};

struct CountArgs {
    Rows rows;
    int32_t experts, top_k, ranks;
    const int32_t *index, *place;
    int32_t *counts, *rank_tokens;
    int32_t *part;               // [chunks + segments][experts if counts][ranks if rank_tokens]
    int32_t whole;               // segments of up to so many rows are not counted in parts
};

// Rows of a chunk: about `most` chunks, but more where a lane would add up the values of more than `chain` rows
// of one chunk.
int32_t route_chunk(int32_t tokens, int32_t experts, int32_t segments, int32_t most, int32_t chain);
int32_t count_chunk(int32_t tokens, int32_t top_k);

hipError_t launch_route(const RouteArgs &a, int32_t dtype, hipStream_t stream);
hipError_t launch_balance_loss(int32_t segments, int32_t experts, int32_t top_k,
                               const int32_t *counts, const int32_t *routed,
                               const float *prob_sum, float alpha, float *loss,
                               hipStream_t stream);
hipError_t launch_route_backward(const BackwardArgs &a, int32_t dtype, hipStream_t stream);
hipError_t launch_counts(const CountArgs &a, hipStream_t stream);
hipError_t launch_traffic(int32_t batch, int32_t ranks, const int32_t *rank_tokens, double bytes,
                          int32_t n_comm, const int32_t *src, const int32_t *dst, bool way_back,
                          double *traffic, hipStream_t stream);

}  // namespace nimble::moe
