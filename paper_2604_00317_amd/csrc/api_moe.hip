// C ABI of the routing operators: argument checks and scratch layout (include/nimble_moe.h).
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "../../include/nimble_moe.h"
#include "kernels_moe.hpp"
#include "report.hpp"

using nimble::report;

namespace {

namespace moe = nimble::moe;

constexpr int32_t kChunks = 1 << 13, kChunksOfSums = 1 << 9, kChunksOfGradient = 1 << 9;

// Chunks of rows whose probabilities are summed: 512, two workgroups per CU, all of them at work at once, unless that
// makes a lane add up more than 64 rows in binary32 before the parts are added in binary64: sums of 2^28 equal rows
// in 512 chunks were off by 1600 roundings (1e-4); in chains of 64 by 7, and of 600 experts by 16 instead of 128.
constexpr int32_t kChain = 64, kNoSums = NIMBLE_MOE_MAX_TOKENS;

int32_t chunk_of_sums(int32_t tokens, int32_t experts, int32_t n_segments)
{
    return moe::route_chunk(tokens, experts, n_segments, kChunksOfSums, kChain);
}

nimble_status_t bad(const char *what) { return report(NIMBLE_ERR_INVALID, what); }
nimble_status_t too_large(const char *what) { return report(NIMBLE_ERR_RANGE, what); }

nimble_status_t check_sizes(int32_t tokens, int32_t experts, int32_t top_k)
{
    if (tokens < 0) return bad("tokens must be >= 0");
    if (experts < 1) return bad("experts must be >= 1");
    if (top_k < 1) return bad("top_k must be >= 1");
    if (experts > NIMBLE_MOE_MAX_EXPERTS) return too_large("more than 2048 experts");
    if (top_k > NIMBLE_MOE_MAX_TOP_K) return too_large("top_k is more than 16");
    // (row numbers a pass beyond the last one fit 32 bits)
    if (tokens > NIMBLE_MOE_MAX_TOKENS) return too_large("more than 2^31 - 2^16 tokens");
    return NIMBLE_OK;
}

nimble_status_t check_segments(int32_t n_segments, const int32_t *d_seg_ptr)
{
    if (n_segments < 1) return bad("n_segments must be >= 1");
    if (n_segments > NIMBLE_MOE_MAX_SEGMENTS) return too_large("more than 2^20 segments");
    if (!d_seg_ptr && n_segments != 1)
        return bad("d_seg_ptr must not be NULL unless there is one segment");
    return NIMBLE_OK;
}

nimble_status_t check_scratch(const void *d_scratch, int64_t have, int64_t need)
{
    if (need == 0) return NIMBLE_OK;
    if (!d_scratch) return bad("d_scratch must not be NULL");
    if (reinterpret_cast<uintptr_t>(d_scratch) % 16 != 0) return bad("d_scratch must be aligned to 16 bytes");
    if (have < need) return bad("scratch_bytes is less than the call needs");
    return NIMBLE_OK;
}

moe::Rows rows_of(int32_t tokens, int32_t chunk, int32_t n_segments, const int32_t *d_seg_ptr)
{
    const int64_t chunks = (static_cast<int64_t>(tokens) + chunk - 1) / chunk;
    return {tokens, chunk, static_cast<int32_t>(chunks), n_segments, d_seg_ptr};
}

int64_t round16(int64_t n) { return (n + 15) / 16 * 16; }

// Parts of the rows, and bytes of an array with `words` words per part.
int64_t part_bytes(int32_t tokens, int32_t chunk, int32_t n_segments, int64_t words)
{
    const int64_t chunks = (static_cast<int64_t>(tokens) + chunk - 1) / chunk;
    return round16((chunks + n_segments) * words * 4);
}

nimble_status_t check_route(uint32_t flags, int32_t dtype, int32_t experts, int32_t top_k,
                            int64_t row_stride, float scale)
{
    if ((flags & ~static_cast<uint32_t>(NIMBLE_MOE_SIGMOID | NIMBLE_MOE_RENORM)) != 0)
        return bad("unknown flag");
    if (dtype != NIMBLE_F32 && dtype != NIMBLE_F16 && dtype != NIMBLE_BF16) return bad("unknown dtype");
    if (top_k > experts) return bad("top_k is more than the number of experts");
    if (row_stride < experts) return bad("row_stride is less than the number of experts");
    if (!(scale > 0.0f) || !std::isnormal(scale)) return bad("scale must be finite, > 0 and no denormal number");
    return NIMBLE_OK;
}

}  // namespace

int64_t nimble_moe_route_scratch_bytes(int32_t tokens, int32_t experts, int32_t n_segments)
{
    if (tokens < 0 || tokens > NIMBLE_MOE_MAX_TOKENS || experts < 1 || experts > NIMBLE_MOE_MAX_EXPERTS ||
        n_segments < 1 || n_segments > NIMBLE_MOE_MAX_SEGMENTS)
        return -1;
    const int32_t chunk = chunk_of_sums(tokens, experts, n_segments);
    return 2 * part_bytes(tokens, chunk, n_segments, experts) + part_bytes(tokens, chunk, n_segments, 1);
}

nimble_status_t nimble_moe_route(int32_t tokens, int32_t experts, int32_t top_k, uint32_t flags,
                                 int32_t dtype, const void *d_logits, int64_t row_stride,
                                 const float *d_bias, const uint8_t *d_keep, float scale,
                                 int32_t n_segments, const int32_t *d_seg_ptr, int32_t *d_index,
                                 float *d_weight, int32_t *d_counts, int32_t *d_routed,
                                 float *d_prob_sum, void *d_scratch, int64_t scratch_bytes,
                                 void *hip_stream)
{
    nimble::report_clear();
    nimble_status_t st = check_sizes(tokens, experts, top_k);
    if (st == NIMBLE_OK) st = check_route(flags, dtype, experts, top_k, row_stride, scale);
    if (st == NIMBLE_OK) st = check_segments(n_segments, d_seg_ptr);
    if (st != NIMBLE_OK) return st;
    if (tokens > 0 && (!d_logits || !d_index || !d_weight))
        return bad("logits, index and weight pointers must not be NULL");
    const bool sums = d_counts || d_routed || d_prob_sum;
    if (sums && !(d_counts && d_routed && d_prob_sum))
        return bad("counts, routed and prob_sum are wanted together or not at all");
    const int32_t chunk = sums ? chunk_of_sums(tokens, experts, n_segments)
                               : moe::route_chunk(tokens, experts, n_segments, kChunks, kNoSums);
    moe::RouteArgs a{};
    a.rows = rows_of(tokens, chunk, n_segments, d_seg_ptr);
    if (sums) {
        st = check_scratch(d_scratch, scratch_bytes,
                           nimble_moe_route_scratch_bytes(tokens, experts, n_segments));
        if (st != NIMBLE_OK) return st;
        const int64_t bytes = part_bytes(tokens, chunk, n_segments, experts);
        auto *p = static_cast<unsigned char *>(d_scratch);
        a.part_prob = reinterpret_cast<float *>(p);
        a.part_count = reinterpret_cast<int32_t *>(p + bytes);
        a.part_routed = reinterpret_cast<int32_t *>(p + 2 * bytes);
    }
    a.experts = experts;
    a.top_k = top_k;
    a.flags = flags;
    a.logits = d_logits;
    a.stride = row_stride;
    a.bias = d_bias;
    a.bias_runs = reinterpret_cast<uintptr_t>(d_bias) % 16 == 0 && experts % 4 == 0;
    a.keep = d_keep;
    a.scale = scale;
    a.index = d_index;
    a.weight = d_weight;
    a.counts = d_counts;
    a.routed = d_routed;
    a.prob_sum = d_prob_sum;
    const hipError_t e = moe::launch_route(a, dtype, static_cast<hipStream_t>(hip_stream));
    if (e != hipSuccess) return nimble::report_hip(e, "kernel launch (routing)");
    return NIMBLE_OK;
}

nimble_status_t nimble_moe_balance_loss(int32_t n_segments, int32_t experts, int32_t top_k,
                                        const int32_t *d_counts, const int32_t *d_routed,
                                        const float *d_prob_sum, float alpha, float *d_loss,
                                        void *hip_stream)
{
    nimble::report_clear();
    nimble_status_t st = check_sizes(0, experts, top_k);
    if (st != NIMBLE_OK) return st;
    if (top_k > experts) return bad("top_k is more than the number of experts");
    if (n_segments < 1) return bad("n_segments must be >= 1");
    if (n_segments > NIMBLE_MOE_MAX_SEGMENTS) return too_large("more than 2^20 segments");
    if (!d_counts || !d_routed || !d_prob_sum || !d_loss)
        return bad("counts, routed, prob_sum and loss pointers must not be NULL");
    if (!std::isfinite(alpha)) return bad("alpha must be finite");
    const hipError_t e = moe::launch_balance_loss(n_segments, experts, top_k, d_counts, d_routed,
                                                  d_prob_sum, alpha, d_loss,
                                                  static_cast<hipStream_t>(hip_stream));
    if (e != hipSuccess) return nimble::report_hip(e, "kernel launch (balance loss)");
    return NIMBLE_OK;
}

nimble_status_t nimble_moe_route_backward(int32_t tokens, int32_t experts, int32_t top_k,
                                          uint32_t flags, int32_t dtype, const void *d_logits,
                                          int64_t row_stride, const uint8_t *d_keep, float scale,
                                          int32_t n_segments, const int32_t *d_seg_ptr,
                                          const int32_t *d_index, const float *d_weight,
                                          const float *d_grad_weight, float alpha,
                                          const int32_t *d_counts, const int32_t *d_routed,
                                          const float *d_grad_loss, void *d_grad_logits,
                                          int64_t grad_stride, void *hip_stream)
{
    nimble::report_clear();
    nimble_status_t st = check_sizes(tokens, experts, top_k);
    if (st == NIMBLE_OK) st = check_route(flags, dtype, experts, top_k, row_stride, scale);
    if (st == NIMBLE_OK) st = check_segments(n_segments, d_seg_ptr);
    if (st != NIMBLE_OK) return st;
    if (grad_stride < experts) return bad("grad_stride is less than the number of experts");
    if (tokens > 0 && (!d_logits || !d_index || !d_weight || !d_grad_logits))
        return bad("logits, index, weight and gradient pointers must not be NULL");
    if ((d_counts || d_routed || d_grad_loss) && !(d_counts && d_routed && d_grad_loss))
        return bad("counts, routed and grad_loss are given together or not at all");
    if (!std::isfinite(alpha)) return bad("alpha must be finite");
    moe::BackwardArgs a{};
    a.rows = rows_of(tokens, moe::route_chunk(tokens, experts, n_segments, kChunksOfGradient, kNoSums), n_segments,
                     d_seg_ptr);
    a.experts = experts;
    a.top_k = top_k;
    a.flags = flags;
    a.logits = d_logits;
    a.stride = row_stride;
    a.keep = d_keep;
    a.scale = scale;
    a.index = d_index;
    a.weight = d_weight;
    a.grad_weight = d_grad_weight;
    a.alpha = alpha;
    a.counts = d_counts;
    a.routed = d_routed;
    a.count_runs = reinterpret_cast<uintptr_t>(d_counts) % 16 == 0 && experts % 4 == 0;
    a.grad_loss = d_grad_loss;
    a.grad = d_grad_logits;
    a.grad_stride = grad_stride;
    const hipError_t e = moe::launch_route_backward(a, dtype, static_cast<hipStream_t>(hip_stream));
    if (e != hipSuccess) return nimble::report_hip(e, "kernel launch (gradient of the routing)");
    return NIMBLE_OK;
}

// n_ranks = 0: no rank tokens are counted (the scratch memory has room for the counts all the same).
int64_t nimble_moe_counts_scratch_bytes(int32_t tokens, int32_t top_k, int32_t experts,
                                        int32_t n_ranks, int32_t n_segments)
{
    if (tokens < 0 || tokens > NIMBLE_MOE_MAX_TOKENS || top_k < 1 || top_k > NIMBLE_MOE_MAX_TOP_K || experts < 1 ||
        experts > NIMBLE_MOE_MAX_EXPERTS || n_ranks < 0 || n_ranks > NIMBLE_MOE_MAX_RANKS ||
        n_segments < 1 || n_segments > NIMBLE_MOE_MAX_SEGMENTS)
        return -1;
    return part_bytes(tokens, moe::count_chunk(tokens, top_k), n_segments,
                      static_cast<int64_t>(experts) + n_ranks);
}

nimble_status_t nimble_moe_counts(int32_t tokens, int32_t top_k, const int32_t *d_index,
                                  int32_t experts, int32_t n_segments, const int32_t *d_seg_ptr,
                                  const int32_t *d_expert_rank, int32_t n_ranks,
                                  int32_t *d_counts, int32_t *d_rank_tokens, void *d_scratch,
                                  int64_t scratch_bytes, void *hip_stream)
{
    nimble::report_clear();
    nimble_status_t st = check_sizes(tokens, experts, top_k);
    if (st == NIMBLE_OK) st = check_segments(n_segments, d_seg_ptr);
    if (st != NIMBLE_OK) return st;
    if (tokens > 0 && !d_index) return bad("index pointer must not be NULL");
    if (!d_counts && !d_rank_tokens) return bad("counts and rank_tokens are both NULL");
    if (n_ranks < 0) return bad("n_ranks must be >= 0");
    if (n_ranks > NIMBLE_MOE_MAX_RANKS) return too_large("more than 4096 ranks");
    if (d_rank_tokens && (n_ranks < 1 || !d_expert_rank))
        return bad("rank_tokens need n_ranks >= 1 and expert_rank");
    st = check_scratch(d_scratch, scratch_bytes,
                       nimble_moe_counts_scratch_bytes(tokens, top_k, experts,
                                                       d_rank_tokens ? n_ranks : 0, n_segments));
    if (st != NIMBLE_OK) return st;
    moe::CountArgs a{};
    a.rows = rows_of(tokens, moe::count_chunk(tokens, top_k), n_segments, d_seg_ptr);
    a.experts = experts;
    a.top_k = top_k;
    a.ranks = n_ranks;
    a.index = d_index;
    a.place = d_expert_rank;
    a.counts = d_counts;
    a.rank_tokens = d_rank_tokens;
    a.part = static_cast<int32_t *>(d_scratch);
    const hipError_t e = moe::launch_counts(a, static_cast<hipStream_t>(hip_stream));
    if (e != hipSuccess) return nimble::report_hip(e, "kernel launch (counts of routed tokens)");
    return NIMBLE_OK;
}

nimble_status_t nimble_moe_traffic(int32_t batch, int32_t n_ranks, const int32_t *d_rank_tokens,
                                   double bytes_per_token, int32_t n_comm, const int32_t *d_src,
                                   const int32_t *d_dst, uint32_t flags, double *d_traffic,
                                   void *hip_stream)
{
    nimble::report_clear();
    if (batch < 1) return bad("batch must be >= 1");
    if (n_ranks < 1) return bad("n_ranks must be >= 1");
    if (n_comm < 1) return bad("n_comm must be >= 1");
    if (n_ranks > NIMBLE_MOE_MAX_RANKS) return too_large("more than 4096 ranks");
    if (static_cast<int64_t>(batch) * n_comm >= (1LL << 31)) return too_large("2^31 demands or more");
    if ((flags & ~static_cast<uint32_t>(NIMBLE_MOE_WAY_BACK)) != 0) return bad("unknown flag");
    if (!d_rank_tokens || !d_traffic) return bad("rank_tokens and traffic pointers must not be NULL");
    if ((d_src == nullptr) != (d_dst == nullptr)) return bad("src and dst are given together or not at all");
    if (!d_src && static_cast<int64_t>(n_comm) != static_cast<int64_t>(n_ranks) * (n_ranks - 1))
        return bad("without src and dst n_comm must be n_ranks * (n_ranks - 1)");
    if (!(bytes_per_token >= 0.0) || !std::isfinite(bytes_per_token))
        return bad("bytes_per_token must be finite and >= 0");
    const hipError_t e = moe::launch_traffic(batch, n_ranks, d_rank_tokens, bytes_per_token, n_comm, d_src,
                                             d_dst, (flags & NIMBLE_MOE_WAY_BACK) != 0, d_traffic,
                                             static_cast<hipStream_t>(hip_stream));
    if (e != hipSuccess) return nimble::report_hip(e, "kernel launch (demand of routed tokens)");
    return NIMBLE_OK;
}
