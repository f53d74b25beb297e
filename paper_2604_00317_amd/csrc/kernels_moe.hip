// Routing kernels that work on sums and indices: end of the sums, balance loss, counts per expert and
// destination GPU, demand vectors (definitions in include/nimble_moe.h), and the launchers.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "kernels_moe.hpp"
#include "moe_device.hpp"

namespace nimble::moe {

// one per element type, kernels_moe_*.hip
hipError_t route_f32(const RouteArgs &a, hipStream_t stream);
hipError_t route_f16(const RouteArgs &a, hipStream_t stream);
hipError_t route_bf16(const RouteArgs &a, hipStream_t stream);
hipError_t backward_f32(const BackwardArgs &a, hipStream_t stream);
hipError_t backward_f16(const BackwardArgs &a, hipStream_t stream);
hipError_t backward_bf16(const BackwardArgs &a, hipStream_t stream);

namespace {

constexpr int kFinishWaves = 16;

// The parts of a segment, 64 columns per workgroup: every wave adds each 16th part, in double.
__global__ __launch_bounds__(kFinishWaves *kWave) void k_route_finish(RouteArgs a)
{
    __shared__ double sums[kFinishWaves][kWave];
    __shared__ int hits[kFinishWaves][kWave];
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int s = blockIdx.x;
    const int col = blockIdx.y * kWave + lane;
    const int lo = begin_of(a.rows, s), hi = end_of(a.rows, s);
    const int64_t p0 = static_cast<int64_t>(lo / a.rows.chunk) + s;
    const int64_t p1 = lo < hi ? static_cast<int64_t>((hi - 1) / a.rows.chunk) + s : p0 - 1;
    double t = 0.0;
    int n = 0;
    if (col < a.experts) {
#pragma unroll 4
        for (int64_t p = p0 + wave; p <= p1; p += kFinishWaves) {
            t = t + static_cast<double>(a.part_prob[p * a.experts + col]);
            n += a.part_count[p * a.experts + col];
        }
    }
    sums[wave][lane] = t;
    hits[wave][lane] = n;
    __syncthreads();
    if (wave == 0 && col < a.experts) {
        for (int w = 1; w < kFinishWaves; ++w) {
            t = t + sums[w][lane];
            n += hits[w][lane];
        }
        a.prob_sum[static_cast<int64_t>(s) * a.experts + col] = static_cast<float>(t);
        a.counts[static_cast<int64_t>(s) * a.experts + col] = n;
    }
    if (blockIdx.y == 0) {
        int m = 0;
        for (int64_t p = p0 + threadIdx.x; p <= p1; p += kFinishWaves * kWave) m += a.part_routed[p];
        __syncthreads();
        hits[wave][lane] = m;
        __syncthreads();
        if (wave == 0) {
            for (int w = 1; w < kFinishWaves; ++w) m += hits[w][lane];
            for (int step = 1; step < kWave; step *= 2) m += __shfl_xor(m, step, kWave);
            if (lane == 0) a.routed[s] = m;
        }
    }
}

// ---- loss ------------------------------------------------------------------------------------

__global__ __launch_bounds__(256) void k_balance_loss(int experts, double unit, const int32_t *counts,
                                                      const int32_t *routed, const float *prob_sum,
                                                      float *loss)
{
    __shared__ double part[4];
    const int64_t at = static_cast<int64_t>(blockIdx.x) * experts;
    double t = 0.0;
    for (int e = threadIdx.x; e < experts; e += 256)
        t = t + static_cast<double>(counts[at + e]) * static_cast<double>(prob_sum[at + e]);
    for (int step = 1; step < kWave; step *= 2) t = t + __shfl_xor(t, step, kWave);
    if ((threadIdx.x & (kWave - 1)) == 0) part[threadIdx.x / kWave] = t;
    __syncthreads();
    if (threadIdx.x == 0) {
        const double n = static_cast<double>(routed[blockIdx.x]);
        t = ((part[0] + part[1]) + part[2]) + part[3];
        loss[blockIdx.x] = routed[blockIdx.x] == 0 ? 0.0f : static_cast<float>(unit * t / (n * n));
    }
}

// ---- counts and demand -----------------------------------------------------------------------

constexpr int kCountBlock = 512;

__global__ __launch_bounds__(kCountBlock) void k_counts(CountArgs a)
{
    extern __shared__ int lds[];
    const int E = a.experts, M = (a.counts ? E : 0) + (a.rank_tokens ? a.ranks : 0);
    int *bins = lds;                                 // experts, then ranks
    int *by_rank = bins + (a.counts ? E : 0);
    int *place = lds + M;
    const int lane = threadIdx.x & (kWave - 1);
    const int64_t first = static_cast<int64_t>(blockIdx.x) * a.rows.chunk;
    const int lo = static_cast<int>(first);
    const int hi = static_cast<int>(min(first + a.rows.chunk, static_cast<int64_t>(a.rows.tokens)));
    if (a.rank_tokens)
        for (int e = threadIdx.x; e < E; e += kCountBlock) place[e] = a.place[e];
    for (int s = first_segment(a.rows, lo, lane); s < a.rows.segments; ++s) {
        if (begin_of(a.rows, s) >= hi) break;
        const int from = max(lo, begin_of(a.rows, s)), to = min(hi, end_of(a.rows, s));
        if (from >= to) continue;
        for (int c = threadIdx.x; c < M; c += kCountBlock) bins[c] = 0;
        __syncthreads();
        for (int row = from + threadIdx.x; row < to; row += kCountBlock) {
            const int32_t *idx = a.index + static_cast<int64_t>(row) * a.top_k;
            int to_rank[NIMBLE_MOE_MAX_TOP_K];
#pragma unroll
            for (int j = 0; j < NIMBLE_MOE_MAX_TOP_K; ++j) {
                to_rank[j] = -1;
                if (j < a.top_k) {
                    const int e = idx[j];
                    const bool there = static_cast<uint32_t>(e) < static_cast<uint32_t>(E);
                    if (there && a.counts) atomicAdd(&bins[e], 1);
                    if (there && a.rank_tokens) {
                        const int r = place[e];
                        bool fresh = static_cast<uint32_t>(r) < static_cast<uint32_t>(a.ranks);
#pragma unroll
                        for (int i = 0; i < j; ++i) fresh = fresh && to_rank[i] != r;
                        if (fresh) {
                            to_rank[j] = r;
                            atomicAdd(&by_rank[r], 1);
                        }
                    }
                }
            }
        }
        __syncthreads();
        const int64_t part = static_cast<int64_t>(blockIdx.x) + s;
        for (int c = threadIdx.x; c < M; c += kCountBlock) a.part[part * M + c] = bins[c];
        __syncthreads();
    }
}

__global__ __launch_bounds__(kFinishWaves *kWave) void k_counts_finish(CountArgs a)
{
    __shared__ int hits[kFinishWaves][kWave];
    const int E = a.counts ? a.experts : 0, M = E + (a.rank_tokens ? a.ranks : 0);
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int s = blockIdx.x;
    const int col = blockIdx.y * kWave + lane;
    const int lo = begin_of(a.rows, s), hi = end_of(a.rows, s);
    const int64_t p0 = static_cast<int64_t>(lo / a.rows.chunk) + s;
    const int64_t p1 = lo < hi ? static_cast<int64_t>((hi - 1) / a.rows.chunk) + s : p0 - 1;
    int n = 0;
    if (col < M) {
#pragma unroll 4
        for (int64_t p = p0 + wave; p <= p1; p += kFinishWaves) n += a.part[p * M + col];
    }
    hits[wave][lane] = n;
    __syncthreads();
    if (wave != 0 || col >= M) return;
    for (int w = 1; w < kFinishWaves; ++w) n += hits[w][lane];
    if (col < E) a.counts[static_cast<int64_t>(s) * E + col] = n;
    else a.rank_tokens[static_cast<int64_t>(s) * a.ranks + col - E] = n;
}

__global__ __launch_bounds__(256) void k_traffic(int64_t total, int ranks, const int32_t *tokens,
                                                 double bytes, int n_comm, const int32_t *src,
                                                 const int32_t *dst, bool way_back, double *traffic)
{
    const int64_t at = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (at >= total) return;
    const int64_t b = at / n_comm;
    const int k = static_cast<int>(at - b * n_comm);
    int r, q;
    if (src) {
        r = src[k];
        q = dst[k];
    } else {
        r = k / (ranks - 1);
        q = k - r * (ranks - 1);
        q += q >= r ? 1 : 0;
    }
    const uint32_t n = static_cast<uint32_t>(ranks);
    double v = __builtin_nan("");
    if (static_cast<uint32_t>(r) < n && static_cast<uint32_t>(q) < n) {
        const int64_t cell = way_back ? static_cast<int64_t>(q) * ranks + r
                                      : static_cast<int64_t>(r) * ranks + q;
        v = static_cast<double>(tokens[b * ranks * ranks + cell]) * bytes;
    }
    traffic[at] = v;
}

}  // namespace

// Whole passes of a workgroup's rows, and no more than 1024 chunks with sums to add up: about four
// workgroups per CU.
int32_t route_chunk(int32_t tokens, int32_t experts, bool sums)
{
    const int32_t pass = kRowWaves * (experts <= 256 ? 4 : experts <= 512 ? 2 : 1);
    const int32_t most = sums ? 1 << 10 : 1 << 20;
    const int64_t rows = (static_cast<int64_t>(tokens) + most - 1) / most;
    return static_cast<int32_t>((std::max<int64_t>(rows, 1) + pass - 1) / pass * pass);
}

int32_t count_chunk(int32_t tokens, int32_t)
{
    return std::max(kCountBlock, (tokens + 1023) / 1024);
}

hipError_t launch_route(const RouteArgs &a, int32_t dtype, hipStream_t stream)
{
    if (a.rows.chunks > 0) {
        const hipError_t e = dtype == NIMBLE_F32   ? route_f32(a, stream)
                             : dtype == NIMBLE_F16 ? route_f16(a, stream)
                                                   : route_bf16(a, stream);
        if (e != hipSuccess || !a.counts) return e;
    }
    if (!a.counts) return hipSuccess;
    k_route_finish<<<dim3(a.rows.segments, (a.experts + kWave - 1) / kWave), kFinishWaves * kWave, 0,
                     stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_balance_loss(int32_t segments, int32_t experts, int32_t top_k,
                               const int32_t *counts, const int32_t *routed,
                               const float *prob_sum, float alpha, float *loss, hipStream_t stream)
{
    const double unit = static_cast<double>(alpha) * experts / top_k;
    k_balance_loss<<<segments, 256, 0, stream>>>(experts, unit, counts, routed, prob_sum, loss);
    return hipGetLastError();
}

hipError_t launch_route_backward(const BackwardArgs &a, int32_t dtype, hipStream_t stream)
{
    if (a.rows.chunks == 0) return hipSuccess;
    return dtype == NIMBLE_F32   ? backward_f32(a, stream)
           : dtype == NIMBLE_F16 ? backward_f16(a, stream)
                                 : backward_bf16(a, stream);
}

hipError_t launch_counts(const CountArgs &a, hipStream_t stream)
{
    const int M = (a.counts ? a.experts : 0) + (a.rank_tokens ? a.ranks : 0);
    const size_t lds = sizeof(int) * (static_cast<size_t>(M) + (a.rank_tokens ? a.experts : 0));
    if (a.rows.chunks > 0) {
        k_counts<<<a.rows.chunks, kCountBlock, lds, stream>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    k_counts_finish<<<dim3(a.rows.segments, (M + kWave - 1) / kWave), kFinishWaves * kWave, 0,
                      stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_traffic(int32_t batch, int32_t ranks, const int32_t *rank_tokens, double bytes,
                          int32_t n_comm, const int32_t *src, const int32_t *dst, bool way_back,
                          double *traffic, hipStream_t stream)
{
    const int64_t total = static_cast<int64_t>(batch) * n_comm;
    const int64_t blocks = (total + 255) / 256;
    k_traffic<<<static_cast<unsigned>(blocks), 256, 0, stream>>>(total, ranks, rank_tokens, bytes, n_comm,
                                                               src, dst, way_back, traffic);
    return hipGetLastError();
}

}  // namespace nimble::moe
