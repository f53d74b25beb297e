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

// ---- end of the sums -------------------------------------------------------------------------

// The parts of segment s are p0 .. p1 (none: p1 < p0).
struct Parts {
    int lo, hi;                  // its rows
    int64_t p0, p1;
    __device__ __forceinline__ Parts(const Rows &r, int s)
    {
        lo = r.seg_ptr ? min(max(r.seg_ptr[s], 0), r.tokens) : 0;
        hi = r.seg_ptr ? min(max(r.seg_ptr[s + 1], 0), r.tokens) : r.tokens;
        p0 = static_cast<int64_t>(lo / r.chunk) + s;
        p1 = lo < hi ? static_cast<int64_t>((hi - 1) / r.chunk) + s : p0 - 1;
    }
};

// Parts are added by the threads of a workgroup in COLS columns and 1024 / COLS (or one) rows: every row
// adds each rows-th part, and the first one the rows' sums in order.  What bounds these kernels is the time
// of a few dependent reads, so many parts (of few segments) take many rows and few columns, and few parts
// one row and a workgroup of one wave: 3.4 to 5.9 us for 32 to 512 parts of 64 to 1024 columns.
template <int COLS, int ROWS>
__global__ __launch_bounds__(COLS *ROWS) void k_route_finish(RouteArgs a)
{
    __shared__ double sums[ROWS][COLS];
    __shared__ int hits[ROWS][COLS];
    const int x = threadIdx.x % COLS, y = threadIdx.x / COLS;
    const int64_t s = blockIdx.x;
    const int col = blockIdx.y * COLS + x;
    const Parts parts(a.rows, blockIdx.x);
    double t = 0.0;
    int n = 0;
    if (col < a.experts) {
#pragma unroll 8
        for (int64_t p = parts.p0 + y; p <= parts.p1; p += ROWS) {
            t = t + static_cast<double>(a.part_prob[p * a.experts + col]);
            n += a.part_count[p * a.experts + col];
        }
    }
    int m = 0;                                       // rows with a choice, by the first columns' workgroup
    if (blockIdx.y == 0)
        for (int64_t p = parts.p0 + threadIdx.x; p <= parts.p1; p += COLS * ROWS) m += a.part_routed[p];
    if constexpr (ROWS > 1) {
        sums[y][x] = t;
        hits[y][x] = n;
        __syncthreads();
        if (y == 0) {
            for (int i = 1; i < ROWS; ++i) {
                t = t + sums[i][x];
                n += hits[i][x];
            }
        }
    }
    if (y == 0 && col < a.experts) {
        a.prob_sum[s * a.experts + col] = static_cast<float>(t);
        a.counts[s * a.experts + col] = n;
    }
    if (blockIdx.y == 0) {
        for (int step = 1; step < kWave; step *= 2) m += __shfl_xor(m, step, kWave);
        if constexpr (ROWS > 1) {
            __syncthreads();
            int *each = &hits[0][0];
            if (threadIdx.x % kWave == 0) each[threadIdx.x / kWave] = m;
            __syncthreads();
            m = 0;
            for (int i = 0; i < COLS * ROWS / kWave; ++i) m += each[i];
        }
        if (threadIdx.x == 0) a.routed[s] = m;
    }
}

// ---- loss ------------------------------------------------------------------------------------

// A workgroup per segment, of up to 1024 threads: all reads are under way at once (1.6 us for one segment of 64
// experts, 3.8 for one of 1024; no more than a launch and the reads' latency).
__global__ __launch_bounds__(1024) void k_balance_loss(int experts, double unit, const int32_t *counts,
                                                       const int32_t *routed, const float *prob_sum,
                                                       float *loss)
{
    __shared__ double part[1024 / kWave];
    const int64_t at = static_cast<int64_t>(blockIdx.x) * experts;
    const int rows = routed[blockIdx.x];
    double t = 0.0;
    for (int e = threadIdx.x; e < experts; e += blockDim.x)
        t = t + static_cast<double>(counts[at + e]) * static_cast<double>(prob_sum[at + e]);
    for (int step = 1; step < kWave; step *= 2) t = t + __shfl_xor(t, step, kWave);
    if ((threadIdx.x & (kWave - 1)) == 0) part[threadIdx.x / kWave] = t;
    __syncthreads();
    if (threadIdx.x == 0) {
        const double n = static_cast<double>(rows);
        for (int w = 1; w < static_cast<int>(blockDim.x) / kWave; ++w) t = t + part[w];
        loss[blockIdx.x] = rows == 0 ? 0.0f : static_cast<float>(unit * t / (n * n));
    }
}

// ---- counts and demand -----------------------------------------------------------------------

// Counts.  A thread has whole rows.  What bounds the kernel, behind the reading of the indices, is LDS
// additions to few places -- most rows of a skewed router choose the same experts -- and the
// comparisons of a row's destinations.  So every bin is there several times, side by side in different
// banks, a copy for every so many'th lane; indices of no expert have a bin of their own instead of a branch.
// GPUs are not counted slot by slot: their tokens are the slots of their experts, added up at the
// end, less the slots that go where an earlier slot of the same row goes, which are few.  8.4 M tokens, 8 of 1024
// experts on 512 GPUs: 64 us, 4.2 TB/s of indices; 83 with branches for missing experts, 195 with one copy of the bins.
constexpr int kCountBlock = 512;

// Segments of up to kShort rows, whole, are counted by the workgroup that ends a segment (k_counts_segment), so
// that thousands of short ones -- the tokens of every layer and source of a decoding step -- are not counted
// one after the other by the few workgroups whose rows they are.
constexpr int kShort = 512;

// Rows a thread reads before it counts them.
template <int K>
constexpr int rows_at_once() { return K <= 4 ? 4 : K <= 8 ? 2 : 1; }

// A thread's view of the bins in LDS.
struct Bins {
    int *experts;                // [experts + 1][copies]
    int *dups;                   // [ranks][copies of theirs]
    int log_copies, copy, log_dups, dup_copy;
};

// Counts rows from .. to-1, BLOCK of them at a time.  place_of(e), e <= experts, is the GPU of an expert, or
// below 0, another for each, where it has none.
template <int K, int BLOCK, class Place>
__device__ __forceinline__ void count_rows(const CountArgs &a, bool aligned, int64_t from, int64_t to, bool ranks,
                                           const Bins &bins, const Place &place_of)
{
    constexpr int N = rows_at_once<K>();
    const uint32_t E = static_cast<uint32_t>(a.experts);
    for (int64_t u0 = from; u0 < to; u0 += N * BLOCK) {
        int idx[N][K];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            if (u0 + n * BLOCK >= to) break;
            // (a row that is not there is read as the last one)
            const int64_t row = u0 + n * BLOCK + threadIdx.x;
            const int32_t *p = a.index + min(row, to - 1) * K;
            if (K % 4 == 0 && aligned) {
#pragma unroll
                for (int j = 0; j + 3 < K; j += 4) {
                    const int4 v = *reinterpret_cast<const int4 *>(p + j);
                    idx[n][j] = v.x;
                    idx[n][j + 1] = v.y;
                    idx[n][j + 2] = v.z;
                    idx[n][j + 3] = v.w;
                }
            } else if (K % 2 == 0 && aligned) {
#pragma unroll
                for (int j = 0; j + 1 < K; j += 2) {
                    const int2 v = *reinterpret_cast<const int2 *>(p + j);
                    idx[n][j] = v.x;
                    idx[n][j + 1] = v.y;
                }
            } else {
#pragma unroll
                for (int j = 0; j < K; ++j) idx[n][j] = p[j];
            }
        }
#pragma unroll
        for (int n = 0; n < N; ++n) {
            if (u0 + n * BLOCK >= to) break;
            if (u0 + (n + 1) * BLOCK > to && u0 + n * BLOCK + threadIdx.x >= to) continue;   // the last rows
            int rank[K];
#pragma unroll
            for (int j = 0; j < K; ++j) {
                const uint32_t e = min(static_cast<uint32_t>(idx[n][j]), E);
                atomicAdd(&bins.experts[(e << bins.log_copies) + bins.copy], 1);
                if (ranks) rank[j] = place_of(e);
            }
            if (ranks) {
#pragma unroll
                for (int j = 1; j < K; ++j) {
                    bool again = false;
#pragma unroll
                    for (int i = 0; i < j; ++i) again = again | (rank[i] == rank[j]);
                    if (again && rank[j] >= 0) atomicAdd(&bins.dups[(rank[j] << bins.log_dups) + bins.dup_copy], 1);
                }
            }
        }
    }
}

__device__ __forceinline__ int place_or_none(int r, int ranks, int e)
{
    return static_cast<uint32_t>(r) < static_cast<uint32_t>(ranks) ? r : -1 - e;
}

template <int K>
__global__ __launch_bounds__(kCountBlock) void k_counts(CountArgs a, int log_copies, int log_dups, bool aligned)
{
    extern __shared__ int lds[];
    const int E = a.experts, R = a.rank_tokens ? a.ranks : 0;
    const int copies = 1 << log_copies, dup_copies = 1 << log_dups;
    Bins bins{lds, lds + ((E + 1) << log_copies), log_copies, static_cast<int>(threadIdx.x) & (copies - 1), log_dups,
              static_cast<int>(threadIdx.x) & (dup_copies - 1)};
    int *totals = bins.dups + (R << log_dups);       // [ranks]
    int *place = totals + R;                         // [experts + 1]
    const int lane = threadIdx.x & (kWave - 1);
    const int64_t first = static_cast<int64_t>(blockIdx.x) * a.rows.chunk;
    const int lo = static_cast<int>(first);
    const int hi = static_cast<int>(min(first + a.rows.chunk, static_cast<int64_t>(a.rows.tokens)));
    if (R)
        for (int e = threadIdx.x; e <= E; e += kCountBlock) place[e] = place_or_none(e < E ? a.place[e] : -1, R, e);
    Segments segments(a.rows, lane);
    for (int s = segments.longer(segments.first(lo), a.whole, hi); s < a.rows.segments;
         s = segments.longer(s + 1, a.whole, hi)) {
        const int begin = segments.begin(s), from = max(lo, begin), to = min(hi, segments.end(s));
        if (begin >= hi) break;
        if (from >= to) continue;
        for (int c = threadIdx.x; c < ((E + 1) << log_copies) + (R << log_dups) + R; c += kCountBlock) lds[c] = 0;
        __syncthreads();
        count_rows<K, kCountBlock>(a, aligned, from, to, R != 0, bins, [&](uint32_t e) { return place[e]; });
        __syncthreads();
        const int M = (a.counts ? E : 0) + R;
        int32_t *part = a.part + (static_cast<int64_t>(blockIdx.x) + s) * M;
        for (int e = threadIdx.x; e < E; e += kCountBlock) {
            int t = 0;
            for (int c = 0; c < copies; ++c) t += bins.experts[(e << log_copies) + ((c + e) & (copies - 1))];
            if (a.counts) part[e] = t;
            if (R && place[e] >= 0) atomicAdd(&totals[place[e]], t);
        }
        if (R) {
            __syncthreads();
            for (int r = threadIdx.x; r < R; r += kCountBlock) {
                int t = totals[r];
                for (int c = 0; c < dup_copies; ++c) t -= bins.dups[(r << log_dups) + ((c + r) & (dup_copies - 1))];
                part[M - R + r] = t;
            }
        }
        __syncthreads();
    }
}

// A workgroup per segment: the parts of a long one are added, a short one is counted here (3.9 to 5.2 us).
constexpr int kSegmentBlock = 256;

template <int K>
__global__ __launch_bounds__(kSegmentBlock) void k_counts_segment(CountArgs a, bool aligned)
{
    extern __shared__ int lds[];
    const int E = a.experts, R = a.rank_tokens ? a.ranks : 0, M = (a.counts ? E : 0) + R;
    const int64_t s = blockIdx.x;
    const Parts parts(a.rows, blockIdx.x);
    int32_t *counts = a.counts + s * E, *tokens = a.rank_tokens + s * R;
    if (parts.hi - parts.lo > a.whole) {
        for (int c0 = threadIdx.x; c0 < M; c0 += 4 * kSegmentBlock) {    // four columns' reads at a time
            int n[4] = {0, 0, 0, 0};
#pragma unroll 2
            for (int64_t p = parts.p0; p <= parts.p1; ++p) {
#pragma unroll
                for (int i = 0; i < 4; ++i) n[i] += a.part[p * M + min(c0 + i * kSegmentBlock, M - 1)];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int col = c0 + i * kSegmentBlock;
                if (col < M - R) counts[col] = n[i];
                else if (col < M) tokens[col - (M - R)] = n[i];
            }
        }
        return;
    }
    Bins bins{lds, lds + E + 1, 0, 0, 0, 0};
    int *totals = bins.dups + R;
    for (int c = threadIdx.x; c < E + 1 + 2 * R; c += kSegmentBlock) lds[c] = 0;
    __syncthreads();
    count_rows<K, kSegmentBlock>(a, aligned, parts.lo, parts.hi, R != 0, bins, [&](uint32_t e) {
        const int i = static_cast<int>(e);
        return place_or_none(i < E ? a.place[i] : -1, R, i);
    });
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += kSegmentBlock) {
        const int t = bins.experts[e];
        if (a.counts) counts[e] = t;
        if (R && t != 0) {
            const int r = place_or_none(a.place[e], R, e);
            if (r >= 0) atomicAdd(&totals[r], t);
        }
    }
    if (!R) return;
    __syncthreads();
    for (int r = threadIdx.x; r < R; r += kSegmentBlock) tokens[r] = totals[r] - bins.dups[r];
}

// The parts of a segment, as in k_route_finish.
template <int COLS, int ROWS>
__global__ __launch_bounds__(COLS *ROWS) void k_counts_finish(CountArgs a)
{
    __shared__ int hits[ROWS][COLS];
    const int E = a.counts ? a.experts : 0, M = E + (a.rank_tokens ? a.ranks : 0);
    const int x = threadIdx.x % COLS, y = threadIdx.x / COLS;
    const int64_t s = blockIdx.x;
    const int col = blockIdx.y * COLS + x;
    const Parts parts(a.rows, blockIdx.x);
    int n = 0;
    if (col < M) {
#pragma unroll 8
        for (int64_t p = parts.p0 + y; p <= parts.p1; p += ROWS) n += a.part[p * M + col];
    }
    if constexpr (ROWS > 1) {
        hits[y][x] = n;
        __syncthreads();
        if (y == 0)
            for (int i = 1; i < ROWS; ++i) n += hits[i][x];
    }
    if (y != 0 || col >= M) return;
    if (col < E) a.counts[s * E + col] = n;
    else a.rank_tokens[s * a.ranks + col - E] = n;
}

// A thread per commodity; 1.9 to 4.8 us, a launch and two dependent reads.
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

namespace {

int32_t round_up(int64_t rows, int32_t pass)
{
    return static_cast<int32_t>((std::max<int64_t>(rows, 1) + pass - 1) / pass * pass);
}

// A segment has about chunks / segments parts.
bool many_parts(const Rows &r) { return r.chunks > 8 * static_cast<int64_t>(r.segments); }

}  // namespace

// Whole passes of a workgroup's rows.  Where segments are shorter than a pass, chunks are too: the parts of a
// chunk are worked on one after the other.
int32_t route_chunk(int32_t tokens, int32_t experts, int32_t segments, int32_t most, int32_t chain)
{
    const int32_t rows = experts <= 256 ? 4 : experts <= 512 ? 2 : 1;    // of a wave, with any top_k
    int32_t pass = kRowWaves * (experts <= 128 ? 8 : rows);
    if (segments > 1) pass = std::min(pass, round_up(tokens / segments, 8));
    const int64_t even = (static_cast<int64_t>(tokens) + most - 1) / most;
    return round_up(std::min<int64_t>(even, static_cast<int64_t>(chain) * kRowWaves * rows), pass);
}

int32_t count_chunk(int32_t tokens, int32_t) { return round_up((static_cast<int64_t>(tokens) + 1023) / 1024, kCountBlock); }

hipError_t launch_route(const RouteArgs &a, int32_t dtype, hipStream_t stream)
{
    if (a.rows.chunks > 0) {
        const hipError_t e = dtype == NIMBLE_F32   ? route_f32(a, stream)
                             : dtype == NIMBLE_F16 ? route_f16(a, stream)
                                                   : route_bf16(a, stream);
        if (e != hipSuccess || !a.counts) return e;
    }
    if (!a.counts) return hipSuccess;
    if (many_parts(a.rows))
        k_route_finish<16, 64><<<dim3(a.rows.segments, (a.experts + 15) / 16), 1024, 0, stream>>>(a);
    else
        k_route_finish<64, 1><<<dim3(a.rows.segments, (a.experts + 63) / 64), 64, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_balance_loss(int32_t segments, int32_t experts, int32_t top_k,
                               const int32_t *counts, const int32_t *routed,
                               const float *prob_sum, float alpha, float *loss, hipStream_t stream)
{
    const double unit = static_cast<double>(alpha) * experts / top_k;
    const int threads = std::min(1024, round_up(experts, kWave));
    k_balance_loss<<<segments, threads, 0, stream>>>(experts, unit, counts, routed, prob_sum, loss);
    return hipGetLastError();
}

hipError_t launch_route_backward(const BackwardArgs &a, int32_t dtype, hipStream_t stream)
{
    if (a.rows.chunks == 0) return hipSuccess;
    return dtype == NIMBLE_F32   ? backward_f32(a, stream)
           : dtype == NIMBLE_F16 ? backward_f16(a, stream)
                                 : backward_bf16(a, stream);
}

namespace {

template <int K>
hipError_t counts_of(CountArgs a, hipStream_t stream)
{
    const int E = a.experts, R = a.rank_tokens ? a.ranks : 0, M = (a.counts ? E : 0) + R;
    const bool aligned = reinterpret_cast<uintptr_t>(a.index) % 16 == 0;
    const bool few_segments = many_parts(a.rows);
    a.whole = few_segments ? 0 : kShort;
    if (a.rows.tokens > a.whole) {
        // as many copies as 32 KiB hold, up to 32 (and 8 KiB, up to 8, of the bins of double visits), and no more
        // bins than a chunk has slots: 47 KB for 1024 experts on 512 GPUs, three workgroups to a CU; 74 KB, two,
        // for 2048 on 4096
        int log_copies = 5, log_dups = 3;
        const int64_t slots = std::min<int64_t>(static_cast<int64_t>(a.rows.chunk) * K, 8192);
        while (log_copies > 0 && static_cast<int64_t>(E) << log_copies > slots) --log_copies;
        while (log_dups > 0 && static_cast<int64_t>(R) << log_dups > 2048) --log_dups;
        const size_t bins = E + 1, ranks = R;
        const size_t lds = sizeof(int) * ((bins << log_copies) + bins + (ranks << log_dups) + ranks);
        k_counts<K><<<a.rows.chunks, kCountBlock, lds, stream>>>(a, log_copies, log_dups, aligned);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (few_segments)
        k_counts_finish<16, 64><<<dim3(a.rows.segments, (M + 15) / 16), 1024, 0, stream>>>(a);
    else
        k_counts_segment<K><<<a.rows.segments, kSegmentBlock, sizeof(int) * (E + 1 + 2 * R), stream>>>(a, aligned);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_counts(const CountArgs &a, hipStream_t stream)
{
    switch (a.top_k) {
    case 1: return counts_of<1>(a, stream);
    case 2: return counts_of<2>(a, stream);
    case 3: return counts_of<3>(a, stream);
    case 4: return counts_of<4>(a, stream);
    case 5: return counts_of<5>(a, stream);
    case 6: return counts_of<6>(a, stream);
    case 7: return counts_of<7>(a, stream);
    case 8: return counts_of<8>(a, stream);
    case 9: return counts_of<9>(a, stream);
    case 10: return counts_of<10>(a, stream);
    case 11: return counts_of<11>(a, stream);
    case 12: return counts_of<12>(a, stream);
    case 13: return counts_of<13>(a, stream);
    case 14: return counts_of<14>(a, stream);
    case 15: return counts_of<15>(a, stream);
    default: return counts_of<16>(a, stream);
    }
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
