// Routing kernels: choice of experts with its sums, balance loss, gradient of the logits, counts
// per expert and destination GPU, demand vectors (definitions in include/nimble_moe.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "../../include/nimble_moe.h"
#include "kernels_moe.hpp"
#include "wave_ops.hpp"

namespace nimble::moe {

namespace {

constexpr float kInf = __builtin_inff();
constexpr int kStatWaves = 8;        // waves of a workgroup that makes sums
constexpr int kRowWaves = 4;         // of one that does not

// ---- element types ---------------------------------------------------------------------------

struct F32 {
    using Raw = float;
    static __device__ __forceinline__ float up(float v) { return v; }
    static __device__ __forceinline__ float down(float v) { return v; }
};
struct F16 {
    using Raw = uint16_t;
    static __device__ __forceinline__ float up(uint16_t v)
    {
        return static_cast<float>(__builtin_bit_cast(_Float16, v));
    }
    static __device__ __forceinline__ uint16_t down(float v)
    {
        return __builtin_bit_cast(uint16_t, static_cast<_Float16>(v));
    }
};
struct BF16 {
    using Raw = uint16_t;
    static __device__ __forceinline__ float up(uint16_t v)
    {
        return __builtin_bit_cast(float, static_cast<uint32_t>(v) << 16);
    }
    static __device__ __forceinline__ uint16_t down(float v)
    {
        return __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
    }
};

// A row lies in a wave as V values per lane, in groups of W neighbours (one load each): lane l
// has columns q * 64 W + l W + 0 .. W-1 for q = 0 .. V/W - 1.
template <int V>
constexpr int group_width() { return V < 4 ? V : 4; }

template <class D, int W>
struct alignas(sizeof(typename D::Raw) * W) Group {
    typename D::Raw v[W];
};

// Columns beyond the row's end come as -inf, like masked ones.  `whole`: groups inside the row are
// aligned to their size.
template <class D, int V>
__device__ __forceinline__ void load_row(const typename D::Raw *row, int experts, int lane,
                                         bool whole, float (&x)[V])
{
    constexpr int W = group_width<V>();
#pragma unroll
    for (int q = 0; q < V / W; ++q) {
        const int col = q * (kWave * W) + lane * W;
        if (whole && col + W <= experts) {
            const auto g = *reinterpret_cast<const Group<D, W> *>(row + col);
#pragma unroll
            for (int i = 0; i < W; ++i) x[q * W + i] = D::up(g.v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < W; ++i) x[q * W + i] = col + i < experts ? D::up(row[col + i]) : -kInf;
        }
    }
}

template <class D, int V>
__device__ __forceinline__ void store_row(typename D::Raw *row, int experts, int lane, bool whole,
                                          const float (&x)[V])
{
    constexpr int W = group_width<V>();
#pragma unroll
    for (int q = 0; q < V / W; ++q) {
        const int col = q * (kWave * W) + lane * W;
        if (whole && col + W <= experts) {
            Group<D, W> g;
#pragma unroll
            for (int i = 0; i < W; ++i) g.v[i] = D::down(x[q * W + i]);
            *reinterpret_cast<Group<D, W> *>(row + col) = g;
        } else {
#pragma unroll
            for (int i = 0; i < W; ++i)
                if (col + i < experts) row[col + i] = D::down(x[q * W + i]);
        }
    }
}

// ---- reductions over lanes -------------------------------------------------------------------

struct TwoF32 {
    float a, b;
};
__device__ __forceinline__ TwoF32 rows_f32(float v)          // both rows of a pair of rows
{
    const int i = __builtin_bit_cast(int, v);
    const auto r = __builtin_amdgcn_permlane16_swap(i, i, false, false);
    return {__builtin_bit_cast(float, static_cast<int>(r[0])),
            __builtin_bit_cast(float, static_cast<int>(r[1]))};
}
__device__ __forceinline__ TwoF32 halves_f32(float v)        // both halves of the wave
{
    const int i = __builtin_bit_cast(int, v);
    const auto r = __builtin_amdgcn_permlane32_swap(i, i, false, false);
    return {__builtin_bit_cast(float, static_cast<int>(r[0])),
            __builtin_bit_cast(float, static_cast<int>(r[1]))};
}
template <int CTRL>
__device__ __forceinline__ float dpp_f32(float v)
{
    return __builtin_bit_cast(float, dpp_i32<CTRL>(__builtin_bit_cast(int, v)));
}

// over aligned groups of 16 lanes, and over the wave; the same bits in all lanes
__device__ __forceinline__ float max16(float v)
{
    v = fmaxf(v, dpp_f32<kDppXor1>(v));
    v = fmaxf(v, dpp_f32<kDppXor2>(v));
    v = fmaxf(v, dpp_f32<kDppHalfMirror>(v));
    return fmaxf(v, dpp_f32<kDppMirror>(v));
}
__device__ __forceinline__ float sum16(float v)
{
    v = v + dpp_f32<kDppXor1>(v);
    v = v + dpp_f32<kDppXor2>(v);
    v = v + dpp_f32<kDppHalfMirror>(v);
    return v + dpp_f32<kDppMirror>(v);
}
__device__ __forceinline__ float max64(float v)
{
    v = max16(v);
    const TwoF32 r = rows_f32(v);
    const TwoF32 h = halves_f32(fmaxf(r.a, r.b));
    return fmaxf(h.a, h.b);
}
__device__ __forceinline__ float sum64(float v)
{
    v = sum16(v);
    const TwoF32 r = rows_f32(v);
    const TwoF32 h = halves_f32(r.a + r.b);
    return h.a + h.b;
}

__device__ __forceinline__ float uniform(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v)));
}
__device__ __forceinline__ float of_lane(float v, int lane)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}

// exp by the hardware's exp2: off by 2^-23 |x| and a step or so, relative; results below 2^-126 are 0
__device__ __forceinline__ float exp_of(float x)
{
    return __builtin_amdgcn_exp2f(x * 1.44269504f);
}

// Sigmoids are summed and compared as s(x) exp(-shift) = exp(min(x, 0) - shift) / (1 + exp(-|x|)), shift
// = 0 unless the row's largest logit is so low that all sigmoids would vanish in 32 bits.
__device__ __forceinline__ float sigmoid_shift(float top) { return top < -60.0f ? top : 0.0f; }
__device__ __forceinline__ float shifted_sigmoid(float x, float shift)
{
    const float e = exp_of(-fabsf(x));
    float n = x > 0.0f ? 1.0f : e;
    if (shift != 0.0f) n = exp_of(x - shift);
    return n * __builtin_amdgcn_rcpf(1.0f + e);
}

// ---- segments --------------------------------------------------------------------------------

__device__ __forceinline__ int offset(const Rows &r, int s)
{
    return min(max(r.seg_ptr[s], 0), r.tokens);
}
__device__ __forceinline__ int begin_of(const Rows &r, int s) { return r.seg_ptr ? offset(r, s) : 0; }
__device__ __forceinline__ int end_of(const Rows &r, int s)
{
    return r.seg_ptr ? offset(r, s + 1) : r.tokens;
}

// The first segment that ends behind `row`, by a search with 64 tries at a time (a round trip to
// memory each).  All lanes of the wave are active and get the same answer.
__device__ __forceinline__ int first_segment(const Rows &r, int row, int lane)
{
    if (!r.seg_ptr) return 0;
    int at = 0, n = r.segments;
    while (n > 0) {
        const int step = (n + kWave - 1) / kWave;
        const int s = at + lane * step + step - 1;
        const bool behind = s >= at + n || r.seg_ptr[s + 1] > row;
        const unsigned long long hit = __ballot(behind);
        if (hit == 0) return at + n;
        const int to = at + (__ffsll(hit) - 1) * step;
        n = min(step - 1, at + n - to);
        at = to;
    }
    return at;
}

// ---- choice ----------------------------------------------------------------------------------

// The top_k largest keys of a row, lane j gets column and logit of slot j (-1 and -inf where there
// is none).  Per slot: the largest key of the wave (each lane has the largest of every group of W
// at hand), the first group and lane that hold it in column order, and that one key taken out.
// All of the bookkeeping is in scalars: the lanes' answers are ballots.
template <int V>
__device__ __forceinline__ void choose(float (&key)[V], const float (&x)[V], int top_k, int lane,
                                       int &index, float &logit)
{
    constexpr int W = group_width<V>(), Q = V / W;
    float top[Q];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        top[q] = key[q * W];
#pragma unroll
        for (int i = 1; i < W; ++i) top[q] = fmaxf(top[q], key[q * W + i]);
    }
    index = -1;
    logit = -kInf;
    for (int slot = 0; slot < top_k; ++slot) {
        float best = top[0];
#pragma unroll
        for (int q = 1; q < Q; ++q) best = fmaxf(best, top[q]);
        best = uniform(max64(best));
        if (best == -kInf) return;
        bool found = false;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const unsigned long long any = __ballot(top[q] == best);
            if (found || any == 0) continue;
            found = true;
            const int owner = __ffsll(any) - 1;
            const unsigned long long bit = 1ull << owner;
            bool taken = false;
            float value = -kInf;
            int col = q * (kWave * W) + owner * W;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const bool here = !taken && (__ballot(key[q * W + i] == best) & bit) != 0;
                if (here) {
                    value = of_lane(x[q * W + i], owner);
                    col += i;
                    key[q * W + i] = lane == owner ? -kInf : key[q * W + i];
                }
                taken = taken || here;
            }
            top[q] = key[q * W];
#pragma unroll
            for (int i = 1; i < W; ++i) top[q] = fmaxf(top[q], key[q * W + i]);
            if (lane == slot) {
                index = col;
                logit = value;
            }
        }
    }
}

// One row: choice, weights, statistics; p gets the probabilities (0 or NaN where there are none).
// Returns whether the row has a choice.
template <class D, int V>
__device__ __forceinline__ bool route_row(const RouteArgs &a, int64_t row, int lane, bool whole,
                                          const float (&bias)[V], float (&p)[V], int &index)
{
    const bool sigmoid = (a.flags & NIMBLE_MOE_SIGMOID) != 0;
    const bool renorm = (a.flags & NIMBLE_MOE_RENORM) != 0;
    const int64_t slot = row * a.top_k + lane;
    if (a.keep && a.keep[row] == 0) {
        index = -1;
#pragma unroll
        for (int j = 0; j < V; ++j) p[j] = 0.0f;
        if (lane < a.top_k) {
            a.index[slot] = -1;
            a.weight[slot] = 0.0f;
        }
        return false;
    }
    float x[V], key[V];
    load_row<D, V>(static_cast<const typename D::Raw *>(a.logits) + row * a.stride, a.experts, lane,
                   whole, x);
    float top = x[0];
#pragma unroll
    for (int j = 1; j < V; ++j) top = fmaxf(top, x[j]);
    top = max64(top);
    const float shift = sigmoid ? sigmoid_shift(top == -kInf ? 0.0f : top) : (top == -kInf ? 0.0f : top);
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        p[j] = sigmoid ? shifted_sigmoid(x[j], shift) : exp_of(x[j] - shift);
        sum = sum + p[j];
    }
    sum = sum64(sum);
    const bool bad = !(sum == sum) || top == kInf;
    const bool empty = !bad && top == -kInf;
    const float inv = bad ? __builtin_nanf("") : (empty ? 0.0f : 1.0f / sum);
#pragma unroll
    for (int j = 0; j < V; ++j) p[j] = p[j] * inv;

    index = -1;
    float logit = -kInf;
    if (!bad && !empty) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float k = x[j] + bias[j];
            key[j] = x[j] == -kInf || !(k == k) ? -kInf : k;
        }
        choose<V>(key, x, a.top_k, lane, index, logit);
    }
    float w;
    if (renorm) {
        const float t = max16(logit);
        const float u = sigmoid ? shifted_sigmoid(logit, sigmoid_shift(t)) : exp_of(logit - t);
        w = u / sum16(u);
    } else {
        w = sigmoid ? shifted_sigmoid(logit, 0.0f) : exp_of(logit - shift) * inv;
    }
    w = bad ? __builtin_nanf("") : (index < 0 ? 0.0f : w * a.scale);
    if (lane < a.top_k) {
        a.index[slot] = index;
        a.weight[slot] = w;
    }
    const bool chosen = __builtin_amdgcn_readfirstlane(index) >= 0;
    if (!bad && !chosen) {                       // nothing but keys of -inf
#pragma unroll
        for (int j = 0; j < V; ++j) p[j] = 0.0f;
    }
    return chosen;
}

template <int V>
__device__ __forceinline__ void load_bias(const RouteArgs &a, int lane, float (&bias)[V])
{
    constexpr int W = group_width<V>();
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int col = (j / W) * (kWave * W) + lane * W + j % W;
        bias[j] = a.bias && col < a.experts ? a.bias[col] : 0.0f;   // (+0: the keys' zeros are +0)
    }
}

// A wave per row, no sums.
template <class D, int V>
__global__ __launch_bounds__(kRowWaves *kWave) void k_route(RouteArgs a, bool whole)
{
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    float bias[V];
    load_bias<V>(a, lane, bias);
    for (int64_t row = static_cast<int64_t>(blockIdx.x) * kRowWaves + wave; row < a.rows.tokens;
         row += static_cast<int64_t>(gridDim.x) * kRowWaves) {
        if (a.rows.seg_ptr) {
            const int s = first_segment(a.rows, static_cast<int>(row), lane);
            if (s >= a.rows.segments || begin_of(a.rows, s) > row) continue;
        }
        float p[V];
        int index;
        route_row<D, V>(a, row, lane, whole, bias, p, index);
    }
}

// A workgroup per chunk, a wave per row in turn; probabilities are summed in registers, slots
// counted in LDS, and the waves' sums added in order at the end of every part.
template <class D, int V>
__global__ __launch_bounds__(kStatWaves *kWave) void k_route_sums(RouteArgs a, bool whole)
{
    constexpr int C = V * kWave;
    __shared__ float sums[kStatWaves][C];
    __shared__ int hits[C];
    __shared__ int routed[kStatWaves];
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t first = static_cast<int64_t>(blockIdx.x) * a.rows.chunk;
    const int lo = static_cast<int>(first);
    const int hi = static_cast<int>(min(first + a.rows.chunk, static_cast<int64_t>(a.rows.tokens)));
    float bias[V];
    load_bias<V>(a, lane, bias);
    for (int s = first_segment(a.rows, lo, lane); s < a.rows.segments; ++s) {
        const int from = max(lo, begin_of(a.rows, s)), to = min(hi, end_of(a.rows, s));
        if (begin_of(a.rows, s) >= hi) break;
        if (from >= to) continue;
        for (int c = threadIdx.x; c < C; c += kStatWaves * kWave) hits[c] = 0;
        __syncthreads();
        float acc[V];
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] = 0.0f;
        int n = 0;
        for (int row = from + wave; row < to; row += kStatWaves) {
            float p[V];
            int index;
            n += route_row<D, V>(a, row, lane, whole, bias, p, index) ? 1 : 0;
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] = acc[j] + p[j];
            if (lane < a.top_k && index >= 0) atomicAdd(&hits[index], 1);
        }
        constexpr int W = group_width<V>();
#pragma unroll
        for (int j = 0; j < V; ++j)
            sums[wave][(j / W) * (kWave * W) + lane * W + j % W] = acc[j];
        if (lane == 0) routed[wave] = n;
        __syncthreads();
        const int64_t part = static_cast<int64_t>(blockIdx.x) + s;
        for (int c = threadIdx.x; c < a.experts; c += kStatWaves * kWave) {
            float t = sums[0][c];
#pragma unroll
            for (int w = 1; w < kStatWaves; ++w) t = t + sums[w][c];
            a.part_prob[part * a.experts + c] = t;
            a.part_count[part * a.experts + c] = hits[c];
        }
        if (threadIdx.x == 0) {
            int t = 0;
            for (int w = 0; w < kStatWaves; ++w) t += routed[w];
            a.part_routed[part] = t;
        }
        __syncthreads();
    }
}

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

// ---- gradient --------------------------------------------------------------------------------

template <class D, int V>
__global__ __launch_bounds__(kStatWaves *kWave) void k_route_backward(BackwardArgs a, bool whole)
{
    constexpr int W = group_width<V>(), C = V * kWave;
    __shared__ float slots[kStatWaves][C];       // the weights' part of a wave's row, by column
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int64_t first = static_cast<int64_t>(blockIdx.x) * a.rows.chunk;
    const int lo = static_cast<int>(first);
    const int hi = static_cast<int>(min(first + a.rows.chunk, static_cast<int64_t>(a.rows.tokens)));
    const bool sigmoid = (a.flags & NIMBLE_MOE_SIGMOID) != 0;
    const bool renorm = (a.flags & NIMBLE_MOE_RENORM) != 0;
    float *mine = slots[wave];
    for (int c = lane; c < C; c += kWave) mine[c] = 0.0f;
    for (int s = first_segment(a.rows, lo, lane); s < a.rows.segments; ++s) {
        if (begin_of(a.rows, s) >= hi) break;
        const int from = max(lo, begin_of(a.rows, s)), to = min(hi, end_of(a.rows, s));
        if (from >= to) continue;
        float coef[V];
        double unit = 0.0;
        if (a.counts) {
            const double n = static_cast<double>(a.routed[s]);
            if (a.routed[s] != 0)
                unit = static_cast<double>(a.grad_loss[s]) * static_cast<double>(a.alpha) * a.experts /
                       (static_cast<double>(a.top_k) * n * n);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int col = (j / W) * (kWave * W) + lane * W + j % W;
            coef[j] = a.counts && col < a.experts
                          ? static_cast<float>(unit * a.counts[static_cast<int64_t>(s) * a.experts + col])
                          : 0.0f;
        }
        for (int row = from + wave; row < to; row += kStatWaves) {
            float x[V];
            const int64_t at = row;
            auto *out = static_cast<typename D::Raw *>(a.grad) + at * a.grad_stride;
            const bool kept = !a.keep || a.keep[row] != 0;
            const float first_w = kept ? a.weight[at * a.top_k] : 0.0f;
            int index = -1;
            float wg = 0.0f, w = 0.0f, g = 0.0f;
            if (kept && lane < a.top_k) {
                index = a.index[at * a.top_k + lane];
                if (static_cast<uint32_t>(index) >= static_cast<uint32_t>(a.experts)) index = -1;
                if (index >= 0) {
                    w = a.weight[at * a.top_k + lane];
                    if (a.grad_weight) g = a.grad_weight[at * a.top_k + lane];
                    wg = w * g;
                }
            }
            const bool nan = kept && !(first_w == first_w);
            if (__ballot(index >= 0) == 0) {                     // left out, or without a choice
#pragma unroll
                for (int j = 0; j < V; ++j) x[j] = nan ? __builtin_nanf("") : 0.0f;
                store_row<D, V>(out, a.experts, lane, whole, x);
                continue;
            }
            load_row<D, V>(static_cast<const typename D::Raw *>(a.logits) + at * a.stride, a.experts,
                           lane, whole, x);
            const float all = uniform(sum16(wg));
            const float slope = w * (g - (renorm ? all / a.scale : 0.0f));
            if (index >= 0) atomicAdd(&mine[index], slope);
            float top = x[0], sum = 0.0f, rest = 0.0f, p[V], r[V];
#pragma unroll
            for (int j = 1; j < V; ++j) top = fmaxf(top, x[j]);
            top = max64(top);
            const float shift = sigmoid ? sigmoid_shift(top) : top;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if (sigmoid) {
                    const float e = exp_of(-fabsf(x[j]));
                    const float d = __builtin_amdgcn_rcpf(1.0f + e);
                    r[j] = x[j] > 0.0f ? e * d : d;              // 1 - s
                    p[j] = (shift != 0.0f ? exp_of(x[j] - shift) : (x[j] > 0.0f ? 1.0f : e)) * d;
                } else {
                    r[j] = 1.0f;
                    p[j] = exp_of(x[j] - shift);
                }
                sum = sum + p[j];
                rest = rest + p[j] * coef[j];
            }
            const float inv = 1.0f / sum64(sum);
#pragma unroll
            for (int j = 0; j < V; ++j) p[j] = p[j] * inv;
            rest = sum64(rest) * inv;
            if (!sigmoid && !renorm) rest = rest + all;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int col = (j / W) * (kWave * W) + lane * W + j % W;
                x[j] = r[j] * (p[j] * (coef[j] - rest) + mine[col]);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (index >= 0) mine[index] = 0.0f;
            store_row<D, V>(out, a.experts, lane, whole, x);
        }
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

// ---- launches --------------------------------------------------------------------------------

// Rows can be read and written in groups: those inside a row are aligned to their size.
bool groups_align(const void *base, int64_t stride, int width, int bytes)
{
    const auto at = reinterpret_cast<uintptr_t>(base);
    return at % static_cast<uintptr_t>(width * bytes) == 0 && stride % width == 0;
}

template <class D, int V>
hipError_t route_as(const RouteArgs &a, hipStream_t stream)
{
    const bool whole = groups_align(a.logits, a.stride, group_width<V>(), sizeof(typename D::Raw));
    if (!a.counts) {
        if (a.rows.tokens == 0) return hipSuccess;
        const int64_t grid = std::min<int64_t>((static_cast<int64_t>(a.rows.tokens) + kRowWaves - 1) / kRowWaves,
                                               1 << 20);
        k_route<D, V><<<static_cast<unsigned>(grid), kRowWaves * kWave, 0, stream>>>(a, whole);
        return hipGetLastError();
    }
    if (a.rows.chunks > 0) {
        k_route_sums<D, V><<<a.rows.chunks, kStatWaves * kWave, 0, stream>>>(a, whole);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    k_route_finish<<<dim3(a.rows.segments, (a.experts + kWave - 1) / kWave), kFinishWaves * kWave, 0,
                     stream>>>(a);
    return hipGetLastError();
}

template <class D, int V>
hipError_t backward_as(const BackwardArgs &a, hipStream_t stream)
{
    constexpr int W = group_width<V>(), B = sizeof(typename D::Raw);
    if (a.rows.chunks == 0) return hipSuccess;
    const bool whole = groups_align(a.logits, a.stride, W, B) && groups_align(a.grad, a.grad_stride, W, B);
    k_route_backward<D, V><<<a.rows.chunks, kStatWaves * kWave, 0, stream>>>(a, whole);
    return hipGetLastError();
}

template <class D>
hipError_t route_of(const RouteArgs &a, hipStream_t stream)
{
    if (a.experts <= 64) return route_as<D, 1>(a, stream);
    if (a.experts <= 128) return route_as<D, 2>(a, stream);
    if (a.experts <= 256) return route_as<D, 4>(a, stream);
    if (a.experts <= 512) return route_as<D, 8>(a, stream);
    if (a.experts <= 1024) return route_as<D, 16>(a, stream);
    return route_as<D, 32>(a, stream);
}

template <class D>
hipError_t backward_of(const BackwardArgs &a, hipStream_t stream)
{
    if (a.experts <= 64) return backward_as<D, 1>(a, stream);
    if (a.experts <= 128) return backward_as<D, 2>(a, stream);
    if (a.experts <= 256) return backward_as<D, 4>(a, stream);
    if (a.experts <= 512) return backward_as<D, 8>(a, stream);
    if (a.experts <= 1024) return backward_as<D, 16>(a, stream);
    return backward_as<D, 32>(a, stream);
}

}  // namespace

// About four workgroups per CU, and no fewer rows than waves.
int32_t route_chunk(int32_t tokens, int32_t)
{
    return std::max(kStatWaves, (tokens + 1023) / 1024);
}

int32_t count_chunk(int32_t tokens, int32_t)
{
    return std::max(kCountBlock, (tokens + 1023) / 1024);
}

hipError_t launch_route(const RouteArgs &a, int32_t dtype, hipStream_t stream)
{
    if (dtype == NIMBLE_F32) return route_of<F32>(a, stream);
    if (dtype == NIMBLE_F16) return route_of<F16>(a, stream);
    return route_of<BF16>(a, stream);
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
    if (dtype == NIMBLE_F32) return backward_of<F32>(a, stream);
    if (dtype == NIMBLE_F16) return backward_of<F16>(a, stream);
    return backward_of<BF16>(a, stream);
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
