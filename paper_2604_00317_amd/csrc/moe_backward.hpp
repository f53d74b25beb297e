// Gradient of the logits (include/nimble_moe.h).  Rows lie in lanes as in moe_route.hpp.  One pass over the
// logits: probabilities are made again (a stored sum would save 4 bytes of 2 KB, and lose accuracy for
// large logits), the choice's part comes through LDS, a float per column of every row at work.  Reading
// and writing bound it: 16384 rows of 1024 in f32 25 us (5.4 TB/s), 1 M rows of 256 in bf16 263 us (4.5 TB/s; the
// vector units are busy for 62 % of the cycles in which waves are there).
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>

#include "kernels_moe.hpp"
#include "moe_device.hpp"

namespace nimble::moe {

namespace {

template <class D, int L, int V>
__global__ __launch_bounds__(kRowWaves *kWave) void k_route_backward(BackwardArgs a, int shape)
{
    constexpr int C = L * V, G = kWave / L;
    constexpr int kSlots = L < 16 ? L : 16;              // lanes of a group that have slots
    __shared__ __align__(16) float slots[kRowWaves * G][C];
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int l = lane & (L - 1), g = lane / L;
    const bool sigmoid = (a.flags & NIMBLE_MOE_SIGMOID) != 0;
    const bool renorm = (a.flags & NIMBLE_MOE_RENORM) != 0;
    const float per_scale = 1.0f / a.scale;
    const int64_t first = static_cast<int64_t>(blockIdx.x) * a.rows.chunk;
    const int lo = static_cast<int>(first);
    const int hi = static_cast<int>(min(first + a.rows.chunk, static_cast<int64_t>(a.rows.tokens)));
    float *mine = slots[wave * G + g];
#pragma unroll
    for (int j = 0; j < V; ++j) mine[column_of<L>(j) + l * kRun] = 0.0f;
    // Rows are read a pass ahead; the first ones before it is known which segment they are in.  Divided softmax
    // weights alone have a gradient that the weights give: no logits are read for it.
    const bool dense = a.counts || sigmoid || !renorm;
    const auto *const logits = static_cast<const typename D::Raw *>(a.logits);
    RowOf<D, L, V> ahead{};
    int ahead_of = lo + wave * G;
    if (dense) ahead.load(logits + static_cast<int64_t>(min(ahead_of + g, hi - 1)) * a.stride, a.experts, l, shape);
    Segments segments(a.rows, lane);
    for (int s = segments.first(lo); s < a.rows.segments; ++s) {
        const int begin = segments.begin(s), from = max(lo, begin), to = min(hi, segments.end(s));
        if (begin >= hi) break;
        if (from >= to) continue;
        float coef[V];
#pragma unroll
        for (int j = 0; j < V; ++j) coef[j] = 0.0f;
        if (a.counts) {
            const int32_t *counts = a.counts + static_cast<int64_t>(s) * a.experts;
            const int at = anew(l * kRun);
            int count[V];
            if (shape != kSingle && a.count_runs) {
#pragma unroll
                for (int q = 0; q < V / kRun; ++q) {
                    const int col = q * (L * kRun) + at;
                    const int4 c = *reinterpret_cast<const int4 *>(counts + (col < a.experts ? col : 0));
                    count[q * kRun] = c.x;
                    count[q * kRun + 1] = c.y;
                    count[q * kRun + 2] = c.z;
                    count[q * kRun + 3] = c.w;
                }
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) count[j] = counts[min(column_of<L>(j) + at, a.experts - 1)];
            }
            const double n = static_cast<double>(a.routed[s]);
            const double unit = static_cast<double>(a.grad_loss[s]) * static_cast<double>(a.alpha) * a.experts /
                                (static_cast<double>(a.top_k) * n * n);
            const float per_count = n != 0.0 ? static_cast<float>(unit) : 0.0f;
            // (columns beyond the row's end have probability 0)
#pragma unroll
            for (int j = 0; j < V; ++j) coef[j] = per_count * static_cast<float>(count[j]);
        }
        for (int r0 = from + wave * G; r0 < to; r0 += kRowWaves * G) {
            const bool inside = r0 + g < to;
            const int64_t row = inside ? r0 + g : to - 1;       // (no group reads outside the part)
            if (dense && r0 != ahead_of)
                ahead.load(logits + row * a.stride, a.experts, l, shape);
            RowOf<D, L, V> raw = ahead;
            const int64_t slot = row * a.top_k + min(l, a.top_k - 1);   // (lanes without a slot read the last)
            int index = a.index[slot];
            float w = a.weight[slot], gw = a.grad_weight ? a.grad_weight[slot] : 0.0f;
            if (r0 + kRowWaves * G < to) {
                ahead_of = r0 + kRowWaves * G;
                if (dense) ahead.load(logits + static_cast<int64_t>(min(ahead_of + g, to - 1)) * a.stride, a.experts, l, shape);
            }
            const bool kept = !a.keep || a.keep[row] != 0;
            const bool nan = kept && l == 0 && !(w == w);
            const bool there = kept && l < a.top_k && static_cast<uint32_t>(index) < static_cast<uint32_t>(a.experts);
            index = there ? index : -1;
            w = there ? w : 0.0f;
            const float wg = there ? w * gw : 0.0f;
            const float all = group_sum<kSlots>(wg);
            const float slope = w * ((there ? gw : 0.0f) - (renorm ? all * per_scale : 0.0f));
            float before = 0.0f;
            if (index >= 0 && inside) before = atomicAdd(&mine[index], slope);
            float x[V], sum = 0.0f, rest = 0.0f, r[V];
            raw.end_at(a.experts, l, shape);
            raw.values(x);
            float top = x[0];
#pragma unroll
            for (int j = 1; j < V; ++j) top = fmaxf(top, x[j]);
            top = group_max<L>(top);
            const Shifted by(shift_of(sigmoid, top));
            if (sigmoid) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float e = exp_of(-fabsf(x[j]));
                    r[j] = __builtin_amdgcn_rcpf(1.0f + e) * (x[j] > 0.0f ? e : 1.0f);       // 1 - s
                }
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) r[j] = 1.0f;
            }
            scores_of<V>(sigmoid, x, by);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                sum = sum + x[j];
                rest = __builtin_fmaf(x[j], coef[j], rest);
            }
            const float inv = 1.0f / group_sum<L>(sum);
            rest = group_sum<L>(rest) * inv;
            // sums over the slots are in the lanes that have them
            if (!sigmoid && !renorm) rest = rest + __shfl(all, lane & ~(L - 1));
            // LDS adds slots of the same expert (a router's choice has none) in any order; where a column got more than
            // one, all are added again in the order of the slots.  (Looking costs 0 to 3 % of the kernel's time, 5 with 64 experts, top-8, sigmoids.)
            if (__ballot(before != 0.0f) != 0) {
                float total = 0.0f;
                for (int i = 0; i < a.top_k; ++i) {
                    const float other = __shfl(slope, (lane & ~(L - 1)) + i);
                    total = __shfl(index, (lane & ~(L - 1)) + i) == index ? total + other : total;
                }
                if (index >= 0 && inside) mine[index] = total;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
            for (int q = 0; q < V / kRun; ++q) {
                const float4 m = *reinterpret_cast<const float4 *>(&mine[column_of<L>(q * kRun) + l * kRun]);
                const float v[kRun] = {m.x, m.y, m.z, m.w};
#pragma unroll
                for (int i = 0; i < kRun; ++i) {
                    const int j = q * kRun + i;
                    x[j] = r[j] * __builtin_fmaf(x[j] * inv, coef[j] - rest, v[i]);
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (index >= 0 && inside) mine[index] = 0.0f;
            // rows that are left out, and rows without a choice
            const unsigned long long with = __ballot(index >= 0), without = __ballot(nan);
            const unsigned long long group = (L == kWave ? ~0ull : (1ull << (L & 63)) - 1) << (lane & ~(L - 1));
            if ((with & group) == 0) {
                const float fill = (without & group) != 0 ? __builtin_nanf("") : 0.0f;
#pragma unroll
                for (int j = 0; j < V; ++j) x[j] = fill;
            }
            if (inside)
                store_row<D, L, V>(static_cast<typename D::Raw *>(a.grad) + row * a.grad_stride, a.experts, l,
                                   shape, x);
        }
    }
}

template <class D, int L, int V>
hipError_t run(const BackwardArgs &a, hipStream_t stream)
{
    constexpr size_t B = sizeof(typename D::Raw);
    const int shape = std::max(shape_of(a.logits, a.stride, a.experts, L * V, B),
                               shape_of(a.grad, a.grad_stride, a.experts, L * V, B));
    k_route_backward<D, L, V><<<a.rows.chunks, kRowWaves * kWave, 0, stream>>>(a, shape);
    return hipGetLastError();
}

}  // namespace

template <class D>
hipError_t backward_rows(const BackwardArgs &a, hipStream_t stream)
{
    if (a.experts <= 128 && a.top_k <= 8) {
        if (a.experts <= 32) return run<D, 8, 4>(a, stream);
        if (a.experts <= 64) return run<D, 8, 8>(a, stream);
        return run<D, 8, 16>(a, stream);
    }
    if (a.experts <= 64) return run<D, 16, 4>(a, stream);
    if (a.experts <= 128) return run<D, 16, 8>(a, stream);
    if (a.experts <= 256) return run<D, 16, 16>(a, stream);
    if (a.experts <= 512) return run<D, 32, 16>(a, stream);
    if (a.experts <= 1024) return run<D, 64, 16>(a, stream);
    return run<D, 64, 32>(a, stream);
}

}  // namespace nimble::moe
