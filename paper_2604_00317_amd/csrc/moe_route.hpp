// Choice of experts, their weights, and the sums of the balance loss (include/nimble_moe.h).
//
// A row lies in a group of 8 to 64 lanes (moe_device.hpp), so a wave works on up to eight rows at a
// time.  What bounds the kernel is the choice: everything else is half a dozen operations per logit.  It
// is made of minima and maxima of 32-bit whole numbers, without branches:
//   - a logit becomes a key whose order as a whole number is its order as a float, with the column, turned
//     round, in the lowest bits: keys are distinct, and among equal values the lower column is the larger;
//   - every lane sorts its V keys down to the KL largest (sorting networks of KL keys, then merges
//     of two lists: the larger ones of one list and the other backwards, sorted again);
//   - slot after slot, the largest head of all lanes is the next choice, and its lane's list moves up.
// A 16-bit logit and its column fit a key.  Binary32 logits, and sums with a bias, lose their last bits to
// the column (ROUNDED), so one slot more is looked at: where neighbours in the order agree in the bits that are
// left, the chosen are put in order by whole values, and where that happens at the last one, the wave
// chooses again by whole values.  (Standard normal logits, counted: top-2 of 64 to top-8 of 1024 experts in
// binary32, 0.04 to 0.3 % of waves choose again and 0.04 to 1 % put in order; all where most are equal.)
//
// Measured, top-8 of the experts: 1 M tokens on 256 experts in bf16 with sums 277 us (2.2 TB/s; vector units busy for
// 93 % of the cycles in which waves are there, 436 instructions per four rows), 16384 tokens on 1024 experts in f32
// with sums 30 us (2.3 TB/s, 61 %: a wave's one row is a chain of eight slots), in bf16 without 15 us (79 %); a wave
// per row with a ballot per value took 1052, 62 and 31 us.
#pragma once
#include <hip/hip_runtime.h>

#include <climits>

#include "kernels_moe.hpp"
#include "moe_device.hpp"

namespace nimble::moe {

namespace {

// ---- choice ----------------------------------------------------------------------------------

// The order of binary32 numbers as an order of whole numbers (of +0 and -0 the first is larger).
__device__ __forceinline__ int in_order(int bits) { return bits ^ ((bits >> 31) & 0x7FFFFFFF); }

// The order of two 16-bit numbers, in the halves of a word: sign and magnitude as a number (0 is 0), and back.
typedef short Pair __attribute__((ext_vector_type(2)));
__device__ __forceinline__ Pair pair_in_order(uint32_t w)
{
    const Pair sign = __builtin_bit_cast(Pair, w) >> 15;
    return (__builtin_bit_cast(Pair, w & 0x7FFF7FFFu) ^ sign) - sign;
}
__device__ __forceinline__ uint16_t half_of_order(int order)
{
    return static_cast<uint16_t>(order < 0 ? 0x8000 | -order : order);
}

// The key of a value: its order, with the column's bits in the place of the lowest.
__device__ __forceinline__ int key_of(float y, int cols, int column)
{
    return __builtin_amdgcn_bitop3_b32(in_order(bits_of(y)), cols, column, 0xBA);       // (a & ~b) | c
}

// Keys up to kNoKey stand for -inf: the order of binary32 -inf, and of a 16-bit one in the upper half, with
// any column below.
template <class D, bool ROUNDED>
constexpr int no_key()
{
    if constexpr (ROUNDED) return static_cast<int>(0x807FFFFFu);
    else return static_cast<int>(((0x10000u - D::kInfBits) << 16) | 0xFFFFu);
}

__device__ __forceinline__ void order(int &a, int &b)     // the larger one first
{
    const int hi = max(a, b), lo = min(a, b);
    a = hi;
    b = lo;
}

// Every place in a list is a constant of the program: keys stay in registers.

// Sorts a[A .. A+N-1], the largest first (odd-even merge sort: runs of P, compared Q apart).
template <int N, int A, int P = 1, int Q = 1, int S>
__device__ __forceinline__ void sort_keys(int (&a)[S])
{
    if constexpr (P < N) {
#pragma unroll
        for (int i = 0; i < N - Q; ++i) {
            const bool pair = i >= Q % P && (i - Q % P) / Q % 2 == 0 && i / (2 * P) == (i + Q) / (2 * P);
            if (pair) order(a[A + i], a[A + i + Q]);
        }
        if constexpr (Q > 1) sort_keys<N, A, P, Q / 2>(a);
        else sort_keys<N, A, 2 * P, 2 * P>(a);
    }
}

// Sorts a[A .. A+N-1] that rises and then falls, the largest first.
template <int N, int A, int D = N / 2, int S>
__device__ __forceinline__ void sort_bitonic(int (&a)[S])
{
    if constexpr (D >= 1) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if ((i & D) == 0) order(a[A + i], a[A + i + D]);
        sort_bitonic<N, A, D / 2>(a);
    }
}

// The N largest keys of a[A .. A+S-1], sorted, in a[A .. A+N-1]: of two sorted halves the larger ones of one
// list and the other backwards, sorted again.
template <int N, int A, int M, int S>
__device__ __forceinline__ void largest(int (&a)[S])
{
    if constexpr (M == N) {
        sort_keys<N, A>(a);
    } else {
        largest<N, A, M / 2>(a);
        largest<N, A + M / 2, M / 2>(a);
#pragma unroll
        for (int i = 0; i < N; ++i) a[A + i] = max(a[A + i], a[A + M / 2 + N - 1 - i]);
        sort_bitonic<N, A>(a);
    }
}

struct Choice {
    int slot;                    // key of the lane's slot; kNoKey or less: there is none
    int top;                     // the largest key of the row, in all lanes
    bool close;                  // keys do not tell the order of two slots
    bool unsure;                 // keys do not tell the last slot
};

// Lanes that are number R of their group.
template <int L>
constexpr uint64_t lanes_at(int r)
{
    uint64_t m = 0;
    for (int i = r; i < kWave; i += L) m |= 1ull << i;
    return m;
}

// Slot R: the largest head of all lists in key[0 .. N-1] is taken, and its list moves up.
template <int L, int V, int KL, int N, int R, bool ROUNDED, int NONE>
__device__ __forceinline__ void take(int (&key)[V], int top_k, int mine, int before, Choice &c)
{
    constexpr int kCols = L * V - 1;
    if (R > top_k || (R == top_k && !ROUNDED)) return;
    const int head = key[0] | mine;
    int best;
    if constexpr (L == kWave) best = wave_max(head);
    else best = group_max<L>(head);
    if constexpr (R == 0) c.top = best;
    bool same = false;
    if constexpr (ROUNDED && R > 0) same = ((best ^ before) & ~kCols) == 0 && best > NONE;
    if (R == top_k) {
        c.unsure = same;
        if constexpr (N < V) c.unsure = c.unsure || key[0] == INT_MIN;   // a list that ends too early
        return;
    }
    if constexpr (R < KL) {
        c.close = c.close || same;
        c.slot = __builtin_amdgcn_inverse_ballot_w64(lanes_at<L>(R)) ? best : c.slot;
        const bool won = head == best;
        // (both values are read before one is picked: a pick between two places would make the list memory)
#pragma unroll
        for (int i = 0; i + 1 < N; ++i) {
            const int here = key[i], next = key[i + 1];
            if (i + R < KL) key[i] = won ? next : here;
        }
        if constexpr (N + R <= KL) key[N - 1] = won ? INT_MIN : key[N - 1];
        take<L, V, KL, N, R + 1, ROUNDED, NONE>(key, top_k, mine, best, c);
    }
}

// The top_k <= KL largest keys of every group, slot j's in lane j.  The keys are used up.
template <int L, int V, int KL, bool ROUNDED, int NONE>
__device__ __forceinline__ Choice choose(int (&key)[V], int top_k, int l)
{
    constexpr int N = V < KL ? V : KL;
    largest<N, 0, V>(key);
    // (the lists are done here: the compiler would put off their last steps into the slots that need them, and
    // keep twice the registers until then)
#pragma unroll
    for (int i = 0; i < N; ++i) key[i] = anew(key[i]);
    Choice c{NONE, NONE, false, false};
    take<L, V, KL, N, 0, ROUNDED, NONE>(key, top_k, ((L - 1) ^ l) * kRun, 0, c);    // (the lane's part of the column)
    return c;
}

// The right columns in the wrong order: every slot goes as many places down as slots are ahead of it by
// whole values y and columns.
template <int L>
__device__ __forceinline__ int by_value(int index, float y, int top_k, int lane)
{
    const int first = lane & ~(L - 1), l = lane & (L - 1);
    const int col = index >= 0 ? index : INT_MAX - kWave + l;
    int rank = 0;
    for (int r = 0; r < top_k; ++r) {
        const float other = __shfl(y, first + r);
        const int at = __shfl(col, first + r);
        rank += other > y || (other == y && at < col) ? 1 : 0;
    }
    // (lanes beyond the slots keep to themselves)
    return __builtin_amdgcn_ds_permute((first + (l < top_k ? rank : l)) * 4, index);
}

// The choice by whole values y (-inf: not to be chosen): column of slot l, or -1.
template <int L, int V>
__device__ __forceinline__ int choose_by_value(float (&y)[V], int top_k, int l)
{
    int index = -1;
    for (int r = 0; r < top_k; ++r) {
        float best = y[0];
#pragma unroll
        for (int j = 1; j < V; ++j) best = fmaxf(best, y[j]);
        best = group_max<L>(best);
        int col = INT_MIN;                               // the largest of -1 - column
#pragma unroll
        for (int j = 0; j < V; ++j) col = max(col, y[j] == best ? ~(column_of<L>(j) + l * kRun) : INT_MIN);
        col = ~group_max<L>(col);
        if (!(best > -kInf)) col = -1;                   // nothing left, or NaN
        if (l == r) index = col;
#pragma unroll
        for (int j = 0; j < V; ++j) y[j] = column_of<L>(j) + l * kRun == col ? -kInf : y[j];
    }
    return index;
}

// ---- rows ------------------------------------------------------------------------------------

// A bias as it is added: NaN counts as -inf and +inf as the largest number, so that the sum with -inf stays
// -inf; +0 for -0, so that zeros are alike.
__device__ __forceinline__ float bias_of(float b)
{
    return (b == b ? fminf(b, 3.402823466e38f) : -kInf) + 0.0f;
}

// y = x + bias, the order of the choice; without a bias -0 becomes +0, which equals it.
template <int L, int V>
__device__ __forceinline__ void add_bias(const RouteArgs &a, int l, int shape, const float (&x)[V], float (&y)[V])
{
    if (!a.bias) {
#pragma unroll
        for (int j = 0; j < V; ++j) y[j] = x[j] + 0.0f;
        return;
    }
    const int at = anew(l * kRun);
    if (shape != kSingle && a.bias_runs) {
        float4 b[V / kRun];
#pragma unroll
        for (int q = 0; q < V / kRun; ++q) {
            const int col = q * (L * kRun) + at;
            b[q] = *reinterpret_cast<const float4 *>(a.bias + (col < a.experts ? col : 0));
        }
#pragma unroll
        for (int q = 0; q < V / kRun; ++q) {
            y[q * kRun] = x[q * kRun] + bias_of(b[q].x);
            y[q * kRun + 1] = x[q * kRun + 1] + bias_of(b[q].y);
            y[q * kRun + 2] = x[q * kRun + 2] + bias_of(b[q].z);
            y[q * kRun + 3] = x[q * kRun + 3] + bias_of(b[q].w);
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            y[j] = x[j] + bias_of(a.bias[min(column_of<L>(j) + at, a.experts - 1)]);
    }
}

// A workgroup per chunk of rows, cut where a segment ends; probabilities are summed in registers,
// slots counted in LDS, and the waves' sums added in order at the end of every part.
template <class D, int L, int V, int KL, bool ROUNDED, bool SUMS>
__global__ __launch_bounds__(kRowWaves *kWave, waves_per_simd(V)) void k_route(RouteArgs a, int shape)
{
    constexpr int C = L * V, G = kWave / L, kCols = C - 1;
    constexpr int kSlots = L < 16 ? L : 16;              // lanes of a group that have slots
    extern __shared__ float lds[];
    float *sums = lds;                                   // [kRowWaves][C]
    int *hits = reinterpret_cast<int *>(lds + kRowWaves * C);
    int *routed = hits + C;                              // [kRowWaves]
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int l = lane & (L - 1), g = lane / L;
    const bool sigmoid = (a.flags & NIMBLE_MOE_SIGMOID) != 0;
    const bool renorm = (a.flags & NIMBLE_MOE_RENORM) != 0;
    constexpr int kNoKey = no_key<D, ROUNDED>();
    // (made anew, so that the compiler does not fold it into what it is multiplied with)
    const float nan = float_of(anew(0x7FC00000));
    // scores of all experts are wanted for sums and for weights that are divided by their sum
    const bool all_scores = SUMS || !(renorm || sigmoid);
    const int64_t first = static_cast<int64_t>(blockIdx.x) * a.rows.chunk;
    const int lo = static_cast<int>(first);
    const int hi = static_cast<int>(min(first + a.rows.chunk, static_cast<int64_t>(a.rows.tokens)));
    // Rows are read a pass ahead; the first ones before it is known which segment they are in.
    const auto *const logits = static_cast<const typename D::Raw *>(a.logits);
    RowOf<D, L, V> ahead;
    int ahead_of = lo + wave * G;
    ahead.load(logits + static_cast<int64_t>(min(ahead_of + g, hi - 1)) * a.stride, a.experts, l, shape);
    Segments segments(a.rows, lane);
    for (int s = segments.first(lo); s < a.rows.segments; ++s) {
        const int begin = segments.begin(s), from = max(lo, begin), to = min(hi, segments.end(s));
        if (begin >= hi) break;
        if (from >= to) continue;
        if constexpr (SUMS) {
            for (int c = threadIdx.x; c < C; c += kRowWaves * kWave) hits[c] = 0;
            __syncthreads();
        }
        float acc[V];
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] = 0.0f;
        int n = 0;
        for (int r0 = from + wave * G; r0 < to; r0 += kRowWaves * G) {
            const bool inside = r0 + g < to;
            const int64_t row = inside ? r0 + g : to - 1;       // (no group reads outside the part)
            const auto *const mine = logits + row * a.stride;
            const int top_k = anew_uniform(a.top_k);
            if (r0 != ahead_of) ahead.load(mine, a.experts, l, shape);
            RowOf<D, L, V> raw = ahead;
            if (r0 + kRowWaves * G < to) {
                ahead_of = r0 + kRowWaves * G;
                ahead.load(logits + static_cast<int64_t>(min(ahead_of + g, to - 1)) * a.stride, a.experts, l, shape);
            }
            const bool live = inside && (!a.keep || a.keep[row] != 0);
            raw.end_at(a.experts, l, shape);
            if (__ballot(live) != ~0ull) raw.drop(live);
            float x[V], logit, top = 0.0f;
            int index;
            bool bad = false;                                   // in one lane of a group, or in all of them
            if constexpr (ROUNDED) {
                float y[V];
                int key[V];
                raw.values(x);
                add_bias<L, V>(a, l, shape, x, y);
                const int cols = anew(kCols);
#pragma unroll
                for (int j = 0; j < V; ++j)
                    key[j] = key_of(y[j], cols, kCols ^ column_of<L>(j) ^ ((L - 1) * kRun));
                const Choice c = choose<L, V, KL, true, kNoKey>(key, top_k, anew(l));
                index = c.slot > kNoKey ? ~c.slot & kCols : -1;
                if (__ballot(c.unsure) != 0) {
                    add_bias<L, V>(a, l, shape, x, y);
                    index = choose_by_value<L, V>(y, top_k, l);
                }
                logit = index >= 0 ? D::up(mine[index]) : -kInf;
                if (__ballot(c.close && !c.unsure) != 0) {
                    // (in a wave that has chosen by value already, this changes nothing)
                    const float b = index >= 0 && a.bias ? bias_of(a.bias[index]) : 0.0f;
                    index = by_value<L>(index, logit + b, top_k, lane);
                    logit = index >= 0 ? D::up(mine[index]) : -kInf;
                }
                if (all_scores) {
                    // any shift near the largest logit does, so without a bias the largest key gives one
                    top = c.top > kNoKey ? float_of(in_order(c.top)) : -kInf;
                    if (a.bias || __ballot(top == -kInf || fabsf(top) <= 512.0f) != ~0ull) {
                        top = x[0];
#pragma unroll
                        for (int j = 1; j < V; ++j) top = fmaxf(top, x[j]);
                        top = group_max<L>(top);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < V; ++j) bad = bad || !(x[j] < kInf);
                }
            } else {
                int key[V];
                Pair low{0, 0};
#pragma unroll
                for (int w = 0; w < V / 2; ++w) {
                    const Pair u = pair_in_order(raw.word[w]);
                    const uint32_t both = __builtin_bit_cast(uint32_t, u);
                    key[2 * w] = static_cast<int>(both << 16 | (kCols ^ column_of<L>(2 * w) ^ ((L - 1) * kRun)));
                    key[2 * w + 1] = static_cast<int>((both & 0xFFFF0000u) |
                                                      (kCols ^ column_of<L>(2 * w + 1) ^ ((L - 1) * kRun)));
                    low = __builtin_elementwise_min(low, u);
                }
                const Choice c = choose<L, V, KL, false, kNoKey>(key, top_k, anew(l));
                index = c.slot > kNoKey ? ~c.slot & kCols : -1;
                logit = index >= 0 ? D::up(half_of_order(c.slot >> 16)) : -kInf;
                top = c.top > kNoKey ? D::up(half_of_order(c.top >> 16)) : -kInf;
                if (all_scores) raw.values(x);
                else bad = min(low.x, low.y) < -D::kInfBits || c.top >> 16 >= D::kInfBits;
            }
            const bool chosen = __shfl(index, lane & ~(L - 1)) >= 0;
            const Shifted by(shift_of(sigmoid, top));
            float inv = 0.0f;
            if (all_scores) {
                scores_of<V>(sigmoid, x, by);
                float sum = 0.0f;
#pragma unroll
                for (int j = 0; j < V; ++j) sum = sum + x[j];
                sum = group_sum<L>(sum);
                bad = !(sum == sum) || top == kInf;
                inv = __builtin_amdgcn_rcpf(sum);
            } else {
                const unsigned long long group = (L == kWave ? ~0ull : (1ull << (L & 63)) - 1) << (lane & ~(L - 1));
                bad = (__ballot(bad) & group) != 0;
            }
            float w;
            if (renorm) {
                const float t = group_max<kSlots>(logit);
                const float u = score_of(sigmoid, logit, Shifted(shift_of(sigmoid, t)));
                w = u * __builtin_amdgcn_rcpf(group_sum<kSlots>(u));
            } else {
                w = sigmoid ? sigmoid_of(logit) : by.exp(logit) * inv;
            }
            if (bad) index = -1;
            w = bad ? nan : (index < 0 ? 0.0f : w * a.scale);
            if (l < a.top_k && inside) {
                a.index[row * a.top_k + l] = index;
                a.weight[row * a.top_k + l] = w;
            }
            if constexpr (SUMS) {
                const float of_row = bad ? nan : (chosen ? inv : 0.0f);
#pragma unroll
                for (int j = 0; j < V; ++j) acc[j] = __builtin_fmaf(x[j], of_row, acc[j]);
                n += chosen && !bad ? 1 : 0;
                if (l < a.top_k && index >= 0) atomicAdd(&hits[index], 1);
            }
        }
        if constexpr (SUMS) {
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] = over_groups<L>(acc[j]);
            if (g == 0) {
#pragma unroll
                for (int j = 0; j < V; ++j) sums[wave * C + column_of<L>(j) + l * kRun] = acc[j];
            }
            int m = 0;
#pragma unroll
            for (int i = 0; i < G; ++i) m += __builtin_amdgcn_readlane(n, i * L);
            if (lane == 0) routed[wave] = m;
            __syncthreads();
            const int64_t part = static_cast<int64_t>(blockIdx.x) + s;
            for (int c = threadIdx.x; c < a.experts; c += kRowWaves * kWave) {
                float t = sums[c];
#pragma unroll
                for (int w = 1; w < kRowWaves; ++w) t = t + sums[w * C + c];
                a.part_prob[part * a.experts + c] = t;
                a.part_count[part * a.experts + c] = hits[c];
            }
            if (threadIdx.x == 0) {
                int t = 0;
                for (int w = 0; w < kRowWaves; ++w) t += routed[w];
                a.part_routed[part] = t;
            }
            __syncthreads();
        }
    }
}

template <class D, int L, int V, int KL, bool ROUNDED>
hipError_t run(const RouteArgs &a, hipStream_t stream)
{
    const int shape = shape_of(a.logits, a.stride, a.experts, L * V, sizeof(typename D::Raw));
    const dim3 grid(a.rows.chunks), block(kRowWaves * kWave);
    if (a.counts) {
        const size_t lds = sizeof(float) * ((kRowWaves + 1) * L * V + kRowWaves);
        k_route<D, L, V, KL, ROUNDED, true><<<grid, block, lds, stream>>>(a, shape);
    } else {
        k_route<D, L, V, KL, ROUNDED, false><<<grid, block, 0, stream>>>(a, shape);
    }
    return hipGetLastError();
}

template <class D, int L, int V, int KL>
hipError_t run(const RouteArgs &a, hipStream_t stream)
{
    if constexpr (!D::kWide)
        if (!a.bias) return run<D, L, V, KL, false>(a, stream);
    return run<D, L, V, KL, true>(a, stream);
}

// Lists of one more than top_k where there are few: a lane that holds all the chosen ones of a row cannot
// tell what comes next.
template <class D, int L, int V>
hipError_t run(const RouteArgs &a, hipStream_t stream)
{
    if constexpr (L > 8)
        if (a.top_k > 8) return run<D, L, V, 16>(a, stream);
    if (a.top_k <= 3) return run<D, L, V, 4>(a, stream);
    return run<D, L, V, 8>(a, stream);
}

}  // namespace

// Sixteen values to a lane where there are enough; as few lanes to a row as that makes, but as many as there
// are slots.
template <class D>
hipError_t route_rows(const RouteArgs &a, hipStream_t stream)
{
    if (a.experts <= 128 && a.top_k <= 8) {
        if (a.experts <= 32) return run<D, 8, 4>(a, stream);
        if (a.experts <= 64) return run<D, 8, 8>(a, stream);
        return run<D, 8, 16>(a, stream);
    }
    if (a.experts <= 64) return run<D, 16, 4, 16>(a, stream);
    if (a.experts <= 128) return run<D, 16, 8, 16>(a, stream);
    if (a.experts <= 256) return run<D, 16, 16>(a, stream);
    if (a.experts <= 512) return run<D, 32, 16>(a, stream);
    if (a.experts <= 1024) return run<D, 64, 16>(a, stream);
    return run<D, 64, 32>(a, stream);
}

}  // namespace nimble::moe
