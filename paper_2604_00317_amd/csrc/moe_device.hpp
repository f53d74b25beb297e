// Device code shared by the routing kernels: element types, reductions over lanes, segments, scores.
#pragma once
#include <hip/hip_runtime.h>

#include <climits>

#include "../../include/nimble_moe.h"
#include "kernels_moe.hpp"
#include "wave_ops.hpp"

namespace nimble::moe {

namespace {

constexpr float kInf = __builtin_inff();
constexpr int kRowWaves = 8;         // waves of a workgroup that works on rows

// Waves a SIMD should hold: two workgroups to a CU, where 128 registers do.
constexpr int waves_per_simd(int values) { return values <= 16 ? 4 : 2; }

// ---- element types ---------------------------------------------------------------------------

struct F32 {
    using Raw = float;
    static constexpr bool kWide = true;      // its bits do not leave room for a column
    static __device__ __forceinline__ float up(float v) { return v; }
    static __device__ __forceinline__ float down(float v) { return v; }
};
struct F16 {
    using Raw = uint16_t;
    static constexpr bool kWide = false;
    static constexpr int kInfBits = 0x7C00;
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
    static constexpr bool kWide = false;
    static constexpr int kInfBits = 0x7F80;
    static __device__ __forceinline__ float up(uint16_t v)
    {
        return __builtin_bit_cast(float, static_cast<uint32_t>(v) << 16);
    }
    static __device__ __forceinline__ uint16_t down(float v)
    {
        return __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
    }
};

// ---- reductions over lanes -------------------------------------------------------------------

struct TwoI32 {
    int a, b;
};
__device__ __forceinline__ TwoI32 both_rows(int v)           // of a pair of rows of 16 lanes
{
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return {static_cast<int>(r[0]), static_cast<int>(r[1])};
}
__device__ __forceinline__ TwoI32 both_halves(int v)         // of the wave
{
    const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return {static_cast<int>(r[0]), static_cast<int>(r[1])};
}
__device__ __forceinline__ int bits_of(float v) { return __builtin_bit_cast(int, v); }
__device__ __forceinline__ float float_of(int v) { return __builtin_bit_cast(float, v); }
template <int CTRL>
__device__ __forceinline__ float dpp_f32(float v)
{
    return float_of(dpp_i32<CTRL>(bits_of(v)));
}

// Over aligned groups of L lanes (8 to 64); the same bits in all lanes of a group.
template <int L>
__device__ __forceinline__ int group_max(int v)
{
    v = max(v, dpp_i32<kDppXor1>(v));
    v = max(v, dpp_i32<kDppXor2>(v));
    v = max(v, dpp_i32<kDppHalfMirror>(v));
    if constexpr (L > 8) v = max(v, dpp_i32<kDppMirror>(v));
    if constexpr (L > 16) {
        const TwoI32 r = both_rows(v);
        v = max(r.a, r.b);
    }
    if constexpr (L > 32) {
        const TwoI32 h = both_halves(v);
        v = max(h.a, h.b);
    }
    return v;
}
// Over the wave, as a scalar: rows pass theirs on to the last one, half the instructions of an exchange.
__device__ __forceinline__ int wave_max(int v)
{
    v = group_max<16>(v);
    v = max(v, __builtin_amdgcn_update_dpp(INT_MIN, v, 0x142, 0xA, 0xF, false));   // row_bcast:15
    v = max(v, __builtin_amdgcn_update_dpp(INT_MIN, v, 0x143, 0xC, 0xF, false));   // row_bcast:31
    return __builtin_amdgcn_readlane(v, kWave - 1);
}
template <int L>
__device__ __forceinline__ float group_max(float v)
{
    v = fmaxf(v, dpp_f32<kDppXor1>(v));
    v = fmaxf(v, dpp_f32<kDppXor2>(v));
    v = fmaxf(v, dpp_f32<kDppHalfMirror>(v));
    if constexpr (L > 8) v = fmaxf(v, dpp_f32<kDppMirror>(v));
    if constexpr (L > 16) {
        const TwoI32 r = both_rows(bits_of(v));
        v = fmaxf(float_of(r.a), float_of(r.b));
    }
    if constexpr (L > 32) {
        const TwoI32 h = both_halves(bits_of(v));
        v = fmaxf(float_of(h.a), float_of(h.b));
    }
    return v;
}
template <int L>
__device__ __forceinline__ float group_sum(float v)
{
    v = v + dpp_f32<kDppXor1>(v);
    v = v + dpp_f32<kDppXor2>(v);
    v = v + dpp_f32<kDppHalfMirror>(v);
    if constexpr (L > 8) v = v + dpp_f32<kDppMirror>(v);
    if constexpr (L > 16) {
        const TwoI32 r = both_rows(bits_of(v));
        v = float_of(r.a) + float_of(r.b);
    }
    if constexpr (L > 32) {
        const TwoI32 h = both_halves(bits_of(v));
        v = float_of(h.a) + float_of(h.b);
    }
    return v;
}
constexpr int kDppRotate8 = 0x128;                           // row_ror:8, the other half of a row of 16

// The sum of a value over the groups of a wave, by lane of a group; the same bits in all groups.
template <int L>
__device__ __forceinline__ float over_groups(float v)
{
    if constexpr (L < 16) v = v + dpp_f32<kDppRotate8>(v);
    if constexpr (L < 32) {
        const TwoI32 r = both_rows(bits_of(v));
        v = float_of(r.a) + float_of(r.b);
    }
    if constexpr (L < 64) {
        const TwoI32 h = both_halves(bits_of(v));
        v = float_of(h.a) + float_of(h.b);
    }
    return v;
}

// ---- scores ----------------------------------------------------------------------------------

constexpr float kLog2E = 1.44269504f;

// exp by the hardware's exp2: off by 2^-23 |x| and a step or so, relative; results below 2^-126 are 0
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2E); }

// 1 / (1 + exp(-x)); 0 below -88 or so
__device__ __forceinline__ float sigmoid_of(float x)
{
    return __builtin_amdgcn_rcpf(1.0f + exp_of(-x));
}

// exp(x - shift) and exp(shift - x) up to a factor that is the same for all x (2 to the rounding of `at`,
// shift * log2(e)), in a multiply-add and an exp2.  far(): `at` is so large that the factor may leave the range,
// or no number.
struct Shifted {
    float shift, at;
    __device__ __forceinline__ explicit Shifted(float s) : shift(s), at(s * kLog2E) {}
    __device__ __forceinline__ bool far() const { return !(fabsf(at) <= 16777216.0f); }
    __device__ __forceinline__ float near_exp(float x) const
    {
        return __builtin_amdgcn_exp2f(__builtin_fmaf(x, kLog2E, -at));
    }
    __device__ __forceinline__ float exp(float x) const { return far() ? exp_of(x - shift) : near_exp(x); }
    // 1 / (exp(shift) + exp(shift - x)), the factor in both terms; `one` is near_one()
    __device__ __forceinline__ float near_one() const { return __builtin_amdgcn_exp2f(at); }
    __device__ __forceinline__ float near_sigmoid(float x, float one) const
    {
        return __builtin_amdgcn_rcpf(one + __builtin_amdgcn_exp2f(__builtin_fmaf(x, -kLog2E, at)));
    }
    __device__ __forceinline__ float sigmoid(float x) const
    {
        return far() ? __builtin_amdgcn_rcpf(exp_of(shift) + exp_of(shift - x)) : near_sigmoid(x, near_one());
    }
};

// Scores of a row are summed and compared as s(x) exp(-shift), so that the largest is about one.  Softmax: shift is
// the largest logit.  Sigmoid: that logit where it is below 0, else 0 (sigmoids as they are); a row of low logits
// keeps the ratios of its scores, where sigmoids of logits below -87 would be zeros.
__device__ __forceinline__ float shift_of(bool sigmoid, float top)
{
    return top == -kInf ? 0.0f : sigmoid ? fminf(top, 0.0f) : top;
}
__device__ __forceinline__ float score_of(bool sigmoid, float x, const Shifted &by)
{
    return sigmoid ? by.sigmoid(x) : by.exp(x);
}
// All scores of a row's lane; the choice between forms is the wave's.
template <int V>
__device__ __forceinline__ void scores_of(bool sigmoid, float (&x)[V], const Shifted &by)
{
    if (__ballot(by.far()) != 0) {
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = score_of(sigmoid, x[j], by);
    } else if (sigmoid) {
        const float one = by.near_one();
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = by.near_sigmoid(x[j], one);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = by.near_exp(x[j]);
    }
}

// ---- segments --------------------------------------------------------------------------------

// The segments' offsets, 64 of them at a time in the lanes of a wave: one round trip to memory finds the
// segment of a row and its ends where there are up to 63 segments.  All lanes are active in every call, and
// all waves of a workgroup get the same answers.
class Segments {
public:
    __device__ __forceinline__ Segments(const Rows &rows, int lane) : r(rows), lane(lane) {}

    // The first segment that ends behind `row` (the number of segments, if none does).
    __device__ __forceinline__ int first(int row)
    {
        if (!r.seg_ptr) return 0;
        if (r.segments >= kWave) {                   // 64 tries at a time
            int at = 0, n = r.segments;
            while (n > 0) {
                const int step = (n + kWave - 1) / kWave;
                const int s = at + lane * step + step - 1;
                const unsigned long long hit = __ballot(s >= at + n || r.seg_ptr[s + 1] > row);
                if (hit == 0) return at + n;
                const int to = at + (__ffsll(hit) - 1) * step;
                n = min(step - 1, at + n - to);
                at = to;
            }
            fetch(at);
            return at;
        }
        fetch(0);
        const unsigned long long hit = __ballot(lane >= 1 && lane <= r.segments && offsets > row);
        return hit == 0 ? r.segments : __ffsll(hit) - 2;
    }
    // The first segment from s on that has more than `rows` rows (the number of segments, if there is none that
    // begins before row `end`), 63 at a time.
    __device__ __forceinline__ int longer(int s, int rows, int end)
    {
        if (!r.seg_ptr) return s == 0 && r.tokens <= rows ? r.segments : s;
        while (s < r.segments) {
            if (s + 1 - base >= kWave) fetch(s);
            if (__builtin_amdgcn_readlane(offsets, s - base) >= end) break;
            const int next = __shfl_down(offsets, 1);
            const unsigned long long hit = __ballot(lane >= s - base && lane < kWave - 1 && base + lane < r.segments &&
                                                    next - offsets > rows);
            if (hit != 0) return base + __ffsll(hit) - 1;
            s = min(base + kWave - 1, r.segments);
        }
        return r.segments;
    }
    __device__ __forceinline__ int begin(int s) { return r.seg_ptr ? offset(s) : 0; }
    __device__ __forceinline__ int end(int s) { return r.seg_ptr ? offset(s + 1) : r.tokens; }

private:
    __device__ __forceinline__ void fetch(int s)
    {
        base = s;
        offsets = min(max(r.seg_ptr[min(s + lane, r.segments)], 0), r.tokens);
    }
    __device__ __forceinline__ int offset(int s)
    {
        if (s - base >= kWave) fetch(s - 1);
        return __builtin_amdgcn_readlane(offsets, s - base);
    }
    const Rows &r;
    int lane, base = 0, offsets = 0;
};

// ---- rows in lanes ---------------------------------------------------------------------------

// A row lies in a group of L lanes (8 to 64), V values per lane in runs of W neighbours (one load each): lane
// l of the group has columns q * L W + l W + 0 .. W-1 for q = 0 .. V/W - 1.  A wave holds 64/L rows.
constexpr int kRun = 4;

template <class D, int W>
struct alignas(sizeof(typename D::Raw) * W) Run {
    typename D::Raw v[W];
};

// Column of value j without the lane's part, l * kRun.
template <int L>
constexpr int column_of(int j) { return (j / kRun) * (L * kRun) + j % kRun; }

// The value, but where the compiler cannot see what it depends on: what is worked out from it inside a
// loop stays there, where a dozen comparisons kept over the loop would take all scalar registers.
__device__ __forceinline__ int anew(int v)
{
    asm volatile("" : "+v"(v));
    return v;
}
__device__ __forceinline__ int anew_uniform(int v)
{
    asm volatile("" : "+s"(v));
    return v;
}

// How a row is read and written: kFull, its runs fill the lanes and are aligned to their size; kWhole, it is
// made of such runs, but does not fill the lanes; kSingle, value by value.
enum Shape : int { kFull, kWhole, kSingle };

// A row's values as they are read: binary32 one by one, 16-bit ones in pairs.  Columns beyond the row's end
// come as -inf, like masked ones.  (No read waits for a branch: lanes without a column read one that is there.)
template <class D, int L, int V>
struct RowOf {
    static constexpr int kPer = D::kWide ? 1 : 2;            // values of a word
    static constexpr int kWords = V / kPer;
    uint32_t word[kWords];

    static constexpr uint32_t none()
    {
        if constexpr (D::kWide) return 0xFF800000u;
        else return (0x8000u | D::kInfBits) * 0x10001u;
    }
    __device__ __forceinline__ void load(const typename D::Raw *row, int experts, int l, int shape)
    {
        const int at = anew(l * kRun);
        if (shape == kFull) {
#pragma unroll
            for (int q = 0; q < V / kRun; ++q)
                put(q, *reinterpret_cast<const Run<D, kRun> *>(row + q * (L * kRun) + at));
        } else if (shape == kWhole) {
#pragma unroll
            for (int q = 0; q < V / kRun; ++q) {
                const int col = q * (L * kRun) + at;
                put(q, *reinterpret_cast<const Run<D, kRun> *>(row + (col < experts ? col : 0)));
            }
        } else {
            typename D::Raw r[V];
#pragma unroll
            for (int j = 0; j < V; ++j) r[j] = row[min(column_of<L>(j) + at, experts - 1)];
#pragma unroll
            for (int w = 0; w < kWords; ++w) {
                uint32_t v;
                if constexpr (D::kWide) {
                    v = static_cast<uint32_t>(bits_of(r[w]));
                    v = column_of<L>(w) + at < experts ? v : none();
                } else {
                    const uint32_t a = r[2 * w], b = r[2 * w + 1], no = none() & 0xFFFFu;
                    v = (column_of<L>(2 * w) + at < experts ? a : no) |
                        (column_of<L>(2 * w + 1) + at < experts ? b : no) << 16;
                }
                word[w] = v;
            }
        }
    }
    // What load() leaves of columns beyond the row's end, once the values are there: reading ahead does not
    // wait for them.
    __device__ __forceinline__ void end_at(int experts, int l, int shape)
    {
        if (shape != kWhole) return;
        const int at = anew(l * kRun);
#pragma unroll
        for (int w = 0; w < kWords; ++w) word[w] = column_of<L>(w * kPer) - w * kPer % kRun + at < experts ? word[w] : none();
    }
    __device__ __forceinline__ void drop(bool keep)
    {
#pragma unroll
        for (int w = 0; w < kWords; ++w) word[w] = keep ? word[w] : none();
    }
    __device__ __forceinline__ float value(int j) const
    {
        if constexpr (D::kWide) return float_of(static_cast<int>(word[j]));
        else return D::up(static_cast<uint16_t>(word[j / 2] >> (j % 2 * 16)));
    }
    __device__ __forceinline__ void values(float (&x)[V]) const
    {
#pragma unroll
        for (int j = 0; j < V; ++j) x[j] = value(j);
    }

private:
    __device__ __forceinline__ void put(int q, const Run<D, kRun> &r)
    {
        constexpr int kWordsOfRun = kRun / kPer;
        struct Words {
            uint32_t w[kWordsOfRun];
        };
        const Words words = __builtin_bit_cast(Words, r);
#pragma unroll
        for (int i = 0; i < kWordsOfRun; ++i) word[q * kWordsOfRun + i] = words.w[i];
    }
};

template <class D, int L, int V>
__device__ __forceinline__ void store_row(typename D::Raw *row, int experts, int l, int shape,
                                          const float (&x)[V])
{
    const int at = anew(l * kRun);
    if (shape != kSingle) {
#pragma unroll
        for (int q = 0; q < V / kRun; ++q) {
            const int col = q * (L * kRun) + at;
            Run<D, kRun> r;
#pragma unroll
            for (int i = 0; i < kRun; ++i) r.v[i] = D::down(x[q * kRun + i]);
            if (col < experts) *reinterpret_cast<Run<D, kRun> *>(row + col) = r;
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (column_of<L>(j) + at < experts) row[column_of<L>(j) + at] = D::down(x[j]);
    }
}

inline int shape_of(const void *base, int64_t stride, int experts, int columns, size_t bytes)
{
    const bool aligned = reinterpret_cast<uintptr_t>(base) % (kRun * bytes) == 0 && stride % kRun == 0;
    if (!aligned || experts % kRun != 0) return kSingle;
    return experts == columns ? kFull : kWhole;
}

}  // namespace

}  // namespace nimble::moe
