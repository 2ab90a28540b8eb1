// Sampling of one token per row of logits: temperature, top-k, top-p, min-p, and a race of given
// exponential numbers.
//
// The race needs no prefix sums: of independent E_j ~ Exp(1), E_j / p_j is least at j with
// probability p_j, so the token is the largest y_j - log E_j over what is kept, and neither the
// normalisation nor the order of addition can move it.
//
// What top-k and top-p keep are the elements above a threshold in the order (logit falling, index
// rising). The general way to it is a descent through the 32-bit keys of the logits, eight bits a
// level: a histogram of the elements that share the prefix, by count for top-k, by mass for top-p,
// names the next eight bits. Masses are integers (multiples of 2^-38 of the largest weight), so
// that LDS atomics add them in any order to the same sum.
#pragma once

#include "rlcs_softmax.h"

namespace rlcs {

struct SampleArgs {
    const void* logits;
    const float* noise;
    const float* temperature;
    const int32_t* top_k;
    const float *top_p, *min_p;
    int32_t* tokens;
    float* logp;
    int64_t M, V, ld, ld_noise;
    float all_temperature, all_top_p, all_min_p;
    int32_t all_top_k;
};

constexpr double kMassUnit = 274877906944.0;  // 2^38: 2^24 elements of weight 1 stay below 2^63
constexpr int kDigits = 256;

// A row's settings, and its largest logit.
struct SampleRow {
    float temperature, top_p, min_p;
    int64_t top_k;  // >= V: all
};

__device__ __forceinline__ SampleRow sample_row(const SampleArgs& a, int64_t row) {
    SampleRow r;
    r.temperature = a.temperature ? a.temperature[row] : a.all_temperature;
    r.top_p = a.top_p ? a.top_p[row] : a.all_top_p;
    r.min_p = a.min_p ? a.min_p[row] : a.all_min_p;
    const int32_t k = a.top_k ? a.top_k[row] : a.all_top_k;
    r.top_k = k > 0 ? k : a.V;
    return r;
}

// The best of (key, index) pairs, the lower index among equal keys, as one integer to maximise.
__device__ __forceinline__ uint64_t race_entry(uint32_t key, uint32_t index) {
    return (uint64_t(key) << 32) | uint32_t(~index);
}
__device__ __forceinline__ uint32_t race_index(uint64_t e) { return ~uint32_t(e); }

__device__ __forceinline__ uint64_t max_lanes(uint64_t v) {
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const uint64_t o = __shfl_xor(v, d);
        v = o > v ? o : v;
    }
    return v;
}
// Over the workgroup; every lane has the result. `slots`: one word a wave.
template <int W>
__device__ __forceinline__ uint64_t max_group(uint64_t v, uint64_t* slots) {
    v = max_lanes(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
    __syncthreads();
    v = slots[0];
#pragma unroll
    for (int i = 1; i < W; ++i) v = slots[i] > v ? slots[i] : v;
    return v;
}
template <int W>
__device__ __forceinline__ float sum_group(float v, uint64_t* slots) {
    v = sum_lanes(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = __float_as_uint(v);
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) v += __uint_as_float(uint32_t(slots[i]));
    return v;
}

// The digit at which the bins' sum from the highest digit down first reaches `target` (>= 1), what
// lies above it and its own bin; digit -1 if the whole sum does not. By every wave for itself.
struct Crossing {
    int digit;
    uint64_t above, own;
};
__device__ __forceinline__ Crossing find_crossing(const uint64_t* bins, uint64_t target) {
    const int lane = threadIdx.x & 63;
    uint64_t b[4], sum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        b[i] = bins[kDigits - 1 - (4 * lane + i)];
        sum += b[i];
    }
    uint64_t upto = sum;  // inclusive scan over the lanes
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        const uint64_t o = __shfl_up(upto, d);
        if (lane >= d) upto += o;
    }
    const uint64_t reached = __ballot(upto >= target);
    if (!reached) return Crossing{-1, 0, 0};
    const int first = __ffsll((unsigned long long)reached) - 1;
    uint64_t above = upto - sum, own = 0;
    int at = 4 * lane;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        own = b[i];
        at = 4 * lane + i;
        if (above + own >= target) break;
        above += own;
    }
    return Crossing{kDigits - 1 - __shfl(at, first), __shfl(above, first), __shfl(own, first)};
}

// What of a row is kept: keys above `key`, and the first `quota` of those equal to it. `cut`: there
// are more equal ones than that.
struct Threshold {
    uint32_t key;
    uint64_t quota;
    bool cut;
};

// A row in memory, its weights' scale.
template <typename DT>
struct RowView {
    const DT* x;
    int64_t V;
    Scale scale;
    __device__ __forceinline__ float logit(int64_t j) const {
        const float v = widen(x[j]);
        return v == v ? v : kNegInf;
    }
    __device__ __forceinline__ float log2_weight(float v) const { return scale.log2_weight(v); }
    __device__ __forceinline__ uint64_t mass(float v) const {
        return uint64_t(double(exp2_fast(log2_weight(v))) * kMassUnit);
    }
};

// The k-th largest logit (k < V).
template <typename DT, int W>
__device__ Threshold descend_count(const RowView<DT>& r, uint64_t k, uint64_t* bins) {
    const int tid = threadIdx.x;
    uint32_t prefix = 0;
    uint64_t want = k, equal = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        for (int i = tid; i < kDigits; i += W * kWave) bins[i] = 0;
        __syncthreads();
        for (int64_t j = tid; j < r.V; j += W * kWave) {
            const float v = r.logit(j);
            const uint32_t key = order_key(v);
            if (v > kNegInf && (shift == 24 || (key >> (shift + 8)) == (prefix >> (shift + 8))))
                atomicAdd(reinterpret_cast<unsigned long long*>(&bins[(key >> shift) & 255u]), 1ull);
        }
        __syncthreads();
        const Crossing c = find_crossing(bins, want);
        if (c.digit < 0) return Threshold{0u, ~0ull, false};  // fewer than k are not masked
        prefix |= uint32_t(c.digit) << shift;
        want -= c.above;
        equal = c.own;
    }
    return Threshold{prefix, want, want < equal};
}

// The element of what `t` keeps before which the mass first is p of the whole.
template <typename DT, int W>
__device__ Threshold descend_mass(const RowView<DT>& r, Threshold t, float p, uint64_t* bins) {
    const int tid = threadIdx.x;
    uint32_t prefix = 0;
    uint64_t target = 0, equal = 0;
    const uint64_t tied = t.key ? r.mass(key_value(t.key)) * t.quota : 0;  // (no threshold: key 0)
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        for (int i = tid; i < kDigits; i += W * kWave) bins[i] = 0;
        __syncthreads();
        auto shares = [&](uint32_t key) { return shift == 24 || (key >> (shift + 8)) == (prefix >> (shift + 8)); };
        auto add = [&](uint32_t key, uint64_t m) {
            atomicAdd(reinterpret_cast<unsigned long long*>(&bins[(key >> shift) & 255u]), (unsigned long long)m);
        };
        for (int64_t j = tid; j < r.V; j += W * kWave) {
            const float v = r.logit(j);
            const uint32_t key = order_key(v);
            if (v > kNegInf && key > t.key && shares(key)) add(key, r.mass(v));
        }
        if (tid == 0 && t.key && shares(t.key)) add(t.key, tied);
        __syncthreads();
        if (shift == 24) {
            uint64_t all = 0;
            for (int i = tid & 63; i < kDigits; i += kWave) all += bins[i];
#pragma unroll
            for (int d = 1; d < kWave; d <<= 1) all += __shfl_xor(all, d);
            const double want = ceil(double(p) * double(all));
            target = want < 1.0 ? 1 : uint64_t(want);
            if (target > all) target = all;
        }
        const Crossing c = find_crossing(bins, target);
        prefix |= uint32_t(c.digit) << shift;
        target -= c.above;
        equal = c.own;
    }
    const uint64_t one = r.mass(key_value(prefix));
    const uint64_t quota = (target + one - 1) / one, count = equal / one;
    return Threshold{prefix, quota, quota < count || (prefix == t.key && t.cut)};
}

// One row per workgroup of W waves, element by element: any alignment, length and settings.
template <typename DT, int W>
__global__ __launch_bounds__(W * kWave) void sample_rows_kernel(SampleArgs a) {
    __shared__ uint64_t s_bins[kDigits];
    __shared__ uint64_t s_slots[W];
    constexpr int kLanes = W * kWave;
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    RowView<DT> r{reinterpret_cast<const DT*>(a.logits) + row * a.ld, a.V, {}};
    const float* noise = a.noise ? a.noise + row * a.ld_noise : nullptr;

    uint64_t best = 0;
    for (int64_t j = tid; j < a.V; j += kLanes) {
        const uint64_t e = race_entry(order_key(r.logit(j)), uint32_t(j));
        best = e > best ? e : best;
    }
    best = max_group<W>(best, s_slots);
    const float top = r.logit(race_index(best));
    const SampleRow s = sample_row(a, row);
    const float c = kLog2e / s.temperature;
    const bool greedy = !(s.temperature > 0.f) || !(c < __builtin_inff());
    r.scale = scale_of(top, c);
    if (top == kNegInf || greedy) {
        if (tid == 0) {
            a.tokens[row] = top == kNegInf ? -1 : int32_t(race_index(best));
            if (a.logp) a.logp[row] = top == kNegInf ? kNegInf : 0.f;
        }
        return;
    }
    Threshold t{0u, ~0ull, false};
    if (s.top_k < a.V) t = descend_count<DT, W>(r, uint64_t(s.top_k), s_bins);
    if (s.top_p < 1.f) t = descend_mass<DT, W>(r, t, s.top_p, s_bins);
    // (the largest logit is always kept)
    const float least = s.min_p > 0.f ? fminf(s.min_p, 1.f) * exp2_fast(r.log2_weight(top)) : 0.f;

    float z = 0.f;
    uint64_t winner = 0, ties = 0;
    for (int64_t j0 = 0; j0 < a.V; j0 += kLanes) {
        const int64_t j = j0 + tid;
        const float v = j < a.V ? r.logit(j) : kNegInf;
        const uint32_t key = order_key(v);
        bool keep = v > kNegInf && key >= t.key;
        if (t.cut) {  // the first `quota` of the equal ones, by index
            const bool tie = keep && key == t.key;
            const uint64_t votes = __ballot(tie);
            __syncthreads();
            if (lane == 0) s_slots[wave] = __popcll(votes);
            __syncthreads();
            uint64_t before = ties + __popcll(votes & ((1ull << lane) - 1));
#pragma unroll
            for (int i = 0; i < W; ++i) {
                if (i < wave) before += s_slots[i];
                ties += s_slots[i];
            }
            keep = keep && (!tie || before < t.quota);
        }
        if (!keep) continue;
        const float u = r.log2_weight(v), w = exp2_fast(u);
        if (!(w >= least)) continue;
        z += w;
        const float score = noise ? u - log2_fast(noise[j]) : v;
        const uint64_t e = race_entry(order_key(score), uint32_t(j));
        winner = e > winner ? e : winner;
    }
    winner = max_group<W>(winner, s_slots);
    z = sum_group<W>(z, s_slots);
    if (tid == 0) {
        const uint32_t token = race_index(winner);
        a.tokens[row] = int32_t(token);
        if (a.logp) a.logp[row] = kLn2 * (r.log2_weight(r.logit(token)) - log2_fast(z));
    }
}

}  // namespace rlcs
