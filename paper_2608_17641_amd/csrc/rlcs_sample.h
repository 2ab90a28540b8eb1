// Sampling of one token per row of logits: temperature, top-k, top-p, min-p, and a race of given
// exponential numbers.
//
// The race needs no prefix sums: of independent E_j ~ Exp(1), E_j / p_j is least at j with
// probability p_j, so the token is the largest y_j - log E_j over what is kept, and neither the
// normalisation nor the order of addition can move it.
//
// What top-k and top-p keep are the elements above a threshold in the order (logit falling, index
// rising). Each row takes the shortest way to it:
//   no filter    one pass: the race and the sum of weights.
//   short rows   one wave a row: halving the range of keys, in registers.
//   few kept     (a top-k of at most kFewest) the k-th largest of the lanes' maxima is a lower bound of the
//                k-th logit; the elements from there on, little more than k, are ranked by comparing
//                each with each.
//   a mass       (top-p without top-k) a histogram of masses over 1/64 of an octave each; its
//                crossing bin is ranked the same way, everything above it is kept.
//   otherwise    a descent through the 32-bit keys of the logits, eight bits a level, by histograms of
//                counts or masses.
// Masses in histograms are integers (multiples of 2^-38 of the largest weight), so that LDS atomics
// add them in any order to the same sum.
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

// log2(e) / temperature, or infinity for a temperature of 0 (or none, or too small to divide by). Not 0 for
// one of infinity: -inf times that has to stay -inf.
__device__ __forceinline__ float sample_scale(const SampleRow& s) {
    return s.temperature > 0.f ? fmaxf(kLog2e / s.temperature, 1.1754944e-38f) : kInf;
}

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

// Logarithm of a random number. v_log_f32 takes what lies below 2^-126 for 0: those are scaled first.
__device__ __forceinline__ float noise_log2(float e) {
    const bool small = e < 0x1p-126f;
    return log2_fast(small ? e * 0x1p32f : e) - (small ? 32.f : 0.f);
}
// Whether a race with the plain logarithm was won by such a number: by a score of +inf. It is run again then (a comparison
// a row, where the scaling takes five operations a logit: 8192 x 1000 12.3 us against 13.0).
__device__ __forceinline__ bool won_by_small(uint64_t winner) { return uint32_t(winner >> 32) == 0xff800000u; }
template <int L>
__device__ __forceinline__ uint64_t max_lanes(uint64_t v) {
#pragma unroll
    for (int d = 1; d < L; d <<= 1) {
        const uint64_t o = __shfl_xor(v, d);
        v = o > v ? o : v;
    }
    return v;
}
// Over the workgroup; every lane has the result. `slots`: one word a wave.
template <int W>
__device__ __forceinline__ uint64_t max_group(uint64_t v, uint64_t* slots) {
    v = max_wave(v);
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
    v = sum_wave(v);
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

__device__ __forceinline__ void sample_outputs(const SampleArgs& a, int64_t row, uint32_t token, float log2_p) {
    a.tokens[row] = int32_t(token);
    if (a.logp) a.logp[row] = kLn2 * log2_p;
}
__device__ __forceinline__ void sample_none(const SampleArgs& a, int64_t row) {  // every logit is masked
    a.tokens[row] = -1;
    if (a.logp) a.logp[row] = kNegInf;
}

// What of a row is kept: keys above `key`, and the first `quota` of those equal to it. `cut`: there
// are more equal ones than that.
struct Threshold {
    uint32_t key;
    uint64_t quota;
    bool cut;
};

// Scales of up to this much have scores x c - log E that are rounded to 2^-12 at most, and weights at most
// 2^(2^-13) of the largest; rows beyond it (a temperature small against their logits, or finite masks
// everywhere) go the general way.
constexpr float kNear = 4096.f;
__device__ __forceinline__ bool near_scale(float top, float c) { return fabsf(top * c) < kNear; }

// A row in memory, its weights' scale (Scale or Above). NaN counts as -inf and +inf as the type's largest
// number, so that all weights are numbers of at most a little over 1.
template <typename DT, class S>
struct RowView {
    const DT* x;
    int64_t V;
    S scale;
    static __device__ __forceinline__ float finite(float v) { return fminf(v, sizeof(DT) == 4 ? 0x1.fffffep127f : 0x1.fep127f); }
    static __device__ __forceinline__ float number(DT v) { return finite(fmaxf(widen(v), kNegInf)); }
    __device__ __forceinline__ float logit(int64_t j) const { return number(x[j]); }
    // Element j of a short row, or what stands for the ones past its end; all of a lane's are asked for
    // before any is looked at.
    __device__ __forceinline__ DT ask(int j) const { return x[j < V ? j : int(V) - 1]; }
    __device__ __forceinline__ float log2_weight(float v) const { return scale.log2_weight(v); }
    // A weight (at most a little over 1) as an integer: its 2^-6 and 2^-38 parts, exact in float32.
    static __device__ __forceinline__ uint64_t mass_of(float w) {
        const float x = w * 64.f;
        return (uint64_t(uint32_t(x)) << 32) | uint32_t(__builtin_amdgcn_fractf(x) * 4294967296.f);
    }
    __device__ __forceinline__ uint64_t mass(float v) const { return mass_of(exp2_fast(log2_weight(v))); }
};

// The weight that min-p asks for (the largest logit always has it).
template <class R>
__device__ __forceinline__ float least_weight(const SampleRow& s, const R& r, float top) {
    return s.min_p > 0.f ? fminf(s.min_p, 1.f) * exp2_fast(r.log2_weight(top)) : 0.f;
}

// The k-th largest logit (k < V).
template <class R, int W>
__device__ Threshold descend_count(const R& r, uint64_t k, uint64_t* bins) {
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
template <class R, int W>
__device__ Threshold descend_mass(const R& r, Threshold t, float p, uint64_t* bins) {
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

// The general way: one row, any settings but a temperature of 0, by a workgroup of W waves. `top`: its largest
// logit, not -inf.
template <typename DT, int W>
__device__ __forceinline__ void sample_general(const SampleArgs& a, const SampleRow& s, const DT* x, const float* noise, float top, int64_t row,
                                               uint64_t* bins, uint64_t* slots) {
    typedef RowView<DT, Above> Row;
    top = Row::finite(top);
    const Row r{x, a.V, above(top, sample_scale(s))};
    constexpr int kLanes = W * kWave;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    Threshold t{0u, ~0ull, false};
    if (s.top_k < a.V) t = descend_count<Row, W>(r, uint64_t(s.top_k), bins);
    if (s.top_p < 1.f) t = descend_mass<Row, W>(r, t, s.top_p, bins);
    const float least = least_weight(s, r, top);
    double zl = 0.;
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
            if (lane == 0) slots[wave] = __popcll(votes);
            __syncthreads();
            uint64_t before = ties + __popcll(votes & ((1ull << lane) - 1));
#pragma unroll
            for (int i = 0; i < W; ++i) {
                if (i < wave) before += slots[i];
                ties += slots[i];
            }
            keep = keep && (!tie || before < t.quota);
        }
        if (!keep) continue;
        const float u = r.log2_weight(v), w = exp2_fast(u);
        if (!(w >= least)) continue;
        zl += w;
        const float score = noise ? u - noise_log2(noise[j]) : v;
        const uint64_t e = race_entry(order_key(score), uint32_t(j));
        winner = e > winner ? e : winner;
    }
    winner = max_group<W>(winner, slots);
    const float z = sum_group<W>(float(zl), slots);
    if (tid == 0) sample_outputs(a, row, race_index(winner), r.log2_weight(r.logit(race_index(winner))) - log2_fast(z));
}

constexpr int kList = 512;       // elements that can be ranked
constexpr int kFewest = 256;     // top-k that goes by lanes' maxima
constexpr int kMassBins = 2048;  // 64 an octave of weight: down to 2^-32 of the largest
constexpr float kBinsPerOctave = 64.f;
constexpr int kBatch = 256;  // kept elements a wave draws from at a time
// What holds them: less than a batch is left over when a wave adds up to four from each lane.
constexpr int kRoom = 2 * kBatch;
static_assert(kBatch - 1 + 4 * kWave <= kRoom, "a wave's kept elements fit their buffer");

// A row as its workgroup walks it, U vectors a lane at a time: f(vectors, index of the first; the
// others follow kLanes vectors apart). Past the row's end vectors are -inf. With ONE the row is no longer
// than that, and stays in registers.
template <typename DT, int W, int U, bool ONE>
struct RowWalk {
    static constexpr int K = RowVec<DT>::K, kLanes = W * kWave;
    const DT* x;
    int64_t V;
    RowVec<DT> kept[ONE ? U : 1];

    __device__ __forceinline__ void read(RowVec<DT> (&v)[U], int64_t i0) const {
#pragma unroll
        for (int u = 0; u < U; ++u) v[u].load(x, i0 + u * kLanes, V);
    }
    __device__ __forceinline__ RowWalk(const DT* row, int64_t n) : x(row), V(n) {
        if constexpr (ONE) read(kept, threadIdx.x);
    }
    template <class F>
    __device__ __forceinline__ void chunks(F&& f) const {
        if constexpr (ONE) {
            f(kept, int64_t(threadIdx.x));
        } else {
            // (a wave's lanes all make the same rounds, some of them past the end: f may vote)
            const int64_t vecs = (V + K - 1) / K, lane = threadIdx.x & 63;
            for (int64_t i0 = threadIdx.x & ~63u; i0 < vecs; i0 += U * kLanes) {
                RowVec<DT> v[U];
                read(v, i0 + lane);
                f(v, i0 + lane);
            }
        }
    }
    // f(value, index) for every element, NaN as -inf
    template <class F>
    __device__ __forceinline__ void each(F&& f) const {
        chunks([&](const RowVec<DT>(&v)[U], int64_t i0) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int k = 0; k < K; ++k) f(fmaxf(v[u].at(k), kNegInf), uint32_t((i0 + u * kLanes) * K + k));
        });
    }
    // The lane's largest element, its scale, and the sum of its weights by that (its
    // chunks' in 64 bits: a lane of the longest rows adds 2^16 weights). NaN as -inf.
    __device__ __forceinline__ void statistics(float c, float& top, Scale& sc, float& z) const {
        top = kNegInf;
        double zl = 0.;
        sc = scale_of(top, c);
        chunks([&](const RowVec<DT>(&v)[U], int64_t) {
            float t = top;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int k = 0; k < K; ++k) t = fmaxf(t, v[u].at(k));
            if (t > top) {
                const Scale to = scale_of(t, c);
                zl *= exp2_fast(scale_step(sc, to));
                sc = to;
                top = t;
            }
            float zc = 0.f;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int k = 0; k < K; ++k) zc += fmaxf(exp2_fast(sc.log2_weight(v[u].at(k))), 0.f);
            zl += zc;
        });
        z = float(zl);
    }
};

template <int W>
struct SampleShared {
    union {
        uint64_t bins[kMassBins];
        float maxima[W * kWave];
        struct {
            float v[W][kRoom];
            uint32_t j[W][kRoom];
        } kept;
    };
    uint64_t list[kList], sorted[kList];
    uint64_t slots[W];
    float slots_f[2 * W];
    uint32_t count, pivot;
    float top;
};

template <int W>
__device__ __forceinline__ float max_group_f(float v, float* slots) {
    v = max_wave(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
    __syncthreads();
    v = slots[0];
#pragma unroll
    for (int i = 1; i < W; ++i) v = fmaxf(v, slots[i]);
    return v;
}

// list[0, n) into `sorted`, largest first.
template <int W>
__device__ __forceinline__ void rank_list(const uint64_t* list, uint64_t* sorted, int n) {
    for (int i = threadIdx.x; i < n; i += W * kWave) {
        const uint64_t e = list[i];
        int rank = 0;
        int j = 0;
        for (; j + 4 <= n; j += 4)
            rank += int(list[j] > e) + int(list[j + 1] > e) + int(list[j + 2] > e) + int(list[j + 3] > e);
        for (; j < n; ++j) rank += int(list[j] > e);
        sorted[rank] = e;
    }
    __syncthreads();
}

// What a wave finds among sorted elements: of the first `most`, in their order, those before which the
// weights' sum (from `above` on) is below `target` and that weigh `least`.
struct Drawn {
    uint64_t winner;
    float z;
};
template <class R>
__device__ __forceinline__ Drawn draw_sorted(const uint64_t* sorted, int most, const R& r, const float* noise, float above,
                                             float target, float least, bool first_kept) {
    const int lane = threadIdx.x & 63;
    Drawn d{0, 0.f};
    for (int i0 = 0; i0 < most; i0 += kWave) {
        const int i = i0 + lane;
        const bool in = i < most;
        const uint64_t e = in ? sorted[i] : 0;
        const uint32_t j = race_index(e);
        const float v = key_value(uint32_t(e >> 32)), u = in ? r.log2_weight(v) : kNegInf, w = in ? exp2_fast(u) : 0.f;
        float upto = w;  // inclusive
#pragma unroll
        for (int step = 1; step < kWave; step <<= 1) {
            const float o = __shfl_up(upto, step);
            if (lane >= step) upto += o;
        }
        float before = __shfl_up(upto, 1);
        before = above + (lane == 0 ? 0.f : before);
        const bool keep = in && (before < target || (first_kept && i == 0)) && w >= least;
        if (keep) {
            d.z += w;
            const float score = noise ? u - noise_log2(noise[j]) : v;
            const uint64_t x = race_entry(order_key(score), j);
            d.winner = x > d.winner ? x : d.winner;
        }
        above += __shfl(upto, kWave - 1);
        if (!(above < target)) break;
    }
    d.winner = max_wave(d.winner);
    d.z = sum_wave(d.z);
    return d;
}

// What a part of a row without filters comes to: its race's winner, its largest logit, the sum of weights
// relative to that.
struct OpenPart {
    uint64_t winner;
    float top, z;
};

// Part of a row without filters: the race and the sum of weights in one pass. `first`: index of the
// part's first element.
template <typename DT, int W, int U, bool ONE>
__device__ __forceinline__ OpenPart open_part(const RowWalk<DT, W, U, ONE>& walk, const float* noise, float c, uint32_t first,
                                              uint64_t* slots, float* slots_f) {
    constexpr int K = RowVec<DT>::K, kLanes = W * kWave;
    const bool greedy = !(c < kInf);  // (temperature 0)
    const bool race = noise && !greedy;
    float top = kNegInf, best = kNegInf;
    double z = 0.;  // (chunk by chunk, as in statistics())
    Scale sc = scale_of(top, c);
    uint32_t at = 0;
    walk.chunks([&](const RowVec<DT>(&v)[U], int64_t i0) {
        RowVec<float> e[U][K / 4];
        if (race) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int q = 0; q < K / 4; ++q) e[u][q].load(noise, (i0 + u * kLanes) * (K / 4) + q, walk.V);
        }
        float t = top;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int k = 0; k < K; ++k) t = fmaxf(t, v[u].at(k));
        if (t > top) {
            const Scale to = scale_of(t, c);
            z *= exp2_fast(scale_step(sc, to));
            sc = to;
            top = t;
        }
        int where = -1;  // in this chunk
        float zc = 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const float x = v[u].at(k);
                zc += fmaxf(exp2_fast(sc.log2_weight(x)), 0.f);  // (NaN, of a NaN or while all is -inf: 0)
                const float score = race ? fmaf(x, c, -log2_fast(e[u][k / 4].at(k % 4))) : x;
                if (score > best) {  // (never of NaN or of a masked logit)
                    best = score;
                    where = u * K + k;
                }
            }
        z += zc;
        if (where >= 0) at = uint32_t((i0 + where / K * kLanes) * K + where % K);
    });
    OpenPart p;
    p.top = max_group_f<W>(top, slots_f);
    p.winner = max_group<W>(best == kNegInf ? 0 : race_entry(order_key(best), first + at), slots);
    p.z = sum_group<W>(top == kNegInf || greedy ? 0.f : float(z) * exp2_fast(scale_step(sc, scale_of(p.top, c))), slots);
    return p;
}

// The row's outputs from its whole part. False: the general way has to take it, as its logits are not near
// (infinity among them), no score is above -inf (noise out of its range), or the best is infinite (noise
// below 2^-126, whose logarithm one operation does not give: a check here costs nothing a logit).
template <typename DT>
__device__ __forceinline__ bool open_finish(const SampleArgs& a, const OpenPart& p, const DT* x, float c, int64_t row) {
    if (p.top == kNegInf) {
        if (threadIdx.x == 0) sample_none(a, row);
        return true;
    }
    const bool greedy = !(c < kInf);
    if (!greedy && (!near_scale(p.top, c) || p.winner == 0 || won_by_small(p.winner))) return false;
    if (threadIdx.x == 0) {
        const uint32_t j = race_index(p.winner);
        sample_outputs(a, row, j, greedy ? 0.f : scale_of(p.top, c).log2_weight(widen(x[j])) - log2_fast(p.z));
    }
    return true;
}

// A row without filters, one per workgroup: a pass over logits and noise, 6 bytes a bfloat16 logit,
// with the running maximum and sum of a softmax beside the race, so bound by memory: 512 x 128000 bfloat16
// (393 MB) 70 us, 5.6 TB/s.
template <typename DT, int W, int U, bool ONE>
__global__ __launch_bounds__(W * kWave) void sample_open_kernel(SampleArgs a) {
    __shared__ uint64_t s_bins[kDigits], s_slots[W];
    __shared__ float s_slots_f[W];
    const int64_t row = grid_row();
    if (row >= a.M) return;
    const DT* x = reinterpret_cast<const DT*>(a.logits) + row * a.ld;
    const float* noise = a.noise ? a.noise + row * a.ld_noise : nullptr;
    const SampleRow s = sample_row(a, row);
    const float c = sample_scale(s);
    const OpenPart p = open_part<DT, W, U, ONE>(RowWalk<DT, W, U, ONE>(x, a.V), noise, c, 0u, s_slots, s_slots_f);
    if (!open_finish<DT>(a, p, x, c, row)) sample_general<DT, W>(a, s, x, noise, p.top, row, s_bins, s_slots);
}

// Few long rows, on which one CU's loads are what bounds: parts of `length` elements (a multiple of a
// vector) on workgroups of their own (4 x 128000 bfloat16 5.5 us),
template <typename DT, int W, int U>
__global__ __launch_bounds__(W * kWave) void sample_parts_kernel(SampleArgs a, OpenPart* parts, int64_t length) {
    __shared__ uint64_t s_slots[W];
    __shared__ float s_slots_f[W];
    const int64_t row = blockIdx.y, first = int64_t(blockIdx.x) * length;
    const DT* x = reinterpret_cast<const DT*>(a.logits) + row * a.ld + first;
    const float* noise = a.noise ? a.noise + row * a.ld_noise + first : nullptr;
    const RowWalk<DT, W, U, false> walk(x, a.V - first < length ? a.V - first : length);
    const OpenPart p = open_part<DT, W, U, false>(walk, noise, sample_scale(sample_row(a, row)), uint32_t(first), s_slots, s_slots_f);
    if (threadIdx.x == 0) parts[row * gridDim.x + blockIdx.x] = p;
}

// and their join, four waves a row (one does, unless the general way has to take it; 2 us).
template <typename DT>
__global__ __launch_bounds__(4 * kWave) void sample_join_kernel(SampleArgs a, const OpenPart* parts, int count) {
    __shared__ uint64_t s_bins[kDigits], s_slots[4];
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x & 63;
    const DT* x = reinterpret_cast<const DT*>(a.logits) + row * a.ld;
    const SampleRow s = sample_row(a, row);
    const float c = sample_scale(s);
    const OpenPart mine = lane < count ? parts[row * count + lane] : OpenPart{0, kNegInf, 0.f};
    OpenPart p;
    p.top = max_wave(mine.top);
    p.winner = max_wave(mine.winner);
    p.z = sum_wave(mine.top == kNegInf ? 0.f : mine.z * exp2_fast(scale_step(scale_of(mine.top, c), scale_of(p.top, c))));
    if (!open_finish<DT>(a, p, x, c, row))
        sample_general<DT, 4>(a, s, x, a.noise ? a.noise + row * a.ld_noise : nullptr, p.top, row, s_bins, s_slots);
}

// One row per workgroup of W waves, with its filters. Bound by the vector unit and by barriers, a row having
// a CU or a part of one: 64 x 32000 bfloat16 with top-k of 50 11 us, top-p of 0.9 19, min-p 12; 256 x 128000
// float32 with top-k 45 us (2.9 TB/s), with top-p of 0.95 83: the first pass, at the memory's rate, 27, the
// histogram 22 (16 vector operations a logit above its bound), what picks out the kept ones, to weigh
// them with full waves, 15, and their noise 18, as some 9000 of a row touch nine tenths of its lines.
// Measured and left: the next vectors read ahead (85 us), the kept ones in a column of LDS for each lane
// with no count over lanes (85). top-k beyond 256 takes the general way (64 x 32000 of 2000 78 us).
// The cases that the quicker ways leave end in
// the general one, at the end (one place, so that it is compiled into the kernel, not called).
template <typename DT, int W, int U, bool ONE>
__global__ __launch_bounds__(W * kWave) void sample_rows_kernel(SampleArgs a) {
    __shared__ SampleShared<W> sh;
    constexpr int kLanes = W * kWave, K = RowVec<DT>::K;
    const int64_t row = grid_row();
    if (row >= a.M) return;
    const int tid = threadIdx.x, lane = tid & 63;
    const DT* x = reinterpret_cast<const DT*>(a.logits) + row * a.ld;
    const float* noise = a.noise ? a.noise + row * a.ld_noise : nullptr;
    const SampleRow s = sample_row(a, row);
    const RowWalk<DT, W, U, ONE> walk(x, a.V);
    const float c = sample_scale(s);
    const bool by_k = s.top_k < a.V, by_p = s.top_p < 1.f, by_min = s.min_p > 0.f;
    float top = kNegInf;

    auto quick = [&]() -> bool {
        if (!(c < kInf) || (!by_k && !by_p && !by_min))
        {
            const OpenPart p = open_part<DT, W, U, ONE>(walk, noise, c, 0u, sh.slots, sh.slots_f);
            top = p.top;
            return open_finish<DT>(a, p, x, c, row);
        }

        if (by_k && s.top_k <= kFewest) {
            walk.chunks([&](const RowVec<DT>(&v)[U], int64_t) {
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int k = 0; k < K; ++k) top = fmaxf(top, v[u].at(k));
            });
            sh.maxima[tid] = top;
            if (tid == 0) sh.count = 0;
            __syncthreads();
            if (tid < kWave) {
                // the largest 16-bit prefix of a key that k lanes' maxima reach; of fours of lanes while
                // there are plenty (fewer to compare, hardly more elements)
                constexpr int E = W;
                uint32_t key[E];
                float all = kNegInf;
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const float m = sh.maxima[lane + kWave * i];
                    all = fmaxf(all, m);
                    key[i] = m > kNegInf ? order_key(m) >> 16 : 0u;
                }
                int used = E;
                if constexpr (E % 4 == 0) {
                    if (s.top_k <= kLanes / 8) {
#pragma unroll
                        for (int i = 0; i < E / 4; ++i) {
                            const uint32_t x = key[4 * i] > key[4 * i + 1] ? key[4 * i] : key[4 * i + 1];
                            const uint32_t y = key[4 * i + 2] > key[4 * i + 3] ? key[4 * i + 2] : key[4 * i + 3];
                            key[i] = x > y ? x : y;
                        }
                        used = E / 4;
                    }
                }
                uint32_t prefix = 0;
                for (int bit = 15; bit >= 0; --bit) {
                    const uint32_t tried = prefix | (1u << bit);
                    int reached = 0;
#pragma unroll
                    for (int i = 0; i < E; ++i)
                        if (i < used) reached += __popcll(__ballot(key[i] >= tried));
                    if (reached >= s.top_k) prefix = tried;
                }
                all = max_wave(all);
                if (lane == 0) {
                    sh.pivot = prefix << 16;
                    sh.top = all;
                }
            }
            __syncthreads();
            top = sh.top;
            if (top == kNegInf) {
                if (tid == 0) sample_none(a, row);
                return true;
            }
            const RowView<DT, Above> r{x, a.V, above(top, c)};
            if (top == kInf) return false;
            const float from = sh.pivot > order_key(kNegInf) ? key_value(sh.pivot) : kNegInf;
            walk.each([&](float v, uint32_t j) {
                if (v >= from && v > kNegInf) {
                    const uint32_t i = atomicAdd(&sh.count, 1u);
                    if (i < kList) sh.list[i] = race_entry(order_key(v), j);
                }
            });
            __syncthreads();
            const int n = int(sh.count);
            if (n > kList) return false;
            rank_list<W>(sh.list, sh.sorted, n);
            if (tid >= kWave) return true;
            const int most = n < s.top_k ? n : int(s.top_k);
            float target = kInf;
            if (by_p) {
                float sum = 0.f;
                for (int i = lane; i < most; i += kWave) sum += exp2_fast(r.log2_weight(key_value(uint32_t(sh.sorted[i] >> 32))));
                target = s.top_p * sum_wave(sum);
            }
            const Drawn d = draw_sorted(sh.sorted, most, r, noise, 0.f, target, least_weight(s, r, top), true);
            if (lane == 0) sample_outputs(a, row, race_index(d.winner), r.log2_weight(r.logit(race_index(d.winner))) - log2_fast(d.z));
            return true;
        }

        // the largest logit and the sum of weights
        float own_top, z;
        Scale own;
        walk.statistics(c, own_top, own, z);
        top = max_group_f<W>(own_top, sh.slots_f);
        if (top == kNegInf) {
            if (tid == 0) sample_none(a, row);
            return true;
        }
        if (by_k || !near_scale(top, c)) return false;
        const RowView<DT, Scale> r{x, a.V, scale_of(top, c)};
        const float least = least_weight(s, r, top);
        z = own_top == kNegInf ? 0.f : z * exp2_fast(scale_step(own, r.scale));
        z = sum_group<W>(z, sh.slots);

        // without top-p everything is above the crossing bin
        int cross = kMassBins;
        float above = 0.f;
        const float target = by_p ? s.top_p * z : kInf;
        if (by_p) {
            // the smallest elements, of less than 1 - p in all, cannot be in: at most V of them below this
            const float low = log2_fast(0.99f * (1.f - s.top_p) * z / float(a.V));
            for (int i = tid; i < kMassBins; i += kLanes) sh.bins[i] = 0;
            if (tid == 0) sh.count = 0;
            __syncthreads();
            const float from = fmaxf(low, -float(kMassBins) / kBinsPerOctave * 0.9999f);  // (in the last bin still)
            walk.chunks([&](const RowVec<DT>(&v)[U], int64_t) {
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        const float l = r.log2_weight(v[u].at(k));
                        if (l >= from)  // (not of NaN)
                            atomicAdd(reinterpret_cast<unsigned long long*>(&sh.bins[uint32_t(fmaxf(l * -kBinsPerOctave, 0.f))]),
                                      (unsigned long long)(r.mass_of(exp2_fast(l))));
                    }
            });
            __syncthreads();
            // the first bin at which the sum reaches p of the mass (at least the largest element's)
            const uint64_t want0 = uint64_t(ceil(double(target) * kMassUnit)), want = want0 < 1 ? 1 : want0;
            constexpr int kEach = kMassBins / kLanes;  // bins a lane, in order
            uint64_t bin[kEach], sum = 0;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                bin[i] = sh.bins[tid * kEach + i];
                sum += bin[i];
            }
            uint64_t upto = sum;
#pragma unroll
            for (int d = 1; d < kWave; d <<= 1) {
                const uint64_t o = __shfl_up(upto, d);
                if (lane >= d) upto += o;
            }
            if (lane == kWave - 1) sh.slots[tid >> 6] = upto;
            if (tid == 0) sh.pivot = kMassBins;
            __syncthreads();
            uint64_t before = upto - sum;
#pragma unroll
            for (int i = 0; i < W; ++i) before += i < (tid >> 6) ? sh.slots[i] : 0;
            if (before < want && before + sum >= want) {  // one lane's
                bool found = false;
#pragma unroll
                for (int i = 0; i < kEach; ++i) {
                    if (found) continue;
                    if (before + bin[i] >= want) {
                        found = true;
                        sh.pivot = uint32_t(tid * kEach + i);
                        sh.top = float(double(before) / kMassUnit);
                    }
                    before += bin[i];
                }
            }
            __syncthreads();
            cross = int(sh.pivot);
            above = sh.top;
            if (cross == kMassBins) return false;  // (so flat that the cut lies below 2^-32)
        }
        // Above `sure` everything is kept, between the two edges lies the crossing bin. What passes goes
        // through a buffer of the wave's own, so that the few kept ones of many are weighed, and their
        // noise fetched, by full waves.
        // (the first bin takes logarithms that rounding leaves above 0, too)
        const float sure = !by_p ? kNegInf : cross > 0 ? -float(cross) / kBinsPerOctave : kInf;
        // (min-p's bound, less the rounding of a logarithm and an exponential, spares what lies below it the trip)
        const float edge = fmaxf(by_p ? -float(cross + 1) / kBinsPerOctave : kNegInf, by_min ? log2_fast(least) - 0.01f : kNegInf);
        __syncthreads();  // (the bins' memory)
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        float* kept_v = sh.kept.v[wave];
        uint32_t* kept_j = sh.kept.j[wave];
        double zl = 0.;
        uint64_t winner = 0;
        auto draw = [&](int n) {  // the buffer's first n (at most kBatch)
            float x[kBatch / kWave], e[kBatch / kWave];
            uint32_t j[kBatch / kWave];
            float zb = 0.f;
            wave_lds_sync();
#pragma unroll
            for (int q = 0; q < kBatch / kWave; ++q) {
                const int i = q * kWave + lane;
                x[q] = i < n ? kept_v[i] : kNegInf;
                j[q] = i < n ? kept_j[i] : 0u;
                e[q] = noise ? noise[j[q]] : 1.f;
            }
#pragma unroll
            for (int q = 0; q < kBatch / kWave; ++q) {
                if (!(x[q] > kNegInf)) continue;
                const float l = r.log2_weight(x[q]), w = exp2_fast(l);
                if (!(w >= least)) continue;
                if (l <= sure) {
                    const uint32_t i = atomicAdd(&sh.count, 1u);
                    if (i < kList) sh.list[i] = race_entry(order_key(x[q]), j[q]);
                    continue;
                }
                zb += w;
                const uint64_t y = race_entry(order_key(noise ? l - noise_log2(e[q]) : x[q]), j[q]);
                winner = y > winner ? y : winner;
            }
            zl += zb;
        };
        int held = 0;
        walk.chunks([&](const RowVec<DT>(&v)[U], int64_t i0) {
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    const float x = v[u].at(k);
                    const bool in = r.log2_weight(x) > edge;  // (not of NaN, nor of a masked logit)
                    const uint64_t passed = __ballot(in);
                    if (in) {
                        const int i = held + __popcll(passed & ((1ull << lane) - 1));
                        kept_v[i] = x;
                        kept_j[i] = uint32_t((i0 + u * kLanes) * K + k);
                    }
                    held += __popcll(passed);
                    if (k % 4 == 3 && held >= kBatch) {  // (every four elements of a lane: up to kRoom by then)
                        draw(kBatch);
                        held -= kBatch;
                        wave_lds_sync();
                        float xs[kBatch / kWave];
                        uint32_t js[kBatch / kWave];
#pragma unroll
                        for (int q = 0; q < kBatch / kWave; ++q) {
                            xs[q] = kept_v[kBatch + q * kWave + lane];
                            js[q] = kept_j[kBatch + q * kWave + lane];
                        }
                        wave_lds_sync();
#pragma unroll
                        for (int q = 0; q < kBatch / kWave; ++q) {
                            kept_v[q * kWave + lane] = xs[q];
                            kept_j[q * kWave + lane] = js[q];
                        }
                    }
                }
        });
        if (held) draw(held);
        float zk = sum_group<W>(float(zl), sh.slots);
        winner = max_group<W>(winner, sh.slots);
        if (by_p) {
            __syncthreads();
            const int n = int(sh.count);
            if (n > kList) return false;
            rank_list<W>(sh.list, sh.sorted, n);
            if (tid >= kWave) return true;
            const Drawn d = draw_sorted(sh.sorted, n, r, noise, above, target, least, true);
            zk += d.z;
            winner = d.winner > winner ? d.winner : winner;
        }
        if (tid == 0) sample_outputs(a, row, race_index(winner), r.log2_weight(r.logit(race_index(winner))) - log2_fast(zk));
        return true;
    };
    if (!quick()) sample_general<DT, W>(a, s, x, noise, top, row, sh.bins, sh.slots);
}

// Rows of up to 64 * E logits with filters, one per wave, logits and keys in registers (lane i has
// elements i, 64 + i, ...). A threshold is searched for by halving the range of logits: each step counts,
// or weighs, what lies above the middle, and the search ends when the cut falls between two elements
// (about ten steps on random logits) or at equal ones, of which the first by index stay. Bound by the
// latency of these steps, some 50 instructions each for a count of 1000 logits, 100 for a mass: 8 x 1000
// bfloat16 8 us with top-k, 10 with top-p, 14 with both and min-p; halving the range of keys alone, most of
// which lie near 0, took twice the steps (31 among equal bfloat16 logits), and loads of a lane one
// after another 3 us more: 14, 18 and 20.
template <typename DT, int E>
__global__ __launch_bounds__(4 * kWave) void sample_wave_kernel(SampleArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t row = grid_row() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (row >= a.M) return;
    RowView<DT, Above> r{reinterpret_cast<const DT*>(a.logits) + row * a.ld, a.V, {}};
    const float* noise = a.noise ? a.noise + row * a.ld_noise : nullptr;
    const SampleRow s = sample_row(a, row);
    const float c = sample_scale(s);
    const bool greedy = !(c < kInf);
    // Keys in as many bits as the type has; 0 is a dropped element's.
    constexpr uint32_t kOut = 0u;
    constexpr int kShift = 32 - 8 * int(sizeof(DT));
    auto key_of = [](float x) { return order_key(x) >> kShift; };
    auto value_of = [](uint32_t k) {
        const uint32_t u = k << kShift;
        return key_value(u & 0x80000000u ? u : u | ((1u << kShift) - 1));
    };
    DT asked[E];
    float v[E], n[E], top = kNegInf, low = kInf;
    uint32_t key[E];
#pragma unroll
    for (int e = 0; e < E; ++e) asked[e] = r.ask(lane + kWave * e);
#pragma unroll
    for (int e = 0; e < E; ++e) n[e] = noise && !greedy ? noise[lane + kWave * e < a.V ? lane + kWave * e : int(a.V) - 1] : 1.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        v[e] = lane + kWave * e < a.V ? r.number(asked[e]) : kNegInf;
        key[e] = v[e] > kNegInf ? key_of(v[e]) : kOut;
        top = fmaxf(top, v[e]);
        low = v[e] > kNegInf ? fminf(low, v[e]) : low;
    }
    top = max_wave(top);
    if (top == kNegInf) {
        if (lane == 0) sample_none(a, row);
        return;
    }
    r.scale = above(top, c);
    auto count = [&](uint32_t from) {
        int x = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) x += __popcll(__ballot(key[e] >= from));
        return x;
    };
    // Drops what lies below `from`, and of the elements equal to it all but the first `quota`.
    auto drop = [&](uint32_t from, int quota) {
        int before = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const uint64_t ties = __ballot(key[e] == from);
            const int rank = before + __popcll(ties & ((1ull << lane) - 1));
            before += __popcll(ties);
            if (key[e] < from || (key[e] == from && rank >= quota)) key[e] = kOut;
        }
    };
    if (!greedy) {
        // The middle is that of the values first, then of the keys, which ends where values are far from even.
        constexpr int kByValue = 14;
        auto middle = [&](uint32_t lo, uint32_t hi, int step) {
            if (step >= kByValue) return lo + (hi - lo) / 2;
            const uint32_t m = key_of(0.5f * value_of(lo) + 0.5f * value_of(hi));
            return m <= lo ? lo + 1 : m >= hi ? hi - 1 : m;
        };
        const uint32_t first = key_of(-max_wave(-low)), last = key_of(top) + 1;  // (of all; above all)
        if (s.top_k < a.V) {
            const int k = int(s.top_k);
            uint32_t lo = first, hi = last;
            int above_lo = count(lo), above_hi = 0;
            if (above_lo > k) {
                for (int step = 0; hi - lo > 1 && above_lo > k; ++step) {
                    const uint32_t mid = middle(lo, hi, step);
                    const int x = count(mid);
                    if (x >= k) {
                        lo = mid;
                        above_lo = x;
                    } else {
                        hi = mid;
                        above_hi = x;
                    }
                }
                drop(lo, above_lo > k ? k - above_hi : kWave * E);
            }
        }
        if (s.top_p < 1.f) {
            float w[E], z = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                w[e] = key[e] != kOut ? exp2_fast(r.log2_weight(v[e])) : 0.f;
                z += w[e];
            }
            const float target = fmaxf(s.top_p * sum_wave(z), 1e-30f);
            uint32_t lo = first, hi = last;
            int above_lo = count(lo), above_hi = 0;
            float mass_hi = 0.f;
            for (int step = 0; hi - lo > 1 && above_lo - above_hi > 1; ++step) {
                const uint32_t mid = middle(lo, hi, step);
                float m = 0.f;
                int x = 0;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const bool in = key[e] >= mid;
                    m += in ? w[e] : 0.f;
                    x += __popcll(__ballot(in));
                }
                m = sum_wave(m);
                if (m >= target) {
                    lo = mid;
                    above_lo = x;
                } else {
                    hi = mid;
                    above_hi = x;
                    mass_hi = m;
                }
            }
            int quota = kWave * E;
            if (above_lo - above_hi > 1) {  // equal ones: as many as begin below the target
                const float one = exp2_fast(r.log2_weight(value_of(lo)));
                quota = one > 0.f ? int(fminf(fmaxf(ceilf((target - mass_hi) / one), 1.f), float(kWave * E))) : 1;
            }
            drop(lo, quota);
        }
        if (s.min_p > 0.f) {
            const float least = least_weight(s, r, top);
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (!(exp2_fast(r.log2_weight(v[e])) >= least)) key[e] = kOut;
        }
    }
    float z = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) z += key[e] != kOut ? exp2_fast(r.log2_weight(v[e])) : 0.f;
    z = sum_wave(z);
    auto race = [&](auto log2_of) {
        uint64_t best = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (key[e] == kOut) continue;
            const uint64_t x = race_entry(noise && !greedy ? order_key(r.log2_weight(v[e]) - log2_of(n[e])) : key[e], uint32_t(lane + kWave * e));
            best = x > best ? x : best;
        }
        return max_wave(best);
    };
    uint64_t winner = race([](float e) { return log2_fast(e); });
    if (won_by_small(winner)) winner = race([](float e) { return noise_log2(e); });
    const uint32_t j = race_index(winner);
    if (lane == 0) sample_outputs(a, row, j, greedy ? 0.f : r.log2_weight(r.logit(j)) - log2_fast(z));
}

// Rows of up to L * E logits, L lanes a row, no filters: all of a lane's loads at once, then one fold for
// the maximum and one each for the sum and the race. Bound by a launch's latency up to some thousand rows
// (8192 x 18 float32 3.2 us), then by memory (8192 x 1000 bfloat16 12.3 us, 4 TB/s).
template <typename DT, int L, int E>
__global__ __launch_bounds__(4 * kWave) void sample_small_kernel(SampleArgs a) {
    const int lane = threadIdx.x & 63, i = lane % L;
    const int64_t row = (grid_row() * 4 + (threadIdx.x >> 6)) * (kWave / L) + lane / L;
    if (row >= a.M) return;  // (a whole group of L lanes leaves together)
    RowView<DT, Above> r{reinterpret_cast<const DT*>(a.logits) + row * a.ld, a.V, {}};
    const float* noise = a.noise ? a.noise + row * a.ld_noise : nullptr;
    const SampleRow s = sample_row(a, row);
    const float c = sample_scale(s);
    const bool greedy = !(c < kInf);
    DT asked[E];
    float v[E], n[E], top = kNegInf;
#pragma unroll
    for (int e = 0; e < E; ++e) asked[e] = r.ask(i + L * e);
#pragma unroll
    for (int e = 0; e < E; ++e) n[e] = noise && !greedy ? noise[i + L * e < a.V ? i + L * e : int(a.V) - 1] : 1.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        v[e] = i + L * e < a.V ? r.number(asked[e]) : kNegInf;
        top = fmaxf(top, v[e]);
    }
    top = max_lanes<L>(top);
    if (top == kNegInf) {
        if (i == 0) sample_none(a, row);
        return;
    }
    r.scale = above(top, c);
    float z = 0.f;
    uint64_t winner = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float u = r.log2_weight(v[e]);
        z += exp2_fast(u);
        const float score = noise && !greedy ? u - log2_fast(n[e]) : v[e];
        const uint64_t x = v[e] > kNegInf ? race_entry(order_key(score), uint32_t(i + L * e)) : 0;
        winner = x > winner ? x : winner;
    }
    z = sum_lanes<L>(z);
    winner = max_lanes<L>(winner);
    if (won_by_small(winner)) {  // (from memory: 8192 x 1000 takes 12.3 us, 12.5 where the loop above keeps its registers for it)
        winner = 0;
#pragma unroll 1
        for (int j = i; j < a.V; j += L) {
            const float x = r.logit(j);
            const uint64_t y = x > kNegInf ? race_entry(order_key(r.log2_weight(x) - noise_log2(noise[j])), uint32_t(j)) : 0;
            winner = y > winner ? y : winner;
        }
        winner = max_lanes<L>(winner);
    }
    const uint32_t j = race_index(winner);
    float won = kNegInf;  // the winner's logit, from the lane that has it
#pragma unroll
    for (int e = 0; e < E; ++e) won = uint32_t(i + L * e) == j ? v[e] : won;
    won = max_lanes<L>(won);
    if (i == 0) sample_outputs(a, row, j, greedy ? 0.f : r.log2_weight(won) - log2_fast(z));
}

}  // namespace rlcs
