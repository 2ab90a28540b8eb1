// Distillation from a teacher's largest logits: the loss of each row and its gradient by the logits.
//
// With u = (x - max x) * log2(e) / temperature and z = sum 2^u, log p_j = ln 2 (u_j - log2 z). The gradient is
// S p_j - t_j at the K listed tokens, S the sum of all shares that count, and p_j times one factor a row everywhere else: a
// row is written as if nothing were listed, then the listed places again. S is 1 but where the class of the rest is left out: then what the
// list has, whatever it adds up to. What lies outside the list is summed apart, by a bit for each logit in LDS (as the difference of two
// sums it would be lost where the list has almost all of the mass). Where it lies so far below the row's largest logit that its weights
// underflow, it is summed again relative to its own: p' is a number however small, and the gradient there is each logit's share of it.
#pragma once

#include "rlcs_softmax.h"

namespace rlcs {

constexpr int kMaxListed = 1024;
constexpr int64_t kBits = 1 << 18;  // logits whose bits are in LDS at a time

struct DistillArgs {
    const void* logits;
    const int32_t* ids;
    const float *top, *weight;
    float* loss;
    void* grad;
    int64_t M, V, ld, ld_grad;
    int32_t K, words;  // words: of a row's bits, a multiple of 4
    float inv_temp;
};

// LDS of a row: its bits, and the listed tokens: id (-1: none), logit, share t, and log t.
struct DistillLds {
    uint32_t* bits;
    int32_t* id;
    float *x, *t, *lt;
    __device__ __forceinline__ DistillLds(char* mem, const DistillArgs& a) {
        bits = reinterpret_cast<uint32_t*>(mem);
        id = reinterpret_cast<int32_t*>(bits + a.words);
        x = reinterpret_cast<float*>(id + a.K);
        t = x + a.K;
        lt = t + a.K;
    }
};
inline size_t distill_lds(const DistillArgs& a) { return (size_t(a.words) * 4 + size_t(a.K) * 16 + 15) / 16 * 16; }

// The lanes of a row: W waves of a workgroup, or with W = 1 a wave of a workgroup of four. Folds take several values with one
// wait; `slots`: kFolds floats a wave, every fold of a row with its own (from `at` on), so that none waits for the one before.
template <int W>
struct Team {
    static constexpr int kLanes = W * kWave, kFolds = 11;
    float* slots;
    int lane;
    __device__ __forceinline__ void sync() const {
        if constexpr (W == 1) wave_lds_sync();
        else __syncthreads();
    }
    // Stores of any lane before it come before stores of any lane after it.
    __device__ __forceinline__ void order_stores() const {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
        if constexpr (W > 1) __syncthreads();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
    }
    // v[i] folded over the waves by f.
    template <int N, class F>
    __device__ __forceinline__ void fold(float (&v)[N], int at, F&& f) const {
        if constexpr (W > 1) {
            if ((lane & 63) == 0) {
#pragma unroll
                for (int i = 0; i < N; ++i) slots[(at + i) * W + (lane >> 6)] = v[i];
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i) {
                v[i] = slots[(at + i) * W];
#pragma unroll
                for (int w = 1; w < W; ++w) v[i] = f(v[i], slots[(at + i) * W + w]);
            }
        }
    }
    template <int N>
    __device__ __forceinline__ void largest(float (&v)[N], int at) const {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = max_wave(v[i]);
        fold(v, at, [](float x, float y) { return fmaxf(x, y); });
    }
    template <int N>
    __device__ __forceinline__ void sums(float (&v)[N], int at) const {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = sum_wave(v[i]);
        fold(v, at, [](float x, float y) { return x + y; });
    }
};

__device__ __forceinline__ void mark(uint32_t* bits, int64_t id, bool& twice) {
    const uint32_t at = uint32_t(id) & uint32_t(kBits - 1), bit = 1u << (at & 31);
    twice |= (atomicOr(&bits[at >> 5], bit) & bit) != 0;
}

// The listed ids and their bits, first of all; true: one may be there twice (ids that are kBits apart share a bit).
template <int W>
__device__ __forceinline__ bool read_ids(const DistillArgs& a, const DistillLds& l, const Team<W>& team, int64_t row) {
    for (int i = team.lane; i < a.words; i += Team<W>::kLanes) l.bits[i] = 0;
    team.sync();
    bool twice = false;
    for (int k = team.lane; k < a.K; k += Team<W>::kLanes) {
        const int32_t id = a.ids[row * a.K + k];
        const bool is = id >= 0 && id < a.V;
        l.id[k] = is ? id : -1;
        if (is) mark(l.bits, id, twice);
    }
    return twice;
}

// The largest logit of the row, and of its list.
struct RowStats {
    float top;
    Scale sc;
    float top_listed;
    bool some, twice;  // a share is not 0; a token may be listed twice
};
// From each lane's largest logit; the logits of the listed tokens and the logarithms of their shares are read here, by the
// lanes that keep them.
template <typename DT, int W>
__device__ __forceinline__ RowStats row_tops(const DistillArgs& a, const DistillLds& l, const Team<W>& team, int64_t row, float top, bool twice) {
    const DT* x = reinterpret_cast<const DT*>(a.logits) + row * a.ld;
    float listed = kNegInf;
    bool some = false;
    for (int k = team.lane; k < a.K; k += Team<W>::kLanes) {
        const int32_t id = l.id[k];
        const float lt = id >= 0 ? a.top[row * a.K + k] : kNegInf;
        l.x[k] = id >= 0 ? widen(x[id]) : 0.f;
        l.lt[k] = lt;
        some |= !(lt == kNegInf);  // (NaN is some)
        listed = fmaxf(listed, lt);
    }
    float v[4] = {top, listed, some ? 1.f : 0.f, twice ? 1.f : 0.f};
    team.largest(v, 0);
    return RowStats{v[0], scale_of(v[0], kLog2e * a.inv_temp), v[1], v[2] > 0.f, v[3] > 0.f};
}

// A row once its sums are known: weights' scale, the sum's inverse (0: every logit is masked), what a logit that is not listed has as
// its gradient's factor.
struct DistillRow {
    Scale sc;
    float inv, factor, amount, share;  // share: what the weights of the list are multiplied by
    float mass;                        // of all shares that count
    // Of a class summed apart: what its weights, relative to its largest, are multiplied by; 0: it was not.
    float apart;
    Scale sc_out;
    // f times the probability of logit x. (The weight times the sum's inverse and not by the logarithm of the sum: the
    // rounding of the scale is in both, and cancels.)
    __device__ __forceinline__ float times(float f, float x) const { return exp2_fast(sc.log2_weight(x)) * f; }
};

// The largest logit outside the list and the sum of the weights relative to it; each(f): f(vector, its bits) for all of a lane's vectors.
// (Bits of a list, a word's low ones for a vector; past the row's end -inf.)
struct RowRest {
    float top, sum;
    Scale sc;
};
template <int W, class F>
__device__ __forceinline__ RowRest row_rest(const Team<W>& team, float c, F&& each) {
    float top = kNegInf;
    double sum = 0.;
    Scale sc = scale_of(top, c);
    auto rebase = [&](float t) {
        const Scale to = scale_of(t, c);
        sum *= top == kNegInf ? 0. : double(exp2_fast(scale_step(sc, to)));
        top = t;
        sc = to;
    };
    each([&](const auto& v, uint32_t bits) {
        constexpr int K = std::decay<decltype(v)>::type::K;
        float t = top;
#pragma unroll
        for (int k = 0; k < K; ++k) t = bits >> k & 1 ? t : fmaxf(t, v.at(k));
        if (t > top) rebase(t);
        float z = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) z += bits >> k & 1 ? 0.f : exp2_fast(sc.log2_weight(v.at(k)));
        sum += z;
    });
    float v[1] = {top};
    team.largest(v, 9);
    if (top > kNegInf && v[0] > top) rebase(v[0]);
    float z[1] = {float(sum)};
    team.sums(z, 10);
    return RowRest{v[0], z[0], scale_of(v[0], c)};
}

// Sums of weights outside the list below this are taken again by row_rest(): of larger ones, what underflowed is less than 2^-36. (Rows
// where it is so are read once more for the sum and once for the gradient: 4096 of 32000 bfloat16 logits 178 us, else 97; 2048 of
// 128000 343 and 222.)
constexpr float kLeastRest = 0x1p-60f;

// From each lane's sums of the weights outside the list and in it: the row's, and its loss. each: as row_rest() takes it.
template <bool TAIL, int W, class F>
__device__ __forceinline__ DistillRow row_loss(const DistillArgs& a, const DistillLds& l, const Team<W>& team, const RowStats& st, float z_out,
                                               float z_in, float w, int64_t row, F&& each) {
    DistillRow r;
    r.sc = st.sc;
    r.amount = w * a.inv_temp;
    r.factor = r.amount;
    r.mass = 1.f;
    r.apart = 0.f;
    float rest = 0.f, log_sum = 0.f, loss = 0.f, z;
    if constexpr (TAIL) {
        // (in 64 bits: what is left of 1 may be small. Over the waves as two floats, the sum's high part and what it leaves out)
        double sum = 0.;
        for (int k = team.lane; k < a.K; k += Team<W>::kLanes) {
            const double t = exp(double(l.lt[k]));
            l.t[k] = float(t);
            sum += t;
        }
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) sum += __shfl_xor(sum, d);
        const float high = float(sum);
        if (W > 1 && (team.lane & 63) == 0) {
            team.slots[6 * W + (team.lane >> 6)] = high;
            team.slots[7 * W + (team.lane >> 6)] = float(sum - double(high));
        }
        float v[2] = {z_out, z_in};
        team.sums(v, 4);
        double left = 1.;
        if constexpr (W > 1) {
#pragma unroll
            for (int i = 0; i < W; ++i) left -= double(team.slots[6 * W + i]) + double(team.slots[7 * W + i]);
        } else {
            left -= sum;
        }
        z_out = v[0];
        z = v[0] + v[1];
        rest = left < 0. ? 0.f : float(left);
        r.mass = float(1. - left);
        r.share = 1.f;
    } else {
        float sum = 0.f;
        for (int k = team.lane; k < a.K; k += Team<W>::kLanes) {
            const float t = l.lt[k] == kNegInf ? 0.f : exp2_fast((l.lt[k] - st.top_listed) * kLog2e);
            l.t[k] = t;
            sum += t;
        }
        float v[2] = {z_out, sum};
        team.sums(v, 4);
        z = v[0];
        r.share = 1.f / v[1];
        log_sum = kLn2 * log2_fast(v[1]);
    }
    const bool unmasked = !(z == 0.f);  // (NaN counts)
    r.inv = unmasked ? 1.f / z : 0.f;
    // log z relative to the top itself: the scale's m is rounded, by what this product leaves over
    const float log_z = unmasked ? kLn2 * (log2_fast(z) - fmaf(st.top, st.sc.c, -st.sc.m)) : 0.f;
    const float top_listed = TAIL ? 0.f : st.top_listed;
    for (int k = team.lane; k < a.K; k += Team<W>::kLanes) {
        // (not by way of the base 2: 1.44 times a finite mask of the type's lowest value overflows)
        const float t = l.t[k] * r.share, lp = unmasked ? fmaf(l.x[k] - st.top, a.inv_temp, -log_z) : kNegInf;
        if (!(t == 0.f)) loss = fmaf(t, (l.lt[k] - top_listed) - log_sum - lp, loss);
    }
    if constexpr (TAIL) {
        bool some = !(rest == 0.f);
        float log_ratio = 0.f, ratio = 0.f;  // of the class's share to its probability
        if (some && z_out < kLeastRest) {
            const RowRest o = row_rest(team, kLog2e * a.inv_temp, each);
            some = unmasked && !(o.top == kNegInf);
            if (some) {
                const float log_p = fmaf(o.top - st.top, a.inv_temp, kLn2 * (log2_fast(o.sum) - fmaf(o.top, o.sc.c, -o.sc.m)) - log_z);
                log_ratio = kLn2 * log2_fast(rest) - log_p;
                r.apart = r.amount * (rest / o.sum);
                r.sc_out = o.sc;
            }
        } else {
            const float p_out = z_out / z;
            log_ratio = kLn2 * (log2_fast(rest) - log2_fast(p_out));
            ratio = rest / p_out;
        }
        if (some) {
            if (team.lane == 0) loss = fmaf(rest, log_ratio, loss);
            r.mass = 1.f;
            r.factor = r.amount * (1.f - ratio);
        } else {
            r.factor = r.amount * r.mass;
        }
    }
    float v[1] = {loss};
    team.sums(v, 8);
    if (team.lane == 0) a.loss[row] = w * v[0];
    return r;
}

// The gradient of a row whose class was summed apart, as if nothing were listed. (It reads the row again: beside vectors in registers
// it would take half as many more of these, and rows like this are rare.)
template <typename DT, int L>
__device__ __forceinline__ void gradient_apart(const DT* x, DT* g, int64_t V, int lane, const DistillRow& r, float factor) {
    constexpr int K = RowVec<DT>::K;
    const int64_t vecs = (V + K - 1) / K;
#pragma unroll 1
    for (int64_t i = lane; i < vecs; i += L) {
        RowVec<DT> v;
        v.load(x, i, V);
        float d[K];
#pragma unroll
        for (int k = 0; k < K; ++k) d[k] = r.times(factor, v.at(k)) - r.apart * exp2_fast(r.sc_out.log2_weight(v.at(k)));
        store_row_vec<DT>(g, i, V, d);
    }
}

// The listed places of the gradient, once everything else of the row is written.
template <typename DT, int W>
__device__ __forceinline__ void listed_gradient(const DistillArgs& a, const DistillLds& l, const Team<W>& team, bool twice, const DistillRow& r, DT* g) {
    team.order_stores();
    for (int k = team.lane; k < a.K; k += Team<W>::kLanes) {
        const int32_t id = l.id[k];
        if (id < 0) continue;
        float t = l.t[k];
        if (twice) {  // the first of a token's places writes the sum of its shares
            bool first = true;
            t = 0.f;
            for (int j = 0; j < a.K; ++j) {
                if (l.id[j] != id) continue;
                first = first && j >= k;
                t += l.t[j];
            }
            if (!first) continue;
        }
        g[id] = narrow(r.amount * (r.times(r.inv * r.mass, l.x[k]) - t * r.share), DT{});
    }
}

template <typename DT, int L>
__device__ __forceinline__ void zero_row(DT* g, int64_t V, int lane) {
    constexpr int K = RowVec<DT>::K;
    const float zero[K] = {};
    const int64_t vecs = (V + K - 1) / K;
    for (int64_t i = lane; i < vecs; i += L) store_row_vec<DT>(g, i, V, zero);
}

// Bits of the logits of vector i.
template <int K>
__device__ __forceinline__ uint32_t vector_bits(const uint32_t* bits, int64_t i) {
    if constexpr (K == 8) return reinterpret_cast<const uint8_t*>(bits)[i];
    else return reinterpret_cast<const uint8_t*>(bits)[i >> 1] >> (4 * (i & 1)) & 15u;
}

// A vector's weights, added to what they belong to.
template <bool TAIL, class V>
__device__ __forceinline__ void add_weights(const V& v, const Scale& sc, uint32_t bits, float& z_out, float& z_in) {
    float e[V::K];
#pragma unroll
    for (int k = 0; k < V::K; ++k) e[k] = exp2_fast(sc.log2_weight(v.at(k)));
    if (TAIL && bits) {
#pragma unroll
        for (int k = 0; k < V::K; ++k) {
            const bool in = bits >> k & 1;
            z_out += in ? 0.f : e[k];
            z_in += in ? e[k] : 0.f;
        }
    } else {
#pragma unroll
        for (int k = 0; k < V::K; ++k) z_out += e[k];
    }
}

// Rows of up to U vectors a lane of W waves, which stay in registers. Every logit is read and every gradient
// written once. Bound by memory: 4096 rows of 32000 bfloat16 logits (8 waves of 8 vectors) 88 us for 438 MB, 5.0 TB/s; by 4 waves of
// 16 vectors 91, by 16 of 4 128 us.
// (Waves a SIMD as without row_rest(), beside which the compiler would hold a few registers more than these allow.)
template <typename DT, bool TAIL, int W, int U>
__global__ __launch_bounds__((W == 1 ? 4 : W) * kWave) __attribute__((amdgpu_waves_per_eu(!TAIL ? 1 : U == 8 ? 4 : sizeof(DT) == 2 ? 6 : 8)))
void distill_vec_kernel(DistillArgs a, int row_lds) {
    extern __shared__ __attribute__((aligned(16))) char s_mem[];
    __shared__ float s_slots[Team<W>::kFolds * W];
    constexpr int K = RowVec<DT>::K, kLanes = W * kWave;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row = W == 1 ? grid_row() * 4 + wave : grid_row();
    if (row >= a.M) return;
    const Team<W> team{s_slots, W == 1 ? int(threadIdx.x) & 63 : int(threadIdx.x)};
    const DistillLds l(s_mem + (W == 1 ? wave * row_lds : 0), a);
    const DT* x = reinterpret_cast<const DT*>(a.logits) + row * a.ld;
    DT* g = a.grad ? reinterpret_cast<DT*>(a.grad) + row * a.ld_grad : nullptr;
    const float w = a.weight ? a.weight[row] : 1.f;
    RowVec<DT> v[U];
    RowStats st{};
    float top = kNegInf;
    if (w != 0.f) {
#pragma unroll
        for (int u = 0; u < U; ++u) v[u].load(x, team.lane + u * kLanes, a.V);  // (past the end: -inf)
        const bool twice = read_ids<W>(a, l, team, row);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int k = 0; k < K; ++k) top = fmaxf(top, v[u].at(k));
        st = row_tops<DT, W>(a, l, team, row, top, twice);
        if (TAIL && W == 1) team.sync();  // (all bits are there)
    }
    if (w == 0.f || !(TAIL || st.some)) {
        if (team.lane == 0) a.loss[row] = 0.f;
        if (g) zero_row<DT, kLanes>(g, a.V, team.lane);
        return;
    }
    float z_out = 0.f, z_in = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t i = team.lane + u * kLanes;
        const uint32_t bits = TAIL && i * K < a.V ? vector_bits<K>(l.bits, i) : 0u;
        add_weights<TAIL>(v[u], st.sc, bits, z_out, z_in);
    }
    const DistillRow r = row_loss<TAIL, W>(a, l, team, st, z_out, z_in, w, row, [&](auto&& f) {
#pragma unroll 1
        for (int64_t i = team.lane; i * K < a.V; i += kLanes) {
            RowVec<DT> one;
            one.load(x, i, a.V);
            f(one, vector_bits<K>(l.bits, i));
        }
    });
    if (!g) return;
    const float factor = r.factor * r.inv;
    if (TAIL && r.apart != 0.f) {
        gradient_apart<DT, kLanes>(x, g, a.V, team.lane, r, factor);
    } else {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t i = team.lane + u * kLanes;
            float d[K];
#pragma unroll
            for (int k = 0; k < K; ++k) d[k] = r.times(factor, v[u].at(k));
            if (i * K < a.V) store_row_vec<DT>(g, i, a.V, d);
        }
    }
    listed_gradient<DT, W>(a, l, team, st.twice, r, g);
}

// Longer rows, one per workgroup of W waves: one pass for the sums, each lane relative to its own running
// maximum, and one backwards that writes the gradient, from the registers of the first pass's last vectors. Both passes spend about eight vector operations a logit, one of them an exponential.
// 8192 rows of 128000 bfloat16 logits, a third of weight 0: 710 us, 8 waves with eight vectors a lane at a time; the caches
// fetch 2.5 GB for 1.4 and write 2.1, 6.5 TB/s of that. Four vectors: 772 us, twelve 884, sixteen 841; eight by 4 waves 824, by 16
// 753; all of a row in 16 waves' registers 2294 us.
template <typename DT, bool TAIL, int W>
__global__ __launch_bounds__(W * kWave) void distill_rows_kernel(DistillArgs a) {
    extern __shared__ __attribute__((aligned(16))) char s_mem[];
    __shared__ float s_slots[Team<W>::kFolds * W];
    constexpr int K = RowVec<DT>::K, U = 8, kLanes = W * kWave;
    const int64_t row = grid_row();
    if (row >= a.M) return;
    const int tid = threadIdx.x;
    const Team<W> team{s_slots, tid};
    const DistillLds l(s_mem, a);
    const DT* x = reinterpret_cast<const DT*>(a.logits) + row * a.ld;
    DT* g = a.grad ? reinterpret_cast<DT*>(a.grad) + row * a.ld_grad : nullptr;
    const float w = a.weight ? a.weight[row] : 1.f;
    if (w == 0.f) {
        if (tid == 0) a.loss[row] = 0.f;
        if (g) zero_row<DT, kLanes>(g, a.V, tid);
        return;
    }
    const bool twice = read_ids<W>(a, l, team, row);
    __syncthreads();
    const float c = kLog2e * a.inv_temp;
    const int64_t vecs = (a.V + K - 1) / K;
    // (sums from chunk to chunk in 64 bits: one addition after another in 32 drifts in the longest rows)
    float top = kNegInf;
    Scale sc = scale_of(top, c);
    double out = 0., in = 0.;
    auto rebase = [&](float t) {
        const Scale to = scale_of(t, c);
        const double f = top == kNegInf ? 0. : double(exp2_fast(scale_step(sc, to)));
        out *= f;
        in *= f;
        top = t;
        sc = to;
    };
    const int64_t span = TAIL ? kBits / K : vecs;  // vectors whose bits are there
    RowVec<DT> v[U];
    auto part_bits = [&](int64_t from, int64_t end) {  // the bits of this part of a longer row
        if (!TAIL || a.V <= kBits) return;
        __syncthreads();
        for (int i = tid; i < a.words; i += kLanes) l.bits[i] = 0;
        __syncthreads();
        bool unused = false;
        for (int k = tid; k < a.K; k += kLanes) {
            const int64_t id = l.id[k];
            if (id >= from * K && id < end * K) mark(l.bits, id, unused);
        }
        __syncthreads();
    };
    for (int64_t from = 0; from < vecs; from += span) {
        const int64_t end = from + span < vecs ? from + span : vecs;
        part_bits(from, end);
        for (int64_t i0 = from + tid; i0 < end; i0 += U * kLanes) {
#pragma unroll
            for (int u = 0; u < U; ++u) v[u].load(x, i0 + u * kLanes, i0 + u * kLanes < end ? a.V : 0);  // (past the end: -inf)
            float t = top;
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int k = 0; k < K; ++k) t = fmaxf(t, v[u].at(k));
            if (t > top) rebase(t);
            float z_out = 0.f, z_in = 0.f;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t i = i0 + u * kLanes;
                const uint32_t bits = TAIL && i < end ? vector_bits<K>(l.bits, i - from) : 0u;
                add_weights<TAIL>(v[u], sc, bits, z_out, z_in);
            }
            out += z_out;
            in += z_in;
        }
    }
    const RowStats st = row_tops<DT, W>(a, l, team, row, top, twice);
    if (!TAIL && !st.some) {
        if (tid == 0) a.loss[row] = 0.f;
        if (g) zero_row<DT, kLanes>(g, a.V, tid);
        return;
    }
    if (top > kNegInf && st.top > top) rebase(st.top);
    const DistillRow r = row_loss<TAIL, W>(a, l, team, st, float(out), float(in), w, row, [&](auto&& f) {
        for (int64_t from = 0; from < vecs; from += span) {
            const int64_t end = from + span < vecs ? from + span : vecs;
            part_bits(from, end);
#pragma unroll 1
            for (int64_t i = from + tid; i < end; i += kLanes) {
                RowVec<DT> one;
                one.load(x, i, a.V);
                f(one, vector_bits<K>(l.bits, i - from));
            }
        }
    });
    if (!g) return;
    const float factor = r.factor * r.inv;
    if (TAIL && r.apart != 0.f) {
        gradient_apart<DT, kLanes>(x, g, a.V, tid, r, factor);
        listed_gradient<DT, W>(a, l, team, st.twice, r, g);
        return;
    }
    // backwards: what the first pass read last is nearest in the caches
    const int64_t last = (vecs - 1) / (U * kLanes) * (U * kLanes) + tid;
    for (int64_t i0 = last; i0 >= 0; i0 -= U * kLanes) {
        if (i0 != last) {  // (which is still there)
#pragma unroll
            for (int u = 0; u < U; ++u) v[u].load(x, i0 + u * kLanes, a.V);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t i = i0 + u * kLanes;
            float d[K];
#pragma unroll
            for (int k = 0; k < K; ++k) d[k] = r.times(factor, v[u].at(k));
            if (i < vecs) store_row_vec<DT>(g, i, a.V, d);
        }
    }
    listed_gradient<DT, W>(a, l, team, st.twice, r, g);
}

}  // namespace rlcs
