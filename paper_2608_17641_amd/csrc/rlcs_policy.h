// Log-probability, entropy and the clipped policy loss of rows of logits.
//
// With u = (x - max x) * log2(e) / temperature, z = sum 2^u and s = sum 2^u u:
//   log p_j = ln 2 (u_j - log2 z),  entropy = ln 2 (log2 z - s / z),
// and the gradient of the loss by x_j is p_j (a log2 p_j + b) + 1{j = token} d with three numbers a
// row.
#pragma once

#include "rlcs_softmax.h"

namespace rlcs {

struct PolicyArgs {
    const void* logits;
    const int32_t* tokens;
    const float *logp_old, *adv, *weight;
    float *loss, *logp, *ent;
    void* grad;
    int64_t M, V, ld, ld_grad;
    float low, high;  // bounds of the probability ratio: 1 - clip_low, 1 + clip_high
    float ent_coef, inv_temp;
};

// At least kLog2Zero, or NaN: a NaN or +inf among the logits makes all of the row's outputs NaN.
__device__ __forceinline__ float clamp_log2(float x) { return __builtin_elementwise_maximum(x, kLog2Zero); }

// What the gradient of a row needs, from its statistics.
struct PolicyRow {
    float logp, ent, loss;
    float a, b, d;  // gradient: p (a log2 p + b) + 1{taken} d
    bool some;      // a logit is not masked
};

template <bool LOSS>
__device__ __forceinline__ PolicyRow policy_row(const PolicyArgs& p, float z, float s, float u_taken,
                                                float logp_old, float adv, float w) {
    PolicyRow r{};
    const bool some = !(z == 0.f);  // (NaN is some)
    r.some = some;
    const float l2z = some ? log2_fast(z) : 0.f;
    r.logp = some ? kLn2 * (u_taken - l2z) : kNegInf;
    r.ent = some ? kLn2 * (l2z - s / z) : 0.f;
    if (LOSS) {
        const float rho = exp2_fast(kLog2e * (r.logp - logp_old));
        const float free = rho * adv, held = fminf(fmaxf(rho, p.low), p.high) * adv;
        // (fminf and fmaxf pass over NaN, and so does a comparison: one in logp_old or adv has to show. An infinite
        // ratio with an advantage of 0, whose product is NaN too, is held at the bound, and adds 0.)
        const bool bad = __builtin_isunordered(rho, adv);
        const float gain = bad ? __builtin_nanf("") : fminf(free, held);
        r.loss = w * (-gain - p.ent_coef * r.ent);
        const float g = bad ? gain : free <= held ? -w * free : 0.f;
        const float c = w * p.ent_coef;
        r.a = c * kLn2 * p.inv_temp;
        r.b = (c * r.ent - g) * p.inv_temp;
        r.d = g * p.inv_temp;
    }
    return r;
}

// The row's inputs beside its logits; false: the row is left out.
template <bool LOSS>
__device__ __forceinline__ bool policy_inputs(const PolicyArgs& p, int64_t row, int64_t& a, float& w, float& old, float& adv) {
    a = p.tokens[row];
    w = LOSS && p.weight ? p.weight[row] : 1.f;
    old = adv = 0.f;
    const bool part = a >= 0 && a < p.V && w != 0.f;
    if (LOSS && part) {
        old = p.logp_old[row];
        adv = p.adv[row];
    }
    return part;
}

template <bool LOSS>
__device__ __forceinline__ void policy_outputs(const PolicyArgs& p, int64_t row, const PolicyRow& r) {
    if (p.logp) p.logp[row] = r.logp;
    if (p.ent) p.ent[row] = r.ent;
    if (LOSS) p.loss[row] = r.loss;
}

// The gradient by a logit that is not the taken one.
__device__ __forceinline__ float policy_gradient(const PolicyRow& r, const Above& sc, float l2z, float x) {
    const float l = clamp_log2(fmaf(x - sc.top, sc.c, -l2z));
    return exp2_fast(l) * fmaf(r.a, l, r.b);
}

// Rows of up to L * E logits, L lanes a row, E logits a lane in registers: neighbours, where they make a
// vector, else L apart. Four lanes for the shortest, so that what is done once a row (a logarithm, two
// exponentials, the clip: some 150 operations) is done four times, not 64. 131072 x 18 float32, loss and gradient, 8.2 us (2.7 TB/s): one round of waves, which loads,
// computes (278 vector operations a wave, 3.7 us of a SIMD's eight) and stores. 65536 x 200 bfloat16 17.5 (3 TB/s).
template <typename DT, bool LOSS, int L, int E>
__global__ __launch_bounds__(4 * kWave) void policy_small_kernel(PolicyArgs p) {
    constexpr bool VEC = E == RowVec<DT>::K;
    const int lane = threadIdx.x & 63, i = lane % L;
    const int64_t row = (grid_row() * 4 + (threadIdx.x >> 6)) * (kWave / L) + lane / L;
    if (row >= p.M) return;  // (a whole group of L lanes leaves together)
    const DT* x = reinterpret_cast<const DT*>(p.logits) + row * p.ld;
    int64_t a;
    float w, old, adv, v[E];
    const bool part = policy_inputs<LOSS>(p, row, a, w, old, adv);
    PolicyRow r{};
    Above sc{};
    float l2z = 0.f;
    if (part) {
        // (all of a lane's logits are asked for before any is looked at)
        float top = kNegInf, taken;
        if constexpr (VEC) {
            RowVec<DT> asked;
            asked.load(x, i, p.V);
            taken = widen(x[a]);
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = asked.at(e);
        } else {
            DT asked[E];
#pragma unroll
            for (int e = 0; e < E; ++e) asked[e] = x[i + L * e < p.V ? i + L * e : int(p.V) - 1];
            taken = widen(x[a]);
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = i + L * e < p.V ? widen(asked[e]) : kNegInf;
        }
#pragma unroll
        for (int e = 0; e < E; ++e) top = fmaxf(top, v[e]);
        top = max_lanes<L>(top);
        sc = above(top, kLog2e * p.inv_temp);
        float z = 0.f, s = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float u = clamp_log2(sc.log2_weight(v[e])), q = exp2_fast(u);
            z += q;
            s = fmaf(q, u, s);
        }
        z = sum_lanes<L>(z);
        s = sum_lanes<L>(s);
        r = policy_row<LOSS>(p, z, s, sc.log2_weight(taken), old, adv, w);
        l2z = log2_fast(z);
    }
    if (LOSS && p.grad) {
        DT* g = reinterpret_cast<DT*>(p.grad) + row * p.ld_grad;
        float d[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            d[e] = part && r.some ? policy_gradient(r, sc, l2z, v[e]) : 0.f;
            if (part && (VEC ? i * E + e : i + L * e) == a) d[e] += r.d;
        }
        if constexpr (VEC) {
            if (i * E < p.V) store_row_vec<DT>(g, i, p.V, d);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (i + L * e < p.V) g[i + L * e] = narrow(d[e], DT{});
        }
    }
    if (i == 0) policy_outputs<LOSS>(p, row, r);
}

// Rows of up to U vectors a lane of W waves, which stay in registers: the maximum, the sums, the
// gradient. With W = 1 the four waves of a workgroup take a row each. Every logit is read and every gradient
// written once, and stores pass the caches by, which hold nothing that is read again. Bound by
// memory: 4096 x 32000 bfloat16 with gradient (524 MB) 102 us, 5.1 TB/s, without 52 us, 5.0; 65536 x 1000
// 43 us, 6 TB/s, some of it in the Infinity Cache.
template <typename DT, bool LOSS, int W, int U>
__global__ __launch_bounds__((W == 1 ? 4 : W) * kWave) void policy_vec_kernel(PolicyArgs p) {
    __shared__ float s_m[W], s_z[W], s_s[W];
    constexpr int K = RowVec<DT>::K, kLanes = W * kWave;
    const int tid = W == 1 ? int(threadIdx.x) & 63 : int(threadIdx.x), wave = tid >> 6;
    const int64_t row = W == 1 ? grid_row() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : grid_row();
    if (row >= p.M) return;
    const DT* x = reinterpret_cast<const DT*>(p.logits) + row * p.ld;
    DT* g = LOSS && p.grad ? reinterpret_cast<DT*>(p.grad) + row * p.ld_grad : nullptr;
    const int64_t vecs = (p.V + K - 1) / K;
    int64_t a;
    float w, old, adv;
    if (!policy_inputs<LOSS>(p, row, a, w, old, adv)) {
        if (tid == 0) policy_outputs<LOSS>(p, row, PolicyRow{});
        if (g) {
            const float zero[K] = {};
            for (int64_t i = tid; i < vecs; i += kLanes) store_row_vec<DT>(g, i, p.V, zero);
        }
        return;
    }
    RowVec<DT> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u].load(x, tid + u * kLanes, p.V);  // (past the end: -inf)
    const float taken = widen(x[a]);
    float top = kNegInf;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int k = 0; k < K; ++k) top = fmaxf(top, v[u].at(k));
    top = max_wave(top);
    if constexpr (W > 1) {
        if ((tid & 63) == 0) s_m[wave] = top;
        __syncthreads();  // (and everyone has read the taken logit, which the gradient may overwrite)
#pragma unroll
        for (int i = 0; i < W; ++i) top = fmaxf(top, s_m[i]);
    }
    const Above sc = above(top, kLog2e * p.inv_temp);
    float z = 0.f, s = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const float l = clamp_log2(sc.log2_weight(v[u].at(k))), e = exp2_fast(l);
            z += e;
            s = fmaf(e, l, s);
        }
    z = sum_wave(z);
    s = sum_wave(s);
    if constexpr (W > 1) {
        if ((tid & 63) == 0) {
            s_z[wave] = z;
            s_s[wave] = s;
        }
        __syncthreads();
        z = s = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            z += s_z[i];
            s += s_s[i];
        }
    }
    const PolicyRow r = policy_row<LOSS>(p, z, s, sc.log2_weight(taken), old, adv, w);
    if (tid == 0) policy_outputs<LOSS>(p, row, r);
    if (!g) return;
    const float l2z = log2_fast(z);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t i = tid + u * kLanes;
        float d[K];
#pragma unroll
        for (int k = 0; k < K; ++k) d[k] = r.some ? policy_gradient(r, sc, l2z, v[u].at(k)) : 0.f;
        if (i == a / K) {
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (k == a % K) d[k] += r.d;
        }
        if (i < vecs) store_row_vec<DT>(g, i, p.V, d);
    }
}

// Longer rows, one per workgroup of W waves: one pass for the statistics, each lane relative to its own
// running maximum, and one that writes the gradient, for which the row comes out of the caches. Bound by
// memory: 2048 x 50001 float32 without gradient (410 MB) 72 us, 5.7 TB/s; 8192 x 128000 bfloat16 with
// gradient (4.2 GB, and what the caches miss of another 2.1) 875 us, 4.8 TB/s, 685 with a third of the
// rows of weight 0. Sixteen waves with rows of up to 64 logits a lane in registers in place of the second
// reading are slower: one workgroup a CU waits where two take turns.
template <typename DT, bool LOSS, int W>
__global__ __launch_bounds__(W * kWave) void policy_rows_kernel(PolicyArgs p) {
    __shared__ float s_m[W], s_z[W], s_s[W];
    constexpr int K = RowVec<DT>::K, U = 4, kLanes = W * kWave;
    const int64_t row = grid_row();
    if (row >= p.M) return;
    const int tid = threadIdx.x;
    const DT* x = reinterpret_cast<const DT*>(p.logits) + row * p.ld;
    DT* g = LOSS && p.grad ? reinterpret_cast<DT*>(p.grad) + row * p.ld_grad : nullptr;
    const int64_t vecs = (p.V + K - 1) / K;
    int64_t a;
    float w, old, adv;
    if (!policy_inputs<LOSS>(p, row, a, w, old, adv)) {
        if (tid == 0) policy_outputs<LOSS>(p, row, PolicyRow{});
        if (g) {
            const float zero[K] = {};
            for (int64_t i = tid; i < vecs; i += kLanes) store_row_vec<DT>(g, i, p.V, zero);
        }
        return;
    }
    const float c = kLog2e * p.inv_temp;
    const float taken = widen(x[a]);
    // A lane's sums go chunk by chunk into 64 bits: one addition after another in 32 bits, 2^20 of them in the
    // longest rows, drifts by as much as a hundredth where weights are alike.
    float top = kNegInf;
    double zl = 0., sl = 0.;
    // sums relative to `top`, brought to a new maximum
    auto rebase = [&](auto& z, auto& s, float& top, float t) {
        const float d = top == t ? 0.f : fmaxf((top - t) * c, kLog2Zero), f = exp2_fast(d);
        s = f * (d * z + s);
        z *= f;
        top = t;
    };
    for (int64_t i0 = tid; i0 < vecs; i0 += U * kLanes) {
        RowVec<DT> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u].load(x, i0 + u * kLanes, p.V);  // (past the end: -inf)
        float t = top;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int k = 0; k < K; ++k) t = fmaxf(t, v[u].at(k));
        if (t > top) rebase(zl, sl, top, t);
        const Above sc = above(top, c);
        float z = 0.f, s = 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const float l = clamp_log2(sc.log2_weight(v[u].at(k))), e = exp2_fast(l);
                z += e;
                s = fmaf(e, l, s);
            }
        zl += z;
        sl += s;
    }
    // over the wave, then the workgroup: every lane's sums relative to one maximum
    rebase(zl, sl, top, max_wave(top));
    const float z = sum_wave(float(zl)), s = sum_wave(float(sl));
    if ((tid & 63) == 0) {
        s_m[tid >> 6] = top;
        s_z[tid >> 6] = z;
        s_s[tid >> 6] = s;
    }
    __syncthreads();  // (and everyone has read the taken logit, which the gradient may overwrite)
    float m = s_m[0];
#pragma unroll
    for (int i = 1; i < W; ++i) m = fmaxf(m, s_m[i]);
    float z1 = 0.f, s1 = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        float zw = s_z[i], sw = s_s[i], mw = s_m[i];
        rebase(zw, sw, mw, m);
        z1 += zw;
        s1 += sw;
    }
    const Above sc = above(m, c);
    const PolicyRow r = policy_row<LOSS>(p, z1, s1, sc.log2_weight(taken), old, adv, w);
    if (tid == 0) policy_outputs<LOSS>(p, row, r);
    if (!g) return;
    const float l2z = log2_fast(z1);
    // backwards: what the first pass read last is nearest in the caches
    for (int64_t i0 = (vecs - 1) / (U * kLanes) * (U * kLanes) + tid; i0 >= 0; i0 -= U * kLanes) {
        RowVec<DT> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u].load(x, i0 + u * kLanes, p.V);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t i = i0 + u * kLanes;
            float d[K];
#pragma unroll
            for (int k = 0; k < K; ++k) d[k] = r.some ? policy_gradient(r, sc, l2z, v[u].at(k)) : 0.f;
            if (i == a / K) {
#pragma unroll
                for (int k = 0; k < K; ++k)
                    if (k == a % K) d[k] += r.d;
            }
            if (i < vecs) store_row_vec<DT>(g, i, p.V, d);
        }
    }
}

}  // namespace rlcs
