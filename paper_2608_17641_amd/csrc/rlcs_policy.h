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

// What the gradient of a row needs, from its statistics.
struct PolicyRow {
    float logp, ent, loss;
    float a, b, d;  // gradient: p (a log2 p + b) + 1{taken} d
};

template <bool LOSS>
__device__ __forceinline__ PolicyRow policy_row(const PolicyArgs& p, float z, float s, float u_taken,
                                                float logp_old, float adv, float w) {
    PolicyRow r{};
    const bool some = z > 0.f;  // a logit that is not masked
    const float l2z = some ? log2_fast(z) : 0.f;
    r.logp = some ? kLn2 * (u_taken - l2z) : kNegInf;
    r.ent = some ? kLn2 * (l2z - s / z) : 0.f;
    if (LOSS) {
        const float rho = exp2_fast(kLog2e * (r.logp - logp_old));
        const float free = rho * adv, held = fminf(fmaxf(rho, p.low), p.high) * adv;
        r.loss = w * (-fminf(free, held) - p.ent_coef * r.ent);
        const float g = free <= held ? -w * free : 0.f;
        const float c = w * p.ent_coef;
        r.a = c * kLn2 * p.inv_temp;
        r.b = (c * r.ent - g) * p.inv_temp;
        r.d = g * p.inv_temp;
    }
    return r;
}

// One row per workgroup of W waves, element by element: any alignment, any length.
template <typename DT, bool LOSS, int W>
__global__ __launch_bounds__(W * kWave) void policy_rows_kernel(PolicyArgs p) {
    __shared__ float s_a[W], s_b[W], s_c[W];
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x;
    const DT* x = reinterpret_cast<const DT*>(p.logits) + row * p.ld;
    DT* g = p.grad ? reinterpret_cast<DT*>(p.grad) + row * p.ld_grad : nullptr;
    const int64_t a = p.tokens[row];
    const float w = LOSS && p.weight ? p.weight[row] : 1.f;
    const bool part = a >= 0 && a < p.V && w != 0.f;
    if (!part) {
        if (tid == 0) {
            if (p.logp) p.logp[row] = 0.f;
            if (p.ent) p.ent[row] = 0.f;
            if (LOSS) p.loss[row] = 0.f;
        }
        if (LOSS && g)
            for (int64_t j = tid; j < p.V; j += W * kWave) g[j] = narrow(0.f, DT{});
        return;
    }
    float top = kNegInf;
    for (int64_t j = tid; j < p.V; j += W * kWave) top = fmaxf(top, widen(x[j]));
    top = max_lanes(top);
    if ((tid & 63) == 0) s_a[tid >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < W; ++i) top = fmaxf(top, s_a[i]);
    const Scale sc = scale_of(top, kLog2e * p.inv_temp);
    float z = 0.f, s = 0.f;
    for (int64_t j = tid; j < p.V; j += W * kWave) {
        const float u = sc.log2_weight(widen(x[j])), e = exp2_fast(u);
        if (e > 0.f) {
            z += e;
            s = fmaf(e, u, s);
        }
    }
    z = sum_lanes(z);
    s = sum_lanes(s);
    if ((tid & 63) == 0) {
        s_b[tid >> 6] = z;
        s_c[tid >> 6] = s;
    }
    const float u_taken = sc.log2_weight(widen(x[a]));
    __syncthreads();  // (and everyone has read the taken logit, which the gradient may overwrite)
    z = s = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        z += s_b[i];
        s += s_c[i];
    }
    const PolicyRow r = policy_row<LOSS>(p, z, s, u_taken, LOSS ? p.logp_old[row] : 0.f, LOSS ? p.adv[row] : 0.f, w);
    if (LOSS && g) {
        const float l2z = log2_fast(z);
        for (int64_t j = tid; j < p.V; j += W * kWave) {
            const float l = sc.log2_weight(widen(x[j])) - l2z, q = exp2_fast(l);
            float v = q > 0.f ? q * fmaf(r.a, l, r.b) : 0.f;
            if (j == a) v += r.d;
            g[j] = narrow(v, DT{});
        }
    }
    if (tid == 0) {
        if (p.logp) p.logp[row] = r.logp;
        if (p.ent) p.ent[row] = r.ent;
        if (LOSS) p.loss[row] = r.loss;
    }
}

}  // namespace rlcs
