// Attention of single-token queries over a group's shared prefix and each sequence's own suffix.
#pragma once

#include "rlcs.h"
#include "rlcs_softmax.h"

namespace rlcs {

struct AttnArgs {
    const void *q, *kp, *vp, *ks, *vs;
    const int32_t *prefix_len, *suffix_len;
    void* o;
    float* lse;
    int64_t N, G, Hq, Hkv, D, P, S;
    rlcs_attn_layout at;
    float scale2;  // scale * log2(e): scores in base 2
};

__device__ __forceinline__ int64_t clamp_len(const int32_t* p, int64_t i, int64_t most) {
    if (!p) return most;
    const int64_t n = p[i];
    return n < 0 ? 0 : n > most ? most : n;
}

constexpr int kAttnSlots = 4;  // elements of a head a lane holds: D <= 256

// One wave per query head: key after key, a dot product over the lanes each.
template <typename DT>
__global__ __launch_bounds__(kWave) void attn_heads_kernel(AttnArgs a) {
    const int lane = threadIdx.x;
    const int64_t h = blockIdx.x, g = blockIdx.y, n = blockIdx.z;
    const int64_t hk = h / (a.Hq / a.Hkv);
    const DT* q = reinterpret_cast<const DT*>(a.q) + n * a.at.q[0] + g * a.at.q[1] + h * a.at.q[2];
    float x[kAttnSlots], acc[kAttnSlots] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kAttnSlots; ++i) {
        const int d = lane + 64 * i;
        x[i] = d < a.D ? widen(q[d]) * a.scale2 : 0.f;
    }
    float m = kNegInf, z = 0.f;
    auto part = [&](const DT* k, const DT* v, int64_t len, int64_t sk, int64_t sv) {
        for (int64_t j = 0; j < len; ++j) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < kAttnSlots; ++i)
                if (lane + 64 * i < a.D) s = fmaf(x[i], widen(k[j * sk + lane + 64 * i]), s);
#pragma unroll
            for (int d = 1; d < kWave; d <<= 1) s += __shfl_xor(s, d);
            const float m1 = fmaxf(m, s), keep = exp2_fast(m - m1), w = exp2_fast(s - m1);
            m = m1;
            z = fmaf(z, keep, w);
#pragma unroll
            for (int i = 0; i < kAttnSlots; ++i)
                if (lane + 64 * i < a.D) acc[i] = fmaf(acc[i], keep, w * widen(v[j * sv + lane + 64 * i]));
        }
    };
    part(reinterpret_cast<const DT*>(a.kp) + n * a.at.kp[0] + hk * a.at.kp[2],
         reinterpret_cast<const DT*>(a.vp) + n * a.at.vp[0] + hk * a.at.vp[2],
         clamp_len(a.prefix_len, n, a.P), a.at.kp[1], a.at.vp[1]);
    part(reinterpret_cast<const DT*>(a.ks) + n * a.at.ks[0] + g * a.at.ks[1] + hk * a.at.ks[3],
         reinterpret_cast<const DT*>(a.vs) + n * a.at.vs[0] + g * a.at.vs[1] + hk * a.at.vs[3],
         clamp_len(a.suffix_len, n * a.G + g, a.S), a.at.ks[2], a.at.vs[2]);
    const int64_t row = (n * a.G + g) * a.Hq + h;
    DT* o = reinterpret_cast<DT*>(a.o) + row * a.D;
#pragma unroll
    for (int i = 0; i < kAttnSlots; ++i)
        if (lane + 64 * i < a.D) o[lane + 64 * i] = narrow(z > 0.f ? acc[i] / z : 0.f, DT{});
    if (a.lse && lane == 0) a.lse[row] = z > 0.f ? kLn2 * (m + log2_fast(z)) : kNegInf;
}

}  // namespace rlcs
