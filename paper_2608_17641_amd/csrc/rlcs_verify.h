// Drafted tokens against the target policy: which stand, and the token that follows them.
//
// Token x_i stands if u_i q_i(x_i) < p_i(x_i); after the first that falls one is drawn from max(p - q, 0). The
// draw is a race as the sampler's: of independent E_j ~ Exp(1) the largest log(w_j) - log(E_j) is at j with
// probability w_j / sum w, so neither the normalisation of what is left of p nor a prefix sum is needed.
//
// First the maximum and the sum of weights of every row of both (a row is cut into parts, where there are few
// rows); then, a few workgroups a sequence, the comparison of all its drafted tokens at once, and the race over the
// row that it comes down to; then, where a row's race was cut into parts, their best. The sums are bound by memory, the rest by
// latency and by what the race computes a logit. 64 sequences of up to 7 drafted tokens, 128000 bfloat16 logits: sums 44 us (205 MB
// fetched, 4.7 TB/s), race 19 us, its join 5; 8 of 4, 32000 float32: 5.5, 7.3 and 3.
#pragma once

#include "rlcs_sample.h"

namespace rlcs {

constexpr int kVerifyWaves = 4;

struct VerifyArgs {
    const void *target, *draft;
    const int32_t *draft_tokens, *n_draft;
    const float *u, *noise, *temperature, *draft_temperature;
    int32_t *tokens, *count;
    float* logp;
    int64_t B, V, target_seq, target_ld, draft_seq, draft_ld, noise_ld;
    int32_t K;
    float all_temperature, all_draft_temperature;
    // parts of a row in the sums and in the race, and their lengths (multiples of a vector)
    int32_t sum_parts, race_parts;
    int64_t sum_length, race_length;
    struct RowSum* sums;    // [row][sum_parts]: target rows, then draft rows
    struct Verdict* verdict;  // [B]
    uint64_t* best;         // [B][race_parts]
};

// A part of a row: its largest logit and the sum of the weights relative to it; of a temperature of 0 the place of the
// largest logit, as race_entry().
struct RowSum {
    union {
        struct {
            float top, sum;
        };
        uint64_t entry;
    };
};

// A sequence's row to draw from.
struct Verdict {
    int32_t n, greedy;  // tokens that stand; greedy: the drawn token, -2 where there is a race
    float top, c, l2z;
};

__device__ __forceinline__ float temperature_scale(float t) { return t > 0.f ? fmaxf(kLog2e / t, 1.1754944e-38f) : kInf; }
__device__ __forceinline__ float target_scale(const VerifyArgs& a, int64_t b) {
    return temperature_scale(a.temperature ? a.temperature[b] : a.all_temperature);
}
// (of a temperature of 0: what differs from the largest logit at all weighs nothing)
__device__ __forceinline__ float draft_scale(const VerifyArgs& a, int64_t b) {
    return fminf(temperature_scale(a.draft_temperature ? a.draft_temperature[b] : a.all_draft_temperature), 0x1p127f);
}
__device__ __forceinline__ int drafted(const VerifyArgs& a, int64_t b) {
    const int n = a.n_draft ? a.n_draft[b] : a.K;
    return n < 0 ? 0 : n > a.K ? a.K : n;
}
template <typename DT>
__device__ __forceinline__ const DT* target_row(const VerifyArgs& a, int64_t b, int i) {
    return reinterpret_cast<const DT*>(a.target) + b * a.target_seq + i * a.target_ld;
}
template <typename DT>
__device__ __forceinline__ const DT* draft_row(const VerifyArgs& a, int64_t b, int i) {
    return reinterpret_cast<const DT*>(a.draft) + b * a.draft_seq + i * a.draft_ld;
}
// A logit as it counts: NaN as -inf, +inf as the type's largest number.
template <typename DT>
__device__ __forceinline__ float counted(float v) {
    return RowView<DT, Above>::finite(fmaxf(v, kNegInf));
}

// The largest logit and the sum of weights of part blockIdx.x of a row, by W waves.
template <typename DT, int W>
__global__ __launch_bounds__(W * kWave) void verify_sums_kernel(VerifyArgs a) {
    constexpr int K = RowVec<DT>::K, U = 4, kLanes = W * kWave;
    __shared__ float s_top[W], s_sum[W];
    __shared__ uint64_t s_slots[W];
    const int64_t item = grid_row(), rows = a.B * (2 * int64_t(a.K) + 1);
    const int64_t row = item / a.sum_parts, part = item % a.sum_parts;
    if (row >= rows) return;
    const bool is_target = row < a.B * (a.K + 1);
    const int64_t in_kind = is_target ? row : row - a.B * (a.K + 1);
    const int of_seq = is_target ? a.K + 1 : a.K;
    const int64_t b = in_kind / of_seq;
    const int i = int(in_kind % of_seq), n = drafted(a, b);
    if (i > n || (!is_target && (i == n || !a.draft))) return;
    const DT* x = is_target ? target_row<DT>(a, b, i) : draft_row<DT>(a, b, i);
    const float c = is_target ? target_scale(a, b) : draft_scale(a, b);
    const int tid = threadIdx.x;
    const int64_t from = part * a.sum_length / K, most = (a.V + K - 1) / K;
    const int64_t end = from + a.sum_length / K < most ? from + a.sum_length / K : most;
    RowSum* out = a.sums + item;
    if (is_target && c == kInf) {
        uint64_t best = 0;
        for (int64_t v = from + tid; v < end; v += kLanes) {
            RowVec<DT> r;
            r.load(x, v, a.V);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const float y = counted<DT>(r.at(k));
                const uint64_t e = y > kNegInf ? race_entry(order_key(y), uint32_t(v * K + k)) : 0;
                best = e > best ? e : best;
            }
        }
        best = max_group<W>(best, s_slots);
        if (tid == 0) out->entry = best;
        return;
    }
    float top = kNegInf;
    double sum = 0.;
    auto rebase = [&](auto& z, float t) {
        z *= top == t ? 1.f : exp2_fast(fmaxf((top - t) * c, kLog2Zero));
        top = t;
    };
    for (int64_t v0 = from + tid; v0 < end; v0 += U * kLanes) {
        RowVec<DT> r[U];
#pragma unroll
        for (int q = 0; q < U; ++q) r[q].load(x, v0 + q * kLanes, v0 + q * kLanes < end ? a.V : 0);  // (past the end: -inf)
        float y[U][K], t = top;
#pragma unroll
        for (int q = 0; q < U; ++q)
#pragma unroll
            for (int k = 0; k < K; ++k) {
                y[q][k] = counted<DT>(r[q].at(k));
                t = fmaxf(t, y[q][k]);
            }
        if (t > top) rebase(sum, t);
        const Above sc = above(top, c);
        float z = 0.f;
#pragma unroll
        for (int q = 0; q < U; ++q)
#pragma unroll
            for (int k = 0; k < K; ++k) z += exp2_fast(sc.log2_weight(y[q][k]));
        sum += z;
    }
    rebase(sum, max_wave(top));
    float z = sum_wave(float(sum));
    if constexpr (W > 1) {
        if ((tid & 63) == 0) {
            s_top[tid >> 6] = top;
            s_sum[tid >> 6] = z;
        }
        __syncthreads();
        float m = s_top[0];
#pragma unroll
        for (int w = 1; w < W; ++w) m = fmaxf(m, s_top[w]);
        z = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            top = s_top[w];
            float zw = s_sum[w];
            rebase(zw, m);
            z += zw;
        }
    }
    if (tid == 0) {
        out->top = top;
        out->sum = z;
    }
}

// A row's softmax: weights 2^((x - top) c) and one over their sum (0 where there is none).
struct RowSoftmax {
    Above sc;
    float sum;
    __device__ __forceinline__ float weight(float x) const { return exp2_fast(sc.log2_weight(x)); }
    __device__ __forceinline__ float probability(float x) const { return sum > 0.f ? weight(x) / sum : 0.f; }
};
// By a wave, from the row's parts, one a lane.
__device__ __forceinline__ RowSoftmax row_softmax(const VerifyArgs& a, int64_t row, float c) {
    const int lane = threadIdx.x & 63;
    RowSum s;
    s.top = kNegInf;
    s.sum = 0.f;
    if (lane < a.sum_parts) s = a.sums[row * a.sum_parts + lane];
    const float top = max_wave(s.top);
    const float f = s.top == top ? 1.f : exp2_fast(fmaxf((s.top - top) * c, kLog2Zero));
    return RowSoftmax{above(top, c), sum_wave(f * s.sum)};
}
__device__ __forceinline__ uint64_t row_largest(const VerifyArgs& a, int64_t row) {
    const int lane = threadIdx.x & 63;
    return max_wave(lane < a.sum_parts ? a.sums[row * a.sum_parts + lane].entry : uint64_t(0));
}

// The drawn token of sequence b: place n, and what is -1 and 0 after it.
__device__ __forceinline__ void verify_finish(const VerifyArgs& a, int64_t b, int n, int32_t token, float logp) {
    const int64_t row = b * (a.K + 1);
    a.tokens[row + n] = token;
    a.count[b] = n + 1;
    if (a.logp) a.logp[row + n] = logp;
}
template <typename DT>
__device__ __forceinline__ void verify_drawn(const VerifyArgs& a, int64_t b, const Verdict& v, uint64_t winner) {
    if (!winner) {
        verify_finish(a, b, v.n, -1, kNegInf);
        return;
    }
    const int32_t token = int32_t(race_index(winner));
    const float u = Above{v.top, v.c}.log2_weight(counted<DT>(widen(target_row<DT>(a, b, v.n)[token])));
    verify_finish(a, b, v.n, token, kLn2 * (u - v.l2z));
}

// A lane's share of a race over vectors [from, end) of a row, as an entry (0: it has none). w(logits, i, k) is the weight of
// element k of vector i, a number from 0 to 1; none has a weight of 0. Scores are w / E, which order as log w - log E does; where the best is
// near an end of float32's range (numbers E that no exponential draw gives) the lane takes logarithms.
template <typename DT, class F>
__device__ __forceinline__ uint64_t race_lane(const DT* x, const float* noise, int64_t V, int64_t from, int64_t end, int step, F&& weight) {
    constexpr int K = RowVec<DT>::K;
    auto run = [&](auto logs) {
        float best = kNegInf;
        uint32_t at = 0;
        bool some = false;
        for (int64_t i = from; i < end; i += step) {
            RowVec<DT> r;
            r.load(x, i, V);
            float e[K], w[K];
            if ((i + 1) * K <= V) {
#pragma unroll
                for (int k = 0; k < K; k += 4) {
                    const u32x4 word = *reinterpret_cast<const u32x4_any*>(noise + i * K + k);
#pragma unroll
                    for (int m = 0; m < 4; ++m) e[k + m] = __uint_as_float(word[m]);
                }
            } else {
#pragma unroll
                for (int k = 0; k < K; ++k) e[k] = i * K + k < V ? noise[i * K + k] : 1.f;
            }
            weight(r, i, w);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const float score = decltype(logs)::value ? noise_log2(w[k]) - noise_log2(e[k]) : w[k] * __builtin_amdgcn_rcpf(e[k]);
                const bool ahead = w[k] > 0.f && (score > best || !some);
                best = ahead ? score : best;
                at = ahead ? uint32_t(i * K + k) : at;
                some |= ahead;
            }
        }
        if (!some) return uint64_t(0);
        if (!decltype(logs)::value) {
            if (!(best > 0x1p-100f && best < 0x1p100f)) return ~uint64_t(0);
            best = log2_fast(best);
        }
        return race_entry(order_key(best), at);
    };
    const uint64_t fast = run(std::false_type{});
    return fast == ~uint64_t(0) ? run(std::true_type{}) : fast;
}
// The race over all of p: where no token fell, and where q leaves nothing.
template <typename DT>
__device__ __forceinline__ uint64_t race_all(const DT* x, const float* noise, int64_t V, int64_t from, int64_t end, int step, Above sc) {
    return race_lane<DT>(x, noise, V, from, end, step, [&](const RowVec<DT>& r, int64_t, float (&w)[RowVec<DT>::K]) {
#pragma unroll
        for (int k = 0; k < RowVec<DT>::K; ++k) {
            const float y = counted<DT>(r.at(k));
            // (a token that is not masked takes part, however little it weighs)
            w[k] = y > kNegInf ? fmaxf(exp2_fast(sc.log2_weight(y)), 0x1p-126f) : 0.f;
        }
    });
}

// Part blockIdx of a sequence's race, after the comparison of its drafted tokens, which every part makes for itself.
template <typename DT>
__global__ __launch_bounds__(kVerifyWaves * kWave) void verify_race_kernel(VerifyArgs a) {
    constexpr int K = RowVec<DT>::K, W = kVerifyWaves, kLanes = W * kWave;
    __shared__ uint64_t s_slots[W];
    __shared__ int s_first;
    const int64_t item = grid_row();
    const int64_t b = item / a.race_parts, part = item % a.race_parts;
    if (b >= a.B) return;
    const int tid = threadIdx.x, n_draft = drafted(a, b);
    const float c = target_scale(a, b);
    const bool greedy = c == kInf;
    const int64_t targets = b * (a.K + 1), drafts = a.B * (a.K + 1) + b * a.K;
    if (tid == 0) s_first = n_draft;
    __syncthreads();
    // a wave a drafted token; the ones after a token that fell do not matter
    for (int i = tid >> 6; i < n_draft && i < *static_cast<volatile int*>(&s_first); i += W) {
        const int64_t token = a.draft_tokens[b * a.K + i];
        bool stands = false;
        float logp = 0.f;
        if (token >= 0 && token < a.V) {
            const float u = a.u[b * a.K + i], x = counted<DT>(widen(target_row<DT>(a, b, i)[token]));
            float q = 1.f, p;
            if (a.draft) {
                const float y = counted<DT>(widen(draft_row<DT>(a, b, i)[token]));
                q = row_softmax(a, drafts + i, draft_scale(a, b)).probability(y);
            }
            if (greedy) {
                const uint64_t e = row_largest(a, targets + i);
                p = e && race_index(e) == uint32_t(token) ? 1.f : 0.f;
            } else {
                const RowSoftmax s = row_softmax(a, targets + i, c);
                p = s.probability(x);
                logp = kLn2 * (s.sc.log2_weight(x) - log2_fast(s.sum));
            }
            stands = u * q < p;
        }
        if ((tid & 63) == 0) {
            if (!stands) atomicMin(&s_first, i);
            if (part == 0) {  // (places from the first that falls on are written again)
                a.tokens[targets + i] = int32_t(token);
                if (a.logp) a.logp[targets + i] = logp;
            }
        }
    }
    __syncthreads();
    const int n = s_first;
    if (part == 0) {
        for (int i = n + 1 + tid; i <= a.K; i += kLanes) {
            a.tokens[targets + i] = -1;
            if (a.logp) a.logp[targets + i] = 0.f;
        }
    }
    Verdict v{n, -2, 0.f, c, 0.f};
    if (greedy) {
        const uint64_t e = row_largest(a, targets + n);
        v.greedy = e ? int32_t(race_index(e)) : -1;
        if (part == 0 && tid == 0) {
            a.verdict[b] = v;
            verify_finish(a, b, n, v.greedy, e ? 0.f : kNegInf);
        }
        return;
    }
    const RowSoftmax p = row_softmax(a, targets + n, c);
    const bool fell = n < n_draft;
    // (a draft without logits has all of its mass on the token that fell)
    const int64_t fallen = fell && !a.draft ? a.draft_tokens[b * a.K + n] : -1;
    const bool minus = fell && a.draft;
    const RowSoftmax q = minus ? row_softmax(a, drafts + n, draft_scale(a, b)) : RowSoftmax{Above{0.f, 0.f}, 0.f};
    v.top = p.sc.top;
    v.l2z = log2_fast(p.sum);
    const DT *xp = target_row<DT>(a, b, n), *xq = minus ? draft_row<DT>(a, b, n) : xp;
    const float* noise = a.noise + b * a.noise_ld;
    const float inv_p = 1.f / p.sum, inv_q = q.sum > 0.f ? 1.f / q.sum : 0.f;
    const int64_t from = part * a.race_length / K + tid, most = (a.V + K - 1) / K;
    const int64_t past = (part + 1) * a.race_length / K, end = past < most ? past : most;
    uint64_t winner;
    if (minus) {
        winner = race_lane<DT>(xp, noise, a.V, from, end, kLanes, [&](const RowVec<DT>& r, int64_t i, float (&w)[K]) {
            RowVec<DT> rq;
            rq.load(xq, i, a.V);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                // (each product rounded by itself, so that of equal rows nothing is left)
#pragma clang fp contract(off)
                const float of_p = p.weight(counted<DT>(r.at(k))) * inv_p, of_q = q.weight(counted<DT>(rq.at(k))) * inv_q;
                w[k] = of_p - of_q;
            }
        });
    } else if (fell) {
        winner = race_lane<DT>(xp, noise, a.V, from, end, kLanes, [&](const RowVec<DT>& r, int64_t i, float (&w)[K]) {
#pragma unroll
            for (int k = 0; k < K; ++k) w[k] = i * K + k == fallen ? 0.f : p.weight(counted<DT>(r.at(k)));
        });
    } else {
        winner = race_all<DT>(xp, noise, a.V, from, end, kLanes, p.sc);
    }
    winner = max_group<W>(winner, s_slots);
    if (a.race_parts > 1) {
        if (tid == 0) {
            if (part == 0) a.verdict[b] = v;
            a.best[item] = winner;
        }
        return;
    }
    if (!winner) winner = max_group<W>(race_all<DT>(xp, noise, a.V, tid, most, kLanes, p.sc), s_slots);
    if (tid == 0) verify_drawn<DT>(a, b, v, winner);
}

// The best of a race's parts, a workgroup a sequence; where q has left nothing, the race over all of p.
template <typename DT>
__global__ __launch_bounds__(kVerifyWaves * kWave) void verify_join_kernel(VerifyArgs a) {
    constexpr int W = kVerifyWaves, K = RowVec<DT>::K;
    __shared__ uint64_t s_slots[W];
    const int64_t b = grid_row();
    if (b >= a.B) return;
    const Verdict v = a.verdict[b];
    if (v.greedy != -2) return;  // (written already)
    const int tid = threadIdx.x, lane = tid & 63;
    uint64_t winner = max_wave(lane < a.race_parts ? a.best[b * a.race_parts + lane] : uint64_t(0));
    if (!winner)
        winner = max_group<W>(race_all<DT>(target_row<DT>(a, b, v.n), a.noise + b * a.noise_ld, a.V, tid, (a.V + K - 1) / K, W * kWave, Above{v.top, v.c}),
                              s_slots);
    if (tid == 0) verify_drawn<DT>(a, b, v, winner);
}

}  // namespace rlcs
