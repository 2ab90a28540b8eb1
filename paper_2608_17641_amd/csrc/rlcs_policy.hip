// Entry points of the policy's log-probabilities, entropies and loss.
#include "rlcs_dispatch.h"
#include "rlcs_policy.h"

#include <cmath>

using namespace rlcs;
using namespace rlcs::host;

namespace {

template <typename DT, bool LOSS, int L, int E>
void launch_small(const PolicyArgs& p, hipStream_t s) {
    const int64_t rows = 4 * (kWave / L);
    hipLaunchKernelGGL((policy_small_kernel<DT, LOSS, L, E>), row_grid((p.M + rows - 1) / rows), dim3(4 * kWave), 0, s, p);
}

template <typename DT, bool LOSS, int W, int U>
void launch_vec(const PolicyArgs& p, hipStream_t s) {
    const int64_t rows = W == 1 ? 4 : 1;
    hipLaunchKernelGGL((policy_vec_kernel<DT, LOSS, W, U>), row_grid((p.M + rows - 1) / rows), dim3((W == 1 ? 4 : W) * kWave), 0, s, p);
}

// Rows of up to 64 * E logits, a wave a row: float32 logits apart, bfloat16 ones in vectors.
template <typename DT, bool LOSS, int E>
void launch_wave(const PolicyArgs& p, hipStream_t s) {
    if constexpr (sizeof(DT) == 4) launch_small<DT, LOSS, 64, E>(p, s);
    else launch_vec<DT, LOSS, 1, E / 8>(p, s);
}

// Rows that do not fit the registers of eight waves (with sixteen, one workgroup would have the CU to
// itself and nothing to do while it waits: 4096 x 40000 bfloat16 196 us against 148) take sixteen
// waves where few rows leave CUs to them (64 x 128000 bfloat16 27 -> 24 us), and from this length
// on, where eight waves have twice as many rows in the caches between their two readings (2048 rows of
// 208 KB 195 -> 185 us, 256 KB 237 -> 215 float32 and 254 -> 230 bfloat16, 512 KB 594 -> 460); otherwise eight
// (8192 x 20000 float32 272 us against 330).
constexpr int64_t kFewRows = 256, kLongRow = 200 << 10;

template <typename DT, bool LOSS, int W>
void launch_rows(const PolicyArgs& p, hipStream_t s) {
    hipLaunchKernelGGL((policy_rows_kernel<DT, LOSS, W>), row_grid(p.M), dim3(W * kWave), 0, s, p);
}

// Short rows: as few lanes a row as hold it, four at least (131072 x 18 float32 8.5 us with four lanes of six
// logits, 9.8 with eight of four; 65536 x 120 14.5 with sixteen of eight, 15.4 with 32 of four; 65536 x 250
// 23 with 32 of eight, 31 with 64 of four), neighbours in a vector where that has as many (131072 x 31
// float32 11 us with eight lanes' vectors, 13 with four lanes of eight logits apart; 65536 x 200 bfloat16 17.5 and 23).
template <typename DT, bool LOSS>
rlcs_status run_policy(const PolicyArgs& p, hipStream_t s) {
    constexpr bool kWide = sizeof(DT) == 4;
    if (p.V <= 8) launch_small<DT, LOSS, 4, 2>(p, s);
    else if (p.V <= 16) launch_small<DT, LOSS, 4, 4>(p, s);
    else if (p.V <= 24) launch_small<DT, LOSS, 4, 6>(p, s);
    else if (p.V <= 32) launch_small<DT, LOSS, kWide ? 8 : 4, kWide ? 4 : 8>(p, s);
    else if (p.V <= 64) launch_small<DT, LOSS, 8, 8>(p, s);
    else if (p.V <= 128) launch_small<DT, LOSS, 16, 8>(p, s);
    else if (p.V <= 256) launch_small<DT, LOSS, 32, 8>(p, s);
    else if (p.V <= 512) launch_wave<DT, LOSS, 8>(p, s);
    else if (p.V <= 1024) launch_wave<DT, LOSS, 16>(p, s);
    else if (p.V <= 2048) launch_vec<DT, LOSS, 1, kWide ? 8 : 4>(p, s);
    else if (p.V <= 4096) launch_vec<DT, LOSS, kWide ? 4 : 1, kWide ? 4 : 8>(p, s);
    else if (p.V <= 8192) launch_vec<DT, LOSS, 4, kWide ? 8 : 4>(p, s);
    else if (p.V <= 16384) launch_vec<DT, LOSS, kWide ? 8 : 4, 8>(p, s);
    else if (!kWide && p.V <= 32768) launch_vec<DT, LOSS, 8, 8>(p, s);
    else if (p.M <= kFewRows || p.V * int64_t(sizeof(DT)) >= kLongRow) launch_rows<DT, LOSS, 16>(p, s);
    else launch_rows<DT, LOSS, 8>(p, s);
    return hipGetLastError() == hipSuccess ? RLCS_OK : RLCS_ERR_LAUNCH;
}

// Sizes, type and alignment of what both entry points share.
rlcs_status check_rows(int64_t M, int64_t V, int64_t ld, float temperature, rlcs_dtype dtype, const void* logits,
                       std::initializer_list<const void*> words) {
    if (M < 0 || V < 0) return RLCS_ERR_INVALID_ARG;
    if (dtype != RLCS_F32 && dtype != RLCS_BF16) return RLCS_ERR_DTYPE;
    if (M > INT32_MAX || V > kMaxT || ld < V || (ld > 0 && M > INT64_MAX / 4 / ld)) return RLCS_ERR_INVALID_ARG;
    if (!positive(temperature) || !std::isfinite(temperature) || !std::isfinite(kLog2e / temperature)) return RLCS_ERR_INVALID_ARG;
    if (logits && !aligned(logits, dtype_size(dtype))) return RLCS_ERR_INVALID_ARG;
    for (const void* p : words)
        if (p && !aligned(p, 4)) return RLCS_ERR_INVALID_ARG;
    return RLCS_OK;
}

}  // namespace

extern "C" {

rlcs_status rlcs_token_logp(const void* logits, const int32_t* tokens, float* logp, float* ent,
                            int64_t M, int64_t V, int64_t ld, float temperature, rlcs_dtype dtype,
                            rlcs_stream_t stream) {
    const rlcs_status st = check_rows(M, V, ld, temperature, dtype, logits, {tokens, logp, ent});
    if (st != RLCS_OK) return st;
    if (M == 0 || V == 0) return RLCS_OK;
    if (!logits || !tokens || !logp) return RLCS_ERR_INVALID_ARG;
    PolicyArgs p{};
    p.logits = logits; p.tokens = tokens; p.logp = logp; p.ent = ent;
    p.M = M; p.V = V; p.ld = ld; p.inv_temp = 1.f / temperature;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    return dtype == RLCS_BF16 ? run_policy<bf16_t, false>(p, s) : run_policy<float, false>(p, s);
}

rlcs_status rlcs_policy_loss(const void* logits, const int32_t* tokens, const float* logp_old,
                             const float* adv, const float* weight, float* loss, void* dlogits,
                             float* logp, float* ent, int64_t M, int64_t V, int64_t ld,
                             int64_t ld_grad, float clip_low, float clip_high, float ent_coef,
                             float temperature, rlcs_dtype dtype, rlcs_stream_t stream) {
    const rlcs_status st = check_rows(M, V, ld, temperature, dtype, logits, {tokens, logp_old, adv, weight, loss, logp, ent});
    if (st != RLCS_OK) return st;
    if (!unit_interval(clip_low) || !(clip_high >= 0.f) || !std::isfinite(ent_coef)) return RLCS_ERR_INVALID_ARG;
    if (dlogits && (!aligned(dlogits, dtype_size(dtype)) || ld_grad < V || (ld_grad > 0 && M > INT64_MAX / 4 / ld_grad)))
        return RLCS_ERR_INVALID_ARG;
    if (dlogits && dlogits == logits && ld_grad != ld) return RLCS_ERR_INVALID_ARG;
    if (M == 0 || V == 0) return RLCS_OK;
    if (!logits || !tokens || !logp_old || !adv || !loss) return RLCS_ERR_INVALID_ARG;
    PolicyArgs p{};
    p.logits = logits; p.tokens = tokens; p.logp_old = logp_old; p.adv = adv; p.weight = weight;
    p.loss = loss; p.logp = logp; p.ent = ent; p.grad = dlogits;
    p.M = M; p.V = V; p.ld = ld; p.ld_grad = ld_grad;
    p.low = 1.f - clip_low; p.high = 1.f + clip_high; p.ent_coef = ent_coef; p.inv_temp = 1.f / temperature;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    return dtype == RLCS_BF16 ? run_policy<bf16_t, true>(p, s) : run_policy<float, true>(p, s);
}

}  // extern "C"
