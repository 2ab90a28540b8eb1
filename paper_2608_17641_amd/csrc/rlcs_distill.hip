// Entry point of the distillation loss.
#include "rlcs_dispatch.h"
#include "rlcs_distill.h"

#include <cmath>

using namespace rlcs;
using namespace rlcs::host;

namespace {

template <typename DT, bool TAIL, int W, int U>
void launch_vec(const DistillArgs& a, hipStream_t s) {
    const int64_t rows = W == 1 ? 4 : 1;
    const size_t lds = distill_lds(a);
    hipLaunchKernelGGL((distill_vec_kernel<DT, TAIL, W, U>), row_grid((a.M + rows - 1) / rows), dim3((W == 1 ? 4 : W) * kWave), unsigned(rows * lds), s,
                       a, int(lds));
}
template <typename DT, bool TAIL, int W>
void launch_rows(const DistillArgs& a, hipStream_t s) {
    hipLaunchKernelGGL((distill_rows_kernel<DT, TAIL, W>), row_grid(a.M), dim3(W * kWave), unsigned(distill_lds(a)), s, a);
}

// As many waves and vectors a lane as hold the row in registers; longer rows are read twice, by 16 waves where there is no more
// than a row for each CU (128 rows of 128000 bfloat16: 22.7 us, 8 waves 27.6) and else by 8 (8192 rows: 710 us, 16 waves 753).
constexpr int64_t kFewRows = 256;

template <typename DT, bool TAIL>
rlcs_status run_distill(const DistillArgs& a, hipStream_t s) {
    constexpr bool kWide = sizeof(DT) == 4;
    constexpr int64_t k = kWide ? 1 : 2;  // rows of twice as many bfloat16 logits
    if (a.V <= 256 * k) launch_vec<DT, TAIL, 1, 1>(a, s);
    else if (a.V <= 512 * k) launch_vec<DT, TAIL, 1, 2>(a, s);
    else if (a.V <= 1024 * k) launch_vec<DT, TAIL, 1, 4>(a, s);
    else if (a.V <= 2048 * k) launch_vec<DT, TAIL, 1, 8>(a, s);
    else if (a.V <= 4096 * k) launch_vec<DT, TAIL, 4, 4>(a, s);
    else if (a.V <= 8192 * k) launch_vec<DT, TAIL, 4, 8>(a, s);
    else if (a.V <= 16384 * k) launch_vec<DT, TAIL, 8, 8>(a, s);
    else if (a.M <= kFewRows) launch_rows<DT, TAIL, 16>(a, s);
    else launch_rows<DT, TAIL, 8>(a, s);
    return hipGetLastError() == hipSuccess ? RLCS_OK : RLCS_ERR_LAUNCH;
}

template <typename DT>
rlcs_status run_distill(const DistillArgs& a, bool tail, hipStream_t s) {
    return tail ? run_distill<DT, true>(a, s) : run_distill<DT, false>(a, s);
}

}  // namespace

extern "C" {

rlcs_status rlcs_distill_loss(const void* logits, const int32_t* top_ids, const float* top_logp,
                              const float* weight, float* loss, void* dlogits, int64_t M,
                              int64_t V, int64_t K, int64_t ld, int64_t ld_grad, float temperature,
                              int tail, rlcs_dtype dtype, rlcs_stream_t stream) {
    if (M < 0 || V < 0 || K < 0) return RLCS_ERR_INVALID_ARG;
    if (dtype != RLCS_F32 && dtype != RLCS_BF16) return RLCS_ERR_DTYPE;
    if (M > INT32_MAX || V > kMaxT || K > kMaxListed || ld < V || (ld > 0 && M > INT64_MAX / 4 / ld)) return RLCS_ERR_INVALID_ARG;
    if (!positive(temperature) || !std::isfinite(temperature) || !std::isfinite(kLog2e / temperature)) return RLCS_ERR_INVALID_ARG;
    if (tail != 0 && tail != 1) return RLCS_ERR_INVALID_ARG;
    if (logits && !aligned(logits, dtype_size(dtype))) return RLCS_ERR_INVALID_ARG;
    for (const void* p : {static_cast<const void*>(top_ids), static_cast<const void*>(top_logp), static_cast<const void*>(weight),
                          static_cast<const void*>(loss)})
        if (p && !aligned(p, 4)) return RLCS_ERR_INVALID_ARG;
    if (dlogits && (!aligned(dlogits, dtype_size(dtype)) || ld_grad < V || (ld_grad > 0 && M > INT64_MAX / 4 / ld_grad)))
        return RLCS_ERR_INVALID_ARG;
    if (dlogits && dlogits == logits && ld_grad != ld) return RLCS_ERR_INVALID_ARG;
    if (M == 0 || V == 0) return RLCS_OK;
    if (!logits || !loss || (K && (!top_ids || !top_logp))) return RLCS_ERR_INVALID_ARG;
    DistillArgs a{};
    a.logits = logits; a.ids = top_ids; a.top = top_logp; a.weight = weight;
    a.loss = loss; a.grad = dlogits;
    a.M = M; a.V = V; a.ld = ld; a.ld_grad = ld_grad;
    a.K = int32_t(K);
    a.words = int32_t(((V < kBits ? V : kBits) + 127) / 128 * 4);
    a.inv_temp = 1.f / temperature;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    return dtype == RLCS_BF16 ? run_distill<bf16_t>(a, tail != 0, s) : run_distill<float>(a, tail != 0, s);
}

}  // extern "C"
