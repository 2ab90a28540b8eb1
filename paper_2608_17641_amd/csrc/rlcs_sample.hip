// Entry point of token sampling.
#include "rlcs_dispatch.h"
#include "rlcs_sample.h"

using namespace rlcs;
using namespace rlcs::host;

namespace {

template <typename DT, int L, int E>
void launch_small(const SampleArgs& a, hipStream_t s) {
    const int64_t rows = 4 * (kWave / L);
    hipLaunchKernelGGL((sample_small_kernel<DT, L, E>), row_grid((a.M + rows - 1) / rows), dim3(4 * kWave), 0, s, a);
}

template <typename DT, int W, int U, bool ONE>
void launch_rows(const SampleArgs& a, bool open, hipStream_t s) {
    const dim3 grid = row_grid(a.M), block(W * kWave);
    if (open) hipLaunchKernelGGL((sample_open_kernel<DT, W, U, ONE>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((sample_rows_kernel<DT, W, U, ONE>), grid, block, 0, s, a);
}

template <typename DT, int E>
void launch_wave(const SampleArgs& a, hipStream_t s) {
    hipLaunchKernelGGL((sample_wave_kernel<DT, E>), row_grid((a.M + 3) / 4), dim3(4 * kWave), 0, s, a);
}

// Unfiltered rows of at least kSplitFrom logits are split over workgroups where there are few of them:
// parts of at least kMinPart, as many as make kWantParts in all, up to 64 a row (a wave joins them).
constexpr int64_t kSplitFrom = 32768, kMinPart = 8192, kWantParts = 512;

int64_t open_parts(int64_t M, int64_t V) {
    if (V < kSplitFrom || M * 2 > kWantParts) return 1;
    int64_t parts = kWantParts / M;
    if (parts > V / kMinPart) parts = V / kMinPart;
    return parts > 64 ? 64 : parts;
}

// Waves a row: sixteen where a row has a CU to itself, four where there are rows enough to fill the
// CUs with small workgroups, whose waves spend less time at barriers and behind the one that ranks
// and draws (1024 x 30000 bfloat16 top-k 45 us with sixteen, 26 with four; top-p 107 and 86; 512 x 30000
// 24 with sixteen, 18 with eight; 64 x 32000 11 with sixteen).
template <typename DT>
rlcs_status run_sample(const SampleArgs& a, void* ws, size_t ws_bytes, hipStream_t s) {
    constexpr int kVec = 16 / sizeof(DT);
    // no row has a filter, as far as the host can tell
    const bool open = !a.top_k && !a.top_p && !a.min_p && (a.all_top_k <= 0 || a.all_top_k >= a.V) && a.all_top_p >= 1.f &&
                      !(a.all_min_p > 0.f);
    const int64_t parts = open ? open_parts(a.M, a.V) : 1;
    if (parts > 1 && ws && aligned(ws, 16) && ws_bytes >= size_t(a.M * parts) * sizeof(OpenPart)) {
        const int64_t length = ((a.V + parts - 1) / parts + kVec - 1) / kVec * kVec;  // (shorter than V / (parts - 1))
        const int count = int((a.V + length - 1) / length);
        OpenPart* p = static_cast<OpenPart*>(ws);
        hipLaunchKernelGGL((sample_parts_kernel<DT, 8, 2>), dim3(unsigned(count), unsigned(a.M)), dim3(8 * kWave), 0, s, a, p, length);
        hipLaunchKernelGGL((sample_join_kernel<DT>), dim3(unsigned(a.M)), dim3(4 * kWave), 0, s, a, p, count);
    } else if (open && a.V <= 1024) {
        if (a.V <= 32) launch_small<DT, 8, 4>(a, s);
        else if (a.V <= 64) launch_small<DT, 16, 4>(a, s);
        else if (a.V <= 128) launch_small<DT, 32, 4>(a, s);
        else if (a.V <= 256) launch_small<DT, 64, 4>(a, s);
        else launch_small<DT, 64, 16>(a, s);
    } else if (a.V <= 128) {
        launch_wave<DT, 2>(a, s);
    } else if (a.V <= 256) {
        launch_wave<DT, 4>(a, s);
    } else if (a.V <= 512) {
        launch_wave<DT, 8>(a, s);
    } else if (a.V <= 1024) {
        launch_wave<DT, 16>(a, s);
    } else if (a.V <= 2 * 256 * kVec) {  // rows that four waves hold in registers, two vectors a lane
        launch_rows<DT, 4, 2, true>(a, open, s);
    } else if (a.M >= 1024) {
        launch_rows<DT, 4, 2, false>(a, open, s);
    } else if (a.M > 256) {
        launch_rows<DT, 8, 2, false>(a, open, s);
    } else if (a.V <= 4 * 1024 * kVec) {
        launch_rows<DT, 16, 4, true>(a, open, s);
    } else {
        launch_rows<DT, 16, 4, false>(a, open, s);
    }
    return hipGetLastError() == hipSuccess ? RLCS_OK : RLCS_ERR_LAUNCH;
}

}  // namespace

extern "C" {

size_t rlcs_workspace_size_sample(int64_t M, int64_t V) {
    if (M < 1 || V < 1) return 0;
    const int64_t parts = open_parts(M, V);
    return parts > 1 ? size_t(M * parts) * sizeof(OpenPart) : 0;
}

rlcs_status rlcs_sample(const void* logits, const float* noise, const float* temperature,
                        const int32_t* top_k, const float* top_p, const float* min_p,
                        int32_t* tokens, float* logp, int64_t M, int64_t V, int64_t ld,
                        int64_t ld_noise, float all_temperature, int32_t all_top_k,
                        float all_top_p, float all_min_p, rlcs_dtype dtype, void* ws,
                        size_t ws_bytes, rlcs_stream_t stream) {
    if (M < 0 || V < 0) return RLCS_ERR_INVALID_ARG;
    if (dtype != RLCS_F32 && dtype != RLCS_BF16) return RLCS_ERR_DTYPE;
    if (M > INT32_MAX || V > (int64_t(1) << 24) || ld < V || (ld > 0 && M > INT64_MAX / 4 / ld)) return RLCS_ERR_INVALID_ARG;
    if (noise && (ld_noise < V || (ld_noise > 0 && M > INT64_MAX / 4 / ld_noise))) return RLCS_ERR_INVALID_ARG;
    if (all_temperature != all_temperature || all_top_p != all_top_p || all_min_p != all_min_p) return RLCS_ERR_INVALID_ARG;
    if (all_min_p > 1.f) return RLCS_ERR_INVALID_ARG;
    if (logits && !aligned(logits, dtype_size(dtype))) return RLCS_ERR_INVALID_ARG;
    for (const void* p : {static_cast<const void*>(noise), static_cast<const void*>(temperature), static_cast<const void*>(top_k),
                          static_cast<const void*>(top_p), static_cast<const void*>(min_p), static_cast<const void*>(tokens),
                          static_cast<const void*>(logp)})
        if (p && !aligned(p, 4)) return RLCS_ERR_INVALID_ARG;
    if (M == 0 || V == 0) return RLCS_OK;
    if (!logits || !tokens) return RLCS_ERR_INVALID_ARG;
    SampleArgs a{};
    a.logits = logits; a.noise = noise;
    a.temperature = temperature; a.top_k = top_k; a.top_p = top_p; a.min_p = min_p;
    a.tokens = tokens; a.logp = logp;
    a.M = M; a.V = V; a.ld = ld; a.ld_noise = ld_noise;
    a.all_temperature = all_temperature; a.all_top_k = all_top_k; a.all_top_p = all_top_p; a.all_min_p = all_min_p;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    return dtype == RLCS_BF16 ? run_sample<bf16_t>(a, ws, ws_bytes, s) : run_sample<float>(a, ws, ws_bytes, s);
}

}  // extern "C"
