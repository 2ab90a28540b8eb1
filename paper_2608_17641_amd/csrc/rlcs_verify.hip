// Entry point of the check of drafted tokens.
#include "rlcs_dispatch.h"
#include "rlcs_verify.h"

using namespace rlcs;
using namespace rlcs::host;

namespace {

constexpr int64_t kMaxDrafted = 1024;
// Parts of a row: as many as give kWantItems workgroups in all, each of at least kMinPart logits. (64 sequences of 7 tokens, 128000
// logits: 67 us; with 2048 workgroups 72, with 512 68. 256 of one token, 32000 logits: 33 us, 39, 34. Parts of at least 4096: alike.)
constexpr int64_t kWantItems = 1024, kMinPart = 2048, kMostParts = 64;

int64_t parts_of(int64_t rows, int64_t V) {
    int64_t parts = (kWantItems + rows - 1) / rows;
    if (parts > V / kMinPart) parts = V / kMinPart;
    if (parts > kMostParts) parts = kMostParts;
    return parts < 1 ? 1 : parts;
}

struct VerifySpace {
    int64_t sum_parts, race_parts;
    size_t sums, verdict, best, bytes;
};
VerifySpace space_of(int64_t B, int64_t K, int64_t V) {
    VerifySpace s{};
    const int64_t rows = B * (2 * K + 1);
    s.sum_parts = parts_of(rows, V);
    s.race_parts = parts_of(B, V);
    auto take = [&](size_t bytes) {
        const size_t at = s.bytes;
        s.bytes += (bytes + 15) / 16 * 16;
        return at;
    };
    s.sums = take(size_t(rows * s.sum_parts) * sizeof(RowSum));
    s.verdict = take(size_t(B) * sizeof(Verdict));
    s.best = take(size_t(B * s.race_parts) * 8);
    return s;
}
// Length of a part, a multiple of eight logits, with which there are no more than `parts`.
int64_t part_length(int64_t V, int64_t parts) { return ((V + parts - 1) / parts + 7) / 8 * 8; }

bool sizes_fit(int64_t B, int64_t K, int64_t V) {
    return B >= 0 && K >= 0 && V >= 0 && K <= kMaxDrafted && V <= (int64_t(1) << 24) && B <= INT32_MAX / (2 * K + 1) / kMostParts;
}

// Parts of at most this many logits are a wave's: a lane of four waves would have one vector or two.
constexpr int64_t kWaveRow = 2048;

template <typename DT>
rlcs_status run_verify(const VerifyArgs& a, hipStream_t s) {
    const int64_t rows = a.B * (a.K + 1) + (a.draft ? a.B * a.K : 0);
    if (a.sum_length <= kWaveRow) hipLaunchKernelGGL((verify_sums_kernel<DT, 1>), row_grid(rows * a.sum_parts), dim3(kWave), 0, s, a);
    else hipLaunchKernelGGL((verify_sums_kernel<DT, kVerifyWaves>), row_grid(rows * a.sum_parts), dim3(kVerifyWaves * kWave), 0, s, a);
    hipLaunchKernelGGL((verify_race_kernel<DT>), row_grid(a.B * a.race_parts), dim3(kVerifyWaves * kWave), 0, s, a);
    if (a.race_parts > 1) hipLaunchKernelGGL((verify_join_kernel<DT>), row_grid(a.B), dim3(kVerifyWaves * kWave), 0, s, a);
    return hipGetLastError() == hipSuccess ? RLCS_OK : RLCS_ERR_LAUNCH;
}

// Whether rows (b, i) at b * seq + i * ld of V elements have offsets within 63 bits.
bool reachable(int64_t B, int64_t rows, int64_t V, int64_t seq, int64_t ld) {
    const int64_t most = INT64_MAX / 8;
    if (seq < 0 || ld < 0) return false;
    if (rows > 1 && ld > (most - V) / rows) return false;
    return !(B > 1 && seq > (most - V - rows * ld) / B);
}

}  // namespace

extern "C" {

size_t rlcs_workspace_size_verify(int64_t B, int64_t K, int64_t V) {
    if (!sizes_fit(B, K, V) || B == 0 || V == 0) return 0;
    return space_of(B, K, V).bytes;
}

rlcs_status rlcs_verify_draft(const void* target, const void* draft, const int32_t* draft_tokens,
                              const float* u, const float* noise, const int32_t* n_draft,
                              const float* temperature, const float* draft_temperature,
                              int32_t* tokens, int32_t* count, float* logp, int64_t B, int64_t K,
                              int64_t V, int64_t target_seq, int64_t target_ld, int64_t draft_seq,
                              int64_t draft_ld, int64_t noise_ld, float all_temperature,
                              float all_draft_temperature, rlcs_dtype dtype, void* ws,
                              size_t ws_bytes, rlcs_stream_t stream) {
    if (B < 0 || K < 0 || V < 0) return RLCS_ERR_INVALID_ARG;
    if (dtype != RLCS_F32 && dtype != RLCS_BF16) return RLCS_ERR_DTYPE;
    if (!sizes_fit(B, K, V)) return RLCS_ERR_INVALID_ARG;
    if (all_temperature != all_temperature || all_draft_temperature != all_draft_temperature) return RLCS_ERR_INVALID_ARG;
    const size_t es = dtype_size(dtype);
    if (!aligned(target, es) || !aligned(draft, es)) return RLCS_ERR_INVALID_ARG;
    for (const void* p : {static_cast<const void*>(draft_tokens), static_cast<const void*>(u), static_cast<const void*>(noise),
                          static_cast<const void*>(n_draft), static_cast<const void*>(temperature), static_cast<const void*>(draft_temperature),
                          static_cast<const void*>(tokens), static_cast<const void*>(count), static_cast<const void*>(logp)})
        if (!aligned(p, 4)) return RLCS_ERR_INVALID_ARG;
    if (!reachable(B, K + 1, V, target_seq, target_ld) || !reachable(B, 1, V, noise_ld, 0)) return RLCS_ERR_INVALID_ARG;
    if (draft && !reachable(B, K, V, draft_seq, draft_ld)) return RLCS_ERR_INVALID_ARG;
    if (B == 0 || V == 0) return RLCS_OK;
    if (!target || !noise || !tokens || !count || (K && (!draft_tokens || !u))) return RLCS_ERR_INVALID_ARG;
    const VerifySpace space = space_of(B, K, V);
    if (!ws || ws_bytes < space.bytes) return RLCS_ERR_WORKSPACE;
    if (!aligned(ws, 16)) return RLCS_ERR_INVALID_ARG;
    VerifyArgs a{};
    a.target = target; a.draft = K ? draft : nullptr;
    a.draft_tokens = draft_tokens; a.n_draft = n_draft;
    a.u = u; a.noise = noise; a.temperature = temperature; a.draft_temperature = draft_temperature;
    a.tokens = tokens; a.count = count; a.logp = logp;
    a.B = B; a.V = V; a.K = int32_t(K);
    a.target_seq = target_seq; a.target_ld = target_ld; a.draft_seq = draft_seq; a.draft_ld = draft_ld; a.noise_ld = noise_ld;
    a.all_temperature = all_temperature; a.all_draft_temperature = all_draft_temperature;
    a.sum_length = part_length(V, space.sum_parts);
    a.race_length = part_length(V, space.race_parts);
    a.sum_parts = int32_t((V + a.sum_length - 1) / a.sum_length);
    a.race_parts = int32_t((V + a.race_length - 1) / a.race_length);
    char* w = static_cast<char*>(ws);
    a.sums = reinterpret_cast<RowSum*>(w + space.sums);
    a.verdict = reinterpret_cast<Verdict*>(w + space.verdict);
    a.best = reinterpret_cast<uint64_t*>(w + space.best);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    return dtype == RLCS_BF16 ? run_verify<bf16_t>(a, s) : run_verify<float>(a, s);
}

}  // extern "C"
