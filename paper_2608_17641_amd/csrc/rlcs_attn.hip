// Entry point of attention over a shared prefix.
#include "rlcs_attn.h"
#include "rlcs_dispatch.h"

#include <cmath>

using namespace rlcs;
using namespace rlcs::host;

namespace {

constexpr int64_t kMaxHeadDim = 256;

// Whether the elements that an array's strides reach have 63-bit offsets: the sum of
// (size - 1) * stride over its dimensions.
bool reachable(std::initializer_list<int64_t> sizes, const int64_t* strides) {
    int64_t last = kMaxHeadDim;
    int i = 0;
    for (const int64_t n : sizes) {
        const int64_t s = strides[i++];
        if (s < 0) return false;
        if (n <= 1 || s == 0) continue;
        if (s > (INT64_MAX / 8 - last) / (n - 1)) return false;
        last += (n - 1) * s;
    }
    return true;
}

template <typename DT>
rlcs_status run_attn(const AttnArgs& a, hipStream_t s) {
    hipLaunchKernelGGL((attn_heads_kernel<DT>), dim3(unsigned(a.Hq), unsigned(a.G), unsigned(a.N)), dim3(kWave), 0, s, a);
    return hipGetLastError() == hipSuccess ? RLCS_OK : RLCS_ERR_LAUNCH;
}

}  // namespace

extern "C" {

size_t rlcs_workspace_size_attn(int64_t, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t) { return 0; }

rlcs_status rlcs_shared_prefix_attn(const void* q, const void* kp, const void* vp, const void* ks,
                                    const void* vs, const int32_t* prefix_len,
                                    const int32_t* suffix_len, void* o, float* lse, int64_t N,
                                    int64_t G, int64_t Hq, int64_t Hkv, int64_t D, int64_t P,
                                    int64_t S, const rlcs_attn_layout* layout, float scale,
                                    rlcs_dtype dtype, void* ws, size_t ws_bytes,
                                    rlcs_stream_t stream) {
    if (N < 0 || G < 0 || Hq < 0 || Hkv < 0 || D < 0 || P < 0 || S < 0) return RLCS_ERR_INVALID_ARG;
    if (dtype != RLCS_F32 && dtype != RLCS_BF16) return RLCS_ERR_DTYPE;
    if (!std::isfinite(scale)) return RLCS_ERR_INVALID_ARG;
    if (N == 0 || G == 0 || Hq == 0 || D == 0) return RLCS_OK;
    // grid dimensions and row counts that the kernels index with 32 bits
    if (N > 65535 || G > 65535 || Hq > 65535 || Hkv < 1 || Hq % Hkv || N * G > INT32_MAX / Hq) return RLCS_ERR_INVALID_ARG;
    if (D > kMaxHeadDim || D % 8 || P > kMaxT || S > kMaxT) return RLCS_ERR_INVALID_ARG;
    if (!q || !o || (P && (!kp || !vp)) || (S && (!ks || !vs))) return RLCS_ERR_INVALID_ARG;
    for (const void* p : {q, kp, vp, ks, vs, static_cast<const void*>(o)})
        if (!aligned(p, 16)) return RLCS_ERR_INVALID_ARG;
    for (const void* p : {static_cast<const void*>(prefix_len), static_cast<const void*>(suffix_len), static_cast<const void*>(lse)})
        if (!aligned(p, 4)) return RLCS_ERR_INVALID_ARG;
    AttnArgs a{};
    if (layout) {
        a.at = *layout;
    } else {
        const int64_t t = Hkv * D;  // (at most 2^24; a group's suffixes may be more than 63 bits count)
        if (S > 0 && G > INT64_MAX / 8 / S / t) return RLCS_ERR_INVALID_ARG;
        a.at = rlcs_attn_layout{{G * Hq * D, Hq * D, D}, {P * t, t, D}, {P * t, t, D}, {G * S * t, S * t, t, D}, {G * S * t, S * t, t, D}};
    }
    const int64_t vec = 16 / int64_t(dtype_size(dtype));
    auto whole = [&](const int64_t* s, int n) {
        for (int i = 0; i < n; ++i)
            if (s[i] % vec) return false;
        return true;
    };
    if (!whole(a.at.q, 3) || !whole(a.at.kp, 3) || !whole(a.at.vp, 3) || !whole(a.at.ks, 4) || !whole(a.at.vs, 4))
        return RLCS_ERR_INVALID_ARG;
    if (!reachable({N, G, Hq}, a.at.q) || !reachable({N, P, Hkv}, a.at.kp) || !reachable({N, P, Hkv}, a.at.vp) ||
        !reachable({N, G, S, Hkv}, a.at.ks) || !reachable({N, G, S, Hkv}, a.at.vs))
        return RLCS_ERR_INVALID_ARG;
    if (ws_bytes < rlcs_workspace_size_attn(N, G, Hq, Hkv, D, P, S)) return RLCS_ERR_WORKSPACE;
    (void)ws;
    a.q = q; a.kp = kp; a.vp = vp; a.ks = ks; a.vs = vs;
    a.prefix_len = prefix_len; a.suffix_len = suffix_len;
    a.o = o; a.lse = lse;
    a.N = N; a.G = G; a.Hq = Hq; a.Hkv = Hkv; a.D = D; a.P = P; a.S = S;
    a.scale2 = scale * kLog2e;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    return dtype == RLCS_BF16 ? run_attn<bf16_t>(a, s) : run_attn<float>(a, s);
}

}  // extern "C"
