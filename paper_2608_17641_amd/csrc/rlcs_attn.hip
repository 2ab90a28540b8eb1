// Entry point of attention over a shared prefix.
#include "rlcs_attn.h"
#include "rlcs_dispatch.h"

#include <cmath>

using namespace rlcs;
using namespace rlcs::host;

namespace {

constexpr int64_t kMaxHeadDim = 256;
constexpr int64_t kMaxTokenStride = int64_t(1) << 24;

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

// Keys of a part: no fewer than kMinChunk (a part of r rows costs r * D * 8 bytes written and read
// again), and as many parts as give the workgroups, or waves, wanted.
constexpr int64_t kMinChunk = 256;
constexpr int64_t kWantPrefix = 512, kWantSuffix = 1536, kWantSolo = 4096;
// From this many pieces of kMinChunk keys (two for each SIMD) every wave takes items of its own, which
// needs no join in the workgroup; with fewer the waves of a workgroup split an item's keys.
constexpr int64_t kSoloFrom = 2048;
// Calls of at most this many keys, and of at most kWholeItems workgroups so, run as one kernel in which
// each sequence takes its prefix itself: no second reading of partial outputs (1 x 64, 32 heads on 8,
// 400 + 100 keys 17 us against 31 in three kernels; with 8 x 64 sequences 105 against 85).
constexpr int64_t kWholeKeys = 512, kWholeItems = 2048;

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

PrefixRows prefix_rows(int64_t rows, int64_t D, bool bf16) {
    if (rows <= kTileRows) return kPrefixOne;
    if (rows <= 64 || D > 128) return kPrefixShared64;
    return rows <= 128 || !bf16 ? kPrefixShared128 : kPrefixShared256;
}
int64_t rows_of(PrefixRows p) {  // of a workgroup
    return p == kPrefixOne ? kTileRows : p == kPrefixShared64 ? 64 : p == kPrefixShared128 ? 128 : 256;
}

bool make_plan(AttnPlan& p, int64_t N, int64_t G, int64_t Hq, int64_t Hkv, int64_t D, int64_t P, int64_t S, bool bf16) {
    const int64_t r = Hq / Hkv;
    const PrefixRows pr = prefix_rows(G * r, D, bf16);
    p = AttnPlan{};
    p.suffix_tiles = int32_t(ceil_div(r, kTileRows));
    p.prefix_tiles = int32_t(ceil_div(G * r, rows_of(pr)));
    const int64_t suffix_base = N * G * Hkv * p.suffix_tiles, prefix_base = N * Hkv * p.prefix_tiles;
    p.whole = P == 0 || (P + S <= kWholeKeys && suffix_base <= kWholeItems);
    p.solo = !(p.whole && P > 0) &&
             suffix_base * ceil_div(S, kMinChunk) + (pr == kPrefixOne ? prefix_base * ceil_div(P, kMinChunk) : 0) >= kSoloFrom;
    auto split = [](int64_t keys, int64_t base, int64_t items, int32_t& chunk, int32_t& parts) {
        int64_t want = ceil_div(items, base), most = ceil_div(keys, kMinChunk);
        if (want > most) want = most;
        if (want < 1) want = 1;
        chunk = int32_t(keys > 0 ? ceil_div(ceil_div(keys, want), 64) * 64 : 1);
        parts = int32_t(keys > 0 ? ceil_div(keys, chunk) : 1);
    };
    p.suffix_chunk = 1;
    p.prefix_chunk = 1;
    if (p.whole && P > 0) {
        p.suffix_parts = 1;
        p.suffix_chunk = int32_t(S > 0 ? S : 1);
    } else if (S > 0 || P == 0) {
        split(S, suffix_base, p.solo ? kWantSolo : kWantSuffix, p.suffix_chunk, p.suffix_parts);
    }
    const int64_t suffix_items = suffix_base * p.suffix_parts;
    int64_t prefix_items = 0;
    const bool prefix_solo = p.solo && pr == kPrefixOne;
    if (!p.whole) {
        split(P, prefix_base, prefix_solo ? kWantSolo : pr == kPrefixShared256 ? kWantPrefix / 2 : kWantPrefix, p.prefix_chunk, p.prefix_parts);
        prefix_items = prefix_base * p.prefix_parts;
    }
    const int64_t prefix_groups = ceil_div(prefix_items, kGroup * (prefix_solo ? kAttnWaves : 1));
    const int64_t groups = prefix_groups + ceil_div(suffix_items, kGroup * (p.solo ? kAttnWaves : 1));
    if (prefix_items + suffix_items > INT32_MAX - 4 * kGroup * kAttnWaves || groups > (INT32_MAX >> kGridBits << kGridBits) / kGroup) return false;
    p.prefix_items = int32_t(prefix_items);
    p.suffix_items = int32_t(suffix_items);
    p.prefix_groups = int32_t(prefix_groups);
    p.groups = int32_t(groups);
    return true;
}

size_t part_bytes(const AttnPlan& p, int64_t rows, int64_t D) {
    const int64_t parts = p.prefix_parts + p.suffix_parts;
    return parts > 1 ? size_t(parts * rows) * size_t(4 * D + 8) : 0;
}

// The workgroups of the prefix alone, or of the suffix alone, of a plan that has both.
AttnPlan only(AttnPlan p, bool prefix) {
    if (prefix) {
        p.groups = p.prefix_groups;
    } else {
        p.groups -= p.prefix_groups;
        p.prefix_groups = 0;
    }
    return p;
}

template <typename DT, int ND, PrefixRows PR, bool SOLO>
void launch_attn(const AttnArgs& a, const AttnPlan& p, hipStream_t s) {
    const dim3 grid = row_grid(int64_t(p.groups) * kGroup), block(kAttnWaves * kWave);
    if (a.D == 16 * ND) hipLaunchKernelGGL((attn_kernel<DT, ND, PR, SOLO, true>), grid, block, 0, s, a, p);
    else hipLaunchKernelGGL((attn_kernel<DT, ND, PR, SOLO, false>), grid, block, 0, s, a, p);
}
template <typename DT, int ND, PrefixRows PR>
void launch_attn(const AttnArgs& a, const AttnPlan& p, hipStream_t s) {
    if (p.groups == 0) return;
    if (p.solo) launch_attn<DT, ND, PR, true>(a, p, s);
    else launch_attn<DT, ND, PR, false>(a, p, s);
}

template <typename DT, int ND, int QT, int W>
void launch_prefix(const AttnArgs& a, const AttnPlan& p, hipStream_t s) {
    const dim3 grid = row_grid(int64_t(p.groups) * kGroup), block(W * kWave);
    if (a.D == 16 * ND) hipLaunchKernelGGL((attn_prefix_kernel<DT, ND, QT, W, true>), grid, block, 0, s, a, p);
    else hipLaunchKernelGGL((attn_prefix_kernel<DT, ND, QT, W, false>), grid, block, 0, s, a, p);
}

template <typename DT, int ND>
rlcs_status run_attn(const AttnArgs& a, const AttnPlan& p, hipStream_t s) {
    const PrefixRows pr = p.prefix_items ? prefix_rows(a.G * (a.Hq / a.Hkv), a.D, sizeof(DT) == 2) : kPrefixOne;
    if (pr == kPrefixOne) launch_attn<DT, ND, kPrefixOne>(a, p, s);
    if (pr == kPrefixShared64) launch_attn<DT, ND, kPrefixShared64>(a, p, s);
    if constexpr (ND <= 8) {
        if (pr == kPrefixShared128 || pr == kPrefixShared256) {
            if constexpr (sizeof(DT) == 4) {
                launch_prefix<DT, ND, 1, 8>(a, only(p, true), s);
            } else {
                if (pr == kPrefixShared128) launch_prefix<DT, ND, 2, 4>(a, only(p, true), s);
                else launch_prefix<DT, ND, 2, 8>(a, only(p, true), s);
            }
            launch_attn<DT, ND, kPrefixOne>(a, only(p, false), s);
        }
    }
    if (p.part_acc)
        hipLaunchKernelGGL((attn_join_kernel<DT>), row_grid(int64_t(a.N) * a.G * a.Hq), dim3(256), 0, s, a, p);
    return hipGetLastError() == hipSuccess ? RLCS_OK : RLCS_ERR_LAUNCH;
}

template <typename DT>
rlcs_status run_attn(const AttnArgs& a, const AttnPlan& p, hipStream_t s) {
    return a.D <= 64 ? run_attn<DT, 4>(a, p, s) : a.D <= 128 ? run_attn<DT, 8>(a, p, s) : run_attn<DT, 16>(a, p, s);
}

bool sizes_fit(int64_t N, int64_t G, int64_t Hq, int64_t Hkv, int64_t D, int64_t P, int64_t S) {
    if (N < 1 || G < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv || P < 0 || S < 0) return false;
    return N <= INT32_MAX && G <= INT32_MAX && Hq <= INT32_MAX && N <= INT32_MAX / G && N * G <= INT32_MAX / Hq && D >= 8 &&
           D <= kMaxHeadDim && D % 8 == 0 && P <= kMaxT && S <= kMaxT;
}

}  // namespace

extern "C" {

size_t rlcs_workspace_size_attn(int64_t N, int64_t G, int64_t Hq, int64_t Hkv, int64_t D, int64_t P, int64_t S) {
    if (!sizes_fit(N, G, Hq, Hkv, D, P, S)) return 0;
    AttnPlan b, f;
    if (!make_plan(b, N, G, Hq, Hkv, D, P, S, true) || !make_plan(f, N, G, Hq, Hkv, D, P, S, false)) return 0;
    const size_t x = part_bytes(b, N * G * Hq, D), y = part_bytes(f, N * G * Hq, D);
    return x > y ? x : y;
}

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
    if (!sizes_fit(N, G, Hq, Hkv, D, P, S)) return RLCS_ERR_INVALID_ARG;
    if (!q || !o || (P && (!kp || !vp)) || (S && (!ks || !vs))) return RLCS_ERR_INVALID_ARG;
    for (const void* p : {q, kp, vp, ks, vs, static_cast<const void*>(o)})
        if (!aligned(p, 16)) return RLCS_ERR_INVALID_ARG;
    for (const void* p : {static_cast<const void*>(prefix_len), static_cast<const void*>(suffix_len), static_cast<const void*>(lse)})
        if (!aligned(p, 4)) return RLCS_ERR_INVALID_ARG;
    AttnArgs a{};
    if (layout) {
        a.at = *layout;
    } else {
        const int64_t t = Hkv * D;  // (refused from 2^24; a group's suffixes may be more than 63 bits count)
        if (S > 0 && G > INT64_MAX / 8 / S / t) return RLCS_ERR_INVALID_ARG;
        a.at = rlcs_attn_layout{{G * Hq * D, Hq * D, D}, {P * t, t, D}, {P * t, t, D}, {G * S * t, S * t, t, D}, {G * S * t, S * t, t, D}};
    }
    const int64_t vec = 16 / int64_t(dtype_size(dtype));
    auto whole = [&](const int64_t* s, int n) {
        for (int i = 0; i < n; ++i)
            if (s[i] % vec) return false;
        return true;
    };
    // a block's rows lie within 31 bits of bytes of each other
    if (a.at.kp[1] >= kMaxTokenStride || a.at.vp[1] >= kMaxTokenStride || a.at.ks[2] >= kMaxTokenStride || a.at.vs[2] >= kMaxTokenStride)
        return RLCS_ERR_INVALID_ARG;
    if (!whole(a.at.q, 3) || !whole(a.at.kp, 3) || !whole(a.at.vp, 3) || !whole(a.at.ks, 4) || !whole(a.at.vs, 4))
        return RLCS_ERR_INVALID_ARG;
    if (!reachable({N, G, Hq}, a.at.q) || !reachable({N, P, Hkv}, a.at.kp) || !reachable({N, P, Hkv}, a.at.vp) ||
        !reachable({N, G, S, Hkv}, a.at.ks) || !reachable({N, G, S, Hkv}, a.at.vs))
        return RLCS_ERR_INVALID_ARG;
    const bool bf16 = dtype == RLCS_BF16;
    AttnPlan p;
    if (!make_plan(p, N, G, Hq, Hkv, D, P, S, bf16)) return RLCS_ERR_INVALID_ARG;
    if (const size_t need = part_bytes(p, N * G * Hq, D)) {
        if (!ws || ws_bytes < need) return RLCS_ERR_WORKSPACE;
        if (!aligned(ws, 16)) return RLCS_ERR_INVALID_ARG;
        const int64_t slots = int64_t(p.prefix_parts + p.suffix_parts) * N * G * Hq;
        p.part_acc = static_cast<float*>(ws);
        p.part_ml = reinterpret_cast<float2*>(p.part_acc + slots * D);
    }
    a.q = q; a.kp = kp; a.vp = vp; a.ks = ks; a.vs = vs;
    a.prefix_len = prefix_len; a.suffix_len = suffix_len;
    a.o = o; a.lse = lse;
    a.N = int32_t(N); a.G = int32_t(G); a.Hq = int32_t(Hq); a.Hkv = int32_t(Hkv); a.D = int32_t(D);
    a.P = int32_t(P); a.S = int32_t(S);
    a.scale2 = scale * kLog2e;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    return bf16 ? run_attn<bf16_t>(a, p, s) : run_attn<float>(a, p, s);
}

}  // extern "C"
