// Attention of single-token queries over a group's shared prefix and each sequence's own suffix.
//
// A tile of 16 * QT query rows that read the same keys is one workgroup's: for a prefix, rows of any
// sequence of the group, for a suffix, the query heads of one key head of one sequence. Its keys
// are dealt to the waves block by block; a wave keeps running maxima, sums and outputs of its
// own (no barrier), and the waves join at the end. Long key ranges are split over workgroups, whose
// parts a second kernel joins.
//
// Both products run on the matrix cores in the transposed form S^T = K Q^T, O^T = V^T P^T: a lane
// then holds scores of one query (lane % 16), so the maximum needs two shuffles, the rescaling none,
// and P^T leaves the first product in the layout the second wants, if V's keys are taken in the
// same order. Keys are read from memory straight into the operand's layout; bfloat16 values pass
// through LDS, whose transposing read turns rows of V into columns.
#pragma once

#include "rlcs.h"
#include "rlcs_softmax.h"

namespace rlcs {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

struct AttnArgs {
    const void *q, *kp, *vp, *ks, *vs;
    const int32_t *prefix_len, *suffix_len;
    void* o;
    float* lse;
    int64_t N, G, Hq, Hkv, D, P, S;
    rlcs_attn_layout at;
    float scale2;  // scale * log2(e): scores in base 2
};

// How a call is cut into workgroups: `prefix_parts` pieces of `prefix_chunk` keys of every prefix tile
// (`prefix_tiles` a key head), then the suffix's. With `whole` a suffix tile takes the prefix too. With
// one part in all (`part_acc` null) results go straight to the outputs.
struct AttnPlan {
    int64_t prefix_chunk, suffix_chunk;
    int32_t prefix_parts, suffix_parts, prefix_tiles, suffix_tiles;
    int32_t prefix_items, items;  // workgroups of the prefix, and all
    bool whole;
    float* part_acc;  // [part][row][D]: outputs relative to the part's own maximum
    float2* part_ml;  // [part][row]: maximum (base 2) and sum
};

__device__ __forceinline__ int64_t clamp_len(const int32_t* p, int64_t i, int64_t most) {
    if (!p) return most;
    const int64_t n = p[i];
    return n < 0 ? 0 : n > most ? most : n;
}

constexpr int kTileRows = 16;  // queries of a matrix product's columns

// Keys of one block, as operands: of bfloat16 32 keys, of float32 16. ND: the head's dimensions in
// sixteens.
template <typename DT, int ND>
struct KeyBlock;

template <int ND>
struct KeyBlock<bf16_t, ND> {
    static constexpr int kKeys = 32;
    static constexpr int kRow = 16 * ND + 16;  // elements of a row of V in LDS: 32 bytes more, so that
                                               // the eight rows of half a wave's read lie in different banks
    u32x4 k[ND];  // k[kt * ND / 2 + s]: key 16 kt + lane % 16, dimensions 32 s + 8 (lane / 16) ...
    u32x4 v[ND];  // rows of V, 16 bytes a lane

    __device__ __forceinline__ void load(const bf16_t* kb, const bf16_t* vb, int64_t sk, int64_t sv, int64_t j0, int64_t end,
                                         int D, int lane) {
        const int c = lane & 15, g = lane >> 4;
        const bool all = j0 + kKeys <= end;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            int64_t j = j0 + 16 * kt + c;
            if (!all) j = j < end ? j : end - 1;
            const bf16_t* p = kb + j * sk + 8 * g;
#pragma unroll
            for (int s = 0; s < ND / 2; ++s)
                k[kt * (ND / 2) + s] = 32 * s + 8 * g < D ? *reinterpret_cast<const u32x4*>(p + 32 * s) : u32x4{0, 0, 0, 0};
        }
        constexpr int kVecs = 2 * ND;  // 16-byte pieces of a row
#pragma unroll
        for (int i = 0; i < ND; ++i) {
            const int at = lane + 64 * i, piece = at % kVecs;
            const int64_t j = j0 + at / kVecs;
            v[i] = (all || j < end) && 8 * piece < D ? *reinterpret_cast<const u32x4*>(vb + j * sv + 8 * piece) : u32x4{0, 0, 0, 0};
        }
    }
    __device__ __forceinline__ void stage(bf16_t* lds, int lane) const {
        constexpr int kVecs = 2 * ND;
        wave_lds_sync();  // the block before has been read
#pragma unroll
        for (int i = 0; i < ND; ++i) {
            const int at = lane + 64 * i;
            *reinterpret_cast<u32x4*>(lds + (at / kVecs) * kRow + 8 * (at % kVecs)) = v[i];
        }
        wave_lds_sync();
    }
};

template <int ND>
struct KeyBlock<float, ND> {
    static constexpr int kKeys = 16;
    f32x4 k[ND];     // key lane % 16, dimensions 16 j + 4 (lane / 16) ...
    float v[ND][4];  // key 4 (lane / 16) + i, dimension 16 t + lane % 16

    __device__ __forceinline__ void load(const float* kb, const float* vb, int64_t sk, int64_t sv, int64_t j0, int64_t end, int D,
                                         int lane) {
        const int c = lane & 15, g = lane >> 4;
        const bool all = j0 + kKeys <= end;
        int64_t j = j0 + c;
        if (!all) j = j < end ? j : end - 1;
        const float* p = kb + j * sk + 4 * g;
#pragma unroll
        for (int t = 0; t < ND; ++t)
            k[t] = 16 * t + 4 * g < D ? *reinterpret_cast<const f32x4*>(p + 16 * t) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t jv = j0 + 4 * g + i;
            const bool in = all || jv < end;
            const float* pv = vb + (in ? jv : end - 1) * sv + c;
#pragma unroll
            for (int t = 0; t < ND; ++t) v[t][i] = in && 16 * t + c < D ? pv[16 * t] : 0.f;
        }
    }
};

// A wave's state: queries, running maxima, sums (of its lane's keys only) and outputs.
template <typename DT, int ND, int QT>
struct AttnWave {
    static constexpr int kKeys = KeyBlock<DT, ND>::kKeys;
    typedef typename std::conditional<sizeof(DT) == 2, u32x4, f32x4>::type QVec;
    static constexpr int kQVecs = sizeof(DT) == 2 ? ND / 2 : ND;
    QVec q[QT][kQVecs];
    f32x4 acc[QT][ND];  // query lane % 16, dimensions 16 t + 4 (lane / 16) ...
    float m[QT], l[QT];

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int x = 0; x < QT; ++x) {
            m[x] = kNegInf;
            l[x] = 0.f;
#pragma unroll
            for (int t = 0; t < ND; ++t) acc[x][t] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
    // Query row of this lane's column of tile x, or null past the last.
    __device__ __forceinline__ void load_query(int x, const DT* p, int D, int lane) {
        const int g = lane >> 4;
        constexpr int kVec = 16 / sizeof(DT);
#pragma unroll
        for (int s = 0; s < kQVecs; ++s) {
            const int d = 4 * kVec * s + kVec * g;
            q[x][s] = p && d < D ? *reinterpret_cast<const QVec*>(p + d) : QVec{0, 0, 0, 0};
        }
    }

    // Scores of a block, its softmax step and its part of the outputs.
    __device__ __forceinline__ void step(const KeyBlock<DT, ND>& b, bf16_t* lds, int64_t j0, int64_t end, float scale2, int lane) {
        const int c = lane & 15, g = lane >> 4;
        constexpr int KT = kKeys / 16;
        f32x4 s[QT][KT];
#pragma unroll
        for (int x = 0; x < QT; ++x)
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) s[x][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
        if constexpr (sizeof(DT) == 2) {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int d = 0; d < ND / 2; ++d)
#pragma unroll
                    for (int x = 0; x < QT; ++x)
                        s[x][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, b.k[kt * (ND / 2) + d]),
                                                                          __builtin_bit_cast(bf16x8, q[x][d]), s[x][kt], 0, 0, 0);
        } else {
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int x = 0; x < QT; ++x)
                        s[x][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(b.k[d][i], q[x][d][i], s[x][0], 0, 0, 0);
        }
        const bool all = j0 + kKeys <= end;
#pragma unroll
        for (int x = 0; x < QT; ++x) {
            float top = kNegInf;
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
                s[x][kt] *= scale2;
                if (!all) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (j0 + 16 * kt + 4 * g + i >= end) s[x][kt][i] = kNegInf;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) top = fmaxf(top, s[x][kt][i]);
            }
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float m1 = fmaxf(m[x], top);
            if (__any(m1 > m[x])) {
                const float keep = exp2_fast(m[x] - m1);
                l[x] *= keep;
#pragma unroll
                for (int t = 0; t < ND; ++t) acc[x][t] *= keep;
                m[x] = m1;
            }
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[x][kt][i] = exp2_fast(s[x][kt][i] - m[x]);
                    l[x] += s[x][kt][i];
                }
        }
        if constexpr (sizeof(DT) == 2) {
            bf16x8 p[QT];  // rounded to nearest for the product; the sums keep all bits
#pragma unroll
            for (int x = 0; x < QT; ++x)
#pragma unroll
                for (int i = 0; i < 8; ++i) p[x][i] = static_cast<__bf16>(s[x][i >> 2][i & 3]);
            // rows 4 g ... of each sixteen keys, columns 16 t ...
            const bf16_t* at = lds + (4 * g + (c >> 2)) * KeyBlock<DT, ND>::kRow + 4 * (c & 3);
#pragma unroll
            for (int t = 0; t < ND; ++t) {
                union {
                    s16x4 half[2];
                    bf16x8 all;
                } v;
                v.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at + 16 * t));
                v.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) s16x4*)(at + 16 * KeyBlock<DT, ND>::kRow + 16 * t));
#pragma unroll
                for (int x = 0; x < QT; ++x) acc[x][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v.all, p[x], acc[x][t], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int t = 0; t < ND; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int x = 0; x < QT; ++x)
                        acc[x][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(b.v[t][i], s[x][0][i], acc[x][t], 0, 0, 0);
        }
    }

    // Keys [from, end) of one array: blocks wave, wave + W, ... The next block's loads are under way
    // while one is worked on.
    template <int W>
    __device__ __forceinline__ void run(const DT* kb, const DT* vb, int64_t sk, int64_t sv, int64_t from, int64_t end, int D,
                                        float scale2, bf16_t* lds, int wave, int lane) {
        int64_t j = from + wave * kKeys;
        if (j >= end) return;
        KeyBlock<DT, ND> b;
        b.load(kb, vb, sk, sv, j, end, D, lane);
        for (;;) {
            const int64_t next = j + W * kKeys;
            KeyBlock<DT, ND> cur = b;
            if constexpr (sizeof(DT) == 2) cur.stage(lds, lane);
            if (next < end) b.load(kb, vb, sk, sv, next, end, D, lane);
            step(cur, lds, j, end, scale2, lane);
            if (next >= end) return;
            j = next;
        }
    }
};

template <typename DT, int ND, int W>
constexpr size_t attn_lds() {
    const size_t join = size_t(W) * kTileRows * (16 * ND + 4) * 4;
    const size_t v = sizeof(DT) == 2 ? size_t(W) * 32 * (16 * ND + 16) * 2 : 0;
    return join > v ? join : v;
}

template <typename DT, int ND, int QT, int W>
__global__ __launch_bounds__(W * kWave) void attn_kernel(AttnArgs a, AttnPlan plan, int first_item) {
    __shared__ __attribute__((aligned(16))) char s_mem[attn_lds<DT, ND, W>()];
    __shared__ float s_m[W][kTileRows], s_l[W][kTileRows];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c = lane & 15, g4 = lane >> 4;
    const int D = int(a.D), r = int(a.Hq / a.Hkv);
    bf16_t* lds = reinterpret_cast<bf16_t*>(s_mem) + wave * 32 * (16 * ND + 16);

    // what this workgroup takes
    int item = first_item + int(blockIdx.x);
    const bool prefix = item < plan.prefix_items;
    if (!prefix) item -= plan.prefix_items;
    const int tiles = prefix ? plan.prefix_tiles : plan.suffix_tiles;
    const int parts = prefix ? plan.prefix_parts : plan.suffix_parts;
    const int tile = item % tiles;
    item /= tiles;
    const int64_t hk = item % a.Hkv;
    item /= int(a.Hkv);
    const int part = item % parts;
    item /= parts;
    const int64_t n = prefix ? item : item / a.G, own = prefix ? 0 : item % a.G;
    const int64_t rows = prefix ? a.G * r : r;
    const int64_t row0 = int64_t(tile) * kTileRows * QT;

    const int64_t plen = clamp_len(a.prefix_len, n, a.P), slen = prefix ? 0 : clamp_len(a.suffix_len, n * a.G + own, a.S);
    const int64_t chunk = prefix ? plan.prefix_chunk : plan.suffix_chunk;
    const int64_t from = part * chunk;
    int64_t end = prefix ? plen : slen;
    if (end > from + chunk) end = from + chunk;
    const int slot = prefix ? part : (plan.whole ? 0 : plan.prefix_parts) + part;
    // (a part past the length: the joining kernel knows, and does not look at it)
    if (plan.part_acc && from >= end) return;

    auto row_of = [&](int64_t i, int64_t& g, int64_t& h) {
        g = prefix ? i / r : own;
        h = hk * r + (prefix ? i % r : i);
    };
    AttnWave<DT, ND, QT> w;
    w.clear();
#pragma unroll
    for (int x = 0; x < QT; ++x) {
        const int64_t i = row0 + x * kTileRows + c;
        const DT* p = nullptr;
        if (i < rows) {
            int64_t g, h;
            row_of(i, g, h);
            p = reinterpret_cast<const DT*>(a.q) + n * a.at.q[0] + g * a.at.q[1] + h * a.at.q[2];
        }
        w.load_query(x, p, D, lane);
    }
    const DT* kp = reinterpret_cast<const DT*>(a.kp) + n * a.at.kp[0] + hk * a.at.kp[2];
    const DT* vp = reinterpret_cast<const DT*>(a.vp) + n * a.at.vp[0] + hk * a.at.vp[2];
    const DT* ks = reinterpret_cast<const DT*>(a.ks) + n * a.at.ks[0] + own * a.at.ks[1] + hk * a.at.ks[3];
    const DT* vs = reinterpret_cast<const DT*>(a.vs) + n * a.at.vs[0] + own * a.at.vs[1] + hk * a.at.vs[3];
    if (prefix) {
        w.template run<W>(kp, vp, a.at.kp[1], a.at.vp[1], from, end, D, a.scale2, lds, wave, lane);
    } else {
        if (plan.whole) w.template run<W>(kp, vp, a.at.kp[1], a.at.vp[1], 0, plen, D, a.scale2, lds, wave, lane);
        w.template run<W>(ks, vs, a.at.ks[2], a.at.vs[2], from, end, D, a.scale2, lds, wave, lane);
    }

    // the waves join, tile by tile
    float* join = reinterpret_cast<float*>(s_mem);
    constexpr int kJoinRow = 16 * ND + 4;
#pragma unroll
    for (int x = 0; x < QT; ++x) {
        float l = w.l[x];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        __syncthreads();
        if (g4 == 0) {
            s_m[wave][c] = w.m[x];
            s_l[wave][c] = l;
        }
#pragma unroll
        for (int t = 0; t < ND; ++t)
            *reinterpret_cast<f32x4*>(join + (wave * kTileRows + c) * kJoinRow + 16 * t + 4 * g4) = w.acc[x][t];
        __syncthreads();
        for (int at = tid; at < kTileRows * 4 * ND; at += W * kWave) {
            const int i = at / (4 * ND), d = 4 * (at % (4 * ND));
            const int64_t row = row0 + x * kTileRows + i;
            if (row >= rows || d >= D) continue;
            float m = kNegInf;
#pragma unroll
            for (int v = 0; v < W; ++v) m = fmaxf(m, s_m[v][i]);
            float z = 0.f;
            f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int v = 0; v < W; ++v) {
                const float keep = s_m[v][i] == kNegInf ? 0.f : exp2_fast(s_m[v][i] - m);
                z = fmaf(keep, s_l[v][i], z);
                o += keep * *reinterpret_cast<const f32x4*>(join + (v * kTileRows + i) * kJoinRow + d);
            }
            int64_t g, h;
            row_of(row, g, h);
            const int64_t out = (n * a.G + g) * a.Hq + h;
            if (plan.part_acc) {
                const int64_t at_part = int64_t(slot) * a.N * a.G * a.Hq + out;
                *reinterpret_cast<f32x4*>(plan.part_acc + at_part * D + d) = o;
                if (d == 0) plan.part_ml[at_part] = float2{m, z};
            } else {
                o = z > 0.f ? o / z : f32x4{0.f, 0.f, 0.f, 0.f};
                DT* po = reinterpret_cast<DT*>(a.o) + out * D + d;
#pragma unroll
                for (int e = 0; e < 4; ++e) po[e] = narrow(o[e], DT{});
                if (d == 0 && a.lse) a.lse[out] = z > 0.f ? kLn2 * (m + log2_fast(z)) : kNegInf;
            }
        }
    }
}

// Joins the parts of every row: 4 dimensions a lane.
template <typename DT>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a, AttnPlan plan) {
    const int lanes = int(a.D / 4);  // of a row
    const int64_t rows = a.N * a.G * a.Hq;
    const int64_t out = int64_t(blockIdx.x) * (256 / lanes) + threadIdx.x / lanes;
    const int d = 4 * (int(threadIdx.x) % lanes);
    if (int(threadIdx.x) >= 256 / lanes * lanes || out >= rows) return;
    const int64_t seq = out / a.Hq;
    const int64_t plen = plan.whole ? 0 : clamp_len(a.prefix_len, seq / a.G, a.P), slen = clamp_len(a.suffix_len, seq, a.S);
    // parts that hold keys
    const int np = plen > 0 ? int((plen + plan.prefix_chunk - 1) / plan.prefix_chunk) : 0;
    const int ns = slen > 0 ? int((slen + plan.suffix_chunk - 1) / plan.suffix_chunk) : 0;
    float m = kNegInf;
    for (int i = 0; i < np + ns; ++i) m = fmaxf(m, plan.part_ml[(i < np ? i : plan.prefix_parts + i - np) * rows + out].x);
    float z = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < np + ns; ++i) {
        const int64_t at = (i < np ? i : plan.prefix_parts + i - np) * rows + out;
        const float2 ml = plan.part_ml[at];
        const float keep = exp2_fast(ml.x - m);
        z = fmaf(keep, ml.y, z);
        o += keep * *reinterpret_cast<const f32x4*>(plan.part_acc + at * a.D + d);
    }
    o = z > 0.f ? o / z : f32x4{0.f, 0.f, 0.f, 0.f};
    DT* po = reinterpret_cast<DT*>(a.o) + out * a.D + d;
#pragma unroll
    for (int e = 0; e < 4; ++e) po[e] = narrow(o[e], DT{});
    if (d == 0 && a.lse) a.lse[out] = z > 0.f ? kLn2 * (m + log2_fast(z)) : kNegInf;
}

}  // namespace rlcs
