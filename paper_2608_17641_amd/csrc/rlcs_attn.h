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
    int32_t N, G, Hq, Hkv, D, P, S;  // (N * G * Hq below 2^31, P and S up to 2^30)
    rlcs_attn_layout at;
    float scale2;  // scale * log2(e): scores in base 2
};

// How a call is cut into items, each a workgroup's, or with `solo` a wave's (but a prefix that waves
// share): `prefix_parts` pieces of `prefix_chunk` keys of every prefix tile
// (`prefix_tiles` a key head), then the suffix's. With `whole` a suffix tile takes the prefix too. With
// one part in all (`part_acc` null) results go straight to the outputs.
struct AttnPlan {
    int32_t prefix_chunk, suffix_chunk, prefix_parts, suffix_parts, prefix_tiles, suffix_tiles;
    int32_t prefix_items, suffix_items;
    int32_t prefix_groups, groups;  // workgroups of the prefix, and all, in groups of kGroup, as they are dealt
    bool whole, solo;
    float* part_acc;  // [part][row][D]: outputs relative to the part's own maximum
    float2* part_ml;  // [part][row]: maximum (base 2) and sum
};

__device__ __forceinline__ int clamp_len(const int32_t* p, int64_t i, int most) {
    if (!p) return most;
    const int n = p[i];
    return n < 0 ? 0 : n > most ? most : n;
}

// The prefix's workgroups, which compute, and the suffix's, which wait for memory, are dealt in turn,
// kGroup of each kind at a time in proportion to their numbers, so that a CU has both.
constexpr int kGroup = 16;

constexpr int kAttnWaves = 4;

constexpr int kTileRows = 16;  // queries of a matrix product's columns

// One array of keys and values as a wave walks it: byte offsets of its lane's pieces of a block from
// the block's first row (below 2^31: token strides are below 2^24 elements), and the rows' strides. A
// piece past the head's dimensions reads the head's last one instead: its query is 0, its output
// column is not stored. Rows past the end read the last row: their weights are 0, and it holds
// ordinary numbers. So no load depends on a lane's condition.
template <typename DT, int ND, bool EXACT>
struct KeyBlock {
    static constexpr bool kWide = sizeof(DT) == 4;
    static constexpr int kKeys = kWide ? 16 : 32;
    static constexpr int kRow = 16 * ND + 16;  // bfloat16: elements of a row of V in LDS, 32 bytes more than it
                                               // has, so that the rows of half a wave's read lie in different banks
    static constexpr int kVecs = 2 * ND;       // its 16-byte pieces
    static constexpr int kKRows = kKeys / 16, kVRows = kWide ? 4 : ND;
    // bfloat16: k[kt * ND / 2 + s] is key 16 kt + lane % 16, dimensions 32 s + 8 (lane / 16) ..., v rows
    // of V, 16 bytes a lane. float32: k[t] is key lane % 16, dimensions 16 t + 4 (lane / 16) ..., v[t][i]
    // is key 4 (lane / 16) + i, dimension 16 t + lane % 16.
    u32x4 k[ND], v[ND];
    uint32_t at_k[kKRows], at_v[kVRows];

    // `rows` of the block that exist
    __device__ __forceinline__ void aim(int rows, int64_t sk, int64_t sv, int D, int lane) {
        const int c = lane & 15, g = lane >> 4;
        auto row = [&](int j) { return uint32_t(j < rows ? j : rows - 1); };
#pragma unroll
        for (int kt = 0; kt < kKRows; ++kt) at_k[kt] = (row(16 * kt + c) * uint32_t(sk)) * uint32_t(sizeof(DT)) + 16u * g;
#pragma unroll
        for (int i = 0; i < kVRows; ++i) {
            if constexpr (kWide) {
                at_v[i] = (row(4 * g + i) * uint32_t(sv) + c) * 4u;
            } else {
                const int at = lane + 64 * i, piece = at % kVecs;
                at_v[i] = (row(at / kVecs) * uint32_t(sv) + 8u * (EXACT || 8 * piece < D ? piece : D / 8 - 1)) * 2u;
            }
        }
    }
    __device__ __forceinline__ void load_k(const char* base, int D, int lane) {
        constexpr int kSteps = ND / kKRows;
#pragma unroll
        for (int kt = 0; kt < kKRows; ++kt)
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                uint32_t at = at_k[kt] + 64u * s;
                if constexpr (!EXACT) {  // (64 bytes a step, 16 a lane)
                    const uint32_t d = 64u * s + 16u * (lane >> 4), last = uint32_t(D) * sizeof(DT) - 16u;
                    if (d > last) at -= d - last;
                }
                k[kt * kSteps + s] = *reinterpret_cast<const u32x4*>(base + at);
            }
    }
    __device__ __forceinline__ void load_v(const char* base, int D, int lane) {
        if constexpr (kWide) {
#pragma unroll
            for (int t = 0; t < ND; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t at = at_v[i] + 64u * t;
                    if constexpr (!EXACT) {
                        const int d = 16 * t + (lane & 15);
                        if (d >= D) at -= 4u * uint32_t(d - D + 1);
                    }
                    v[t][i] = *reinterpret_cast<const uint32_t*>(base + at);
                }
        } else {
#pragma unroll
            for (int i = 0; i < ND; ++i) v[i] = *reinterpret_cast<const u32x4*>(base + at_v[i]);
        }
    }
    __device__ __forceinline__ void stage(bf16_t* lds, int lane) const {
        wave_lds_sync();  // the block before has been read
#pragma unroll
        for (int i = 0; i < ND; ++i) {
            const int at = lane + 64 * i;
            *reinterpret_cast<u32x4*>(lds + (at / kVecs) * kRow + 8 * (at % kVecs)) = v[i];
        }
        wave_lds_sync();
    }
};

// The largest over the four lanes that share lane % 16.
__device__ __forceinline__ float max_of_four(float x) {
    typedef unsigned u32x2v __attribute__((ext_vector_type(2)));
    u32x2v p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
    p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}

// One softmax step of a query tile: scores of 16 * KT keys become their weights, in place, and the
// running maximum, sum and outputs are brought to the new maximum.
template <int KT, int ND>
__device__ __forceinline__ void softmax_step(f32x4 (&s)[KT], float scale, float& m, float& l, f32x4 (&acc)[ND]) {
    float top = kNegInf;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[kt][i]);
    const float m1 = fmaxf(m, max_of_four(top) * scale);
    if (__any(m1 > m)) {
        const float keep = exp2_fast(m - m1);
        l *= keep;
#pragma unroll
        for (int t = 0; t < ND; ++t) acc[t] *= keep;
        m = m1;
    }
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s[kt][i] = exp2_fast(fmaf(s[kt][i], scale, -m));
            l += s[kt][i];
        }
}

// Weights of 32 keys (two tiles of scores) as an operand, rounded to bfloat16, to nearest, for the product alone:
// their sum keeps all bits.
__device__ __forceinline__ bf16x8 weights_operand(f32x4 a, f32x4 b) {
    bf16x8 p;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        p[i] = static_cast<__bf16>(a[i]);
        p[4 + i] = static_cast<__bf16>(b[i]);
    }
    return p;
}

// Values of 32 keys and 16 dimensions in LDS as an operand, keys in the order that scores come in:
// `at` is the lane's place, row 4 (lane / 16) + lane % 16 / 4 and column 4 (lane % 4) of the block.
__device__ __forceinline__ bf16x8 values_operand(const bf16_t* at, int row) {
    union {
        s16x4 half[2];
        bf16x8 all;
    } v;
    v.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at));
    v.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(at + 16 * row));
    return v.all;
}

// A wave's state: queries, running maxima (base 2), sums (of its lane's keys only) and outputs.
template <typename DT, int ND, int QT, bool EXACT>
struct AttnWave {
    typedef KeyBlock<DT, ND, EXACT> Block;
    static constexpr bool kWide = sizeof(DT) == 4;
    static constexpr int kKeys = Block::kKeys;
    static constexpr int kQVecs = kWide ? ND : ND / 2;
    u32x4 q[QT][kQVecs];
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
    // Query row of this lane's column of tile x, or null past the last; `sign` flips its elements' signs.
    __device__ __forceinline__ void load_query(int x, const DT* p, int D, uint32_t sign, int lane) {
        const int g = lane >> 4;
        constexpr int kVec = 16 / sizeof(DT);
#pragma unroll
        for (int s = 0; s < kQVecs; ++s) {
            const int d = 4 * kVec * s + kVec * g;
            q[x][s] = p && d < D ? *reinterpret_cast<const u32x4*>(p + d) ^ sign : u32x4{0, 0, 0, 0};
        }
    }

    // Keys [from, end) of one array: blocks wave, wave + W, ... A block's values are on their way while
    // the scores of the one before are worked out, its keys while those weigh their values. `scale` >= 0.
    template <int W>
    __device__ __forceinline__ void run(const DT* keys, const DT* values, int64_t sk, int64_t sv, int from, int end, int D,
                                        float scale, bf16_t* lds, int wave, int lane) {
        const int c = lane & 15, g = lane >> 4;
        constexpr int KT = kKeys / 16;
        int j = from + wave * kKeys;
        if (j >= end) return;
        Block b;
        const char* kb = reinterpret_cast<const char*>(keys + j * sk);
        const char* vb = reinterpret_cast<const char*>(values + j * sv);
        const int64_t hop_k = W * kKeys * sk * int64_t(sizeof(DT)), hop_v = W * kKeys * sv * int64_t(sizeof(DT));
        b.aim(end - j < kKeys ? int(end - j) : kKeys, sk, sv, D, lane);
        b.load_k(kb, D, lane);
        b.load_v(vb, D, lane);
        for (;;) {
            const int rows = end - j < kKeys ? int(end - j) : kKeys;
            j += W * kKeys;
            const bool more = j < end;
            kb += hop_k;
            vb += hop_v;
            if (end - j < kKeys && more) b.aim(int(end - j), sk, sv, D, lane);
            u32x4 now[kWide ? ND : 1];
            if constexpr (kWide) {
#pragma unroll
                for (int t = 0; t < ND; ++t) now[t] = b.v[t];
            } else {
                b.stage(lds, lane);
            }
            if (more) b.load_v(vb, D, lane);

            f32x4 s[QT][KT];
#pragma unroll
            for (int x = 0; x < QT; ++x)
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) s[x][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
            if constexpr (!kWide) {
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
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
                            s[x][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(b.k[d][i]), __uint_as_float(q[x][d][i]),
                                                                          s[x][0], 0, 0, 0);
            }
            if (more) b.load_k(kb, D, lane);

            if (rows < kKeys) {
#pragma unroll
                for (int x = 0; x < QT; ++x)
#pragma unroll
                    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (16 * kt + 4 * g + i >= rows) s[x][kt][i] = kNegInf;
            }
#pragma unroll
            for (int x = 0; x < QT; ++x) softmax_step<KT, ND>(s[x], scale, m[x], l[x], acc[x]);
            if constexpr (!kWide) {
                bf16x8 p[QT];
#pragma unroll
                for (int x = 0; x < QT; ++x) p[x] = weights_operand(s[x][0], s[x][1]);
                const bf16_t* at = lds + (4 * g + (c >> 2)) * Block::kRow + 4 * (c & 3);
#pragma unroll
                for (int t = 0; t < ND; ++t) {
                    const bf16x8 v = values_operand(at + 16 * t, Block::kRow);
#pragma unroll
                    for (int x = 0; x < QT; ++x) acc[x][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[x], acc[x][t], 0, 0, 0);
                }
            } else {
#pragma unroll
                for (int t = 0; t < ND; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int x = 0; x < QT; ++x)
                            acc[x][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(now[t][i]), s[x][0][i], acc[x][t], 0, 0, 0);
            }
            if (!more) return;
        }
    }
};

// Keys [from, end) of one array for a workgroup whose waves have queries of their own: all of
// its lanes bring blocks of keys and values to LDS, every wave reads them from there. While one
// block is worked on, the next is in the other half of LDS and the one after it on its way.
template <typename DT, int ND, int QT, int W, bool EXACT>
struct SharedKeys {
    static constexpr bool kWide = sizeof(DT) == 4;
    static constexpr int kKeys = (ND > 8 ? 32 : 64) / (kWide ? 2 : 1);
    static constexpr int kVecs = ND * int(sizeof(DT));  // 16-byte pieces of a row
    static constexpr int kVec = 16 / int(sizeof(DT));
    // elements of a row in LDS: the sixteen rows of a key operand's read, and the eight of half a wave's
    // of bfloat16 values, or the four of a wave's of float32 ones, in different banks
    static constexpr int kKRow = 16 * ND + kVec;
    static constexpr int kVRow = 16 * ND + (kWide ? 4 : 16);
    static constexpr int kPieces = kKeys * kVecs / (W * kWave);
    static constexpr int kHalf = kKeys * (kKRow + kVRow);  // elements
    static constexpr size_t kLds = size_t(2 * kHalf) * sizeof(DT);

    static __device__ __forceinline__ void run(AttnWave<DT, ND, QT, EXACT>& w, const DT* keys, const DT* values, int64_t sk, int64_t sv,
                                               int from, int end, int D, float scale, DT* lds, int tid) {
        const int lane = tid & 63, c = lane & 15, g = lane >> 4;
        constexpr int KT = kKeys / 16;
        u32x4 k[kPieces], v[kPieces];
        uint32_t at_k[kPieces], at_v[kPieces];
        auto aim = [&](int rows) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int at = tid + W * kWave * i, piece = at % kVecs;
                const uint32_t row = at / kVecs < rows ? at / kVecs : rows - 1;
                const uint32_t d = uint32_t(kVec) * (EXACT || kVec * piece < D ? piece : D / kVec - 1);
                at_k[i] = (row * uint32_t(sk) + d) * uint32_t(sizeof(DT));
                at_v[i] = (row * uint32_t(sv) + d) * uint32_t(sizeof(DT));
            }
        };
        auto load = [&](int j) {
            if (end - j < kKeys) aim(int(end - j));
            const char* kb = reinterpret_cast<const char*>(keys + j * sk);
            const char* vb = reinterpret_cast<const char*>(values + j * sv);
#pragma unroll
            for (int i = 0; i < kPieces; ++i) k[i] = *reinterpret_cast<const u32x4*>(kb + at_k[i]);
#pragma unroll
            for (int i = 0; i < kPieces; ++i) v[i] = *reinterpret_cast<const u32x4*>(vb + at_v[i]);
        };
        auto put = [&](DT* half) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int at = tid + W * kWave * i;
                *reinterpret_cast<u32x4*>(half + (at / kVecs) * kKRow + kVec * (at % kVecs)) = k[i];
                *reinterpret_cast<u32x4*>(half + kKeys * kKRow + (at / kVecs) * kVRow + kVec * (at % kVecs)) = v[i];
            }
        };
        if (from >= end) return;
        aim(kKeys);
        load(from);
        put(lds);
        if (from + kKeys < end) load(from + kKeys);
        int turn = 0;
        for (int j = from; j < end; j += kKeys) {
            const int rows = end - j < kKeys ? int(end - j) : kKeys;
            const DT* lk = lds + turn * kHalf;
            const DT* lv = lk + kKeys * kKRow;
            turn ^= 1;
            __syncthreads();  // this block is there, and the one before has been read
            if (j + kKeys < end) put(lds + turn * kHalf);
            if (j + 2 * kKeys < end) load(j + 2 * kKeys);
            f32x4 s[QT][KT];
#pragma unroll
            for (int x = 0; x < QT; ++x)
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) s[x][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
            if constexpr (kWide) {
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                    for (int t = 0; t < ND; ++t) {
                        const f32x4 k4 = *reinterpret_cast<const f32x4*>(lk + (16 * kt + c) * kKRow + 16 * t + 4 * g);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int x = 0; x < QT; ++x)
                                s[x][kt] = __builtin_amdgcn_mfma_f32_16x16x4f32(k4[i], __uint_as_float(w.q[x][t][i]), s[x][kt], 0, 0, 0);
                    }
            } else {
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                    for (int d = 0; d < ND / 2; ++d) {
                        const bf16x8 k8 = *reinterpret_cast<const bf16x8*>(lk + (16 * kt + c) * kKRow + 32 * d + 8 * g);
#pragma unroll
                        for (int x = 0; x < QT; ++x)
                            s[x][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k8, __builtin_bit_cast(bf16x8, w.q[x][d]), s[x][kt], 0, 0, 0);
                    }
            }
            if (rows < kKeys) {
#pragma unroll
                for (int x = 0; x < QT; ++x)
#pragma unroll
                    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (16 * kt + 4 * g + i >= rows) s[x][kt][i] = kNegInf;
            }
#pragma unroll
            for (int x = 0; x < QT; ++x) softmax_step<KT, ND>(s[x], scale, w.m[x], w.l[x], w.acc[x]);
            if constexpr (kWide) {
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int t = 0; t < ND; ++t) {
                            const float v1 = lv[(16 * kt + 4 * g + i) * kVRow + 16 * t + c];
#pragma unroll
                            for (int x = 0; x < QT; ++x)
                                w.acc[x][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(v1, s[x][kt][i], w.acc[x][t], 0, 0, 0);
                        }
            } else {
#pragma unroll
                for (int h = 0; h < KT / 2; ++h) {
                    bf16x8 p[QT];
#pragma unroll
                    for (int x = 0; x < QT; ++x) p[x] = weights_operand(s[x][2 * h], s[x][2 * h + 1]);
                    const DT* at = lv + (32 * h + 4 * g + (c >> 2)) * kVRow + 4 * (c & 3);
#pragma unroll
                    for (int t = 0; t < ND; ++t) {
                        const bf16x8 b = values_operand(reinterpret_cast<const bf16_t*>(at + 16 * t), kVRow);
#pragma unroll
                        for (int x = 0; x < QT; ++x)
                            w.acc[x][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, p[x], w.acc[x][t], 0, 0, 0);
                    }
                }
            }
        }
    }
};

template <typename DT, int ND, int W>
constexpr size_t attn_lds() {
    const size_t join = size_t(W) * kTileRows * (16 * ND + 4) * 4;
    const size_t v = sizeof(DT) == 2 ? size_t(W) * 32 * (16 * ND + 16) * 2 : 0;
    return join > v ? join : v;
}

// What a workgroup takes, and where its rows' results go.
struct AttnItem {
    bool prefix;
    int tile, hk, part, own, rows;  // own: the sequence of a suffix; rows: query rows that share its keys
    int64_t n;
    int plen, from, end, r, Hq, G, slot;

    // false: nothing to do (past the last item, or a part past the length, which the joining kernel
    // does not look at)
    // `solo_prefix`, `solo_suffix`: the wave, where waves have items of their own, else -1.
    __device__ __forceinline__ bool of(const AttnArgs& a, const AttnPlan& plan, int block, int solo_prefix, int solo_suffix) {
        const int group = block / kGroup;
        const int before = int(int64_t(group) * plan.prefix_groups / plan.groups);
        prefix = int64_t(group + 1) * plan.prefix_groups / plan.groups > before;
        // Workgroups that run on one XCD are eight apart: there, two tiles of a prefix read the same keys.
        // The XCDs take turns at a group's places, which else could be the same part of every
        // sequence (with eight parts and suffixes half their longest, half of the XCDs had no work).
        const int within = ((block + group) % 8) * (kGroup / 8) + block % kGroup / 8;
        int item = (prefix ? before : group - before) * kGroup + within;
        if ((prefix ? solo_prefix : solo_suffix) >= 0) item = item * kAttnWaves + (prefix ? solo_prefix : solo_suffix);
        if (item >= (prefix ? +plan.prefix_items : +plan.suffix_items)) return false;
        // (all of these are below 2^31, so 32-bit divisions do)
        Hq = a.Hq;
        G = a.G;
        const int Hkv = a.Hkv;
        r = Hq / Hkv;
        const int tiles = prefix ? +plan.prefix_tiles : +plan.suffix_tiles;
        const int parts = prefix ? +plan.prefix_parts : +plan.suffix_parts;
        tile = item % tiles;
        item /= tiles;
        hk = item % Hkv;
        item /= Hkv;
        part = item % parts;
        item /= parts;
        n = prefix ? item : item / G;
        own = prefix ? 0 : item % G;
        rows = prefix ? G * r : r;
        plen = clamp_len(a.prefix_len, n, a.P);
        const int chunk = prefix ? +plan.prefix_chunk : +plan.suffix_chunk;
        from = part * chunk;  // (parts reach past 2^30 by less than a chunk)
        end = prefix ? plen : clamp_len(a.suffix_len, n * G + own, a.S);
        if (end - from > chunk) end = from + chunk;
        slot = prefix ? part : (plan.whole ? 0 : plan.prefix_parts) + part;
        return !plan.part_acc || from < end;
    }
    // Row of the outputs that row i of the item is.
    __device__ __forceinline__ int64_t out_row(int i) const {
        const int g = prefix ? i / r : own, h = hk * r + (prefix ? i % r : i);
        return (n * G + g) * Hq + h;
    }
    template <typename DT>
    __device__ __forceinline__ const DT* query(const AttnArgs& a, int i) const {
        if (i >= rows) return nullptr;
        const int g = prefix ? i / r : own, h = hk * r + (prefix ? i % r : i);
        return reinterpret_cast<const DT*>(a.q) + n * a.at.q[0] + g * a.at.q[1] + h * a.at.q[2];
    }
    // Four dimensions of a row: to the part, or finished.
    template <typename DT>
    __device__ __forceinline__ void store(const AttnArgs& a, const AttnPlan& plan, int i, int d, f32x4 o, float m, float z) const {
        const int64_t out = out_row(i);
        if (plan.part_acc) {
            const int64_t at = int64_t(slot) * (a.N * G * Hq) + out;
            *reinterpret_cast<f32x4*>(plan.part_acc + at * a.D + d) = o;
            if (d == 0) plan.part_ml[at] = float2{m, z};
        } else {
            finish<DT>(a, out, d, o, m, z);
        }
    }
    template <typename DT>
    // (a sum of 0 has no keys; one of NaN, of a NaN among them or the query, makes the row NaN)
    static __device__ __forceinline__ void finish(const AttnArgs& a, int64_t out, int d, f32x4 o, float m, float z) {
        const bool none = z == 0.f;
        o = none ? f32x4{0.f, 0.f, 0.f, 0.f} : o / z;
        DT* p = reinterpret_cast<DT*>(a.o) + out * a.D + d;
        if constexpr (sizeof(DT) == 4) {
            *reinterpret_cast<f32x4*>(p) = o;
        } else {
            bf16x4 b;
#pragma unroll
            for (int e = 0; e < 4; ++e) b[e] = static_cast<__bf16>(o[e]);
            *reinterpret_cast<bf16x4*>(p) = b;
        }
        if (d == 0 && a.lse) a.lse[out] = none ? kNegInf : kLn2 * (m + log2_fast(z));
    }
};

// A negative scale is its amount with the queries' signs flipped, so that maxima are taken before
// scaling; and not 0, so that a masked score stays -inf.
template <typename DT>
__device__ __forceinline__ uint32_t query_sign(float scale2) {
    return scale2 < 0.f ? (sizeof(DT) == 4 ? 0x80000000u : 0x80008000u) : 0u;
}
__device__ __forceinline__ float score_scale(float scale2) { return fmaxf(fabsf(scale2), 1e-30f); }

// The prefix's or the suffix's keys and values of an item.
template <typename DT>
struct ItemKeys {
    const DT *k, *v;
    int64_t sk, sv;
    __device__ __forceinline__ ItemKeys(const AttnArgs& a, const AttnItem& it, bool prefix) {
        int64_t ak, av;
        if (prefix) {
            k = reinterpret_cast<const DT*>(a.kp);
            v = reinterpret_cast<const DT*>(a.vp);
            ak = it.n * a.at.kp[0] + it.hk * a.at.kp[2];
            av = it.n * a.at.vp[0] + it.hk * a.at.vp[2];
            sk = a.at.kp[1];
            sv = a.at.vp[1];
        } else {
            k = reinterpret_cast<const DT*>(a.ks);
            v = reinterpret_cast<const DT*>(a.vs);
            ak = it.n * a.at.ks[0] + it.own * a.at.ks[1] + it.hk * a.at.ks[3];
            av = it.n * a.at.vs[0] + it.own * a.at.vs[1] + it.hk * a.at.vs[3];
            sk = a.at.ks[2];
            sv = a.at.vs[2];
        }
        k += ak;
        v += av;
    }
};

// Waves of the workgroup on the same sixteen rows and keys of their own.
template <typename DT, int ND, int W, bool EXACT>
__device__ __forceinline__ void attn_split_keys(const AttnArgs& a, const AttnPlan& plan, const AttnItem& it, char* mem,
                                                float (*s_m)[kTileRows], float (*s_l)[kTileRows]) {
    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int D = EXACT ? 16 * ND : int(a.D);
    bf16_t* lds = reinterpret_cast<bf16_t*>(mem) + wave * 32 * (16 * ND + 16);
    const int row0 = it.tile * kTileRows;
    AttnWave<DT, ND, 1, EXACT> w;
    w.clear();
    w.load_query(0, it.template query<DT>(a, row0 + c), D, query_sign<DT>(a.scale2), lane);
    // the prefix (for a suffix tile only if it takes all), then the suffix
    for (int pass = it.prefix || plan.whole ? 0 : 1; pass < (it.prefix ? 1 : 2); ++pass) {
        const bool all = pass == 0 && !it.prefix;
        const ItemKeys<DT> x(a, it, pass == 0);
        w.template run<W>(x.k, x.v, x.sk, x.sv, all ? 0 : it.from, all ? it.plen : it.end, D, score_scale(a.scale2), lds, wave, lane);
    }

    // the waves join
    float* join = reinterpret_cast<float*>(mem);
    constexpr int kJoinRow = 16 * ND + 4;
    float l = w.l[0];
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    __syncthreads();
    if (g4 == 0) {
        s_m[wave][c] = w.m[0];
        s_l[wave][c] = l;
    }
#pragma unroll
    for (int t = 0; t < ND; ++t)
        *reinterpret_cast<f32x4*>(join + (wave * kTileRows + c) * kJoinRow + 16 * t + 4 * g4) = w.acc[0][t];
    __syncthreads();
    for (int at = tid; at < kTileRows * 4 * ND; at += W * kWave) {
        const int i = at / (4 * ND), d = 4 * (at % (4 * ND));
        const int row = row0 + i;
        if (row >= it.rows || d >= D) continue;
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
        it.template store<DT>(a, plan, row, d, o, m, z);
    }
}

// The rows of a wave that has worked out all of their keys.
template <typename DT, int ND, int QT, bool EXACT>
__device__ __forceinline__ void attn_store_wave(const AttnArgs& a, const AttnPlan& plan, const AttnItem& it, int row0,
                                                const AttnWave<DT, ND, QT, EXACT>& w) {
    const int lane = threadIdx.x & 63, c = lane & 15, g4 = lane >> 4;
    const int D = EXACT ? 16 * ND : int(a.D);
#pragma unroll
    for (int x = 0; x < QT; ++x) {
        float l = w.l[x];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        const int row = row0 + x * kTileRows + c;
        if (row >= it.rows) continue;
#pragma unroll
        for (int t = 0; t < ND; ++t)
            if (EXACT || 16 * t + 4 * g4 < D) it.template store<DT>(a, plan, row, 16 * t + 4 * g4, w.acc[x][t], w.m[x], l);
    }
}

// A wave on rows and keys of its own: no barrier, nothing to join. (Prefix or suffix is a matter of
// compilation: a choice between members of the arguments at run time kept those in memory.)
template <typename DT, int ND, bool PREFIX, bool EXACT>
__device__ __forceinline__ void attn_solo(const AttnArgs& a, const AttnPlan& plan, const AttnItem& it, char* mem) {
    const int lane = threadIdx.x & 63, c = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int D = EXACT ? 16 * ND : int(a.D);
    bf16_t* lds = reinterpret_cast<bf16_t*>(mem) + wave * 32 * (16 * ND + 16);
    const int row0 = it.tile * kTileRows;
    AttnWave<DT, ND, 1, EXACT> w;
    w.clear();
    w.load_query(0, it.template query<DT>(a, row0 + c), D, query_sign<DT>(a.scale2), lane);
    const ItemKeys<DT> x(a, it, PREFIX);
    w.template run<1>(x.k, x.v, x.sk, x.sv, it.from, it.end, D, score_scale(a.scale2), lds, 0, lane);
    attn_store_wave<DT, ND, 1, EXACT>(a, plan, it, row0, w);
}

// Waves of the workgroup on rows of their own, 16 * QT each, and the same keys: prefixes of many rows.
template <typename DT, int ND, int QT, int W, bool EXACT>
__device__ __forceinline__ void attn_share_keys(const AttnArgs& a, const AttnPlan& plan, const AttnItem& it, char* mem) {
    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15;
    const int D = EXACT ? 16 * ND : int(a.D);
    const int row0 = (it.tile * W + (tid >> 6)) * kTileRows * QT;
    AttnWave<DT, ND, QT, EXACT> w;
    w.clear();
#pragma unroll
    for (int x = 0; x < QT; ++x)
        w.load_query(x, it.template query<DT>(a, row0 + x * kTileRows + c), D, query_sign<DT>(a.scale2), lane);
    const ItemKeys<DT> x(a, it, true);
    SharedKeys<DT, ND, QT, W, EXACT>::run(w, x.k, x.v, x.sk, x.sv, it.from, it.end, D, score_scale(a.scale2), reinterpret_cast<DT*>(mem), tid);
    attn_store_wave<DT, ND, QT, EXACT>(a, plan, it, row0, w);
}

// How the rows of a prefix are taken: like a suffix's; by waves of their own, four of one tile; or, in a
// kernel of its own, by more rows: bfloat16 four or eight waves of two tiles, float32 eight of one.
enum PrefixRows { kPrefixOne, kPrefixShared64, kPrefixShared128, kPrefixShared256 };

template <typename DT, int ND, PrefixRows PR, bool EXACT>
constexpr size_t attn_mem() {
    const size_t n = attn_lds<DT, ND, kAttnWaves>(), k = SharedKeys<DT, ND, 1, kAttnWaves, EXACT>::kLds;
    return PR == kPrefixShared64 && k > n ? k : n;
}

// Every item but a prefix of more than 64 rows. Bound by memory: a key and its value
// (512 bytes in bfloat16, D = 128) meet 256 multiply-adds of each query row, of which a suffix has as many as a
// key head serves heads.
// Solo waves on full suffixes, 64 sequences x 4096 tokens x 8 heads x 128 bfloat16 (1.07 GB): 190 us,
// 5.7 TB/s, 512 sequences 1393 us, 6.2 TB/s; with lengths at random 126 us for half the bytes, 4.3 TB/s: what
// is left when the short ones have ended does not fill the CUs. A launch bound of four waves a SIMD
// spills and is slower; keys loaded straight into the operand's layout spare LDS one of its two passes.
template <typename DT, int ND, PrefixRows PR, bool SOLO, bool EXACT>
__global__ __launch_bounds__(kAttnWaves * kWave) void attn_kernel(AttnArgs a, AttnPlan plan) {
    __shared__ __attribute__((aligned(16))) char s_mem[attn_mem<DT, ND, PR, EXACT>()];
    const int wave = SOLO ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : -1;
    AttnItem it;
    if (!it.of(a, plan, int(grid_row()), PR == kPrefixOne ? wave : -1, wave)) return;
    if constexpr (PR == kPrefixShared64) {
        if (it.prefix) {
            attn_share_keys<DT, ND, 1, kAttnWaves, EXACT>(a, plan, it, s_mem);
            return;
        }
    }
    if constexpr (SOLO) {
        if (PR == kPrefixOne && it.prefix) attn_solo<DT, ND, true, EXACT>(a, plan, it, s_mem);
        else attn_solo<DT, ND, false, EXACT>(a, plan, it, s_mem);
    } else {
        __shared__ float s_m[kAttnWaves][kTileRows], s_l[kAttnWaves][kTileRows];
        attn_split_keys<DT, ND, kAttnWaves, EXACT>(a, plan, it, s_mem, s_m, s_l);
    }
}

// The prefix alone: its registers (two tiles a wave) would halve the suffix's waves on a CU. Bound by the
// vector unit: a step's weights take some 6 of its operations for each matrix instruction, and a SIMD's two
// waves, which meet at a barrier every 64 keys, want both units at the same time. 256 rows of 32768
// keys, 8 heads, D = 128, bfloat16 (34 GFLOP): 54 us, 640 TFLOP/s, where a product of 8192^3 reaches 1227.
// Measured and left: four waves of two tiles, two workgroups a CU, 86 us (every key is staged twice); one
// tile a wave in the launch of the suffixes 137; the next step's scores issued before this step's
// weights, with a third block in LDS, 58; the products' accumulators held in vector registers, the same.
template <typename DT, int ND, int QT, int W, bool EXACT>
__global__ __launch_bounds__(W * kWave) void attn_prefix_kernel(AttnArgs a, AttnPlan plan) {
    __shared__ __attribute__((aligned(16))) char s_mem[SharedKeys<DT, ND, QT, W, EXACT>::kLds];
    AttnItem it;
    if (!it.of(a, plan, int(grid_row()), -1, -1)) return;
    attn_share_keys<DT, ND, QT, W, EXACT>(a, plan, it, s_mem);
}

// Joins the parts of a row, o = sum_i 2^(m_i - m) o_i / sum_i 2^(m_i - m) l_i: one row a workgroup,
// `groups` of D / 4 lanes (four dimensions each) on every groups-th part. Bound by latency and by reading
// again what the parts wrote, 4 D + 8 bytes a part and row: 512 rows 4 us, 4096 rows 10, 16384 rows 22.
template <typename DT>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a, AttnPlan plan) {
    __shared__ f32x4 s_o[256];
    __shared__ float s_z[256];
    const int lanes = a.D / 4, groups = 256 / lanes;
    const int64_t rows = a.N * a.G * a.Hq, out = grid_row();
    if (out >= rows) return;
    const int group = int(threadIdx.x) / lanes, d = 4 * (int(threadIdx.x) % lanes);
    const int seq = int(out) / a.Hq;
    const int plen = plan.whole ? 0 : clamp_len(a.prefix_len, seq / a.G, a.P), slen = clamp_len(a.suffix_len, seq, a.S);
    // parts that hold keys
    const int np = (plen + plan.prefix_chunk - 1) / plan.prefix_chunk, ns = (slen + plan.suffix_chunk - 1) / plan.suffix_chunk;
    auto slot = [&](int i) { return (i < np ? i : plan.prefix_parts + i - np) * rows + out; };
    float m = kNegInf;
    for (int i = int(threadIdx.x) & 63; i < np + ns; i += kWave) m = fmaxf(m, plan.part_ml[slot(i)].x);
    m = max_wave(m);
    float z = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    if (group < groups) {
        for (int i = group; i < np + ns; i += groups) {
            const float2 ml = plan.part_ml[slot(i)];
            const float keep = exp2_fast(ml.x - m);
            z = fmaf(keep, ml.y, z);
            o += keep * *reinterpret_cast<const f32x4*>(plan.part_acc + slot(i) * a.D + d);
        }
    }
    s_o[threadIdx.x] = o;
    s_z[threadIdx.x] = z;
    __syncthreads();
    if (group != 0) return;
    for (int i = 1; i < groups; ++i) {
        o += s_o[threadIdx.x + i * lanes];
        z += s_z[threadIdx.x + i * lanes];
    }
    AttnItem::finish<DT>(a, out, d, o, m, z);
}

}  // namespace rlcs
