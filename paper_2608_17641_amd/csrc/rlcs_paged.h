// Attention of a chunk of new tokens a sequence over a paged cache, and the writing of their keys and values.
//
// A tile is up to R rows (token, query head of one key head) of one sequence, in the order of tokens; row i of a
// sequence with T new tokens and L in all sees the first L - T + i / r + 1 keys, r query heads to a key head.
// Sequences of up to kFewRows rows a key head are one tile, whose keys are dealt to the waves of a workgroup, each
// with running maxima, sums and outputs of its own, which join at the end: bound by reading the keys. Longer
// chunks are tiles of more rows, each wave with rows of its own and all with the same keys, in LDS: bound by the
// matrix and the vector units. Long key ranges are cut into parts, which a second kernel joins; how long a part is
// follows from the lengths on the device, which every workgroup adds up for itself.
//
// Products, operand layouts and softmax are those of attention over a shared prefix (rlcs_attn.h). Keys are
// addressed sixteen at a time, as sixteen lie in one page: a wave holds the next page numbers of its way in its
// lanes, one load for many blocks, and hands them to scalar registers.
#pragma once

#include "rlcs_attn.h"

namespace rlcs {

struct PagedArgs {
    const void *q, *k, *v;
    const int32_t *table, *length, *q_start;
    void* o;
    float* lse;
    int64_t ld_table, tokens;
    int64_t qs[2], ks[3], vs[3];
    int32_t B, W, pages, shift, Hq, Hkv, D, r, max_chunk;
    float scale2;  // scale * log2(e)
    // Tiles of at most few_rows rows are the first kernel's, the others the second's.
    int32_t few_rows;
    // How many items a key head the parts of this kernel should come to (0: no parts), at least how many keys a part
    // has, and places for parts in the workspace.
    int32_t want, least, slots;
    float* part_acc;   // [key head][slot][row][D]: outputs relative to the part's own maximum
    float2* part_ml;   // [key head][slot][row]: maximum (base 2) and sum
};

constexpr int kKeyGroup = 16;  // keys that are addressed together

// A sequence: its first row of q, its new tokens, how many of these count, and all of its tokens.
struct PagedSeq {
    int64_t first;
    int n, taken, length;
};
__device__ __forceinline__ PagedSeq paged_seq(const PagedArgs& a, int b) {
    PagedSeq s;
    if (a.q_start) {
        int64_t x = a.q_start[b], y = a.q_start[b + 1];
        x = x < 0 ? 0 : x > a.tokens ? a.tokens : x;
        y = y < x ? x : y > a.tokens ? a.tokens : y;
        s.first = x;
        s.n = int(y - x);
    } else {
        const int64_t n = a.tokens / a.B;
        s.first = b * n;
        s.n = int(n);
    }
    s.taken = s.n < a.max_chunk ? s.n : a.max_chunk;
    const int length = a.length[b], most = a.pages ? a.W << a.shift : 0;
    s.length = length < 0 ? 0 : length > most ? most : length;
    return s;
}

// How a kernel's tiles of R rows are cut: tiles of a sequence (none, if it is the other kernel's), and parts of each.
struct PagedCut {
    int chunk;  // keys of a part (a multiple of 64), or 0: one part
    template <bool FEW, int R>
    static __device__ __forceinline__ int tiles(const PagedArgs& a, const PagedSeq& s) {
        const int64_t rows = int64_t(s.taken) * a.r;
        if (FEW) return rows > 0 && rows <= a.few_rows ? 1 : 0;
        return rows > a.few_rows ? int((rows + R - 1) / R) : 0;
    }
    __device__ __forceinline__ int parts(const PagedSeq& s) const {
        if (chunk == 0 || s.length <= chunk) return 1;
        return (s.length + chunk - 1) / chunk;
    }
    // From the sum over all sequences of keys that tiles read: every wave for itself.
    template <bool FEW, int R>
    __device__ __forceinline__ void plan(const PagedArgs& a) {
        chunk = 0;
        if (a.want == 0) return;
        int64_t blocks = 0;
        for (int b = int(threadIdx.x) & 63; b < a.B; b += kWave) {
            const PagedSeq s = paged_seq(a, b);
            blocks += int64_t(tiles<FEW, R>(a, s)) * ((s.length + 63) / 64);
        }
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) blocks += __shfl_xor(blocks, d);
        int64_t each = (blocks + a.want - 1) / a.want * 64;
        if (each < a.least) each = a.least;
        chunk = int(each < (int64_t(1) << 30) ? each : int64_t(1) << 30);
        chunk = __builtin_amdgcn_readfirstlane(chunk);
    }
};

// What a workgroup takes.
struct PagedItem {
    PagedSeq s;
    int b, hk, tile, parts, part, from, end;  // end: past the last key that any of the tile's rows sees
    int slot;
    int64_t rows;  // of the sequence

    // Item `item` of a key head; false: there are fewer.
    template <bool FEW, int R>
    __device__ __forceinline__ bool of(const PagedArgs& a, const PagedCut& cut, int item, int head) {
        const int lane = threadIdx.x & 63;
        int64_t base = 0;
        int found = -1, local = 0;
        for (int b0 = 0; b0 < a.B; b0 += kWave) {
            int items = 0;
            if (b0 + lane < a.B) {
                const PagedSeq s = paged_seq(a, b0 + lane);
                items = tiles_of<FEW, R>(a, s) * cut.parts(s);
            }
            int upto = items;
#pragma unroll
            for (int d = 1; d < kWave; d <<= 1) {
                const int o = __shfl_up(upto, d);
                if (lane >= d) upto += o;
            }
            const uint64_t past = __ballot(base + upto > item);
            if (past) {
                const int at = __ffsll((unsigned long long)past) - 1;
                found = b0 + at;
                local = int(item - base) - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(items, at));
                break;
            }
            base += __builtin_amdgcn_readlane(upto, 63);
        }
        if (found < 0) return false;
        b = __builtin_amdgcn_readfirstlane(found);
        hk = head;
        s = paged_seq(a, b);
        rows = int64_t(s.taken) * a.r;
        parts = cut.parts(s);
        const int tiles = tiles_of<FEW, R>(a, s);
        part = local % parts;
        tile = tiles - 1 - local / parts;  // (those that see the most keys first)
        slot = item;
        end = sees(int64_t(tile + 1) * R - 1, a);
        from = part * cut.chunk;
        if (parts > 1 && end - from > cut.chunk) end = from + cut.chunk;
        return true;
    }
    template <bool FEW, int R>
    static __device__ __forceinline__ int tiles_of(const PagedArgs& a, const PagedSeq& s) {
        return PagedCut::tiles<FEW, R>(a, s);
    }
    // How many keys row i of the sequence sees (a row past its last: as many as that).
    __device__ __forceinline__ int sees(int64_t i, const PagedArgs& a) const {
        if (i >= rows) i = rows - 1;
        const int n = s.length - s.n + int(i / a.r) + 1;
        return n < 0 ? 0 : n > s.length ? s.length : n;
    }
    __device__ __forceinline__ int64_t out_row(int64_t i, const PagedArgs& a) const { return (s.first + i / a.r) * a.Hq + hk * a.r + i % a.r; }
    template <typename DT>
    __device__ __forceinline__ const DT* query(int64_t i, const PagedArgs& a) const {
        if (i >= rows) return nullptr;
        return reinterpret_cast<const DT*>(a.q) + (s.first + i / a.r) * a.qs[0] + (hk * a.r + i % a.r) * a.qs[1];
    }
    // Four dimensions of row i: to the part, or finished. R: rows of a tile.
    template <typename DT, int R>
    __device__ __forceinline__ void store(int64_t i, int d, f32x4 o, float m, float z, const PagedArgs& a) const {
        if (parts > 1) {
            const int64_t at = (int64_t(hk) * a.slots + slot) * R + i % R;
            *reinterpret_cast<f32x4*>(a.part_acc + at * a.D + d) = o;
            if (d == 0) a.part_ml[at] = float2{m, z};
        } else {
            finish<DT>(out_row(i, a), d, o, m, z, a);
        }
    }
    // (a sum of 0 has no keys; one of NaN, of a NaN among them or the query, makes the row NaN)
    template <typename DT>
    static __device__ __forceinline__ void finish(int64_t out, int d, f32x4 o, float m, float z, const PagedArgs& a) {
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

// Page numbers of the groups of keys on a wave's way: G groups a block, group x of block n at key
// first + n * hop + offset(x). Lane n % (64 / G) * G + x holds the one of (n, x), the lanes of the next 64 / G blocks
// are on their way while these are used. Keys past the last one count as that.
template <int G>
struct PageNumbers {
    const int32_t* row;
    int first, hop, last, shift, lane_offset;
    int now, next;

    template <class F>
    __device__ __forceinline__ void begin(const int32_t* table_row, int first_, int hop_, int end, int shift_, F&& offset) {
        row = table_row;
        first = first_;
        hop = hop_;
        last = end - 1;
        shift = shift_;
        lane_offset = offset((int(threadIdx.x) & 63) % G);
        now = ask(0);
        next = ask(64 / G);
    }
    __device__ __forceinline__ int ask(int n) const {
        const int64_t key = int64_t(first) + int64_t(n + (int(threadIdx.x) & 63) / G) * hop + lane_offset;
        return row[(key < last ? int(key) : last) >> shift];
    }
    // Blocks in order, each once for every group, the groups in order.
    __device__ __forceinline__ int get(int n, int x) {
        constexpr int kBlocks = 64 / G;
        if (x == 0 && n && n % kBlocks == 0) {
            now = next;
            next = ask(n + kBlocks);
        }
        return __builtin_amdgcn_readlane(now, n % kBlocks * G + x);
    }
};

// Sixteen keys: where the first is, how far the last that exists is from it, and whether there is a page.
struct KeyGroup {
    int64_t at_k, at_v;  // bytes from the caches' begin
    int last;
    bool there;
    template <typename DT>
    __device__ __forceinline__ void of(const PagedArgs& a, int page, int key, int end, int hk) {
        const int in_end = (end - 1) & ~(kKeyGroup - 1);
        key = key < in_end ? key : in_end;
        last = end - 1 - key < kKeyGroup - 1 ? end - 1 - key : kKeyGroup - 1;
        there = unsigned(page) < unsigned(a.pages);
        const int64_t p = there ? page : 0, t = key & ((1 << a.shift) - 1);
        at_k = (p * a.ks[0] + t * a.ks[1] + hk * a.ks[2]) * int64_t(sizeof(DT));
        at_v = (p * a.vs[0] + t * a.vs[1] + hk * a.vs[2]) * int64_t(sizeof(DT));
    }
};

// One softmax step as softmax_step(), of rows that may have seen no key yet.
template <int KT, int ND>
__device__ __forceinline__ void chunk_softmax_step(f32x4 (&s)[KT], float scale, float& m, float& l, f32x4 (&acc)[ND]) {
    float top = kNegInf;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[kt][i]);
    const float m1 = fmaxf(m, max_of_four(top) * scale);
    const float by = m1 == kNegInf ? 0.f : m1;
    if (__any(m1 > m)) {
        const float keep = exp2_fast(m - by);
        l *= keep;
#pragma unroll
        for (int t = 0; t < ND; ++t) acc[t] *= keep;
        m = m1;
    }
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            s[kt][i] = exp2_fast(fmaf(s[kt][i], scale, -by));
            l += s[kt][i];
        }
}

// Scores of keys that a row does not see, or that have no page, count as -inf. `first`: key of the lane's first score;
// `out`: bits of the groups without a page.
template <int KT>
__device__ __forceinline__ void hide_scores(f32x4 (&s)[KT], int first, int sees, uint32_t out) {
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (first + 16 * kt + i >= sees || (out >> kt & 1)) s[kt][i] = kNegInf;
}

// ------------------------------------------------------------- few rows: keys dealt to waves

// Keys [from, end) of one item, blocks wave, wave + W, ..., by a wave with QT tiles of sixteen rows.
template <typename DT, int ND, int QT, int W, bool EXACT>
__device__ __forceinline__ void paged_run(AttnWave<DT, ND, QT, EXACT>& w, const PagedArgs& a, const PagedItem& it, const int (&sees)[QT], int least,
                                          int D, float scale, bf16_t* lds, int wave, int lane) {
    typedef KeyBlock<DT, ND, EXACT> Block;
    constexpr bool kWide = sizeof(DT) == 4;
    constexpr int kKeys = Block::kKeys, KT = kKeys / 16, G = kKeys / kKeyGroup, kVecs = Block::kVecs;
    const int c = lane & 15, g = lane >> 4, end = it.end;
    int j = it.from + wave * kKeys;
    if (j >= end) return;
    PageNumbers<G> numbers;
    numbers.begin(a.table + int64_t(it.b) * a.ld_table, j, W * kKeys, end, a.shift, [](int x) { return kKeyGroup * x; });
    Block b;
    KeyGroup at[G];
    const uint32_t sk = uint32_t(a.ks[1]), sv = uint32_t(a.vs[1]);
    auto aim = [&](int n, int key) {  // block n of the wave, at `key`
#pragma unroll
        for (int x = 0; x < G; ++x) at[x].template of<DT>(a, numbers.get(n, x), key + kKeyGroup * x, end, it.hk);
    };
    auto row = [&](int r, const KeyGroup& k) { return uint32_t(r < k.last ? r : k.last); };
    auto load_k = [&]() {
        constexpr int kSteps = ND / Block::kKRows;
#pragma unroll
        for (int kt = 0; kt < Block::kKRows; ++kt) {
            const char* base = reinterpret_cast<const char*>(a.k) + at[kt].at_k;
            const uint32_t first = row(c, at[kt]) * sk * uint32_t(sizeof(DT)) + 16u * g;
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                uint32_t o = first + 64u * s;
                if constexpr (!EXACT) {
                    const uint32_t d = 64u * s + 16u * g, most = uint32_t(D) * sizeof(DT) - 16u;
                    if (d > most) o -= d - most;
                }
                b.k[kt * kSteps + s] = *reinterpret_cast<const u32x4*>(base + o);
            }
        }
    };
    auto load_v = [&]() {
        if constexpr (kWide) {
            const char* base = reinterpret_cast<const char*>(a.v) + at[0].at_v;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t first = (row(4 * g + i, at[0]) * sv + c) * 4u;
#pragma unroll
                for (int t = 0; t < ND; ++t) {
                    uint32_t o = first + 64u * t;
                    if constexpr (!EXACT) {
                        const int d = 16 * t + c;
                        if (d >= D) o -= 4u * uint32_t(d - D + 1);
                    }
                    b.v[t][i] = *reinterpret_cast<const uint32_t*>(base + o);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < ND; ++i) {
                constexpr int kRows = 64 / kVecs;  // of a load
                const KeyGroup& k = at[i * kRows / kKeyGroup];
                const int r = (lane / kVecs + i * kRows) % kKeyGroup, piece = lane % kVecs;
                const uint32_t o = (row(r, k) * sv + 8u * (EXACT || 8 * piece < D ? piece : D / 8 - 1)) * 2u;
                b.v[i] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(a.v) + k.at_v + o);
            }
        }
    };
    auto missing = [&]() {
        uint32_t m = 0;
#pragma unroll
        for (int x = 0; x < G; ++x) m |= at[x].there ? 0u : 1u << x;
        return m;
    };
    aim(0, j);
    uint32_t out = missing();
    load_k();
    load_v();
    for (int n = 1;; ++n) {
        const int here = j;
        const uint32_t out_here = out;
        j += W * kKeys;
        const bool more = j < end;
        if (out_here) {  // what is read in place of no page may be anything: its values become 0
#pragma unroll
            for (int i = 0; i < ND; ++i) {
                constexpr int kRows = kWide ? 0 : 64 / kVecs;
                if (out_here >> (i * kRows / kKeyGroup) & 1) b.v[i] = u32x4{0, 0, 0, 0};
            }
        }
        if (more) {
            aim(n, j);
            out = missing();
        }
        u32x4 now[kWide ? ND : 1];
        if constexpr (kWide) {
#pragma unroll
            for (int t = 0; t < ND; ++t) now[t] = b.v[t];
        } else {
            b.stage(lds, lane);
        }
        if (more) load_v();

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
                                                                          __builtin_bit_cast(bf16x8, w.q[x][d]), s[x][kt], 0, 0, 0);
        } else {
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int x = 0; x < QT; ++x)
                        s[x][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(b.k[d][i]), __uint_as_float(w.q[x][d][i]), s[x][0], 0, 0, 0);
        }
        if (more) load_k();

        if (here + kKeys > least || out_here) {
#pragma unroll
            for (int x = 0; x < QT; ++x) hide_scores<KT>(s[x], here + 4 * g, sees[x], out_here);
        }
#pragma unroll
        for (int x = 0; x < QT; ++x) chunk_softmax_step<KT, ND>(s[x], scale, w.m[x], w.l[x], w.acc[x]);
        if constexpr (!kWide) {
            bf16x8 p[QT];
#pragma unroll
            for (int x = 0; x < QT; ++x) p[x] = weights_operand(s[x][0], s[x][1]);
            const bf16_t* from = lds + (4 * g + (c >> 2)) * Block::kRow + 4 * (c & 3);
#pragma unroll
            for (int t = 0; t < ND; ++t) {
                const bf16x8 v = values_operand(from + 16 * t, Block::kRow);
#pragma unroll
                for (int x = 0; x < QT; ++x) w.acc[x][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[x], w.acc[x][t], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int t = 0; t < ND; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int x = 0; x < QT; ++x)
                        w.acc[x][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(now[t][i]), s[x][0][i], w.acc[x][t], 0, 0, 0);
        }
        if (!more) return;
    }
}

// Sequences of few rows: four waves on the same rows, each with keys of its own.
template <typename DT, int ND, int QT, bool EXACT>
__global__ __launch_bounds__(kAttnWaves * kWave) void paged_few_kernel(PagedArgs a) {
    constexpr int W = kAttnWaves, R = QT * kTileRows;
    __shared__ __attribute__((aligned(16))) char s_mem[attn_lds<DT, ND, W>()];
    __shared__ float s_m[W][kTileRows], s_l[W][kTileRows];
    const int block = int(grid_row());
    PagedCut cut;
    cut.plan<true, R>(a);
    PagedItem it;
    if (!it.template of<true, R>(a, cut, block / a.Hkv, block % a.Hkv)) return;
    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int D = EXACT ? 16 * ND : int(a.D);
    AttnWave<DT, ND, QT, EXACT> w;
    w.clear();
    int sees[QT];
#pragma unroll
    for (int x = 0; x < QT; ++x) {
        w.load_query(x, it.template query<DT>(kTileRows * x + c, a), D, query_sign<DT>(a.scale2), lane);
        sees[x] = it.sees(kTileRows * x + c, a);
        if (sees[x] > it.end) sees[x] = it.end;
    }
    int least = it.sees(0, a);
    if (least > it.end) least = it.end;
    paged_run<DT, ND, QT, W, EXACT>(w, a, it, sees, least, D, score_scale(a.scale2), reinterpret_cast<bf16_t*>(s_mem) + wave * 32 * (16 * ND + 16), wave,
                                    lane);

    // the waves join, sixteen rows at a time
    float* join = reinterpret_cast<float*>(s_mem);
    constexpr int kJoinRow = 16 * ND + 4;
#pragma unroll
    for (int x = 0; x < QT; ++x) {
        const int row0 = kTileRows * x, left = int(it.rows) - row0, rows = left < kTileRows ? left : kTileRows;
        if (rows <= 0) break;
        float l = w.l[x];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        __syncthreads();  // (the values, or the tile before, have been read)
        if (g4 == 0) {
            s_m[wave][c] = w.m[x];
            s_l[wave][c] = l;
        }
#pragma unroll
        for (int t = 0; t < ND; ++t) *reinterpret_cast<f32x4*>(join + (wave * kTileRows + c) * kJoinRow + 16 * t + 4 * g4) = w.acc[x][t];
        __syncthreads();
        for (int at = tid; at < rows * 4 * ND; at += W * kWave) {
            const int i = at / (4 * ND), d = 4 * (at % (4 * ND));
            if (d >= D) continue;
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
            it.template store<DT, R>(row0 + i, d, o, m, z, a);
        }
    }
}

// ------------------------------------------------------------- many rows: waves share keys

// Keys [from, end) of an item for a workgroup whose waves have rows of their own: all of its lanes bring blocks of keys and
// values to LDS, every wave reads them from there. While one block is worked on, the next is in the other half of
// LDS and the one after it on its way.
template <typename DT, int ND, int QT, int W, bool EXACT>
struct PagedShared {
    static constexpr bool kWide = sizeof(DT) == 4;
    static constexpr int kKeys = (ND > 8 ? 32 : 64) / (kWide ? 2 : 1);
    static constexpr int kVecs = ND * int(sizeof(DT));
    static constexpr int kVec = 16 / int(sizeof(DT));
    static constexpr int kKRow = 16 * ND + kVec;
    static constexpr int kVRow = 16 * ND + (kWide ? 4 : 16);
    static constexpr int kPieces = kKeys * kVecs / (W * kWave);
    static constexpr int kHalf = kKeys * (kKRow + kVRow);
    static constexpr size_t kLds = size_t(2 * kHalf) * sizeof(DT);
    static constexpr int kGroups = kKeys / kKeyGroup;

    static __device__ __forceinline__ void run(AttnWave<DT, ND, QT, EXACT>& w, const PagedArgs& a, const PagedItem& it, const int (&sees)[QT], int least,
                                               int most, int D, float scale, DT* lds, uint32_t (*s_out)[4], int tid) {
        const int lane = tid & 63, c = lane & 15, g = lane >> 4, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        constexpr int KT = kKeys / 16;
        const int from = it.from, end = it.end;
        if (from >= end) return;
        // piece i of a wave's lanes: rows (64 wave + 64 W i) / kVecs ... of a block, all in one group
        auto first_row = [&](int i) { return (64 * wave + 64 * W * i) / kVecs; };
        PageNumbers<kPieces> numbers;
        numbers.begin(a.table + int64_t(it.b) * a.ld_table, from, kKeys, end, a.shift,
                      [&](int i) { return first_row(i) / kKeyGroup * kKeyGroup; });
        const uint32_t sk = uint32_t(a.ks[1]), sv = uint32_t(a.vs[1]);
        u32x4 k[kPieces], v[kPieces];
        uint32_t out = 0;  // pieces without a page
        auto load = [&](int n) {
            const int j = from + n * kKeys;
            out = 0;
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                KeyGroup at;
                at.template of<DT>(a, numbers.get(n, i), j + first_row(i) / kKeyGroup * kKeyGroup, end, it.hk);
                out |= at.there ? 0u : 1u << i;
                const int piece = lane % kVecs, r = (first_row(i) + lane / kVecs) % kKeyGroup;
                const uint32_t row = r < at.last ? r : at.last, d = uint32_t(kVec) * (EXACT || kVec * piece < D ? piece : D / kVec - 1);
                k[i] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(a.k) + at.at_k + (row * sk + d) * uint32_t(sizeof(DT)));
                v[i] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(a.v) + at.at_v + (row * sv + d) * uint32_t(sizeof(DT)));
            }
        };
        auto put = [&](int turn) {
            DT* half = lds + turn * kHalf;
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int at = tid + W * kWave * i;
                const bool none = out >> i & 1;
                if (none) v[i] = u32x4{0, 0, 0, 0};  // (what is read in place of no page may be anything)
                *reinterpret_cast<u32x4*>(half + (at / kVecs) * kKRow + kVec * (at % kVecs)) = k[i];
                *reinterpret_cast<u32x4*>(half + kKeys * kKRow + (at / kVecs) * kVRow + kVec * (at % kVecs)) = v[i];
                if (lane == 0 && first_row(i) % kKeyGroup == 0) s_out[turn][first_row(i) / kKeyGroup] = none ? 1u : 0u;
            }
        };
        const int blocks = (end - from + kKeys - 1) / kKeys;
        load(0);
        put(0);
        if (blocks > 1) load(1);
        for (int n = 0; n < blocks; ++n) {
            const int j = from + n * kKeys, turn = n & 1;
            const DT* lk = lds + turn * kHalf;
            const DT* lv = lk + kKeys * kKRow;
            __syncthreads();  // this block is there, and the one before has been read
            if (n + 1 < blocks) put(turn ^ 1);
            if (n + 2 < blocks) load(n + 2);
            if (j >= most) continue;  // (none of the wave's rows sees it)
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
            uint32_t hidden = 0;
#pragma unroll
            for (int x = 0; x < kGroups; ++x) hidden |= s_out[turn][x] << x;
            hidden = __builtin_amdgcn_readfirstlane(hidden);
            if (j + kKeys > least || hidden) {
#pragma unroll
                for (int x = 0; x < QT; ++x) hide_scores<KT>(s[x], j + 4 * g, sees[x], hidden);
            }
#pragma unroll
            for (int x = 0; x < QT; ++x) chunk_softmax_step<KT, ND>(s[x], scale, w.m[x], w.l[x], w.acc[x]);
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
                        for (int x = 0; x < QT; ++x) w.acc[x][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, p[x], w.acc[x][t], 0, 0, 0);
                    }
                }
            }
        }
    }
};

template <typename DT, int ND, int QT, int W, bool EXACT>
__global__ __launch_bounds__(W * kWave) void paged_many_kernel(PagedArgs a) {
    constexpr int R = W * QT * kTileRows;
    typedef PagedShared<DT, ND, QT, W, EXACT> Shared;
    __shared__ __attribute__((aligned(16))) char s_mem[Shared::kLds];
    __shared__ uint32_t s_out[2][4];
    const int block = int(grid_row());
    PagedCut cut;
    cut.plan<false, R>(a);
    PagedItem it;
    if (!it.template of<false, R>(a, cut, block / a.Hkv, block % a.Hkv)) return;
    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int D = EXACT ? 16 * ND : int(a.D);
    const int64_t row0 = int64_t(it.tile) * R + wave * QT * kTileRows;
    AttnWave<DT, ND, QT, EXACT> w;
    w.clear();
    int sees[QT];
#pragma unroll
    for (int x = 0; x < QT; ++x) {
        w.load_query(x, it.template query<DT>(row0 + kTileRows * x + c, a), D, query_sign<DT>(a.scale2), lane);
        sees[x] = it.sees(row0 + kTileRows * x + c, a);
        if (sees[x] > it.end) sees[x] = it.end;
    }
    int least = it.sees(row0, a), most = row0 < it.rows ? it.sees(row0 + QT * kTileRows - 1, a) : 0;
    if (least > it.end) least = it.end;
    Shared::run(w, a, it, sees, least, most, D, score_scale(a.scale2), reinterpret_cast<DT*>(s_mem), s_out, tid);
    const int g4 = lane >> 4;
#pragma unroll
    for (int x = 0; x < QT; ++x) {
        float l = w.l[x];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        const int64_t row = row0 + x * kTileRows + c;
        if (row >= it.rows) continue;
#pragma unroll
        for (int t = 0; t < ND; ++t)
            if (EXACT || 16 * t + 4 * g4 < D) it.template store<DT, R>(row, 16 * t + 4 * g4, w.acc[x][t], w.m[x], l, a);
    }
}

// The sequence that row t of q belongs to, or -1: every lane with the answer. Each round looks at 64 of the
// sequences' ends.
__device__ __forceinline__ int sequence_of(const PagedArgs& a, int64_t t) {
    if (!a.q_start) {
        const int64_t n = a.tokens / a.B;
        return int(t / n);
    }
    const int lane = threadIdx.x & 63;
    int lo = 0, n = a.B;  // the first of [lo, lo + n) whose end is past t
    while (n > 0) {
        const int step = (n + kWave - 1) / kWave, at = lo + (lane + 1) * step - 1;
        const uint64_t past = __ballot(at >= lo + n || a.q_start[at + 1] > t);
        if (!past) return -1;
        const int k = __ffsll((unsigned long long)past) - 1, was = lo;
        lo += k * step;
        const int left = was + n - lo;
        if (left <= 0) return -1;
        if (step == 1) break;
        n = left < step ? left : step;
    }
    return lo < a.B && a.q_start[lo] <= t && t < a.q_start[lo + 1] ? lo : -1;
}

// Joins the parts of a row, o = sum_i 2^(m_i - m) o_i / sum_i 2^(m_i - m) l_i: one row a workgroup,
// `groups` of D / 4 lanes (four dimensions each) on every groups-th part.
template <typename DT, bool FEW, int R>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedArgs a) {
    __shared__ f32x4 s_o[256];
    __shared__ float s_z[256];
    const int64_t out = grid_row(), t = out / a.Hq;
    if (t >= a.tokens) return;
    const int b = __builtin_amdgcn_readfirstlane(sequence_of(a, t));
    if (b < 0) return;
    const int h = int(out % a.Hq), hk = h / a.r;
    const PagedSeq s = paged_seq(a, b);
    const int tiles = PagedCut::tiles<FEW, R>(a, s);
    if (tiles == 0 || t < s.first || t - s.first >= s.taken) return;
    PagedCut cut;
    cut.plan<FEW, R>(a);
    const int parts = cut.parts(s);
    if (parts == 1) return;
    // the sequence's first slot: the items of those before it
    int64_t before = 0;
    for (int i = int(threadIdx.x) & 63; i < b; i += kWave) {
        const PagedSeq o = paged_seq(a, i);
        before += int64_t(PagedCut::tiles<FEW, R>(a, o)) * cut.parts(o);
    }
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) before += __shfl_xor(before, d);
    if (before + int64_t(tiles) * parts > a.slots) return;  // (starts that fall: more rows than there are)
    const int64_t row = (t - s.first) * a.r + h % a.r;
    const int tile = int(row / R);
    const int64_t first = int64_t(hk) * a.slots + before + int64_t(tiles - 1 - tile) * parts;
    auto place = [&](int i) { return (first + i) * R + row % R; };
    const int lanes = a.D / 4, groups = 256 / lanes;
    const int group = int(threadIdx.x) / lanes, d = 4 * (int(threadIdx.x) % lanes);
    float m = kNegInf;
    for (int i = int(threadIdx.x) & 63; i < parts; i += kWave) m = fmaxf(m, a.part_ml[place(i)].x);
    m = max_wave(m);
    float z = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    if (group < groups) {
        for (int i = group; i < parts; i += groups) {
            const float2 ml = a.part_ml[place(i)];
            const float keep = ml.x == kNegInf ? 0.f : exp2_fast(ml.x - m);
            z = fmaf(keep, ml.y, z);
            o += keep * *reinterpret_cast<const f32x4*>(a.part_acc + place(i) * a.D + d);
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
    PagedItem::finish<DT>(out, d, o, m, z, a);
}

// ------------------------------------------------------------- writing

struct PagedWriteArgs {
    PagedArgs at;  // (q: the new keys, o: nothing)
    const void *k_new, *v_new;
    char *k, *v;
    int64_t kn[2], vn[2];
    int32_t pieces;  // 16-byte pieces of a head
};

// A token a wave: its keys and values are on their way before its place is known.
template <typename DT>
__global__ __launch_bounds__(256) void paged_write_kernel(PagedWriteArgs a) {
    constexpr int kVec = 16 / sizeof(DT), U = 2;
    const int64_t t = grid_row() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (t >= a.at.tokens) return;
    const int lane = threadIdx.x & 63, all = a.at.Hkv * a.pieces;
    const DT* k = reinterpret_cast<const DT*>(a.k_new) + t * a.kn[0];
    const DT* v = reinterpret_cast<const DT*>(a.v_new) + t * a.vn[0];
    u32x4 x[U], y[U];
    auto load = [&](int at) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = at + u * kWave, h = i / a.pieces, d = i % a.pieces * kVec;
            if (i < all) {
                x[u] = *reinterpret_cast<const u32x4*>(k + h * a.kn[1] + d);
                y[u] = *reinterpret_cast<const u32x4*>(v + h * a.vn[1] + d);
            }
        }
    };
    load(lane);
    const int b = __builtin_amdgcn_readfirstlane(sequence_of(a.at, t));
    if (b < 0) return;
    const PagedSeq s = paged_seq(a.at, b);
    const int64_t place = s.length - s.n + (t - s.first);
    if (place < 0 || place >= s.length) return;
    const int page = a.at.table[b * a.at.ld_table + (place >> a.at.shift)];
    if (unsigned(page) >= unsigned(a.at.pages)) return;
    const int64_t in = place & ((1 << a.at.shift) - 1);
    DT* to_k = reinterpret_cast<DT*>(a.k) + page * a.at.ks[0] + in * a.at.ks[1];
    DT* to_v = reinterpret_cast<DT*>(a.v) + page * a.at.vs[0] + in * a.at.vs[1];
    for (int at = lane; at < all; at += U * kWave) {
        if (at != lane) load(at);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = at + u * kWave, h = i / a.pieces, d = i % a.pieces * kVec;
            if (i < all) {
                *reinterpret_cast<u32x4*>(to_k + h * a.at.ks[2] + d) = x[u];
                *reinterpret_cast<u32x4*>(to_v + h * a.at.vs[2] + d) = y[u];
            }
        }
    }
}

}  // namespace rlcs
