// Attention of a chunk of new tokens a sequence over a paged cache, and the writing of their keys and values.
//
// With s_j = scale q . k_j over the keys that a token sees, o = sum_j 2^(s_j log2 e - m) v_j / sum_j 2^(s_j log2 e - m), in one pass over
// the keys with a running maximum m, whose rise rescales what is there.
// A tile is up to R rows (token, query head of one key head) of one sequence, in the order of tokens; row i of a
// sequence with T new tokens and L in all sees the first L - T + i / r + 1 keys, r query heads to a key head.
// Sequences of up to few_rows rows a key head are one tile of sixteen or 32 rows: bound by reading the keys, each once. Where no
// sequence can be long, a workgroup takes a tile whole, its four waves with keys of their own, and joins them; else a wave
// takes a piece of the keys. Longer chunks are tiles of more rows, each wave with rows of its own and all with the same
// keys, in LDS: bound by LDS (a wave reads every key and value of its block: 256 KB a CU and 64 keys, as many clocks as the
// products take) and by the vector unit, which turns scores into weights. Tiles are cut into pieces of equal work, as the
// lengths on the device make it, which every wave adds up for itself; a second kernel joins the parts of a tile.
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
    int64_t qs[2];         // strides of q in elements
    int64_t ks[3], vs[3];  // of the caches in bytes: page, token (below 2^26), head
    int32_t B, W, pages, shift, Hq, Hkv, D, r, max_chunk;
    double rise;   // units by which a tile has more keys than the one before
    int32_t unit;  // work is counted in 2^unit keys, 64 at least, so that all of it counts in 31 bits
    float scale2;  // scale * log2(e)
    // Tiles of at most few_rows rows are the first kernel's, the others the second's.
    int32_t few_rows;
    // Pieces a key head that its keys are dealt out in; 0: whole tiles only.
    int32_t pieces;
    float* part_acc;   // [key head][slot][row][D]: outputs relative to the part's own maximum
    float2* part_ml;   // [key head][slot][row]: maximum (base 2) and sum
};

constexpr int kKeyGroup = 16;  // keys that are addressed together

// A sequence: its first row of q, its new tokens, how many of these count, and all of its tokens.
struct PagedSeq {
    int first, n, taken, length;
};
__device__ __forceinline__ PagedSeq paged_seq(const PagedArgs& a, int b) {
    PagedSeq s;
    if (a.q_start) {
        int64_t x = a.q_start[b], y = a.q_start[b + 1];
        x = x < 0 ? 0 : x > a.tokens ? a.tokens : x;
        y = y < x ? x : y > a.tokens ? a.tokens : y;
        s.first = int(x);
        s.n = int(y - x);
    } else {
        const int64_t n = a.tokens / a.B;
        s.first = int(b * n);
        s.n = int(n);
    }
    s.taken = s.n < a.max_chunk ? s.n : a.max_chunk;
    const int length = a.length[b], most = a.pages ? a.W << a.shift : 0;
    s.length = length < 0 ? 0 : length > most ? most : length;
    return s;
}

// What all lanes agree on, in scalar registers.
__device__ __forceinline__ int agreed(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Inclusive sums over the lanes.
__device__ __forceinline__ int scan_wave(int v) {
    auto step = [&](auto ctrl, auto rows) { v += __builtin_amdgcn_update_dpp(0, v, decltype(ctrl)::value, decltype(rows)::value, 0xf, false); };
    step(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});  // row_shr:1
    step(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
    step(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});  // row_bcast:15
    step(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});  // row_bcast:31
    return v;
}

// The sequences, the first 64 of them in the lanes.
struct PagedSeqs {
    const PagedArgs& a;
    PagedSeq mine;
    __device__ __forceinline__ PagedSeqs(const PagedArgs& args) : a(args) {
        const int lane = threadIdx.x & 63;
        mine = lane < a.B ? paged_seq(a, lane) : PagedSeq{0, 0, 0, 0};
    }
    __device__ __forceinline__ PagedSeq of_lane(int b0) const {  // b0 + lane
        if (b0 == 0) return mine;
        const int b = b0 + (int(threadIdx.x) & 63);
        return b < a.B ? paged_seq(a, b) : PagedSeq{0, 0, 0, 0};
    }
    __device__ __forceinline__ PagedSeq get(int b) const {
        if (b >= kWave) return paged_seq(a, b);
        return PagedSeq{__builtin_amdgcn_readlane(mine.first, b), __builtin_amdgcn_readlane(mine.n, b), __builtin_amdgcn_readlane(mine.taken, b),
                        __builtin_amdgcn_readlane(mine.length, b)};
    }
    // The sequence within which x lies, where each is as long as f says: what is left of x there, or -1 past the last.
    template <class F>
    __device__ __forceinline__ int locate(int x, int& b, F&& f) const {
        for (int b0 = 0; b0 < a.B; b0 += kWave) {
            const int own = f(of_lane(b0)), upto = scan_wave(own);
            const uint64_t past = __ballot(upto > x);
            if (past) {
                const int i = __ffsll((unsigned long long)past) - 1;
                b = b0 + i;
                return x - __builtin_amdgcn_readlane(upto - own, i);
            }
            x -= __builtin_amdgcn_readlane(upto, 63);
        }
        return -1;
    }
    template <class F>
    __device__ __forceinline__ int sum(int before, F&& f) const {  // of the sequences before that one
        int all = 0;
        for (int b0 = 0; b0 < before; b0 += kWave) all += b0 + (int(threadIdx.x) & 63) < before ? f(of_lane(b0)) : 0;
        return __builtin_amdgcn_readlane(scan_wave(all), 63);
    }
};

// How the tiles of a kernel, R rows each, are dealt out within a key head. Tiles lie one after the other on a line, each as long
// as its work: its keys, and kTile units for what a tile costs beside them. The line is cut into pieces of equal length, whole tiles and
// parts of tiles, so that all end together however lengths differ. Where they lie follows from the lengths on the device, which
// every wave adds up for itself.
// kTile was measured: of many rows, 4 sequences of 2048 to 16384 keys, the last 2048 of them new: 1366 us with 6, 1381 with 4,
// 1490 with 2, 1380 with 10, and 1421 where tiles are cut only as far as they are no multiple of the pieces.
constexpr int kTileWork = 2, kTileWorkMany = 6;
constexpr int kLeastWork = 4;  // units of a piece, at least
template <bool FEW, int R>
struct PagedLine {
    static constexpr int kTile = FEW ? kTileWork : kTileWorkMany;
    int each, more, pieces;  // their length; the first `more` are longer by one

    // Tiles of a sequence: none, if it is the other kernel's.
    static __device__ __forceinline__ int tiles(const PagedArgs& a, const PagedSeq& s) {
        const int rows = s.taken * a.r;
        if (FEW) return rows > 0 && rows <= a.few_rows ? 1 : 0;
        return rows > a.few_rows ? (rows + R - 1) / R : 0;
    }
    // Where tile t of a sequence begins. (A tile's keys are those before the chunk and as many tokens as its rows and the
    // ones before are.)
    static __device__ __forceinline__ int begin(const PagedArgs& a, const PagedSeq& s, int t) {
        if (FEW) return t * (kTile + (s.length >> a.unit));
        const int before = s.length > s.n ? s.length - s.n : 0;
        return t * (kTile + (before >> a.unit)) + int(double(int64_t(t) * (t + 1) / 2) * a.rise);
    }
    static __device__ __forceinline__ int work(const PagedArgs& a, const PagedSeq& s) { return begin(a, s, tiles(a, s)); }
    __device__ __forceinline__ void plan(const PagedArgs& a, const PagedSeqs& seqs) {
        each = more = 0;
        const int total = seqs.sum(a.B, [&](const PagedSeq& s) { return work(a, s); }), most = (total + kLeastWork - 1) / kLeastWork;
        pieces = most < a.pieces ? most : a.pieces;
        if (pieces <= 0) {
            pieces = 0;
            return;
        }
        each = int(unsigned(total) / unsigned(pieces));
        more = total - each * pieces;
    }
    __device__ __forceinline__ int piece(int w) const { return w * each + (w < more ? w : more); }
    // The key, a multiple of 64 or past the last, at which a tile is cut that many units after its begin; `sees`: its keys.
    static __device__ __forceinline__ int cut(const PagedArgs& a, int at, int length, int sees) {
        if (at >= length) return sees;
        const int64_t key = at <= kTile ? 0 : int64_t(at - kTile) << a.unit;
        return key < sees ? int(key) : sees;
    }
};

// A tile, and what is done of it.
struct PagedItem {
    PagedSeq s;
    int b, hk, tile, tiles;
    int rows;             // of the sequence
    int at, length;       // of the tile: the place in it, and its length on the line
    int all;              // keys that the last of its rows sees
    int from, end, slot;  // keys of this part; slot: of the workspace, or -1: these are all

    template <class Line>
    __device__ __forceinline__ void enter(const PagedArgs& a, const PagedSeq& of) {
        s = of;
        tiles = Line::tiles(a, s);
        rows = s.taken * a.r;
    }
    template <class Line, int R>
    __device__ __forceinline__ void aim(const PagedArgs& a) {
        length = Line::begin(a, s, tile + 1) - Line::begin(a, s, tile);
        all = sees((tile + 1) * R - 1, a);
    }
    // The tile of sequence `of`, where it has one at most, to be taken whole.
    template <int R>
    __device__ __forceinline__ bool only(const PagedArgs& a, int of) {
        typedef PagedLine<true, R> Line;
        b = of;
        tile = at = 0;
        const PagedSeq one = paged_seq(a, b);
        enter<Line>(a, PagedSeq{agreed(one.first), agreed(one.n), agreed(one.taken), agreed(one.length)});
        if (tiles == 0) return false;
        aim<Line, R>(a);
        return true;
    }
    // The tile at place x of the line.
    template <bool FEW, int R>
    __device__ __forceinline__ bool find(const PagedArgs& a, const PagedSeqs& seqs, int x) {
        typedef PagedLine<FEW, R> Line;
        at = seqs.locate(x, b, [&](const PagedSeq& o) { return Line::work(a, o); });
        if (at < 0) return false;
        enter<Line>(a, seqs.get(b));
        int lo = 0, hi = tiles;  // the last tile that begins at `at` or before
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (Line::begin(a, s, mid) <= at) lo = mid;
            else hi = mid;
        }
        tile = lo;
        at -= Line::begin(a, s, tile);
        aim<Line, R>(a);
        return true;
    }
    // The tile after it, if there is one.
    template <bool FEW, int R>
    __device__ __forceinline__ bool next(const PagedArgs& a, const PagedSeqs& seqs) {
        typedef PagedLine<FEW, R> Line;
        at = 0;
        if (++tile >= tiles) {
            tile = 0;
            do {
                if (++b >= a.B) return false;
                enter<Line>(a, seqs.get(b));
            } while (tiles == 0);
        }
        aim<Line, R>(a);
        return true;
    }
    // What piece w does of the tile with `units` of the line from its place on. False: nothing.
    template <class Line>
    __device__ __forceinline__ bool take(const PagedArgs& a, int w, int units) {
        from = Line::cut(a, at, length, all);
        end = Line::cut(a, at + units, length, all);
        if (all == 0) {
            slot = -1;
            return at == 0;
        }
        slot = from == 0 && end == all ? -1 : from > 0 ? 2 * w : 2 * w + 1;
        return true;
    }
    // How many keys row i of the sequence sees (a row past its last: as many as that).
    __device__ __forceinline__ int sees(int i, const PagedArgs& a) const {
        if (i >= rows) i = rows - 1;
        const int n = s.length - s.n + int(unsigned(i) / unsigned(a.r)) + 1;
        return n < 0 ? 0 : n > s.length ? s.length : n;
    }
    __device__ __forceinline__ int64_t out_row(int i, const PagedArgs& a) const {
        const unsigned t = unsigned(i) / unsigned(a.r);
        return int64_t(s.first + t) * a.Hq + hk * a.r + (i - int(t) * a.r);
    }
    template <typename DT>
    __device__ __forceinline__ const DT* query(int i, const PagedArgs& a) const {
        if (i >= rows) return nullptr;
        const unsigned t = unsigned(i) / unsigned(a.r);
        return reinterpret_cast<const DT*>(a.q) + int64_t(s.first + t) * a.qs[0] + (hk * a.r + (i - int(t) * a.r)) * a.qs[1];
    }
    // A row's outputs, four dimensions of them at `d`: to the part, or finished. R: rows of a tile.
    template <typename DT, int R>
    __device__ __forceinline__ void store(int i, int64_t out, int d, f32x4 o, float m, float z, const PagedArgs& a) const {
        if (slot >= 0) {
            const int64_t place = (int64_t(hk) * a.pieces * 2 + slot) * R + i % R;
            *reinterpret_cast<f32x4*>(a.part_acc + place * a.D + d) = o;
            if (d == 0) a.part_ml[place] = float2{m, z};
        } else {
            finish<DT>(out, d, o, m, z, a);
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
    uint64_t at_k, at_v;  // bytes from the key head's begin
    int last;
    bool there;
    __device__ __forceinline__ void of(const PagedArgs& a, int page, int key, int end) {
        const int in_end = (end - 1) & ~(kKeyGroup - 1);
        key = key < in_end ? key : in_end;
        last = end - 1 - key < kKeyGroup - 1 ? end - 1 - key : kKeyGroup - 1;
        there = unsigned(page) < unsigned(a.pages);
        const uint64_t p = there ? page : 0, t = unsigned(key) & ((1u << a.shift) - 1);
        at_k = p * uint64_t(a.ks[0]) + t * uint32_t(a.ks[1]);
        at_v = p * uint64_t(a.vs[0]) + t * uint32_t(a.vs[1]);
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

// Infinite and NaN values of keys that some of the rows do not see: their product with a weight of 0 is NaN. In blocks of such keys they
// count as 0, and are added at the end to the rows that see them.
template <typename DT>
__device__ __forceinline__ bool take_odd(u32x4& w) {  // true: there were some
    uint32_t all = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(DT) == 4) {
            const uint32_t odd = (w[i] & 0x7f800000u) == 0x7f800000u ? ~0u : 0u;
            w[i] &= ~odd;
            all |= odd;
        } else {  // (the top bit of each half whose exponent is all ones)
            const uint32_t odd = ~((~w[i] & 0x7f807f80u) + 0x7fff7fffu) & 0x80008000u;
            w[i] &= ~((odd >> 15) * 0xffffu);
            all |= odd;
        }
    }
    return all != 0;
}
// Where the blocks begin that not all rows see all of; `least`: keys that all rows see.
__device__ __forceinline__ int first_unseen(int from, int least, int keys) { return from + (least > from ? (least - from) / keys * keys : 0); }
// The sum of such values of keys [first, sees), four dimensions at d. (Apart from the products, whose registers a loop over the
// outputs would cost: 1727 us became 1790.)
template <typename DT>
__device__ __forceinline__ f32x4 odd_values(const PagedArgs& a, const PagedItem& it, int first, int sees, int d) {
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int j = first; j < sees; ++j) {
        const int page = a.table[int64_t(it.b) * a.ld_table + (j >> a.shift)];
        if (unsigned(page) >= unsigned(a.pages)) continue;
        const int64_t token = j & ((1 << a.shift) - 1);
        const DT* v = reinterpret_cast<const DT*>(reinterpret_cast<const char*>(a.v) + page * a.vs[0] + token * a.vs[1] + it.hk * a.vs[2]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float value = widen(v[d + e]);
            if ((__float_as_uint(value) & 0x7f800000u) == 0x7f800000u) o[e] += value;
        }
    }
    return o;
}

// Piece w of a key head, tile by tile.
template <bool FEW, int R, class F>
__device__ __forceinline__ void paged_share(const PagedArgs& a, const PagedSeqs& seqs, int w, int hk, F&& tile) {
    PagedLine<FEW, R> line;
    line.plan(a, seqs);
    if (w >= line.pieces) return;
    int x = line.piece(w);
    const int end = line.piece(w + 1);
    PagedItem it;
    it.hk = hk;
    if (!it.find<FEW, R>(a, seqs, x)) return;
    for (;;) {
        const int rest = it.length - it.at, units = rest < end - x ? rest : end - x;
        if (it.take<PagedLine<FEW, R>>(a, w, units)) tile(it);
        x += units;
        if (x >= end || !it.next<FEW, R>(a, seqs)) return;
    }
}

// ------------------------------------------------------------- few rows: keys dealt to waves

// Keys [from, end) of one item, blocks wave, wave + W, ..., by a wave with QT tiles of sixteen rows. True: there were odd values in
// blocks that not all rows see all of.
template <typename DT, int ND, int QT, int W, bool EXACT>
__device__ __forceinline__ bool paged_run(AttnWave<DT, ND, QT, EXACT>& w, const PagedArgs& a, const PagedItem& it, const int (&sees)[QT], int least,
                                          int D, float scale, bf16_t* lds, int wave, int lane) {
    typedef KeyBlock<DT, ND, EXACT> Block;
    constexpr bool kWide = sizeof(DT) == 4;
    constexpr int kKeys = Block::kKeys, KT = kKeys / 16, G = kKeys / kKeyGroup, kVecs = Block::kVecs;
    const int c = lane & 15, g = lane >> 4, end = it.end;
    int j = it.from + wave * kKeys;
    if (j >= end) return false;
    PageNumbers<G> numbers;
    numbers.begin(a.table + int64_t(it.b) * a.ld_table, j, W * kKeys, end, a.shift, [](int x) { return kKeyGroup * x; });
    Block b;
    KeyGroup at[G];
    const uint32_t sk = uint32_t(a.ks[1]), sv = uint32_t(a.vs[1]);
    const char *keys = reinterpret_cast<const char*>(a.k) + it.hk * a.ks[2], *values = reinterpret_cast<const char*>(a.v) + it.hk * a.vs[2];
    auto aim = [&](int n, int key) {  // block n of the wave, at `key`
#pragma unroll
        for (int x = 0; x < G; ++x) at[x].of(a, numbers.get(n, x), key + kKeyGroup * x, end);
    };
    auto row = [&](int r, const KeyGroup& k) { return uint32_t(r < k.last ? r : k.last); };
    auto load_k = [&]() {
        constexpr int kSteps = ND / Block::kKRows;
#pragma unroll
        for (int kt = 0; kt < Block::kKRows; ++kt) {
            const char* base = keys + at[kt].at_k;
            const uint32_t first = row(c, at[kt]) * sk + 16u * g;
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
            const char* base = values + at[0].at_v;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t first = row(4 * g + i, at[0]) * sv + 4u * c;
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
            // (whole rows, past the caches, which keys in pieces of 64 bytes need: 64 sequences of 4096 keys, 8 key heads of 128 dimensions:
            // 180 us, else 197; of 64 dimensions 91 and 113; but four sequences on the same pages each 103 and 91, sixteen 91 and 84)
#pragma unroll
            for (int i = 0; i < ND; ++i) {
                constexpr int kRows = 64 / kVecs;  // of a load
                const KeyGroup& k = at[i * kRows / kKeyGroup];
                const int r = (lane / kVecs + i * kRows) % kKeyGroup, piece = lane % kVecs;
                const uint32_t o = row(r, k) * sv + 16u * (EXACT || 8 * piece < D ? piece : D / 8 - 1);
                b.v[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(values + k.at_v + o));
            }
        }
    };
    auto missing = [&]() {
        uint32_t m = 0;
#pragma unroll
        for (int x = 0; x < G; ++x) m |= at[x].there ? 0u : 1u << x;
        return m;
    };
    bool odd = false;
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
        if (here + kKeys > least) {
#pragma unroll
            for (int i = 0; i < ND; ++i) odd |= take_odd<DT>(b.v[i]);
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
        if (!more) return __any(odd);
    }
}

// Sequences of few rows: four waves on the same rows, each with keys of its own.
template <typename DT, int ND, int QT, bool EXACT>
__device__ __forceinline__ void paged_few_tile(const PagedArgs& a, const PagedItem& it, char* mem, float (*s_m)[kTileRows], float (*s_l)[kTileRows]) {
    constexpr int W = kAttnWaves, R = QT * kTileRows;
    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int D = EXACT ? 16 * ND : int(a.D);
    AttnWave<DT, ND, QT, EXACT> w;
    w.clear();
    int sees[QT];
#pragma unroll
    for (int x = 0; x < QT; ++x) {
        w.load_query(x, it.query<DT>(kTileRows * x + c, a), D, query_sign<DT>(a.scale2), lane);
        sees[x] = it.sees(kTileRows * x + c, a);
        if (sees[x] > it.end) sees[x] = it.end;
    }
    int least = it.sees(0, a);
    if (least > it.end) least = it.end;
    const bool odd = paged_run<DT, ND, QT, W, EXACT>(w, a, it, sees, least, D, score_scale(a.scale2), reinterpret_cast<bf16_t*>(mem) + wave * 32 * (16 * ND + 16), wave, lane);

    const int first = __syncthreads_or(odd) ? first_unseen(it.from, least, KeyBlock<DT, ND, EXACT>::kKeys) : it.end;

    // the waves join, sixteen rows at a time
    float* join = reinterpret_cast<float*>(mem);
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
            if (first < it.end) {
                const int seen = it.sees(row0 + i, a);
                o += odd_values<DT>(a, it, first, seen < it.end ? seen : it.end, d);
            }
            it.template store<DT, R>(row0 + i, it.out_row(row0 + i, a), d, o, m, z, a);
        }
    }
}

// The sequence and key head of a workgroup. False: there is none, as the grid of more than 2^20 workgroups is a multiple of that many.
// (The pairs are below 2^31, and so are the grid's workgroups: one division in 32 bits. Past the last sequence b is the last: what is read of
// it does not wait for the comparison.)
__host__ __device__ __forceinline__ bool whole_tile(int block, int B, int Hkv, int& b, int& hk) {
    b = block / Hkv;
    hk = block - b * Hkv;
    const bool is = b < B;
    b = is ? b : B - 1;
    return is;
}

// Whole tiles. 64 sequences of 1024 keys as below: 42 us (6.3 TB/s); 8 of 300 float32 keys, one head of 64 dimensions: 9.3 us, all of it
// latency (lengths, page numbers, five blocks of keys a wave one after the other).
template <typename DT, int ND, int QT, bool EXACT>
__global__ __launch_bounds__(kAttnWaves * kWave) void paged_few_kernel(PagedArgs a) {
    __shared__ __attribute__((aligned(16))) char s_mem[attn_lds<DT, ND, kAttnWaves>()];
    __shared__ float s_m[kAttnWaves][kTileRows], s_l[kAttnWaves][kTileRows];
    int b;
    PagedItem it;
    const bool is = whole_tile(int(grid_row()), a.B, a.Hkv, b, it.hk);
    if (it.only<QT * kTileRows>(a, b) && is && it.take<PagedLine<true, QT * kTileRows>>(a, 0, it.length))
        paged_few_tile<DT, ND, QT, EXACT>(a, it, s_mem, s_m, s_l);
}

// The same with a wave on each piece of the line: no barrier, and nothing to join within the workgroup. One wave a SIMD, with all of
// its registers for keys on their way. 64 sequences of 5120 keys, 8 key heads of 128 dimensions, bfloat16, 4 query heads
// to a key head: 235 us for one new token each (5.7 TB/s); of up to 8192 keys 238 us for 1.35 GB.
template <typename DT, int ND, int QT, bool EXACT>
__global__ __launch_bounds__(kAttnWaves * kWave) __attribute__((amdgpu_waves_per_eu(1, 1))) void paged_solo_kernel(PagedArgs a) {
    constexpr int R = QT * kTileRows;
    __shared__ __attribute__((aligned(16))) char s_mem[sizeof(DT) == 2 ? kAttnWaves * 32 * (16 * ND + 16) * 2 : 16];
    const int block = int(grid_row()), lane = threadIdx.x & 63, c = lane & 15, g4 = lane >> 4;
    const int wave = agreed(int(threadIdx.x >> 6));
    const int D = EXACT ? 16 * ND : int(a.D);
    const PagedSeqs seqs(a);
    paged_share<true, R>(a, seqs, block / a.Hkv * kAttnWaves + wave, block % a.Hkv, [&](const PagedItem& it) {
        AttnWave<DT, ND, QT, EXACT> w;
        w.clear();
        int sees[QT];
#pragma unroll
        for (int x = 0; x < QT; ++x) {
            w.load_query(x, it.query<DT>(kTileRows * x + c, a), D, query_sign<DT>(a.scale2), lane);
            sees[x] = it.sees(kTileRows * x + c, a);
            if (sees[x] > it.end) sees[x] = it.end;
        }
        int least = it.sees(0, a);
        if (least > it.end) least = it.end;
        const bool odd = paged_run<DT, ND, QT, 1, EXACT>(w, a, it, sees, least, D, score_scale(a.scale2), reinterpret_cast<bf16_t*>(s_mem) + wave * 32 * (16 * ND + 16), 0, lane);
        const int first = odd ? first_unseen(it.from, least, KeyBlock<DT, ND, EXACT>::kKeys) : it.end;
#pragma unroll
        for (int x = 0; x < QT; ++x) {
            float l = w.l[x];
            l += __shfl_xor(l, 16);
            l += __shfl_xor(l, 32);
            const int row = kTileRows * x + c;
            if (row >= it.rows) continue;
            const int64_t out = it.out_row(row, a);
#pragma unroll
            for (int t = 0; t < ND; ++t)
                if (EXACT || 16 * t + 4 * g4 < D) {
                    if (first < it.end) w.acc[x][t] += odd_values<DT>(a, it, first, sees[x], 16 * t + 4 * g4);
                    it.store<DT, R>(row, out, 16 * t + 4 * g4, w.acc[x][t], w.m[x], l, a);
                }
        }
    });
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
    // (rows of LDS longer by a few banks than they are: bfloat16 keys by 32 bytes 1694 us, by 16 1716, by none 2353)
    static constexpr int kKRow = 16 * ND + (kWide ? 4 : 16);
    static constexpr int kVRow = 16 * ND + (kWide ? 4 : 16);
    static constexpr int kPieces = kKeys * kVecs / (W * kWave);
    static constexpr int kHalf = kKeys * (kKRow + kVRow);
    static constexpr size_t kLds = size_t(2 * kHalf) * sizeof(DT);
    static constexpr int kGroups = kKeys / kKeyGroup;

    static __device__ __forceinline__ bool run(AttnWave<DT, ND, QT, EXACT>& w, const PagedArgs& a, const PagedItem& it, const int (&sees)[QT], int least,
                                               int least_of_all, int most, int D, float scale, DT* lds, uint32_t (*s_out)[4], int tid) {
        const int lane = tid & 63, c = lane & 15, g = lane >> 4, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        constexpr int KT = kKeys / 16;
        const int from = it.from, end = it.end;
        if (from >= end) return false;
        // piece i of a wave's lanes: rows (64 wave + 64 W i) / kVecs ... of a block, all in one group
        auto first_row = [&](int i) { return (64 * wave + 64 * W * i) / kVecs; };
        PageNumbers<kPieces> numbers;
        numbers.begin(a.table + int64_t(it.b) * a.ld_table, from, kKeys, end, a.shift,
                      [&](int i) { return first_row(i) / kKeyGroup * kKeyGroup; });
        const uint32_t sk = uint32_t(a.ks[1]), sv = uint32_t(a.vs[1]);
        const char *keys = reinterpret_cast<const char*>(a.k) + it.hk * a.ks[2], *values = reinterpret_cast<const char*>(a.v) + it.hk * a.vs[2];
        u32x4 k[kPieces], v[kPieces];
        uint32_t out = 0;  // pieces without a page
        auto load = [&](int n) {
            const int j = from + n * kKeys;
            out = 0;
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                KeyGroup at;
                at.of(a, numbers.get(n, i), j + first_row(i) / kKeyGroup * kKeyGroup, end);
                out |= at.there ? 0u : 1u << i;
                const int piece = lane % kVecs, r = (first_row(i) + lane / kVecs) % kKeyGroup;
                const uint32_t row = r < at.last ? r : at.last, d = 16u * (EXACT || kVec * piece < D ? piece : D / kVec - 1);
                k[i] = *reinterpret_cast<const u32x4*>(keys + at.at_k + row * sk + d);
                v[i] = *reinterpret_cast<const u32x4*>(values + at.at_v + row * sv + d);
            }
        };
        bool odd = false;
        auto put = [&](int n) {
            const int turn = n & 1;
            DT* half = lds + turn * kHalf;
            if (__builtin_expect(from + (n + 1) * kKeys > least_of_all, 0)) {
#pragma unroll
                for (int i = 0; i < kPieces; ++i) odd |= take_odd<DT>(v[i]);
            }
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
            if (n + 1 < blocks) put(n + 1);
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
                // (the next keys' operand is on its way while this one's products run)
                bf16x8 k8[2][ND / 2];
                auto ask = [&](int kt) {
#pragma unroll
                    for (int d = 0; d < ND / 2; ++d) k8[kt & 1][d] = *reinterpret_cast<const bf16x8*>(lk + (16 * kt + c) * kKRow + 32 * d + 8 * g);
                };
                ask(0);
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) {
                    if (kt + 1 < KT) ask(kt + 1);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int d = 0; d < ND / 2; ++d)
#pragma unroll
                        for (int x = 0; x < QT; ++x)
                            s[x][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k8[kt & 1][d], __builtin_bit_cast(bf16x8, w.q[x][d]), s[x][kt], 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
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
                constexpr int kStep = 4;  // dimensions' tiles asked for at a time
                bf16x8 p[QT][KT / 2], v8[2][kStep];
#pragma unroll
                for (int h = 0; h < KT / 2; ++h)
#pragma unroll
                    for (int x = 0; x < QT; ++x) p[x][h] = weights_operand(s[x][2 * h], s[x][2 * h + 1]);
                const DT* base = lv + (4 * g + (c >> 2)) * kVRow + 4 * (c & 3);
                auto ask = [&](int n) {
#pragma unroll
                    for (int i = 0; i < kStep; ++i) {
                        const int t = n % (ND / kStep) * kStep + i, h = n / (ND / kStep);
                        v8[n & 1][i] = values_operand(reinterpret_cast<const bf16_t*>(base + 32 * h * kVRow + 16 * t), kVRow);
                    }
                };
                ask(0);
                constexpr int kSteps = ND / kStep * (KT / 2);
#pragma unroll
                for (int n = 0; n < kSteps; ++n) {
                    if (n + 1 < kSteps) ask(n + 1);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int i = 0; i < kStep; ++i)
#pragma unroll
                        for (int x = 0; x < QT; ++x) {
                            const int t = n % (ND / kStep) * kStep + i;
                            w.acc[x][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v8[n & 1][i], p[x][n / (ND / kStep)], w.acc[x][t], 0, 0, 0);
                        }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        return __syncthreads_or(odd);
    }
};

template <typename DT, int ND, int QT, int W, bool EXACT>
__device__ __forceinline__ void paged_many_tile(const PagedArgs& a, const PagedItem& it, char* mem, uint32_t (*s_out)[4]) {
    constexpr int R = W * QT * kTileRows;
    typedef PagedShared<DT, ND, QT, W, EXACT> Shared;
    const int tid = threadIdx.x, lane = tid & 63, c = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int D = EXACT ? 16 * ND : int(a.D);
    const int row0 = it.tile * R + wave * QT * kTileRows;
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
    int least_of_all = it.sees(it.tile * R, a);
    if (least_of_all > it.end) least_of_all = it.end;
    const bool odd = Shared::run(w, a, it, sees, least, least_of_all, most, D, score_scale(a.scale2), reinterpret_cast<DT*>(mem), s_out, tid);
    const int first = odd ? first_unseen(it.from, least_of_all, Shared::kKeys) : it.end;
    const int g4 = lane >> 4;
#pragma unroll
    for (int x = 0; x < QT; ++x) {
        float l = w.l[x];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        const int row = row0 + x * kTileRows + c;
        if (row >= it.rows) continue;
        const int64_t out = it.out_row(row, a);
#pragma unroll
        for (int t = 0; t < ND; ++t)
            if (EXACT || 16 * t + 4 * g4 < D) {
                if (first < it.end) w.acc[x][t] += odd_values<DT>(a, it, first, sees[x], 16 * t + 4 * g4);
                it.template store<DT, R>(row, out, 16 * t + 4 * g4, w.acc[x][t], w.m[x], l, a);
            }
    }
}

// Two waves a SIMD; a workgroup a CU in the largest form (256 rows). 4 sequences of 16384 keys, the last 2048 of them new, 32 query heads on
// 8 key heads of 128 dimensions, bfloat16: 2300 us, 890 TFLOP/s; of lengths in between 820 to 870.
template <typename DT, int ND, int QT, int W, bool EXACT>
__global__ __launch_bounds__(W * kWave) __attribute__((amdgpu_waves_per_eu(ND > 8 ? 1 : 2, ND > 8 ? 1 : 2))) void paged_many_kernel(PagedArgs a) {
    constexpr int R = W * QT * kTileRows;
    __shared__ __attribute__((aligned(16))) char s_mem[PagedShared<DT, ND, QT, W, EXACT>::kLds];
    __shared__ uint32_t s_out[2][4];  // groups without a page, of each half
    const int block = int(grid_row());
    const PagedSeqs seqs(a);
    paged_share<false, R>(a, seqs, block / a.Hkv, block % a.Hkv, [&](const PagedItem& it) {
        paged_many_tile<DT, ND, QT, W, EXACT>(a, it, s_mem, s_out);
        __syncthreads();  // (what is in LDS has been read)
    });
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

// Joins the parts of the tiles that are cut, o = sum_i 2^(m_i - m) o_i / sum_i 2^(m_i - m) l_i: a tile by the workgroups of the
// first cut in it, each with kJoinRows of its rows, D / 4 lanes (four dimensions each) a row; where that leaves lanes, several
// groups of them on parts in turn. Bound by latency, the plan first (with 8 rows a workgroup, and twice as many plans, 159 us where
// it took 156 in all, with 4 167). 64 sequences, 20 rows: 16 us of 147; 4 of 2048 tokens 36 of 1720.
constexpr int kJoinRows = 16;
template <typename DT, bool FEW, int R>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedArgs a) {
    __shared__ f32x4 s_o[256];
    __shared__ float s_z[256];
    int64_t item = grid_row();
    const int block = int(item % (R / kJoinRows));
    item /= R / kJoinRows;
    const int hk = int(item % a.Hkv), w0 = int(item / a.Hkv);  // the cut after piece w0
    const PagedSeqs seqs(a);
    PagedLine<FEW, R> line;
    line.plan(a, seqs);
    if (w0 + 1 >= line.pieces) return;
    PagedItem it;
    it.hk = hk;
    const int x = line.piece(w0 + 1);
    if (!it.find<FEW, R>(a, seqs, x) || it.at == 0 || it.all == 0) return;
    const int tile = x - it.at;  // its begin on the line
    if (line.piece(w0) > tile) return;  // (a piece before ends in it, too)
    const int first_row = it.tile * R + block * kJoinRows;
    if (first_row >= it.rows) return;
    int parts = 2;
    while (w0 + parts < line.pieces && line.piece(w0 + parts) < tile + it.length) ++parts;
    // nothing to join where one of them has all of the keys
    bool alone = false;
    for (int i = int(threadIdx.x) & 63; i < parts; i += kWave) {
        const int y = line.piece(w0 + i), z = line.piece(w0 + i + 1);
        alone |= line.cut(a, y > tile ? y - tile : 0, it.length, it.all) == 0 && line.cut(a, z - tile, it.length, it.all) == it.all;
    }
    if (__any(alone)) return;
    const int lanes = a.D / 4, fit = 256 / lanes;
    const int count = it.rows - first_row < kJoinRows ? it.rows - first_row : kJoinRows;
    const int at_once = count < fit ? count : fit, groups = fit / at_once;
    const int which = int(threadIdx.x) / lanes, d = 4 * (int(threadIdx.x) % lanes);
    for (int r0 = 0; r0 < count; r0 += at_once) {
        const int row = r0 + which % at_once, group = which / at_once;
        const bool on = group < groups && row < count;
        auto place = [&](int i) {
            const int w = w0 + i;
            const int y = line.piece(w);
            const bool later = y > tile && line.cut(a, y - tile, it.length, it.all) > 0;
            return (int64_t(hk) * a.pieces * 2 + 2 * w + (later ? 0 : 1)) * R + block * kJoinRows + row;
        };
        float m = kNegInf, z = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
        if (on) {
            for (int i = 0; i < parts; ++i) m = fmaxf(m, a.part_ml[place(i)].x);
            for (int i = group; i < parts; i += groups) {
                const float2 ml = a.part_ml[place(i)];
                const float keep = ml.x == kNegInf ? 0.f : exp2_fast(ml.x - m);
                z = fmaf(keep, ml.y, z);
                o += keep * *reinterpret_cast<const f32x4*>(a.part_acc + place(i) * a.D + d);
            }
        }
        if (groups > 1) {
            __syncthreads();
            s_o[threadIdx.x] = o;
            s_z[threadIdx.x] = z;
            __syncthreads();
            if (on && group == 0)
                for (int i = 1; i < groups; ++i) {
                    o += s_o[threadIdx.x + i * at_once * lanes];
                    z += s_z[threadIdx.x + i * at_once * lanes];
                }
        }
        if (on && group == 0) {
            PagedItem::finish<DT>(it.out_row(first_row + row, a), d, o, m, z, a);
        }
    }
}

// ------------------------------------------------------------- writing

struct PagedWriteArgs {
    PagedArgs at;  // (q: the new keys, o: nothing)
    const void *k_new, *v_new;
    char *k, *v;
    int64_t kn[2], vn[2];
    int32_t pieces;  // 16-byte pieces of a head
};

// A token a wave: its keys and values are on their way before its place is known. Bound by memory: 16384 tokens of 8 heads of
// 128 dimensions, bfloat16, 134 MB read and written in 23 us (5.8 TB/s); the smallest calls by the launch, 3.7 us.
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
    char* to_k = a.k + page * a.at.ks[0] + in * a.at.ks[1];
    char* to_v = a.v + page * a.at.vs[0] + in * a.at.vs[1];
    for (int at = lane; at < all; at += U * kWave) {
        if (at != lane) load(at);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = at + u * kWave, h = i / a.pieces, d = i % a.pieces * kVec;
            if (i < all) {
                *reinterpret_cast<u32x4*>(to_k + h * a.at.ks[2] + d * int(sizeof(DT))) = x[u];
                *reinterpret_cast<u32x4*>(to_v + h * a.at.vs[2] + d * int(sizeof(DT))) = y[u];
            }
        }
    }
}

}  // namespace rlcs
