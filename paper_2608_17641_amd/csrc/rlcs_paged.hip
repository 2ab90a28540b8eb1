// Entry points of attention over a paged cache and of writing into it.
#include "rlcs_paged.h"
#include "rlcs_dispatch.h"

#include <cmath>

using namespace rlcs;
using namespace rlcs::host;

namespace {

constexpr int64_t kMaxHeadDim = 256;
constexpr int64_t kMaxTokenStride = int64_t(1) << 24;

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

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
// Whether distinct places are distinct memory, D elements each: each axis steps over all that the ones with smaller steps reach.
bool apart(const int64_t (&sizes)[3], const int64_t* strides, int64_t D) {
    int64_t reach = D;
    bool done[3] = {};
    for (int n = 0; n < 3; ++n) {
        int next = -1;
        for (int i = 0; i < 3; ++i)
            if (!done[i] && sizes[i] > 1 && (next < 0 || strides[i] < strides[next])) next = i;
        if (next < 0) return true;
        if (strides[next] < reach) return false;
        reach += (sizes[next] - 1) * strides[next];
        done[next] = true;
    }
    return true;
}
bool whole_vectors(const int64_t* s, int n, int64_t vec) {
    for (int i = 0; i < n; ++i)
        if (s[i] % vec) return false;
    return true;
}

// Where no sequence can have more keys than this, all are taken whole: no second kernel. (64 sequences of 1024 keys, 8 key
// heads of 128 dimensions, 4 rows: 42 us, in pieces 51; of one to 1024 keys 29 and 35; of 2048 keys 79 and 89, but of one to 2048
// 59 and 54.)
constexpr int64_t kWholeKeys = 1024;
// Tiles of sixteen rows, up to which the rows of a sequence are the first kernel's: two (64 sequences of 4096 bfloat16 keys, 20 rows: 198 us,
// by the second kernel 212; of 64 dimensions 98 and 140; float32, 64 of 2048: 130 and 186; but 8 sequences of 4096 keys, 32 rows: 66 and
// 49). One of more than 128 dimensions, as two do not fit in a wave's registers (192 dimensions: 664 us, by the second 449).
int few_tiles_of(int64_t D) { return D <= 128 ? 2 : 1; }
// Pieces that all keys are dealt out in: as many as the GPU holds at once. Waves of the first kernel, one a SIMD;
// workgroups of the second, one a CU.
constexpr int64_t kPiecesFew = 1024, kPiecesMany = 256;

// Which kernels a call takes, and their parts.
struct PagedPlan {
    bool few, many;
    int few_tiles;       // of sixteen rows, of the first kernel
    int64_t many_rows;   // of a tile of the second: 64, 128 or 256
    int64_t few_pieces, many_pieces;  // a key head
};

// `most_keys`: no sequence has more (0: not known).
bool make_plan(PagedPlan& p, int64_t tokens, int64_t B, int64_t Hq, int64_t Hkv, int64_t D, int64_t max_chunk, bool ragged, bool bf16,
               int64_t most_keys = 0) {
    const int64_t r = Hq / Hkv, most = max_chunk * r;
    p = PagedPlan{};
    const bool whole = most_keys && most_keys <= kWholeKeys;
    p.few_tiles = most <= kTileRows ? 1 : few_tiles_of(D);
    p.few = ragged || most <= p.few_tiles * kTileRows;
    p.many = most > p.few_tiles * kTileRows;
    p.many_rows = D > 128 || tokens * r <= 64 * B ? 64 : bf16 ? 256 : 128;
    p.few_pieces = whole ? 0 : ceil_div(ceil_div(kPiecesFew, Hkv), kAttnWaves) * kAttnWaves;
    p.many_pieces = ceil_div(kPiecesMany, Hkv);
    return B <= INT32_MAX / Hkv && tokens * r / 64 + B <= INT32_MAX / Hkv;
}
size_t part_bytes(int64_t pieces, int64_t rows, int64_t Hkv, int64_t D) { return size_t(Hkv * 2 * pieces * rows) * size_t(4 * D + 8); }
size_t plan_bytes(const PagedPlan& p, int64_t Hkv, int64_t D) {
    const size_t x = p.few ? part_bytes(p.few_pieces, p.few_tiles * kTileRows, Hkv, D) : 0;
    const size_t y = p.many ? part_bytes(p.many_pieces, p.many_rows, Hkv, D) : 0;
    return x > y ? x : y;
}

// Gives a kernel its pieces and their places in the workspace.
void deal(PagedArgs& a, int64_t pieces, int64_t rows, void* ws) {
    a.pieces = int32_t(pieces);
    a.rise = double(rows) / (double(a.r) * double(1 << a.unit));
    a.part_acc = static_cast<float*>(ws);
    a.part_ml = pieces ? reinterpret_cast<float2*>(a.part_acc + int64_t(a.Hkv) * 2 * pieces * rows * a.D) : nullptr;
}

template <typename DT, bool FEW, int R>
void launch_join(const PagedArgs& a, hipStream_t s) {
    if (a.pieces > 1)
        hipLaunchKernelGGL((paged_join_kernel<DT, FEW, R>), row_grid(int64_t(a.pieces - 1) * a.Hkv * (R / kJoinRows)), dim3(256), 0, s, a);
}

template <typename DT, int ND, int QT, bool EXACT>
void launch_few(const PagedArgs& a, hipStream_t s) {
    const dim3 block(kAttnWaves * kWave);
    if (a.pieces == 0) {
        hipLaunchKernelGGL((paged_few_kernel<DT, ND, QT, EXACT>), row_grid(int64_t(a.B) * a.Hkv), block, 0, s, a);
    } else {
        hipLaunchKernelGGL((paged_solo_kernel<DT, ND, QT, EXACT>), row_grid(int64_t(a.pieces / kAttnWaves) * a.Hkv), block, 0, s, a);
        launch_join<DT, true, QT * kTileRows>(a, s);
    }
}
template <typename DT, int ND, int QT>
void launch_few(const PagedArgs& a, hipStream_t s) {
    if (a.D == 16 * ND) launch_few<DT, ND, QT, true>(a, s);
    else launch_few<DT, ND, QT, false>(a, s);
}
template <typename DT, int ND, int QT, int W>
void launch_many(const PagedArgs& a, hipStream_t s) {
    constexpr int64_t R = W * QT * kTileRows;
    const dim3 grid = row_grid(int64_t(a.pieces) * a.Hkv), block(W * kWave);
    if (a.D == 16 * ND) hipLaunchKernelGGL((paged_many_kernel<DT, ND, QT, W, true>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((paged_many_kernel<DT, ND, QT, W, false>), grid, block, 0, s, a);
    launch_join<DT, false, R>(a, s);
}

template <typename DT, int ND>
rlcs_status run_paged(PagedArgs a, const PagedPlan& p, void* ws, hipStream_t s) {
    if (p.few) {
        deal(a, p.few_pieces, p.few_tiles * kTileRows, ws);
        if constexpr (ND <= 8) {
            if (p.few_tiles == 2) launch_few<DT, ND, 2>(a, s);
            else launch_few<DT, ND, 1>(a, s);
        } else {
            launch_few<DT, ND, 1>(a, s);
        }
    }
    if (p.many) {
        deal(a, p.many_pieces, p.many_rows, ws);
        if constexpr (ND > 8) {
            launch_many<DT, ND, 1, 4>(a, s);
        } else {
            if (p.many_rows == 64) launch_many<DT, ND, 1, 4>(a, s);
            else if constexpr (sizeof(DT) == 2) launch_many<DT, ND, 2, 8>(a, s);
            else launch_many<DT, ND, 1, 8>(a, s);
        }
    }
    return hipGetLastError() == hipSuccess ? RLCS_OK : RLCS_ERR_LAUNCH;
}
template <typename DT>
rlcs_status run_paged(const PagedArgs& a, const PagedPlan& p, void* ws, hipStream_t s) {
    return a.D <= 64 ? run_paged<DT, 4>(a, p, ws, s) : a.D <= 128 ? run_paged<DT, 8>(a, p, ws, s) : run_paged<DT, 16>(a, p, ws, s);
}

// The unit of work, in which all of a key head's counts in 31 bits: tiles of 64 rows, of all keys that a table row may hold.
int work_unit(const PagedArgs& a) {
    const double tiles = double(a.tokens) * a.r / 64 + a.B, held = double(a.W) * double(1 << a.shift);
    const double keys = held > double(a.tokens) ? held : double(a.tokens);
    int unit = 6;
    while (unit < 30 && tiles * (kTileWorkMany + 3 + keys / double(1 << unit)) > double(1 << 30)) ++unit;
    return unit;
}

bool good_page(int64_t page) { return page >= 16 && page <= 65536 && (page & (page - 1)) == 0; }
bool good_dim(int64_t D) { return D >= 8 && D <= kMaxHeadDim && D % 8 == 0; }

// What both calls share: the cache, the table and the sequences.
rlcs_status prepare(PagedArgs& a, const int32_t* table, const int32_t* length, const int32_t* q_start, int64_t tokens, int64_t B, int64_t W,
                    int64_t ld_table, int64_t pages, int64_t page, int64_t Hkv, int64_t D, const int64_t* ks, const int64_t* vs, rlcs_dtype dtype) {
    if (!good_page(page) || !good_dim(D) || Hkv < 1) return RLCS_ERR_INVALID_ARG;
    if (tokens > INT32_MAX - (1 << 20) || B > INT32_MAX / 2 || pages > kMaxT || W > kMaxT / page || Hkv > INT32_MAX / D) return RLCS_ERR_INVALID_ARG;
    if (ld_table < W || (B > 1 && ld_table > INT64_MAX / 8 / B)) return RLCS_ERR_INVALID_ARG;
    if (!length || (W && !table)) return RLCS_ERR_INVALID_ARG;
    for (const void* p : {table, length, q_start})
        if (!aligned(p, 4)) return RLCS_ERR_INVALID_ARG;
    if (!q_start && tokens % B) return RLCS_ERR_INVALID_ARG;
    const int64_t vec = 16 / int64_t(dtype_size(dtype));
    if (!whole_vectors(ks, 3, vec) || !whole_vectors(vs, 3, vec)) return RLCS_ERR_INVALID_ARG;
    // (a group's rows lie within 31 bits of bytes of each other)
    if (ks[1] >= kMaxTokenStride || vs[1] >= kMaxTokenStride) return RLCS_ERR_INVALID_ARG;
    if (!reachable({pages, page, Hkv}, ks) || !reachable({pages, page, Hkv}, vs)) return RLCS_ERR_INVALID_ARG;
    a.table = table; a.length = length; a.q_start = q_start;
    a.ld_table = ld_table; a.tokens = tokens;
    a.B = int32_t(B); a.W = int32_t(W); a.pages = int32_t(pages);
    while ((int64_t(1) << a.shift) < page) ++a.shift;
    a.Hkv = int32_t(Hkv); a.D = int32_t(D);
    const int64_t es = int64_t(dtype_size(dtype));
    for (int i = 0; i < 3; ++i) {
        a.ks[i] = ks[i] * es;
        a.vs[i] = vs[i] * es;
    }
    return RLCS_OK;
}

rlcs_paged_layout contiguous(int64_t page, int64_t Hq, int64_t Hkv, int64_t D) {
    const int64_t t = Hkv * D;
    return rlcs_paged_layout{{Hq * D, D}, {t, D}, {t, D}, {page * t, t, D}, {page * t, t, D}};
}

}  // namespace

extern "C" {

size_t rlcs_workspace_size_paged(int64_t tokens, int64_t B, int64_t Hq, int64_t Hkv, int64_t D,
                                 int64_t max_chunk) {
    if (tokens < 1 || B < 1 || Hkv < 1 || Hq < 1 || Hq % Hkv || !good_dim(D) || max_chunk < 0) return 0;
    if (B > INT32_MAX / 2 || Hq > INT32_MAX || tokens > (INT32_MAX - (1 << 20)) / Hq) return 0;
    if (max_chunk == 0 || max_chunk > tokens) max_chunk = tokens;
    size_t most = 0;
    for (const bool bf16 : {false, true})
        for (const bool ragged : {false, true}) {
            PagedPlan p;
            if (!make_plan(p, tokens, B, Hq, Hkv, D, max_chunk, ragged, bf16)) return 0;
            const size_t n = plan_bytes(p, Hkv, D);
            most = n > most ? n : most;
        }
    return most;
}

rlcs_status rlcs_paged_attn(const void* q, const void* k_cache, const void* v_cache,
                            const int32_t* table, const int32_t* length, const int32_t* q_start,
                            void* o, float* lse, int64_t tokens, int64_t B, int64_t W,
                            int64_t ld_table, int64_t pages, int64_t page, int64_t Hq, int64_t Hkv,
                            int64_t D, int64_t max_chunk, const rlcs_paged_layout* layout,
                            float scale, rlcs_dtype dtype, void* ws, size_t ws_bytes,
                            rlcs_stream_t stream) {
    if (tokens < 0 || B < 0 || W < 0 || pages < 0 || page < 0 || Hq < 0 || Hkv < 0 || D < 0 || max_chunk < 0) return RLCS_ERR_INVALID_ARG;
    if (dtype != RLCS_F32 && dtype != RLCS_BF16) return RLCS_ERR_DTYPE;
    if (!std::isfinite(scale)) return RLCS_ERR_INVALID_ARG;
    if (tokens == 0 || B == 0 || Hq == 0 || D == 0) return RLCS_OK;
    if (Hkv < 1 || Hq % Hkv || Hq > INT32_MAX / kMaxHeadDim || tokens > (INT32_MAX - (1 << 20)) / Hq) return RLCS_ERR_INVALID_ARG;
    PagedArgs a{};
    const rlcs_paged_layout at = layout ? *layout : contiguous(page, Hq, Hkv, D);
    const rlcs_status st = prepare(a, table, length, q_start, tokens, B, W, ld_table, pages, page, Hkv, D, at.k_cache, at.v_cache, dtype);
    if (st != RLCS_OK) return st;
    if (!q || !o || (pages && W && (!k_cache || !v_cache))) return RLCS_ERR_INVALID_ARG;
    for (const void* p : {q, k_cache, v_cache, static_cast<const void*>(o)})
        if (!aligned(p, 16)) return RLCS_ERR_INVALID_ARG;
    if (!aligned(lse, 4)) return RLCS_ERR_INVALID_ARG;
    if (!whole_vectors(at.q, 2, 16 / int64_t(dtype_size(dtype))) || !reachable({tokens, Hq}, at.q)) return RLCS_ERR_INVALID_ARG;
    const bool bf16 = dtype == RLCS_BF16;
    if (max_chunk == 0 || max_chunk > tokens) max_chunk = tokens;
    if (!q_start) max_chunk = tokens / B;
    PagedPlan p;
    if (!make_plan(p, tokens, B, Hq, Hkv, D, max_chunk, q_start != nullptr, bf16, W * page)) return RLCS_ERR_INVALID_ARG;
    // (what every call of these sizes may need, though keys taken whole need none)
    if (const size_t need = rlcs_workspace_size_paged(tokens, B, Hq, Hkv, D, max_chunk)) {
        if (!ws || ws_bytes < need) return RLCS_ERR_WORKSPACE;
        if (!aligned(ws, 16)) return RLCS_ERR_INVALID_ARG;
    }
    a.q = q; a.k = k_cache; a.v = v_cache; a.o = o; a.lse = lse;
    a.qs[0] = at.q[0]; a.qs[1] = at.q[1];
    a.Hq = int32_t(Hq); a.r = int32_t(Hq / Hkv);
    a.max_chunk = int32_t(max_chunk);
    a.few_rows = int32_t(p.few_tiles * kTileRows);
    a.unit = work_unit(a);
    a.scale2 = scale * kLog2e;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    return bf16 ? run_paged<bf16_t>(a, p, ws, s) : run_paged<float>(a, p, ws, s);
}

rlcs_status rlcs_paged_write(const void* k, const void* v, void* k_cache, void* v_cache,
                             const int32_t* table, const int32_t* length, const int32_t* q_start,
                             int64_t tokens, int64_t B, int64_t W, int64_t ld_table, int64_t pages,
                             int64_t page, int64_t Hkv, int64_t D,
                             const rlcs_paged_layout* layout, rlcs_dtype dtype,
                             rlcs_stream_t stream) {
    if (tokens < 0 || B < 0 || W < 0 || pages < 0 || page < 0 || Hkv < 0 || D < 0) return RLCS_ERR_INVALID_ARG;
    if (dtype != RLCS_F32 && dtype != RLCS_BF16) return RLCS_ERR_DTYPE;
    if (tokens == 0 || B == 0 || W == 0 || pages == 0 || Hkv == 0 || D == 0) return RLCS_OK;
    PagedWriteArgs a{};
    const rlcs_paged_layout at = layout ? *layout : contiguous(page, 1, Hkv, D);
    const rlcs_status st = prepare(a.at, table, length, q_start, tokens, B, W, ld_table, pages, page, Hkv, D, at.k_cache, at.v_cache, dtype);
    if (st != RLCS_OK) return st;
    if (!k || !v || !k_cache || !v_cache) return RLCS_ERR_INVALID_ARG;
    for (const void* p : {k, v, static_cast<const void*>(k_cache), static_cast<const void*>(v_cache)})
        if (!aligned(p, 16)) return RLCS_ERR_INVALID_ARG;
    if (!apart({pages, page, Hkv}, at.k_cache, D) || !apart({pages, page, Hkv}, at.v_cache, D)) return RLCS_ERR_INVALID_ARG;
    const int64_t vec = 16 / int64_t(dtype_size(dtype));
    if (!whole_vectors(at.k_new, 2, vec) || !whole_vectors(at.v_new, 2, vec) || !reachable({tokens, Hkv}, at.k_new) ||
        !reachable({tokens, Hkv}, at.v_new))
        return RLCS_ERR_INVALID_ARG;
    a.at.max_chunk = INT32_MAX;
    a.k_new = k; a.v_new = v;
    a.k = static_cast<char*>(k_cache); a.v = static_cast<char*>(v_cache);
    for (int i = 0; i < 2; ++i) {
        a.kn[i] = at.k_new[i];
        a.vn[i] = at.v_new[i];
    }
    a.pieces = int32_t(D / vec);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const dim3 grid = row_grid((tokens + 3) / 4);
    if (dtype == RLCS_BF16) hipLaunchKernelGGL((paged_write_kernel<bf16_t>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((paged_write_kernel<float>), grid, dim3(256), 0, s, a);
    return hipGetLastError() == hipSuccess ? RLCS_OK : RLCS_ERR_LAUNCH;
}

}  // extern "C"
