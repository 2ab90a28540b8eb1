// Entry points of a cache's pages.
#include "rlcs_dispatch.h"
#include "rlcs_pages.h"

using namespace rlcs;
using namespace rlcs::host;

namespace {

constexpr int64_t kMaxGroups = 2048;
// Calls of at most this many table entries, and pages that fit in LDS, run as one workgroup. (Resize, one call after another: 256
// pages and 128 entries 4.8 us, in four kernels 11.5; 4096 of both 9.2 and 13.6; 8192 of both 13.3 and 12.9; 8192 and 16384 13.2 and
// 10.7. Fork, resize and copy of 2048 pages and 8704 entries: 19.6 and 31.4.)
constexpr int64_t kLdsEntries = 12288;

bool good_page(int64_t page) { return page >= 16 && page <= 65536 && (page & (page - 1)) == 0; }
int shift_of(int64_t page) {
    int s = 0;
    while ((int64_t(1) << s) < page) ++s;
    return s;
}

struct PagesSpace {
    size_t needs, bits, chunk, before, total, bytes;
};
PagesSpace space_of(int64_t B, int64_t pages) {
    PagesSpace s{};
    auto take = [&](size_t bytes) {
        const size_t at = s.bytes;
        s.bytes += (bytes + 15) / 16 * 16;
        return at;
    };
    const int64_t words = (pages + kWordPages - 1) / kWordPages, chunks = (pages + kChunkPages - 1) / kChunkPages;
    s.needs = take(size_t(B) * sizeof(PageNeed));
    s.bits = take(size_t(words) * 8);
    s.chunk = take(size_t(chunks) * 4);
    s.before = take(size_t(words) * 4);
    s.total = take(16);
    return s;
}

// Sizes and pointers that the three calls share; `need`: pointers that must be there where there is a table.
rlcs_status prepare(PagesArgs& a, int64_t B, int64_t W, int64_t pages, int64_t page, void* ws, size_t ws_bytes,
                    std::initializer_list<const void*> need) {
    if (B < 0 || W < 0 || pages < 0 || !good_page(page)) return RLCS_ERR_INVALID_ARG;
    if (B > INT32_MAX || W > kMaxT / page || pages > kMaxT || (W > 0 && B > INT32_MAX / W)) return RLCS_ERR_INVALID_ARG;
    for (const void* p : need) {
        if (!p) return RLCS_ERR_INVALID_ARG;
        if (!aligned(p, 4)) return RLCS_ERR_INVALID_ARG;
    }
    a.B = int32_t(B); a.W = int32_t(W); a.pages = int32_t(pages); a.shift = shift_of(page);
    const PagesSpace s = space_of(B, pages);
    if (!ws || ws_bytes < s.bytes) return RLCS_ERR_WORKSPACE;
    if (!aligned(ws, 16)) return RLCS_ERR_INVALID_ARG;
    char* w = static_cast<char*>(ws);
    a.needs = reinterpret_cast<PageNeed*>(w + s.needs);
    a.bits = reinterpret_cast<uint64_t*>(w + s.bits);
    a.chunk = reinterpret_cast<int32_t*>(w + s.chunk);
    a.before = reinterpret_cast<int32_t*>(w + s.before);
    a.total = reinterpret_cast<int32_t*>(w + s.total);
    return RLCS_OK;
}

bool small(const PagesArgs& a) { return a.pages <= kLdsPages && int64_t(a.B) * a.W <= kLdsEntries && a.B <= kOffsetsInLds; }
template <PagesCall C>
void whole(const PagesArgs& a, hipStream_t s) {
    hipLaunchKernelGGL((pages_lds_kernel<C>), dim3(1), dim3(kPagesSmall), 0, s, a);
}
template <PagesPhase PH>
void phase(const PagesArgs& a, int64_t lanes, hipStream_t s, int extra = 0) {
    int64_t groups = (lanes + kPagesGroup - 1) / kPagesGroup;
    if (groups > kMaxGroups) groups = kMaxGroups;
    if (groups < 1) groups = 1;
    hipLaunchKernelGGL((pages_phase_kernel<PH>), dim3(unsigned(groups + extra)), dim3(kPagesGroup), 0, s, a);
}
int64_t entries(const PagesArgs& a) { return int64_t(a.B) * a.W; }
int64_t counting(const PagesArgs& a) { return (int64_t(a.pages) + kChunkPages - 1) / kChunkPages * kWave; }
int64_t most_of(int64_t x, int64_t y) { return x > y ? x : y; }

rlcs_status launched() { return hipGetLastError() == hipSuccess ? RLCS_OK : RLCS_ERR_LAUNCH; }

template <typename V>
rlcs_status copy_pages(PagesCopyArgs a, hipStream_t s) {
    const int64_t per = int64_t(kCopyLanes) * kCopyVecs * int64_t(sizeof(V));
    a.pieces = (a.page_bytes + per - 1) / per;
    if (a.layers > (int64_t(1) << 40) / a.pieces || a.n > (int64_t(1) << 40) / (a.pieces * a.layers)) return RLCS_ERR_INVALID_ARG;
    if (a.n * a.layers * a.pieces > (int64_t(1) << 35)) return RLCS_ERR_INVALID_ARG;
    hipLaunchKernelGGL((pages_copy_kernel<V>), row_grid(a.n * a.layers * a.pieces), dim3(kCopyLanes), 0, s, a);
    return launched();
}

}  // namespace

extern "C" {

size_t rlcs_workspace_size_pages(int64_t B, int64_t pages) {
    if (B < 0 || pages < 0 || B > INT32_MAX || pages > kMaxT) return 0;
    return space_of(B, pages).bytes;
}

rlcs_status rlcs_pages_fork(const int32_t* table, const int32_t* length, const int32_t* refs,
                            const int32_t* parent, int32_t* table_out, int32_t* length_out,
                            int32_t* refs_out, int64_t B, int64_t W, int64_t pages, int64_t page,
                            void* ws, size_t ws_bytes, rlcs_stream_t stream) {
    PagesArgs a{};
    if (B < 0 || W < 0 || pages < 0 || !good_page(page)) return RLCS_ERR_INVALID_ARG;
    if (B == 0 || W == 0 || pages == 0) return RLCS_OK;
    const rlcs_status st = prepare(a, B, W, pages, page, ws, ws_bytes, {table, length, refs, parent, table_out, length_out, refs_out});
    if (st != RLCS_OK) return st;
    if (table_out == table || length_out == length) return RLCS_ERR_INVALID_ARG;
    a.table = table; a.length = length; a.refs = refs; a.wanted = parent;
    a.table_out = table_out; a.length_out = length_out; a.refs_out = refs_out;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (small(a)) {
        whole<kCallFork>(a, s);
    } else {
        if (refs_out != refs) phase<kCopyRefs>(a, pages, s);
        phase<kFork>(a, entries(a), s);
    }
    return launched();
}

rlcs_status rlcs_pages_resize(const int32_t* table, const int32_t* length, const int32_t* refs,
                              const int32_t* new_length, int32_t* table_out, int32_t* length_out,
                              int32_t* refs_out, int32_t* moves, int64_t B, int64_t W,
                              int64_t pages, int64_t page, void* ws, size_t ws_bytes,
                              rlcs_stream_t stream) {
    PagesArgs a{};
    if (B < 0 || W < 0 || pages < 0 || !good_page(page)) return RLCS_ERR_INVALID_ARG;
    if (B == 0 || W == 0 || pages == 0) return RLCS_OK;
    const rlcs_status st = prepare(a, B, W, pages, page, ws, ws_bytes, {table, length, refs, new_length, table_out, length_out, refs_out, moves});
    if (st != RLCS_OK) return st;
    a.table = table; a.length = length; a.refs = refs; a.wanted = new_length;
    a.table_out = table_out; a.length_out = length_out; a.refs_out = refs_out; a.moves = moves;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (small(a)) {
        whole<kCallResize>(a, s);
    } else {
        if (refs_out != refs) phase<kCopyRefs>(a, pages, s);
        phase<kRelease>(a, entries(a), s);
        phase<kCountFree>(a, counting(a), s, 1);
        phase<kAssign>(a, most_of(counting(a), B), s);
    }
    return launched();
}

rlcs_status rlcs_pages_compact(const int32_t* table, const int32_t* refs, int32_t* table_out,
                               int32_t* refs_out, int32_t* moves, int32_t* count, int64_t B,
                               int64_t W, int64_t pages, void* ws, size_t ws_bytes,
                               rlcs_stream_t stream) {
    PagesArgs a{};
    if (B < 0 || W < 0 || pages < 0) return RLCS_ERR_INVALID_ARG;
    if (pages == 0) return RLCS_OK;
    const rlcs_status st = prepare(a, B, W, pages, 16, ws, ws_bytes, {refs, refs_out, count});
    if (st != RLCS_OK) return st;
    if (B > 0 && W > 0 && (!table || !table_out)) return RLCS_ERR_INVALID_ARG;
    if (pages > 1 && !moves) return RLCS_ERR_INVALID_ARG;
    for (const void* p : {static_cast<const void*>(table), static_cast<const void*>(table_out), static_cast<const void*>(moves)})
        if (p && !aligned(p, 4)) return RLCS_ERR_INVALID_ARG;
    a.table = table; a.refs = refs; a.table_out = table_out; a.refs_out = refs_out; a.moves = moves; a.count = count;
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (small(a)) {
        whole<kCallCompact>(a, s);
    } else {
        phase<kCountUsed>(a, counting(a), s);
        phase<kPlanMoves>(a, most_of(counting(a), pages / 8), s);
        phase<kRenumber>(a, most_of(entries(a), pages), s);
    }
    return launched();
}

rlcs_status rlcs_pages_copy(void* cache, const int32_t* moves, int64_t n, int64_t layers,
                            int64_t pages, int64_t layer_stride, int64_t page_stride,
                            int64_t page_bytes, rlcs_stream_t stream) {
    if (n < 0 || layers < 0 || pages < 0 || page_bytes < 0 || layer_stride < 0 || page_stride < 0) return RLCS_ERR_INVALID_ARG;
    if (n == 0 || layers == 0 || pages == 0 || page_bytes == 0) return RLCS_OK;
    if (!cache || !moves || !aligned(moves, 4)) return RLCS_ERR_INVALID_ARG;
    if (pages > kMaxT || layers > INT32_MAX || n > INT32_MAX) return RLCS_ERR_INVALID_ARG;
    // distinct (layer, page) are distinct memory, all of it within 63 bits
    const int64_t most = INT64_MAX / 4;
    if (page_bytes > most || (pages > 1 && page_stride > most / pages) || (layers > 1 && layer_stride > most / layers)) return RLCS_ERR_INVALID_ARG;
    const int64_t all_pages = (pages - 1) * page_stride + page_bytes, all_layers = (layers - 1) * layer_stride + page_bytes;
    if (pages > 1 && page_stride < page_bytes) return RLCS_ERR_INVALID_ARG;
    if (layers > 1 && layer_stride < all_pages && !(layer_stride >= page_bytes && (pages == 1 || page_stride >= all_layers))) return RLCS_ERR_INVALID_ARG;
    PagesCopyArgs a{static_cast<char*>(cache), moves, n, layers, pages, layer_stride, page_stride, page_bytes, 0};
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    auto fits = [&](int64_t v) {
        return aligned(cache, size_t(v)) && page_bytes % v == 0 && (pages == 1 || page_stride % v == 0) && (layers == 1 || layer_stride % v == 0);
    };
    if (fits(16)) return copy_pages<u32x4>(a, s);
    if (fits(4)) return copy_pages<uint32_t>(a, s);
    return copy_pages<uint8_t>(a, s);
}

}  // extern "C"
