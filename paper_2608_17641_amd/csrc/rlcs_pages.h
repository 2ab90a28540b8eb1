// The pages of a cache: sequences that take over another's pages, grow, shrink, and a cache whose pages
// move to its front.
//
// refs[p] counts the table entries that hold page p; a page is free if it is 0. Nothing else is kept: a
// page is found by its rank among the free ones, in the order of their numbers, so what a call does follows
// from its inputs alone. Counts change by atomics on integers, whose order does not show.
//
// A call is a few phases, each of which needs all of the one before: barriers of one workgroup that has all counts in LDS, or, of
// more pages or entries than that is good for, kernels of their own. Bound by latency: a phase is one or two dependent loads. (One workgroup with
// its counts in memory, whose atomics pass its cache by, has to fence between phases: 30 us for a resize of 256 pages that takes 5
// in LDS and 12 in four kernels.)
#pragma once

#include "rlcs.h"
#include "rlcs_softmax.h"

namespace rlcs {

constexpr int kWordPages = 64;             // pages whose state is one word of bits
constexpr int kChunkWords = 4;             // words that a wave counts
constexpr int kChunkPages = kWordPages * kChunkWords;
constexpr int kOffsetsInLds = 4096;        // sequences whose offsets a workgroup keeps in LDS
constexpr int kLdsPages = 8192;            // pages whose counts fit in LDS
constexpr int kPagesGroup = 256, kPagesSmall = 1024;  // lanes of a workgroup, and of the only one

// What a sequence asks for: pages from rank `offset` of the free ones on, `need` of them, the first of which
// replaces the last it holds where `copies`.
struct PageNeed {
    int32_t offset, need, held, wanted;  // held, wanted: pages; wanted's top bit: copies
    int32_t length;                      // once it has them
};

struct PagesArgs {
    const int32_t *table, *length, *refs, *wanted;
    int32_t *table_out, *length_out, *refs_out, *moves, *count;
    int32_t B, W, pages, shift;  // (B * W below 2^31)
    PageNeed* needs;             // workspace: [B]
    uint64_t* bits;              // a word of kWordPages pages each
    int32_t *chunk, *before;     // counts of kChunkPages pages; compaction: pages in use before each word
    int32_t* total;              // needed pages; compaction: pages in use, and how many of these lie in front
};

// The lanes that share a phase.
struct Lanes {
    int64_t id, n;
};
__device__ __forceinline__ Lanes grid_lanes() {
    return Lanes{int64_t(blockIdx.x) * blockDim.x + threadIdx.x, int64_t(gridDim.x) * blockDim.x};
}
__device__ __forceinline__ Lanes group_lanes() { return Lanes{threadIdx.x, blockDim.x}; }

__device__ __forceinline__ int pages_of(int tokens, int shift) { return (tokens + (1 << shift) - 1) >> shift; }
__device__ __forceinline__ bool is_page(const PagesArgs& a, int p) { return unsigned(p) < unsigned(a.pages); }
__device__ __forceinline__ int held_length(const PagesArgs& a, int b) {
    const int n = a.length[b], most = a.W << a.shift;
    return n < 0 ? 0 : n > most ? most : n;
}
__device__ __forceinline__ int wanted_length(const PagesArgs& a, int b, int held) {
    const int n = a.wanted[b];
    return n < 0 || n > (a.W << a.shift) ? held : n;
}

__device__ __forceinline__ void pages_copy_refs(const PagesArgs& a, Lanes at) {
    if (a.refs_out == a.refs) return;
    for (int64_t p = at.id; p < a.pages; p += at.n) a.refs_out[p] = a.refs[p];
}

// Sequence b takes what sequence wanted[b] holds.
__device__ __forceinline__ void pages_fork(const PagesArgs& a, Lanes at) {
    const unsigned all = unsigned(a.B) * unsigned(a.W);
    for (int64_t e = at.id; e < all; e += at.n) {
        const int b = int(unsigned(e) / unsigned(a.W)), i = int(unsigned(e) % unsigned(a.W));
        const int w = a.wanted[b], from = unsigned(w) < unsigned(a.B) ? w : b;
        const int mine = i < pages_of(held_length(a, b), a.shift) ? a.table[e] : -1;
        const int n = held_length(a, from);
        const int now = i < pages_of(n, a.shift) ? a.table[int64_t(from) * a.W + i] : -1;
        a.table_out[e] = now;
        if (from != b) {
            if (is_page(a, now)) atomicAdd(&a.refs_out[now], 1);
            if (is_page(a, mine)) atomicSub(&a.refs_out[mine], 1);
        }
        if (i == 0) a.length_out[b] = n;
    }
}

// Entries past what a sequence keeps are given back.
__device__ __forceinline__ void pages_release(const PagesArgs& a, Lanes at) {
    const unsigned all = unsigned(a.B) * unsigned(a.W);
    for (int64_t e = at.id; e < all; e += at.n) {
        const int b = int(unsigned(e) / unsigned(a.W)), i = int(unsigned(e) % unsigned(a.W));
        const int old = held_length(a, b), now = wanted_length(a, b, old);
        const int held = pages_of(old, a.shift), kept = pages_of(now < old ? now : old, a.shift);
        const int p = a.table[e];
        if (i >= kept && i < held && is_page(a, p)) atomicSub(&a.refs_out[p], 1);
        a.table_out[e] = i < kept ? p : -1;
    }
}

// A word of bits for every kWordPages pages, and the number of bits in every kChunkWords words: free pages, or
// pages in use.
template <bool FREE>
__device__ __forceinline__ void pages_count(const PagesArgs& a, const int32_t* refs, int64_t wave, int64_t waves) {
    const int lane = threadIdx.x & 63;
    const int64_t chunks = (int64_t(a.pages) + kChunkPages - 1) / kChunkPages;
    for (int64_t c = wave; c < chunks; c += waves) {
        int n[kChunkWords], sum = 0;
#pragma unroll
        for (int i = 0; i < kChunkWords; ++i) {
            const int64_t p = c * kChunkPages + i * kWordPages + lane;
            n[i] = refs[p < a.pages ? p : a.pages - 1];
        }
#pragma unroll
        for (int i = 0; i < kChunkWords; ++i) {
            const uint64_t word = __ballot(c * kChunkPages + i * kWordPages + lane < a.pages && (FREE ? n[i] <= 0 : n[i] > 0));
            if (lane == 0 && (c * kChunkWords + i) * kWordPages < a.pages) a.bits[c * kChunkWords + i] = word;
            sum += __popcll(word);
        }
        if (lane == 0) a.chunk[c] = sum;
    }
}

// What each sequence needs, and its place among the free pages: by one workgroup of T lanes.
template <int T>
__device__ __forceinline__ void pages_needs(const PagesArgs& a, int* s_scan) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int base = 0;
    for (int b0 = 0; b0 < a.B; b0 += T) {
        const int b = b0 + tid;
        PageNeed n{};
        if (b < a.B) {
            const int old = held_length(a, b), now = wanted_length(a, b, old);
            const bool grows = now > old;
            n.held = pages_of(old, a.shift);
            n.wanted = pages_of(now, a.shift);
            n.length = now;
            bool copies = false;
            if (grows && (old & ((1 << a.shift) - 1))) {  // (the page that it ends in is shared)
                const int last = a.table_out[int64_t(b) * a.W + n.held - 1];
                copies = is_page(a, last) && a.refs_out[last] > 1;
            }
            n.need = grows ? n.wanted - n.held + copies : 0;
            if (copies) n.wanted |= int(0x80000000u);
            a.length_out[b] = grows && n.need ? old : now;  // (until it is known to have its pages)
            a.moves[2 * int64_t(b)] = a.moves[2 * int64_t(b) + 1] = -1;
        }
        // the sum over the sequences before: 64-bit overflow is out of reach, 32-bit too (W * page <= 2^30 tokens
        // of pages of 16 and more, B * W < 2^31)
        int sum = n.need;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const int o = __shfl_up(sum, d);
            if (lane >= d) sum += o;
        }
        if (lane == 63) s_scan[wave] = sum;
        __syncthreads();
        int before = 0, all = 0;
#pragma unroll
        for (int w = 0; w < T / kWave; ++w) {
            if (w < wave) before += s_scan[w];
            all += s_scan[w];
        }
        __syncthreads();
        if (b < a.B) {
            n.offset = base + before + sum - n.need;
            a.needs[b] = n;
        }
        base += all;
    }
    if (tid == 0) a.total[0] = base;
}

// Sum of the chunks' counts before chunk c, and of all, by a wave.
__device__ __forceinline__ int2 chunks_before(const PagesArgs& a, int64_t c) {
    const int lane = threadIdx.x & 63;
    const int64_t chunks = (int64_t(a.pages) + kChunkPages - 1) / kChunkPages;
    int before = 0, all = 0;
    for (int64_t i = lane; i < chunks; i += kWave) {
        const int n = a.chunk[i];
        all += n;
        if (i < c) before += n;
    }
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
        before += __shfl_xor(before, d);
        all += __shfl_xor(all, d);
    }
    return int2{before, all};
}

// Free pages go to the sequences, in order, each wave with chunks that follow one another; a sequence whose pages there are not enough for stays as it was.
__device__ __forceinline__ void pages_assign(const PagesArgs& a, Lanes at, int* s_offset) {
    const int lane = threadIdx.x & 63;
    const int needed = a.total[0];
    const bool in_lds = a.B <= kOffsetsInLds;
    if (in_lds) {
        for (int b = threadIdx.x; b < a.B; b += blockDim.x) s_offset[b] = a.needs[b].offset;
        __syncthreads();
    }
    const int64_t chunks = (int64_t(a.pages) + kChunkPages - 1) / kChunkPages;
    const int64_t per = (chunks + (at.n >> 6) - 1) / (at.n >> 6), c0 = (at.id >> 6) * per, c1 = c0 + per < chunks ? c0 + per : chunks;
    const int2 sums = chunks_before(a, c0);
    int rank = sums.x;
    const int free = sums.y;
    for (int64_t c = c0; c < c1; ++c) {
        for (int i = 0; i < kChunkWords && rank < needed && (c * kChunkWords + i) * kWordPages < a.pages; ++i) {
            const uint64_t word = a.bits[c * kChunkWords + i];
            const int mine = rank + __popcll(word & ((uint64_t(1) << lane) - 1));
            rank += __popcll(word);
            if (!(word >> lane & 1) || mine >= needed) continue;
            int lo = 0, hi = a.B;  // the last sequence whose offset is at most `mine`
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                if ((in_lds ? s_offset[mid] : a.needs[mid].offset) <= mine) lo = mid;
                else hi = mid;
            }
            const PageNeed n = a.needs[lo];
            if (n.offset + n.need > free) continue;
            const int page = int(c * kChunkPages + i * kWordPages + lane), copies = n.wanted < 0 ? 1 : 0, j = mine - n.offset;
            int32_t* entry = a.table_out + int64_t(lo) * a.W + n.held + j - copies;
            a.refs_out[page] = 1;
            if (copies && j == 0) {
                const int last = *entry;
                atomicSub(&a.refs_out[last], 1);
                a.moves[2 * int64_t(lo)] = last;
                a.moves[2 * int64_t(lo) + 1] = page;
            }
            *entry = page;
        }
    }
    for (int64_t b = at.id; b < a.B; b += at.n) {
        const PageNeed n = a.needs[b];
        if (n.need && n.offset + n.need <= free) a.length_out[b] = n.length;
    }
}

// Compaction: U pages are in use. The i-th of these from page U on moves to the i-th free page before U.
__device__ __forceinline__ void pages_plan_moves(const PagesArgs& a, Lanes at) {
    const int lane = threadIdx.x & 63;
    const int64_t chunks = (int64_t(a.pages) + kChunkPages - 1) / kChunkPages, words = (int64_t(a.pages) + kWordPages - 1) / kWordPages;
    const int64_t per = (chunks + (at.n >> 6) - 1) / (at.n >> 6), c0 = (at.id >> 6) * per, c1 = c0 + per < chunks ? c0 + per : chunks;
    const int2 sums = chunks_before(a, c0);
    int rank = sums.x;
    const int64_t U = sums.y, cu = U / kChunkPages;
    int front = 0;  // of the pages in use, those before U
    if (lane < kChunkWords && cu * kChunkWords + lane < words) {
        const int64_t left = U - (cu * kChunkWords + lane) * kWordPages;
        const uint64_t word = a.bits[cu * kChunkWords + lane];
        front = left <= 0 ? 0 : __popcll(left >= kWordPages ? word : word & ((uint64_t(1) << left) - 1));
    }
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) front += __shfl_xor(front, d);
    front += chunks_before(a, cu).x;
    if (at.id == 0) {
        a.total[0] = int(U);
        a.total[1] = front;
        a.count[0] = int(U);
    }
    for (int64_t c = c0; c < c1; ++c) {
        for (int i = 0; i < kChunkWords && c * kChunkWords + i < words; ++i) {
            const int64_t at_word = c * kChunkWords + i, p = at_word * kWordPages + lane;
            const uint64_t word = a.bits[at_word];
            const int mine = rank + __popcll(word & ((uint64_t(1) << lane) - 1));
            if (lane == 0) a.before[at_word] = rank;
            rank += __popcll(word);
            if (p >= a.pages) continue;
            if (word >> lane & 1) {
                if (p >= U) a.moves[2 * int64_t(mine - front)] = int(p);
            } else if (p < U) {
                a.moves[2 * (p - mine) + 1] = int(p);
            }
        }
    }
    const int64_t most = a.pages / 2;
    for (int64_t i = U - front + at.id; i < most; i += at.n) a.moves[2 * i] = a.moves[2 * i + 1] = -1;
}

__device__ __forceinline__ void pages_renumber(const PagesArgs& a, Lanes at) {
    const int64_t U = a.total[0], front = a.total[1];
    auto in_use = [&](int64_t p) { return bool(a.bits[p / kWordPages] >> (p % kWordPages) & 1); };
    for (int64_t p = at.id; p < a.pages; p += at.n) {
        const bool used = in_use(p);
        if (used && p < U) {
            if (a.refs_out != a.refs) a.refs_out[p] = a.refs[p];
        } else if (!used && p >= U) {
            a.refs_out[p] = 0;
        }
    }
    for (int64_t i = at.id; i < U - front; i += at.n) {
        const int src = a.moves[2 * i], dst = a.moves[2 * i + 1];
        a.refs_out[dst] = a.refs[src];
        a.refs_out[src] = 0;
    }
    const unsigned all = unsigned(a.B) * unsigned(a.W);
    for (int64_t e = at.id; e < all; e += at.n) {
        int p = a.table[e];
        if (!is_page(a, p) || !in_use(p)) {
            p = -1;
        } else if (p >= U) {
            const int64_t word = p / kWordPages;
            const int rank = a.before[word] + __popcll(a.bits[word] & ((uint64_t(1) << (p % kWordPages)) - 1));
            p = a.moves[2 * (rank - front) + 1];
        }
        a.table_out[e] = p;
    }
}

enum PagesPhase { kCopyRefs, kFork, kRelease, kCountFree, kAssign, kCountUsed, kPlanMoves, kRenumber };

// One phase by the whole grid. Of kCountFree the last workgroup works out what is needed.
template <PagesPhase PH>
__global__ __launch_bounds__(kPagesGroup) void pages_phase_kernel(PagesArgs a) {
    const Lanes at = grid_lanes();
    if constexpr (PH == kCopyRefs) pages_copy_refs(a, at);
    if constexpr (PH == kFork) pages_fork(a, at);
    if constexpr (PH == kRelease) pages_release(a, at);
    if constexpr (PH == kCountFree) {
        __shared__ int s_scan[kPagesGroup / kWave];
        if (blockIdx.x + 1 == gridDim.x) pages_needs<kPagesGroup>(a, s_scan);
        else pages_count<true>(a, a.refs_out, at.id >> 6, (at.n - kPagesGroup) >> 6);
    }
    if constexpr (PH == kAssign) {
        __shared__ int s_offset[kOffsetsInLds];
        pages_assign(a, at, s_offset);
    }
    if constexpr (PH == kCountUsed) pages_count<false>(a, a.refs, at.id >> 6, at.n >> 6);
    if constexpr (PH == kPlanMoves) pages_plan_moves(a, at);
    if constexpr (PH == kRenumber) pages_renumber(a, at);
}

enum PagesCall { kCallFork, kCallResize, kCallCompact };

// All of a call by one workgroup, with the counts of all pages in LDS, where a barrier is all that lies between two phases.
template <PagesCall C>
__global__ __launch_bounds__(kPagesSmall) void pages_lds_kernel(PagesArgs given) {
    __shared__ int32_t s_refs[kLdsPages], s_chunk[kLdsPages / kChunkPages], s_before[kLdsPages / kWordPages], s_total[2];
    __shared__ uint64_t s_bits[kLdsPages / kWordPages];
    const Lanes at = group_lanes();
    PagesArgs a = given;
    a.bits = s_bits;
    a.chunk = s_chunk;
    a.before = s_before;
    a.total = s_total;
    a.refs_out = s_refs;
    for (int64_t p = at.id; p < a.pages; p += at.n) s_refs[p] = given.refs[p];
    __syncthreads();
    if constexpr (C == kCallFork) pages_fork(a, at);
    if constexpr (C == kCallResize) {
        __shared__ int s_scan[kPagesSmall / kWave], s_offset[kOffsetsInLds];
        pages_release(a, at);
        __syncthreads();
        pages_count<true>(a, s_refs, at.id >> 6, at.n >> 6);
        pages_needs<kPagesSmall>(a, s_scan);
        __syncthreads();
        pages_assign(a, at, s_offset);
    }
    if constexpr (C == kCallCompact) {
        a.refs = s_refs;
        pages_count<false>(a, s_refs, at.id >> 6, at.n >> 6);
        __syncthreads();
        pages_plan_moves(a, at);
        __syncthreads();
        pages_renumber(a, at);
    }
    __syncthreads();
    for (int64_t p = at.id; p < a.pages; p += at.n) given.refs_out[p] = s_refs[p];
}

struct PagesCopyArgs {
    char* cache;
    const int32_t* moves;
    int64_t n, layers, pages, layer_stride, page_stride, page_bytes, pieces;  // pieces: workgroups a page
};

// Moves pages: a piece of 16 KB of a page and layer is one workgroup's, all of a lane's loads on their way before its first
// store; neither is looked at again soon, so both pass the caches by. 4096 pages of 128 KB (1.07 GB read and written): 5.05
// TB/s with the plan, as fast as a copy of as much in one piece; with caches 4.5, with 32 KB a workgroup 3.7.
constexpr int kCopyLanes = 256, kCopyVecs = 4;
template <typename V>
__global__ __launch_bounds__(kCopyLanes) void pages_copy_kernel(PagesCopyArgs a) {
    int64_t item = grid_row();
    const int64_t piece = item % a.pieces;
    item /= a.pieces;
    const int64_t layer = item % a.layers, move = item / a.layers;
    if (move >= a.n) return;
    const int64_t src = a.moves[2 * move], dst = a.moves[2 * move + 1];
    if (src < 0 || dst < 0 || src >= a.pages || dst >= a.pages || src == dst) return;
    const int64_t count = a.page_bytes / int64_t(sizeof(V));
    const V* from = reinterpret_cast<const V*>(a.cache + layer * a.layer_stride + src * a.page_stride);
    V* to = reinterpret_cast<V*>(a.cache + layer * a.layer_stride + dst * a.page_stride);
    const int64_t at = piece * kCopyLanes * kCopyVecs + threadIdx.x;
    V v[kCopyVecs];
#pragma unroll
    for (int i = 0; i < kCopyVecs; ++i)
        if (at + i * kCopyLanes < count) v[i] = __builtin_nontemporal_load(from + at + i * kCopyLanes);
#pragma unroll
    for (int i = 0; i < kCopyVecs; ++i)
        if (at + i * kCopyLanes < count) __builtin_nontemporal_store(v[i], to + at + i * kCopyLanes);
}

}  // namespace rlcs
