// The paged key/value cache: what its calls have in common (pages.cu, paged.cu).
#pragma once

#include "common.cuh"

namespace pulsar {

// Sizes of a pool and a page table that the kernels cover.
inline bool pool_ok(int64_t n_layers, int32_t n_pages, int32_t page_size, int32_t Hkv, int32_t d, int32_t n_slots, int32_t max_pages) {
    const bool page = page_size == 16 || page_size == 32 || page_size == 64 || page_size == 128;
    return page && (d == 64 || d == 128) && Hkv >= 1 && Hkv <= 1024 && n_layers >= 1 && n_pages >= 1 && n_pages < (1 << 24) &&
           n_slots >= 1 && n_slots <= 1024 && max_pages >= 1 && static_cast<int64_t>(max_pages) * page_size <= (int64_t{1} << 30) &&
           static_cast<int64_t>(n_slots) * max_pages < (int64_t{1} << 31);
}
inline int log2_exact(int x) {
    int s = 0;
    while ((1 << s) < x) ++s;
    return s;
}
// Whether [a, a + na) and [b, b + nb) have bytes in common.
inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
    const auto x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return a != nullptr && b != nullptr && x < y + nb && y < x + na;
}

constexpr int kMaxSlots = 1024;
constexpr int kMaxTree = 64;                    // nodes of a drafted tree

// Arguments of the attention kernels.  A work item is some query rows of one KV head against a list of keys, cut into pieces; every
// CTA takes an equal share of all pieces of all slots and leaves a partial (normalised output and l = ln sum exp) where it holds an
// item only in part.
struct Meta {                                   // the item that begins in a CTA and goes on in the next ones
    int first, parts;                           // first partial (those of the CTAs after it are their first ones); 0: there is none
    int token0, head0, row0, rows;              // of its rows: see row_of
};

struct PagedArgs {
    const uint16_t *Q, *Knew, *Vnew;             // [n_slots, T, Hq | Hkv, D]
    uint16_t *K, *V;                             // [n_pages, page_size, Hkv, D]
    const int32_t *table, *len, *n_draft, *parent;
    const int32_t* list;                         // selected pages: [n_slots, T, Hkv, k + 1] page ids, the last row's page among them
    int n_slots, T, Hq, Hkv, g_shift, page_shift, n_pages, max_pages, k;
    float scale_log2;
    void* O;
    int out_f32;
    float* LSE;
    float *part_O, *part_LSE;                    // [2 * CTAs, rows of an item, D], [2 * CTAs, rows of an item]
    Meta* meta;                                  // [CTAs]
    int32_t* status;
};

// Trees with more than eight query rows per KV head (paged_tiles.cu).
size_t tree_tiles_workspace_bytes(int rows, int d);
int32_t launch_tree_tiles(PagedArgs a, int rows, int d, void* workspace, cudaStream_t stream);

// Scratch of an attention launch: what its CTAs leave for the merge.  rows: of an item.
struct PartScratch {
    size_t meta, part_O, part_LSE, total;
    PartScratch(size_t ctas, int rows, int d) {
        meta = 0;
        part_LSE = round_up(ctas * sizeof(Meta), 256);
        part_O = round_up(part_LSE + 2 * ctas * rows * 4, 256);
        total = round_up(part_O + 2 * ctas * rows * d * 4, 256);
    }
    void place(PagedArgs& a, void* workspace) const {
        auto* ws = static_cast<uint8_t*>(workspace);
        a.meta = reinterpret_cast<Meta*>(ws + meta);
        a.part_LSE = reinterpret_cast<float*>(ws + part_LSE);
        a.part_O = reinterpret_cast<float*>(ws + part_O);
    }
};

#ifdef __CUDACC__
// A slot's length within its table; what is outside is reported once (by the thread for which `tell` is set) and clamped.
__device__ __forceinline__ int checked_len(int len, int64_t capacity, bool tell, int32_t* status) {
    if (len >= 0 && len <= capacity) return len;
    if (tell) report(status, PULSAR_DEV_BAD_LENGTH);
    return len < 0 ? 0 : static_cast<int>(capacity);
}

// Bookkeeping of a slot, the same in every CTA.
struct SlotWork {
    int len, n;                                  // rows in the cache; new tokens
    int keys;                                    // cached rows an item reads
    int cache_pieces, pieces, items;
};
template <bool kSparse, int kKeys, int kRows>
__device__ __forceinline__ SlotWork slot_work(const PagedArgs& a, int slot, bool tell) {
    SlotWork w;
    w.len = checked_len(a.len[slot], static_cast<int64_t>(a.max_pages) << a.page_shift, tell, a.status);
    w.n = a.n_draft != nullptr ? min(max(a.n_draft[slot], 0), a.T) : a.T;
    const int full = w.len >> a.page_shift;
    w.keys = kSparse ? (min(a.k, full) << a.page_shift) + (w.len - (full << a.page_shift)) : w.len;
    w.cache_pieces = (w.keys + kKeys - 1) / kKeys;
    w.pieces = w.cache_pieces + (w.n + kKeys - 1) / kKeys;
    const int g = 1 << a.g_shift;
    w.items = kSparse ? w.n * a.Hkv * ((g + kRows - 1) / kRows) : a.Hkv * ((w.n * g + kRows - 1) / kRows);
    return w;
}

// Row r of an item: token token0 + r' / g and head head0 + r' % g, with r' = row0 + r.
__device__ __forceinline__ int64_t row_of(int token0, int head0, int row0, int r, int g_shift, int Hq) {
    const int x = row0 + r;
    return static_cast<int64_t>(token0 + (x >> g_shift)) * Hq + head0 + (x & ((1 << g_shift) - 1));
}

// Pieces of the slots before each slot, in s_pieces [n_slots + 1]; returns those of all.  s_warp: [warps of the CTA].
template <bool kSparse, int kKeys, int kRows, int kThreads>
__device__ __forceinline__ int64_t all_pieces(const PagedArgs& a, int64_t* s_pieces, int64_t* s_warp) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t total = 0;
    for (int s0 = 0; s0 < a.n_slots; s0 += kThreads) {
        const int s = s0 + threadIdx.x;
        int64_t x = 0;
        if (s < a.n_slots) {
            const SlotWork w = slot_work<kSparse, kKeys, kRows>(a, s, blockIdx.x == 0);
            x = static_cast<int64_t>(w.pieces) * w.items;
        }
        int64_t y = x;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int64_t z = __shfl_up_sync(0xffffffffu, y, d);
            if (lane >= d) y += z;
        }
        if (lane == 31) s_warp[warp] = y;
        __syncthreads();
        int64_t before = total;
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w < warp) before += s_warp[w];
            total += s_warp[w];
        }
        if (s < a.n_slots) s_pieces[s] = before + y - x;
        __syncthreads();
    }
    if (threadIdx.x == 0) s_pieces[a.n_slots] = total;
    __syncthreads();
    return total;
}

// This CTA's share of them.
struct Share {
    int64_t total, n_ctas, begin, end;
};
__device__ __forceinline__ Share share_of(int64_t total, int least) {
    Share s;
    s.total = total;
    s.n_ctas = max(static_cast<int64_t>(1), min(static_cast<int64_t>(gridDim.x), total / least));
    s.begin = blockIdx.x < s.n_ctas ? total * blockIdx.x / s.n_ctas : total;
    s.end = blockIdx.x < s.n_ctas ? total * (blockIdx.x + 1) / s.n_ctas : total;
    return s;
}
// The last slot that begins at or before piece `at`.
__device__ __forceinline__ int slot_at(const int64_t* s_pieces, int n_slots, int64_t at) {
    int lo = 0, hi = n_slots - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (s_pieces[mid] <= at) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// A CTA's pieces of one item.
struct Segment {
    SlotWork w;
    int slot, p_begin, p_end;
    int row0, n_rows, kvh, token, token0, head0;
    int64_t item_at;                             // the item's first piece among all
};
template <bool kSparse, int kKeys, int kRows>
__device__ __forceinline__ Segment segment_at(const PagedArgs& a, const int64_t* s_pieces, int64_t at, int64_t end, int& slot) {
    Segment s;
    while (s_pieces[slot + 1] <= at) ++slot;
    s.slot = slot;
    s.w = slot_work<kSparse, kKeys, kRows>(a, slot, false);
    const int item = static_cast<int>((at - s_pieces[slot]) / s.w.pieces), g = 1 << a.g_shift;
    s.item_at = s_pieces[slot] + static_cast<int64_t>(item) * s.w.pieces;
    s.p_begin = static_cast<int>(at - s.item_at);
    s.p_end = static_cast<int>(min(end - s.item_at, static_cast<int64_t>(s.w.pieces)));
    const int rows = kSparse ? g : s.w.n * g, row_blocks = (rows + kRows - 1) / kRows;
    const int unit = item / row_blocks;          // KV head, or token and KV head
    s.row0 = (item % row_blocks) * kRows;
    s.kvh = kSparse ? unit % a.Hkv : unit;
    s.token = kSparse ? unit / a.Hkv : 0;
    s.n_rows = min(kRows, rows - s.row0);
    s.token0 = slot * a.T + s.token;
    s.head0 = s.kvh << a.g_shift;
    return s;
}

// Where row `row` of a slot is written (elements from the pool's first, of KV head 0), or -1 where it has no page: reported.
__device__ __forceinline__ int64_t new_row_at(const PagedArgs& a, int slot, int64_t row, int64_t pitch) {
    if ((row >> a.page_shift) >= a.max_pages) {
        report(a.status, PULSAR_DEV_BAD_LENGTH);
        return -1;
    }
    const int page = a.table[static_cast<int64_t>(slot) * a.max_pages + (row >> a.page_shift)];
    if (page < 0 || page >= a.n_pages) {
        report(a.status, PULSAR_DEV_BAD_PAGE);
        return -1;
    }
    return ((static_cast<int64_t>(page) << a.page_shift) + (row & ((1 << a.page_shift) - 1))) * pitch;
}

// A node's ancestors and itself, as a bit per node, for the first kMaxTree threads that call this together (sync: their barrier,
// sees: their result [kMaxTree], up: scratch [kMaxTree]).  Pointers to ancestors are doubled: six steps for 64 nodes.
template <typename Sync>
__device__ __forceinline__ void ancestors(const PagedArgs& a, int slot, int n, int t, uint64_t* sees, int* up, Sync sync) {
    int to = -1;
    if (t < n) {
        to = a.parent != nullptr ? a.parent[static_cast<int64_t>(slot) * a.T + t] : t - 1;
        if (to < -1 || to >= t) {
            report(a.status, PULSAR_DEV_BAD_TREE);
            to = -1;
        }
    }
    uint64_t mine = t < kMaxTree ? 1ull << t : 0ull;
#pragma unroll 1
    for (int step = 1; step < kMaxTree; step <<= 1) {
        if (t < kMaxTree) {
            sees[t] = mine;
            up[t] = to;
        }
        sync();
        if (t < kMaxTree && to >= 0) {
            mine |= sees[to];
            to = up[to];
        }
        sync();
    }
    if (t < kMaxTree) sees[t] = mine;
    sync();
}
#endif

}  // namespace pulsar
