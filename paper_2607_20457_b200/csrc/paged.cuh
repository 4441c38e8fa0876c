// The paged key/value cache: what its calls have in common (pages.cu, paged.cu).
#pragma once

#include <initializer_list>

#include "common.cuh"

namespace pulsar {

// Sizes of a pool and a page table that the kernels cover.
inline bool pool_ok(int64_t n_layers, int32_t n_pages, int32_t page_size, int32_t Hkv, int32_t d, int32_t n_slots, int32_t max_pages) {
    const bool page = page_size == 16 || page_size == 32 || page_size == 64 || page_size == 128;
    return page && (d == 64 || d == 128) && Hkv >= 1 && Hkv <= 1024 && n_layers >= 1 && n_pages >= 1 && n_pages < (1 << 24) &&
           n_slots >= 1 && n_slots <= 1024 && max_pages >= 1 && static_cast<int64_t>(max_pages) * page_size <= (int64_t{1} << 30) &&
           static_cast<int64_t>(n_slots) * max_pages < (int64_t{1} << 31);
}
// Whether the pieces of an attention call can be counted in 32 bits, whatever the lengths on the device are.
inline bool pieces_ok(int64_t n_slots, int64_t max_items, int64_t keys) { return n_slots * max_items * (keys / 128 + 2) < (int64_t{1} << 31); }
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

struct Bytes {
    const void* p;
    size_t n;
};
using Tensors = std::initializer_list<Bytes>;
// Whether none of the outputs shares memory with another one or with an input.
inline bool apart(Tensors outputs, Tensors inputs) {
    for (const Bytes* o = outputs.begin(); o != outputs.end(); ++o) {
        for (const Bytes* x = o + 1; x != outputs.end(); ++x)
            if (overlap(o->p, o->n, x->p, x->n)) return false;
        for (const Bytes& x : inputs)
            if (overlap(o->p, o->n, x.p, x.n)) return false;
    }
    return true;
}
inline size_t pool_bytes(int64_t n_layers, int64_t n_pages, int64_t page_size, int64_t Hkv, int64_t d) {
    return static_cast<size_t>(n_layers * n_pages * page_size * Hkv * d) * 2;
}

constexpr int kMaxSlots = 1024;
constexpr int kMaxTree = 64;                    // nodes of a drafted tree

// Arguments of the attention kernels.  A work item is some query rows of one KV head against a list of keys, cut into pieces; every
// CTA takes an equal share of all pieces of all slots and leaves a partial (normalised output and l = ln sum exp) where it holds an
// item only in part.
struct Meta {                                   // of an item
    int parts;                                  // partials that it is in: 0 or 1: nothing is to be joined
    int first, cta, step;                       // place of the first one, left by CTA `cta`; the others are the first ones of every step-th CTA after it
    int token0, head0, row0, rows;              // of its rows: see row_of
};

struct PagedArgs {
    const uint16_t *Q, *Knew, *Vnew;             // [n_slots, T, Hq | Hkv, D]
    uint16_t *K, *V;                             // [n_pages, page_size, Hkv, D]
    const int32_t *table, *len, *n_draft, *parent;
    const int32_t* list;                         // selected pages: [n_slots, T, Hkv, k + 1] page ids, the last row's page among them
    int n_slots, T, Hq, Hkv, g_shift, page_shift, n_pages, max_pages, k;
    int fresh_rows;                              // rows of the new tokens' tile that are loaded: T, up to a multiple of 8
    float scale_log2;
    void* O;
    int out_f32;
    float* LSE;
    float *part_O, *part_LSE;                    // [2 * CTAs, rows of an item, D], [2 * CTAs, rows of an item]
    Meta* meta;                                  // [n_slots, items_max, row blocks]
    int items_max;                               // items that a slot can have
    int32_t* status;
};

// Appends the new tokens' rows, and joins the partials of `items` items of `rows` rows (paged_merge.cu).
int32_t launch_parts_merge(const PagedArgs& a, int64_t items, int rows, int d, cudaStream_t stream);

// Attention over the rows of the cache or, where there is a list, over the selected pages (paged_tiles.cu).  rows: of an item.
size_t attn_workspace_bytes(int n_slots, int items, int rows, int d);      // items: of a slot, at the most
int32_t launch_attn(PagedArgs a, int items, int rows, int d, void* workspace, cudaStream_t stream);

// Scratch of an attention launch: what its CTAs leave for the merge.  rows: of an item.
struct PartScratch {
    size_t meta, part_O, part_LSE, total;
    PartScratch(size_t items, size_t ctas, int rows, int d) {
        meta = 0;
        part_LSE = round_up(items * sizeof(Meta), 256);
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

constexpr int kTile = 128;                       // keys of a piece

// Bookkeeping of a slot, the same in every CTA.  Tiles of all slots together are fewer than 2^31 (checked on the host: pieces_ok).
// The new tokens follow the cached rows in the last tile, from the next multiple of 16 on, or have a tile of their own where they do
// not fit: a decoding step behind 100 rows is one tile, not two.
struct SlotWork {
    int len, n;                                  // rows in the cache; new tokens
    int keys;                                    // cached rows an item reads
    int pieces, items;
    int new_tile, new_at;                        // the tile with the new tokens, and their place in it
};
template <bool kSparse>
__device__ __forceinline__ SlotWork slot_work(const PagedArgs& a, int len, int n) {
    SlotWork w;
    w.len = len;
    w.n = n;
    const int full = len >> a.page_shift;
    w.keys = kSparse ? (min(a.k, full) << a.page_shift) + (len - (full << a.page_shift)) : len;
    const int whole = w.keys / kTile, tail = w.keys % kTile, at = (tail + 15) / 16 * 16;
    const bool joint = tail > 0 && at + a.fresh_rows <= kTile;
    w.new_tile = whole + (tail > 0 && !joint ? 1 : 0);
    w.new_at = joint ? at : 0;
    w.pieces = w.new_tile + 1;
    w.items = n == 0 ? 0 : kSparse ? n * a.Hkv : a.Hkv;
    return w;
}

// Row r of an item: token token0 + r' / g and head head0 + r' % g, with r' = row0 + r.
__device__ __forceinline__ int64_t row_of(int token0, int head0, int row0, int r, int g_shift, int Hq) {
    const int x = row0 + r;
    return static_cast<int64_t>(token0 + (x >> g_shift)) * Hq + head0 + (x & ((1 << g_shift) - 1));
}

// What a CTA knows of the slots, in shared memory.
struct Slots {
    int before[kMaxSlots + 1];                   // pieces of the slots before
    int len[kMaxSlots];
    unsigned char n[kMaxSlots];
};
// One warp fills it in; returns the pieces of all slots, and how many items they are of.
template <bool kSparse>
__device__ __forceinline__ int all_pieces(const PagedArgs& a, Slots& slots, int row_blocks, int& items) {
    const int lane = threadIdx.x & 31;
    int total = 0, mine = 0;
    for (int s0 = 0; s0 < a.n_slots; s0 += 32) {
        const int s = s0 + lane;
        int x = 0;
        if (s < a.n_slots) {
            const int len = checked_len(a.len[s], static_cast<int64_t>(a.max_pages) << a.page_shift, blockIdx.x == 0, a.status);
            const int n = a.n_draft != nullptr ? min(max(a.n_draft[s], 0), a.T) : a.T;
            const SlotWork w = slot_work<kSparse>(a, len, n);
            x = w.pieces * w.items;
            mine += w.items;
            if (blockIdx.x == 0)                                         // items that do not exist
                for (int i = w.items * row_blocks; i < a.items_max * row_blocks; ++i) a.meta[static_cast<int64_t>(s) * a.items_max * row_blocks + i].parts = 0;
            slots.len[s] = len;
            slots.n[s] = static_cast<unsigned char>(n);
        }
        int y = x;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int z = __shfl_up_sync(0xffffffffu, y, d);
            if (lane >= d) y += z;
        }
        if (s < a.n_slots) slots.before[s] = total + y - x;
        total += __shfl_sync(0xffffffffu, y, 31);
    }
    if (lane == 0) slots.before[a.n_slots] = total;
    items = __reduce_add_sync(0xffffffffu, mine);
    __syncwarp();
    return total;
}

// Equal shares of `total` pieces: the first `more` of n have one more than the others.
struct Shares {
    uint32_t n, each, more;
    __device__ __forceinline__ Shares(int total, int wanted, int ctas) {
        n = static_cast<uint32_t>(max(1, min(ctas, min(wanted, total))));
        each = static_cast<uint32_t>(total) / n;
        more = static_cast<uint32_t>(total) - each * n;
    }
    __device__ __forceinline__ int begin(int i) const {        // n and beyond: all of them
        const uint32_t c = min(static_cast<uint32_t>(i), n);
        return static_cast<int>(c * each + min(c, more));
    }
    __device__ __forceinline__ int owner(int piece) const {
        const uint32_t p = static_cast<uint32_t>(piece), low = more * (each + 1);
        return static_cast<int>(p < low ? p / (each + 1) : more + (p - low) / each);
    }
};
// The last slot that begins at or before piece `at`.
__device__ __forceinline__ int slot_at(const Slots& slots, int n_slots, int at) {
    int lo = 0, hi = n_slots - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (slots.before[mid] <= at) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// A CTA's pieces of one item.
struct Segment {
    SlotWork w;
    int slot, p_begin, p_end;
    int n_rows, kvh, token, token0, head0;       // query rows; KV head; sparse: the token; first token among all, first head
    int item, item_at;                           // number within the slot; its first piece among all
};
template <bool kSparse>
__device__ __forceinline__ Segment segment_at(const PagedArgs& a, const Slots& slots, int at, int end, int& slot) {
    Segment s;
    while (slots.before[slot + 1] <= at) ++slot;
    s.slot = slot;
    s.w = slot_work<kSparse>(a, slots.len[slot], slots.n[slot]);
    const int first = slots.before[slot];
    const int item = static_cast<int>(static_cast<uint32_t>(at - first) / static_cast<uint32_t>(s.w.pieces));
    s.item = item;
    s.item_at = first + item * s.w.pieces;
    s.p_begin = at - s.item_at;
    s.p_end = min(end - s.item_at, s.w.pieces);
    s.kvh = kSparse ? item % a.Hkv : item;
    s.token = kSparse ? item / a.Hkv : 0;
    s.n_rows = (kSparse ? 1 : s.w.n) << a.g_shift;
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

#endif

}  // namespace pulsar
