// What the attention kernels over a paged cache share: the loader of the pages, and the warps that fetch query rows and work out
// which token sees which.  A kernel's configuration C has its shared-memory layout, its barriers
// and its tile sizes.
#pragma once

#include "paged.cuh"
#include "tensor_map.cuh"

namespace pulsar {

constexpr int kPanelBytes = kTile * 128;         // 64 columns of a tile: 128-byte lines, swizzled
constexpr float kRescale = 8.f;                  // in log2 units
constexpr float kUnset = 1e30f;                  // stands for minus a maximum that no logit has set: every logit exceeds it
// Tiles of a CTA, at the least, where items are cut up: one where that leaves few parts to join (2 items of 5 tiles 20.6 -> 18.0 us with the
// selection), else two (2 items of 48 tiles 12.9 us, with one each 15.0, with four 13.9).
constexpr int kLeastTiles = 2, kFewParts = 8;
constexpr int kQueue = 4;                        // segments that the loader may publish ahead of the slowest consumer

// A CTA's pieces of one item, as the loader publishes them.
struct __align__(16) Work {
    int valid;                                   // 0: no more
    int slot, p_begin, p_end, new_tile;
    int keys, n, row0, n_rows, kvh, token0, head0;
    int part;                                    // place of the partial, -1: all of the item, its outputs are final
    int len, token, new_at;                      // rows in the slot's cache; selected pages: the item's token; see SlotWork
};
static_assert(sizeof(Work) == 64, "");

// Barriers of some warps (whole ones: their lanes come together first).
__device__ __forceinline__ void named_sync(int id, int threads) {
    __syncwarp();
    asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
// Whether any of the barrier's threads says so; the threads wait for each other.
__device__ __forceinline__ bool named_any(int id, int threads, bool x) {
    uint32_t y;
    __syncwarp();
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 q, %1, 0;\n\t"
        "bar.red.or.pred p, %2, %3, q;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(y) : "r"(x ? 1u : 0u), "r"(id), "r"(threads) : "memory");
    return y != 0;
}
__device__ __forceinline__ void arrive_a(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }

// Two fused multiply-adds (x * s + y), two sums, with one instruction each.
__device__ __forceinline__ void fma2(float& x0, float& x1, float s, float y0, float y1) {
    asm("{\n\t.reg .b64 a, b, c;\n\t"
        "mov.b64 a, {%0, %1};\n\tmov.b64 b, {%2, %2};\n\tmov.b64 c, {%3, %4};\n\t"
        "fma.rn.f32x2 a, a, b, c;\n\t"
        "mov.b64 {%0, %1}, a;\n\t}"
        : "+f"(x0), "+f"(x1) : "f"(s), "f"(y0), "f"(y1));
}
__device__ __forceinline__ void add2(float& x0, float& x1, float y0, float y1) {
    asm("{\n\t.reg .b64 a, b;\n\t"
        "mov.b64 a, {%0, %1};\n\tmov.b64 b, {%2, %3};\n\t"
        "add.rn.f32x2 a, a, b;\n\t"
        "mov.b64 {%0, %1}, a;\n\t}"
        : "+f"(x0), "+f"(x1) : "f"(y0), "f"(y1));
}

// Tensor maps of a launch: the pool's pages, runs of 16 rows of them, the new tokens' rows, and the query rows.
struct Maps {
    CUtensorMap K, V, K16, V16, Kn, Vn, Q;
};
__device__ __forceinline__ void prefetch_maps(const Maps& m) {
    tma_prefetch_desc(&m.K);
    tma_prefetch_desc(&m.V);
    tma_prefetch_desc(&m.K16);
    tma_prefetch_desc(&m.V16);
    tma_prefetch_desc(&m.Kn);
    tma_prefetch_desc(&m.Vn);
    tma_prefetch_desc(&m.Q);
}

// How many times 16 keys of tile t the product with V has to read.
__device__ __forceinline__ int used_steps(int t, int keys, int new_tile, int new_end) {
    return ((t == new_tile ? new_end : min(keys - t * kTile, kTile)) + 15) / 16;
}

// Trees with more than 64 query rows per KV head (paged_wide.cu).
int32_t launch_tree_wide(const PagedArgs& a, const Maps& map, int rows, int d, cudaStream_t stream);

// Shared memory that the roles use besides the tiles, and where the barriers are.
struct Roles {
    uint8_t* smem;
    Work* s_work;                                // [kQueue]
    uint64_t* s_sees;                            // [kQueue][kMaxTree] a node's ancestors and itself (C::kBySeen: the nodes that see it)
    uint32_t* s_odd;                             // [kQueue][2] nodes whose value is not finite
    int* s_up;                                   // [kMaxTree]
    Slots* slots;
    uint32_t bar0;
    volatile int* abort_flag;
    __device__ __forceinline__ uint32_t bar(int i) const { return bar0 + 8 * static_cast<uint32_t>(i); }
};

// The page ids of an item: its slot's table, or its token's and KV head's selected pages.
template <bool kSparse>
__device__ __forceinline__ const int32_t* page_list(const PagedArgs& a, int slot, int token0, int kvh) {
    return kSparse ? a.list + (static_cast<int64_t>(token0) * a.Hkv + kvh) * (a.k + 1) : a.table + static_cast<int64_t>(slot) * a.max_pages;
}

// The next published segment (a warp's lanes together); `ok` turns false where a wait has given up.
template <class C>
__device__ __forceinline__ const Work* next_work(const PagedArgs& a, const Roles& r, uint32_t seq, bool& ok) {
    __syncwarp();
    ok = __all_sync(0xffffffffu, ok && mbar_wait_a(r.bar(C::bWorkFull + static_cast<int>(seq % kQueue)), (seq / kQueue) & 1, r.abort_flag, a.status));
    return r.s_work + seq % kQueue;
}

// Copies the tiles of an item's pieces: kFirst .. kLast of K (0) and V (1), which take turns in the ring.
template <class C, int kFirst, int kLast>
struct Ring {
    uint32_t stage = kFirst, phase = 0;
    __device__ __forceinline__ void load(const PagedArgs& a, const Maps& map, const Roles& roles, const Work& s, bool& ok) {
        const int lane = threadIdx.x & 31;
        const int32_t* list = page_list<C::kSparse>(a, s.slot, s.token0, s.kvh);
        // A tile's rows are copied page by page, a page per lane; those before new tokens in the same tile 16 by 16, up to where these begin.
        const auto shift_of = [&](int t) { return t == s.new_tile ? 4 : a.page_shift; };
        const auto row_of_lane = [&](int t) { return t * kTile + (lane << shift_of(t)); };
        const auto has_rows = [&](int t) { return t < s.p_end && lane < kTile >> shift_of(t) && row_of_lane(t) < s.keys; };
        const auto page_of = [&](int t) { return has_rows(t) ? list[row_of_lane(t) >> a.page_shift] : 0; };
        int id = page_of(s.p_begin);
        for (int t = s.p_begin; t < s.p_end && ok; ++t) {
            const int next = page_of(t + 1);                       // (looked at a tile later)
            const bool fresh = t == s.new_tile, rows = has_rows(t);
            int page = id;
            if (rows && (id < 0 || id >= a.n_pages)) {
                report(a.status, PULSAR_DEV_BAD_PAGE);             // (some page is loaded; its rows count as absent)
                page = 0;
            }
            const int shift = shift_of(t), from = (page << a.page_shift) + (row_of_lane(t) & ((1 << a.page_shift) - 1));
            const uint32_t lines = (__popc(__ballot_sync(0xffffffffu, rows)) << shift) + (fresh ? a.fresh_rows : 0);
#pragma unroll
            for (int kv = kFirst; kv <= kLast; ++kv) {
                __syncwarp();
                ok = __all_sync(0xffffffffu, ok && mbar_wait_a(roles.bar(C::bKvEmpty + stage), phase ^ 1, roles.abort_flag, a.status));
                if (!ok) break;
                const uint32_t full = roles.bar(C::bKvFull + stage), dst = smem_u32(roles.smem) + stage * C::kTileBytes;
                if (lane == 0) mbar_expect_tx_a(full, static_cast<uint32_t>(C::kPanels) * lines * 128);
                __syncwarp();
                const CUtensorMap* pool = fresh ? (kv ? &map.V16 : &map.K16) : (kv ? &map.V : &map.K);
#pragma unroll
                for (int p = 0; p < C::kPanels; ++p) {
                    if (rows) tma_load_3d_a(dst + p * kPanelBytes + (lane << (shift + 7)), pool, full, p * 64, s.kvh, from);
                    if (fresh && lane == 0) tma_load_3d_a(dst + p * kPanelBytes + s.new_at * 128, kv ? &map.Vn : &map.Kn, full, p * 64, s.kvh, s.slot * a.T);
                }
                stage += kFirst == kLast ? 2 : 1;
                if (stage >= C::kStages) {
                    stage -= C::kStages;
                    phase ^= 1;
                }
            }
            id = next;
        }
    }
};

// ---- loader (one warp): shares out the work, and copies K and V, or K alone ----
template <class C>
__device__ __forceinline__ void load_role(const PagedArgs& a, const Maps& map, int row_blocks, const Roles& roles) {
    const int lane = threadIdx.x & 31;
    Work* s_work = roles.s_work;
    Slots& slots = *roles.slots;
    volatile int* abort_flag = roles.abort_flag;
    const auto bar = [&](int i) { return roles.bar(i); };
    Ring<C, 0, C::kTwoLoaders ? 0 : 1> ring;
    bool ok = true;
    // More rows than a CTA takes: neighbouring CTAs have the same keys at the same time, and a share of the rows each.
    const int cta = static_cast<int>(blockIdx.x) / row_blocks, n_ctas = static_cast<int>(gridDim.x) / row_blocks;
    int items;
    const int total = all_pieces<C::kSparse>(a, slots, row_blocks, items);
    const Shares shares(total, total <= kFewParts * items ? total : max(total / kLeastTiles, items), n_ctas);
    const int begin = shares.begin(cta), end = shares.begin(cta + 1);
    int slot_now = begin < end ? slot_at(slots, a.n_slots, begin) : 0, at = begin;
    for (uint32_t seq = 0;; ++seq) {
        const uint32_t place = seq % kQueue;
        __syncwarp();
        ok = __all_sync(0xffffffffu, ok && mbar_wait_a(bar(C::bWorkEmpty + static_cast<int>(place)), ((seq / kQueue) & 1) ^ 1, abort_flag, a.status));
        if (!ok) break;
        if (at >= end) {
            if (lane == 0) {
                s_work[place].valid = 0;
                arrive_a(bar(C::bWorkFull + static_cast<int>(place)));
            }
            break;
        }
        const Segment s = segment_at<C::kSparse>(a, slots, at, end, slot_now);
        const int row0 = static_cast<int>(blockIdx.x) % row_blocks * C::kRows, n_rows = min(s.n_rows - row0, C::kRows);
        const int part = 2 * static_cast<int>(blockIdx.x) + (at == begin ? 0 : 1);
        at = s.item_at + s.p_end;
        Meta* meta = a.meta + (static_cast<int64_t>(s.slot) * a.items_max + s.item) * row_blocks + static_cast<int>(blockIdx.x) % row_blocks;
        if (n_rows <= 0) {                   // (this slot has fewer rows)
            if (lane == 0 && s.p_begin == 0) meta->parts = 0;
            --seq;
            continue;
        }
        const bool all = s.p_begin == 0 && s.p_end == s.w.pieces;
        const Work work{1, s.slot, s.p_begin, s.p_end, s.w.new_tile, s.w.keys, s.w.n, row0, n_rows, s.kvh, s.token0, s.head0, all ? -1 : part,
                        s.w.len, s.token, s.w.new_at};
        if (lane == 0) {
            s_work[place] = work;
            arrive_a(bar(C::bWorkFull + static_cast<int>(place)));
            if (s.p_begin == 0)
                *meta = {all ? 1 : shares.owner(s.item_at + s.w.pieces - 1) - cta + 1, part, static_cast<int>(blockIdx.x), row_blocks, s.token0, s.head0, row0,
                         n_rows};
        }
        if (C::kSparse && seq == 0) grid_dependency_wait();
        ring.load(a, map, roles, work, ok);
    }
}

// ---- a warp that copies V, where the loader copies K alone ----
template <class C>
__device__ __forceinline__ void values_role(const PagedArgs& a, const Maps& map, const Roles& roles) {
    Ring<C, 1, 1> ring;
    bool ok = true;
    for (uint32_t seq = 0;; ++seq) {
        const Work* work = next_work<C>(a, roles, seq, ok);
        if (!ok || work->valid == 0) break;
        const Work s = *work;
        __syncwarp();
        if ((threadIdx.x & 31) == 0) arrive_a(roles.bar(C::bWorkEmpty + static_cast<int>(seq % kQueue)));
        if (C::kSparse && seq == 0) grid_dependency_wait();
        ring.load(a, map, roles, s, ok);
    }
}

// ---- a warp: query rows (TMA) ----
template <class C>
__device__ __forceinline__ void rows_role(const PagedArgs& a, const Maps& map, const Roles& roles) {
    const int lane = threadIdx.x & 31;
    bool ok = true;
    for (uint32_t seq = 0;; ++seq) {
        const Work* work = next_work<C>(a, roles, seq, ok);
        ok = __all_sync(0xffffffffu, ok && mbar_wait_a(roles.bar(C::bQEmpty), (seq & 1) ^ 1, roles.abort_flag, a.status));
        if (!ok || work->valid == 0) break;
        const Work s = *work;
        __syncwarp();
        if (lane == 0) {                                   // (rows past the item's are other slots', or zeros: nobody reads their outputs)
            arrive_a(roles.bar(C::bWorkEmpty + static_cast<int>(seq % kQueue)));
            mbar_expect_tx_a(roles.bar(C::bQFull), C::kQBytes);
#pragma unroll
            for (int i = 0; i < C::kQTiles; ++i)
#pragma unroll
                for (int p = 0; p < C::kPanels; ++p)
                    tma_load_3d_a(smem_u32(roles.smem) + C::kQ + (i * C::kPanels + p) * (C::kQRows * 128), &map.Q, roles.bar(C::bQFull), p * 64, s.head0,
                                  s.token0 + ((s.row0 + i * C::kQRows) >> a.g_shift));
        }
    }
}

// ---- a warp: which new tokens see which, and which of their values are not finite.  A lane has tokens lane and lane + 32. ----
template <int D, class C>
__device__ __forceinline__ void nodes_role(const PagedArgs& a, const Roles& roles) {
    constexpr int kVecs = D / 8;
    const int lane = threadIdx.x & 31;
    const int64_t pitch = static_cast<int64_t>(a.Hkv) * D;
    int* s_up = roles.s_up;
    bool ok = true;
    for (uint32_t seq = 0;; ++seq) {
        // (the place in the queue, and with it these buffers, is free when the softmax has left the segment kQueue before)
        const Work* work = next_work<C>(a, roles, seq, ok);
        if (!ok || work->valid == 0) break;
        const int n = work->p_end > work->new_tile ? work->n : 0, slot = work->slot, token = work->token;
        uint64_t* sees = roles.s_sees + (seq % kQueue) * kMaxTree;
        uint32_t* s_odd = roles.s_odd + 2 * (seq % kQueue);
        if (lane < 2) s_odd[lane] = 0u;
        __syncwarp();
        const uint4* value = reinterpret_cast<const uint4*>(a.Vnew + static_cast<int64_t>(slot) * a.T * pitch + work->kvh * D);
#pragma unroll 4
        for (int i = lane; i < n * kVecs; i += 32) {
            const uint4 y = value[(i / kVecs) * (pitch / 8) + i % kVecs];
            const uint32_t w[4] = {y.x, y.y, y.z, y.w};
            bool odd = false;
#pragma unroll
            for (int k = 0; k < 4; ++k) odd |= (w[k] & 0x7f80u) == 0x7f80u || (w[k] & 0x7f800000u) == 0x7f800000u;
            if (odd) atomicOr(&s_odd[i / kVecs >> 5], 1u << (i / kVecs & 31));
        }
        uint64_t mine[2] = {1ull << lane, 1ull << (lane + 32)};
        if (C::kSparse) {                                  // (the item's rows are one token's: it sees the tokens up to itself)
            sees[lane] = lane <= token ? 1ull : 0ull;
            sees[lane + 32] = lane + 32 <= token ? 1ull : 0ull;
        } else {
            // Ancestors: pointers to them are doubled.
            int to[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int t = lane + 32 * h;
                to[h] = -1;
                if (t < n) {
                    to[h] = a.parent != nullptr ? a.parent[static_cast<int64_t>(slot) * a.T + t] : t - 1;
                    if (to[h] < -1 || to[h] >= t) {
                        report(a.status, PULSAR_DEV_BAD_TREE);
                        to[h] = -1;
                    }
                }
            }
#pragma unroll 1
            for (int step = 1; step < n; step <<= 1) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    sees[lane + 32 * h] = mine[h];
                    s_up[lane + 32 * h] = to[h];
                }
                __syncwarp();
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    if (to[h] >= 0) {
                        mine[h] |= sees[to[h]];
                        to[h] = s_up[to[h]];
                    }
                __syncwarp();
            }
            if (C::kBySeen) {                              // turned round: the nodes that see a node
                uint32_t* seen = reinterpret_cast<uint32_t*>(sees);
#pragma unroll 4
                for (int node = 0; node < n; ++node) {
                    const uint32_t lo = __ballot_sync(0xffffffffu, ((mine[0] >> node) & 1ull) != 0ull);
                    const uint32_t hi = __ballot_sync(0xffffffffu, ((mine[1] >> node) & 1ull) != 0ull);
                    if (lane < 2) seen[2 * node + lane] = lane == 0 ? lo : hi;
                }
            } else {
                sees[lane] = mine[0];
                sees[lane + 32] = mine[1];
            }
        }
        __syncwarp();
        if (lane == 0) {
            arrive_a(roles.bar(C::bSees + static_cast<int>(seq % kQueue)));
            arrive_a(roles.bar(C::bWorkEmpty + static_cast<int>(seq % kQueue)));
        }
    }
}

}  // namespace pulsar
