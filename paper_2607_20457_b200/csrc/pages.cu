// Pages of a key/value cache: fork, copy, compact, append, summarise (include/pulsar.h has the definitions).
//
// Everything here moves bytes.  The bookkeeping is a pure function of table and lengths: which pages are free follows from the
// tables themselves, so there is no free list that a lost update could corrupt, and the result does not depend on the order
// in which threads run.
//
// Measured (a pass among others): fork of 8 slots 11 us, of 64 slots of 262 pages with half-filled last pages 20 to 22 (floor 7: the copied
// rows); compact of 64 trees of 64 nodes in 8 layers 7.8 (floor 3); key bounds of 131,072 rows of 8 heads 50 us, 5.65 TB/s, 0.87 of the
// copy rate.  The first two are latency: a fork reads lengths, then tables, and cannot hand out a page before all marks are set
// (three cluster barriers of 1 to 2 us each, with what lies between).
#include <algorithm>

#include "paged.cuh"

namespace pulsar {

namespace {

// ---------------------------------------------------------------------------------------------
// Fork: one cluster does the bookkeeping (its barrier is what separates marking, counting and handing out), a second launch
// copies rows.
// ---------------------------------------------------------------------------------------------
constexpr int kForkThreads = 1024;               // one per slot, at least
constexpr int kForkCtas = 8;
constexpr int kForkUnroll = 4;                   // table entries of a thread under way: 64 slots of 262 pages 23 -> 20 us

struct Copy {                                    // rows of page src that page dst receives
    int src, dst, rows, pad_;
};
struct ForkScratch {                             // in the workspace: n_copies | Copy [n_new] | entries in use [n_new] | a byte per page
    static constexpr size_t kHead = 256;
    static size_t used_at(int n_new) { return kHead + round_up(static_cast<size_t>(n_new) * sizeof(Copy), 256); }
    static size_t marks_at(int n_new) { return used_at(n_new) + round_up(static_cast<size_t>(n_new) * 4, 256); }
    static size_t bytes(int n_new, int n_pages) { return marks_at(n_new) + round_up(static_cast<size_t>(n_pages), 256); }
};

struct ForkArgs {
    const int32_t *table, *len, *parent;
    int n_slots, n_new, max_pages, n_pages, page_shift, reserve;
    int32_t *new_table, *new_len, *n_free;
    int32_t* n_copies;
    Copy* copies;
    int32_t* used;                               // entries of a slot of the result that are not -1
    uint8_t* marks;                              // 1: a slot of the result holds the page from its parent
    int32_t* status;
};

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void store_to_rank(void* p, int rank, int v) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(a), "r"(v) : "memory");
}

// Sum over the block's threads before this one; *total: over all of them.  sums: [32] in shared memory.
__device__ __forceinline__ int block_prefix(int x, int* sums, int* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int y = x;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int z = __shfl_up_sync(0xffffffffu, y, d);
        if (lane >= d) y += z;
    }
    __syncthreads();                             // (sums may still be read from the call before)
    if (lane == 31) sums[warp] = y;
    __syncthreads();
    if (warp == 0) {
        int w = lane < static_cast<int>(blockDim.x >> 5) ? sums[lane] : 0;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int z = __shfl_up_sync(0xffffffffu, w, d);
            if (lane >= d) w += z;
        }
        sums[lane] = w;
    }
    __syncthreads();
    *total = sums[31];
    return y - x + (warp > 0 ? sums[warp - 1] : 0);
}

// The last slot whose places begin at or before place r (slots that have none begin where their successor does).
__device__ __forceinline__ int last_at(const int* begins, int r) {
    int lo = 0, hi = kMaxSlots - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (begins[mid] <= r) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

__global__ void __launch_bounds__(kForkThreads) __cluster_dims__(kForkCtas, 1, 1)
fork_kernel(const __grid_constant__ ForkArgs a) {
    __shared__ int s_first[kMaxSlots];           // first child of an old slot
    __shared__ int s_parent[kMaxSlots], s_kept[kMaxSlots];    // (s_parent: -1 for an empty slot)
    __shared__ int s_base[kMaxSlots + 1];        // pages handed out to the slots before
    __shared__ int s_copy[kMaxSlots];            // place in the list of copies, or -1
    __shared__ int s_at[kMaxSlots];              // pages that come from the parents of the slots before
    __shared__ int s_sums[32], s_free[kForkCtas];
    const int t = threadIdx.x, rank = static_cast<int>(cluster_rank());
    const bool tell = rank == 0;
    grid_dependency_wait();
    grid_launch_dependents();

    // ---- marks cleared, and every CTA works out what each slot gets ----
    for (int64_t v = (static_cast<int64_t>(rank) * kForkThreads + t) * 16; v < a.n_pages; v += kForkCtas * kForkThreads * 16)
        *reinterpret_cast<uint4*>(a.marks + v) = make_uint4(0u, 0u, 0u, 0u);       // (padded to 256 bytes)
    s_first[t] = kMaxSlots;
    __syncthreads();
    int parent = -1, len = 0, kept = 0, need = 0;
    const int64_t capacity = static_cast<int64_t>(a.max_pages) << a.page_shift;
    if (t < a.n_new) {
        parent = a.parent != nullptr ? a.parent[t] : t;
        if (parent < -1 || parent >= a.n_slots) {
            if (tell) report(a.status, PULSAR_DEV_BAD_TREE);
            parent = -1;
        }
        if (parent >= 0) {
            atomicMin(&s_first[parent], t);
            len = checked_len(a.len[parent], capacity, tell, a.status);
            kept = (len + (1 << a.page_shift) - 1) >> a.page_shift;
            const int64_t want = (static_cast<int64_t>(len) + a.reserve + (1 << a.page_shift) - 1) >> a.page_shift;
            need = static_cast<int>(min(want, static_cast<int64_t>(a.max_pages)));
            if (want > a.max_pages && tell) report(a.status, PULSAR_DEV_NO_PAGES);
        }
    }
    __syncthreads();
    const int rows = len & ((1 << a.page_shift) - 1);
    const bool copied = parent >= 0 && rows != 0 && s_first[parent] != t;
    int n_fresh, n_copies, n_held;
    const int base = block_prefix(need - kept + (copied ? 1 : 0), s_sums, &n_fresh);
    const int copy_at = block_prefix(copied ? 1 : 0, s_sums, &n_copies);
    s_at[t] = block_prefix(kept, s_sums, &n_held);
    s_parent[t] = parent;
    s_kept[t] = kept;
    s_base[t] = base;
    s_copy[t] = copied ? copy_at : -1;
    if (t == 0) s_base[kMaxSlots] = n_fresh;
    if (tell && t < a.n_new) {
        a.new_len[t] = len;
        a.used[t] = need;
    }
    if (tell && t == 0) *a.n_copies = n_copies;
    cluster_sync();                              // the marks are clear in all CTAs' eyes

    // ---- entries that come from the parents ----
    for (uint64_t e0 = static_cast<uint32_t>(rank) * kForkThreads + t; e0 < static_cast<uint32_t>(n_held); e0 += kForkCtas * kForkThreads * kForkUnroll) {
        int page[kForkUnroll], slot[kForkUnroll], o[kForkUnroll];
#pragma unroll
        for (int k = 0; k < kForkUnroll; ++k) {
            const uint64_t e = e0 + static_cast<uint64_t>(k) * (kForkCtas * kForkThreads);
            slot[k] = -1;
            if (e >= static_cast<uint32_t>(n_held)) continue;
            slot[k] = last_at(s_at, static_cast<int>(e));
            o[k] = static_cast<int>(e) - s_at[slot[k]];
            page[k] = a.table[static_cast<int64_t>(s_parent[slot[k]]) * a.max_pages + o[k]];
        }
#pragma unroll
        for (int k = 0; k < kForkUnroll; ++k) {
            if (slot[k] < 0) continue;
            const int n = s_kept[slot[k]];
            if (page[k] < 0 || page[k] >= a.n_pages) {
                report(a.status, PULSAR_DEV_BAD_PAGE);
                page[k] = -1;
            }
            if (o[k] == n - 1 && s_copy[slot[k]] >= 0) {
                const int l = checked_len(a.len[s_parent[slot[k]]], capacity, false, nullptr);
                a.copies[s_copy[slot[k]]].src = page[k];
                a.copies[s_copy[slot[k]]].rows = l - ((n - 1) << a.page_shift);
            } else {
                a.new_table[static_cast<int64_t>(slot[k]) * a.max_pages + o[k]] = page[k];
                if (page[k] >= 0) a.marks[page[k]] = 1;
            }
        }
    }
    cluster_sync();

    // ---- free pages counted, 16 to a thread, in ranges that ascend with the CTA ----
    const int per_cta = ((a.n_pages + kForkCtas - 1) / kForkCtas + 15) / 16 * 16;
    const int begin = min(rank * per_cta, a.n_pages), end = min(begin + per_cta, a.n_pages);
    const auto free_at = [&](int p) -> uint32_t {                     // bit k: page p + k is free
        if (p >= end) return 0u;
        const uint4 m = *reinterpret_cast<const uint4*>(a.marks + p);
        const uint32_t w[4] = {m.x, m.y, m.z, m.w};
        uint32_t bits = 0;
#pragma unroll
        for (int k = 0; k < 16; ++k) bits |= ((w[k >> 2] >> (8 * (k & 3))) & 1u) << k;
        const int n = min(16, end - p);
        return ~bits & ((1u << n) - 1u);
    };
    int mine = 0, sum;
    for (int p = begin + t * 16; p < end; p += kForkThreads * 16) mine += __popc(free_at(p));
    (void)block_prefix(mine, s_sums, &sum);
    if (t < kForkCtas) store_to_rank(&s_free[rank], t, sum);
    cluster_sync();                              // (behind it nobody writes to another CTA's shared memory: CTAs leave as they finish)
    int before = 0, n_free = 0;
    for (int r = 0; r < kForkCtas; ++r) {
        if (r < rank) before += s_free[r];
        n_free += s_free[r];
    }

    // ---- and handed out: the r-th free page to the r-th place that needs one ----
    const auto give = [&](int r, int page) {
        const int lo = last_at(s_base, r);
        int o = r - s_base[lo] + s_kept[lo];
        if (s_copy[lo] >= 0) {
            --o;
            if (o == s_kept[lo] - 1) a.copies[s_copy[lo]].dst = page;
        }
        a.new_table[static_cast<int64_t>(lo) * a.max_pages + o] = page;
    };
    for (int p0 = begin; p0 < end && before < n_fresh; p0 += kForkThreads * 16) {
        const int p = p0 + t * 16;
        uint32_t bits = free_at(p);
        int n;
        int r = before + block_prefix(__popc(bits), s_sums, &n);
        for (; bits != 0 && r < n_fresh; bits &= bits - 1, ++r) give(r, p + __ffs(bits) - 1);
        before += n;
    }
    if (rank == 0) {
        if (n_free < n_fresh && t == 0) report(a.status, PULSAR_DEV_NO_PAGES);
        for (int r = n_free + t; r < n_fresh; r += kForkThreads) give(r, -1);
        if (t == 0) *a.n_free = max(n_free - n_fresh, 0);
    }
}

constexpr int kCopyThreads = 256, kCopyUnroll = 4;
constexpr int kCopyVecs = kCopyThreads * kCopyUnroll;

// K and V of the copied rows, layer by layer; and -1 in the entries that are not in use (CTAs with y = 1: in wide tables these are most of the
// output; the eight CTAs of the bookkeeping took 30 us for 64 slots of 8192 entries).
__global__ void __launch_bounds__(kCopyThreads)
fork_copy_kernel(const int32_t* __restrict__ n_copies, const Copy* __restrict__ copies, uint4* K, uint4* V, int n_layers, int n_pages,
                 int page_vecs, int row_vecs, const int32_t* __restrict__ used, int n_new, int max_pages, int32_t* new_table) {
    grid_dependency_wait();
    grid_launch_dependents();
    if (blockIdx.y == 1) {
        const int pieces = (max_pages + kCopyVecs - 1) / kCopyVecs;
        for (int64_t u = blockIdx.x; u < static_cast<int64_t>(n_new) * pieces; u += gridDim.x) {
            const int slot = static_cast<int>(u / pieces), o0 = static_cast<int>(u - static_cast<int64_t>(slot) * pieces) * kCopyVecs, n = used[slot];
#pragma unroll
            for (int j = 0; j < kCopyUnroll; ++j) {
                const int o = o0 + static_cast<int>(threadIdx.x) + j * kCopyThreads;
                if (o >= n && o < max_pages) new_table[static_cast<int64_t>(slot) * max_pages + o] = -1;
            }
        }
        return;
    }
    const int n = *n_copies, chunks = (page_vecs + kCopyVecs - 1) / kCopyVecs;
    const int64_t units = static_cast<int64_t>(n) * n_layers * chunks;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int64_t w = u / chunks;
        const int c = static_cast<int>(w / n_layers), layer = static_cast<int>(w - static_cast<int64_t>(c) * n_layers);
        const Copy copy = copies[c];
        if (copy.src < 0 || copy.dst < 0) continue;
        const int n_vecs = copy.rows * row_vecs, i0 = static_cast<int>(u - w * chunks) * kCopyVecs + threadIdx.x;
        const int64_t src = (static_cast<int64_t>(layer) * n_pages + copy.src) * page_vecs;
        const int64_t dst = (static_cast<int64_t>(layer) * n_pages + copy.dst) * page_vecs;
        uint4 k[kCopyUnroll], v[kCopyUnroll];
#pragma unroll
        for (int j = 0; j < kCopyUnroll; ++j)
            if (i0 + j * kCopyThreads < n_vecs) {
                k[j] = K[src + i0 + j * kCopyThreads];
                v[j] = V[src + i0 + j * kCopyThreads];
            }
#pragma unroll
        for (int j = 0; j < kCopyUnroll; ++j)
            if (i0 + j * kCopyThreads < n_vecs) {
                K[dst + i0 + j * kCopyThreads] = k[j];
                V[dst + i0 + j * kCopyThreads] = v[j];
            }
    }
}

// ---------------------------------------------------------------------------------------------
// Compact: rows len + accept[j] move to rows len + j.  A row may be the target of one move and the source of another, so a CTA
// holds its columns of all the slot's moving rows in registers before it writes any of them.
// ---------------------------------------------------------------------------------------------
// K and V of two layers at a time, so that a CTA waits for its rows once: 64 slots, 8 layers 9.4 -> 7.8 us.
constexpr int kCompactThreads = 256, kCompactUnroll = 4, kCompactPools = 4;

struct PoolArgs {
    uint4 *K, *V;
    int n_layers, n_pages, page_shift, row_vecs;
    const int32_t *table, *len;
    int max_pages;
};

// Vector index of a slot's row in layer 0, or -1 (reported) where there is no page for it.
__device__ __forceinline__ int64_t row_at(const PoolArgs& p, int slot, int64_t row, int32_t* status) {
    const int64_t o = row >> p.page_shift;
    if (o >= p.max_pages) {
        report(status, PULSAR_DEV_BAD_LENGTH);
        return -1;
    }
    const int page = p.table[static_cast<int64_t>(slot) * p.max_pages + o];
    if (page < 0 || page >= p.n_pages) {
        report(status, PULSAR_DEV_BAD_PAGE);
        return -1;
    }
    return ((static_cast<int64_t>(page) << p.page_shift) + (row & ((1 << p.page_shift) - 1))) * p.row_vecs;
}

__global__ void __launch_bounds__(kCompactThreads)
compact_kernel(const __grid_constant__ PoolArgs p, const int32_t* __restrict__ accept, int T, int32_t* new_len, int32_t* status) {
    __shared__ int64_t s_src[kMaxTree], s_dst[kMaxTree];
    __shared__ int s_n, s_first;
    const int slot = blockIdx.x, t = threadIdx.x;
    grid_dependency_wait();
    grid_launch_dependents();
    const bool tell = blockIdx.y == 0 && blockIdx.z == 0;
    const int len = checked_len(p.len[slot], static_cast<int64_t>(p.max_pages) << p.page_shift, tell && t == 0, status);
    if (t < 32) {
        // the list ends at the first entry that is not a node after the one before it
        int n = 0, first = 0;
        bool bad = false;
        for (int j0 = 0; j0 < T; j0 += 32) {
            const int j = j0 + t;
            const int x = j < T ? accept[static_cast<int64_t>(slot) * T + j] : -1;
            const int y = j > 0 && j < T ? accept[static_cast<int64_t>(slot) * T + j - 1] : -1;
            const uint32_t stops = __ballot_sync(0xffffffffu, !(x >= 0 && x < T && x > y));
            const uint32_t moved = __ballot_sync(0xffffffffu, x != j);
            bad |= __any_sync(0xffffffffu, j < T && x != -1 && !(x < T && x > y));
            bad |= __any_sync(0xffffffffu, x >= 0 && j > 0 && j < T && y < 0);
            if (n == j0) {
                n = j0 + (stops != 0u ? __ffs(stops) - 1 : 32);
                if (first == j0) first = j0 + (moved != 0u ? __ffs(moved) - 1 : 32);
            }
        }
        n = min(n, T);
        if (t == 0) {
            s_n = n;
            s_first = min(first, n);             // nodes 0 .. first-1 stand where they belong
            if (bad && tell) report(status, PULSAR_DEV_BAD_TREE);
            if (tell) new_len[slot] = static_cast<int>(min(static_cast<int64_t>(len) + n, static_cast<int64_t>(p.max_pages) << p.page_shift));
        }
    }
    __syncthreads();
    const int n = s_n - s_first;
    if (n == 0) return;
    if (t < n) {
        const int j = s_first + t;
        s_src[t] = row_at(p, slot, static_cast<int64_t>(len) + accept[static_cast<int64_t>(slot) * T + j], status);
        s_dst[t] = row_at(p, slot, static_cast<int64_t>(len) + j, status);
    }
    __syncthreads();
    const int cols = kCompactThreads * kCompactUnroll / n;               // columns that a pass of the CTA holds, of kCompactPools pools
    const int64_t layer_vecs = (static_cast<int64_t>(p.n_pages) << p.page_shift) * p.row_vecs;
    for (int l0 = blockIdx.y * kCompactPools; l0 < 2 * p.n_layers; l0 += gridDim.y * kCompactPools) {
        for (int c0 = blockIdx.z * cols; c0 < p.row_vecs; c0 += gridDim.z * cols) {
            const int w = min(cols, p.row_vecs - c0);
            uint4 x[kCompactPools][kCompactUnroll];
#pragma unroll
            for (int l = 0; l < kCompactPools; ++l) {
                const uint4* base = ((l0 + l) & 1 ? p.V : p.K) + ((l0 + l) >> 1) * layer_vecs;
#pragma unroll
                for (int u = 0; u < kCompactUnroll; ++u) {
                    const int i = t + u * kCompactThreads, j = i / w;
                    if (l0 + l < 2 * p.n_layers && j < n && s_src[j] >= 0) x[l][u] = base[s_src[j] + c0 + (i - j * w)];
                }
            }
            __syncthreads();
#pragma unroll
            for (int l = 0; l < kCompactPools; ++l) {
                uint4* base = ((l0 + l) & 1 ? p.V : p.K) + ((l0 + l) >> 1) * layer_vecs;
#pragma unroll
                for (int u = 0; u < kCompactUnroll; ++u) {
                    const int i = t + u * kCompactThreads, j = i / w;
                    if (l0 + l < 2 * p.n_layers && j < n && s_src[j] >= 0 && s_dst[j] >= 0) base[s_dst[j] + c0 + (i - j * w)] = x[l][u];
                }
            }
            // (the next pass has columns of its own: nothing to wait for)
        }
    }
}

// ---------------------------------------------------------------------------------------------
// Append: packed rows into one layer's pages.
// ---------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(kCopyThreads)
append_pages_kernel(const uint4* __restrict__ Knew, const uint4* __restrict__ Vnew, int T, const int32_t* __restrict__ n_new,
                    const __grid_constant__ PoolArgs p, int32_t* status) {
    const int slot = blockIdx.y;
    grid_dependency_wait();
    grid_launch_dependents();
    const bool tell = blockIdx.x == 0 && threadIdx.x == 0;
    const int64_t capacity = static_cast<int64_t>(p.max_pages) << p.page_shift;
    const int len = checked_len(p.len[slot], capacity, tell, status);
    int n = n_new != nullptr ? min(max(n_new[slot], 0), T) : T;
    if (n > capacity - len) {
        if (tell) report(status, PULSAR_DEV_BAD_LENGTH);
        n = static_cast<int>(capacity - len);
    }
    const int64_t vecs = static_cast<int64_t>(n) * p.row_vecs, from = static_cast<int64_t>(slot) * T * p.row_vecs;
    for (int64_t i0 = static_cast<int64_t>(blockIdx.x) * kCopyVecs; i0 < vecs; i0 += static_cast<int64_t>(gridDim.x) * kCopyVecs) {
        uint4 k[kCopyUnroll], v[kCopyUnroll];
#pragma unroll
        for (int u = 0; u < kCopyUnroll; ++u) {
            const int64_t i = i0 + threadIdx.x + u * kCopyThreads;
            if (i < vecs) {
                k[u] = Knew[from + i];
                v[u] = Vnew[from + i];
            }
        }
#pragma unroll
        for (int u = 0; u < kCopyUnroll; ++u) {
            const int64_t i = i0 + threadIdx.x + u * kCopyThreads;
            if (i >= vecs) continue;
            const int64_t row = i / p.row_vecs, to = row_at(p, slot, len + row, status);
            if (to < 0) continue;
            p.K[to + (i - row * p.row_vecs)] = k[u];
            p.V[to + (i - row * p.row_vecs)] = v[u];
        }
    }
}

// ---------------------------------------------------------------------------------------------
// Summarise: smallest and largest component over a page's keys.  bf16 values are compared as they are, so the bounds are exact.
// ---------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t min2(uint32_t a, uint32_t b) {
    uint32_t c;
    asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(c) : "r"(a), "r"(b));
    return c;
}
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
    uint32_t c;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(c) : "r"(a), "r"(b));
    return c;
}
__device__ __forceinline__ uint4 min8(const uint4& a, const uint4& b) {
    return make_uint4(min2(a.x, b.x), min2(a.y, b.y), min2(a.z, b.z), min2(a.w, b.w));
}
__device__ __forceinline__ uint4 max8(const uint4& a, const uint4& b) {
    return make_uint4(max2(a.x, b.x), max2(a.y, b.y), max2(a.z, b.z), max2(a.w, b.w));
}

// A page's rows of one strip (32 vectors of a row) are a warp's work: kSumRows rows' vectors under way per lane, nothing shared and nobody to
// wait for.  (A CTA per page and strip with the rows shared out between its warps and two barriers: 88 us for 131,072 rows of 8 heads, 3.3
// TB/s.)  Pages of 64 and 128 rows of few slots leave warps idle that way, so two or four neighbouring warps share such a page and the first
// one joins them.
constexpr int kSumThreads = 256, kSumRows = 16;
__global__ void __launch_bounds__(kSumThreads)
summarize_kernel(const uint4* __restrict__ K, int n_pages, int page_shift, int row_vecs, int head_shift, int share_shift,
                 const int32_t* __restrict__ table, const int32_t* __restrict__ row_begin, const int32_t* __restrict__ row_end,
                 int max_pages, uint4* __restrict__ summary, int32_t* status) {
    __shared__ uint4 s_min[kSumThreads], s_max[kSumThreads];
    const int slot = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    grid_dependency_wait();
    grid_launch_dependents();
    const int64_t capacity = static_cast<int64_t>(max_pages) << page_shift;
    const bool tell = blockIdx.x == 0 && blockIdx.z == 0 && threadIdx.x == 0;
    const int first = (row_begin != nullptr ? checked_len(row_begin[slot], capacity, tell, status) : 0) >> page_shift;
    const int last = checked_len(row_end[slot], capacity, tell, status) >> page_shift;       // full pages
    const uint32_t strips = static_cast<uint32_t>(row_vecs + 31) / 32;
    const int together = (kSumThreads / 32) >> share_shift;                                  // units of a CTA
    const int part = warp & ((1 << share_shift) - 1), rows = (1 << page_shift) >> share_shift;
    const uint32_t units = last > first ? static_cast<uint32_t>(last - first) * strips : 0u;
    for (uint32_t u0 = blockIdx.x * together; u0 < units; u0 += gridDim.x * together) {
        const uint32_t u = u0 + (warp >> share_shift), o = u / strips;
        const int v = static_cast<int>(u - o * strips) * 32 + lane;
        const int page = u < units ? table[static_cast<int64_t>(slot) * max_pages + first + static_cast<int>(o)] : -1;
        const bool known = page >= 0 && page < n_pages;
        if (u < units && !known && lane == 0) report(status, PULSAR_DEV_BAD_PAGE);
        const int64_t at = static_cast<int64_t>(blockIdx.z) * n_pages + (known ? page : 0);
        uint4 lo, hi;
        if (known && v < row_vecs) {
            const uint4* src = K + ((at << page_shift) + part * rows) * row_vecs + v;
            lo = hi = *src;
            for (int r0 = 0; r0 < rows; r0 += kSumRows) {
                uint4 x[kSumRows];
#pragma unroll
                for (int r = 0; r < kSumRows; ++r) x[r] = __ldcs(src + static_cast<int64_t>(r0 + min(r, rows - 1)) * row_vecs);
#pragma unroll
                for (int r = 0; r < kSumRows; ++r) {
                    lo = min8(lo, x[r]);
                    hi = max8(hi, x[r]);
                }
            }
        }
        if (share_shift > 0) {
            s_min[threadIdx.x] = lo;
            s_max[threadIdx.x] = hi;
            __syncthreads();
            for (int w = 1; w < 1 << share_shift; ++w)
                if (part == 0) {
                    lo = min8(lo, s_min[threadIdx.x + 32 * w]);
                    hi = max8(hi, s_max[threadIdx.x + 32 * w]);
                }
            __syncthreads();
        }
        if (known && v < row_vecs && part == 0) {
            const int head = v >> head_shift, in_head = v - (head << head_shift);
            uint4* to = summary + at * 2 * row_vecs + (static_cast<int64_t>(2 * head) << head_shift) + in_head;
            to[0] = lo;
            to[static_cast<int64_t>(1) << head_shift] = hi;
        }
    }
}

}  // namespace
}  // namespace pulsar

using namespace pulsar;

extern "C" size_t pulsar_pages_fork_workspace_bytes(int32_t n_new, int32_t n_pages) {
    if (n_new < 1 || n_new > kMaxSlots || n_pages < 1 || n_pages >= (1 << 24)) return 0;
    return ForkScratch::bytes(n_new, n_pages);
}

extern "C" int32_t pulsar_pages_fork(const int32_t* page_table, const int32_t* cache_len, int32_t n_slots, int32_t max_pages,
                                     const int32_t* parent, int32_t n_new, uint16_t* K_pages, uint16_t* V_pages, int32_t n_layers,
                                     int32_t n_pages, int32_t page_size, int32_t Hkv, int32_t d, int32_t reserve_rows,
                                     int32_t* new_table, int32_t* new_len, int32_t* n_free, void* workspace, size_t workspace_bytes,
                                     int32_t* device_status, void* stream) {
    if (!pool_ok(n_layers, n_pages, page_size, Hkv, d, n_slots, max_pages) || n_new < 1 || n_new > kMaxSlots || reserve_rows < 0 ||
        static_cast<int64_t>(n_new) * max_pages >= (int64_t{1} << 31))
        return PULSAR_ERR_SHAPE;
    if (page_table == nullptr || cache_len == nullptr || K_pages == nullptr || V_pages == nullptr || new_table == nullptr ||
        new_len == nullptr || n_free == nullptr || workspace == nullptr || (parent == nullptr && n_new != n_slots))
        return PULSAR_ERR_INVALID_ARG;
    const size_t table_bytes = 4 * static_cast<size_t>(max_pages);
    const size_t pool = pool_bytes(n_layers, n_pages, page_size, Hkv, d), scratch = ForkScratch::bytes(n_new, n_pages);
    const Tensors in = {{page_table, n_slots * table_bytes}, {cache_len, 4u * n_slots}, {parent, 4u * n_new}};
    const Tensors out = {{new_table, n_new * table_bytes}, {new_len, 4u * n_new}, {n_free, 4u}, {K_pages, pool}, {V_pages, pool}, {device_status, 4u}};
    if (!apart(out, in)) return PULSAR_ERR_INVALID_ARG;
    if (!aligned(K_pages, 16) || !aligned(V_pages, 16) || !aligned(workspace, 256) || !aligned(page_table, 4) || !aligned(cache_len, 4) ||
        !aligned(parent, 4) || !aligned(new_table, 4) || !aligned(new_len, 4) || !aligned(n_free, 4))
        return PULSAR_ERR_ALIGNMENT;
    if (workspace_bytes < scratch) return PULSAR_ERR_WORKSPACE;
    if (!apart({{workspace, scratch}}, in) || !apart({{workspace, scratch}}, out)) return PULSAR_ERR_INVALID_ARG;
    if (const int32_t rc = check_device(); rc != PULSAR_OK) return rc;

    ForkArgs a{};
    a.table = page_table;
    a.len = cache_len;
    a.parent = parent;
    a.n_slots = n_slots;
    a.n_new = n_new;
    a.max_pages = max_pages;
    a.n_pages = n_pages;
    a.page_shift = log2_exact(page_size);
    a.reserve = reserve_rows;
    a.new_table = new_table;
    a.new_len = new_len;
    a.n_free = n_free;
    a.n_copies = static_cast<int32_t*>(workspace);
    a.copies = reinterpret_cast<Copy*>(static_cast<uint8_t*>(workspace) + ForkScratch::kHead);
    a.used = reinterpret_cast<int32_t*>(static_cast<uint8_t*>(workspace) + ForkScratch::used_at(n_new));
    a.marks = static_cast<uint8_t*>(workspace) + ForkScratch::marks_at(n_new);
    a.status = device_status;
    auto st = static_cast<cudaStream_t>(stream);
    PULSAR_CUDA_OK(launch_kernel(fork_kernel, dim3(kForkCtas), dim3(kForkThreads), 0, st, true, a));
    count_launch();
    const int row_vecs = Hkv * d / 8;
    const int64_t units = static_cast<int64_t>(n_new) * n_layers * ((static_cast<int64_t>(row_vecs) * page_size + kCopyVecs - 1) / kCopyVecs);
    const unsigned ctas = static_cast<unsigned>(std::min<int64_t>(units, 8 * sm_count()));
    PULSAR_CUDA_OK(launch_kernel(fork_copy_kernel, dim3(ctas, 2), dim3(kCopyThreads), 0, st, true, a.n_copies, a.copies,
                                 reinterpret_cast<uint4*>(K_pages), reinterpret_cast<uint4*>(V_pages), n_layers, n_pages,
                                 row_vecs * page_size, row_vecs, a.used, n_new, max_pages, new_table));
    count_launch();
    return PULSAR_OK;
}

namespace {
PoolArgs pool_args(const uint16_t* K, const uint16_t* V, int32_t n_layers, int32_t n_pages, int32_t page_size, int32_t Hkv, int32_t d,
                   const int32_t* table, const int32_t* len, int32_t max_pages) {
    PoolArgs p{};
    p.K = reinterpret_cast<uint4*>(const_cast<uint16_t*>(K));
    p.V = reinterpret_cast<uint4*>(const_cast<uint16_t*>(V));
    p.n_layers = n_layers;
    p.n_pages = n_pages;
    p.page_shift = log2_exact(page_size);
    p.row_vecs = Hkv * d / 8;
    p.table = table;
    p.len = len;
    p.max_pages = max_pages;
    return p;
}
}  // namespace

extern "C" int32_t pulsar_pages_compact(uint16_t* K_pages, uint16_t* V_pages, int32_t n_layers, int32_t n_pages, int32_t page_size,
                                        int32_t Hkv, int32_t d, const int32_t* page_table, const int32_t* cache_len, int32_t n_slots,
                                        int32_t max_pages, const int32_t* accept, int32_t T, int32_t* new_len, int32_t* device_status,
                                        void* stream) {
    if (!pool_ok(n_layers, n_pages, page_size, Hkv, d, n_slots, max_pages) || T < 1 || T > kMaxTree) return PULSAR_ERR_SHAPE;
    if (K_pages == nullptr || V_pages == nullptr || page_table == nullptr || cache_len == nullptr || accept == nullptr || new_len == nullptr)
        return PULSAR_ERR_INVALID_ARG;
    const size_t pool = pool_bytes(n_layers, n_pages, page_size, Hkv, d), slots = static_cast<size_t>(n_slots);
    if (!apart({{K_pages, pool}, {V_pages, pool}, {new_len, 4 * slots}, {device_status, 4u}},
               {{page_table, 4 * slots * max_pages}, {cache_len, 4 * slots}, {accept, 4 * slots * T}}))
        return PULSAR_ERR_INVALID_ARG;
    if (!aligned(K_pages, 16) || !aligned(V_pages, 16) || !aligned(page_table, 4) || !aligned(cache_len, 4) || !aligned(accept, 4) ||
        !aligned(new_len, 4))
        return PULSAR_ERR_ALIGNMENT;
    if (const int32_t rc = check_device(); rc != PULSAR_OK) return rc;
    const PoolArgs p = pool_args(K_pages, V_pages, n_layers, n_pages, page_size, Hkv, d, page_table, cache_len, max_pages);
    // Eight accepted nodes of a row of 128 vectors fill a pass; more of either take several, shared out as far as the chip has room.
    const int64_t groups = (2 * static_cast<int64_t>(n_layers) + kCompactPools - 1) / kCompactPools;
    const int64_t strips = (static_cast<int64_t>(p.row_vecs) * std::min(T, 8) + kCompactThreads * kCompactUnroll - 1) / (kCompactThreads * kCompactUnroll);
    PULSAR_CUDA_OK(launch_kernel(compact_kernel, dim3(n_slots, static_cast<unsigned>(std::min<int64_t>(groups, 65535)), static_cast<unsigned>(strips)),
                                 dim3(kCompactThreads), 0, static_cast<cudaStream_t>(stream), true, p, accept, T, new_len, device_status));
    count_launch();
    return PULSAR_OK;
}

extern "C" int32_t pulsar_pages_append(const uint16_t* Knew, const uint16_t* Vnew, int32_t T, const int32_t* n_new, uint16_t* K_pages,
                                       uint16_t* V_pages, int32_t n_pages, int32_t page_size, int32_t Hkv, int32_t d,
                                       const int32_t* page_table, const int32_t* cache_len, int32_t n_slots, int32_t max_pages,
                                       int32_t* device_status, void* stream) {
    if (!pool_ok(1, n_pages, page_size, Hkv, d, n_slots, max_pages) || T < 0) return PULSAR_ERR_SHAPE;
    if (K_pages == nullptr || V_pages == nullptr || page_table == nullptr || cache_len == nullptr ||
        (T > 0 && (Knew == nullptr || Vnew == nullptr)))
        return PULSAR_ERR_INVALID_ARG;
    const size_t slots = static_cast<size_t>(n_slots), fresh = slots * T * Hkv * d * 2, pool = pool_bytes(1, n_pages, page_size, Hkv, d);
    if (!apart({{K_pages, pool}, {V_pages, pool}, {device_status, 4u}},
               {{Knew, fresh}, {Vnew, fresh}, {n_new, 4 * slots}, {page_table, 4 * slots * max_pages}, {cache_len, 4 * slots}}))
        return PULSAR_ERR_INVALID_ARG;
    if (!aligned(K_pages, 16) || !aligned(V_pages, 16) || !aligned(Knew, 16) || !aligned(Vnew, 16) || !aligned(page_table, 4) ||
        !aligned(cache_len, 4) || !aligned(n_new, 4))
        return PULSAR_ERR_ALIGNMENT;
    if (const int32_t rc = check_device(); rc != PULSAR_OK) return rc;
    if (T == 0) return PULSAR_OK;
    const PoolArgs p = pool_args(K_pages, V_pages, 1, n_pages, page_size, Hkv, d, page_table, cache_len, max_pages);
    const int64_t chunks = (static_cast<int64_t>(T) * p.row_vecs + kCopyVecs - 1) / kCopyVecs;
    const unsigned ctas = static_cast<unsigned>(std::min<int64_t>(chunks, std::max(1, 16 * sm_count() / n_slots)));
    PULSAR_CUDA_OK(launch_kernel(append_pages_kernel, dim3(ctas, n_slots), dim3(kCopyThreads), 0, static_cast<cudaStream_t>(stream), true,
                                 reinterpret_cast<const uint4*>(Knew), reinterpret_cast<const uint4*>(Vnew), T, n_new, p, device_status));
    count_launch();
    return PULSAR_OK;
}

extern "C" int32_t pulsar_pages_summarize(const uint16_t* K_pages, int32_t n_layers, int32_t n_pages, int32_t page_size, int32_t Hkv,
                                          int32_t d, const int32_t* page_table, const int32_t* row_begin, const int32_t* row_end,
                                          int32_t n_slots, int32_t max_pages, uint16_t* summary, int32_t* device_status, void* stream) {
    // (the units of a slot are counted in 32 bits)
    if (!pool_ok(n_layers, n_pages, page_size, Hkv, d, n_slots, max_pages) || n_layers > 65535 ||
        static_cast<int64_t>(max_pages) * ((Hkv * d / 8 + 31) / 32) >= (int64_t{1} << 31))
        return PULSAR_ERR_SHAPE;
    if (K_pages == nullptr || page_table == nullptr || row_end == nullptr || summary == nullptr) return PULSAR_ERR_INVALID_ARG;
    const size_t pool = pool_bytes(n_layers, n_pages, page_size, Hkv, d), slots = static_cast<size_t>(n_slots);
    if (!apart({{summary, pool / page_size * 2}, {device_status, 4u}},
               {{K_pages, pool}, {page_table, 4 * slots * max_pages}, {row_begin, 4 * slots}, {row_end, 4 * slots}}))
        return PULSAR_ERR_INVALID_ARG;
    if (!aligned(K_pages, 16) || !aligned(summary, 16) || !aligned(page_table, 4) || !aligned(row_begin, 4) || !aligned(row_end, 4))
        return PULSAR_ERR_ALIGNMENT;
    if (const int32_t rc = check_device(); rc != PULSAR_OK) return rc;
    const int row_vecs = Hkv * d / 8;
    // Warps of a page: one per 16 rows where there are few pages and strips, else one.  CTAs: eight warps each, as many as the chip holds at
    // a time and a few rounds more, so that the last ones end together.
    const int64_t units = static_cast<int64_t>(max_pages) * ((row_vecs + 31) / 32) * n_slots * n_layers, warps = 64 * static_cast<int64_t>(sm_count());
    int share = 0;
    while (share < 3 && (page_size >> share) > kSumRows && (units << share) < warps) ++share;
    const int64_t ctas = ((static_cast<int64_t>(max_pages) * ((row_vecs + 31) / 32) << share) + 7) / 8;
    const int64_t most = std::max<int64_t>(1, 32 * sm_count() / (static_cast<int64_t>(n_slots) * n_layers));
    PULSAR_CUDA_OK(launch_kernel(summarize_kernel, dim3(static_cast<unsigned>(std::min(ctas, most)), n_slots, n_layers), dim3(kSumThreads), 0,
                                 static_cast<cudaStream_t>(stream), true, reinterpret_cast<const uint4*>(K_pages), n_pages, log2_exact(page_size), row_vecs,
                                 log2_exact(d / 8), share, page_table, row_begin, row_end, max_pages, reinterpret_cast<uint4*>(summary),
                                 device_status));
    count_launch();
    return PULSAR_OK;
}
