// Attention over a paged key/value cache: drafted trees (every cached row) and selected pages (include/pulsar.h).
//
// Lengths live on the device, so a launch does not know how much work it has.  A work item is the query rows of one KV head (tree: nodes
// x heads of the group; selected pages: the group's heads of one token) against a list of keys, cut into tiles of 128.  Every CTA adds
// up the tiles of all slots, takes an equal share of them, whichever items they belong to, and leaves a partial (normalised output and
// l = ln sum exp) where it holds an item only in part; a second launch joins those (paged_merge.cu).  This file has the selection of
// the pages and the entry points.
#include <algorithm>

#include "mma.cuh"
#include "paged.cuh"

namespace pulsar {

namespace {

// ---------------------------------------------------------------------------------------------
// Scores of the full pages and the k best.
//
// sum_j (q_j > 0 ? q_j max_j : q_j min_j) is one product of length 2 d: the negative parts of the query with the smallest components, the
// positive ones with the largest.  The tensor cores form it for all pages and rows in fp32, which is what the memory's rate leaves
// time for (in float64 on the FMA pipe 16 slots of 45,000 rows took 70 us); the ranking is that of the float64 scores all the
// same: a page whose fp32 score lies further from the k-th than both can be off is in or out, and the few others are formed again in
// float64.  With the selection's launch the attention's starts, and waits for the list alone.
//
// Measured with the attention: one slot of 6001 rows, 32 pages of 16 19 us; of 131,072, 64 pages of 32 27; 16 slots of up to 45,011
// with 4 tokens, 48 pages of 16 50 us (cold and one by one the scores take 17, the ranking 14, the attention 27, the joining 7).
// A slot's ranking is a chain of steps over the block (largest and smallest, bins, border, places), each a microsecond.
// ---------------------------------------------------------------------------------------------
constexpr int kScoreThreads = 128, kScorePages = 64;     // of a CTA: 16 pages per warp
constexpr int kScoreRows = 32;                           // query rows in shared memory at a time

struct SelectArgs {
    const uint16_t *Q, *summary;
    const int32_t *table, *len, *n_draft;
    int T, Hq, Hkv, g_shift, page_shift, n_pages, max_pages, k, sink, window;
    float* score;                                // [n_slots, T, Hkv, max_pages] in fp32
    uint64_t* exact;                             // [n_slots, T, Hkv, max_pages] of the pages that are ranked in float64
    float* most;                                 // [n_slots, Hkv, blocks of kScorePages pages] largest magnitude of a bound
    int32_t *sel, *list;                         // [n_slots, T, Hkv, k], [n_slots, T, Hkv, k + 1]
    int32_t* status;
};

__device__ __forceinline__ float max_nan(float a, float b) {
    float c;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(c) : "f"(a), "f"(b));
    return c;
}
__device__ __forceinline__ uint32_t max_abs2(uint32_t a, uint32_t b) {     // of two bf16 each; NaN counts as nothing
    uint32_t c;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(c) : "r"(a), "r"(b & 0x7fff7fffu));
    return c;
}

template <int D>
__global__ void __launch_bounds__(kScoreThreads)
page_score_kernel(const __grid_constant__ SelectArgs a, int blocks) {
    constexpr int kChunks = 2 * D / 32;          // of 32 products: a lane has 8 consecutive ones, 16 bytes, of two pages
    constexpr int kPitch = 2 * D + 32;           // of a query row in shared memory: two rows' vectors fill the banks
    __shared__ __align__(16) uint16_t s_q[kScoreRows * kPitch];
    __shared__ float s_most[kScoreThreads / 32];
    const int slot = blockIdx.z, kvh = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gid = lane >> 2, tig = lane & 3;
    grid_dependency_wait();
    grid_launch_dependents();
    int b0 = blockIdx.x * kScorePages, id[2];    // (ids are asked for beside the length: whether there are such pages shows later)
    const auto ids = [&](int from) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int b = from + warp * 16 + gid + 8 * h;
            id[h] = b < a.max_pages ? a.table[static_cast<int64_t>(slot) * a.max_pages + b] : -1;
        }
    };
    ids(b0);
    const int len = checked_len(a.len[slot], static_cast<int64_t>(a.max_pages) << a.page_shift, false, nullptr);
    const int full = len >> a.page_shift;
    if (full <= a.k) return;                     // (all pages are taken as they are)
    const int n = a.n_draft != nullptr ? min(max(a.n_draft[slot], 0), a.T) : a.T, g = 1 << a.g_shift, rows = n * g;
    if (rows == 0) return;

    for (; b0 < full; b0 += static_cast<int>(gridDim.x) * kScorePages) {
        const int page0 = b0 + warp * 16 + gid;
        // ---- the bounds of pages gid and gid + 8 of the warp's 16, as A fragments: products are summed in the order of these vectors ----
        uint4 f[2][kChunks];
        bool known[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int b = page0 + 8 * h, page = b < full ? id[h] : -1;
            known[h] = page >= 0 && page < a.n_pages;
            if (b < full && !known[h] && tig == 0) report(a.status, PULSAR_DEV_BAD_PAGE);
            const uint4* src = reinterpret_cast<const uint4*>(a.summary + (static_cast<int64_t>(known[h] ? page : 0) * a.Hkv + kvh) * 2 * D) + tig;
#pragma unroll
            for (int c = 0; c < kChunks; ++c) f[h][c] = known[h] ? src[4 * c] : make_uint4(0u, 0u, 0u, 0u);
        }
        float best[2];                               // g = 16: of the row tile before
        for (int r0 = 0; r0 < rows; r0 += kScoreRows) {
            if (r0 > 0) __syncthreads();
            for (int i = threadIdx.x; i < kScoreRows * (D / 2); i += kScoreThreads) {
                const int r = i / (D / 2), j = i % (D / 2);
                uint32_t x = 0, up = 0;
                if (r0 + r < rows) {
                    x = reinterpret_cast<const uint32_t*>(a.Q + row_of(slot * a.T, kvh << a.g_shift, r0, r, a.g_shift, a.Hq) * D)[j];
                    up = (__uint_as_float(x << 16) > 0.f ? 0xffffu : 0u) | (__uint_as_float(x & 0xffff0000u) > 0.f ? 0xffff0000u : 0u);
                }
                uint32_t* to = reinterpret_cast<uint32_t*>(s_q + r * kPitch);
                to[j] = x & ~up;
                to[D / 2 + j] = x & up;
            }
            if (r0 == 0) {                           // the largest magnitude of a bound
                uint32_t m = 0;
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int c = 0; c < kChunks; ++c)
                        m = max_abs2(max_abs2(max_abs2(max_abs2(m, f[h][c].x), f[h][c].y), f[h][c].z), f[h][c].w);
                float most = fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
                if (lane == 0) s_most[warp] = most;
            }
            __syncthreads();
            if (r0 == 0 && threadIdx.x == 0)
                a.most[(static_cast<int64_t>(slot) * a.Hkv + kvh) * blocks + b0 / kScorePages] = fmaxf(fmaxf(s_most[0], s_most[1]), fmaxf(s_most[2], s_most[3]));
            for (int t = 0; t < min(kScoreRows, rows - r0); t += 8) {
                float c[4] = {0.f, 0.f, 0.f, 0.f}, c2[4] = {0.f, 0.f, 0.f, 0.f};       // two chains of products
                const uint4* src = reinterpret_cast<const uint4*>(s_q + (t + gid) * kPitch) + tig;
#pragma unroll
                for (int i = 0; i < kChunks; ++i) {
                    const uint4 q = src[4 * i];
                    const uint32_t lo[4] = {f[0][i].x, f[1][i].x, f[0][i].y, f[1][i].y}, hi[4] = {f[0][i].z, f[1][i].z, f[0][i].w, f[1][i].w};
                    mma_bf16(c, lo, q.x, q.y);
                    mma_bf16(c2, hi, q.z, q.w);
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float x = c[2 * h] + c2[2 * h], y = c[2 * h + 1] + c2[2 * h + 1];  // rows r0 + t + 2 tig and the next
                    const int b = page0 + 8 * h, r = r0 + t + 2 * tig;
                    const auto put = [&](int row, float z) {
                        if (b < full && row < rows)
                            a.score[(static_cast<int64_t>(slot * a.T + (row >> a.g_shift)) * a.Hkv + kvh) * a.max_pages + b] = known[h] ? z : -INFINITY;
                    };
                    if (g == 1) {
                        put(r, x);
                        put(r + 1, y);
                        continue;
                    }
                    x = max_nan(x, y);
                    if (g >= 4) x = max_nan(x, __shfl_xor_sync(0xffffffffu, x, 1));
                    if (g >= 8) x = max_nan(x, __shfl_xor_sync(0xffffffffu, x, 2));
                    if (g == 16) {
                        if ((t & 8) == 0) {
                            best[h] = x;
                            continue;
                        }
                        x = max_nan(x, best[h]);
                    }
                    if ((2 * tig & (min(g, 8) - 1)) == 0) put(r, x);
                }
            }
        }
        ids(b0 + static_cast<int>(gridDim.x) * kScorePages);
        __syncthreads();
    }
}

// The score of a page for one KV head's queries in float64, as a number whose order is the scores'.  A warp together; s_q: [g][D].
__device__ __forceinline__ uint64_t order_key(double x) {
    if (x != x) x = -INFINITY;
    const uint64_t b = static_cast<uint64_t>(__double_as_longlong(x + 0.0));      // (-0 counts as 0)
    return b >> 63 ? ~b : b | (1ull << 63);
}
template <int D>
__device__ __forceinline__ uint64_t exact_score(const SelectArgs& a, const float* s_q, int g, int page, int kvh) {
    if (page < 0 || page >= a.n_pages) return order_key(-INFINITY);
    constexpr int kPer = D / 32;
    const int lane = threadIdx.x & 31;
    const uint16_t* src = a.summary + (static_cast<int64_t>(page) * a.Hkv + kvh) * 2 * D;
    double low[kPer], high[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        low[i] = static_cast<double>(__uint_as_float(static_cast<uint32_t>(src[i * 32 + lane]) << 16));
        high[i] = static_cast<double>(__uint_as_float(static_cast<uint32_t>(src[D + i * 32 + lane]) << 16));
    }
    double best = -INFINITY;
    for (int h = 0; h < g; ++h) {
        double x = 0.0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const double q = static_cast<double>(s_q[h * D + i * 32 + lane]);
            x = fma(q, q > 0.0 ? high[i] : low[i], x);
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
        best = x > best ? x : best;              // (a NaN never is)
    }
    return order_key(best);
}

constexpr int kTopThreads = 512, kTopWarps = kTopThreads / 32;
constexpr int kBins = 2 * kTopThreads;
constexpr int kTopHeld = 8;                      // scores that a thread holds; more are read again
constexpr int kNear = 256;                       // pages that are ranked in float64 within shared memory
// How far an fp32 score can be off, as a share of the sum of the products' magnitudes: 2 d / 16 = 16 matrix instructions (d = 128), each
// of which rounds a sum of 17 terms that are no larger than that; 2^-20 for each is several times what fp32 sums lose.
constexpr float kScoreError = 1.f / 65536.f;

struct TopScratch {
    int bins[kBins];
    float q[16 * 128];
    float value[5][kTopWarps];
    int count[kTopWarps];
    __align__(16) int taken[kTopHeld][kTopWarps];
    uint64_t near_key[kNear], cut_key;
    int near_at[kNear], n_near, cut_at, bin, above;
};

// Largest values over the CTA (smallest: of the negated ones).
template <int N>
__device__ __forceinline__ void block_max(float (&x)[N], float (&s)[5][kTopWarps]) {
    static_assert(N <= 5, "");
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) x[i] = fmaxf(x[i], __shfl_xor_sync(0xffffffffu, x[i], d));
        if ((threadIdx.x & 31) == 0) s[i][threadIdx.x >> 5] = x[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[i] = s[i][threadIdx.x & (kTopWarps - 1)];
#pragma unroll
        for (int d = kTopWarps / 2; d > 0; d >>= 1) x[i] = fmaxf(x[i], __shfl_xor_sync(0xffffffffu, x[i], d));
    }
}
// How many threads before this one have the flag, and how many in all.
__device__ __forceinline__ int block_count(bool flag, int& all, int (&s)[kTopWarps]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t m = __ballot_sync(0xffffffffu, flag);
    __syncthreads();
    if (lane == 0) s[warp] = __popc(m);
    __syncthreads();
    const int c = lane < kTopWarps ? s[lane] : 0;
    all = static_cast<int>(__reduce_add_sync(0xffffffffu, static_cast<unsigned>(c)));
    return static_cast<int>(__reduce_add_sync(0xffffffffu, static_cast<unsigned>(lane < warp ? c : 0))) + __popc(m & ((1u << lane) - 1u));
}

template <int D>
__global__ void __launch_bounds__(kTopThreads, 2)
page_select_kernel(const __grid_constant__ SelectArgs a, int blocks) {
    __shared__ TopScratch s;
    const int row = blockIdx.x, t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const int token0 = row / a.Hkv, kvh = row - token0 * a.Hkv, slot = token0 / a.T, u = token0 - slot * a.T, g = 1 << a.g_shift;
    // This launch is placed when the scores' CTAs have all passed their wait: the caller's tensors are complete and only the scores
    // are waited for.  The attention may be placed as soon as this launch runs, for the same reason.
    grid_launch_dependents();
    const int len = checked_len(a.len[slot], static_cast<int64_t>(a.max_pages) << a.page_shift, false, nullptr);
    const int full = len >> a.page_shift, k = min(a.k, full);
    if (a.n_draft != nullptr && u >= a.n_draft[slot]) {
        grid_dependency_wait();
        return;
    }
    const float* score = a.score + static_cast<int64_t>(row) * a.max_pages;
    uint64_t* exact = a.exact + static_cast<int64_t>(row) * a.max_pages;
    int32_t* sel = a.sel + static_cast<int64_t>(row) * a.k;
    int32_t* list = a.list + static_cast<int64_t>(row) * (a.k + 1);
    const int32_t* table = a.table + static_cast<int64_t>(slot) * a.max_pages;

    // Pages [first, last) are ranked, `want` of them taken; those before and after are taken anyway.
    const bool all = full <= a.k;
    const int first = min(a.sink, full), last = max(first, full - a.window), want = all ? 0 : k - first - (full - last);
    const bool ranked = !all && want > 0;
    // ---- pages that are taken anyway, before the scores are there: they come before and after the ranked ones ----
    const int ahead = all ? full : first, after = all ? full : last;
    for (int b = t; b < ahead; b += kTopThreads) {
        sel[b] = b;
        list[b] = table[b];
    }
    for (int b = after + t; b < full; b += kTopThreads) {
        sel[k - full + b] = b;
        list[k - full + b] = table[b];
    }
    for (int i = k + t; i < a.k; i += kTopThreads) sel[i] = -1;
    if (t == 0 && len > full << a.page_shift) list[k] = table[full];      // the page of the rows after the last full one
    float held[kTopHeld], above = INFINITY, below = INFINITY;      // scores over `above` are taken, under `below` not, the others ranked
    const auto at = [&](int i) { return first + t + i * kTopThreads; };
    const int rounds = (last - first + kTopThreads - 1) / kTopThreads;
#pragma unroll
    for (int i = 0; i < kTopHeld; ++i) held[i] = -INFINITY;
    const auto value = [&](int i) { return at(i) < last ? score[at(i)] : -INFINITY; };
    if (ranked) {
        float q1 = 0.f;                           // sums of the queries' magnitudes, a warp per head
        for (int h = warp; h < g; h += kTopWarps) {
            float x = 0.f;
            for (int j = lane; j < D; j += 32) {
                const float q = __uint_as_float(static_cast<uint32_t>(a.Q[(static_cast<int64_t>(token0) * a.Hq + (kvh << a.g_shift) + h) * D + j]) << 16);
                s.q[h * D + j] = q;
                x += fabsf(q);
            }
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
            q1 = fmaxf(q1, x != x ? INFINITY : x);
        }
        float lo = INFINITY, hi = -INFINITY;
        bool odd = false;                         // a score that is not finite
        if (t == 0) s.n_near = 0;
        for (int i = t; i < kBins; i += kTopThreads) s.bins[i] = 0;
        const auto look = [&](float x) {
            odd |= !(x < INFINITY);
            if (x > -INFINITY) {
                lo = fminf(lo, x);
                hi = fmaxf(hi, x);
            }
        };
        grid_dependency_wait();
#pragma unroll
        for (int i = 0; i < kTopHeld; ++i)
            if (i < rounds) held[i] = value(i);
        float most = 0.f;
        for (int i = t; i < (full + kScorePages - 1) / kScorePages; i += kTopThreads)
            most = fmaxf(most, a.most[(static_cast<int64_t>(slot) * a.Hkv + kvh) * blocks + i]);
#pragma unroll
        for (int i = 0; i < kTopHeld; ++i)
            if (i < rounds) look(held[i]);
        for (int i = kTopHeld; i < rounds; ++i) look(value(i));
        float all5[5] = {-lo, hi, q1, most, odd ? 1.f : 0.f};
        block_max(all5, s.value);
        lo = -all5[0];
        hi = all5[1];
        const float size = all5[2] * all5[3];
        const bool rough = all5[4] > 0.f || !(size < 1e37f) || !(hi > lo);      // fp32 says nothing: all are ranked in float64
        if (!rough) {
            // ---- the bin of the want-th largest score ----
            const float inv = kBins / (hi - lo);
            const auto bin_of = [&](float x) { return min(max(static_cast<int>((x - lo) * inv), 0), kBins - 1); };
#pragma unroll
            for (int i = 0; i < kTopHeld; ++i)
                if (i < rounds && at(i) < last) atomicAdd(&s.bins[bin_of(held[i])], 1);
            for (int i = kTopHeld; i < rounds; ++i)
                if (at(i) < last) atomicAdd(&s.bins[bin_of(value(i))], 1);
            __syncthreads();
            const int top = kBins - 1 - 2 * t, n0 = s.bins[top], n1 = s.bins[top - 1];       // a thread's two, from the largest down
            int x = n0 + n1;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, x, d);
                if (lane >= d) x += y;
            }
            if (lane == 31) s.count[warp] = x;
            __syncthreads();
            int over = x - n0 - n1;
            for (int w = 0; w < warp; ++w) over += s.count[w];
            if (over < want && over + n0 + n1 >= want) s.bin = over + n0 >= want ? top : top - 1;
            __syncthreads();
            const int bin = s.bin;
            float in_lo = INFINITY, in_hi = -INFINITY;                       // smallest and largest score in it
            const auto inside = [&](int i, float v) {
                if (at(i) < last && bin_of(v) == bin) {
                    in_lo = fminf(in_lo, v);
                    in_hi = fmaxf(in_hi, v);
                }
            };
#pragma unroll
            for (int i = 0; i < kTopHeld; ++i)
                if (i < rounds) inside(i, held[i]);
            for (int i = kTopHeld; i < rounds; ++i) inside(i, value(i));
            const float e = 2.f * kScoreError * size;
            float ends[2] = {-in_lo, in_hi};
            block_max(ends, s.value);
            above = nextafterf(ends[1] + e, INFINITY);                       // (outward: the sums are rounded)
            below = nextafterf(-ends[0] - e, -INFINITY);
        } else {
            below = -INFINITY;                    // (`above` is infinite)
        }
    }
    if (!ranked) grid_dependency_wait();
    const auto is_near = [&](float x) { return !(x > above) && !(x < below); };

    // ---- pages between the two borders are ranked in float64 ----
    bool whole = false;
    if (ranked) {
        int taken = 0;
        const auto sort_out = [&](int i, float x) {
            if (at(i) >= last) return;
            if (is_near(x)) {
                const int n = atomicAdd(&s.n_near, 1);
                if (n < kNear) s.near_at[n] = at(i);
            } else if (x > above) {
                ++taken;
            }
        };
#pragma unroll
        for (int i = 0; i < kTopHeld; ++i)
            if (i < rounds) sort_out(i, held[i]);
        for (int i = kTopHeld; i < rounds; ++i) sort_out(i, value(i));
        taken = static_cast<int>(__reduce_add_sync(0xffffffffu, taken));
        __syncthreads();
        if (lane == 0) s.count[warp] = taken;
        __syncthreads();
        int left = want;                          // pages to take from those in between
        for (int w = 0; w < kTopWarps; ++w) left -= s.count[w];
        const int n_near = s.n_near;
        whole = left == n_near;                   // all of them are taken, often the k-th alone: nothing to rank
        if (whole) {
        } else if (n_near <= kNear) {
            for (int i = warp; i < n_near; i += kTopWarps) {
                const int b = s.near_at[i];
                const uint64_t key = exact_score<D>(a, s.q, g, table[b], kvh);
                if (lane == 0) {
                    s.near_key[i] = key;
                    exact[b] = key;
                }
            }
            __syncthreads();
            if (t < n_near) {
                const uint64_t key = s.near_key[t];
                const int b = s.near_at[t];
                int before = 0;
                for (int i = 0; i < n_near; ++i) before += s.near_key[i] > key || (s.near_key[i] == key && s.near_at[i] < b) ? 1 : 0;
                if (before == left - 1) {
                    s.cut_key = key;
                    s.cut_at = b;
                }
            }
            __syncthreads();
        } else {
            for (int b = first + warp; b < last; b += kTopWarps)
                if (is_near(score[b])) {
                    const uint64_t key = exact_score<D>(a, s.q, g, table[b], kvh);
                    if (lane == 0) exact[b] = key;
                }
            // the left-th largest key, a byte at a time
            uint64_t kth = 0, settled = 0;
            for (int shift = 56; shift >= 0; shift -= 8) {
                __syncthreads();
                for (int i = t; i < 256; i += kTopThreads) s.bins[i] = 0;
                __syncthreads();
                for (int b = first + t; b < last; b += kTopThreads)
                    if (is_near(score[b])) {
                        const uint64_t x = exact[b];
                        if ((x & settled) == kth) atomicAdd(&s.bins[(x >> shift) & 255], 1);
                    }
                __syncthreads();
                if (t == 0) {
                    int bin = 255, over = 0;
                    while (over + s.bins[bin] < left) over += s.bins[bin--];
                    s.bin = bin;
                    s.above = over;
                }
                __syncthreads();
                kth |= static_cast<uint64_t>(s.bin) << shift;
                settled |= 255ull << shift;
                left -= s.above;
            }
            // and the left-th page of those that have it
            int done = 0;
            for (int b0 = first; b0 < last; b0 += kTopThreads) {
                const int b = b0 + t;
                const bool same = b < last && is_near(score[b]) && exact[b] == kth;
                int total;
                const int before = block_count(same, total, s.count);
                if (same && done + before == left - 1) {
                    s.cut_key = kth;
                    s.cut_at = b;
                }
                done += total;
            }
            __syncthreads();
        }
    }

    // ---- the ranked pages that are taken, in ascending order ----
    if (ranked) {
        const uint64_t cut_key = whole ? 0 : s.cut_key;
        const int cut_at = whole ? 0 : s.cut_at;
        int done = first;
        for (int i0 = 0; i0 < rounds; i0 += kTopHeld) {
            uint32_t takes[kTopHeld];
            if (i0 > 0) __syncthreads();
#pragma unroll
            for (int i = 0; i < kTopHeld; ++i) {
                takes[i] = 0u;
                if (i0 + i >= rounds) {
                    if (lane == 0) s.taken[i][warp] = 0;
                    continue;
                }
                const int b = at(i0 + i);
                const float x = i0 == 0 ? held[i] : value(i0 + i);
                bool take = b < last && x > above;
                if (b < last && is_near(x) && whole) {
                    take = true;
                } else if (b < last && is_near(x)) {
                    const uint64_t key = exact[b];
                    take = key > cut_key || (key == cut_key && b <= cut_at);
                }
                takes[i] = __ballot_sync(0xffffffffu, take);
                if (lane == 0) s.taken[i][warp] = __popc(takes[i]);
            }
            __syncthreads();
            static_assert(kTopHeld * kTopWarps == 128, "");
            const int4 c = reinterpret_cast<const int4*>(s.taken)[lane];     // four of the 128 counts, in the pages' order
            int x = c.x + c.y + c.z + c.w;
            const int own = x;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, x, d);
                if (lane >= d) x += y;
            }
            const int total = __shfl_sync(0xffffffffu, x, 31), p0 = x - own, p1 = p0 + c.x, p2 = p1 + c.y, p3 = p2 + c.z;
#pragma unroll
            for (int i = 0; i < kTopHeld; ++i) {
                if (i0 + i >= rounds) break;
                const int from = i * (kTopWarps / 4) + (warp >> 2);          // the lane with this warp's count of the i-th round
                const int q0 = __shfl_sync(0xffffffffu, p0, from), q1 = __shfl_sync(0xffffffffu, p1, from);
                const int q2 = __shfl_sync(0xffffffffu, p2, from), q3 = __shfl_sync(0xffffffffu, p3, from);
                const int before = (warp & 2) ? ((warp & 1) ? q3 : q2) : ((warp & 1) ? q1 : q0);
                if ((takes[i] >> lane) & 1u) {
                    const int to = done + before + __popc(takes[i] & ((1u << lane) - 1u)), b = at(i0 + i);
                    sel[to] = b;
                    list[to] = table[b];
                }
            }
            done += total;
        }
    }
}

// ---------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------
bool heads_ok(int32_t Hq, int32_t Hkv) {
    if (Hkv < 1 || Hq < Hkv || Hq % Hkv != 0) return false;
    const int g = Hq / Hkv;
    return g == 1 || g == 2 || g == 4 || g == 8 || g == 16;
}

float scale_log2(float softmax_scale, int32_t d) {
    return (softmax_scale > 0.f ? softmax_scale : 1.f / sqrtf(static_cast<float>(d))) * 1.4426950408889634f;
}

}  // namespace
}  // namespace pulsar

using namespace pulsar;

extern "C" size_t pulsar_tree_attn_workspace_bytes(int32_t n_slots, int32_t T, int32_t Hq, int32_t Hkv, int32_t d) {
    if (n_slots < 1 || n_slots > kMaxSlots || T < 1 || T > kMaxTree || !heads_ok(Hq, Hkv) || (d != 64 && d != 128)) return 0;
    return attn_workspace_bytes(n_slots, Hkv, T * (Hq / Hkv), d);
}

extern "C" int32_t pulsar_tree_attn(const uint16_t* Q, const uint16_t* Knew, const uint16_t* Vnew, int32_t T, uint16_t* K_pages,
                                    uint16_t* V_pages, int32_t n_pages, int32_t page_size, const int32_t* page_table,
                                    const int32_t* cache_len, int32_t n_slots, int32_t max_pages, const int32_t* parent,
                                    const int32_t* n_draft, int32_t Hq, int32_t Hkv, int32_t d, float softmax_scale, void* O,
                                    int32_t out_is_f32, float* LSE, void* workspace, size_t workspace_bytes, int32_t* device_status,
                                    void* stream) {
    if (!pool_ok(1, n_pages, page_size, Hkv, d, n_slots, max_pages) || !heads_ok(Hq, Hkv) || T < 1 || T > kMaxTree) return PULSAR_ERR_SHAPE;
    if (Q == nullptr || Knew == nullptr || Vnew == nullptr || K_pages == nullptr || V_pages == nullptr || page_table == nullptr ||
        cache_len == nullptr || O == nullptr || workspace == nullptr)
        return PULSAR_ERR_INVALID_ARG;
    const size_t slots = static_cast<size_t>(n_slots), rows = slots * T, pool = pool_bytes(1, n_pages, page_size, Hkv, d);
    const Tensors in = {{Q, rows * Hq * d * 2}, {Knew, rows * Hkv * d * 2}, {Vnew, rows * Hkv * d * 2}, {page_table, 4 * slots * max_pages},
                        {cache_len, 4 * slots}, {parent, 4 * rows}, {n_draft, 4 * slots}};
    const Tensors out = {{O, rows * Hq * d * (out_is_f32 ? 4 : 2)}, {K_pages, pool}, {V_pages, pool}, {LSE, rows * Hq * 4}, {device_status, 4u}};
    if (!apart(out, in)) return PULSAR_ERR_INVALID_ARG;
    for (const void* p : {static_cast<const void*>(Q), static_cast<const void*>(Knew), static_cast<const void*>(Vnew),
                          static_cast<const void*>(K_pages), static_cast<const void*>(V_pages), static_cast<const void*>(O)})
        if (!aligned(p, 16)) return PULSAR_ERR_ALIGNMENT;
    if (!aligned(page_table, 4) || !aligned(cache_len, 4) || !aligned(parent, 4) || !aligned(n_draft, 4) || !aligned(LSE, 4) ||
        !aligned(workspace, 256))
        return PULSAR_ERR_ALIGNMENT;
    if (!pieces_ok(n_slots, Hkv, static_cast<int64_t>(max_pages) * page_size)) return PULSAR_ERR_SHAPE;
    const size_t scratch = pulsar_tree_attn_workspace_bytes(n_slots, T, Hq, Hkv, d);
    if (workspace_bytes < scratch) return PULSAR_ERR_WORKSPACE;
    if (!apart({{workspace, scratch}}, in) || !apart({{workspace, scratch}}, out)) return PULSAR_ERR_INVALID_ARG;
    if (const int32_t rc = check_device(); rc != PULSAR_OK) return rc;
    PagedArgs a{};
    a.Q = Q;
    a.Knew = Knew;
    a.Vnew = Vnew;
    a.K = K_pages;
    a.V = V_pages;
    a.table = page_table;
    a.len = cache_len;
    a.n_draft = n_draft;
    a.parent = parent;
    a.n_slots = n_slots;
    a.T = T;
    a.Hq = Hq;
    a.Hkv = Hkv;
    a.g_shift = log2_exact(Hq / Hkv);
    a.page_shift = log2_exact(page_size);
    a.n_pages = n_pages;
    a.max_pages = max_pages;
    a.scale_log2 = scale_log2(softmax_scale, d);
    a.O = O;
    a.out_f32 = out_is_f32;
    a.LSE = LSE;
    a.status = device_status;
    return launch_attn(a, Hkv, T * (Hq / Hkv), d, workspace, static_cast<cudaStream_t>(stream));
}

namespace {
struct SparseScratch {
    size_t exact, score, most, list, total;
    SparseScratch(int64_t n_slots, int64_t T, int64_t Hkv, int64_t max_pages, int64_t k, int g, int d) {
        const int64_t rows = n_slots * T * Hkv;
        exact = attn_workspace_bytes(static_cast<int>(n_slots), static_cast<int>(T * Hkv), g, d);
        score = round_up(exact + static_cast<size_t>(rows * max_pages) * 8, 256);
        most = round_up(score + static_cast<size_t>(rows * max_pages) * 4, 256);
        list = round_up(most + static_cast<size_t>(n_slots * Hkv * ((max_pages + kScorePages - 1) / kScorePages)) * 4, 256);
        total = round_up(list + static_cast<size_t>(rows * (k + 1)) * 4, 256);
    }
};
bool sparse_ok(int32_t n_slots, int32_t T, int32_t k, int32_t Hq, int32_t Hkv, int32_t d) {
    return n_slots >= 1 && n_slots <= kMaxSlots && T >= 1 && T <= kMaxTree && heads_ok(Hq, Hkv) && Hkv <= 1024 && (d == 64 || d == 128) &&
           k >= 1 && k <= 65536 && static_cast<int64_t>(n_slots) * T * Hkv <= (1 << 20);
}
}  // namespace

extern "C" size_t pulsar_sparse_attn_workspace_bytes(int32_t n_slots, int32_t T, int32_t max_pages, int32_t k, int32_t Hq, int32_t Hkv,
                                                     int32_t d) {
    if (!sparse_ok(n_slots, T, k, Hq, Hkv, d) || max_pages < 1) return 0;
    return SparseScratch(n_slots, T, Hkv, max_pages, k, Hq / Hkv, d).total;
}

extern "C" int32_t pulsar_sparse_attn(const uint16_t* Q, const uint16_t* Knew, const uint16_t* Vnew, int32_t T, uint16_t* K_pages,
                                      uint16_t* V_pages, const uint16_t* summary, int32_t n_pages, int32_t page_size,
                                      const int32_t* page_table, const int32_t* cache_len, int32_t n_slots, int32_t max_pages,
                                      const int32_t* n_draft, int32_t k, int32_t sink, int32_t window, int32_t Hq, int32_t Hkv, int32_t d,
                                      float softmax_scale, uint16_t* O, float* LSE, int32_t* sel, void* workspace,
                                      size_t workspace_bytes, int32_t* device_status, void* stream) {
    if (!pool_ok(1, n_pages, page_size, Hkv, d, n_slots, max_pages) || !sparse_ok(n_slots, T, k, Hq, Hkv, d) || sink < 0 || window < 0 ||
        static_cast<int64_t>(sink) + window > k ||
        !pieces_ok(n_slots, static_cast<int64_t>(T) * Hkv, (static_cast<int64_t>(k) + 1) * page_size))
        return PULSAR_ERR_SHAPE;
    if (Q == nullptr || Knew == nullptr || Vnew == nullptr || K_pages == nullptr || V_pages == nullptr || summary == nullptr ||
        page_table == nullptr || cache_len == nullptr || O == nullptr || sel == nullptr || workspace == nullptr)
        return PULSAR_ERR_INVALID_ARG;
    const size_t slots = static_cast<size_t>(n_slots), tokens = slots * T, pool = pool_bytes(1, n_pages, page_size, Hkv, d);
    const Tensors in = {{Q, tokens * Hq * d * 2}, {Knew, tokens * Hkv * d * 2}, {Vnew, tokens * Hkv * d * 2}, {summary, pool / page_size * 2},
                        {page_table, 4 * slots * max_pages}, {cache_len, 4 * slots}, {n_draft, 4 * slots}};
    const Tensors out = {{O, tokens * Hq * d * 2}, {K_pages, pool}, {V_pages, pool}, {LSE, tokens * Hq * 4}, {sel, tokens * Hkv * k * 4},
                         {device_status, 4u}};
    if (!apart(out, in)) return PULSAR_ERR_INVALID_ARG;
    for (const void* p : {static_cast<const void*>(Q), static_cast<const void*>(Knew), static_cast<const void*>(Vnew), static_cast<const void*>(summary),
                          static_cast<const void*>(K_pages), static_cast<const void*>(V_pages), static_cast<const void*>(O)})
        if (!aligned(p, 16)) return PULSAR_ERR_ALIGNMENT;
    if (!aligned(page_table, 4) || !aligned(cache_len, 4) || !aligned(n_draft, 4) || !aligned(LSE, 4) || !aligned(sel, 4) || !aligned(workspace, 256))
        return PULSAR_ERR_ALIGNMENT;
    const int64_t rows = static_cast<int64_t>(n_slots) * T * Hkv;
    const SparseScratch y(n_slots, T, Hkv, max_pages, k, Hq / Hkv, d);
    if (workspace_bytes < y.total) return PULSAR_ERR_WORKSPACE;
    if (!apart({{workspace, y.total}}, in) || !apart({{workspace, y.total}}, out)) return PULSAR_ERR_INVALID_ARG;
    if (const int32_t rc = check_device(); rc != PULSAR_OK) return rc;
    auto* ws = static_cast<uint8_t*>(workspace);
    auto st = static_cast<cudaStream_t>(stream);

    SelectArgs b{};
    b.Q = Q;
    b.summary = summary;
    b.table = page_table;
    b.len = cache_len;
    b.n_draft = n_draft;
    b.T = T;
    b.Hq = Hq;
    b.Hkv = Hkv;
    b.g_shift = log2_exact(Hq / Hkv);
    b.page_shift = log2_exact(page_size);
    b.n_pages = n_pages;
    b.max_pages = max_pages;
    b.k = k;
    b.sink = sink;
    b.window = window;
    b.exact = reinterpret_cast<uint64_t*>(ws + y.exact);
    b.score = reinterpret_cast<float*>(ws + y.score);
    b.most = reinterpret_cast<float*>(ws + y.most);
    b.sel = sel;
    b.list = reinterpret_cast<int32_t*>(ws + y.list);
    b.status = device_status;
    const int blocks = (max_pages + kScorePages - 1) / kScorePages;
    // A CTA per 64 pages of a head, up to 32 per SM: then they take more in turn, so that a table for far longer contexts than the slots
    // have costs little (64 slots of 2000 rows with room for 131,072: 134 -> 78 us).
    const unsigned score_ctas = static_cast<unsigned>(std::min<int64_t>(blocks, std::max<int64_t>(1, 32 * sm_count() / (static_cast<int64_t>(Hkv) * n_slots))));
    PULSAR_CUDA_OK(launch_kernel(d == 128 ? page_score_kernel<128> : page_score_kernel<64>, dim3(score_ctas, Hkv, n_slots), dim3(kScoreThreads), 0,
                                 st, true, b, blocks));
    count_launch();
    PULSAR_CUDA_OK(launch_kernel(d == 128 ? page_select_kernel<128> : page_select_kernel<64>, dim3(static_cast<unsigned>(rows)), dim3(kTopThreads), 0,
                                 st, true, b, blocks));
    count_launch();

    PagedArgs a{};
    a.Q = Q;
    a.Knew = Knew;
    a.Vnew = Vnew;
    a.K = K_pages;
    a.V = V_pages;
    a.table = page_table;
    a.len = cache_len;
    a.n_draft = n_draft;
    a.list = b.list;
    a.n_slots = n_slots;
    a.T = T;
    a.Hq = Hq;
    a.Hkv = Hkv;
    a.g_shift = b.g_shift;
    a.page_shift = b.page_shift;
    a.n_pages = n_pages;
    a.max_pages = max_pages;
    a.k = k;
    a.scale_log2 = scale_log2(softmax_scale, d);
    a.O = O;
    a.LSE = LSE;
    a.status = device_status;
    return launch_attn(a, T * Hkv, Hq / Hkv, d, workspace, st);
}
