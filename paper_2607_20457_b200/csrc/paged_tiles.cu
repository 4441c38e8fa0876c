// Attention over a paged cache for up to 64 query rows per KV head (drafted trees, decoding steps, selected pages), on the tensor
// cores (tcgen05).
//
// S^T = K Q^T: the 128 keys of a tile stand in the rows (TMEM lanes) and the query rows -- nodes x heads of the group, 16, 32 or 64
// with those that do not exist -- in the columns, so that the products cost what the rows need and every softmax thread has one key.
// O^T += V^T P^T takes the V tile as it lies in memory (d contiguous) as its first operand and P^T from shared memory.
//
//   warp 0      loader: shares out the work; pages of K and V by TMA into a ring of tiles, the new tokens' own rows with the last one
//   warp 1      issues the matrix instructions: S of the next tile before PV of this one
//   warp 2      query rows (TMA)
//   warp 3      which nodes see which
//   warps 4-..  softmax: a thread per key and 32 columns (or all, if fewer); epilogue: a thread per output component and 32 rows
//   last warp   pages of 16 rows: copies V (see Cfg)
//
// A column's maximum lies across lanes, so it is not formed for every tile: P is formed with the largest logit seen when it was
// last moved, and moved (and O^T and the sums rescaled) when a logit exceeds it by more than 2^8.  P, O^T and the sums use the same
// stale maximum, so the result is unchanged.  The sums stay with their keys' threads, in fp32, until an item ends.
//
// The product with V takes P in bf16.  Rounded once, every probability is off by up to 2^-8 of itself and the outputs by as much as
// their own last rounding; so P is split into two bf16 numbers (2^-16 is left), which are neighbouring columns of one product with
// twice the columns, and the epilogue adds the two results where the upper part's is finite (one slot of 6001 rows 12.9 -> 13.2 us, 16 trees of 52
// rows 33.6 -> 35.3, long caches the same; to look at the upper part first costs the small trees 0.3 us).
//
// What bounds it (measured in a pass of many, with the joining launch): long caches the memory -- 32 slots of up to 8192 rows of 8
// heads, one token each, 97 to 102 us, 5.4 to 5.7 TB/s; short ones latency -- one slot of 6001 rows 13 us, of which the first tile's way (length,
// page ids, TMA) takes 3.5, an item's end 1.5 and the joining launch 3; a tile of 64 rows itself about 1100 cycles.
#include <algorithm>

#include "mma.cuh"
#include "paged_roles.cuh"

namespace pulsar {

namespace {

// kSplit: a warp behind the softmax copies V, and the loader K alone.  Pages of 16 rows are many copies, of which a warp issues one in 100
// cycles or so: 1800 for K and V of a tile of d = 64, whose softmax takes 1900.  8 slots of 6000 rows 33.3 -> 29.1 us (d = 64),
// 47.7 -> 41.5 (d = 128); with pages of 64 rows, which are few copies, 28.2 -> 29.3 and 39.5 -> 40.6.  Selected pages lie apart and
// come no faster for it: 16 slots, 48 pages of 16 rows 53.8 -> 56.7 with the scores.
template <int D, int N, bool kSelected, bool kSplit>
struct Cfg {
    static constexpr int kPanels = D / 64;
    static constexpr int kTileBytes = kPanels * kPanelBytes;
    static constexpr int kCols = N < 32 ? N : 32;                // columns of a softmax thread
    static constexpr int kGroups = N / kCols;                    // softmax warpgroups
    static constexpr int kSoftWarps = 4 * kGroups;
    static constexpr int kThreads = 128 + 128 * kGroups + (kSplit ? 32 : 0);
    static constexpr int kRows = N, kQTiles = 1, kQRows = N;
    static constexpr bool kBySeen = true, kSparse = kSelected, kTwoLoaders = kSplit;
    static constexpr int kPBytes = (2 * N + 63) / 64 * kPanelBytes;              // P's upper and lower parts side by side
    static constexpr int kQBytes = kPanels * N * 128;
    static constexpr int kMisc = static_cast<int>(sizeof(Slots)) + 12 + kQueue * kMaxTree * 8 + kQueue * (8 + 64) + 64 * 8 + 7 * N * 4 + N * 8 +
                                 kMaxTree * 4 + 8;
    static constexpr int kFit = (232448 - kPBytes - kQBytes - kMisc) / kTileBytes;
    static constexpr int kStages = kFit < 10 ? kFit : 10;
    // The product with V reads 128 components; with d = 64 the second half is whatever follows the tile (and is not used), so
    // something has to follow the last tile of the ring: P does.
    static constexpr int kP = kStages * kTileBytes;
    static constexpr int kQ = kP + kPBytes;
    static constexpr int kRest = kQ + kQBytes;
    static constexpr int kSmem = kRest + kMisc;
    static constexpr int kTmemCols = 4 * N;                                      // S of two tiles; O of P's two parts
    // barriers
    static constexpr int bKvFull = 0, bKvEmpty = kStages, bQFull = 2 * kStages, bQEmpty = bQFull + 1, bSFull = bQEmpty + 1, bSEmpty = bSFull + 2,
                         bPFull = bSEmpty + 2, bPEmpty = bPFull + 1, bOFull = bPEmpty + 1, bOEmpty = bOFull + 1, bSees = bOEmpty + 1, bWorkFull = bSees + kQueue, bWorkEmpty = bWorkFull + kQueue,
                         kBars = bWorkEmpty + kQueue;
    static_assert(kBars <= 64 && kStages >= 3, "");
};

// Where columns c & ~7 .. of key `key` stand in P.
__device__ __forceinline__ int p_at(int key, int c) { return (c >> 6) * kPanelBytes + key * 128 + (((c >> 3 & 7) ^ (key & 7)) << 4); }

// Columns [0, C) of TMEM, 32 lanes per warp.
template <int C>
__device__ __forceinline__ void load_columns(uint32_t taddr, float (&x)[C]) {
    if constexpr (C == 16) {
        uint32_t r[16];
        tmem_ld16(taddr, r);
        tmem_wait_ld();
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = __uint_as_float(r[i]);
    } else {
        static_assert(C == 32, "");
        uint32_t r[32];
        tmem_ld32(taddr, r);
        tmem_wait_ld();
#pragma unroll
        for (int i = 0; i < 32; ++i) x[i] = __uint_as_float(r[i]);
    }
}

// Column sums over a warp's lanes: lane l ends with those of columns [l * C / 32, ...) (C = 16: lanes 2 c and 2 c + 1 with column c).
// Every step hands half of the columns to the other half of the lanes.
template <int C>
__device__ __forceinline__ void column_sums(float (&x)[C], int lane) {
    int n = C;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        if (n > 1) {
            n >>= 1;
#pragma unroll
            for (int i = 0; i < C / 2; ++i)
                if (i < n) {
                    const bool upper = (lane & off) != 0;
                    const float keep = upper ? x[i + n] : x[i], give = upper ? x[i] : x[i + n];
                    x[i] = keep + __shfl_xor_sync(0xffffffffu, give, off);
                }
        } else {
            x[0] += __shfl_xor_sync(0xffffffffu, x[0], off);
        }
    }
}

template <int D, int N, bool kSparse, bool kSplit>
__global__ void __launch_bounds__(Cfg<D, N, kSparse, kSplit>::kThreads, 1)
paged_tiles_kernel(const __grid_constant__ PagedArgs a, const __grid_constant__ Maps map, int row_blocks) {
    using C = Cfg<D, N, kSparse, kSplit>;
    constexpr int kCols = C::kCols;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint8_t* rest = smem + C::kRest;
    uint64_t* s_seen = reinterpret_cast<uint64_t*>(rest);                              // [kQueue][kMaxTree] the nodes that see a node
    Work* s_work = reinterpret_cast<Work*>(s_seen + kQueue * kMaxTree);                // [kQueue]
    uint64_t* bars = reinterpret_cast<uint64_t*>(s_work + kQueue);                     // [64]
    float* s_col = reinterpret_cast<float*>(bars + 64);                                // [4][N] of each warp's keys: largest logits, sums
    float* s_neg = s_col + 4 * N;                                                      // [N] minus the maximum in use
    float* s_alpha = s_neg + N;                                                        // [N] rescaling factors
    float* s_inv = s_alpha + N;                                                        // [N] 1 / sum
    int64_t* s_to = reinterpret_cast<int64_t*>(s_inv + N);                             // [N] where a row's outputs go
    int* s_up = reinterpret_cast<int*>(s_to + N);                                      // [kMaxTree]
    uint32_t* s_odd = reinterpret_cast<uint32_t*>(s_up + kMaxTree);                    // [kQueue][2] nodes whose value is not finite
    uint32_t* tmem_ptr = s_odd + 2 * kQueue;
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_ptr + 1);
    Slots& slots = *reinterpret_cast<Slots*>(tmem_ptr + 2);

    const int lane = threadIdx.x & 31;
    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0);
    const uint32_t bar0 = smem_u32(bars);
    const auto bar = [&](int i) { return bar0 + 8 * static_cast<uint32_t>(i); };
    if (threadIdx.x == 0) {
        *abort_flag = 0;
        for (int i = 0; i < C::kStages; ++i) {
            mbar_init(bars + C::bKvFull + i, 1);
            mbar_init(bars + C::bKvEmpty + i, 1);
        }
        mbar_init(bars + C::bQFull, 1);
        mbar_init(bars + C::bQEmpty, 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(bars + C::bSFull + i, 1);
            mbar_init(bars + C::bSEmpty + i, C::kSoftWarps);
        }
        mbar_init(bars + C::bPFull, C::kSoftWarps);
        mbar_init(bars + C::bPEmpty, 1);
        mbar_init(bars + C::bOFull, 1);
        mbar_init(bars + C::bOEmpty, C::kSoftWarps);
        for (int i = 0; i < kQueue; ++i) {
            mbar_init(bars + C::bSees + i, 1);
            mbar_init(bars + C::bWorkFull + i, 1);
            mbar_init(bars + C::bWorkEmpty + i, C::kSoftWarps + 3 + (kSplit ? 1 : 0));         // and the issuer, warps 2 and 3, the one for V
        }
        mbar_fence_init();
        prefetch_maps(map);
    }
    if (warp == 1) {
        tmem_alloc(tmem_ptr, C::kTmemCols);
        tmem_relinquish();
    }
    // Behind a selection everything but its list is complete when this launch is placed (paged.cu): those who read the list wait.
    if (!kSparse) grid_dependency_wait();
    grid_launch_dependents();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_ptr, tO = tmem + 2 * N;
    const int64_t pitch = static_cast<int64_t>(a.Hkv) * D;
    const Roles roles{smem, s_work, s_seen, s_odd, s_up, &slots, bar0, abort_flag};

    if (warp == 0) {
        load_role<C>(a, map, row_blocks, roles);
    } else if (warp == 1) {
        // ---- matrix instructions: S of a tile, then PV of the tile before it ----
        const bool leader = elect_one();
        constexpr uint32_t kIdescS = umma_idesc_bf16(kTile, N, false, false), kIdescO = umma_idesc_bf16(kTile, 2 * N, true, true);
        const uint64_t desc_k = umma_smem_desc_sw128(smem_u32(smem), 16, 1024);
        const uint64_t desc_v = umma_smem_desc_sw128(smem_u32(smem), kPanelBytes, 1024);
        const uint64_t desc_q = umma_smem_desc_sw128(smem_u32(smem + C::kQ), 16, 1024);
        const uint64_t desc_p = umma_smem_desc_sw128(smem_u32(smem + C::kP), kPanelBytes, 1024);
        uint32_t tile = 0, n_done = 0;                     // tiles issued, segments finished
        uint32_t stage = 0, phase = 0;                     // of the next K or V
        bool ok = true, first = false, last = false;       // of the tile whose PV is due
        int steps = 0;                                     // and 16 keys times this many of it
        const auto wait = [&](int b, uint32_t parity) {
            __syncwarp();
            ok = __all_sync(0xffffffffu, ok && mbar_wait_a(bar(b), parity, abort_flag, a.status));
        };
        uint32_t v_stage = 0, v_phase = 0;
        const auto issue_pv = [&](uint32_t t) {
            wait(C::bKvFull + static_cast<int>(v_stage), v_phase);
            if (first) wait(C::bOEmpty, (n_done & 1) ^ 1);
            wait(C::bPFull, t & 1);
            if (!ok) return;
            tc_fence_after();
            if (leader) {
#pragma unroll
                for (int kk = 0; kk < kTile / 16; ++kk)
                    if (kk < steps) umma_ss(tO, desc_v + static_cast<uint64_t>(v_stage * (C::kTileBytes >> 4) + kk * 128), desc_p + static_cast<uint64_t>(kk * 128),
                            kIdescO, first && kk == 0 ? 0u : 1u);
                umma_commit_a(bar(C::bKvEmpty + static_cast<int>(v_stage)));
                umma_commit_a(bar(C::bPEmpty));
                if (last) umma_commit_a(bar(C::bOFull));
            }
            if (last) ++n_done;
        };
        for (uint32_t seq = 0;; ++seq) {
            const Work* s = next_work<C>(a, roles, seq, ok);
            if (!ok || s->valid == 0) break;
            const int p_begin = s->p_begin, p_end = s->p_end, keys = s->keys, new_tile = s->new_tile, new_end = s->new_at + s->n;
            __syncwarp();
            if (lane == 0) arrive_a(bar(C::bWorkEmpty + static_cast<int>(seq % kQueue)));
            for (int t = p_begin; t < p_end && ok; ++t, ++tile) {
                wait(C::bKvFull + static_cast<int>(stage), phase);
                if (t == p_begin) wait(C::bQFull, seq & 1);
                wait(C::bSEmpty + static_cast<int>(tile & 1), ((tile >> 1) & 1) ^ 1);
                if (!ok) break;
                tc_fence_after();
                if (leader) {
#pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk) {
                        const uint64_t off_k = static_cast<uint64_t>(stage * (C::kTileBytes >> 4) + (((kk >> 2) * kPanelBytes + (kk & 3) * 32) >> 4));
                        const uint64_t off_q = static_cast<uint64_t>(((kk >> 2) * (N * 128) + (kk & 3) * 32) >> 4);
                        umma_ss(tmem + (tile & 1) * N, desc_k + off_k, desc_q + off_q, kIdescS, kk > 0 ? 1u : 0u);
                    }
                    umma_commit_a(bar(C::bSFull + static_cast<int>(tile & 1)));
                    umma_commit_a(bar(C::bKvEmpty + static_cast<int>(stage)));
                    if (t + 1 == p_end) umma_commit_a(bar(C::bQEmpty));
                }
                if (++stage == C::kStages) {
                    stage = 0;
                    phase ^= 1;
                }
                if (tile > 0) issue_pv(tile - 1);
                v_stage = stage;
                v_phase = phase;
                if (++stage == C::kStages) {
                    stage = 0;
                    phase ^= 1;
                }
                first = t == p_begin;
                last = t + 1 == p_end;
                steps = used_steps(t, keys, new_tile, new_end);
            }
        }
        if (ok && tile > 0) issue_pv(tile - 1);
    } else if (warp == 2) {
        rows_role<C>(a, map, roles);
    } else if (warp == 3) {
        nodes_role<D, C>(a, roles);
    } else if (kSplit && warp == 4 + C::kSoftWarps) {
        values_role<C>(a, map, roles);
    } else {
        // ---- softmax and epilogue ----
        const int quarter = warp & 3, group = (warp - 4) >> 2;
        const int key = quarter * 32 + lane, col0 = group * kCols;
        const int id = 1 + group;                          // barrier of the warpgroup
        const uint32_t my_lanes = static_cast<uint32_t>(quarter * 32) << 16;
        const int tg = threadIdx.x - 128 - group * 128;    // thread of the warpgroup
        uint32_t tile = 0;
        uint32_t v_stage = 1, v_phase = 0;                 // ring place of the tile's V
        bool ok = true;
        for (uint32_t seg = 0;; ++seg) {
            const Work& s = *next_work<C>(a, roles, seg, ok);
            if (named_any(id, 128, !ok) || s.valid == 0) break;
            if (kSparse && seg == 0) grid_dependency_wait();
            const int32_t* list = page_list<kSparse>(a, s.slot, s.token0, s.kvh);
            const int p_begin = s.p_begin, p_end = s.p_end, new_tile = s.new_tile, n_rows = s.n_rows;
            float sum[kCols];
#pragma unroll
            for (int c = 0; c < kCols; ++c) sum[c] = 0.f;
            const auto page_of = [&](int t) {              // the page of this thread's key of tile t, -1: there is no such key
                const int row = t * kTile + key;
                return t < p_end && row < s.keys ? list[row >> a.page_shift] : -1;
            };
            int page = page_of(p_begin);
            bool failed = false;
            for (int t = p_begin; t < p_end; ++t, ++tile) {
                const int next = page_of(t + 1);           // (looked at a tile later)
                const bool fresh = t == new_tile;
                const int node = fresh ? key - s.new_at : -1;                  // of the new tokens, where this key is one
                const bool cached = page >= 0 && page < a.n_pages, is_node = node >= 0 && node < s.n;
                const uint32_t tS = tmem + (tile & 1) * N + col0 + my_lanes;
                __syncwarp();
                ok = ok && mbar_wait_a(bar(C::bSFull + static_cast<int>(tile & 1)), (tile >> 1) & 1, abort_flag, a.status);
                tc_fence_after();
                uint32_t visible = ~0u;                    // columns that see this key
                if (fresh) {
                    __syncwarp();
                    ok = ok && mbar_wait_a(bar(C::bSees + static_cast<int>(seg % kQueue)), (seg / kQueue) & 1, abort_flag, a.status);
                    const int gs = a.g_shift, per = 1 << gs;
                    const uint64_t seen = is_node ? s_seen[(seg % kQueue) * kMaxTree + node] >> ((s.row0 + col0) >> gs) : cached ? ~0ull : 0ull;
                    visible = 0u;                          // every node's bit becomes the bits of its rows
                    for (int c = 0; c < kCols; c += per)
                        if (((seen >> (c >> gs)) & 1ull) != 0ull) visible |= (per == 32 ? ~0u : (1u << per) - 1u) << c;
                } else if (!cached) {
                    visible = 0u;
                }
                const bool masked = fresh || __any_sync(0xffffffffu, visible != ~0u);
                float x[kCols];
                // x = logits (log2 units) minus the maximum in use
                const auto logits = [&]() {
                    __syncwarp();
                    load_columns<kCols>(tS, x);
                    if (masked) {
#pragma unroll
                        for (int c = 0; c < kCols; ++c)
                            if (((visible >> c) & 1u) == 0u) x[c] = -INFINITY;
                    }
                };
                const auto below = [&]() {
                    float most = -INFINITY;
#pragma unroll
                    for (int c = 0; c < kCols; c += 4) {
                        const float4 neg = *reinterpret_cast<const float4*>(s_neg + col0 + c);
                        fma2(x[c], x[c + 1], a.scale_log2, neg.x, neg.y);
                        fma2(x[c + 2], x[c + 3], a.scale_log2, neg.z, neg.w);
                        most = max3(max3(most, x[c], x[c + 1]), x[c + 2], x[c + 3]);
                    }
                    return most;
                };
                logits();
                if (t == p_begin) {
                    // To begin with, a column's maximum is its logit at the tile's first key, if it sees that key.
                    if (tg == 0) {
#pragma unroll
                        for (int c = 0; c < kCols; ++c) s_neg[col0 + c] = x[c] > -INFINITY ? x[c] * -a.scale_log2 : kUnset;
                    }
                    named_sync(id, 128);
                }
                if (named_any(id, 128, below() > kRescale || !ok)) {
                    // ---- the maximum moves ----
                    __syncwarp();
                    ok = ok && mbar_wait_a(bar(C::bPEmpty), (tile & 1) ^ 1, abort_flag, a.status);       // PV of the tile before is done
                    if (named_any(id, 128, !ok)) {
                        failed = true;
                        break;
                    }
                    tc_fence_after();
                    logits();
#pragma unroll
                    for (int c = 0; c < kCols; ++c) {
                        const float most = warp_max(x[c]);
                        if (lane == 0) s_col[quarter * N + col0 + c] = most;
                    }
                    named_sync(id, 128);
                    if (tg < kCols) {
                        const int c = col0 + tg;
                        const float most = fmaxf(fmaxf(s_col[c], s_col[N + c]), fmaxf(s_col[2 * N + c], s_col[3 * N + c])) * a.scale_log2;
                        const float old = s_neg[c];
                        const bool moves = most > -INFINITY && (old == kUnset || most > -old);
                        s_alpha[c] = !moves ? 1.f : old == kUnset ? 0.f : ex2(-old - most);
                        if (moves) s_neg[c] = -most;
                    }
                    named_sync(id, 128);
#pragma unroll
                    for (int c = 0; c < kCols; ++c) sum[c] *= s_alpha[col0 + c];
                    if (t > p_begin) {
#pragma unroll 1
                        for (int c0 = 0; c0 < 2 * kCols; c0 += 16) {
                            const int from = col0 + c0 % kCols;
                            const uint32_t at = tO + (c0 < kCols ? 0 : N) + from + my_lanes;
                            uint32_t o[16];
                            __syncwarp();
                            tmem_ld16(at, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int c = 0; c < 16; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * s_alpha[from + c]);
                            tmem_st16(at, o);
                        }
                        tmem_wait_st();
                    }
                    (void)below();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) arrive_a(bar(C::bSEmpty + static_cast<int>(tile & 1)));
                uint32_t p[kCols / 2], rest[kCols / 2];    // rounded to bf16, and what that leaves, rounded again
#pragma unroll
                for (int c = 0; c < kCols; c += 2) {
                    const float p0 = ex2(x[c]), p1 = ex2(x[c + 1]);
                    add2(sum[c], sum[c + 1], p0, p1);
                    const uint32_t upper = pack_bf16x2(p0, p1);
                    p[c / 2] = upper;
                    rest[c / 2] = pack_bf16x2(p0 - __uint_as_float(upper << 16), p1 - __uint_as_float(upper & 0xffff0000u));
                }
                // P^T: lines of 64 columns per key, where the product before has been read
                __syncwarp();
                ok = ok && mbar_wait_a(bar(C::bPEmpty), (tile & 1) ^ 1, abort_flag, a.status);
#pragma unroll
                for (int v = 0; v < kCols / 8; ++v) {
                    *reinterpret_cast<uint4*>(smem + C::kP + p_at(key, col0 + 8 * v)) = make_uint4(p[4 * v], p[4 * v + 1], p[4 * v + 2], p[4 * v + 3]);
                    *reinterpret_cast<uint4*>(smem + C::kP + p_at(key, N + col0 + 8 * v)) = make_uint4(rest[4 * v], rest[4 * v + 1], rest[4 * v + 2], rest[4 * v + 3]);
                }
                if (masked && group == 0) {
                    // Rows of V that do not exist may hold anything, and 0 * NaN is NaN: they become zeros, as far as the product
                    // reads.  So does a new token's value that is not finite: those that do not see it have weight 0.  The epilogue adds
                    // it where it is seen.
                    __syncwarp();
                    ok = ok && mbar_wait_a(bar(C::bKvFull + static_cast<int>(v_stage)), v_phase, abort_flag, a.status);
                    const bool odd = is_node && ((s_odd[2 * (seg % kQueue) + (node >> 5)] >> (node & 31)) & 1u) != 0u;
                    if ((odd || (!cached && !is_node)) && key < 16 * used_steps(t, s.keys, new_tile, s.new_at + s.n)) {
                        uint8_t* value = smem + v_stage * C::kTileBytes + key * 128;
#pragma unroll
                        for (int v = 0; v < D / 8; ++v)
                            *reinterpret_cast<uint4*>(value + (v >> 3) * kPanelBytes + (((v ^ key) & 7) << 4)) = make_uint4(0u, 0u, 0u, 0u);
                    }
                }
                fence_proxy_async_smem();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) arrive_a(bar(C::bPFull));
                v_stage += 2;
                if (v_stage >= C::kStages) {
                    v_stage -= C::kStages;
                    v_phase ^= 1;
                }
                page = next;
            }
            if (failed) break;

            // ---- sums over the keys, and the item's outputs: a thread per component ----
            column_sums<kCols>(sum, lane);
            if constexpr (kCols == 32) {
                s_col[quarter * N + col0 + lane] = sum[0];
            } else {
                if ((lane & 1) == 0) s_col[quarter * N + col0 + (lane >> 1)] = sum[0];
            }
            named_sync(id, 128);
            const bool whole = s.part < 0;
            if (tg < kCols) {
                const int c = col0 + tg;
                const float total = (s_col[c] + s_col[N + c]) + (s_col[2 * N + c] + s_col[3 * N + c]);
                s_inv[c] = total == 0.f ? 0.f : 1.f / total;
                const float lse = total == 0.f ? -INFINITY : (log2f(total) - s_neg[c]) * 0.6931471805599453f;
                const int64_t row = whole ? row_of(s.token0, s.head0, s.row0, c, a.g_shift, a.Hq) : static_cast<int64_t>(s.part) * N + c;
                s_to[c] = row * D;
                float* to_lse = whole ? a.LSE : a.part_LSE;
                if (c < n_rows && to_lse != nullptr) to_lse[row] = lse;
            }
            __syncwarp();
            ok = ok && mbar_wait_a(bar(C::bOFull), seg & 1, abort_flag, a.status);
            if (named_any(id, 128, !ok)) break;
            tc_fence_after();
            const uint64_t odd = p_end <= new_tile ? 0ull : s_odd[2 * (seg % kQueue)] | static_cast<uint64_t>(s_odd[2 * (seg % kQueue) + 1]) << 32;
#pragma unroll 1
            for (int c0 = 0; c0 < kCols; c0 += 16) {
                uint32_t r[16], r2[16];
                __syncwarp();
                tmem_ld16(tO + col0 + c0 + my_lanes, r);
                tmem_ld16(tO + N + col0 + c0 + my_lanes, r2);
                tmem_wait_ld();
                if (key >= D) continue;                    // (d = 64: the lower half of the lanes)
                float o[16];
#pragma unroll
                for (int c = 0; c < 16; ++c) {
                    // An infinite value makes the upper part's sum what it is to be; the lower part's, whose weights are 0 or negative as
                    // often as not, would turn it into a NaN.
                    const float upper = __uint_as_float(r[c]);
                    o[c] = fabsf(upper) < INFINITY ? upper + __uint_as_float(r2[c]) : upper;
                }
                for (uint64_t left = odd; left != 0ull; left &= left - 1ull) {
                    const int node = __ffsll(static_cast<long long>(left)) - 1;
                    const uint64_t seen = s_seen[(seg % kQueue) * kMaxTree + node];
                    const float v = __uint_as_float(static_cast<uint32_t>(a.Vnew[(static_cast<int64_t>(s.slot) * a.T + node) * pitch + s.kvh * D + key]) << 16);
                    const int at = s.new_at + node;
#pragma unroll
                    for (int c = 0; c < 16; ++c) {
                        const int col = col0 + c0 + c;
                        if (((seen >> ((s.row0 + col) >> a.g_shift)) & 1ull) == 0ull) continue;
                        const uint32_t p = *reinterpret_cast<const uint16_t*>(smem + C::kP + p_at(at, col) + (col & 7) * 2);
                        o[c] = fmaf(__uint_as_float(p << 16), v, o[c]);
                        if (fabsf(v) < INFINITY) {          // (a component beside the one that is not finite: both parts of its weight)
                            const uint32_t lower = *reinterpret_cast<const uint16_t*>(smem + C::kP + p_at(at, N + col) + (col & 7) * 2);
                            o[c] = fmaf(__uint_as_float(lower << 16), v, o[c]);
                        }
                    }
                }
                int64_t to[16];                            // (read before the first store, which they could depend on)
#pragma unroll
                for (int c = 0; c < 16; ++c) {
                    to[c] = s_to[col0 + c0 + c] + key;
                    o[c] *= s_inv[col0 + c0 + c];
                }
                const int n = min(16, n_rows - (col0 + c0));
                if (!whole || a.out_f32) {
                    float* out = whole ? static_cast<float*>(a.O) : a.part_O;
#pragma unroll
                    for (int c = 0; c < 16; ++c)
                        if (c < n) out[to[c]] = o[c];
                } else {
#pragma unroll
                    for (int c = 0; c < 16; ++c)
                        if (c < n) static_cast<__nv_bfloat16*>(a.O)[to[c]] = __float2bfloat16_rn(o[c]);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_a(bar(C::bOEmpty));
            __syncwarp();
            if (lane == 0) arrive_a(bar(C::bWorkEmpty + static_cast<int>(seg % kQueue)));
        }
    }

    if (kSparse) grid_dependency_wait();
    tc_fence_before();
    __syncthreads();
    if (*abort_flag != 0) {                                // copies that are still under way land before the memory is given back
        const uint64_t t0 = globaltimer_ns();
        while (globaltimer_ns() - t0 < 5000000ull) {
        }
        __syncthreads();
    }
    if (warp == 1) tmem_dealloc(tmem, C::kTmemCols);
}

// Query rows of a CTA: with more than 64 the rows stand in the lanes (paged_wide.cu).
int item_rows(int rows) { return rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : rows <= 128 ? 128 : 256; }

template <int D, int N, bool kSparse, bool kSplit>
int32_t launch(const PagedArgs& a, const Maps& map, cudaStream_t stream) {
    using C = Cfg<D, N, kSparse, kSplit>;
    const auto kernel = paged_tiles_kernel<D, N, kSparse, kSplit>;
    const unsigned ctas = static_cast<unsigned>(sm_count());
    PULSAR_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem));
    PULSAR_CUDA_OK(launch_kernel(kernel, dim3(ctas), dim3(C::kThreads), C::kSmem, stream, true, a, map, 1));
    count_launch();
    return launch_parts_merge(a, static_cast<int64_t>(a.n_slots) * a.items_max, N, D, stream);
}
template <int D, bool kSplit>
int32_t launch_rows(const PagedArgs& a, const Maps& map, int n, cudaStream_t stream) {
    switch (n) {
        case 16: return launch<D, 16, false, kSplit>(a, map, stream);
        case 32: return launch<D, 32, false, kSplit>(a, map, stream);
        default: return launch<D, 64, false, kSplit>(a, map, stream);
    }
}

}  // namespace

// CTAs of a launch that share an item's rows.
int row_blocks(int rows) { return (rows + 255) / 256; }

size_t attn_workspace_bytes(int n_slots, int items, int rows, int d) {
    return PartScratch(static_cast<size_t>(n_slots) * items * row_blocks(rows), sm_count(), item_rows(rows), d).total;
}

int32_t launch_attn(PagedArgs a, int items, int rows, int d, void* workspace, cudaStream_t stream) {
    const int n = item_rows(rows);
    a.items_max = items;
    PartScratch(static_cast<size_t>(a.n_slots) * items * row_blocks(rows), sm_count(), n, d).place(a, workspace);
    a.fresh_rows = static_cast<int>(round_up(a.T, 8));
    Maps map;
    const int64_t pool_rows = static_cast<int64_t>(a.n_pages) << a.page_shift, fresh_rows = static_cast<int64_t>(a.n_slots) * a.T;
    bool ok = make_map_3d(&map.K, a.K, pool_rows, a.Hkv, d, 1, 1 << a.page_shift) && make_map_3d(&map.V, a.V, pool_rows, a.Hkv, d, 1, 1 << a.page_shift) &&
              make_map_3d(&map.Kn, a.Knew, fresh_rows, a.Hkv, d, 1, a.fresh_rows) && make_map_3d(&map.Vn, a.Vnew, fresh_rows, a.Hkv, d, 1, a.fresh_rows) &&
              make_map_3d(&map.Q, a.Q, fresh_rows, a.Hq, d, 1 << a.g_shift, std::min(n, 128) >> a.g_shift);
    map.K16 = map.K;
    map.V16 = map.V;
    if (a.page_shift != 4)
        ok = ok && make_map_3d(&map.K16, a.K, pool_rows, a.Hkv, d, 1, 16) && make_map_3d(&map.V16, a.V, pool_rows, a.Hkv, d, 1, 16);
    if (!ok) return PULSAR_ERR_CUDA;
    if (n > 64) return launch_tree_wide(a, map, rows, d, stream);
    if (a.list != nullptr) return d == 128 ? launch<128, 16, true, false>(a, map, stream) : launch<64, 16, true, false>(a, map, stream);
    if (a.page_shift == 4) return d == 128 ? launch_rows<128, true>(a, map, n, stream) : launch_rows<64, true>(a, map, n, stream);
    return d == 128 ? launch_rows<128, false>(a, map, n, stream) : launch_rows<64, false>(a, map, n, stream);
}

}  // namespace pulsar
