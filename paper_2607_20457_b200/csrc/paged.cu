// Attention over a paged key/value cache: drafted trees (every cached row) and selected pages (include/pulsar.h).
//
// Lengths live on the device, so a launch does not know how much work it has.  A work item is up to eight query rows of one KV
// head (tree: nodes x heads of the group; selected pages: the group's heads of one token) against a list of keys, cut into pieces
// of 16 keys (d = 128; 32 with d = 64).  Every CTA adds up the pieces of all slots, takes an equal share of them, whichever items they
// belong to, and leaves a partial (normalised output and l = ln sum exp) where it holds an item only in part; a second
// launch joins those (paged_merge.cu).
#include <algorithm>

#include "mma.cuh"
#include "paged.cuh"

namespace pulsar {

namespace {

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kRows = 8;                        // query rows of an item: the columns of a matrix fragment
constexpr int kUnitBytes = 4096;
constexpr int kUnits = 3;                       // of a warp's ring: one in use, two on their way
constexpr int kRingBytes = kWarps * kUnits * kUnitBytes;
constexpr int kLeastKeys = 16;                  // of a piece
constexpr int kLeastPieces = 3 * kWarps;        // of a CTA: three per warp, unless all CTAs have fewer

// Two CTAs per SM: while the keys of one are on their way, the other computes.
template <int D, bool kSparse>
__global__ void __launch_bounds__(kThreads, 2)
paged_rows_kernel(const __grid_constant__ PagedArgs a) {
    constexpr int kKeys = kUnitBytes / (2 * D);                // keys of a piece: 16 (d = 128), 32 (d = 64)
    constexpr int kHalves = kKeys / 16;                        // runs of 16 keys lie in one page
    constexpr int kVecs = D / 8;                               // 16-byte vectors of a row
    constexpr int kRowsPerCopy = 32 / kVecs;                   // rows a warp copies with one instruction
    constexpr int kCopies = kKeys / kRowsPerCopy;
    constexpr int kPitch = D + 4;                              // floats of a partial row: 2 * kPitch = 8 modulo the banks
    static_assert(kWarps * kRows * kPitch * 4 <= kRingBytes, "the warps' partials take the ring's place");
    extern __shared__ __align__(1024) uint8_t smem[];
    float2* w_ml = reinterpret_cast<float2*>(smem + kRingBytes);               // [kRows][kWarps]
    uint64_t* s_sees = reinterpret_cast<uint64_t*>(w_ml + kRows * kWarps);     // [kMaxTree] a node's ancestors and itself
    int* s_up = reinterpret_cast<int*>(s_sees + kMaxTree);                     // [kMaxTree]
    Slots& slots = *reinterpret_cast<Slots*>(s_up + kMaxTree);
    float* w_o = reinterpret_cast<float*>(smem);                               // [kWarps][kRows][kPitch], where the rings were

    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int gid = lane >> 2, tig = lane & 3;
    grid_dependency_wait();
    grid_launch_dependents();

    // ---- this CTA's share of all pieces of all slots ----
    if (warp == 0) (void)all_pieces<kSparse, kKeys, kRows>(a, slots);
    __syncthreads();
    const Shares shares(slots.before[a.n_slots], kLeastPieces, gridDim.x);
    const int begin = shares.begin(blockIdx.x), end = shares.begin(blockIdx.x + 1);
    if (begin >= end) {
        if (threadIdx.x == 0) a.meta[blockIdx.x].parts = 0;
        return;
    }
    int slot_now = slot_at(slots, a.n_slots, begin);

    const uint32_t ring = smem_u32(smem) + warp * (kUnits * kUnitBytes);
    const int copy_row = lane / kVecs, copy_vec = lane % kVecs;
    const int64_t pitch = static_cast<int64_t>(a.Hkv) * D;     // elements between the rows of a head
    const int page_mask = (1 << a.page_shift) - 1;
    const int mi = lane >> 3, l8 = lane & 7;
    const uint32_t k_lane = ring + ((mi & 1) * 8 + l8) * (D * 2), k_x = ((mi >> 1) ^ l8) << 4;     // K: rows are keys
    const uint32_t v_lane = ring + ((mi >> 1) * 8 + l8) * (D * 2), v_x = ((mi & 1) ^ l8) << 4;     // V: read transposed
    bool meta_written = false;

    for (int at = begin; at < end;) {
        // ---- the next item and this CTA's pieces of it ----
        const Segment seg = segment_at<kSparse, kKeys, kRows>(a, slots, at, end, slot_now);
        const SlotWork& w = seg.w;
        const int slot = seg.slot, p_begin = seg.p_begin, p_end = seg.p_end, row0 = seg.row0, n_rows = seg.n_rows, kvh = seg.kvh;
        const int token = seg.token, token0 = seg.token0, head0 = seg.head0;
        const bool appends = row0 == 0 && token == 0;
        const int head_at = kvh * D + copy_vec * 8;
        const int32_t* list = kSparse ? a.list + (static_cast<int64_t>(token0) * a.Hkv + kvh) * (a.k + 1)
                                      : a.table + static_cast<int64_t>(slot) * a.max_pages;
        const uint16_t* fresh_k = a.Knew + (static_cast<int64_t>(slot) * a.T) * pitch + head_at;
        const uint16_t* fresh_v = a.Vnew + (static_cast<int64_t>(slot) * a.T) * pitch + head_at;

        // Page ids of a piece; -1 where there is no row.
        struct Ids { int id[kHalves]; };
        const auto pages_of = [&](int p) {
            Ids x;
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
                const int row = p * kKeys + 16 * h;
                x.id[h] = p < p_end && row < w.keys ? list[row >> a.page_shift] : -1;
            }
            return x;
        };
        // Bit h: the rows of half h exist.
        const auto good = [&](const Ids& x, int p) {
            uint32_t ok = 0;
#pragma unroll
            for (int h = 0; h < kHalves; ++h) {
                const bool in = x.id[h] >= 0 && x.id[h] < a.n_pages;
                if (!in && p < p_end && p * kKeys + 16 * h < w.keys && lane == 0) report(a.status, PULSAR_DEV_BAD_PAGE);
                ok |= (in ? 1u : 0u) << h;
            }
            return ok;
        };
        // A unit is K or V of a piece.  Row r goes to line r, its vector v to place v ^ (r & 7), so that the eight rows of a
        // matrix fragment lie in different banks.  Rows that do not exist are zeros.
        const auto load = [&](const uint16_t* pool, const uint16_t* fresh, const Ids& x, uint32_t ok, int p, int place) {
            if (p < p_end) {
                const uint32_t dst = ring + place * kUnitBytes + copy_row * (D * 2);
#pragma unroll
                for (int i = 0; i < kCopies; ++i) {
                    const int r = i * kRowsPerCopy + copy_row, h = i / (kCopies / kHalves);
                    const uint32_t to = dst + i * (kRowsPerCopy * D * 2) + ((copy_vec ^ (r & 7)) << 4);
                    bool in;
                    const uint16_t* src;
                    if (p < w.cache_pieces) {
                        const int row = p * kKeys + r;
                        in = row < w.keys && ((ok >> h) & 1u) != 0u;
                        src = pool + ((static_cast<int64_t>(x.id[h]) << a.page_shift) + (row & page_mask)) * pitch + head_at;
                    } else {
                        const int row = (p - w.cache_pieces) * kKeys + r;
                        in = row < w.n;
                        src = fresh + row * pitch;
                    }
                    cp_async16(to, in ? src : pool, in ? 16 : 0);
                }
            }
            cp_async_commit();                                     // an empty group past the end keeps the count
        };

        const int p_first = p_begin + warp;
        Ids now_ids = pages_of(p_first), next_ids = pages_of(p_first + kWarps);
        uint32_t now_ok = good(now_ids, min(p_first, w.cache_pieces)), next_ok = 0;
        load(a.K, fresh_k, now_ids, now_ok, p_first, 0);
        load(a.V, fresh_v, now_ids, now_ok, p_first, 1);

        // ---- which nodes a node sees ----
        const bool has_new = p_end > w.cache_pieces;
        if (!kSparse && has_new && a.parent != nullptr)
            ancestors(a, slot, w.n, threadIdx.x, s_sees, s_up, [] { __syncthreads(); });
        uint64_t sees[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int r = 2 * tig + k, x = kSparse ? token : (row0 + r) >> a.g_shift;
            sees[k] = r >= n_rows || !has_new ? 0ull : kSparse || a.parent == nullptr ? ~0ull >> (63 - x) : s_sees[x];
        }

        // ---- the query rows as B fragments ----
        uint32_t q[D / 16][2];
        {
            const uint32_t* src = reinterpret_cast<const uint32_t*>(a.Q + row_of(token0, head0, row0, gid < n_rows ? gid : 0, a.g_shift, a.Hq) * D) + tig;
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                q[kk][0] = gid < n_rows ? src[kk * 8] : 0u;
                q[kk][1] = gid < n_rows ? src[kk * 8 + 4] : 0u;
            }
        }
        // rows 2 tig and 2 tig + 1; o[c]: outputs 16 c + gid and 16 c + 8 + gid of both
        float o[D / 16][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
        for (int c = 0; c < D / 16; ++c)
#pragma unroll
            for (int k = 0; k < 4; ++k) o[c][k] = 0.f;

        // Units are consumed in the order K, V, K, V, ... and refilled in that order, each where the unit before it was.
        int place = 0, free_place = kUnits - 1;
        const auto next_unit = [&](const uint16_t* pool, const uint16_t* fresh, int p) {
            cp_async_wait<kUnits - 2>();
            __syncwarp();
            load(pool, fresh, next_ids, next_ok, p, free_place);
            const int here = place;
            free_place = here;
            place = here + 1 == kUnits ? 0 : here + 1;
            return here * kUnitBytes;
        };
        for (int p = p_first; p < p_end; p += kWarps) {
            next_ok = good(next_ids, min(p + kWarps, w.cache_pieces));
            const int at_k = next_unit(a.K, fresh_k, p + kWarps);
            const Ids later_ids = pages_of(p + 2 * kWarps);
            // ---- S^T = K Q^T: keys gid and gid + 8 of each 16, rows 2 tig and 2 tig + 1 ----
            float s[kKeys / 16][4];
#pragma unroll
            for (int j = 0; j < kKeys / 16; ++j) {
                float t[2][4] = {};                                // two chains of products
#pragma unroll
                for (int kk = 0; kk < D / 16; ++kk) {
                    uint32_t f[4];
                    ldmatrix4(k_lane + at_k + j * (16 * D * 2) + ((kk * 32) ^ k_x), f);
                    mma_bf16(t[kk & 1], f, q[kk][0], q[kk][1]);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) s[j][k] = t[0][k] + t[1][k];
            }
            // keys that do not exist, or that the node of a row must not see
            if (p >= w.cache_pieces) {
                const int first = (p - w.cache_pieces) * kKeys;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint32_t bits = static_cast<uint32_t>(sees[k] >> first);        // (node rows past n are nobody's ancestors)
#pragma unroll
                    for (int j = 0; j < kKeys / 16; ++j) {
                        if (((bits >> (16 * j + gid)) & 1u) == 0u) s[j][k] = -INFINITY;
                        if (((bits >> (16 * j + gid + 8)) & 1u) == 0u) s[j][k + 2] = -INFINITY;
                    }
                }
            } else if (w.keys - p * kKeys < kKeys || now_ok != (1u << kHalves) - 1u) {
                const int n_vis = w.keys - p * kKeys;
#pragma unroll
                for (int j = 0; j < kKeys / 16; ++j)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (16 * j + gid + (k >> 1) * 8 >= n_vis || ((now_ok >> j) & 1u) == 0u) s[j][k] = -INFINITY;
            }
            float x[2], alpha[2], neg[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                x[k] = fmaxf(s[0][k], s[0][k + 2]);
#pragma unroll
                for (int j = 1; j < kKeys / 16; ++j) x[k] = max3(x[k], s[j][k], s[j][k + 2]);
            }
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) {
                x[0] = fmaxf(x[0], __shfl_xor_sync(0xffffffffu, x[0], d));
                x[1] = fmaxf(x[1], __shfl_xor_sync(0xffffffffu, x[1], d));
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float m_new = fmaxf(m[k], x[k] * a.scale_log2);
                alpha[k] = m_new == -INFINITY ? 1.f : ex2(m[k] - m_new);
                neg[k] = m_new == -INFINITY ? 0.f : -m_new;
                m[k] = m_new;
            }
            uint32_t pb[kKeys / 16][2];
            l[0] *= alpha[0];
            l[1] *= alpha[1];
#pragma unroll
            for (int j = 0; j < kKeys / 16; ++j) {
#pragma unroll
                for (int k = 0; k < 4; ++k) s[j][k] = ex2(fmaf(s[j][k], a.scale_log2, neg[k & 1]));
                l[0] += s[j][0] + s[j][2];
                l[1] += s[j][1] + s[j][3];
                pb[j][0] = movmatrix(pack_bf16x2(s[j][0], s[j][1]));      // [key][row] -> [row][key]
                pb[j][1] = movmatrix(pack_bf16x2(s[j][2], s[j][3]));
            }
            if (__any_sync(0xffffffffu, alpha[0] != 1.f || alpha[1] != 1.f)) {
#pragma unroll
                for (int c = 0; c < D / 16; ++c)
#pragma unroll
                    for (int k = 0; k < 4; ++k) o[c][k] *= alpha[k & 1];
            }
            // ---- O^T += V^T P^T ----
            const int at_v = next_unit(a.V, fresh_v, p + kWarps);
            bool plain = true;
            if (p >= w.cache_pieces) {
                // A node that a row does not see has weight 0, and 0 times an infinity or a NaN in its value would still reach the
                // row.  Units with such values are added up one visible product at a time.
                const uint16_t* unit_v = reinterpret_cast<const uint16_t*>(smem + warp * (kUnits * kUnitBytes) + at_v);
                uint32_t odd = 0;
                for (int i = lane; i < kUnitBytes / 4; i += 32) {
                    const uint32_t x = reinterpret_cast<const uint32_t*>(unit_v)[i];
                    odd |= (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u ? 1u : 0u;
                }
                plain = !__any_sync(0xffffffffu, odd != 0u);
                if (!plain) {
                    const int first = (p - w.cache_pieces) * kKeys;
#pragma unroll 1
                    for (int key = 0; key < kKeys; ++key) {
                        const uint16_t* v = unit_v + key * D + (gid & 7);
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const float a0 = s[0][k], a1 = s[0][k + 2];
                            float x = key & 8 ? a1 : a0;
                            if (kKeys > 16) x = key & 16 ? (key & 8 ? s[kKeys / 16 - 1][k + 2] : s[kKeys / 16 - 1][k]) : x;
                            x = __shfl_sync(0xffffffffu, x, (key & 7) * 4 + tig);
                            if (((sees[k] >> (first + key)) & 1u) == 0u) continue;
#pragma unroll
                            for (int c = 0; c < D / 16; ++c) {
                                const uint32_t v0 = v[((2 * c) ^ (key & 7)) * 8], v1 = v[((2 * c + 1) ^ (key & 7)) * 8];
                                o[c][k] = fmaf(x, __uint_as_float(v0 << 16), o[c][k]);
                                o[c][k + 2] = fmaf(x, __uint_as_float(v1 << 16), o[c][k + 2]);
                            }
                        }
                    }
                }
            }
            if (plain) {
#pragma unroll
                for (int j = 0; j < kKeys / 16; ++j)
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) {
                        uint32_t f[4];
                        ldmatrix4_trans(v_lane + at_v + j * (16 * D * 2) + ((c * 32) ^ v_x), f);
                        mma_bf16(o[c], f, pb[j][0], pb[j][1]);
                    }
            }
            // The new tokens' rows go to their pages from the warp that has just read them (nobody reads those rows in this launch).
            if (appends && p >= w.cache_pieces) {
#pragma unroll 1
                for (int i = 0; i < kCopies; ++i) {
                    const int row = (p - w.cache_pieces) * kKeys + i * kRowsPerCopy + copy_row;
                    if (row >= w.n) continue;
                    int64_t to = new_row_at(a, slot, static_cast<int64_t>(w.len) + row, pitch);
                    if (to < 0) continue;
                    to += head_at;
                    *reinterpret_cast<uint4*>(a.K + to) = *reinterpret_cast<const uint4*>(fresh_k + row * pitch);
                    *reinterpret_cast<uint4*>(a.V + to) = *reinterpret_cast<const uint4*>(fresh_v + row * pitch);
                }
            }
            now_ok = next_ok;
            next_ids = later_ids;
        }
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) {
            l[0] += __shfl_xor_sync(0xffffffffu, l[0], d);
            l[1] += __shfl_xor_sync(0xffffffffu, l[1], d);
        }

        // ---- the warps' partials, brought to the CTA's maximum and added up, 32 outputs of a row per warp ----
        if (gid == 0) {
            w_ml[(2 * tig) * kWarps + warp] = make_float2(m[0], l[0]);
            w_ml[(2 * tig + 1) * kWarps + warp] = make_float2(m[1], l[1]);
        }
        __syncthreads();
        float f[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) f[k] = w_ml[(2 * tig + k) * kWarps + gid].x;
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) {
            f[0] = fmaxf(f[0], __shfl_xor_sync(0xffffffffu, f[0], d));
            f[1] = fmaxf(f[1], __shfl_xor_sync(0xffffffffu, f[1], d));
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            f[k] = weight(m[k], f[k]);
            if (2 * tig + k < n_rows) {
                float* dst = w_o + (warp * kRows + 2 * tig + k) * kPitch + gid;
#pragma unroll
                for (int c = 0; c < D / 16; ++c) {
                    dst[16 * c] = o[c][k] * f[k];
                    dst[16 * c + 8] = o[c][k + 2] * f[k];
                }
            }
        }
        __syncthreads();
        const bool whole = p_begin == 0 && p_end == w.pieces;
        const int64_t part = 2 * static_cast<int64_t>(blockIdx.x) + (at == begin ? 0 : 1);
        for (int c = warp; c < n_rows * (D / 32); c += kWarps) {
            const int r = c / (D / 32), at_d = (c % (D / 32)) * 32 + lane;
            const float* src = w_o + r * kPitch + at_d;
            float y[2] = {0.f, 0.f};
#pragma unroll
            for (int v = 0; v < kWarps; ++v) y[v & 1] += src[v * (kRows * kPitch)];
            const float2 ml = lane < kWarps ? w_ml[r * kWarps + lane] : make_float2(-INFINITY, 0.f);
            const float M = warp_max(ml.x), sum = low_lanes_sum<kWarps>(weight(ml.x, M) * ml.y);
            const float out = (y[0] + y[1]) * (sum == 0.f ? 0.f : 1.f / sum);
            const float lse = sum == 0.f ? -INFINITY : (M + log2f(sum)) * 0.6931471805599453f;
            if (!whole) {
                a.part_O[(part * kRows + r) * D + at_d] = out;
                if (at_d == 0) a.part_LSE[part * kRows + r] = lse;
                continue;
            }
            const int64_t row = row_of(token0, head0, row0, r, a.g_shift, a.Hq);
            if (a.out_f32) {
                static_cast<float*>(a.O)[row * D + at_d] = out;
            } else {
                const float z = __shfl_xor_sync(0xffffffffu, out, 1);
                if ((lane & 1) == 0) *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.O) + row * D + at_d) = pack_bf16x2(out, z);
            }
            if (at_d == 0 && a.LSE != nullptr) a.LSE[row] = lse;
        }
        // An item that begins here and goes on elsewhere is this CTA's last; the CTAs up to the one with its last piece have a part each.
        if (p_begin == 0 && p_end < w.pieces) {
            if (threadIdx.x == 0) {
                a.meta[blockIdx.x] = {static_cast<int>(part), shares.owner(seg.item_at + w.pieces - 1) - static_cast<int>(blockIdx.x) + 1, 1, token0, head0, row0, n_rows};
            }
            meta_written = true;
        }
        at = seg.item_at + p_end;
        __syncthreads();                         // the ring is loaded into again
    }
    if (!meta_written && threadIdx.x == 0) a.meta[blockIdx.x].parts = 0;
}

// ---------------------------------------------------------------------------------------------
// Scores of the full pages and the k best.
//
// sum_j (q_j > 0 ? q_j max_j : q_j min_j) is one product of length 2 d: the negative parts of the query with the smallest components, the
// positive ones with the largest.  The tensor cores form it for all pages and rows in fp32, which is what the memory's rate leaves
// time for (in float64 on the FMA pipe 16 slots of 45,000 rows took 70 us); the ranking is that of the float64 scores all the
// same: a page whose fp32 score lies further from the k-th than both can be off is in or out, and the few others are formed again in
// float64.
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
page_score_kernel(const __grid_constant__ SelectArgs a) {
    constexpr int kChunks = 2 * D / 32;          // of 32 products: a lane has 8 consecutive ones, 16 bytes, of two pages
    constexpr int kPitch = 2 * D + 32;           // of a query row in shared memory: two rows' vectors fill the banks
    __shared__ __align__(16) uint16_t s_q[kScoreRows * kPitch];
    __shared__ float s_most[kScoreThreads / 32];
    const int slot = blockIdx.z, kvh = blockIdx.y, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gid = lane >> 2, tig = lane & 3;
    grid_dependency_wait();
    grid_launch_dependents();
    const int len = checked_len(a.len[slot], static_cast<int64_t>(a.max_pages) << a.page_shift, false, nullptr);
    const int full = len >> a.page_shift, b0 = blockIdx.x * kScorePages;
    if (full <= a.k || b0 >= full) return;       // (all pages are taken as they are)
    const int n = a.n_draft != nullptr ? min(max(a.n_draft[slot], 0), a.T) : a.T, g = 1 << a.g_shift, rows = n * g;
    if (rows == 0) return;

    // ---- the bounds of pages gid and gid + 8 of the warp's 16, as A fragments: products are summed in the order of these vectors ----
    uint4 f[2][kChunks];
    bool known[2];
    const int page0 = b0 + warp * 16 + gid;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int b = page0 + 8 * h;
        const int page = b < full ? a.table[static_cast<int64_t>(slot) * a.max_pages + b] : -1;
        known[h] = page >= 0 && page < a.n_pages;
        if (b < full && !known[h] && tig == 0) report(a.status, PULSAR_DEV_BAD_PAGE);
        const uint4* src = reinterpret_cast<const uint4*>(a.summary + (static_cast<int64_t>(known[h] ? page : 0) * a.Hkv + kvh) * 2 * D) + tig;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) f[h][c] = known[h] ? src[4 * c] : make_uint4(0u, 0u, 0u, 0u);
    }
    {
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
    float best[2];                               // g = 16: of the row tile before
    for (int r0 = 0; r0 < rows; r0 += kScoreRows) {
        __syncthreads();
        if (r0 == 0 && threadIdx.x == 0)
            a.most[(static_cast<int64_t>(slot) * a.Hkv + kvh) * gridDim.x + blockIdx.x] = fmaxf(fmaxf(s_most[0], s_most[1]), fmaxf(s_most[2], s_most[3]));
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
        __syncthreads();
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
    float value[kTopWarps];
    int count[2][kTopWarps];
    uint64_t near_key[kNear], cut_key;
    int near_at[kNear], n_near, cut_at, bin, above;
    int odd;                                     // a score that is not finite
};

// Largest (or smallest: of the negated values) over the CTA.
__device__ __forceinline__ float block_max(float x, float* s) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = x;
    __syncthreads();
    x = s[threadIdx.x & (kTopWarps - 1)];
#pragma unroll
    for (int d = kTopWarps / 2; d > 0; d >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
    return x;
}
// Of two flags: how many threads before this one have them, and how many in all.
__device__ __forceinline__ void block_counts(const bool (&flag)[2], int (&before)[2], int (&all)[2], int (&s)[2][kTopWarps]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t m[2] = {__ballot_sync(0xffffffffu, flag[0]), __ballot_sync(0xffffffffu, flag[1])};
    __syncthreads();
    if (lane < 2) s[lane][warp] = __popc(m[lane]);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int c = s[i][lane & (kTopWarps - 1)];
        int x = lane < warp ? c : 0, y = lane < kTopWarps ? c : 0;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) {
            x += __shfl_xor_sync(0xffffffffu, x, d);
            y += __shfl_xor_sync(0xffffffffu, y, d);
        }
        before[i] = x + __popc(m[i] & ((1u << lane) - 1u));
        all[i] = y;
    }
}

template <int D>
__global__ void __launch_bounds__(kTopThreads)
page_select_kernel(const __grid_constant__ SelectArgs a, int blocks) {
    __shared__ TopScratch s;
    const int row = blockIdx.x, t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const int token0 = row / a.Hkv, kvh = row - token0 * a.Hkv, slot = token0 / a.T, u = token0 - slot * a.T, g = 1 << a.g_shift;
    grid_dependency_wait();
    grid_launch_dependents();
    const int len = checked_len(a.len[slot], static_cast<int64_t>(a.max_pages) << a.page_shift, false, nullptr);
    const int full = len >> a.page_shift, k = min(a.k, full);
    if (a.n_draft != nullptr && u >= a.n_draft[slot]) return;
    const float* score = a.score + static_cast<int64_t>(row) * a.max_pages;
    uint64_t* exact = a.exact + static_cast<int64_t>(row) * a.max_pages;
    int32_t* sel = a.sel + static_cast<int64_t>(row) * a.k;
    int32_t* list = a.list + static_cast<int64_t>(row) * (a.k + 1);
    const int32_t* table = a.table + static_cast<int64_t>(slot) * a.max_pages;

    // Pages [first, last) are ranked, `want` of them taken; those before and after are taken anyway.
    const bool all = full <= a.k;
    const int first = min(a.sink, full), last = max(first, full - a.window), want = all ? 0 : k - first - (full - last);
    const bool ranked = !all && want > 0;
    float held[kTopHeld], above = INFINITY, below = INFINITY;      // scores over `above` are taken, under `below` not, the others ranked
    const auto at = [&](int i) { return first + t + i * kTopThreads; };
    const int rounds = (last - first + kTopThreads - 1) / kTopThreads;
    const auto value = [&](int i) { return at(i) < last ? score[at(i)] : -INFINITY; };
    if (ranked) {
        float lo = INFINITY, hi = -INFINITY;
        bool odd = false;
        if (t == 0) {
            s.odd = 0;
            s.n_near = 0;
        }
        for (int i = t; i < kBins; i += kTopThreads) s.bins[i] = 0;
        const auto look = [&](float x) {
            odd |= !(x < INFINITY);
            if (x > -INFINITY) {
                lo = fminf(lo, x);
                hi = fmaxf(hi, x);
            }
        };
#pragma unroll
        for (int i = 0; i < kTopHeld; ++i) held[i] = value(i);
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
        float most = 0.f;
        for (int i = t; i < (full + kScorePages - 1) / kScorePages; i += kTopThreads)
            most = fmaxf(most, a.most[(static_cast<int64_t>(slot) * a.Hkv + kvh) * blocks + i]);
#pragma unroll
        for (int i = 0; i < kTopHeld; ++i) look(held[i]);
        for (int i = kTopHeld; i < rounds; ++i) look(value(i));
        lo = -block_max(-lo, s.value);
        hi = block_max(hi, s.value);
        const float size = block_max(q1, s.value) * block_max(most, s.value);
        if (odd) s.odd = 1;
        __syncthreads();
        const bool rough = s.odd != 0 || !(size < 1e37f) || !(hi > lo);      // fp32 says nothing: all are ranked in float64
        if (!rough) {
            // ---- the bin of the want-th largest score ----
            const float inv = kBins / (hi - lo);
            const auto bin_of = [&](float x) { return min(max(static_cast<int>((x - lo) * inv), 0), kBins - 1); };
#pragma unroll
            for (int i = 0; i < kTopHeld; ++i)
                if (at(i) < last) atomicAdd(&s.bins[bin_of(held[i])], 1);
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
            if (lane == 31) s.count[0][warp] = x;
            __syncthreads();
            int over = x - n0 - n1;
            for (int w = 0; w < warp; ++w) over += s.count[0][w];
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
            for (int i = 0; i < kTopHeld; ++i) inside(i, held[i]);
            for (int i = kTopHeld; i < rounds; ++i) inside(i, value(i));
            const float e = 2.f * kScoreError * size;
            in_lo = -block_max(-in_lo, s.value);
            in_hi = block_max(in_hi, s.value);
            above = nextafterf(in_hi + e, INFINITY);                         // (outward: the sums are rounded)
            below = nextafterf(in_lo - e, -INFINITY);
        } else {
            below = -INFINITY;                    // (`above` is infinite)
        }
    }
    const auto is_near = [&](float x) { return !(x > above) && !(x < below); };

    // ---- pages between the two borders are ranked in float64 ----
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
        for (int i = 0; i < kTopHeld; ++i) sort_out(i, held[i]);
        for (int i = kTopHeld; i < rounds; ++i) sort_out(i, value(i));
        taken = static_cast<int>(__reduce_add_sync(0xffffffffu, taken));
        __syncthreads();
        if (lane == 0) s.count[0][warp] = taken;
        __syncthreads();
        int left = want;                          // pages to take from those in between
        for (int w = 0; w < kTopWarps; ++w) left -= s.count[0][w];
        const int n_near = s.n_near;
        if (n_near <= kNear) {
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
                const bool flag[2] = {b < last && is_near(score[b]) && exact[b] == kth, false};
                int before[2], total[2];
                block_counts(flag, before, total, s.count);
                if (flag[0] && done + before[0] == left - 1) {
                    s.cut_key = kth;
                    s.cut_at = b;
                }
                done += total[0];
            }
            __syncthreads();
        }
    }

    // ---- the taken pages in ascending order ----
    const uint64_t cut_key = ranked ? s.cut_key : 0;
    const int cut_at = ranked ? s.cut_at : 0;
    int done = 0;
    for (int b0 = 0; b0 < full; b0 += kTopThreads) {
        const int b = b0 + t;
        bool take = b < full && (all || b < first || b >= last);
        if (ranked && b >= first && b < last) {
            const float x = score[b];
            if (!is_near(x)) {
                take = x > above;
            } else {
                const uint64_t key = exact[b];
                take = key > cut_key || (key == cut_key && b <= cut_at);
            }
        }
        const bool flag[2] = {take, false};
        int before[2], total[2];
        block_counts(flag, before, total, s.count);
        if (take) {
            sel[done + before[0]] = b;
            list[done + before[0]] = table[b];
        }
        done += total[0];
    }
    for (int i = k + t; i < a.k; i += kTopThreads) sel[i] = -1;
    if (t == 0 && len > full << a.page_shift) list[k] = table[full];      // the page of the rows after the last full one
}

// ---------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------
constexpr int kSmemBytes = kRingBytes + kRows * kWarps * 8 + kMaxTree * 8 + kMaxTree * 4 + static_cast<int>(sizeof(Slots));

bool heads_ok(int32_t Hq, int32_t Hkv) {
    if (Hkv < 1 || Hq < Hkv || Hq % Hkv != 0) return false;
    const int g = Hq / Hkv;
    return g == 1 || g == 2 || g == 4 || g == 8 || g == 16;
}

PartScratch rows_scratch(int d) { return PartScratch(2 * static_cast<size_t>(sm_count()), kRows, d); }

template <typename Kernel>
int32_t launch_rows(Kernel kernel, const PagedArgs& a, int d, cudaStream_t st) {
    const unsigned ctas = 2 * static_cast<unsigned>(sm_count());
    PULSAR_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes));
    PULSAR_CUDA_OK(launch_kernel(kernel, dim3(ctas), dim3(kThreads), kSmemBytes, st, true, a));
    count_launch();
    return launch_parts_merge(a, ctas, kRows, d, st);
}

float scale_log2(float softmax_scale, int32_t d) {
    return (softmax_scale > 0.f ? softmax_scale : 1.f / sqrtf(static_cast<float>(d))) * 1.4426950408889634f;
}

}  // namespace
}  // namespace pulsar

using namespace pulsar;

extern "C" size_t pulsar_tree_attn_workspace_bytes(int32_t n_slots, int32_t T, int32_t Hq, int32_t Hkv, int32_t d) {
    if (n_slots < 1 || n_slots > kMaxSlots || T < 1 || T > kMaxTree || !heads_ok(Hq, Hkv) || (d != 64 && d != 128)) return 0;
    const int rows = T * (Hq / Hkv);
    return rows > kRows ? tree_tiles_workspace_bytes(rows, d) : rows_scratch(d).total;
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
    for (const void* p : {static_cast<const void*>(Q), static_cast<const void*>(Knew), static_cast<const void*>(Vnew),
                          static_cast<const void*>(K_pages), static_cast<const void*>(V_pages), static_cast<const void*>(O)})
        if (!aligned(p, 16)) return PULSAR_ERR_ALIGNMENT;
    if (!aligned(page_table, 4) || !aligned(cache_len, 4) || !aligned(parent, 4) || !aligned(n_draft, 4) || !aligned(LSE, 4) ||
        !aligned(workspace, 256))
        return PULSAR_ERR_ALIGNMENT;
    if (!(T * (Hq / Hkv) > kRows ? tree_tiles_ok(n_slots, Hkv, static_cast<int64_t>(max_pages) * page_size, T)
                                 : pieces_ok(n_slots, Hkv, static_cast<int64_t>(max_pages) * page_size, T, kLeastKeys)))
        return PULSAR_ERR_SHAPE;
    if (workspace_bytes < pulsar_tree_attn_workspace_bytes(n_slots, T, Hq, Hkv, d)) return PULSAR_ERR_WORKSPACE;
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
    const int rows = T * (Hq / Hkv);
    if (rows > kRows) return launch_tree_tiles(a, rows, d, workspace, static_cast<cudaStream_t>(stream));
    rows_scratch(d).place(a, workspace);
    return launch_rows(d == 128 ? paged_rows_kernel<128, false> : paged_rows_kernel<64, false>, a, d, static_cast<cudaStream_t>(stream));
}

namespace {
struct SparseScratch {
    size_t exact, score, most, list, total;
    SparseScratch(int64_t n_slots, int64_t T, int64_t Hkv, int64_t max_pages, int64_t k, int d) {
        const int64_t rows = n_slots * T * Hkv;
        exact = rows_scratch(d).total;
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
    return SparseScratch(n_slots, T, Hkv, max_pages, k, d).total;
}

extern "C" int32_t pulsar_sparse_attn(const uint16_t* Q, const uint16_t* Knew, const uint16_t* Vnew, int32_t T, uint16_t* K_pages,
                                      uint16_t* V_pages, const uint16_t* summary, int32_t n_pages, int32_t page_size,
                                      const int32_t* page_table, const int32_t* cache_len, int32_t n_slots, int32_t max_pages,
                                      const int32_t* n_draft, int32_t k, int32_t sink, int32_t window, int32_t Hq, int32_t Hkv, int32_t d,
                                      float softmax_scale, uint16_t* O, float* LSE, int32_t* sel, void* workspace,
                                      size_t workspace_bytes, int32_t* device_status, void* stream) {
    if (!pool_ok(1, n_pages, page_size, Hkv, d, n_slots, max_pages) || !sparse_ok(n_slots, T, k, Hq, Hkv, d) || sink < 0 || window < 0 ||
        static_cast<int64_t>(sink) + window > k ||
        !pieces_ok(n_slots, static_cast<int64_t>(T) * Hkv * 2, std::min<int64_t>(k + 1, max_pages) * page_size, T, kLeastKeys))
        return PULSAR_ERR_SHAPE;
    if (Q == nullptr || Knew == nullptr || Vnew == nullptr || K_pages == nullptr || V_pages == nullptr || summary == nullptr ||
        page_table == nullptr || cache_len == nullptr || O == nullptr || sel == nullptr || workspace == nullptr)
        return PULSAR_ERR_INVALID_ARG;
    for (const void* p : {static_cast<const void*>(Q), static_cast<const void*>(Knew), static_cast<const void*>(Vnew), static_cast<const void*>(summary),
                          static_cast<const void*>(K_pages), static_cast<const void*>(V_pages), static_cast<const void*>(O)})
        if (!aligned(p, 16)) return PULSAR_ERR_ALIGNMENT;
    if (!aligned(page_table, 4) || !aligned(cache_len, 4) || !aligned(n_draft, 4) || !aligned(LSE, 4) || !aligned(sel, 4) || !aligned(workspace, 256))
        return PULSAR_ERR_ALIGNMENT;
    const int64_t rows = static_cast<int64_t>(n_slots) * T * Hkv;
    const SparseScratch y(n_slots, T, Hkv, max_pages, k, d);
    if (workspace_bytes < y.total) return PULSAR_ERR_WORKSPACE;
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
    PULSAR_CUDA_OK(launch_kernel(d == 128 ? page_score_kernel<128> : page_score_kernel<64>, dim3(blocks, Hkv, n_slots), dim3(kScoreThreads), 0, st,
                                 true, b));
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
    rows_scratch(d).place(a, ws);
    return launch_rows(d == 128 ? paged_rows_kernel<128, true> : paged_rows_kernel<64, true>, a, d, st);
}
