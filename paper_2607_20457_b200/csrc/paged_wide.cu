// Attention of drafted trees with more than 64 query rows per KV head, on the tensor cores (tcgen05).
//
// S = Q K^T with 128 query rows (nodes x heads of the group) in the TMEM lanes, so that a softmax thread has a row: its maximum and its
// sum need no other thread, and P goes back to TMEM as the first operand of O += P V.  (With the keys in the lanes, as for fewer rows in
// paged_tiles.cu, four warpgroups wait for each other at every tile: a tile of 96 rows took 3050 cycles of which HBM's share is
// 2800.)
//
// Two streams, each with its own S (and P), O, maximum and sum in 128 + D columns of TMEM and a softmax warpgroup:
//   kTwo     up to 256 rows: stream h has rows 128 h .., every tile of keys is both streams' -- one computes while the other is
//            exponentiated
//   else     up to 128 rows: the streams take the tiles of keys in turn and are joined when the item ends
//
//   warp 0 loader, warp 1 issues the matrix instructions, warps 2-3 query rows and nodes (paged_roles.cuh), warps 4-11 softmax and epilogue
//
// As in paged_tiles.cu the maximum is moved, and O rescaled, only when a logit exceeds it by more than 2^8 (in the first 96 keys of a tile:
// when their probabilities sum to more than 96 * 2^8).  The sums stay in fp32; P is rounded to bf16, each probability by at most 2^-8 of
// itself, which makes the outputs 0.0023 off the 64-bit result where their own last rounding is 0.0017.  In two bf16 parts, as in
// paged_tiles.cu, it would cost a second product on the pipe that sets the pace: 99 -> 125 us (96 rows), 169 -> 219 (256 rows).
//
// P is handed to the issuer in two pieces (96 and 32 keys), so that the first piece of PV runs beside the rest.
//
// What bounds it: up to 128 rows, 4 slots of up to 32,768 rows with 24 nodes (96 rows) 94 to 101 us, 0.7 of HBM's rate; more, one slot of
// 131,072 rows with 64 nodes (256 rows) 159 to 171 us, 0.5 of the tensor cores' burst rate: the chain S -> softmax -> PV -> S of a stream, of
// which the other stream hides a part (its products take 2048 cycles of a tile of about 3200).  The twelve warps have 168 registers each,
// and a row of 128 logits is most of them: up to 128 rows 72 bytes are spilled and 60 read back per thread, with more rows 28 and 12.
#include "mma.cuh"
#include "paged_roles.cuh"

namespace pulsar {

namespace {

constexpr int kThreads = 384;
constexpr int kJoinCols = 16;                    // outputs of a row that the streams exchange at a time
constexpr int kJoinPitch = kJoinCols + 1;
constexpr int kFirst = 96;                       // keys of a tile whose P is handed over first, so that their product runs beside the rest
constexpr int kJoinBarrier = 1;                  // named barrier of both softmax warpgroups

template <int D, bool kTwo>
struct Wide {
    static constexpr int kPanels = D / 64, kTileBytes = kPanels * kPanelBytes;
    static constexpr int kQTiles = kTwo ? 2 : 1, kQRows = 128, kRows = kQTiles * 128;
    static constexpr int kQBytes = kQTiles * kTileBytes;
    static constexpr bool kBySeen = false, kSparse = false, kTwoLoaders = false;
    static constexpr int kJoinBytes = kTwo ? 0 : 2 * 128 * kJoinPitch * 4 + 2 * 128 * 8;
    static constexpr int kMisc = kQueue * (kMaxTree * 8 + 64 + 8) + 64 * 8 + kMaxTree * 4 + 8 + static_cast<int>(sizeof(Slots)) + 12;
    static constexpr int kFit = (232448 - kQBytes - kJoinBytes - kMisc) / kTileBytes;
    static constexpr int kStages = kFit < 10 ? kFit : 10;
    static constexpr int kQ = kStages * kTileBytes, kJoin = kQ + kQBytes, kRest = kJoin + kJoinBytes, kSmem = kRest + kMisc;
    static constexpr int bKvFull = 0, bKvEmpty = kStages, bQFull = 2 * kStages, bQEmpty = bQFull + 1, bSFull = bQEmpty + 1, bPFull = bSFull + 2,
                         bPRest = bPFull + 2, bOFull = bPRest + 2, bOEmpty = bOFull + 2, bSees = bOEmpty + 2, bWorkFull = bSees + kQueue, bWorkEmpty = bWorkFull + kQueue,
                         kBars = bWorkEmpty + kQueue;
    static_assert(kBars <= 64 && kStages >= 4 && kRest % 16 == 0, "");
};

// x * s + n for two logits.
__device__ __forceinline__ void scaled2(float& y0, float& y1, float x0, float x1, float s, float n) {
    asm("{\n\t.reg .b64 a, b, c;\n\t"
        "mov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %4};\n\tmov.b64 c, {%5, %5};\n\t"
        "fma.rn.f32x2 a, a, b, c;\n\t"
        "mov.b64 {%0, %1}, a;\n\t}"
        : "=f"(y0), "=f"(y1) : "f"(x0), "f"(x1), "f"(s), "f"(n));
}

// The low n bits (n from 0 to 32).
__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; }

template <int D, bool kTwo>
__global__ void __launch_bounds__(kThreads, 1)
tree_wide_kernel(const __grid_constant__ PagedArgs a, const __grid_constant__ Maps map, int row_blocks) {
    using C = Wide<D, kTwo>;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint64_t* s_sees = reinterpret_cast<uint64_t*>(smem + C::kRest);
    Work* s_work = reinterpret_cast<Work*>(s_sees + kQueue * kMaxTree);
    uint64_t* bars = reinterpret_cast<uint64_t*>(s_work + kQueue);
    int* s_up = reinterpret_cast<int*>(bars + 64);
    uint32_t* s_odd = reinterpret_cast<uint32_t*>(s_up + kMaxTree);
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
        for (int h = 0; h < 2; ++h) {
            mbar_init(bars + C::bSFull + h, 1);
            mbar_init(bars + C::bPFull + h, 4);
            mbar_init(bars + C::bPRest + h, 4);
            mbar_init(bars + C::bOFull + h, 1);
            mbar_init(bars + C::bOEmpty + h, 4);
        }
        for (int i = 0; i < kQueue; ++i) {
            mbar_init(bars + C::bSees + i, 1);
            mbar_init(bars + C::bWorkFull + i, 1);
            mbar_init(bars + C::bWorkEmpty + i, 8 + 3);
        }
        mbar_fence_init();
        prefetch_maps(map);
    }
    if (warp == 1) {
        tmem_alloc(tmem_ptr, 512);
        tmem_relinquish();
    }
    grid_dependency_wait();
    grid_launch_dependents();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_ptr;
    const Roles roles{smem, s_work, s_sees, s_odd, s_up, &slots, bar0, abort_flag};

    if (warp == 0) {
        load_role<C>(a, map, row_blocks, roles);
    } else if (warp == 1) {
        // ---- matrix instructions.  They run in the order of issue, so S of a stream's next tile may follow PV of the tile before into the
        // same columns, and a full S means that the PV before it is done. ----
        const bool leader = elect_one();
        constexpr uint32_t kIdescS = umma_idesc_bf16(128, kTile, false, false), kIdescO = umma_idesc_bf16(128, D, false, true);
        const uint64_t desc_k = umma_smem_desc_sw128(smem_u32(smem), 16, 1024);
        const uint64_t desc_v = umma_smem_desc_sw128(smem_u32(smem), kPanelBytes, 1024);
        const uint64_t desc_q = umma_smem_desc_sw128(smem_u32(smem + C::kQ), 16, 1024);
        uint32_t tile = 0, stage = 0, phase = 0, v_stage = 0, v_phase = 0;
        int steps = 0;                                     // of 16 keys, of the tile whose PV is due
        uint32_t o_use[2] = {0, 0};                        // items that the stream has begun
        bool ok = true, first = false, last = false;       // of the tile whose PV is due (kTwo: the item's first, last; else the stream's)
        const auto wait = [&](int b, uint32_t parity) {
            __syncwarp();
            ok = __all_sync(0xffffffffu, ok && mbar_wait_a(bar(b), parity, abort_flag, a.status));
        };
        const auto issue_s = [&](int h, int q_tile, bool release_k, bool release_q) {
            tc_fence_after();
            if (!leader) return;
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
                const uint32_t off = static_cast<uint32_t>((kk >> 2) * kPanelBytes + (kk & 3) * 32) >> 4;
                umma_ss(tmem + h * 128, desc_q + static_cast<uint64_t>(q_tile * (C::kTileBytes >> 4) + off),
                        desc_k + static_cast<uint64_t>(stage * (C::kTileBytes >> 4) + off), kIdescS, kk > 0 ? 1u : 0u);
            }
            umma_commit_a(bar(C::bSFull + h));
            if (release_k) umma_commit_a(bar(C::bKvEmpty + static_cast<int>(stage)));
            if (release_q) umma_commit_a(bar(C::bQEmpty));
        };
        const auto issue_pv = [&](int h, uint32_t parity, bool release_v) {
            if (first) wait(C::bOEmpty + h, (o_use[h] & 1) ^ 1);
            wait(C::bPFull + h, parity);
            if (!ok) return;
            tc_fence_after();
            const auto product = [&](int kk) {
                if (kk < steps) umma_ts(tmem + 256 + h * 128, tmem + h * 128 + kk * 8, desc_v + static_cast<uint64_t>(v_stage * (C::kTileBytes >> 4) + kk * 128), kIdescO,
                        first && kk == 0 ? 0u : 1u);
            };
            if (leader) {
#pragma unroll
                for (int kk = 0; kk < kFirst / 16; ++kk) product(kk);
            }
            wait(C::bPRest + h, parity);
            if (!ok) return;
            tc_fence_after();
            if (leader) {
#pragma unroll
                for (int kk = kFirst / 16; kk < kTile / 16; ++kk) product(kk);
                if (release_v) umma_commit_a(bar(C::bKvEmpty + static_cast<int>(v_stage)));
                if (last) umma_commit_a(bar(C::bOFull + h));
            }
            if (first) ++o_use[h];
        };
        const auto next_stage = [&] {
            if (++stage == C::kStages) {
                stage = 0;
                phase ^= 1;
            }
        };
        for (uint32_t seq = 0;; ++seq) {
            const Work* s = next_work<C>(a, roles, seq, ok);
            if (!ok || s->valid == 0) break;
            const int p_begin = s->p_begin, p_end = s->p_end, keys = s->keys, new_tile = s->new_tile, new_end = s->new_at + s->n;
            __syncwarp();
            if (lane == 0) arrive_a(bar(C::bWorkEmpty + static_cast<int>(seq % kQueue)));
            for (int t = p_begin; t < p_end && ok; ++t, ++tile) {
                const bool due = tile > 0, end = t + 1 == p_end;
                if (kTwo) {
                    if (due) {
                        wait(C::bKvFull + static_cast<int>(v_stage), v_phase);
                        issue_pv(0, (tile - 1) & 1, false);
                    }
                    wait(C::bKvFull + static_cast<int>(stage), phase);
                    if (t == p_begin) wait(C::bQFull, seq & 1);
                    if (!ok) break;
                    issue_s(0, 0, false, false);
                    if (due) issue_pv(1, (tile - 1) & 1, true);
                    if (!ok) break;
                    issue_s(1, 1, true, end);
                } else {
                    wait(C::bKvFull + static_cast<int>(stage), phase);
                    if (t == p_begin) wait(C::bQFull, seq & 1);
                    if (!ok) break;
                    issue_s(static_cast<int>(tile & 1), 0, true, end);
                    if (due) {
                        wait(C::bKvFull + static_cast<int>(v_stage), v_phase);
                        issue_pv(static_cast<int>((tile - 1) & 1), ((tile - 1) >> 1) & 1, true);
                    }
                }
                next_stage();
                v_stage = stage;
                v_phase = phase;
                next_stage();
                first = t - p_begin < (kTwo ? 1 : 2);
                last = t >= p_end - (kTwo ? 1 : 2);
                steps = used_steps(t, keys, new_tile, new_end);
            }
        }
        if (ok && tile > 0) {
            wait(C::bKvFull + static_cast<int>(v_stage), v_phase);
            if (kTwo) {
                issue_pv(0, (tile - 1) & 1, false);
                if (ok) issue_pv(1, (tile - 1) & 1, true);
            } else {
                issue_pv(static_cast<int>((tile - 1) & 1), ((tile - 1) >> 1) & 1, true);
            }
        }
    } else if (warp == 2) {
        rows_role<C>(a, map, roles);
    } else if (warp == 3) {
        nodes_role<D, C>(a, roles);
    } else {
        // ---- softmax and epilogue: a thread per row ----
        const int h = (warp - 4) >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t my_lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t tS = tmem + h * 128 + my_lanes, tO = tmem + 256 + h * 128 + my_lanes;
        const int64_t pitch = static_cast<int64_t>(a.Hkv) * D;
        const int per_tile = kTile >> a.page_shift;
        const bool wide = (reinterpret_cast<uintptr_t>(a.O) & 31) == 0;
        uint32_t tile = 0, v_stage = 1, v_phase = 0, o_done = 0;
        bool ok = true;
        for (uint32_t seg = 0;; ++seg) {
            const Work& s = *next_work<C>(a, roles, seg, ok);
            if (!kTwo) {
                if (named_any(kJoinBarrier, 256, !ok)) break;
            } else if (!ok) {
                break;
            }
            if (s.valid == 0) break;
            const int p_begin = s.p_begin, p_end = s.p_end, new_tile = s.new_tile, keys = s.keys;
            const int my_row = (kTwo ? h * 128 : 0) + row;                  // of the CTA's rows
            const bool exists = my_row < s.n_rows;
            const int32_t* list = a.table + static_cast<int64_t>(s.slot) * a.max_pages;
            const auto has_page = [&](int t) { return lane < per_tile && t < p_end && ((t * per_tile + lane) << a.page_shift) < keys; };
            const auto page_of = [&](int t) { return has_page(t) ? list[t * per_tile + lane] : 0; };
            constexpr int kStep = kTwo ? 1 : 2;
            const int t_first = kTwo ? p_begin : p_begin + static_cast<int>((h ^ tile) & 1u);      // this stream's first tile
            int id = page_of(t_first);
            float m = -INFINITY, l0 = 0.f, l1 = 0.f;       // the maximum in use, and the sum
            bool any_tile = false, had_fresh = false;
            uint64_t sees = 0ull;
            for (int t = p_begin; t < p_end; ++t, ++tile) {
                if (kTwo || t >= t_first && ((t - t_first) & 1) == 0) {
                    const int next = page_of(t + kStep);                    // (looked at a tile later)
                    const bool fresh = t == new_tile;
                    __syncwarp();
                    ok = __all_sync(0xffffffffu, ok && mbar_wait_a(bar(C::bSFull + h), (kTwo ? tile : tile >> 1) & 1, abort_flag, a.status));
                    // ---- which of the tile's keys the row sees: a bit each ----
                    uint32_t see[4] = {~0u, ~0u, ~0u, ~0u};
                    bool plain = true, is_key = true;
                    const uint32_t bad = __ballot_sync(0xffffffffu, has_page(t) && (id < 0 || id >= a.n_pages));
                    if (fresh || bad != 0u || keys - t * kTile < kTile) {
                        plain = false;
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            see[c] = low_bits(keys - t * kTile - 32 * c);
                            for (int k = 0; k < 32; k += 16)                // (pages are 16 rows or more)
                                if ((bad >> ((32 * c + k) >> a.page_shift)) & 1u) see[c] &= ~(0xffffu << k);
                        }
                    }
                    if (!plain && (!kTwo || h == 0)) is_key = ((row < 32 ? see[0] : row < 64 ? see[1] : row < 96 ? see[2] : see[3]) >> (row & 31)) & 1u;
                    if (fresh) {
                        ok = __all_sync(0xffffffffu, ok && mbar_wait_a(bar(C::bSees + static_cast<int>(seg % kQueue)), (seg / kQueue) & 1, abort_flag, a.status));
                        sees = exists ? s_sees[(seg % kQueue) * kMaxTree + ((s.row0 + my_row) >> a.g_shift)] : 0ull;
                        // its nodes from new_at on: 64 bits moved up by a multiple of 16
                        const int up = s.new_at & 31, word = s.new_at >> 5;
                        const uint32_t lo = static_cast<uint32_t>(sees), hi = static_cast<uint32_t>(sees >> 32);
                        const uint32_t b[3] = {lo << up, __funnelshift_l(lo, hi, up), up == 0 ? 0u : hi >> (32 - up)};
#pragma unroll
                        for (int c = 0; c < 4; ++c)
#pragma unroll
                            for (int k = 0; k < 3; ++k)
                                if (c == word + k) see[c] |= b[k];
                        had_fresh = true;
                    }
                    tc_fence_after();
                    float x[kTile];
                    {
                        uint32_t r[kTile];
                        __syncwarp();
                        PULSAR_TMEM_LD32_AT(tS, r, 0);
                        PULSAR_TMEM_LD32_AT(tS + 32, r, 32);
                        PULSAR_TMEM_LD32_AT(tS + 64, r, 64);
                        PULSAR_TMEM_LD32_AT(tS + 96, r, 96);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < kTile; ++i) x[i] = __uint_as_float(r[i]);
                    }
                    if (!plain) {
#pragma unroll
                        for (int i = 0; i < kTile; ++i)
                            if (((see[i / 32] >> (i % 32)) & 1u) == 0u) x[i] = -INFINITY;
                    }
                    float sum0, sum1;
                    // P of keys [from, from + 32 n): stored, and added to the two sums.
                    const auto form = [&](int from, int n, float neg) {
#pragma unroll
                        for (int c = from / 32; c < from / 32 + n; ++c) {
                            uint32_t p[16];
#pragma unroll
                            for (int i = 0; i < 32; i += 2) {
                                float y0, y1;
                                scaled2(y0, y1, x[c * 32 + i], x[c * 32 + i + 1], a.scale_log2, neg);
                                const float p0 = ex2(y0), p1 = ex2(y1);
                                add2(sum0, sum1, p0, p1);
                                p[i / 2] = pack_bf16x2(p0, p1);
                            }
                            tmem_st16(tS + c * 16, p);
                        }
                    };
                    // Behind the first tile the first piece is formed with the maximum in use at once: its sum, needed anyway, bounds its
                    // probabilities (a single one may reach 96 * 2^8), and the other logits are compared.  Where that fails the maximum is
                    // taken over the tile and the piece is formed again.
                    const bool ahead = any_tile && plain;
                    bool again = true;
                    sum0 = sum1 = 0.f;
                    if (ahead) {
                        form(0, kFirst / 32, -m);
                        float most = -INFINITY;
#pragma unroll
                        for (int i = kFirst; i < kTile; i += 2) most = max3(most, x[i], x[i + 1]);
                        again = __any_sync(0xffffffffu, !(sum0 + sum1 <= kFirst * 256.f) || m == -INFINITY || !(most * a.scale_log2 <= m + kRescale));
                    }
                    if (again) {
                        float most = -INFINITY, most2 = -INFINITY;
#pragma unroll
                        for (int i = 0; i < kTile; i += 4) {
                            most = max3(most, x[i], x[i + 1]);
                            most2 = max3(most2, x[i + 2], x[i + 3]);
                        }
                        most = fmaxf(most, most2) * a.scale_log2;
                        const float m_new = fmaxf(m, most), alpha = m_new == -INFINITY ? 1.f : ex2(m - m_new);
                        m = m_new;
                        l0 *= alpha;
                        l1 *= alpha;
                        if (any_tile) {
#pragma unroll 1
                            for (int c = 0; c < D; c += 16) {
                                uint32_t o[16];
                                __syncwarp();
                                tmem_ld16(tO + c, o);
                                tmem_wait_ld();
#pragma unroll
                                for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                                tmem_st16(tO + c, o);
                            }
                        }
                        tmem_wait_st();                                      // (two stores to the same columns have no order of their own)
                        sum0 = sum1 = 0.f;
                        form(0, kFirst / 32, m == -INFINITY ? 0.f : -m);
                    }
                    if (!plain && (!kTwo || h == 0)) {
                        // Rows of V that do not exist become zeros, and so does a node's value that is not finite (0 * NaN is NaN): see
                        // paged_tiles.cu.  Thread `row` has key `row` here.
                        ok = __all_sync(0xffffffffu, ok && mbar_wait_a(bar(C::bKvFull + static_cast<int>(v_stage)), v_phase, abort_flag, a.status));
                        const int node = fresh ? row - s.new_at : -1;
                        const bool is_node = node >= 0 && node < s.n;
                        const bool odd = is_node && ((s_odd[2 * (seg % kQueue) + (node >> 5)] >> (node & 31)) & 1u) != 0u;
                        if ((odd || (!is_key && !is_node)) && row < 16 * used_steps(t, keys, new_tile, s.new_at + s.n)) {
                            uint8_t* value = smem + v_stage * C::kTileBytes + row * 128;
#pragma unroll
                            for (int v = 0; v < D / 8; ++v)
                                *reinterpret_cast<uint4*>(value + (v >> 3) * kPanelBytes + (((v ^ row) & 7) << 4)) = make_uint4(0u, 0u, 0u, 0u);
                        }
                        fence_proxy_async_smem();
                    }
                    __syncwarp();
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) arrive_a(bar(C::bPFull + h));
                    form(kFirst, (kTile - kFirst) / 32, m == -INFINITY ? 0.f : -m);
                    l0 += sum0;
                    l1 += sum1;
                    __syncwarp();
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) arrive_a(bar(C::bPRest + h));
                    any_tile = true;
                    id = next;
                }
                v_stage += 2;
                if (v_stage >= C::kStages) {
                    v_stage -= C::kStages;
                    v_phase ^= 1;
                }
            }

            // ---- outputs ----
            const bool whole = s.part < 0;
            const int64_t out_row = whole ? row_of(s.token0, s.head0, s.row0, my_row, a.g_shift, a.Hq) : static_cast<int64_t>(s.part) * C::kRows + my_row;
            float* to_lse = whole ? a.LSE : a.part_LSE;
            if (any_tile) {
                __syncwarp();
                ok = __all_sync(0xffffffffu, ok && mbar_wait_a(bar(C::bOFull + h), o_done & 1, abort_flag, a.status));
                ++o_done;
            }
            tc_fence_after();
            float l = l0 + l1, factor;
            uint64_t odd = 0ull;
            if (had_fresh) odd = (s_odd[2 * (seg % kQueue)] | static_cast<uint64_t>(s_odd[2 * (seg % kQueue) + 1]) << 32) & sees;
            const float neg = m == -INFINITY ? 0.f : -m;
            // kJoinCols outputs of this stream from column c on, before they are divided by the sum.
            const auto outputs = [&](int c, float (&o)[kJoinCols]) {
                uint32_t r[16];
                __syncwarp();
                tmem_ld16(tO + c, r);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 16; ++i) o[i] = __uint_as_float(r[i]);
                for (uint64_t left = odd; left != 0ull; left &= left - 1ull) {          // (rare: the weight is formed again)
                    const int64_t node = (static_cast<int64_t>(s.slot) * a.T + (__ffsll(static_cast<long long>(left)) - 1)) * pitch + s.kvh * D;
                    const uint16_t* q = a.Q + row_of(s.token0, s.head0, s.row0, my_row, a.g_shift, a.Hq) * D;
                    float dot = 0.f;
                    for (int j = 0; j < D; ++j)
                        dot = fmaf(__uint_as_float(static_cast<uint32_t>(q[j]) << 16), __uint_as_float(static_cast<uint32_t>(a.Knew[node + j]) << 16), dot);
                    const float w = ex2(fmaf(dot, a.scale_log2, neg));
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[i] = fmaf(w, __uint_as_float(static_cast<uint32_t>(a.Vnew[node + c + i]) << 16), o[i]);
                }
            };
            const auto store = [&](int c, const float (&o)[kJoinCols]) {
                if (!exists) return;
                if (!whole) {                                               // [D, rows]: 32 rows write together
                    float* to = a.part_O + static_cast<int64_t>(s.part) * C::kRows * D + c * C::kRows + my_row;
#pragma unroll
                    for (int i = 0; i < 16; ++i) to[i * C::kRows] = o[i];
                } else if (a.out_f32) {
                    float* to = static_cast<float*>(a.O) + out_row * D + c;
#pragma unroll
                    for (int i = 0; i < 16; i += 4) *reinterpret_cast<float4*>(to + i) = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                } else {
                    uint16_t* to = static_cast<uint16_t*>(a.O) + out_row * D + c;
                    uint32_t v[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = pack_bf16x2(o[2 * i], o[2 * i + 1]);
                    store_32b(to, v, wide);
                }
            };
            if (kTwo) {
                if (!ok) break;
                factor = l == 0.f ? 0.f : 1.f / l;
#pragma unroll 1
                for (int c = 0; c < D; c += kJoinCols) {
                    float o[kJoinCols];
                    outputs(c, o);
#pragma unroll
                    for (int i = 0; i < kJoinCols; ++i) o[i] *= factor;
                    store(c, o);
                }
            } else {
                float* join = reinterpret_cast<float*>(smem + C::kJoin);            // [2][128][kJoinPitch]: for each stream, from the other
                float2* ml = reinterpret_cast<float2*>(join + 2 * 128 * kJoinPitch);  // [2][128]
                ml[h * 128 + row] = make_float2(m, l);
                if (named_any(kJoinBarrier, 256, !ok)) break;
                const float2 other = ml[(h ^ 1) * 128 + row];
                const float M = fmaxf(m, other.x), f = weight(m, M);
                l = f * l + weight(other.x, M) * other.y;
                factor = l == 0.f ? 0.f : f / l;
                m = M;
                float* give = join + ((h ^ 1) * 128 + row) * kJoinPitch;
                const float* take = join + (h * 128 + row) * kJoinPitch;
#pragma unroll 1
                for (int c = 0; c < D; c += 2 * kJoinCols) {
                    const int mine = c + h * kJoinCols, others = c + (h ^ 1) * kJoinCols;
                    float o[kJoinCols] = {}, o2[kJoinCols] = {};
                    if (any_tile) {
                        outputs(others, o2);
                        outputs(mine, o);
                    }
#pragma unroll
                    for (int i = 0; i < kJoinCols; ++i) give[i] = o2[i] * factor;
                    named_sync(kJoinBarrier, 256);
#pragma unroll
                    for (int i = 0; i < kJoinCols; ++i) o[i] = fmaf(o[i], factor, take[i]);
                    store(mine, o);
                    named_sync(kJoinBarrier, 256);
                }
            }
            if (exists && (kTwo || h == 0) && to_lse != nullptr)
                to_lse[out_row] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (any_tile) arrive_a(bar(C::bOEmpty + h));
                arrive_a(bar(C::bWorkEmpty + static_cast<int>(seg % kQueue)));
            }
        }
    }

    tc_fence_before();
    __syncthreads();
    if (*abort_flag != 0) {                                // copies that are still under way land before the memory is given back
        const uint64_t t0 = globaltimer_ns();
        while (globaltimer_ns() - t0 < 5000000ull) {
        }
        __syncthreads();
    }
    if (warp == 1) tmem_dealloc(tmem, 512);
}

template <int D, bool kTwo>
int32_t launch(const PagedArgs& a, const Maps& map, int rows, cudaStream_t stream) {
    using C = Wide<D, kTwo>;
    const unsigned ctas = static_cast<unsigned>(sm_count());
    const int blocks = (rows + C::kRows - 1) / C::kRows;
    PULSAR_CUDA_OK(cudaFuncSetAttribute(tree_wide_kernel<D, kTwo>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem));
    PULSAR_CUDA_OK(launch_kernel(tree_wide_kernel<D, kTwo>, dim3(ctas), dim3(kThreads), C::kSmem, stream, true, a, map, blocks));
    count_launch();
    return launch_parts_merge(a, static_cast<int64_t>(a.n_slots) * a.items_max * blocks, C::kRows, D, stream);
}

}  // namespace

int32_t launch_tree_wide(const PagedArgs& a, const Maps& map, int rows, int d, cudaStream_t stream) {
    if (d == 128) return rows > 128 ? launch<128, true>(a, map, rows, stream) : launch<128, false>(a, map, rows, stream);
    return rows > 128 ? launch<64, true>(a, map, rows, stream) : launch<64, false>(a, map, rows, stream);
}

}  // namespace pulsar
