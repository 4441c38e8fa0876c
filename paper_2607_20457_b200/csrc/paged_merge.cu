// Behind an attention launch: writes the new tokens' rows to their pages, and joins the parts of the items that several of its CTAs
// share: O = sum_j e^{l_j - l} A_j (Appendix H's closed form), in the order of the keys, whatever order the CTAs ran in.
//
// What bounds it is latency: reads of l, then of the outputs, from L2, so many of them are under way at once.  (One row of a warp after
// the other, 128 rows of nine parts of eight items took 8 us; a CTA for each row of each CTA's possible item 4.3 us to find that
// nothing is to be joined.)
#include <algorithm>
#include <type_traits>

#include "paged.cuh"

namespace pulsar {

namespace {

constexpr int kWarps = 8;
constexpr int kUnder = 8;                        // parts of a row under way
constexpr int kTogether = 2;                     // rows of a warp

// The new tokens' rows to their pages: copied here, by CTAs of their own, because the attention's warps have better things to do (a
// warp of its own took 16 us for 64 rows) and nobody reads those rows before the next call.
template <int D>
__device__ __forceinline__ void append_rows(const PagedArgs& a) {
    constexpr int kVecs = D / 8;
    const uint32_t row_vecs = static_cast<uint32_t>(a.Hkv * kVecs), step = gridDim.x * 32 * kWarps;
    const uint64_t all = static_cast<uint64_t>(a.n_slots) * a.T * row_vecs;
    for (uint64_t i = blockIdx.x * (32 * kWarps) + threadIdx.x; i < all; i += step) {
        const uint32_t token = static_cast<uint32_t>(i / row_vecs), v = static_cast<uint32_t>(i - static_cast<uint64_t>(token) * row_vecs);
        const int slot = static_cast<int>(token / a.T), t = static_cast<int>(token - slot * a.T);
        const uint4 k = reinterpret_cast<const uint4*>(a.Knew)[i], x = reinterpret_cast<const uint4*>(a.Vnew)[i];
        if (a.n_draft != nullptr && t >= a.n_draft[slot]) continue;
        const int len = checked_len(a.len[slot], static_cast<int64_t>(a.max_pages) << a.page_shift, false, nullptr);
        const int64_t to = new_row_at(a, slot, static_cast<int64_t>(len) + t, static_cast<int64_t>(a.Hkv) * D);
        if (to < 0) continue;
        reinterpret_cast<uint4*>(a.K + to)[v] = k;
        reinterpret_cast<uint4*>(a.V + to)[v] = x;
    }
}

// Parts as [rows, D] (paged_tiles.cu): a warp takes kTogether rows side by side, with the parts' l in its lanes (32 parts at a time) and kUnder
// parts' outputs of every row under way.
template <int D>
__global__ void __launch_bounds__(32 * kWarps)
paged_merge_kernel(const __grid_constant__ PagedArgs a, int n, int64_t items) {
    constexpr int kPer = D / 32;                 // consecutive outputs of a lane
    using Vec = typename std::conditional<kPer == 4, float4, float2>::type;
    const float *part_O = a.part_O, *part_LSE = a.part_LSE;
    grid_dependency_wait();
    grid_launch_dependents();
    if (blockIdx.y == 0) {
        append_rows<D>(a);
        return;
    }
    const int lane = threadIdx.x & 31, r0 = ((blockIdx.y - 1) * kWarps + (threadIdx.x >> 5)) * kTogether;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const Meta x = a.meta[item];
        if (x.parts < 2 || r0 >= x.rows) continue;
        const auto place_of = [&](int j) { return static_cast<int64_t>(j == 0 ? x.first : 2 * (x.cta + j * x.step)) * n + r0; };
        float m[kTogether], total[kTogether], acc[kTogether][kPer];
#pragma unroll
        for (int r = 0; r < kTogether; ++r) {
            m[r] = -INFINITY;
            total[r] = 0.f;
#pragma unroll
            for (int i = 0; i < kPer; ++i) acc[r][i] = 0.f;
        }
        for (int j0 = 0; j0 < x.parts; j0 += 32) {
            const int count = min(32, x.parts - j0);
            float w[kTogether];
#pragma unroll
            for (int r = 0; r < kTogether; ++r) w[r] = lane < count && r0 + r < x.rows ? part_LSE[place_of(j0 + lane) + r] : -INFINITY;
#pragma unroll
            for (int r = 0; r < kTogether; ++r) {
                const float l = w[r];
                float most = l;
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
                const float m_new = fmaxf(m[r], most), neg = m_new == -INFINITY ? 0.f : -m_new;      // (no key so far: weights of 0, and a NaN still shows)
                const float alpha = ex2((m[r] + neg) * 1.4426950408889634f);                          // 0 from -infinity
                m[r] = m_new;
                total[r] *= alpha;
#pragma unroll
                for (int i = 0; i < kPer; ++i) acc[r][i] *= alpha;
                w[r] = ex2((l + neg) * 1.4426950408889634f);
            }
#pragma unroll 1
            for (int j = 0; j < count; j += kUnder) {
                Vec v[kUnder][kTogether];
#pragma unroll
                for (int u = 0; u < kUnder; ++u) {
                    const Vec* src = reinterpret_cast<const Vec*>(part_O + place_of(j0 + min(j + u, count - 1)) * D) + lane;
#pragma unroll
                    for (int r = 0; r < kTogether; ++r)
                        if (j + u < count && r0 + r < x.rows) v[u][r] = src[r * 32];
                }
#pragma unroll
                for (int u = 0; u < kUnder; ++u) {
                    if (j + u >= count) break;
#pragma unroll
                    for (int r = 0; r < kTogether; ++r) {
                        const float wj = __shfl_sync(0xffffffffu, w[r], j + u);
                        total[r] += wj;
                        if (r0 + r >= x.rows) continue;
                        const float* y = reinterpret_cast<const float*>(&v[u][r]);
#pragma unroll
                        for (int i = 0; i < kPer; ++i) acc[r][i] = fmaf(wj, y[i], acc[r][i]);
                    }
                }
            }
        }
#pragma unroll
        for (int r = 0; r < kTogether; ++r) {
            if (r0 + r >= x.rows) break;
            const float inv = total[r] == 0.f ? 0.f : 1.f / total[r];
            const int64_t row = row_of(x.token0, x.head0, x.row0, r0 + r, a.g_shift, a.Hq);
            if (a.out_f32) {
#pragma unroll
                for (int i = 0; i < kPer; ++i) static_cast<float*>(a.O)[row * D + lane * kPer + i] = acc[r][i] * inv;
            } else {
#pragma unroll
                for (int i = 0; i < kPer; i += 2)
                    reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.O) + row * D + lane * kPer)[i / 2] = pack_bf16x2(acc[r][i] * inv, acc[r][i + 1] * inv);
            }
            if (lane == 0 && a.LSE != nullptr) a.LSE[row] = total[r] == 0.f ? -INFINITY : m[r] + logf(total[r]);
        }
    }
}

// Parts as [D, n] (paged_wide.cu: its threads have a row each, and 32 rows write an output together).  A CTA takes 32 rows, a lane each,
// and kSlice outputs; its warps share the parts and are joined like these.
constexpr int kSlice = 16;
template <int D>
__global__ void __launch_bounds__(32 * kWarps)
paged_merge_wide_kernel(const __grid_constant__ PagedArgs a, int n, int64_t items) {
    constexpr int kSlices = D / kSlice, kPitch = kSlice + 1;
    __shared__ float s_o[kWarps][32 * kPitch];
    __shared__ float2 s_ml[kWarps][32];
    grid_dependency_wait();
    grid_launch_dependents();
    if (blockIdx.y == 0) {
        append_rows<D>(a);
        return;
    }
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r0 = (blockIdx.y - 1) / kSlices * 32, r = r0 + lane;
    const int c0 = (blockIdx.y - 1) % kSlices * kSlice;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const Meta x = a.meta[item];
        if (x.parts < 2 || r0 >= x.rows) continue;
        float m = -INFINITY, total = 0.f, acc[kSlice] = {};
        for (int j = warp; j < x.parts; j += kWarps) {
            const int64_t at = static_cast<int64_t>(j == 0 ? x.first : 2 * (x.cta + j * x.step)) * n;
            const float l = a.part_LSE[at + r];
            const float* src = a.part_O + at * D + static_cast<int64_t>(c0) * n + r;
            float v[kSlice];
#pragma unroll
            for (int i = 0; i < kSlice; ++i) v[i] = src[i * n];
            const float m_new = fmaxf(m, l), neg = m_new == -INFINITY ? 0.f : -m_new;
            const float alpha = ex2((m + neg) * 1.4426950408889634f), w = ex2((l + neg) * 1.4426950408889634f);
            m = m_new;
            total = fmaf(total, alpha, w);
#pragma unroll
            for (int i = 0; i < kSlice; ++i) acc[i] = fmaf(acc[i], alpha, w * v[i]);
        }
        s_ml[warp][lane] = make_float2(m, total);
#pragma unroll
        for (int i = 0; i < kSlice; ++i) s_o[warp][lane * kPitch + i] = acc[i];
        __syncthreads();
        // two outputs of a row per thread
        const int row = threadIdx.x / (kSlice / 2), c = threadIdx.x % (kSlice / 2) * 2;
        float M = -INFINITY, sum = 0.f, y0 = 0.f, y1 = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) M = fmaxf(M, s_ml[w][row].x);
        const float neg = M == -INFINITY ? 0.f : -M;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float2 ml = s_ml[w][row];
            const float f = ex2((ml.x + neg) * 1.4426950408889634f);
            sum = fmaf(f, ml.y, sum);
            y0 = fmaf(f, s_o[w][row * kPitch + c], y0);
            y1 = fmaf(f, s_o[w][row * kPitch + c + 1], y1);
        }
        if (r0 + row < x.rows) {
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            const int64_t to = row_of(x.token0, x.head0, x.row0, r0 + row, a.g_shift, a.Hq);
            if (a.out_f32) *reinterpret_cast<float2*>(static_cast<float*>(a.O) + to * D + c0 + c) = make_float2(y0 * inv, y1 * inv);
            else *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.O) + to * D + c0 + c) = pack_bf16x2(y0 * inv, y1 * inv);
            if (c0 == 0 && c == 0 && a.LSE != nullptr) a.LSE[to] = sum == 0.f ? -INFINITY : M + logf(sum);
        }
        __syncthreads();
    }
}

}  // namespace

int32_t launch_parts_merge(const PagedArgs& a, int64_t items, int rows, int d, cudaStream_t stream) {
    // CTAs with y = 0 append; the others have an item each, as far as the chip has room for them at once.
    const unsigned x = static_cast<unsigned>(std::min<int64_t>(items, 2 * sm_count()));
    if (rows > 64) {
        PULSAR_CUDA_OK(launch_kernel(d == 128 ? paged_merge_wide_kernel<128> : paged_merge_wide_kernel<64>, dim3(x, 1 + rows / 32 * (d / kSlice)),
                                     dim3(32 * kWarps), 0, stream, true, a, rows, items));
    } else {
        PULSAR_CUDA_OK(launch_kernel(d == 128 ? paged_merge_kernel<128> : paged_merge_kernel<64>, dim3(x, 1 + (rows + kTogether * kWarps - 1) / (kTogether * kWarps)),
                                     dim3(32 * kWarps), 0, stream, true, a, rows, items));
    }
    count_launch();
    return PULSAR_OK;
}

}  // namespace pulsar
