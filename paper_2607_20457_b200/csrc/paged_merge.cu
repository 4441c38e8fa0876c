// Joins the parts of the items that several CTAs of an attention launch share: O = sum_j e^{l_j - l} A_j (Appendix H's closed form),
// in the order of the keys, whatever order the CTAs ran in.
//
// A warp takes a row: 32 parts' l at a time, one per lane, and eight parts' outputs under way.  What bounds it is latency: two
// dependent reads from L2 and as many more as there are eighths of the parts.
#include "paged.cuh"

namespace pulsar {

namespace {

constexpr int kWarps = 8;

template <int D>
__global__ void __launch_bounds__(32 * kWarps)
paged_merge_kernel(const Meta* __restrict__ meta, const float* __restrict__ part_O, const float* __restrict__ part_LSE, int n, int g_shift, int Hq,
                   void* O, int out_f32, float* LSE) {
    constexpr int kPer = D / 32;                 // consecutive outputs of a lane
    using Vec = typename std::conditional<kPer == 4, float4, float2>::type;
    grid_dependency_wait();
    grid_launch_dependents();
    const Meta x = meta[blockIdx.x];
    const int lane = threadIdx.x & 31;
    if (x.parts < 2) return;
    const auto place_of = [&](int j) { return static_cast<int64_t>(j == 0 ? x.first : 2 * (static_cast<int>(blockIdx.x) + j * x.step)) * n; };
    for (int r = blockIdx.y * kWarps + (threadIdx.x >> 5); r < x.rows; r += gridDim.y * kWarps) {
        float m = -INFINITY, total = 0.f, acc[kPer] = {};
        for (int j0 = 0; j0 < x.parts; j0 += 32) {
            const float l = j0 + lane < x.parts ? part_LSE[place_of(j0 + lane) + r] : -INFINITY;
            float most = l;
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
            const float m_new = fmaxf(m, most);
            if (m_new == -INFINITY) {                                        // no key so far (a NaN still shows)
                if (__any_sync(0xffffffffu, l != l)) total = acc[0] = nanf("");
                continue;
            }
            const float alpha = ex2((m - m_new) * 1.4426950408889634f);      // 0 from -inf
            m = m_new;
            total *= alpha;
#pragma unroll
            for (int i = 0; i < kPer; ++i) acc[i] *= alpha;
            const float w = ex2((l - m) * 1.4426950408889634f);
            const int count = min(32, x.parts - j0);
#pragma unroll 1
            for (int j = 0; j < count; j += 8) {
                Vec v[8];
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    if (j + u < count) v[u] = reinterpret_cast<const Vec*>(part_O + (place_of(j0 + j + u) + r) * D)[lane];
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    if (j + u >= count) break;
                    const float wj = __shfl_sync(0xffffffffu, w, j + u);
                    total += wj;
                    const float* y = reinterpret_cast<const float*>(&v[u]);
#pragma unroll
                    for (int i = 0; i < kPer; ++i) acc[i] = fmaf(wj, y[i], acc[i]);
                }
            }
        }
        const float inv = total == 0.f ? 0.f : 1.f / total;
        const int64_t row = row_of(x.token0, x.head0, x.row0, r, g_shift, Hq);
        if (out_f32) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) static_cast<float*>(O)[row * D + lane * kPer + i] = acc[i] * inv;
        } else {
#pragma unroll
            for (int i = 0; i < kPer; i += 2)
                reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(O) + row * D + lane * kPer)[i / 2] = pack_bf16x2(acc[i] * inv, acc[i + 1] * inv);
        }
        if (lane == 0 && LSE != nullptr) LSE[row] = total == 0.f ? -INFINITY : m + logf(total);
    }
}

}  // namespace

int32_t launch_parts_merge(const PagedArgs& a, unsigned ctas, int rows, int d, cudaStream_t stream) {
    const unsigned row_ctas = static_cast<unsigned>((rows + 4 * kWarps - 1) / (4 * kWarps));        // four rows of a warp at most
    PULSAR_CUDA_OK(launch_kernel(d == 128 ? paged_merge_kernel<128> : paged_merge_kernel<64>, dim3(ctas, row_ctas), dim3(32 * kWarps), 0, stream, true,
                                 a.meta, a.part_O, a.part_LSE, rows, a.g_shift, a.Hq, a.O, a.out_f32, a.LSE));
    count_launch();
    return PULSAR_OK;
}

}  // namespace pulsar
