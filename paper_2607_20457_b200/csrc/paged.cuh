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

#ifdef __CUDACC__
// A slot's length within its table; what is outside is reported once (by the thread for which `tell` is set) and clamped.
__device__ __forceinline__ int checked_len(int len, int64_t capacity, bool tell, int32_t* status) {
    if (len >= 0 && len <= capacity) return len;
    if (tell) report(status, PULSAR_DEV_BAD_LENGTH);
    return len < 0 ? 0 : static_cast<int>(capacity);
}
#endif

}  // namespace pulsar
