// Tensor maps for the tiled bulk copies (attn.cu).
#pragma once

#include <cuda.h>
#include <stdint.h>

namespace pulsar {

// [rows, heads, d] bf16 viewed as (d, heads, rows); box = (64, box_heads, box_rows), 128-byte swizzle.
bool make_map_3d(CUtensorMap* m, const void* base, int64_t rows, int heads, int d, int box_heads, int box_rows);

}  // namespace pulsar
