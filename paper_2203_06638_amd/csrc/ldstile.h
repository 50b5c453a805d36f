// ldstile.h -- LDS layout of operand tiles that are read with the LDS transpose read.
#pragma once
#include <hip/hip_runtime.h>

namespace lpp {

// Where logical 16-byte chunk c (8 channels) of tile row `row` lies in a row of W
// chunks: XOR-swizzled in pairs by row, so that the 8 rows a half-wave's
// transposed reads touch (p .. p + 3 and p + 8 .. p + 11) hit all 64 banks once.
template <int W>
__device__ __forceinline__ int wg_chunk(int c, int row) {
    const int f = W >= 16 ? ((row & 3) | (((row >> 3) & 1) << 2)) : (((row >> 1) & 1) | (((row >> 3) & 1) << 1));
    return (((c >> 1) ^ f) << 1) | (c & 1);
}

}  // namespace lpp
