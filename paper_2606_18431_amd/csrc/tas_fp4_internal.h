// tas_fp4_internal.h - arguments of the kernels that work in four bits, and their launchers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tas_fp4.h"
#include "tas_step_internal.h"

namespace tas_step_impl {

struct Append4Args : AppendArgs {  // (its cache is not used)
    tas_cache_fp4 f;
};
struct Attn4Args : AttnArgs {  // (its cache is not used)
    tas_cache_fp4 f;
};

// Units of eight elements of a tensor's rows, one a thread.
struct Tensor4Args {
    tas_rows x, codes, scales;
    uint32_t units, per_row, n1, n2;  // units in all and of a row; rows i0 n1 n2 + i1 n2 + i2
};

struct Values4Args {
    Tensor4Args t[2];  // of as many units
};

// Weights as the products read them: tiles of 16 rows and 128 columns, the tiles of a run
// of rows one after another, so that a tile is one load of adjacent 16 bytes a lane. Lane
// 16 g + r has the words g (elements 8 g .. 8 g + 7) of row r's four blocks: a product's 32
// k-slots are one block, and adjacent in x. A tile's scales are 64 bytes, byte 4 r + j that of
// row r, block j. Rows and blocks beyond the matrix are zeros.
constexpr int kTileRows = 16, kTileCols = 128;
struct WeightsShape {
    int64_t tiles_n, tiles_k;
    int64_t scales_at, bytes;  // byte offset of the scales; size
};
inline WeightsShape weights_shape(int64_t rows, int64_t cols) {
    WeightsShape w;
    w.tiles_n = (rows + kTileRows - 1) / kTileRows;
    w.tiles_k = (cols + kTileCols - 1) / kTileCols;
    w.scales_at = w.tiles_n * w.tiles_k * 1024;
    w.bytes = w.scales_at + w.tiles_n * w.tiles_k * 64;
    return w;
}
struct Weights4Args {
    const char *codes, *scales;
    char *out;
    int64_t codes_stride, scales_stride, rows, blocks;  // blocks of a row
    WeightsShape w;
};
struct Linear4Args {
    const void *x;
    const char *codes, *scales;
    void *y;
    int64_t x_stride, y_stride;
    int32_t tokens, rows, blocks;  // blocks of a row
    int32_t tiles_n, tiles_k;
    int32_t y_fours;  // y can be written four elements at once
    int32_t x_much;   // x has more than 16 times the weights' bytes
};

// Return hipSuccess or the launch's error.
hipError_t launch_append4(const Append4Args &a, int dtype, int head_dim, hipStream_t s);
hipError_t launch_attention4(const Attn4Args &a, int n_items, int n_merge, int dtype,
                             int head_dim, hipStream_t s);
hipError_t launch_pack4(const Tensor4Args &a, int dtype, hipStream_t s);
// (of one tensor or two)
hipError_t launch_values4(const Values4Args &a, int n, int dtype, hipStream_t s);
hipError_t launch_weights4(const Weights4Args &a, hipStream_t s);
hipError_t launch_linear4(const Linear4Args &a, int dtype, hipStream_t s);
// The number of the kernel that it takes, by the sizes alone.
int linear4_kernel(const Linear4Args &a);

}  // namespace tas_step_impl
