// tas_fp4_linear.hip - products of a step's tokens with weights in four bits.
//
// y[t][n] = sum over k of x[t][k] W[n][k], with W's values exact in the 16-bit type (a
// conversion of two elements an instruction), sums in 32 bits, rounded once. The transposed
// product Y^T = W X^T leaves four adjacent n of a token in a lane. The left operand is a
// tile of W as it lies in memory, one load of adjacent 16 bytes a lane: lane 16 g + r has
// block g of row r, so that the k-slots of its four products stand for the elements
// 32 g + 8 i + 0..7, in x too.
//
// Few tokens: bound by the weights' bytes. A workgroup has all of K for some rows, its
// eight waves take every eighth unit of 512 columns, and their sums are joined in LDS, in
// one order: no partial results in memory, no second launch.
#include <hip/hip_runtime.h>

#include "tas_fp4_convert.h"
#include "tas_fp4_internal.h"

namespace tas_step_impl {
namespace {

typedef float f4 __attribute__((ext_vector_type(4)));

__device__ f4 mfma16(vec8<__bf16> a, vec8<__bf16> b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ f4 mfma16(vec8<_Float16> a, vec8<_Float16> b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

constexpr int kWaves = 8;

// Four adjacent n of token t.
template <typename T>
__device__ void store_four(const Linear4Args &a, int64_t t, int n, f4 x) {
    typedef T four __attribute__((ext_vector_type(4)));
    if (n >= a.rows) return;
    T *y = (T *)a.y + t * a.y_stride + n;
    if (a.y_fours) {
        *(four *)y = four{(T)x[0], (T)x[1], (T)x[2], (T)x[3]};
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++)
            if (n + i < a.rows) y[i] = (T)x[i];
    }
}

// 16 RT rows, 16 TT tokens.
template <typename T, int RT, int TT>
__global__ __launch_bounds__(64 * kWaves) void stream_kernel(Linear4Args a) {
    using V = vec8<T>;
    __shared__ f4 part[kWaves][RT * TT][64];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    const uint32_t groups_n = (a.tiles_n + RT - 1) / RT, at_t = blockIdx.x / groups_n;
    const int tile0 = (blockIdx.x - at_t * groups_n) * RT, t0 = at_t * 16 * TT;
    const char *codes[RT], *scales[RT];
#pragma unroll
    for (int i = 0; i < RT; i++) {  // (of tiles that there are not, the last one's)
        const int64_t tile = min(tile0 + i, a.tiles_n - 1);
        codes[i] = a.codes + tile * a.tiles_k * 1024 + lane * 16;
        scales[i] = a.scales + tile * a.units_k * 256 + lane * 4;
    }
    const T *x[TT];
#pragma unroll
    for (int i = 0; i < TT; i++)
        x[i] = (const T *)a.x + (int64_t)min(t0 + i * 16 + col, a.tokens - 1) * a.x_stride + g * 32;
    f4 sum[RT][TT];
#pragma unroll
    for (int i = 0; i < RT; i++)
#pragma unroll
        for (int j = 0; j < TT; j++) sum[i][j] = f4{0, 0, 0, 0};
    for (int u = wave; u < a.units_k; u += kWaves) {
        uint32_t sc[RT];
#pragma unroll
        for (int i = 0; i < RT; i++) sc[i] = *(const uint32_t *)(scales[i] + u * 256);
#pragma unroll
        for (int n = 0; n < 4; n++) {
            const int tk = u * 4 + n;
            if (tk >= a.tiles_k) break;
            u4 c[RT];
#pragma unroll
            for (int i = 0; i < RT; i++)
                c[i] = __builtin_nontemporal_load((const u4 *)(codes[i] + tk * 1024ll));
            // blocks beyond the matrix are zeros: so is x there, whatever lies behind its rows
            const bool in = tk * 4 + g < a.blocks;
            V b[TT][4];
#pragma unroll
            for (int j = 0; j < TT; j++)
#pragma unroll
                for (int k = 0; k < 4; k++)
                    b[j][k] = in ? *(const V *)(x[j] + tk * kTileCols + k * 8) : V{};
#pragma unroll
            for (int i = 0; i < RT; i++) {
                const float s = scale_of(sc[i] >> (8 * n) & 255);
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    const V w = values_of<T>(c[i][k], s);
#pragma unroll
                    for (int j = 0; j < TT; j++) sum[i][j] = mfma16(w, b[j][k], sum[i][j]);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < RT; i++)
#pragma unroll
        for (int j = 0; j < TT; j++) part[wave][i * TT + j][lane] = sum[i][j];
    __syncthreads();
    for (int i = wave; i < RT * TT; i += kWaves) {
        f4 y = part[0][i][lane];
#pragma unroll
        for (int w = 1; w < kWaves; w++) y += part[w][i][lane];
        const int t = t0 + i % TT * 16 + col;
        if (t < a.tokens) store_four<T>(a, t, (tile0 + i / TT) * 16 + g * 4, y);
    }
}

template <typename T, int RT, int TT>
hipError_t launch_stream(const Linear4Args &a, hipStream_t s) {
    Linear4Args copy = a;
    void *args[] = {&copy};
    const dim3 grid((uint32_t)((a.tiles_n + RT - 1) / RT) * ((a.tokens + 16 * TT - 1) / (16 * TT)));
    return hipLaunchKernel((const void *)stream_kernel<T, RT, TT>, grid, dim3(64 * kWaves), args,
                           0, s);
}
template <typename T, int TT>
hipError_t launch_rows(const Linear4Args &a, hipStream_t s) {
    if (a.tiles_n >= 1024) return launch_stream<T, 4, TT>(a, s);
    if (a.tiles_n >= 512) return launch_stream<T, 2, TT>(a, s);
    return launch_stream<T, 1, TT>(a, s);
}
template <typename T>
hipError_t launch(const Linear4Args &a, hipStream_t s) {
    if (a.tokens <= 16) return launch_rows<T, 1>(a, s);
    if (a.tokens <= 32) return launch_rows<T, 2>(a, s);
    return launch_rows<T, 4>(a, s);
}

}  // namespace

hipError_t launch_linear4(const Linear4Args &a, int dtype, hipStream_t s) {
    return dtype == TAS_F16 ? launch<_Float16>(a, s) : launch<__bf16>(a, s);
}

}  // namespace tas_step_impl
