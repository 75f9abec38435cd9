// tas_fp4_pack.hip - tensors to four bits and back, and the layout of weights.
//
// All three move data: a thread has eight elements (16 bytes in 16 bits, 4 in four), so
// that the wider side's accesses are whole lines; a block is four adjacent threads. Each
// is bound by the bytes. (Pack of 16384 x 4096 in bf16 34 us, 5.1 TB/s, and of 65536 x 8192 263 us,
// 5.2 TB/s; values of a pool of 16 MB 16 us, 4.6 TB/s. The layout of 6144 x 4096 weights, 13 MB,
// 10 us, and of 32768 x 16384 153 us, 3.7 TB/s: a lane reads four words of a row, 16 bytes apart,
// and is left so, since it runs once for a matrix.)
#include <hip/hip_runtime.h>

#include "tas_fp4_convert.h"
#include "tas_fp4_internal.h"

namespace tas_step_impl {
namespace {

__device__ char *row_at(const tas_rows &r, uint32_t row, uint32_t n1, uint32_t n2) {
    const uint32_t i2 = row % n2, i01 = row / n2, i1 = i01 % n1, i0 = i01 / n1;
    return (char *)r.p + i0 * r.stride[0] + i1 * r.stride[1] + i2 * r.stride[2];
}

template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(Tensor4Args a) {
    const uint32_t u = blockIdx.x * 256 + threadIdx.x;
    if (u >= a.units) return;  // whole blocks
    const uint32_t row = u / a.per_row, c = u - row * a.per_row;
    const vec8<T> v = *(const vec8<T> *)(row_at(a.x, row, a.n1, a.n2) + c * 16ull);
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; e++) x[e] = (float)v[e];
    uint32_t most = largest(x);
    most = max(most, __shfl_xor(most, 1));
    most = max(most, __shfl_xor(most, 2));
    const uint32_t byte = scale_byte<T>(most);
    *(uint32_t *)(row_at(a.codes, row, a.n1, a.n2) + c * 4ull) = codes_of(x, byte);
    if (c % 4 == 0) *(uint8_t *)(row_at(a.scales, row, a.n1, a.n2) + c / 4) = (uint8_t)byte;
}

template <typename T>
__global__ __launch_bounds__(256) void values_kernel(Values4Args both) {
    const Tensor4Args &a = both.t[blockIdx.y];
    const uint32_t u = blockIdx.x * 256 + threadIdx.x;
    if (u >= a.units) return;
    const uint32_t row = u / a.per_row, c = u - row * a.per_row;
    const uint32_t codes = *(const uint32_t *)(row_at(a.codes, row, a.n1, a.n2) + c * 4ull);
    const uint32_t byte = *(const uint8_t *)(row_at(a.scales, row, a.n1, a.n2) + c / 4);
    *(vec8<T> *)(row_at(a.x, row, a.n1, a.n2) + c * 16ull) = values_of<T>(codes, scale_of(byte));
}

// A thread's 16 bytes of codes are those of one lane and tile, its byte of scale that of a
// row and block of it.
__global__ __launch_bounds__(256) void weights_kernel(Weights4Args a) {
    const int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t tile = u >> 6, tn = tile / a.w.tiles_k, tk = tile - tn * a.w.tiles_k;
    if (tn >= a.w.tiles_n) return;
    const int lane = u & 63, r = lane & 15, g = lane >> 4;
    const int64_t row = tn * kTileRows + r;
    u4 codes = {0, 0, 0, 0};
    uint8_t scale = 0;
    if (row < a.rows) {
#pragma unroll
        for (int j = 0; j < 4; j++)
            if (tk * 4 + j < a.blocks)
                codes[j] = *(const uint32_t *)(a.codes + row * a.codes_stride +
                                               (tk * 4 + j) * 16 + g * 4);
        if (tk * 4 + g < a.blocks) scale = a.scales[row * a.scales_stride + tk * 4 + g];
    }
    *(u4 *)(a.out + tile * 1024 + lane * 16) = codes;
    a.out[a.w.scales_at + tile * 64 + r * 4 + g] = (char)scale;
}

}  // namespace

hipError_t launch_pack4(const Tensor4Args &a, int dtype, hipStream_t s) {
    const int64_t n = ((int64_t)a.units + 255) / 256;
    return launch_kernel(dtype == TAS_F16 ? pack_kernel<_Float16> : pack_kernel<__bf16>, n, a, s);
}
hipError_t launch_values4(const Values4Args &a, int n, int dtype, hipStream_t s) {
    Values4Args copy = a;
    void *args[] = {&copy};
    return hipLaunchKernel(dtype == TAS_F16 ? (const void *)values_kernel<_Float16>
                                            : (const void *)values_kernel<__bf16>,
                           dim3((uint32_t)(((int64_t)a.t[0].units + 255) / 256), n), dim3(256),
                           args, 0, s);
}
hipError_t launch_weights4(const Weights4Args &a, hipStream_t s) {
    return launch_kernel(weights_kernel, (a.w.tiles_n * a.w.tiles_k + 3) / 4, a, s);
}

}  // namespace tas_step_impl
