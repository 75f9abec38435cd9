// tas_step_matrix.h - what the kernels that work on the matrix unit have in common: vectors, the
// product of 16 by 16 by 32, loads to LDS and their waits (device code).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tas_step_impl {
namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

template <typename T>
using vec8 = T __attribute__((ext_vector_type(8)));
template <typename T>
using vec2 = T __attribute__((ext_vector_type(2)));

template <int N>
struct Const {
    static constexpr int value = N;
};

__device__ f4 mfma16(vec8<__bf16> a, vec8<__bf16> b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ f4 mfma16(vec8<_Float16> a, vec8<_Float16> b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

typedef const __attribute__((address_space(1))) char *Global;
__device__ void load_to_lds(Global from, char *to) {
    __builtin_amdgcn_global_load_lds(from, (__attribute__((address_space(3))) void *)to, 16, 0,
                                     0);
}
constexpr int kWaitLoads = 0x0F70;  // s_waitcnt: no load or store outstanding

}  // namespace
}  // namespace tas_step_impl
