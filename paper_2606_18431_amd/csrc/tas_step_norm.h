// tas_step_norm.h - the end of a head's norm, which the appends share (device code).
#pragma once
#include <hip/hip_runtime.h>

namespace tas_step_impl {
namespace {

// y <- y f w of a lane's 16 elements, with f = 1 / sqrt(mean + eps). Heads and weights of
// bfloat16 can be of opposite sizes that take f w out of the range of 32 bits (to 0, or to an
// infinity that makes NaN of a y of 0) though the result is in it. So f's power of two goes to y,
// which is 2 sqrt(head size) at most then, and its mantissa, from 1/2 to 1, to w: the roundings
// are those of y (f w). A float16 has not the exponents for that.
template <typename T, typename V>
__device__ __forceinline__ void weighted(float (&y0)[8], float (&y1)[8], float f, const V &w0,
                                         const V &w1) {
    float power = 1;
    if constexpr (!__is_same(T, _Float16)) {
        power = __builtin_amdgcn_ldexpf(1.0f, __builtin_amdgcn_frexp_expf(f));
        f = __builtin_amdgcn_frexp_mantf(f);
    }
#pragma unroll
    for (int e = 0; e < 8; e++) {
        y0[e] = y0[e] * power * (f * (float)w0[e]);
        y1[e] = y1[e] * power * (f * (float)w1[e]);
    }
}

}  // namespace
}  // namespace tas_step_impl
