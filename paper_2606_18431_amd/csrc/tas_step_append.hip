// tas_step_append.hip - norm, rotation and append of a step's new tokens.
//
// For every head u of a token (queries and keys):
//     u <- u / sqrt(mean(u^2) + eps) * weight
//     (a, b) <- (a cos x - b sin x, b cos x + a sin x)    x: the position's angles
// in 32 bits, rounded once. Queries go to q_out, keys to their slot of the cache,
// values are copied there. Nothing is read twice and nothing in between is
// written, so the bound is the copy of the tensor.
//
// A head is D / 16 lanes with two 16-byte chunks each, chosen so that a lane holds
// both members of its rotated pairs: chunks i and i + R / 16 of the halves (R / 8
// chunks are rotated), or 2 i and 2 i + 1 of interleaved pairs. Either way lane i
// needs the angles 8 i .. 8 i + 7, and only the norm's sum crosses lanes.
#include <hip/hip_runtime.h>

#include "tas_step_internal.h"
#include "tas_step_norm.h"

namespace tas_step_impl {
namespace {

typedef float f4 __attribute__((ext_vector_type(4)));

template <typename T>
using vec8 = T __attribute__((ext_vector_type(8)));

template <typename T, int D>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a) {
    constexpr int LPH = D / 16, HPW = heads_of_wave(D);  // lanes of a head, heads of a wave
    using V = vec8<T>;
    const int lane = threadIdx.x & 63, i = lane % LPH;
    const uint32_t per_tok = (a.heads + 2 * a.kv_heads + HPW - 1) / HPW;
    const uint32_t unit = blockIdx.x * 4 + (threadIdx.x >> 6);
    const uint32_t tok = unit / per_tok;
    if (tok >= (uint32_t)a.n_tok) return;
    const int h = (unit - tok * per_tok) * HPW + lane / LPH;
    if (h >= a.heads + 2 * a.kv_heads) return;  // whole heads: the sum below stays in one

    const int RL = a.rot / 16;
    const bool turned = i < RL;
    int c0 = 2 * i, c1 = 2 * i + 1;
    if (!a.interleaved && turned) c0 = i, c1 = i + RL;
    const T *src = (const T *)a.qkv + tok * a.qkv_stride + (int64_t)h * D;
    V x0 = *(const V *)(src + c0 * 8), x1 = *(const V *)(src + c1 * 8);

    const Req &r = a.reqs[a.tok_req[tok]];
    const int j = (int)tok - r.t0, own = r.kv_len - r.n_new + j;
    const int page = a.tables[r.table + (own >> a.blk_shift)];
    const int at = own & ((1 << a.blk_shift) - 1);

    const bool is_q = h < a.heads, is_v = h >= a.heads + a.kv_heads;
    if (!is_v) {
        float y0[8], y1[8];
        for (int e = 0; e < 8; e++) y0[e] = (float)x0[e], y1[e] = (float)x1[e];
        if (a.q_weight) {
            float sum = 0;
            for (int e = 0; e < 8; e++) sum += y0[e] * y0[e] + y1[e] * y1[e];
            for (int m = 1; m < LPH; m *= 2) sum += __shfl_xor(sum, m);
            const float f = 1.0f / sqrtf(sum / D + a.eps);
            const T *w = (const T *)(is_q ? a.q_weight : a.k_weight);
            const V w0 = *(const V *)(w + c0 * 8), w1 = *(const V *)(w + c1 * 8);
            weighted<T>(y0, y1, f, w0, w1);
        }
        if (turned) {
            const int64_t p = (int64_t)(r.prefix_len + own) * (a.rot / 2) + i * 8;
            float c[8], s[8];
            *(f4 *)c = *(const f4 *)(a.cos + p), *(f4 *)(c + 4) = *(const f4 *)(a.cos + p + 4);
            *(f4 *)s = *(const f4 *)(a.sin + p), *(f4 *)(s + 4) = *(const f4 *)(a.sin + p + 4);
            if (a.interleaved) {
                for (int e = 0; e < 4; e++) {
                    const float u = y0[2 * e], v = y0[2 * e + 1];
                    y0[2 * e] = u * c[e] - v * s[e];
                    y0[2 * e + 1] = v * c[e] + u * s[e];
                    const float w = y1[2 * e], z = y1[2 * e + 1];
                    y1[2 * e] = w * c[4 + e] - z * s[4 + e];
                    y1[2 * e + 1] = z * c[4 + e] + w * s[4 + e];
                }
            } else {
                for (int e = 0; e < 8; e++) {
                    const float u = y0[e], v = y1[e];
                    y0[e] = u * c[e] - v * s[e];
                    y1[e] = v * c[e] + u * s[e];
                }
            }
        }
        for (int e = 0; e < 8; e++) x0[e] = (T)y0[e], x1[e] = (T)y1[e];
    }
    T *to;
    if (is_q)
        to = (T *)a.q_out + tok * a.q_out_stride + (int64_t)h * D;
    else if (is_v)
        to = (T *)a.c.v + page * a.c.v_block + (h - a.heads - a.kv_heads) * a.c.v_head +
             at * a.c.v_token;
    else
        to = (T *)a.c.k + page * a.c.k_block + (h - a.heads) * a.c.k_head + at * a.c.k_token;
    *(V *)(to + c0 * 8) = x0;
    *(V *)(to + c1 * 8) = x1;
}

template <typename T, int D>
hipError_t launch(const AppendArgs &a, hipStream_t s) {
    return launch_kernel(append_kernel<T, D>, append_groups(a.n_tok, a.heads, a.kv_heads, D), a,
                         s);
}

}  // namespace

hipError_t launch_append(const AppendArgs &a, int dtype, int head_dim, hipStream_t s) {
    if (dtype == TAS_F16)
        return head_dim == 64 ? launch<_Float16, 64>(a, s) : launch<_Float16, 128>(a, s);
    return head_dim == 64 ? launch<__bf16, 64>(a, s) : launch<__bf16, 128>(a, s);
}

}  // namespace tas_step_impl
