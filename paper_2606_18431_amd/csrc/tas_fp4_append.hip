// tas_fp4_append.hip - norm, rotation and append of a step's new tokens to a cache in four
// bits.
//
// For every head u of a token (queries and keys):
//     u <- u / sqrt(mean(u^2) + eps) * weight
//     (a, b) <- (a cos x - b sin x, b cos x + a sin x)    x: the position's angles
// Queries in 32 bits, rounded once. Keys and values are rounded to four bits by blocks of
// 32. A key that lies within a rounding error of the border of two codes would get either,
// by the order of the norm's sum, and an error of half a step; so keys are worked out in 64
// bits, which this chip computes at half the rate of 32. Nothing is read twice and nothing in
// between is written, so the bound is the copy of the queries and the reading of the rest.
//
// A head is D / 16 lanes with two chunks of eight elements each, chosen so that a lane
// holds both members of its rotated pairs: chunks i and i + R / 16 of the halves (R / 8
// chunks are rotated), or 2 i and 2 i + 1 of interleaved pairs. Either way lane i needs the
// angles 8 i .. 8 i + 7. A block's four chunks may lie in up to four lanes, in either place:
// their largest magnitudes meet in LDS, within the wave.
#include <hip/hip_runtime.h>

#include "tas_fp4_convert.h"
#include "tas_fp4_internal.h"

namespace tas_step_impl {
namespace {

typedef float f4 __attribute__((ext_vector_type(4)));

__device__ float root(float x) { return sqrtf(x); }
__device__ double root(double x) { return sqrt(x); }

// Chunks c0 and c1 (y0, y1) of a head whose chunks the D / 16 lanes i hold: normed, with
// weights, and rotated by the angles of position `pos`, if `turned`.
template <typename T, int D, typename F>
__device__ __forceinline__ void norm_and_turn(const AppendArgs &a, const void *weight, int c0,
                                              int c1, int i, bool turned, int pos, F (&y0)[8],
                                              F (&y1)[8]) {
    using V = vec8<T>;
    if (weight) {
        F sum = 0;
        for (int e = 0; e < 8; e++) sum += y0[e] * y0[e] + y1[e] * y1[e];
        for (int m = 1; m < D / 16; m *= 2) sum += __shfl_xor(sum, m);
        const F f = F(1) / root(sum / D + a.eps);
        const V w0 = *(const V *)((const T *)weight + c0 * 8);
        const V w1 = *(const V *)((const T *)weight + c1 * 8);
        for (int e = 0; e < 8; e++) y0[e] *= f * (F)w0[e], y1[e] *= f * (F)w1[e];
    }
    if (turned) {
        const int64_t p = (int64_t)pos * (a.rot / 2) + i * 8;
        float c[8], s[8];
        *(f4 *)c = *(const f4 *)(a.cos + p), *(f4 *)(c + 4) = *(const f4 *)(a.cos + p + 4);
        *(f4 *)s = *(const f4 *)(a.sin + p), *(f4 *)(s + 4) = *(const f4 *)(a.sin + p + 4);
        if (a.interleaved) {
            for (int e = 0; e < 4; e++) {
                const F u = y0[2 * e], v = y0[2 * e + 1];
                y0[2 * e] = u * c[e] - v * s[e];
                y0[2 * e + 1] = v * c[e] + u * s[e];
                const F w = y1[2 * e], z = y1[2 * e + 1];
                y1[2 * e] = w * c[4 + e] - z * s[4 + e];
                y1[2 * e + 1] = z * c[4 + e] + w * s[4 + e];
            }
        } else {
            for (int e = 0; e < 8; e++) {
                const F u = y0[e], v = y1[e];
                y0[e] = u * c[e] - v * s[e];
                y1[e] = v * c[e] + u * s[e];
            }
        }
    }
}

template <typename T, int D>
__global__ __launch_bounds__(256) void append4_kernel(Append4Args a) {
    constexpr int LPH = D / 16, HPW = heads_of_wave(D);  // lanes of a head, heads of a wave
    using V = vec8<T>;
    __shared__ __attribute__((aligned(16))) uint32_t most[4][HPW][D / 8];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, i = lane % LPH;
    const uint32_t per_tok = (a.heads + 2 * a.kv_heads + HPW - 1) / HPW;
    const uint32_t unit = blockIdx.x * 4 + wave;
    const uint32_t tok = unit / per_tok;
    if (tok >= (uint32_t)a.n_tok) return;
    const int h = (unit - tok * per_tok) * HPW + lane / LPH;
    if (h >= a.heads + 2 * a.kv_heads) return;  // whole heads: all exchanges stay in one

    const int RL = a.rot / 16;
    const bool turned = i < RL;
    int c0 = 2 * i, c1 = 2 * i + 1;
    if (!a.interleaved && turned) c0 = i, c1 = i + RL;
    const T *src = (const T *)a.qkv + tok * a.qkv_stride + (int64_t)h * D;
    const V x0 = *(const V *)(src + c0 * 8), x1 = *(const V *)(src + c1 * 8);

    const Req &r = a.reqs[a.tok_req[tok]];
    const int j = (int)tok - r.t0, own = r.kv_len - r.n_new + j;
    if (h < a.heads) {
        float y0[8], y1[8];
        for (int e = 0; e < 8; e++) y0[e] = (float)x0[e], y1[e] = (float)x1[e];
        norm_and_turn<T, D>(a, a.q_weight, c0, c1, i, turned, r.prefix_len + own, y0, y1);
        V z0, z1;
        for (int e = 0; e < 8; e++) z0[e] = (T)y0[e], z1[e] = (T)y1[e];
        T *to = (T *)a.q_out + tok * a.q_out_stride + (int64_t)h * D;
        *(V *)(to + c0 * 8) = z0;
        *(V *)(to + c1 * 8) = z1;
        return;
    }
    const int page = a.tables[r.table + (own >> a.blk_shift)];
    const int at = own & ((1 << a.blk_shift) - 1);
    const bool is_v = h >= a.heads + a.kv_heads;
    float y0[8], y1[8];
    if (is_v) {
        for (int e = 0; e < 8; e++) y0[e] = (float)x0[e], y1[e] = (float)x1[e];
    } else {
        double z0[8], z1[8];
        for (int e = 0; e < 8; e++) z0[e] = (double)(float)x0[e], z1[e] = (double)(float)x1[e];
        norm_and_turn<T, D>(a, a.k_weight, c0, c1, i, turned, r.prefix_len + own, z0, z1);
        for (int e = 0; e < 8; e++) y0[e] = odd_float(z0[e]), y1[e] = odd_float(z1[e]);
    }
    uint32_t *mine = most[wave][lane / LPH];
    mine[c0] = largest(y0);
    mine[c1] = largest(y1);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    auto byte_of = [&](int c) {
        const u4 m = *(const u4 *)(mine + (c & ~3));
        return scale_byte<T>(max(max(m[0], m[1]), max(m[2], m[3])));
    };
    const uint32_t b0 = byte_of(c0), b1 = byte_of(c1);
    const tas_rows &codes = is_v ? a.f.v : a.f.k, &scales = is_v ? a.f.v_scale : a.f.k_scale;
    const int64_t hk = is_v ? h - a.heads - a.kv_heads : h - a.heads;
    char *to = (char *)codes.p + page * codes.stride[0] + hk * codes.stride[1] +
               at * codes.stride[2];
    *(uint32_t *)(to + c0 * 4) = codes_of(y0, b0);
    *(uint32_t *)(to + c1 * 4) = codes_of(y1, b1);
    uint8_t *st = (uint8_t *)scales.p + page * scales.stride[0] + hk * scales.stride[1] +
                  at * scales.stride[2];
    if (c0 % 4 == 0) st[c0 / 4] = (uint8_t)b0;
    if (c1 % 4 == 0) st[c1 / 4] = (uint8_t)b1;
}

template <typename T, int D>
hipError_t launch(const Append4Args &a, hipStream_t s) {
    return launch_kernel(append4_kernel<T, D>, append_groups(a.n_tok, a.heads, a.kv_heads, D), a,
                         s);
}

}  // namespace

hipError_t launch_append4(const Append4Args &a, int dtype, int head_dim, hipStream_t s) {
    if (dtype == TAS_F16)
        return head_dim == 64 ? launch<_Float16, 64>(a, s) : launch<_Float16, 128>(a, s);
    return head_dim == 64 ? launch<__bf16, 64>(a, s) : launch<__bf16, 128>(a, s);
}

}  // namespace tas_step_impl
