// tas_fp4_append.hip - norm, rotation and append of a step's new tokens to a cache in four
// bits.
//
// For every head u of a token (queries and keys):
//     u <- u / sqrt(mean(u^2) + eps) * weight
//     (a, b) <- (a cos x - b sin x, b cos x + a sin x)    x: the position's angles
// Queries in 32 bits, rounded once. Keys and values are rounded to four bits by blocks of
// 32. A key that lies within a rounding error of the border of two codes would get either,
// by the order of the norm's sum, and an error of half a step: such keys are worked out again
// in 64 bits. In 32 bits a key is off by 13 roundings of |a cos x| + |b sin x| at most: a term
// of the norm's sum passes 10 in its lane and 3 over the lanes, eps is one more, the root
// halves them to 7 and is one itself, as the division, two products and the rotation's two.
// With two for the comparison that is less than 2^-20; 2^-19 is taken. Where so much moves a
// code or a block's scale (of some hundredths of the waves), or the range of 32 bits does not
// do, the wave's keys take the long way; what 32 bits lose below their smallest normal number is
// in the bound, as it may come back by a weight or an angle. Nothing else is read twice and
// nothing in between is written, so the bound is the copy of the queries and the reading of the
// rest, and the vector work is next to it. (13321 tokens of 32/8 heads of 128: with all keys in 64
// bits 76 us; 65 to 66 so, 4.5 TB/s, where a large copy has 5.1. A flag and a choice for each element
// of the norm took 6 us more.)
//
// A head is D / 16 lanes with two chunks of eight elements each, chosen so that a lane
// holds both members of its rotated pairs: chunks i and i + R / 16 of the halves (R / 8
// chunks are rotated), or 2 i and 2 i + 1 of interleaved pairs. Either way lane i needs the
// angles 8 i .. 8 i + 7. A block's four chunks may lie in up to four lanes, in either place:
// their largest magnitudes meet in LDS, within the wave.
#include <hip/hip_runtime.h>

#include "tas_fp4_convert.h"
#include "tas_fp4_internal.h"
#include "tas_step_norm.h"

namespace tas_step_impl {
namespace {

// A lane's part of a head.
struct Part {
    int c0, c1;   // its chunks
    int i;        // the lane of the head
    bool turned;  // whether they are rotated
    int pos;      // of the token
};

// Chunks c0 and c1 (x0, x1) of a head: normed, with weights, and rotated; and how far the
// results may be off.
template <int D, typename T>
__device__ __forceinline__ float norm_and_turn(const AppendArgs &a, const void *weight,
                                               const Part &p, const vec8<T> &x0,
                                               const vec8<T> &x1, float (&y0)[8], float (&y1)[8]) {
    using V = vec8<T>;
    // Where nothing overflows, roundings are relative ones, but for what is lost below the
    // smallest normal number: 2^-150 of an element before its weight (and of that, times an
    // element), and of each product of the rotation.
    bool in_range = true;
    float lost = 0;
#pragma unroll
    for (int e = 0; e < 8; e++) y0[e] = (float)x0[e], y1[e] = (float)x1[e];
    if (weight) {
        float sum = 0;
#pragma unroll
        for (int e = 0; e < 8; e++) sum += y0[e] * y0[e] + y1[e] * y1[e];
        for (int m = 1; m < D / 16; m *= 2) sum += __shfl_xor(sum, m);
        const float mean = sum / D + a.eps, f = 1.0f / sqrtf(mean);
        in_range = mean > 0x1p-100f && mean < 0x1p120f;
        const V w0 = *(const V *)((const T *)weight + p.c0 * 8);
        const V w1 = *(const V *)((const T *)weight + p.c1 * 8);
        weighted<T>(y0, y1, f, w0, w1);
        float most_w = 0;
#pragma unroll
        for (int e = 0; e < 8; e++)
            most_w = fmaxf(most_w, fmaxf(fabsf((float)w0[e]), fabsf((float)w1[e])));
        in_range &= most_w < 0x1p120f;
        lost = most_w * 0x1p-148f + 0x1p-143f;
    }
    float most = 0, most_turn = 1;
    if (p.turned) {
        const int64_t at = (int64_t)p.pos * (a.rot / 2) + p.i * 8;
        float c[8], s[8];
        *(f4 *)c = *(const f4 *)(a.cos + at), *(f4 *)(c + 4) = *(const f4 *)(a.cos + at + 4);
        *(f4 *)s = *(const f4 *)(a.sin + at), *(f4 *)(s + 4) = *(const f4 *)(a.sin + at + 4);
#pragma unroll
        for (int e = 0; e < 8; e++)
            most_turn = fmaxf(most_turn, fmaxf(fabsf(c[e]), fabsf(s[e])));
        auto turn = [&](float &x, float &y, float c, float s) {
            const float u = x, v = y;
            most = fmaxf(most, fmaxf(fabsf(u * c) + fabsf(v * s), fabsf(v * c) + fabsf(u * s)));
            x = u * c - v * s;
            y = v * c + u * s;
        };
        if (a.interleaved) {
#pragma unroll
            for (int e = 0; e < 4; e++) {
                turn(y0[2 * e], y0[2 * e + 1], c[e], s[e]);
                turn(y1[2 * e], y1[2 * e + 1], c[4 + e], s[4 + e]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; e++) turn(y0[e], y1[e], c[e], s[e]);
        }
    } else if (weight) {
#pragma unroll
        for (int e = 0; e < 8; e++) most = fmaxf(most, fmaxf(fabsf(y0[e]), fabsf(y1[e])));
    }
    if (!weight && !p.turned) return 0;
    const float off = most * 0x1p-19f + (lost * most_turn + 0x1p-148f);
    return in_range && most < 0x1p120f && off < 0x1p120f ? off : INFINITY;
}

// The same in 64 bits, to floats on the same side of every border; `to`: 16 floats of the
// lane in LDS. (Element after element: of doubles, few are held at once.)
template <int D, typename T>
__device__ __forceinline__ void norm_and_turn_exact(const AppendArgs &a, const T *weight,
                                                    const Part &p, vec8<T> x0, vec8<T> x1,
                                                    float *to) {
    using V = vec8<T>;
    double f = 1;
    V w0, w1;
#pragma unroll
    for (int e = 0; e < 8; e++) w0[e] = w1[e] = (T)1.0f;
    if (weight) {
        w0 = *(const V *)(weight + p.c0 * 8);
        w1 = *(const V *)(weight + p.c1 * 8);
        double sum = 0;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const double u = (float)x0[e], v = (float)x1[e];
            sum += u * u + v * v;
            __builtin_amdgcn_sched_barrier(0);
        }
        for (int m = 1; m < D / 16; m *= 2) sum += __shfl_xor(sum, m);
        f = 1.0 / sqrt(sum / D + a.eps);
    }
    const float *cos = a.cos + (int64_t)p.pos * (a.rot / 2) + p.i * 8;
    const float *sin = a.sin + (int64_t)p.pos * (a.rot / 2) + p.i * 8;
    const bool halves = p.turned && !a.interleaved;
    // converted again below, not kept
    u4 k0 = __builtin_bit_cast(u4, x0), k1 = __builtin_bit_cast(u4, x1);
    asm volatile("" : "+v"(k0), "+v"(k1));
    x0 = __builtin_bit_cast(V, k0), x1 = __builtin_bit_cast(V, k1);
#pragma unroll
    for (int e = 0; e < 8; e++) {
        // a rotated pair, or two elements: (c0, e) and (c1, e), or the two of 16 from 2 e on
        const int pair = 2 * e % 8;
        const V &xp = e < 4 ? x0 : x1, &wp = e < 4 ? w0 : w1;
        const float ux = halves ? (float)x0[e] : (float)xp[pair];
        const float vx = halves ? (float)x1[e] : (float)xp[pair + 1];
        const float uw = halves ? (float)w0[e] : (float)wp[pair];
        const float vw = halves ? (float)w1[e] : (float)wp[pair + 1];
        const double u = ux * (f * uw), v = vx * (f * vw);
        double x = u, y = v;
        if (p.turned) {
            const double c = cos[e], s = sin[e];
            x = u * c - v * s;
            y = v * c + u * s;
        }
        to[halves ? e : 2 * e] = odd_float(x);
        to[halves ? 8 + e : 2 * e + 1] = odd_float(y);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// Whether two words of codes differ in more than the sign of zeros.
__device__ bool differ(uint32_t x, uint32_t y) {
    const uint32_t signs = 0x88888888u;
    const uint32_t not_zero = (((x | y) & ~signs) + ~signs) & signs;
    return ((x ^ y) & (not_zero | ~signs)) != 0;
}

template <typename T, int D>
__global__ __launch_bounds__(256) void append4_kernel(Append4Args a) {
    constexpr int LPH = D / 16, HPW = heads_of_wave(D);  // lanes of a head, heads of a wave
    using V = vec8<T>;
    // of a wave's heads: the chunks' largest magnitudes, at least and at most
    __shared__ __attribute__((aligned(16))) uint32_t least[4][HPW][D / 8], most[4][HPW][D / 8];
    __shared__ __attribute__((aligned(16))) float exact[4][64][16];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, i = lane % LPH;
    const uint32_t per_tok = (a.heads + 2 * a.kv_heads + HPW - 1) / HPW;
    const uint32_t unit = blockIdx.x * 4 + wave;
    const uint32_t tok = unit / per_tok;
    if (tok >= (uint32_t)a.n_tok) return;
    const int h = (unit - tok * per_tok) * HPW + lane / LPH;
    if (h >= a.heads + 2 * a.kv_heads) return;  // whole heads: all exchanges stay in one

    const int RL = a.rot / 16;
    Part p;
    p.i = i;
    p.turned = i < RL;
    p.c0 = 2 * i, p.c1 = 2 * i + 1;
    if (!a.interleaved && p.turned) p.c0 = i, p.c1 = i + RL;
    const T *src = (const T *)a.qkv + tok * a.qkv_stride + (int64_t)h * D;
    const V x0 = *(const V *)(src + p.c0 * 8), x1 = *(const V *)(src + p.c1 * 8);

    const Req &r = a.reqs[a.tok_req[tok]];
    const int j = (int)tok - r.t0, own = r.kv_len - r.n_new + j;
    p.pos = r.prefix_len + own;
    float y0[8], y1[8], off = 0;
    if (h < a.heads) {
        norm_and_turn<D, T>(a, a.q_weight, p, x0, x1, y0, y1);
        V z0, z1;
#pragma unroll
        for (int e = 0; e < 8; e++) z0[e] = (T)y0[e], z1[e] = (T)y1[e];
        T *to = (T *)a.q_out + tok * a.q_out_stride + (int64_t)h * D;
        *(V *)(to + p.c0 * 8) = z0;
        *(V *)(to + p.c1 * 8) = z1;
        return;
    }
    const int page = a.tables[r.table + (own >> a.blk_shift)];
    const int at = own & ((1 << a.blk_shift) - 1);
    const bool is_v = h >= a.heads + a.kv_heads;
    if (is_v)
#pragma unroll
        for (int e = 0; e < 8; e++) y0[e] = (float)x0[e], y1[e] = (float)x1[e];
    else
        off = norm_and_turn<D, T>(a, a.k_weight, p, x0, x1, y0, y1);

    uint32_t *lo = least[wave][lane / LPH], *hi = most[wave][lane / LPH];
    auto byte_of = [&](const uint32_t *from, int c) {
        const u4 m = *(const u4 *)(from + (c & ~3));
        return scale_byte<T>(max(max(m[0], m[1]), max(m[2], m[3])));
    };
    const float most0 = __builtin_bit_cast(float, largest(y0));
    const float most1 = __builtin_bit_cast(float, largest(y1));
    auto bits = [](float x) { return __builtin_bit_cast(uint32_t, x); };
    hi[p.c0] = bits(most0 + off);
    hi[p.c1] = bits(most1 + off);
    lo[p.c0] = bits(most0 < off ? 0.0f : most0 - off);
    lo[p.c1] = bits(most1 < off ? 0.0f : most1 - off);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    uint32_t b0 = byte_of(hi, p.c0), b1 = byte_of(hi, p.c1);
    uint32_t k0 = codes_of(y0, b0), k1 = codes_of(y1, b1);
    bool unsure = b0 != byte_of(lo, p.c0) || b1 != byte_of(lo, p.c1);
    if (off != 0) {
        float u0[8], u1[8], v0[8], v1[8];
#pragma unroll
        for (int e = 0; e < 8; e++) {
            u0[e] = y0[e] - off, u1[e] = y1[e] - off;
            v0[e] = y0[e] + off, v1[e] = y1[e] + off;
        }
        unsure |= differ(codes_of(u0, b0), codes_of(v0, b0)) ||
                  differ(codes_of(u1, b1), codes_of(v1, b1));
    }
    if (__any(unsure)) {
        if (!is_v) {
            float *to = exact[wave][lane];
            norm_and_turn_exact<D, T>(a, (const T *)a.k_weight, p, x0, x1, to);
#pragma unroll
            for (int e = 0; e < 8; e++) y0[e] = to[e], y1[e] = to[8 + e];
            hi[p.c0] = largest(y0);
            hi[p.c1] = largest(y1);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        b0 = byte_of(hi, p.c0), b1 = byte_of(hi, p.c1);
        k0 = codes_of(y0, b0), k1 = codes_of(y1, b1);
    }
    const tas_rows &codes = is_v ? a.f.v : a.f.k, &scales = is_v ? a.f.v_scale : a.f.k_scale;
    const int64_t hk = is_v ? h - a.heads - a.kv_heads : h - a.heads;
    char *to = (char *)codes.p + page * codes.stride[0] + hk * codes.stride[1] +
               at * codes.stride[2];
    *(uint32_t *)(to + p.c0 * 4) = k0;
    *(uint32_t *)(to + p.c1 * 4) = k1;
    uint8_t *st = (uint8_t *)scales.p + page * scales.stride[0] + hk * scales.stride[1] +
                  at * scales.stride[2];
    if (p.c0 % 4 == 0) st[p.c0 / 4] = (uint8_t)b0;
    if (p.c1 % 4 == 0) st[p.c1 / 4] = (uint8_t)b1;
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
