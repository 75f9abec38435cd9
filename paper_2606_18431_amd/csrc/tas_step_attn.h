// tas_step_attn.h - what the attention kernels of a step have in common: matrix products,
// the softmax's helpers, partial results and their joins (device code).
#pragma once
#include <hip/hip_runtime.h>

#include "tas_step_internal.h"
#include "tas_step_matrix.h"

namespace tas_step_impl {
namespace {

typedef float f16x __attribute__((ext_vector_type(16)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef short s8 __attribute__((ext_vector_type(8)));
typedef uint64_t u64x2 __attribute__((ext_vector_type(2)));

// Block numbers: constant while a kernel runs, read by scalar loads.
typedef const __attribute__((address_space(4))) int *Table;

__device__ f16x mfma32(vec8<__bf16> a, vec8<__bf16> b, f16x c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ f16x mfma32(vec8<_Float16> a, vec8<_Float16> b, f16x c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// The m of a row is this far below its maximum, so that its weights are that much larger:
// a 16-bit float holds none below 2^-25, and would lose from the row, but not from its
// sum, what many small ones add (8000 keys at 2^-25.5 of the largest: 1.7e-4 of V). With
// 2^7 the largest is at most 2^15, and 2^20 keys below the smallest add 2^-12 at most,
// less than the result's rounding. A bfloat16 has the exponents of 32 bits.
template <typename T>
constexpr float kHeadroom = __is_same(T, _Float16) ? 7.0f : 0.0f;

// m is raised only where it falls behind by 8 more (a weight is then at most 2^8 of what
// it would be): the rescaling of o, as long as it is, is rare.
template <typename T>
constexpr float kRaise = kHeadroom<T> + 8.0f;

__device__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// Maximum and sum over the lanes that hold one column: lane ^ 32, and lane ^ 16.
__device__ float max32(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}
__device__ float max16(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}
__device__ float sum32(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}
__device__ float sum16(float x) {
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}

__device__ s4 read_tr(const char *p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4 *)p);
}

// Partial results. Those that a workgroup of the same launch joins cross dies, whose
// caches do not see each other's writes: they are written through to where the whole
// device reads them, and read from there (DEVICE). That costs their few bytes a trip to
// memory; a release fence would cost every workgroup a write-back of its die's cache
// (decode of 64 requests, 32/8 heads of 128: 181 us with fences, 79 us so). Those that
// the merge kernel joins are ordinary ones.
__device__ void put_part(float *to, float x, bool device) {
    if (device)
        __hip_atomic_store(to, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    else
        *to = x;
}
__device__ void put_part(float *to, f4 x, bool device) {
    if (device) {
        const u64x2 u = __builtin_bit_cast(u64x2, x);
        __hip_atomic_store((uint64_t *)to, u[0], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store((uint64_t *)to + 1, u[1], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    } else {
        *(f4 *)to = x;
    }
}
template <bool DEVICE>
__device__ float get_part(const float *from) {
    if (!DEVICE) return *from;
    return __hip_atomic_load(from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <bool DEVICE>
__device__ f4 get_part4(const float *from) {
    if (!DEVICE) return *(const f4 *)from;
    u64x2 u;
    u[0] = __hip_atomic_load((const uint64_t *)from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    u[1] = __hip_atomic_load((const uint64_t *)from + 1, __ATOMIC_RELAXED,
                             __HIP_MEMORY_SCOPE_AGENT);
    return __builtin_bit_cast(f4, u);
}

// Where elements d .. d + 3 of a row lie among the partial results of a key head's piece.
// Stores should fill whole lines: a wide item's lanes hold rows, so the fours of all its
// rows are adjacent; a thin segment's few rows are whole.
template <int D>
__device__ int64_t part_at(int seg_rows, int64_t first_row, int row, int d) {
    if (seg_rows <= kThinRows) return (first_row + row) * D + d;
    const int tile = row & ~(kWideRows - 1);
    return (first_row + tile) * D + d * min(kWideRows, seg_rows - tile) + (row - tile) * 4;
}
__device__ float lse2(float l, float m) {
    return l > 0 ? m + log2f(l) : (l == l ? -INFINITY : l);  // NaN stays
}
__device__ float reciprocal(float l) { return l > 0 ? 1.0f / l : (l == l ? 0.0f : l); }
constexpr float kLn2 = 0.6931471805599453f;

// Elements d .. d + 7 of row r of an item, in the output.
template <typename T, int D>
__device__ void store_row(const AttnArgs &a, const Seg &s, const Item &it, int r, int d,
                          const float *o, float l, float m) {
    const float f = reciprocal(l);
    const int row = it.row0 + r, j = row / a.group, head = it.hk * a.group + row - j * a.group;
    vec8<T> x;
#pragma unroll
    for (int e = 0; e < 8; e++) x[e] = (T)(o[e] * f);
    const int64_t tok = s.t0 + j;
    *(vec8<T> *)((T *)a.out + tok * a.out_stride + (int64_t)head * D + d) = x;
    if (d == 0 && a.lse) a.lse[tok * a.heads + head] = lse2(l, m) * kLn2;
}

// Keys that some of an item's rows see and others do not: a weight of 0 does not take
// out a value of V that is not finite, so such values are zeroed there and the key is
// marked; a row that sees a marked key becomes NaN.
template <typename T>
__device__ uint32_t not_finite(uint32_t x) {  // bits 15 and 31: of the two values
    constexpr uint32_t E = sizeof(T) == 2 && __is_same(T, _Float16) ? 0x7c00u : 0x7f80u;
    constexpr uint32_t ONE = E & (0u - E);
    return ((x & (E | E << 16)) + (ONE | ONE << 16)) & 0x80008000u;
}
template <typename T>
__device__ bool any_not_finite(u4 x) {
    return (not_finite<T>(x[0]) | not_finite<T>(x[1]) | not_finite<T>(x[2]) |
            not_finite<T>(x[3])) != 0;
}
template <typename T>
__device__ u4 zero_not_finite(u4 x) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const uint32_t b = not_finite<T>(x[i]);
        x[i] &= ~((b >> 15 & 0x10001u) * 0xffffu);
    }
    return x;
}

__device__ uint32_t first_bits(int n) { return n >= 32 ? ~0u : n > 0 ? (1u << n) - 1 : 0; }

// 16 bytes that are read once: they need not stay in the caches (decode of 256 requests,
// 448k tokens of 8 heads of 128: 282 us, with ordinary loads 311).
__device__ u4 stream(const char *p) { return __builtin_nontemporal_load((const u4 *)p); }

constexpr int kMarks = 8;  // words of 32 keys

// The end of a thin item: the four waves' results are joined (each wave's sums through its
// own LDS) and go to the output or to the partial results.
template <typename T, int D>
__device__ __forceinline__ void thin_end(const AttnArgs &a, const Item &it, float l, float m,
                                         const f4 (&o)[D / 16], char *lds01, char *lds23,
                                         float (*stat)[kThinRows][2]) {
    constexpr int VB = kThinKeys * D * 2;  // bytes of a wave's LDS
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int col = lane & 15, g = lane >> 4;
    const Seg &s = it.s;
    auto mine = [&](int w) { return (w < 2 ? lds01 : lds23) + (w & 1) * VB; };
    char *vl = mine(wave);
    // Join the four waves' results.
    l = sum32(sum16(l));
    __syncthreads();
    if (g == 0) stat[wave][col][0] = m, stat[wave][col][1] = l;
    // [row][D], groups of 4 floats swizzled by the row
#pragma unroll
    for (int i = 0; i < D / 16; i++)
        *(f4 *)((float *)vl + col * D + (((i * 4 + g) ^ col) * 4)) = o[i];
    __syncthreads();
    if (it.part >= 0) {
        for (int i = tid; i < s.rows * (D / 4); i += 256) {
            const int r = i / (D / 4), d4 = i % (D / 4);
            float mm = -INFINITY, ll = 0;
            f4 y = {0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < 4; w++) mm = fmaxf(mm, stat[w][r][0]);
            const float mu = mm == -INFINITY ? 0.0f : mm;
#pragma unroll
            for (int w = 0; w < 4; w++) {
                const float f = exp2_(stat[w][r][0] - mu);
                ll += stat[w][r][1] * f;
                y += *(const f4 *)((const float *)mine(w) + r * D + (d4 ^ r) * 4) * f;
            }
            put_part(a.part_o + part_at<D>(s.rows, it.part, r, d4 * 4), y * reciprocal(ll),
                     it.unit >= 0);
            if (d4 == 0) put_part(a.part_lse + it.part + r, lse2(ll, mm), it.unit >= 0);
        }
        return;
    }
    const int r = tid / (D / 8), d = tid % (D / 8) * 8;
    if (r >= s.rows) return;  // (at most 16 rows)
    float mm = -INFINITY, ll = 0, y[8] = {};
#pragma unroll
    for (int w = 0; w < 4; w++) mm = fmaxf(mm, stat[w][r][0]);
    const float mu = mm == -INFINITY ? 0.0f : mm;
#pragma unroll
    for (int w = 0; w < 4; w++) {
        const float f = exp2_(stat[w][r][0] - mu);
        ll += stat[w][r][1] * f;
        const float *from = (const float *)mine(w) + r * D;
        const f4 lo = *(const f4 *)(from + ((d / 4) ^ r) * 4);
        const f4 hi = *(const f4 *)(from + ((d / 4 + 1) ^ r) * 4);
#pragma unroll
        for (int e = 0; e < 4; e++) y[e] += lo[e] * f, y[4 + e] += hi[e] * f;
    }
    store_row<T, D>(a, s, it, r, d, y, ll, mm);
}

// The end of a wide item: its rows go to the output or to the partial results.
template <typename T, int D>
__device__ __forceinline__ void wide_end(const AttnArgs &a, const Item &it, float l, float m,
                                         const f16x (&o)[D / 32]) {
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, half = lane >> 5;
    const Seg &s = it.s;
    const int r = wave * 32 + col;  // row of the item
    l = sum32(l);
    // A lane holds d = 32 i + 8 e + 4 half + 0..3 of its row.
    if (it.part >= 0) {
        if (it.row0 + r >= s.rows) return;
        const float f = reciprocal(l);
        const int64_t first = it.part - it.row0;
#pragma unroll
        for (int i = 0; i < D / 32; i++)
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const f4 x = {o[i][e * 4], o[i][e * 4 + 1], o[i][e * 4 + 2], o[i][e * 4 + 3]};
                put_part(a.part_o + part_at<D>(s.rows, first, it.row0 + r, i * 32 + e * 8 + half * 4),
                         x * f, false);
            }
        if (half == 0) put_part(a.part_lse + it.part + r, lse2(l, m), false);
        return;
    }
    // The halves exchange so that each has 8 adjacent ones.
#pragma unroll
    for (int i = 0; i < D / 32; i++)
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
            float y[8];
#pragma unroll
            for (int c = 0; c < 4; c++) {
                const float ue = o[i][e * 4 + c], we = o[i][e * 4 + 4 + c];
                const uint32_t u = __builtin_bit_cast(uint32_t, ue);
                const uint32_t w = __builtin_bit_cast(uint32_t, we);
                // half 0: {own e, other's e}; half 1: {other's e + 1, own e + 1}
                auto x = __builtin_amdgcn_permlane32_swap(u, w, false, false);
                y[c] = __builtin_bit_cast(float, (uint32_t)x[0]);
                y[4 + c] = __builtin_bit_cast(float, (uint32_t)x[1]);
            }
            if (it.row0 + r < s.rows) store_row<T, D>(a, s, it, r, i * 32 + e * 8 + half * 8, y, l, m);
        }
}

// Joins the partial results of a unit's rows, weights 2^(lse_n - max), in a fixed order
// whoever is last. D / 8 threads to a row, adjacent threads to adjacent rows. What it
// takes is the latency of the loads, so those of eight parts are under way at once, and
// where a unit has fewer than 16 rows, the threads of the others take parts too.
template <typename T, int D, bool DEVICE>
__device__ __forceinline__ void join(const AttnArgs &a, const Unit &u) {
    constexpr int P = 8;
    const int d = threadIdx.x / kJoinRows * 8;
    if (d >= D) return;  // whole waves
    int width = kJoinRows;  // lanes of one set of the rows
    while (width / 2 >= u.rows) width /= 2;
    const int r = threadIdx.x % width, set = threadIdx.x % kJoinRows / width;
    const Seg &us = u.s;
    const int row = u.row0 + min(r, u.rows - 1), j = row / a.group, g = row - j * a.group;
    const int tok = us.t0 + j, head = u.hk * a.group + g;
    Own own{};
    if (u.prefix) own = a.tok_own[tok];
    const int n0 = us.nsplit, all = n0 + own.nsplit;
    const int64_t first0 = us.part + (int64_t)u.hk * us.nsplit * us.rows;
    const int64_t first1 = own.part + (int64_t)u.hk * own.nsplit * own.rows;
    const int own_row = (tok - own.t0) * a.group + g;
    float m = -INFINITY, sum = 0, y[8] = {};
    bool bad = false;  // a NaN among the parts stays
    for (int n = set * P; n < all; n += kJoinRows / width * P) {
        float lse[P];
        f4 o[P][2];
#pragma unroll
        for (int i = 0; i < P; i++) {
            const int k = min(n + i, all - 1);
            const bool mine = k < n0;
            const int rows = mine ? us.rows : own.rows;
            const int64_t first = mine ? first0 + (int64_t)k * rows
                                       : first1 + (int64_t)(k - n0) * rows;
            const int at = mine ? row : own_row;
            lse[i] = get_part<DEVICE>(a.part_lse + first + at);
#pragma unroll
            for (int e = 0; e < 2; e++)
                o[i][e] = get_part4<DEVICE>(a.part_o + part_at<D>(rows, first, at, d + e * 4));
        }
        float mn = m;
#pragma unroll
        for (int i = 0; i < P; i++) {
            bad |= lse[i] != lse[i];
            mn = fmaxf(mn, lse[i]);
        }
        const float mu = mn == -INFINITY ? 0.0f : mn, f = exp2_(m - mu);
        m = mn;
        sum *= f;
#pragma unroll
        for (int e = 0; e < 8; e++) y[e] *= f;
#pragma unroll
        for (int i = 0; i < P; i++) {
            const float w = n + i < all ? exp2_(lse[i] - mu) : 0.0f;
            sum += w;
#pragma unroll
            for (int e = 0; e < 8; e++) y[e] += o[i][e >> 2][e & 3] * w;
        }
    }
    for (int w = width; w < kJoinRows; w *= 2) {
        const float om = __shfl_xor(m, w), mn = fmaxf(m, om);
        const float mu = mn == -INFINITY ? 0.0f : mn;
        const float f = exp2_(m - mu), of = exp2_(om - mu);
        m = mn;
        sum = sum * f + __shfl_xor(sum, w) * of;
#pragma unroll
        for (int e = 0; e < 8; e++) y[e] = y[e] * f + __shfl_xor(y[e], w) * of;
        bad |= __shfl_xor((int)bad, w) != 0;
    }
    if (set || r >= u.rows) return;
    const float f = sum > 0 ? 1.0f / sum : 0.0f;
    vec8<T> x;
#pragma unroll
    for (int e = 0; e < 8; e++) x[e] = (T)(bad ? NAN : y[e] * f);
    *(vec8<T> *)((T *)a.out + (int64_t)tok * a.out_stride + (int64_t)head * D + d) = x;
    if (d == 0 && a.lse)
        a.lse[(int64_t)tok * a.heads + head] =
            bad ? NAN : lse2(sum, m) * kLn2;
}

// A thin item whose partial results have reached the device is counted for its unit, and
// the workgroup that counts the last one joins the unit; the count is left at zero for
// the next launch. (The rows of wide segments are left to the merge kernel: the workgroup that
// came last would join 128 rows one after another. Decode of 64 requests with a shared
// prefix of 2048, 32/8 heads of 128: 71 us so, 23.5 us with the merge kernel.)
template <typename T, int D>
__device__ __forceinline__ void count_item(const AttnArgs &a, const Item &it, int *last) {
    // this wave's results have arrived; then the others' have
    __builtin_amdgcn_s_waitcnt(kWaitLoads);
    __syncthreads();
    const Unit u = a.units[it.unit];
    if (threadIdx.x == 0) {
        uint32_t *done = a.done + it.unit;
        const uint32_t before =
            __hip_atomic_fetch_add(done, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *last = before == (uint32_t)u.items - 1;
        if (*last) __hip_atomic_store(done, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (*last) join<T, D, true>(a, u);
}

}  // namespace
}  // namespace tas_step_impl
