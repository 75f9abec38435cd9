// tas_step_attn.hip - attention of a step's new tokens over the paged cache.
//
// One pass over a row's keys with the running maximum m and sum l of the softmax:
//     m' = max(m, max s),  l <- l 2^(m-m') + sum 2^(s-m'),  o <- o 2^(m-m') + 2^(s-m') V
// with s = scale log2(e) q.k. Scores are computed transposed, S^T = K Q^T, so that
// the matrix unit leaves a query's scores in the lane that holds the query's column:
// the sums over keys stay in lanes, and the weights P^T are in place as the right
// operand of O^T = V^T P^T (which keys its k-slots stand for is free, as long as both
// operands agree). The left operand V^T is read from the rows of V in LDS by the
// transposing LDS read. Scores, statistics and sums are held in 32 bits; the weights
// are rounded to the inputs' type for the second product, as its operands have to be
// (kHeadroom: what a 16-bit float has left of its exponent).
#include <hip/hip_runtime.h>

#include "tas_step_internal.h"

namespace tas_step_impl {
namespace {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f16x __attribute__((ext_vector_type(16)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef short s8 __attribute__((ext_vector_type(8)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

template <typename T>
using vec8 = T __attribute__((ext_vector_type(8)));
template <typename T>
using vec2 = T __attribute__((ext_vector_type(2)));
typedef uint64_t u64x2 __attribute__((ext_vector_type(2)));

// Block numbers: constant while a kernel runs, read by scalar loads.
typedef const __attribute__((address_space(4))) int *Table;

__device__ f4 mfma16(vec8<__bf16> a, vec8<__bf16> b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ f4 mfma16(vec8<_Float16> a, vec8<_Float16> b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
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

// The place in LDS (in 16-byte chunks) of chunk c of a V row: the four rows that
// one transposing read takes lie in different quarters of the banks.
template <int D>
__device__ int v_chunk(int row, int c) {
    if (D == 128) return row * 16 + (c ^ (((row & 3) << 2) | ((row >> 1) & 2)));
    return row * 8 + (c ^ ((row & 3) << 1));
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

// Up to 16 rows against a run of keys: each of the four waves takes every fourth
// 32 keys, K straight into registers as the left operand, V through its own LDS;
// the waves' results are joined at the end. Memory bound: 16 rows make use of at
// most 16 products a byte and a half.
template <typename T, int D>
__device__ __forceinline__ void thin_item(const AttnArgs &a, const Item &it, char *lds01,
                                          char *lds23, float (*stat)[kThinRows][2]) {
    using V = vec8<T>;
    constexpr int QS = D / 32;          // steps of 32 over d
    constexpr int VL = D / 16;          // 16-byte loads of a lane for 32 rows of V
    constexpr int LPR = D / 8;          // lanes of a V row
    constexpr int VB = kThinKeys * D * 2;  // bytes of a wave's V
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int col = lane & 15, g = lane >> 4;
    const Seg &s = it.s;
    const Table tab = (Table)(a.tables + s.table);

    const int row = min(col, s.rows - 1), j = row / a.group;
    const int lim = min(min(s.kv_len, s.lim0 + j), it.k1);
    V q[QS];
    {
        const T *src = (const T *)a.q + (int64_t)(s.t0 + j) * a.q_stride +
                       (int64_t)(it.hk * a.group + row - j * a.group) * D + g * 8;
#pragma unroll
        for (int i = 0; i < QS; i++) q[i] = *(const V *)(src + i * 32);
    }
    const int full = min(min(s.kv_len, s.lim0), it.k1);  // keys that the first row sees
    const int sub_mask = (1 << a.sub_shift) - 1;
    const T *kbase = (const T *)a.c.k + it.hk * a.c.k_head;
    const T *vbase = (const T *)a.c.v + it.hk * a.c.v_head;
    const uint32_t klane = (col * (uint32_t)a.c.k_token + g * 8) * 2;
    const int vrow = lane / LPR, vch = lane % LPR;
    const uint32_t vlane = (vrow * (uint32_t)a.c.v_token + vch * 8) * 2;
    // a wave's 32 rows of V, and in the end its sums (16 rows of floats, as many bytes)
    auto mine = [&](int w) { return (w < 2 ? lds01 : lds23) + (w & 1) * VB; };
    char *vl = mine(wave);
    // (another chunk is an exclusive or, a row 16 on an addition)
    const uint32_t v_at = v_chunk<D>(4 * g + (col >> 2), (col >> 1) & 1) * 16 + (col & 1) * 8;

    f4 o[D / 16];
#pragma unroll
    for (int i = 0; i < D / 16; i++) o[i] = f4{0, 0, 0, 0};
    float m = -INFINITY, l = 0;
    V k[2][QS];
    u4 v[VL];
    int page[2];
    const int last_sub = it.k1 > 0 ? (it.k1 - 1) >> 4 : 0;

    auto look_up = [&](int base) {
#pragma unroll
        for (int n = 0; n < 2; n++)
            page[n] = tab[min((base >> 4) + n, last_sub) >> a.sub_shift];
    };
    auto load = [&](int base) {
#pragma unroll
        for (int n = 0; n < 2; n++) {
            const int64_t off = (min((base >> 4) + n, last_sub) & sub_mask) * 16;
            const char *kp = (const char *)(kbase + page[n] * a.c.k_block + off * a.c.k_token);
            const char *vp = (const char *)(vbase + page[n] * a.c.v_block + off * a.c.v_token);
#pragma unroll
            for (int i = 0; i < QS; i++)
                k[n][i] = __builtin_bit_cast(V, stream(kp + klane + i * 64));
#pragma unroll
            for (int i = 0; i < VL / 2; i++)
                v[n * VL / 2 + i] =
                    stream(vp + (int64_t)(i * (64 / LPR)) * a.c.v_token * 2 + vlane);
        }
    };
    int base = __builtin_amdgcn_readfirstlane(it.k0 + wave * kThinKeys);
    const int stride = 4 * kThinKeys;
    if (base < it.k1) {
        look_up(base);
        load(base);
        look_up(base + stride);
    }
    for (; base < it.k1; base += stride) {
        f4 sc[2];
#pragma unroll
        for (int n = 0; n < 2; n++) {
            sc[n] = f4{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < QS; i++) sc[n] = mfma16(k[n][i], q[i], sc[n]);
        }
        if (base + kThinKeys > it.k1)  // slots past the keys hold anything: weight 0 times it
#pragma unroll
            for (int i = 0; i < VL; i++)
                if (base + i * (64 / LPR) + vrow >= it.k1) v[i] = u4{0, 0, 0, 0};
        uint32_t marked = 0;  // of the 32 keys
        if (base + kThinKeys > full && full < it.k1) {
#pragma unroll
            for (int i = 0; i < VL; i++) {
                const uint64_t lanes = __ballot(any_not_finite<T>(v[i]));
                if (lanes) {
                    v[i] = zero_not_finite<T>(v[i]);
                    for (int y = 0; y < 64 / LPR; y++)
                        if (lanes >> (y * LPR) & ((1u << LPR) - 1))
                            marked |= 1u << (i * (64 / LPR) + y);
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int i = 0; i < VL; i++)
            *(u4 *)(vl + v_chunk<D>(i * (64 / LPR) + vrow, vch) * 16) = v[i];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (base + stride < it.k1) {
            load(base + stride);
            look_up(base + 2 * stride);
        }

        if (base + kThinKeys > full)
#pragma unroll
            for (int n = 0; n < 2; n++)
#pragma unroll
                for (int i = 0; i < 4; i++)
                    if (base + n * 16 + g * 4 + i >= lim) sc[n][i] = -INFINITY;
        // (this lane's keys: 4 g .. 4 g + 3 and 16 on)
        if (marked && (marked & first_bits(lim - base) & (0xf000fu << (g * 4)))) l = NAN;
        float mt = -INFINITY;
#pragma unroll
        for (int n = 0; n < 2; n++)
#pragma unroll
            for (int i = 0; i < 4; i++) mt = fmaxf(mt, sc[n][i]);
        mt = max32(max16(mt)) * a.scale2;
        if (__any(mt > m + kRaise<T>)) {
            const float mn = mt > m + kRaise<T> ? mt - kHeadroom<T> : m;
            const float f = mn == m ? 1.0f : exp2_(m - mn);
            m = mn;
            l *= f;
#pragma unroll
            for (int i = 0; i < D / 16; i++) o[i] *= f;
        }
        const float mu = m == -INFINITY ? 0.0f : m;
        V p;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float y = exp2_(sc[i >> 2][i & 3] * a.scale2 - mu);
            l += y;
            p[i] = (T)y;
        }
#pragma unroll
        for (int i = 0; i < D / 16; i++) {
            // lane c of group g: column d = 16 i + c of the rows 4 g .. 4 g + 3 and 16 on
            const char *at = vl + (v_at ^ (i * 32));
            const s4 lo = read_tr(at), hi = read_tr(at + 256 * LPR);
            const s8 t = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            o[i] = mfma16(__builtin_bit_cast(V, t), p, o[i]);
        }
    }

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

typedef const __attribute__((address_space(1))) char *Global;
__device__ void load_to_lds(Global from, char *to) {
    __builtin_amdgcn_global_load_lds(from, (__attribute__((address_space(3))) void *)to, 16, 0,
                                     0);
}
template <int N>
struct Const {
    static constexpr int value = N;
};
// The order of a stretch: N times a matrix product, a load to LDS at every other of
// them, vector work that does not wait for it, and LDS reads for the next stretch.
template <int N, int VECTOR, int READS, bool LOADS = false>
__device__ __forceinline__ void mix() {
    if constexpr (N > 0) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        if (LOADS && N % 2 == 0) __builtin_amdgcn_sched_group_barrier(0x10, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x2, VECTOR, 0);
        if (READS) __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
        mix<N - 1, VECTOR, READS, LOADS>();
    }
}
constexpr int kMarks = 8;  // words of 32 keys
constexpr int kWaitLoads = 0x0F70;  // s_waitcnt: no load or store outstanding

// 128 rows against a run of keys, 64 keys a step: 32 rows to a wave, K and V of a
// step in LDS for all four waves, loaded there directly and double buffered. A step
// is two stretches in which the matrix unit and the vector unit have independent
// work: S of the next keys beside the exponentials of these, then P V of these beside
// the maximum of the next. One barrier ends a step; the loads it waits for had most of
// the step to arrive. In a stretch the products, the vector work, the LDS reads and the
// loads to LDS alternate: V is read before the weights are worked out, whose end no read
// passes, and the loads go between the products, V's in the first stretch and K's in the
// second. (16 chunks of 11777 tokens, 32/8 heads of 128: 927 us with the products behind
// the vector work, 908 with V read first, 897 with the loads spread as well; 850 to 891 now,
// by the card, 1030 to 983 TFLOP/s.)
template <typename T, int D>
__device__ __forceinline__ void wide_item(const AttnArgs &a, const Item &it, char *k0_lds,
                                          char *k1_lds, char *v0_lds, char *v1_lds,
                                          uint32_t *marked) {
    using V = vec8<T>;
    constexpr int QS = D / 16;             // steps of 16 over d
    constexpr int LPR = D / 8;             // chunks of 16 bytes of a row
    constexpr int TB = kWideKeys * D * 2;  // bytes of a tile
    constexpr int NL = TB / 4096;          // loads of a wave for a tile
    constexpr int RPL = 64 / LPR;          // rows of one wave's load
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, half = lane >> 5;
    const Seg &s = it.s;
    const Table tab = (Table)(a.tables + s.table);

    const int r = wave * 32 + col;  // row of the item
    const int row = min(it.row0 + r, s.rows - 1), j = row / a.group;
    const int lim = min(min(s.kv_len, s.lim0 + j), it.k1);
    V q[QS];
    {
        const T *src = (const T *)a.q + (int64_t)(s.t0 + j) * a.q_stride +
                       (int64_t)(it.hk * a.group + row - j * a.group) * D + half * 8;
#pragma unroll
        for (int i = 0; i < QS; i++) q[i] = *(const V *)(src + i * 16);
    }
    const int full = min(min(s.kv_len, s.lim0 + it.row0 / a.group), it.k1);
    const int sub_mask = (1 << a.sub_shift) - 1;
    const int last_sub = it.k1 > 0 ? (it.k1 - 1) >> 4 : 0;
    const char *kbase = (const char *)((const T *)a.c.k + it.hk * a.c.k_head);
    const char *vbase = (const char *)((const T *)a.c.v + it.hk * a.c.v_head);

    // A wave loads a run of 16 keys of a tile: load i fills 1 KB, rows i RPL on of the run
    // (so that a wave works out two addresses a step: with rows of four runs, and eight
    // addresses, the 16 chunks took 3 % longer). Chunk c of row y of K lies at
    // c ^ (y mod LPR), which spreads the rows of a column over the banks; a lane's place
    // is fixed, so it fetches the chunk that belongs there.
    const int lrow = lane / LPR, lch = lane % LPR;
    uint32_t klane[NL], vlane[NL];
#pragma unroll
    for (int i = 0; i < NL; i++) {
        const int y = i * RPL + lrow;
        klane[i] = y * (uint32_t)(a.c.k_token * 2) + (lch ^ (y & (LPR - 1))) * 16;
        vlane[i] = y * (uint32_t)(a.c.v_token * 2) + (v_chunk<D>(y, lch) - y * LPR) * 16;
    }
    // Even lanes work out where the wave's next run of K lies, odd lanes that of V; the
    // block number is read a step before that.
    const bool of_v = lane & 1;
    const uint64_t base_of = (uint64_t)(of_v ? vbase : kbase);
    const uint32_t block_bytes = (uint32_t)((of_v ? a.c.v_block : a.c.k_block) * 2);
    const uint32_t run_bytes = (uint32_t)((of_v ? a.c.v_token : a.c.k_token) * 32);
    int page = 0, run = 0;
    auto look_up = [&](int v_base, int k_base) {
        const int sub = min(((of_v ? v_base : k_base) >> 4) + wave, last_sub);
        page = tab[sub >> a.sub_shift];
        run = sub & sub_mask;
    };
    uint64_t k_from = 0, v_from = 0;
    auto place = [&]() {
        const uint64_t at = base_of + (uint64_t)(uint32_t)page * block_bytes +
                            (uint64_t)(uint32_t)run * run_bytes;
        const uint32_t lo = (uint32_t)at, hi = (uint32_t)(at >> 32);
        k_from = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(hi, 0) << 32 |
                 (uint32_t)__builtin_amdgcn_readlane(lo, 0);
        v_from = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(hi, 1) << 32 |
                 (uint32_t)__builtin_amdgcn_readlane(lo, 1);
    };
    auto load = [&](char *to, uint64_t from, const uint32_t (&at)[NL]) {
#pragma unroll
        for (int i = 0; i < NL; i++)
            load_to_lds((Global)from + at[i], to + (wave * NL + i) * 1024);
    };
    auto load_k = [&](char *to) { load(to, k_from, klane); };
    auto load_v = [&](char *to) { load(to, v_from, vlane); };
    // The rows see the keys from here on to the end differently (at most 128 + 63 keys;
    // a bit each in `marked`).
    const int differ = full < it.k1 ? full & ~31 : it.k1;
    if (full < it.k1) {
        if (tid < kMarks) marked[tid] = 0;
        __syncthreads();
    }
    // Waits for the loads; slots past the keys hold anything, and weight 0 times it
    // has to be 0: a wave clears what it loaded of them.
    auto arrive = [&](char *v, int base, bool edge) {
        __builtin_amdgcn_s_waitcnt(kWaitLoads);
        if (edge && base + kWideKeys > differ)
#pragma unroll
            for (int i = 0; i < NL; i++) {
                u4 *at = (u4 *)(v + (wave * NL + i) * 1024 + lane * 16);
                const int y = base + wave * 16 + i * RPL + lrow;
                if (y >= it.k1) {
                    *at = u4{0, 0, 0, 0};
                } else if (y >= differ && any_not_finite<T>(*at)) {
                    *at = zero_not_finite<T>(*at);
                    atomicOr(marked + ((y - differ) >> 5), 1u << (y & 31));
                }
            }
        __syncthreads();
    };

    f16x o[D / 32];
#pragma unroll
    for (int i = 0; i < D / 32; i++)
#pragma unroll
        for (int e = 0; e < 16; e++) o[i][e] = 0;
    float m = -INFINITY, l = 0;

    // The chunk's number is in bits 4 and up of an address, so another chunk is an
    // exclusive or, another row (of the same swizzle) an addition.
    const uint32_t k_at = (col * LPR + (half ^ (col & (LPR - 1)))) * 16;
    const int tr = (lane & 15) >> 2, tc = ((lane >> 4) & 1) * 2 + ((lane >> 1) & 1);
    const uint32_t v_at = v_chunk<D>(half * 4 + tr, tc) * 16 + (lane & 1) * 8;
    // The left operands for 32 keys: of the scores, and of the products, whose k-slots
    // of step n are the keys 16 n + 4 half + 0..3 and 8 on, as the scores hold them.
    V kf[QS], vf[2][D / 32];
    auto read_k = [&](const char *kl) {
#pragma unroll
        for (int i = 0; i < QS; i++) kf[i] = *(const V *)(kl + (k_at ^ (i * 32)));
    };
    auto read_v = [&](const char *vl) {
#pragma unroll
        for (int n = 0; n < 2; n++)
#pragma unroll
            for (int i = 0; i < D / 32; i++) {
                const char *at = vl + (v_at ^ (i * 64)) + n * 256 * LPR;
                const s4 lo = read_tr(at), hi = read_tr(at + 128 * LPR);
                const s8 t = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                vf[n][i] = __builtin_bit_cast(V, t);
            }
    };
    auto scores = [&](f16x &sc) {
#pragma unroll
        for (int e = 0; e < 16; e++) sc[e] = 0;
#pragma unroll
        for (int i = 0; i < QS; i++) sc = mfma32(kf[i], q[i], sc);
    };
    auto hide = [&](f16x &sc, int base) {
#pragma unroll
        for (int e = 0; e < 16; e++)
            if (base + (e >> 2) * 8 + half * 4 + (e & 3) >= lim) sc[e] = -INFINITY;
    };
    // (the V of these keys has arrived, so their marks are complete)
    auto poison = [&](int base) {
        if (base < differ || base >= it.k1) return;
        // (this lane's keys: 4 half .. 4 half + 3, and 8, 16 and 24 on)
        if (marked[(base - differ) >> 5] & first_bits(lim - base) & (0xf0f0f0fu << (half * 4)))
            l = NAN;
    };
    auto largest = [&](const f16x &sc) {
        float mt = -INFINITY;
#pragma unroll
        for (int e = 0; e < 16; e++) mt = fmaxf(mt, sc[e]);
        return max32(mt) * a.scale2;
    };
    auto raise = [&](float mt) {
        if (__any(mt > m + kRaise<T>)) {
            const float mn = mt > m + kRaise<T> ? mt - kHeadroom<T> : m;
            const float f = mn == m ? 1.0f : exp2_(m - mn);
            m = mn;
            l *= f;
#pragma unroll
            for (int i = 0; i < D / 32; i++) o[i] *= f;
        }
    };
    auto weights = [&](V (&p)[2], const f16x &sc) {
        const float mu = m == -INFINITY ? 0.0f : m;
#pragma unroll
        for (int e = 0; e < 16; e++) {
            const float y = exp2_(sc[e] * a.scale2 - mu);
            l += y;
            p[e >> 3][e & 7] = (T)y;
        }
        // computed here, beside the scores, and not where they are used
#pragma unroll
        for (int n = 0; n < 2; n++) {
            u4 x = __builtin_bit_cast(u4, p[n]);
            asm volatile("" : "+v"(x));
            p[n] = __builtin_bit_cast(V, x);
        }
    };
    auto products = [&](const V (&p)[2]) {
#pragma unroll
        for (int n = 0; n < 2; n++)
#pragma unroll
            for (int i = 0; i < D / 32; i++) o[i] = mfma32(vf[n][i], p[n], o[i]);
    };

    // The K of a buffer is 32 keys ahead of its V: on entry of a step sa are the scores
    // of the keys base .. + 31, m covers them, buffer B holds the V from base on and
    // the K from base + 32 on.
    constexpr int HB = TB / 2;  // bytes of 32 rows
    f16x sa, sb;
    V p[2];
    // EDGE: its keys and the next ones may be seen by some rows only.
    auto step = [&](auto which, auto edge, int base) {
        constexpr int B = decltype(which)::value, EDGE = decltype(edge)::value;
        const char *kl = B ? k1_lds : k0_lds, *vl = B ? v1_lds : v0_lds;
        const int next = base + kWideKeys;
        if (EDGE) poison(base);
        read_k(kl);
        place();
        look_up(next + kWideKeys, next + kWideKeys + 32);
        __builtin_amdgcn_sched_barrier(0);
        load_v(B ? v0_lds : v1_lds);
        scores(sb);
        read_v(vl);
        weights(p, sa);
        mix<QS, 56 / QS, D / 8 / QS, true>();
        __builtin_amdgcn_sched_barrier(0);
        if (EDGE) hide(sb, base + 32);
        load_k(B ? k0_lds : k1_lds);
        products(p);
        read_k(kl + HB);
        const float mb = largest(sb);
        mix<D / 16, 4, QS / (D / 16), true>();
        raise(mb);
        if (EDGE) poison(base + 32);
        __builtin_amdgcn_sched_barrier(0);
        scores(sa);
        read_v(vl + HB);
        weights(p, sb);
        mix<QS, 56 / QS, D / 8 / QS>();
        __builtin_amdgcn_sched_barrier(0);
        if (EDGE) hide(sa, next);
        products(p);
        const float ma = largest(sa);
        mix<D / 16, 4, 0>();
        raise(ma);
        arrive(B ? v0_lds : v1_lds, next, EDGE);
    };
    if (it.k0 < it.k1) {
        int base = it.k0;
        look_up(base, base);
        place();
        load_k(k1_lds);
        load_v(v0_lds);
        look_up(base, base + 32);
        place();
        load_k(k0_lds);
        look_up(base + kWideKeys, base + kWideKeys + 32);
        arrive(v0_lds, base, true);
        read_k(k1_lds);
        scores(sa);
        hide(sa, base);
        raise(largest(sa));
        __syncthreads();  // the first step loads K where these were
        int steps = (it.k1 - base - 1) / kWideKeys;
        for (; steps >= 2 && base + 3 * kWideKeys <= differ; steps -= 2) {
            step(Const<0>{}, Const<0>{}, base);
            step(Const<1>{}, Const<0>{}, base + kWideKeys);
            base += 2 * kWideKeys;
        }
        for (; steps >= 2; steps -= 2) {
            step(Const<0>{}, Const<1>{}, base);
            step(Const<1>{}, Const<1>{}, base + kWideKeys);
            base += 2 * kWideKeys;
        }
        if (steps) {
            step(Const<0>{}, Const<1>{}, base);
            base += kWideKeys;
        }
        const char *kl = steps ? k1_lds : k0_lds, *vl = steps ? v1_lds : v0_lds;
        poison(base);
        weights(p, sa);
        read_v(vl);
        products(p);
        if (base + 32 < it.k1) {
            read_k(kl);
            scores(sa);
            hide(sa, base + 32);
            poison(base + 32);
            raise(largest(sa));
            weights(p, sa);
            read_v(vl + HB);
            products(p);
        }
    }
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

// One item a workgroup. A thin item whose partial results have reached the device is
// counted for its unit, and the workgroup that counts the last one joins the unit; the
// count is left at zero for the next launch. (The rows of wide segments are left to the merge kernel: the workgroup that
// came last would join 128 rows one after another. Decode of 64 requests with a shared
// prefix of 2048, 32/8 heads of 128: 71 us so, 23.5 us with the merge kernel.)
template <typename T, int D, bool WIDE>
__global__ __launch_bounds__(256, WIDE ? 2 : 3) void attn_kernel(AttnArgs a) {
    constexpr int TB = kWideKeys * D * 2;
    // four objects, so that the compiler sees which loads a read has to wait for
    __shared__ __attribute__((aligned(16))) char k0_lds[TB], k1_lds[TB];
    __shared__ __attribute__((aligned(16))) char v0_lds[WIDE ? TB : 16], v1_lds[WIDE ? TB : 16];
    __shared__ float stat[WIDE ? 1 : 4][kThinRows][2];
    __shared__ uint32_t marked[kMarks];
    const Item it = a.items[blockIdx.x];
    if (WIDE && it.s.rows > kThinRows)
        wide_item<T, D>(a, it, k0_lds, k1_lds, v0_lds, v1_lds, marked);
    else
        thin_item<T, D>(a, it, k0_lds, k1_lds,
                        WIDE ? (float (*)[kThinRows][2])(void *)v0_lds : stat);
    if (it.unit < 0) return;
    // this wave's results have arrived; then the others' have
    __builtin_amdgcn_s_waitcnt(kWaitLoads);
    __syncthreads();
    const Unit u = a.units[it.unit];
    int *last = (int *)k0_lds;
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

template <typename T, int D>
__global__ __launch_bounds__(256) void merge_kernel(AttnArgs a) {
    join<T, D, false>(a, a.merge[blockIdx.x]);
}

template <typename T, int D>
hipError_t launch(const AttnArgs &a, int n, int n_merge, hipStream_t s) {
    const hipError_t e = launch_kernel(
        a.n_wide ? attn_kernel<T, D, true> : attn_kernel<T, D, false>, n, a, s);
    if (e != hipSuccess || !n_merge) return e;
    return launch_kernel(merge_kernel<T, D>, n_merge, a, s);
}

}  // namespace

hipError_t launch_attention(const AttnArgs &a, int n, int n_merge, int dtype, int head_dim,
                            hipStream_t s) {
    if (dtype == TAS_F16)
        return head_dim == 64 ? launch<_Float16, 64>(a, n, n_merge, s)
                              : launch<_Float16, 128>(a, n, n_merge, s);
    return head_dim == 64 ? launch<__bf16, 64>(a, n, n_merge, s)
                          : launch<__bf16, 128>(a, n, n_merge, s);
}

}  // namespace tas_step_impl
