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

#include "tas_step_attn.h"
#include "tas_step_internal.h"

namespace tas_step_impl {
namespace {

// The place in LDS (in 16-byte chunks) of chunk c of a V row: the four rows that
// one transposing read takes lie in different quarters of the banks.
template <int D>
__device__ int v_chunk(int row, int c) {
    if (D == 128) return row * 16 + (c ^ (((row & 3) << 2) | ((row >> 1) & 2)));
    return row * 8 + (c ^ ((row & 3) << 1));
}

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

    thin_end<T, D>(a, it, l, m, o, lds01, lds23, stat);
}

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
    wide_end<T, D>(a, it, l, m, o);
}

// One item a workgroup.
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
    if (it.unit >= 0) count_item<T, D>(a, it, (int *)k0_lds);
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

hipError_t launch_merge(const AttnArgs &a, int n, int dtype, int head_dim, hipStream_t s) {
    if (dtype == TAS_F16)
        return head_dim == 64 ? launch_kernel(merge_kernel<_Float16, 64>, n, a, s)
                              : launch_kernel(merge_kernel<_Float16, 128>, n, a, s);
    return head_dim == 64 ? launch_kernel(merge_kernel<__bf16, 64>, n, a, s)
                          : launch_kernel(merge_kernel<__bf16, 128>, n, a, s);
}

}  // namespace tas_step_impl
