// tas_fp4_attn.hip - attention of a step's new tokens over a paged cache in four bits.
//
// The mathematics, the items and the joins are those of tas_step_attn.hip. What differs is
// the way of K and V to the matrix unit: codes are loaded to registers (a third to a quarter
// of the bytes), converted there to the 16-bit type, exactly, two elements an instruction,
// and go on as 16-bit rows. A lane always has a quarter of a row, D / 8 bytes, which lies in
// one block: one scale to a lane and row.
#include <hip/hip_runtime.h>

#include "tas_fp4_convert.h"
#include "tas_fp4_internal.h"
#include "tas_step_attn.h"

namespace tas_step_impl {
namespace {

// The four bytes of a lane's quarter of a row.
template <int D>
struct Quarter {
    static constexpr int W = D / 32;  // words, of eight elements
    uint32_t w[W];
};

// ONCE: its line is not read again soon. (256 decodes 102 us, 113 with lines kept; 16 chunks, whose
// items share K and V, 812, 850 with lines not kept.)
template <int D, bool ONCE>
__device__ Quarter<D> load_quarter(Global p) {
    typedef uint32_t words __attribute__((ext_vector_type(D / 32)));
    typedef const __attribute__((address_space(1))) words *Words;
    const words x = ONCE ? __builtin_nontemporal_load((Words)p) : *(Words)p;
    Quarter<D> q;
#pragma unroll
    for (int i = 0; i < D / 32; i++) q.w[i] = x[i];
    return q;
}

__device__ uint32_t load_scale(Global p) {
    return *(const __attribute__((address_space(1))) uint8_t *)p;
}

// The block of a row that quarter i lies in.
template <int D>
__device__ int block_of(int i) {
    return D == 128 ? i : i >> 1;
}

// Places in LDS (in 16-byte chunks of eight elements) of chunk c of row y. The banks take 16
// chunks at once: of a write, 16 lanes, which have the quarters of four rows (chunks D / 32
// apart: their low bits are turned by the quarter); of a transposing read, 32 lanes with two
// chunks of eight rows (thin items) or four of four; of a read of K, 16 rows' chunk. Each
// time they lie in different places of 16 (at head size 64 a pair of rows has 16).
template <int D>
__device__ constexpr int turned(int c) {
    return D == 128 ? c ^ (c >> 2) : c;
}
template <int D>
__device__ int v_place(int y, int c) {
    if (D == 128) return y * 16 + (turned<D>(c) ^ ((y & 3) << 2 | (y >> 1 & 2)));
    return y * 8 + (c ^ ((y >> 1 & 1) * 5) ^ (y >> 1 & 2));
}
template <int D>
__device__ int k_place(int y, int c) {
    if (D == 128) return y * 16 + (turned<D>(c) ^ (y & 15));
    return y * 8 + (c ^ (y >> 1 & 7));
}

// Up to 16 rows against a run of keys: each of the four waves takes every fourth 32 keys.
// K goes straight into registers as the left operand: lane 16 g + r has the quarter g of key
// r, so that the k-slots of step i stand for elements g D / 4 + 8 i + 0..7, for the queries
// too. V goes through the wave's own LDS. Memory bound: 256 decodes 99 us, 6.0 TB/s.
template <typename T, int D>
__device__ __forceinline__ void thin_item4(const Attn4Args &a, const Item &it, char *lds01,
                                           char *lds23, float (*stat)[kThinRows][2]) {
    using V = vec8<T>;
    constexpr int QS = D / 32;             // steps of 32 over d, words of a quarter
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
                       (int64_t)(it.hk * a.group + row - j * a.group) * D + g * (D / 4);
#pragma unroll
        for (int i = 0; i < QS; i++) q[i] = *(const V *)(src + i * 8);
    }
    const int full = min(min(s.kv_len, s.lim0), it.k1);  // keys that the first row sees
    const int sub_mask = (1 << a.sub_shift) - 1;
    const int vrow = lane >> 2, vq = lane & 3;
    auto head_of = [&](const tas_rows &r) { return (const char *)r.p + it.hk * r.stride[1]; };
    const char *kbase = head_of(a.f.k), *vbase = head_of(a.f.v);
    const char *ksbase = head_of(a.f.k_scale), *vsbase = head_of(a.f.v_scale);
    const uint32_t klane = col * (uint32_t)a.f.k.stride[2] + g * (D / 8);
    const uint32_t kslane = col * (uint32_t)a.f.k_scale.stride[2] + block_of<D>(g);
    const uint32_t vlane = vrow * (uint32_t)a.f.v.stride[2] + vq * (D / 8);
    const uint32_t vslane = vrow * (uint32_t)a.f.v_scale.stride[2] + block_of<D>(vq);
    // a wave's 32 rows of V, and in the end its sums (16 rows of floats, as many bytes)
    auto mine = [&](int w) { return (w < 2 ? lds01 : lds23) + (w & 1) * VB; };
    char *vl = mine(wave);
    // (another pair of chunks is an exclusive or, a row 16 on an addition)
    const uint32_t v_at = v_place<D>(4 * g + (col >> 2), (col >> 1) & 1) * 16 + (col & 1) * 8;
    char *v_to[QS];
#pragma unroll
    for (int i = 0; i < QS; i++) v_to[i] = vl + v_place<D>(vrow, vq * QS + i) * 16;

    f4 o[D / 16];
#pragma unroll
    for (int i = 0; i < D / 16; i++) o[i] = f4{0, 0, 0, 0};
    float m = -INFINITY, l = 0;
    Quarter<D> k[2], v[2];
    uint32_t ks[2], vs[2];
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
            auto run = [&](const char *p, const tas_rows &r) {
                return (Global)p + page[n] * r.stride[0] + off * r.stride[2];
            };
            k[n] = load_quarter<D, true>(run(kbase, a.f.k) + klane);
            ks[n] = load_scale(run(ksbase, a.f.k_scale) + kslane);
            v[n] = load_quarter<D, true>(run(vbase, a.f.v) + vlane);
            vs[n] = load_scale(run(vsbase, a.f.v_scale) + vslane);
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
            for (int i = 0; i < QS; i++)
                sc[n] = mfma16(values_of<T>(k[n].w[i], scale_of(ks[n])), q[i], sc[n]);
        }
        uint32_t marked = 0;  // of the 32 keys
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int n = 0; n < 2; n++)
#pragma unroll
            for (int i = 0; i < QS; i++)
                *(u4 *)(v_to[i] + n * 32 * D) =
                    __builtin_bit_cast(u4, values_of<T>(v[n].w[i], scale_of(vs[n])));
        if (base + kThinKeys > full) {  // some of them are changed there (what a lane wrote)
#pragma unroll 1
            for (int w = 0; w < 2 * QS; w++) {
                const int n = w / QS;
                u4 *at = (u4 *)(vl + v_place<D>(n * 16 + vrow, vq * QS + w % QS) * 16);
                u4 x = *at;
                // slots past the keys hold anything: weight 0 times it
                if (base + n * 16 + vrow >= it.k1) x = u4{0, 0, 0, 0};
                const uint64_t lanes = __ballot(any_not_finite<T>(x));
                if (lanes && full < it.k1) {
                    x = zero_not_finite<T>(x);
                    for (int y = 0; y < 16; y++)
                        if (lanes >> (y * 4) & 15) marked |= 1u << (n * 16 + y);
                }
                *at = x;
            }
        }
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
            const char *at = vl + (v_at ^ (turned<D>(2 * i) * 16));
            const s4 lo = read_tr(at), hi = read_tr(at + 32 * D);
            const s8 t = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            o[i] = mfma16(__builtin_bit_cast(V, t), p, o[i]);
        }
    }
    thin_end<T, D>(a, it, l, m, o, lds01, lds23, stat);
}

// The order of a stretch: N times a matrix product, vector work that does not wait for it, LDS
// reads for the next stretch and, at every other, an LDS write.
template <int N, int VECTOR, int READS, int WRITES>
__device__ __forceinline__ void mix4() {
    if constexpr (N > 0) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x2, VECTOR, 0);
        if (READS) __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
        if (WRITES && N % 2 == 0) __builtin_amdgcn_sched_group_barrier(0x200, WRITES, 0);
        mix4<N - 1, VECTOR, READS, WRITES>();
    }
}

// 128 rows against a run of keys, as the 16-bit kernel's wide item: 64 keys a step, 32 rows
// to a wave, K and V of a step in LDS as 16-bit rows for all four waves, double buffered.
// A wave fetches a run of 16 keys of K and of V a whole step before it converts them and
// writes them to LDS. Bound by matrix and vector work in turn: 11777 tokens of 16 chunks 803 us,
// 1080 TFLOP/s, the matrix unit busy half of the time.
template <typename T, int D>
__device__ __forceinline__ void wide_item4(const Attn4Args &a, const Item &it, char *k0_lds,
                                           char *k1_lds, char *v0_lds, char *v1_lds,
                                           uint32_t *marked) {
    using V = vec8<T>;
    constexpr int QS = D / 16;             // steps of 16 over d
    constexpr int W = D / 32;              // words of a quarter of a row
    constexpr int LPR = D / 8;             // chunks of 16 bytes of a row
    constexpr int TB = kWideKeys * D * 2;  // bytes of a tile
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

    const int lrow = lane >> 2, lq = lane & 3;
    const uint32_t klane = lrow * (uint32_t)a.f.k.stride[2] + lq * (D / 8);
    const uint32_t vlane = lrow * (uint32_t)a.f.v.stride[2] + lq * (D / 8);
    const uint32_t kslane = lrow * (uint32_t)a.f.k_scale.stride[2] + block_of<D>(lq);
    const uint32_t vslane = lrow * (uint32_t)a.f.v_scale.stride[2] + block_of<D>(lq);
    // Lanes 0 to 3 work out where the wave's next run lies, of K, V and their scales; the
    // block number is read a step before that.
    const bool of_v = lane & 1;
    const tas_rows &mine = lane & 2 ? (of_v ? a.f.v_scale : a.f.k_scale) : (of_v ? a.f.v : a.f.k);
    const uint64_t base_of = (uint64_t)mine.p + it.hk * mine.stride[1];
    const uint32_t block_bytes = (uint32_t)mine.stride[0];
    const uint32_t run_bytes = (uint32_t)mine.stride[2] * 16;
    int page = 0, run = 0;
    auto look_up = [&](int v_base, int k_base) {
        const int sub = min(((of_v ? v_base : k_base) >> 4) + wave, last_sub);
        page = tab[sub >> a.sub_shift];
        run = sub & sub_mask;
    };
    uint32_t at_lo = 0, at_hi = 0;
    auto place = [&]() {
        const uint64_t at = base_of + (uint64_t)(uint32_t)page * block_bytes +
                            (uint64_t)(uint32_t)run * run_bytes;
        at_lo = (uint32_t)at, at_hi = (uint32_t)(at >> 32);
    };
    // (a pointer whose loads do not count as LDS's: those would be waited for with LDS's)
    auto from = [&](int l) {
        return (Global)((uint64_t)(uint32_t)__builtin_amdgcn_readlane(at_hi, l) << 32 |
                        (uint32_t)__builtin_amdgcn_readlane(at_lo, l));
    };
    Quarter<D> kq, vq;
    uint32_t ks, vs;
    auto fetch_k = [&]() {
        kq = load_quarter<D, false>(from(0) + klane);
        ks = load_scale(from(2) + kslane);
    };
    auto fetch_v = [&]() {
        vq = load_quarter<D, false>(from(1) + vlane);
        vs = load_scale(from(3) + vslane);
    };
    // The rows see the keys from here on to the end differently (at most 128 + 63 keys;
    // a bit each in `marked`).
    const int differ = full < it.k1 ? full & ~31 : it.k1;
    if (full < it.k1) {
        if (tid < kMarks) marked[tid] = 0;
        __syncthreads();
    }
    const int y0 = wave * 16 + lrow;  // this lane's row of a tile
    auto put_k = [&](char *to) {
#pragma unroll
        for (int i = 0; i < W; i++)
            *(u4 *)(to + k_place<D>(y0, lq * W + i) * 16) =
                __builtin_bit_cast(u4, values_of<T>(kq.w[i], scale_of(ks)));
    };
    // Slots past the keys hold anything, and weight 0 times it has to be 0.
    auto put_v = [&](char *to, int base, bool edge) {
#pragma unroll
        for (int i = 0; i < W; i++) {
            u4 x = __builtin_bit_cast(u4, values_of<T>(vq.w[i], scale_of(vs)));
            if (edge && base + kWideKeys > differ) {
                const int y = base + y0;
                if (y >= it.k1) {
                    x = u4{0, 0, 0, 0};
                } else if (y >= differ && any_not_finite<T>(x)) {
                    x = zero_not_finite<T>(x);
                    atomicOr(marked + ((y - differ) >> 5), 1u << (y & 31));
                }
            }
            *(u4 *)(to + v_place<D>(y0, lq * W + i) * 16) = x;
        }
    };

    f16x o[D / 32];
#pragma unroll
    for (int i = 0; i < D / 32; i++)
#pragma unroll
        for (int e = 0; e < 16; e++) o[i][e] = 0;
    float m = -INFINITY, l = 0;

    // The chunk's number is in bits 4 and up of an address, so another chunk is an
    // exclusive or, another row (of the same place) an addition.
    const uint32_t k_at = k_place<D>(col, half) * 16;
    const int tr = (lane & 15) >> 2, tc = ((lane >> 4) & 1) * 2 + ((lane >> 1) & 1);
    const uint32_t v_at = v_place<D>(half * 4 + tr, tc) * 16 + (lane & 1) * 8;
    V kf[QS], vf[2][D / 32];
    auto read_k = [&](const char *kl) {
#pragma unroll
        for (int i = 0; i < QS; i++)
            kf[i] = *(const V *)(kl + (k_at ^ (turned<D>(i * 2) * 16)));
    };
    auto read_v = [&](const char *vl) {
#pragma unroll
        for (int n = 0; n < 2; n++)
#pragma unroll
            for (int i = 0; i < D / 32; i++) {
                const char *at = vl + (v_at ^ (turned<D>(i * 4) * 16)) + n * 256 * LPR;
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
    // (the V of these keys is in LDS, so their marks are complete)
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
    // of the keys base .. + 31, m covers them, buffer B holds the V from base on and the K
    // from base + 32 on, and the next ones' codes are in registers.
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
        look_up(next + 2 * kWideKeys, next + 2 * kWideKeys + 32);
        __builtin_amdgcn_sched_barrier(0);
        scores(sb);
        read_v(vl);
        weights(p, sa);
        mix4<QS, 56 / QS, D / 8 / QS, 0>();
        __builtin_amdgcn_sched_barrier(0);
        if (EDGE) hide(sb, base + 32);
        put_k(B ? k0_lds : k1_lds);
        fetch_k();
        products(p);
        read_k(kl + HB);
        const float mb = largest(sb);
        mix4<D / 16, 6, QS / (D / 16), 1>();
        raise(mb);
        if (EDGE) poison(base + 32);
        __builtin_amdgcn_sched_barrier(0);
        scores(sa);
        read_v(vl + HB);
        weights(p, sb);
        mix4<QS, 56 / QS, D / 8 / QS, 0>();
        __builtin_amdgcn_sched_barrier(0);
        if (EDGE) hide(sa, next);
        put_v(B ? v0_lds : v1_lds, next, EDGE);
        fetch_v();
        products(p);
        const float ma = largest(sa);
        mix4<D / 16, 6, 0, 1>();
        raise(ma);
        __syncthreads();
    };
    if (it.k0 < it.k1) {
        int base = it.k0;
        look_up(base, base);
        place();
        fetch_k();
        fetch_v();
        look_up(base + kWideKeys, base + 32);
        put_k(k1_lds);
        put_v(v0_lds, base, true);
        place();
        fetch_k();
        fetch_v();
        look_up(base, base + kWideKeys + 32);
        put_k(k0_lds);
        place();
        fetch_k();
        look_up(base + 2 * kWideKeys, base + 2 * kWideKeys + 32);
        __syncthreads();
        read_k(k1_lds);
        scores(sa);
        hide(sa, base);
        raise(largest(sa));
        __syncthreads();  // the first step writes K where these were
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
__global__ __launch_bounds__(256, WIDE ? 2 : 4) void attn4_kernel(Attn4Args a) {
    constexpr int TB = kWideKeys * D * 2;
    // four objects, so that the compiler sees which loads a read has to wait for
    __shared__ __attribute__((aligned(16))) char k0_lds[TB], k1_lds[TB];
    __shared__ __attribute__((aligned(16))) char v0_lds[WIDE ? TB : 16], v1_lds[WIDE ? TB : 16];
    __shared__ float stat[WIDE ? 1 : 4][kThinRows][2];
    __shared__ uint32_t marked[kMarks];
    const Item it = a.items[blockIdx.x];
    if (WIDE && it.s.rows > kThinRows)
        wide_item4<T, D>(a, it, k0_lds, k1_lds, v0_lds, v1_lds, marked);
    else
        thin_item4<T, D>(a, it, k0_lds, k1_lds,
                         WIDE ? (float (*)[kThinRows][2])(void *)v0_lds : stat);
    if (it.unit >= 0) count_item<T, D>(a, it, (int *)k0_lds);
}

template <typename T, int D>
hipError_t launch(const Attn4Args &a, int n, int n_merge, int dtype, hipStream_t s) {
    const hipError_t e = launch_kernel(
        a.n_wide ? attn4_kernel<T, D, true> : attn4_kernel<T, D, false>, n, a, s);
    if (e != hipSuccess || !n_merge) return e;
    return launch_merge(a, n_merge, dtype, D, s);
}

}  // namespace

hipError_t launch_attention4(const Attn4Args &a, int n, int n_merge, int dtype, int head_dim,
                             hipStream_t s) {
    if (dtype == TAS_F16)
        return head_dim == 64 ? launch<_Float16, 64>(a, n, n_merge, dtype, s)
                              : launch<_Float16, 128>(a, n, n_merge, dtype, s);
    return head_dim == 64 ? launch<__bf16, 64>(a, n, n_merge, dtype, s)
                          : launch<__bf16, 128>(a, n, n_merge, dtype, s);
}

}  // namespace tas_step_impl
