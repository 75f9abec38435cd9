// tas_fp4_linear.hip - products of a step's tokens with weights in four bits.
//
// y[t][n] = sum over k of x[t][k] W[n][k], with W's values exact in the 16-bit type (a
// conversion of two elements an instruction), sums in 32 bits, rounded once. The transposed
// product Y^T = W X^T leaves four adjacent n of a token in a lane. The left operand is a
// tile of W as it lies in memory, one load of adjacent 16 bytes a lane, four products of a
// block each.
#include <hip/hip_runtime.h>

#include <utility>

#include "tas_fp4_convert.h"
#include "tas_fp4_internal.h"

namespace tas_step_impl {
namespace {

constexpr int kWaves = 8;

// Four adjacent n of token t.
template <typename T>
__device__ void store_four(const Linear4Args &a, int64_t t, int n, f4 x) {
    typedef T four __attribute__((ext_vector_type(4)));
    if (n >= a.rows) return;
    T *y = (T *)a.y + t * a.y_stride + n;
    if (a.y_fours) {
        *(four *)y = four{(T)x[0], (T)x[1], (T)x[2], (T)x[3]};
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++)
            if (n + i < a.rows) y[i] = (T)x[i];
    }
}

// A workgroup's part of the product. The eight dies take consecutive workgroups in turn, and each
// has an L2 of its own. Where x is much the larger side a die gets adjacent parts, so that x is
// fetched by one die, not by all that have some of its rows of W. (4096 columns, 8192 tokens, 100
// rows 34.5 us without, 16.0 so; 2000 tokens, 300 rows 18.4, 13.6; 8000 tokens, 1000 rows 61.3,
// 57.0. With sides of like size up to 7 % longer: 1024 tokens, 16384 rows 98.1, 105.2.)
struct Place {
    int n, t;  // of groups_n by some number
};
__device__ Place place_of(const Linear4Args &a, uint32_t groups_n) {
    uint32_t at = blockIdx.x;
    if (a.x_much) {
        const uint32_t die = at & 7, each = gridDim.x >> 3, more = gridDim.x & 7;
        at = die * each + min(die, more) + (at >> 3);
    }
    return {(int)(at % groups_n), (int)(at / groups_n)};
}

constexpr int kWaitLds = 0xC07F;  // s_waitcnt: no LDS access outstanding

// Waits until all but the wave's last N loads are done. (The empty statements keep the compiler
// from moving memory accesses across, the others from using earlier what has arrived later.)
template <int N>
__device__ void wait_loads() {
    static_assert(N < 64, "");
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(kWaitLoads | (N & 15) | (N >> 4) << 14);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// Few tokens: bound by the weights' bytes. A workgroup has all of K for 16 RT rows and 4 XL tokens
// (16 TT in the products). Its eight waves take every eighth tile of 128 columns, each by itself:
// weights in registers, four tiles asked for at once; x, half a tile at a time, through LDS of
// the wave's own, loaded there directly, whole lines of eight tokens a load, NB halves ahead.
// (Read as the product wants it, 16 bytes of 16 rows at a time, x takes more time than the
// weights: 16 tokens, 4096 rows and columns 6.7 us, 4.7 so; loaded to registers and written to
// LDS 6.0.) The waves' sums are joined in LDS, in one order: no partial results in memory, no
// second launch, no barrier before the join. Chunk c (of eight elements) of token t lies at
// c ^ (t / 2 mod 8), which spreads the rows of a column over the banks.
template <typename T, int RT, int XL, int NB>
__global__ __launch_bounds__(64 * kWaves, RT == 4 ? 2 : 4)
void stream_kernel(Linear4Args a) {
    using V = vec8<T>;
    constexpr int H = kWaves / 2, TT = (XL + 3) / 4, PL = XL / 2;  // (loads of half a tile)
    constexpr int XB = TT * 2048;  // bytes of half a tile of x
    static_assert(XL % 2 == 0 && (NB == 2 || NB == 4), "");
    // objects of their own, so that the compiler sees which loads a read has to wait for
    __shared__ __attribute__((aligned(16))) char x0[kWaves * XB], x1[kWaves * XB],
        x2[NB > 2 ? kWaves * XB : 16], x3[NB > 2 ? kWaves * XB : 16];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    const Place at = place_of(a, (a.tiles_n + RT - 1) / RT);
    const int tile0 = at.n * RT, t0 = at.t * 4 * XL;
    const char *codes[RT], *scales[RT];
#pragma unroll
    for (int i = 0; i < RT; i++) {  // (of tiles that there are not, the last one's)
        const int64_t tile = min(tile0 + i, a.tiles_n - 1);
        codes[i] = a.codes + tile * a.tiles_k * 1024;
        scales[i] = a.scales + tile * a.tiles_k * 64;
    }
    // load i: eight rows, 8 lanes each (offsets fit 32 bits: 64 rows of 2^25 bytes)
    const char *x_rows = (const char *)((const T *)a.x + t0 * a.x_stride);
    const int lrow = lane >> 3;
    auto chunk = [&](int i) { return (lane & 7) ^ ((i * 8 + lrow) >> 1 & 7); };
    uint32_t from[PL];
#pragma unroll
    for (int i = 0; i < PL; i++)
        from[i] = (uint32_t)min(i * 8 + lrow, a.tokens - 1 - t0) * (uint32_t)(a.x_stride * 2) +
                  chunk(i) * 16;
    auto buffer = [&](int n) {
        n %= NB;
        return (n == 0 ? x0 : n == 1 ? x1 : n == 2 ? x2 : x3) + wave * XB;
    };
    f4 sum[RT][TT];
#pragma unroll
    for (int i = 0; i < RT; i++)
#pragma unroll
        for (int j = 0; j < TT; j++) sum[i][j] = f4{0, 0, 0, 0};
    // four tiles of each wave, whole ones or those that there are
    auto unit = [&](auto whole, int u) {
        constexpr bool all = decltype(whole)::value;
        uint32_t sc[4][RT];
        u4 c[4][RT];
        auto tile = [&](int n) { return (u * 4 + n) * kWaves + wave; };
        auto load_x = [&](int n) {  // half n % 2 of tile n / 2
            const int b0 = tile(n / 2) * 4 + n % 2 * 2;
            if (!all && b0 >= a.blocks) return;
            const char *rows = x_rows + b0 * 64ll;
#pragma unroll
            for (int i = 0; i < PL; i++) {
                uint32_t at = from[i];
                // past the end: the first chunk, not used
                if (!all && b0 + chunk(i) / 4 >= a.blocks) at -= chunk(i) * 16;
                load_to_lds((Global)rows + at, buffer(n) + i * 1024);
            }
        };
#pragma unroll
        for (int n = 0; n < 4; n++) {
            const int tk = tile(n);
            if (!all && tk >= a.tiles_k) break;
#pragma unroll
            for (int i = 0; i < RT; i++) {
                const u4 *at = (const u4 *)(codes[i] + tk * 1024ll + (uint32_t)lane * 16);
                // (other tokens' workgroups read them too. 2000 tokens, 300 rows: 13.5 us with
                // lines that are not kept, 10.6 so; 256 tokens, 16384 columns 41.7, 39.3)
                c[n][i] = XL > 4 ? *at : __builtin_nontemporal_load(at);
                sc[n][i] = *(const uint32_t *)(scales[i] + tk * 64ll + (uint32_t)col * 4);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < NB; n++) load_x(n);
        auto half = [&](auto at) {
            constexpr int n = decltype(at)::value;
            const int b0 = tile(n / 2) * 4 + n % 2 * 2;
            if (!all && b0 >= a.blocks) return;
            wait_loads<all ? (NB - 1 < 7 - n ? NB - 1 : 7 - n) * PL : 0>();
#pragma unroll
            for (int k = 0; k < 2; k++) {
                V b[TT];
#pragma unroll
                for (int j = 0; j < TT; j++) {  // (rows beyond the tokens hold anything)
                    b[j] = *(const V *)(buffer(n) + (j * 16 + col) * 128 +
                                        ((k * 4 + g) ^ (col >> 1)) * 16);
                    // blocks beyond the matrix: zeros, as the weights are
                    if (!all && b0 + k >= a.blocks) b[j] = V{};
                }
                constexpr int q0 = n % 2 * 2;
#pragma unroll
                for (int i = 0; i < RT; i++) {
                    const V w = values_of<T>(c[n / 2][i][q0 + k],
                                             scale_of(sc[n / 2][i] >> (8 * (q0 + k)) & 255));
#pragma unroll
                    for (int j = 0; j < TT; j++) sum[i][j] = mfma16(w, b[j], sum[i][j]);
                }
            }
            __builtin_amdgcn_s_waitcnt(kWaitLds);  // the buffer has been read
            if (n + NB < 8) load_x(n + NB);
        };
        half(Const<0>{});
        half(Const<1>{});
        half(Const<2>{});
        half(Const<3>{});
        half(Const<4>{});
        half(Const<5>{});
        half(Const<6>{});
        half(Const<7>{});
    };
    const int whole = a.blocks / (16 * kWaves);
    int u = 0;
    for (; u < whole; u++) unit(Const<1>{}, u);
    if (u * 4 * kWaves < a.tiles_k) unit(Const<0>{}, u);
    // the second half's sums are added to the first's, then those to one another
    static_assert(H * RT * TT * 1024 <= kWaves * XB, "");
    f4 *part = (f4 *)x0 + lane;
    auto place = [&](int wave, int i) { return part + (wave * RT * TT + i) * 64; };
    __syncthreads();
    if (wave >= H)
#pragma unroll
        for (int i = 0; i < RT * TT; i++) *place(wave - H, i) = sum[i / TT][i % TT];
    __syncthreads();
    if (wave < H)
#pragma unroll
        for (int i = 0; i < RT * TT; i++) *place(wave, i) += sum[i / TT][i % TT];
    __syncthreads();
    for (int i = wave; i < RT * TT; i += kWaves) {
        f4 y = *place(0, i);
#pragma unroll
        for (int w = 1; w < H; w++) y += *place(w, i);
        const int t = t0 + i % TT * 16 + col;
        if (t < min(a.tokens, t0 + 4 * XL)) store_four<T>(a, t, (tile0 + i / TT) * 16 + g * 4, y);
    }
}

// The same with a barrier, behind which the workgroup's LDS reads are done too. (__syncthreads
// would wait for all loads.)
template <int N>
__device__ void barrier_after_loads() {
    static_assert(N < 64, "");
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | (N >> 4) << 14);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// More tokens, with too few tiles of 256 by 128. 16 RT WN rows and 16 TT tokens a workgroup,
// of KS groups of WN waves, group n with every KS-th step of 128 columns from n on. A wave
// has its weights in registers, converted once for all of its tokens; a step of x is in LDS for
// its group, loaded there directly, S - 1 of the group's steps ahead. Chunk c (of eight
// elements) of row t lies at c ^ (t mod 16). Bound by the loads' latency and LDS.
template <typename T, int WN, int RT, int TT, int S, int KS>
__global__ __launch_bounds__(64 * WN * KS, 2)
void tile_kernel(Linear4Args a) {
    using V = vec8<T>;
    constexpr int BT = 16 * TT, LB = BT * kTileCols * 2;
    constexpr int NL = LB / 1024 / WN;  // loads of a wave for a step
    // objects of their own, so that the compiler sees which loads a read has to wait for
    static_assert(S == 3 || S == 4, "");
    __shared__ __attribute__((aligned(16))) char x0[KS * LB], x1[KS * LB], x2[KS * LB],
        x3[S > 3 ? KS * LB : 16];
    const int lane = threadIdx.x & 63;
    const int all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave = all % WN, group = all / WN;
    const int col = lane & 15, g = lane >> 4;
    const Place at = place_of(a, (a.tiles_n + RT * WN - 1) / (RT * WN));
    const int tile0 = (at.n * WN + wave) * RT, t0 = at.t * BT;
    const char *codes[RT], *scales[RT];
#pragma unroll
    for (int i = 0; i < RT; i++) {  // (of tiles that there are not, the last one's)
        const int64_t tile = min(tile0 + i, a.tiles_n - 1);
        codes[i] = a.codes + tile * a.tiles_k * 1024;
        scales[i] = a.scales + tile * a.tiles_k * 64;
    }
    // load i of a wave: four rows, 16 lanes each (offsets fit 32 bits: 128 rows of 2^25 bytes)
    const int lrow = lane >> 4, lch = lane & 15;
    const char *x_rows = (const char *)((const T *)a.x + t0 * a.x_stride);
    auto chunk = [&](int i) { return lch ^ (((wave * NL + i) * 4 + lrow) & 15); };
    uint32_t from[NL];
#pragma unroll
    for (int i = 0; i < NL; i++)
        from[i] = (uint32_t)min((wave * NL + i) * 4 + lrow, a.tokens - 1 - t0) *
                      (uint32_t)(a.x_stride * 2) + chunk(i) * 16;
    u4 c[S][RT];
    uint32_t sc[S][RT];
    auto buffer = [&](int st) {
        return (st == 0 ? x0 : st == 1 ? x1 : st == 2 ? x2 : x3) + (KS > 1 ? group * LB : 0);
    };
    const int whole = a.blocks / 4 / KS;  // steps of whole tiles
    // (END: the tile may end beyond the rows)
    auto issue = [&](auto stage, auto end, int n) {
        constexpr int st = decltype(stage)::value;
        const int tk = n * KS + group;
        if (decltype(end)::value && tk >= a.tiles_k) return;
#pragma unroll
        for (int i = 0; i < RT; i++) {
            c[st][i] = *(const u4 *)(codes[i] + tk * 1024ll + (uint32_t)lane * 16);
            sc[st][i] = *(const uint32_t *)(scales[i] + tk * 64ll + (uint32_t)col * 4);
        }
        const char *rows = x_rows + tk * 256ll;
#pragma unroll
        for (int i = 0; i < NL; i++) {
            uint32_t at = from[i];
            if constexpr (decltype(end)::value) {
                // past the end: this step's first chunk, cleared when it is there
                if (tk * 4 + chunk(i) / 4 >= a.blocks) at -= chunk(i) * 16;
            }
            load_to_lds((Global)rows + at, buffer(st) + (wave * NL + i) * 1024);
        }
    };
    f4 sum[RT][TT];
#pragma unroll
    for (int i = 0; i < RT; i++)
#pragma unroll
        for (int j = 0; j < TT; j++) sum[i][j] = f4{0, 0, 0, 0};
    auto products = [&](auto stage) {
        constexpr int st = decltype(stage)::value;
        const char *x = buffer(st);
#pragma unroll
        for (int k = 0; k < 4; k++) {
            V w[RT];
#pragma unroll
            for (int i = 0; i < RT; i++)
                w[i] = values_of<T>(c[st][i][k], scale_of(sc[st][i] >> (8 * k) & 255));
#pragma unroll
            for (int j = 0; j < TT; j++) {
                const V b = *(const V *)(x + (j * 16 + col) * 256 + ((k * 4 + g) ^ col) * 16);
#pragma unroll
                for (int i = 0; i < RT; i++) sum[i][j] = mfma16(w[i], b, sum[i][j]);
            }
        }
    };
    // A step in the middle: whole tiles, the S - 2 after it under way. (Their loads of x alone
    // are counted: a step's weights are asked for before its x.)
    auto middle = [&](auto stage, int n) {
        constexpr int st = decltype(stage)::value;
        barrier_after_loads<(S - 2) * NL>();
        issue(Const<(st + S - 1) % S>{}, Const<0>{}, n + S - 1);
        products(stage);
    };
    const int steps = (a.tiles_k + KS - 1) / KS;
    auto last = [&](auto stage, int n) {
        constexpr int st = decltype(stage)::value;
        if (n >= steps) return;
        const int tk = n * KS + group;
        __builtin_amdgcn_s_waitcnt(kWaitLoads);
        if ((tk + 1) * 4 > a.blocks)
#pragma unroll
            for (int i = 0; i < NL; i++) {
                if (tk * 4 + chunk(i) / 4 >= a.blocks)
                    *(u4 *)(buffer(st) + (wave * NL + i) * 1024 + lane * 16) = u4{0, 0, 0, 0};
            }
        __syncthreads();
        issue(Const<(st + S - 1) % S>{}, Const<1>{}, n + S - 1);
        if (tk < a.tiles_k) products(stage);
    };
    auto each = [&](auto &step, int n) {
        step(Const<0>{}, n);
        step(Const<1>{}, n + 1);
        step(Const<2>{}, n + 2);
        if constexpr (S > 3) step(Const<3>{}, n + 3);
    };
    int n = 0;
    if (whole >= 2 * S - 1) {
        issue(Const<0>{}, Const<0>{}, 0);
        issue(Const<1>{}, Const<0>{}, 1);
        if constexpr (S > 3) issue(Const<2>{}, Const<0>{}, 2);
        do {
            each(middle, n);
            n += S;
        } while (n + 2 * S - 1 <= whole);
    } else {
        issue(Const<0>{}, Const<1>{}, 0);
        issue(Const<1>{}, Const<1>{}, 1);
        if constexpr (S > 3) issue(Const<2>{}, Const<1>{}, 2);
    }
    for (; n < steps; n += S) each(last, n);
    if constexpr (KS > 1) {  // the groups' sums are added to the first's, in order
        static_assert((KS - 1) * WN * RT * TT * 1024 <= KS * LB, "");
        auto place = [&](int group) {
            return (f4 *)(x0 + ((group - 1) * WN + wave) * RT * TT * 1024) + lane;
        };
        __syncthreads();
        if (group)
#pragma unroll
            for (int i = 0; i < RT; i++)
#pragma unroll
                for (int j = 0; j < TT; j++) place(group)[(i * TT + j) * 64] = sum[i][j];
        __syncthreads();
        if (group) return;
#pragma unroll
        for (int k = 1; k < KS; k++)
#pragma unroll
            for (int i = 0; i < RT; i++)
#pragma unroll
                for (int j = 0; j < TT; j++) sum[i][j] += place(k)[(i * TT + j) * 64];
    }
#pragma unroll
    for (int j = 0; j < TT; j++) {
        const int t = t0 + j * 16 + col;
        if (t >= a.tokens) break;
#pragma unroll
        for (int i = 0; i < RT; i++) store_four<T>(a, t, (tile0 + i) * 16 + g * 4, sum[i][j]);
    }
}

template <typename T, int WN, int RT, int TT, int S, int KS>
hipError_t launch_tile(const Linear4Args &a, hipStream_t s) {
    Linear4Args copy = a;
    void *args[] = {&copy};
    constexpr int BN = RT * WN, BT = 16 * TT;
    const dim3 grid((uint32_t)((a.tiles_n + BN - 1) / BN) * ((a.tokens + BT - 1) / BT));
    return hipLaunchKernel((const void *)tile_kernel<T, WN, RT, TT, S, KS>, grid,
                           dim3(64 * WN * KS), args, 0, s);
}
// Many tokens: bound by the matrix unit. 256 rows and 128 tokens a workgroup, all tokens to
// each of four waves with 64 rows, so that an operand from LDS goes into four products. As
// above, with a step of x in LDS one step ahead: a step's 128 products a wave last longer than
// its loads. (8192 tokens, 6144 x 4096: 297 us, 1390 TFLOP/s; 128 by 128 a workgroup, 32 rows to
// a wave, 340.)
constexpr int kBigRows = 256, kBigTokens = 128;
template <typename T>
__global__ __launch_bounds__(256, 2) void big_kernel(Linear4Args a) {
    using V = vec8<T>;
    constexpr int RT = kBigRows / 64, TT = kBigTokens / 16;
    constexpr int LB = kBigTokens * kTileCols * 2, NL = LB / 4096;
    __shared__ __attribute__((aligned(16))) char x0[LB], x1[LB];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    const Place at = place_of(a, (a.rows + kBigRows - 1) / kBigRows);
    const int tile0 = at.n * (kBigRows / 16) + wave * RT, t0 = at.t * kBigTokens;
    const char *codes[RT], *scales[RT];
#pragma unroll
    for (int i = 0; i < RT; i++) {  // (of tiles that there are not, the last one's)
        const int64_t tile = min(tile0 + i, a.tiles_n - 1);
        codes[i] = a.codes + tile * a.tiles_k * 1024;
        scales[i] = a.scales + tile * a.tiles_k * 64;
    }
    // load i of a wave: four rows, 16 lanes each (offsets fit 32 bits: 128 rows of 2^25 bytes)
    const int lrow = lane >> 4, lch = lane & 15;
    const char *x_rows = (const char *)((const T *)a.x + t0 * a.x_stride);
    auto chunk = [&](int i) { return lch ^ (((wave * NL + i) * 4 + lrow) & 15); };
    uint32_t from[NL];
#pragma unroll
    for (int i = 0; i < NL; i++)
        from[i] = (uint32_t)min((wave * NL + i) * 4 + lrow, a.tokens - 1 - t0) *
                      (uint32_t)(a.x_stride * 2) + chunk(i) * 16;
    auto load_x = [&](char *to, int tk) {
        const bool end = (tk + 1) * 4 > a.blocks;
        const char *rows = x_rows + tk * 256ll;
#pragma unroll
        for (int i = 0; i < NL; i++) {
            uint32_t at = from[i];
            // past the end: this step's first chunk, cleared when it is there
            if (end && tk * 4 + chunk(i) / 4 >= a.blocks) at -= chunk(i) * 16;
            load_to_lds((Global)rows + at, to + (wave * NL + i) * 1024);
        }
    };
    auto arrive = [&](char *to, int tk) {
        __builtin_amdgcn_s_waitcnt(kWaitLoads);
        if ((tk + 1) * 4 > a.blocks)
#pragma unroll
            for (int i = 0; i < NL; i++)
                if (tk * 4 + chunk(i) / 4 >= a.blocks)
                    *(u4 *)(to + (wave * NL + i) * 1024 + lane * 16) = u4{0, 0, 0, 0};
        __syncthreads();
    };
    u4 c[RT], next_c[RT];
    uint32_t sc[RT], next_sc[RT];
    auto load_w = [&](int tk) {
        tk = min(tk, a.tiles_k - 1);
#pragma unroll
        for (int i = 0; i < RT; i++) {
            next_c[i] = *(const u4 *)(codes[i] + tk * 1024ll + (uint32_t)lane * 16);
            next_sc[i] = *(const uint32_t *)(scales[i] + tk * 64ll + (uint32_t)col * 4);
        }
    };
    f4 sum[RT][TT];
#pragma unroll
    for (int i = 0; i < RT; i++)
#pragma unroll
        for (int j = 0; j < TT; j++) sum[i][j] = f4{0, 0, 0, 0};
    auto step = [&](const char *x, char *next, int tk) {
#pragma unroll
        for (int i = 0; i < RT; i++) c[i] = next_c[i], sc[i] = next_sc[i];
        if (tk + 1 < a.tiles_k) load_x(next, tk + 1);
        load_w(tk + 1);
#pragma unroll
        for (int k = 0; k < 4; k++) {
            V b[TT];
#pragma unroll
            for (int j = 0; j < TT; j++)
                b[j] = *(const V *)(x + (j * 16 + col) * 256 + ((k * 4 + g) ^ col) * 16);
#pragma unroll
            for (int i = 0; i < RT; i++) {
                const V w = values_of<T>(c[i][k], scale_of(sc[i] >> (8 * k) & 255));
#pragma unroll
                for (int j = 0; j < TT; j++) sum[i][j] = mfma16(w, b[j], sum[i][j]);
            }
        }
        if (tk + 1 < a.tiles_k) arrive(next, tk + 1);
    };
    load_x(x0, 0);
    load_w(0);
    arrive(x0, 0);
    for (int tk = 0; tk < a.tiles_k; tk += 2) {
        step(x0, x1, tk);
        if (tk + 1 < a.tiles_k) step(x1, x0, tk + 1);
    }
#pragma unroll
    for (int j = 0; j < TT; j++) {
        const int t = t0 + j * 16 + col;
        if (t >= a.tokens) break;
#pragma unroll
        for (int i = 0; i < RT; i++) store_four<T>(a, t, (tile0 + i) * 16 + g * 4, sum[i][j]);
    }
}

template <typename T, int RT, int XL, int NB>
hipError_t launch_stream(const Linear4Args &a, hipStream_t s) {
    Linear4Args copy = a;
    void *args[] = {&copy};
    const dim3 grid((uint32_t)((a.tiles_n + RT - 1) / RT) * ((a.tokens + 4 * XL - 1) / (4 * XL)));
    return hipLaunchKernel((const void *)stream_kernel<T, RT, XL, NB>, grid, dim3(64 * kWaves),
                           args, 0, s);
}

// The kernels, by number: rows and tokens of a workgroup; tiles: the waves of a group, the steps
// in LDS and the groups; stream: the halves of a tile in LDS; and for more than 16 tokens the
// times measured with 1024 to 16384 columns, us: a first part, one for every round of 256
// workgroups (one a compute unit) and one for every round and 1024 columns; but no less than one
// workgroup takes for its columns, where two on a compute unit hide one another's waits.
enum Kind { kStream, kTile, kBig };
struct Kernel {
    Kind kind;
    int rows, tokens, waves, ahead, groups;
    float base, round, columns, alone;
};
constexpr int kFew = 5;  // for up to 16 tokens
constexpr Kernel kKernels[] = {
    {kStream, 16, 8, 0, 4, 0, 0, 0, 0, 0},
    {kStream, 32, 8, 0, 4, 0, 0, 0, 0, 0},
    {kStream, 16, 16, 0, 2, 0, 0, 0, 0, 0},
    {kStream, 32, 16, 0, 4, 0, 0, 0, 0, 0},
    {kStream, 64, 16, 0, 4, 0, 0, 0, 0, 0},
    // 4096 columns: 32 tokens, 4096 rows 6.0 (the next 6.8)
    {kStream, 16, 32, 0, 2, 0, 2.1f, 0.3f, 0.9f, 0},
    // 32 tokens, 8192 rows 8.1 (10.0 and 10.0); 64 tokens, 4096 rows, 8192 columns 11.5 (15.7)
    {kStream, 32, 32, 0, 2, 0, 3.0f, 0, 1.24f, 0},
    // 128 tokens, 4096 rows 9.2 (11.5, 12.4, 10.5)
    {kStream, 64, 32, 0, 4, 0, 0.5f, 2.2f, 1.75f, 0},
    // 64 tokens, 16384 rows 15.3 (20.7, 16.6)
    {kStream, 64, 64, 0, 2, 0, 1.5f, 3, 2.5f, 0},
    // 32 tokens, 32768 rows 19.3 (21.1, 23.7)
    {kTile, 64, 32, 4, 4, 2, 3.2f, 0.2f, 1.75f, 0},
    // 256 tokens, 8192 rows 21.3 (27.1, 32.3)
    {kTile, 128, 64, 4, 4, 2, 1.5f, 4, 3.45f, 0},
    // 1024 tokens, 4096 rows 34.4 (39.2, 40.5); three stages in LDS instead of four 36.0
    {kTile, 128, 64, 4, 4, 1, 3.5f, 0, 3.85f, 4.9f},
    // 2048 tokens, 4096 rows 57.5 (65.3, 81.5)
    {kTile, 256, 64, 8, 3, 1, 4.5f, 0, 6.6f, 10.3f},
    // 1024 tokens, 16384 rows 97.8 (109.8)
    {kBig, kBigRows, kBigTokens, 0, 0, 0, 3, 0, 11.9f, 19.5f}};
constexpr int kNumber = sizeof(kKernels) / sizeof(Kernel);
static_assert(kNumber == TAS_FP4_LINEAR_KERNELS, "");

// Up to 16 tokens. (4096 columns, one token: 4096 rows 4.3 us with 16 rows and 8 tokens, 5.2 with
// 32 rows, 4.5 with 16 tokens; 16384 rows 9.0 with 32 rows, 9.7 with 64; 32768 14.7, 16.9. 16
// tokens: 4096 rows 4.7 with 16 rows, 5.9 with 32; 6144 rows 7.3, 6.3; 16384 rows 10.6 with 32
// rows, 9.7 with 64; 32768 rows 17.8, 17.2, but of 8192 columns 32.2, 38.6: with 64 rows a compute
// unit has one workgroup, and a wave's second unit of columns waits. With the other of two and
// four halves in LDS: 4 to 8 % longer, or as long.)
int choose_few(const Linear4Args &a) {
    if (a.tokens <= 8) return a.tiles_n <= 256 ? 0 : 1;
    if (a.tiles_n <= 256) return 2;
    return a.tiles_n < 1024 || a.tiles_k > 4 * kWaves ? 3 : 4;
}
// More: the kernel that takes least.
int choose(const Linear4Args &a) {
    if (a.tokens <= 16) return choose_few(a);
    int best = 0;
    float least = 0;
    const float columns = (float)a.blocks / 32;
    for (int i = kFew; i < kNumber; i++) {
        const Kernel &t = kKernels[i];
        const int64_t groups = (int64_t)((a.rows + t.rows - 1) / t.rows) *
                               ((a.tokens + t.tokens - 1) / t.tokens);
        const float rounds = (float)((groups + 255) / 256);
        const float us = fmaxf(t.base + rounds * (t.round + t.columns * columns),
                               t.alone * columns);
        if (i == kFew || us < least) best = i, least = us;
    }
    return best;
}

template <typename T, int N>
hipError_t launch_number(const Linear4Args &a, hipStream_t s) {
    constexpr Kernel k = kKernels[N];
    if constexpr (k.kind == kStream)
        return launch_stream<T, k.rows / 16, k.tokens / 4, k.ahead>(a, s);
    else if constexpr (k.kind == kTile)
        return launch_tile<T, k.waves, k.rows / 16 / k.waves, k.tokens / 16, k.ahead, k.groups>(a, s);
    else
        return launch_kernel(big_kernel<T>, (int64_t)((a.rows + kBigRows - 1) / kBigRows) *
                                                ((a.tokens + kBigTokens - 1) / kBigTokens),
                             a, s);
}
template <typename T, int... N>
hipError_t launch(const Linear4Args &a, hipStream_t s, std::integer_sequence<int, N...>) {
    constexpr hipError_t (*launchers[])(const Linear4Args &, hipStream_t) = {launch_number<T, N>...};
    return launchers[choose(a)](a, s);
}

}  // namespace

hipError_t launch_linear4(const Linear4Args &a, int dtype, hipStream_t s) {
    constexpr std::make_integer_sequence<int, kNumber> all;
    return dtype == TAS_F16 ? launch<_Float16>(a, s, all) : launch<__bf16>(a, s, all);
}
int linear4_kernel(const Linear4Args &a) { return choose(a); }

}  // namespace tas_step_impl
