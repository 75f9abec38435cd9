// tas_fp4_linear.hip - products of a step's tokens with weights in four bits.
//
// y[t][n] = sum over k of x[t][k] W[n][k], with W's values exact in the 16-bit type (a
// conversion of two elements an instruction), sums in 32 bits, rounded once. The transposed
// product Y^T = W X^T leaves four adjacent n of a token in a lane. The left operand is a
// tile of W as it lies in memory, one load of adjacent 16 bytes a lane, four products of a
// block each.
#include <hip/hip_runtime.h>

#include "tas_fp4_convert.h"
#include "tas_fp4_internal.h"

namespace tas_step_impl {
namespace {

typedef float f4 __attribute__((ext_vector_type(4)));

__device__ f4 mfma16(vec8<__bf16> a, vec8<__bf16> b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ f4 mfma16(vec8<_Float16> a, vec8<_Float16> b, f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

constexpr int kWaves = 8;

template <int N>
struct Const {
    static constexpr int value = N;
};

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

// Up to 16 tokens: bound by the weights' bytes. A workgroup has all of K for 16 RT rows, its
// eight waves take every eighth unit of 512 columns, and their sums are joined in LDS, in one
// order: no partial results in memory, no second launch. All of a unit's weights are asked
// for at once.
template <typename T, int RT>
__global__ __launch_bounds__(64 * kWaves) void stream_kernel(Linear4Args a) {
    using V = vec8<T>;
    constexpr int H = kWaves / 2;
    __shared__ f4 part[H][RT][64];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, g = lane >> 4;
    const int tile0 = blockIdx.x * RT;
    const char *codes[RT], *scales[RT];
#pragma unroll
    for (int i = 0; i < RT; i++) {  // (of tiles that there are not, the last one's)
        const int64_t tile = min(tile0 + i, a.tiles_n - 1);
        codes[i] = a.codes + tile * a.tiles_k * 1024;
        scales[i] = a.scales + tile * a.tiles_k * 64;
    }
    const T *x = (const T *)a.x + min(col, a.tokens - 1) * a.x_stride + g * 8;
    f4 sum[RT];
#pragma unroll
    for (int i = 0; i < RT; i++) sum[i] = f4{0, 0, 0, 0};
    auto unit = [&](auto whole, int u) {
        uint32_t sc[4][RT];
        u4 c[4][RT];
#pragma unroll
        for (int n = 0; n < 4; n++) {
            const int64_t tk = decltype(whole)::value ? u * 4 + n : min(u * 4 + n, a.tiles_k - 1);
#pragma unroll
            for (int i = 0; i < RT; i++) {
                c[n][i] = __builtin_nontemporal_load(
                    (const u4 *)(codes[i] + tk * 1024 + (uint32_t)lane * 16));
                sc[n][i] = *(const uint32_t *)(scales[i] + tk * 64 + (uint32_t)col * 4);
            }
        }
#pragma unroll
        for (int n = 0; n < 4; n++) {
            const int tk = u * 4 + n;
            // (not the last tile again: an infinity in it, times zero, is NaN)
            if (!decltype(whole)::value && tk >= a.tiles_k) break;
            V b[4];
#pragma unroll
            for (int k = 0; k < 4; k++)
                // blocks beyond the matrix: x is zero there, whatever lies behind it
                b[k] = decltype(whole)::value || tk * 4 + k < a.blocks
                           ? *(const V *)(x + tk * kTileCols + k * 32) : V{};
#pragma unroll
            for (int i = 0; i < RT; i++)
#pragma unroll
                for (int k = 0; k < 4; k++)
                    sum[i] = mfma16(values_of<T>(c[n][i][k], scale_of(sc[n][i] >> (8 * k) & 255)),
                                    b[k], sum[i]);
        }
    };
    const int whole = a.blocks / 16;
    int u = wave;
    for (; u < whole; u += kWaves) unit(Const<1>{}, u);
    if (u * 4 < a.tiles_k) unit(Const<0>{}, u);
    // the second half's sums are added to the first's, then those to one another
    if (wave >= H)
#pragma unroll
        for (int i = 0; i < RT; i++) part[wave - H][i][lane] = sum[i];
    __syncthreads();
    if (wave < H)
#pragma unroll
        for (int i = 0; i < RT; i++) part[wave][i][lane] += sum[i];
    __syncthreads();
    for (int i = wave; i < RT; i += kWaves) {
        f4 y = part[0][i][lane];
#pragma unroll
        for (int w = 1; w < H; w++) y += part[w][i][lane];
        if (col < a.tokens) store_four<T>(a, col, (tile0 + i) * 16 + g * 4, y);
    }
}

typedef const __attribute__((address_space(1))) char *Global;
__device__ void load_to_lds(Global from, char *to) {
    __builtin_amdgcn_global_load_lds(from, (__attribute__((address_space(3))) void *)to, 16, 0,
                                     0);
}
constexpr int kWaitLoads = 0x0F70;  // s_waitcnt: no load or store outstanding

// A barrier behind which the workgroup's LDS reads and all but the wave's last N loads are
// done. (__syncthreads would wait for all of them. The empty statements keep the compiler from
// moving memory accesses across, the others from working out scales that have not arrived.)
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

// More tokens, with too few tiles of 256 by 128. 16 RT WN rows and 16 TT WT tokens a workgroup,
// of KS groups of WN by WT waves, group n with every KS-th step of 128 columns from n on. A wave
// has its weights in registers, converted once for all of its tokens; a step of x is in LDS for
// its group, loaded there directly, S - 1 of the group's steps ahead. Chunk c (of eight
// elements) of row t lies at c ^ (t mod 16), which spreads the rows of a column over the banks.
// Bound by the loads' latency and LDS.
template <typename T, int WN, int WT, int RT, int TT, int S, int KS>
__global__ __launch_bounds__(64 * WN * WT * KS, (WN * WT * KS > 8 ? WN * WT * KS / 4 : 2))
void tile_kernel(Linear4Args a) {
    using V = vec8<T>;
    constexpr int W = WN * WT, BT = 16 * TT * WT, LB = BT * kTileCols * 2;
    constexpr int NL = LB / 1024 / W;  // loads of a wave for a step
    // objects of their own, so that the compiler sees which loads a read has to wait for
    static_assert(S == 3 || S == 4, "");
    __shared__ __attribute__((aligned(16))) char x0[KS * LB], x1[KS * LB], x2[KS * LB],
        x3[S > 3 ? KS * LB : 16];
    const int lane = threadIdx.x & 63;
    const int all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave = all % W, group = all / W;
    const int wn = wave % WN, wt = wave / WN;
    const int col = lane & 15, g = lane >> 4;
    const uint32_t groups_n = (a.tiles_n + RT * WN - 1) / (RT * WN);
    const uint32_t at_t = blockIdx.x / groups_n;
    const int tile0 = ((blockIdx.x - at_t * groups_n) * WN + wn) * RT;
    const int t0 = at_t * BT;
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
        const char *x = buffer(st) + wt * TT * 16 * 256;
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
    issue(Const<0>{}, Const<1>{}, 0);
    issue(Const<1>{}, Const<1>{}, 1);
    if constexpr (S > 3) issue(Const<2>{}, Const<1>{}, 2);
    int n = 0;
    for (; n + 2 * S - 1 <= whole; n += S) each(middle, n);
    for (; n < steps; n += S) each(last, n);
    if constexpr (KS > 1) {  // the groups' sums are added to the first's, in order
        static_assert((KS - 1) * W * RT * TT * 1024 <= KS * LB, "");
        auto place = [&](int group) {
            return (f4 *)(x0 + ((group - 1) * W + wave) * RT * TT * 1024) + lane;
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
        const int t = t0 + (wt * TT + j) * 16 + col;
        if (t >= a.tokens) break;
#pragma unroll
        for (int i = 0; i < RT; i++) store_four<T>(a, t, (tile0 + i) * 16 + g * 4, sum[i][j]);
    }
}

template <typename T, int WN, int WT, int RT, int TT, int S, int KS>
hipError_t launch_tile(const Linear4Args &a, hipStream_t s) {
    Linear4Args copy = a;
    void *args[] = {&copy};
    constexpr int BN = RT * WN, BT = 16 * TT * WT;
    const dim3 grid((uint32_t)((a.tiles_n + BN - 1) / BN) * ((a.tokens + BT - 1) / BT));
    return hipLaunchKernel((const void *)tile_kernel<T, WN, WT, RT, TT, S, KS>, grid,
                           dim3(64 * WN * WT * KS), args, 0, s);
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
    const uint32_t groups_n = (a.rows + kBigRows - 1) / kBigRows, at_t = blockIdx.x / groups_n;
    const int tile0 = (blockIdx.x - at_t * groups_n) * (kBigRows / 16) + wave * RT;
    const int t0 = at_t * kBigTokens;
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

template <typename T, int RT>
hipError_t launch_stream(const Linear4Args &a, hipStream_t s) {
    Linear4Args copy = a;
    void *args[] = {&copy};
    return hipLaunchKernel((const void *)stream_kernel<T, RT>, dim3((a.tiles_n + RT - 1) / RT),
                           dim3(64 * kWaves), args, 0, s);
}

// Up to 16 tokens. (4096 columns, one token: 4096 rows 4.4 us with RT 1, 5.2 with 2; 16384 rows
// 10.2, 9.2, and 11.7 with 4. 16 tokens: 4096 rows 6.8, 7.6, 9.7; 8192 rows 10.9, 8.7, 10.2;
// 32768 rows 34.7, 22.2, 19.2.)
template <typename T>
hipError_t launch_few(const Linear4Args &a, hipStream_t s) {
    if (a.tiles_n <= 256) return launch_stream<T, 1>(a, s);
    if (a.tiles_n < 1024 || a.tokens <= 8) return launch_stream<T, 2>(a, s);
    return launch_stream<T, 4>(a, s);
}

// More: the tile whose rounds of 256 workgroups (one a compute unit) take least, by the times
// measured with 4096 columns, us: a first part and one for every round, but no less than a
// compute unit takes for one alone.
struct TileCost {
    int rows, tokens;
    float base, round, least;
};
constexpr TileCost kTiles[] = {
    {32, 32, 2, 7, 9},                         // 64 tokens, 4096 rows: 8.9 (the next 11.0)
    {64, 32, 4, 7, 11},                        // 128 tokens, 4096 rows: 11.2 (14.6, 19.4)
    {128, 64, 1, 19, 20},                      // 256 tokens, 8192 rows: 22.4 (26.9, 32.4)
    {128, 64, 8, 13.4, 31},                    // 1024 tokens, 4096 rows: 34.8 (40.5, 75.6)
    {kBigRows, kBigTokens, 0, 49.5, 78}};      // 4096 tokens, 4096 rows: 100 (118)
int choose_tile(const Linear4Args &a) {
    int best = 0;
    float least = 0;
    for (int i = 0; i < 5; i++) {
        const TileCost &t = kTiles[i];
        const int64_t groups = (int64_t)((a.rows + t.rows - 1) / t.rows) *
                               ((a.tokens + t.tokens - 1) / t.tokens);
        const float us = fmaxf(t.base + t.round * (float)((groups + 255) / 256), t.least);
        if (!i || us < least) best = i, least = us;
    }
    return best;
}

template <typename T>
hipError_t launch(const Linear4Args &a, hipStream_t s) {
    if (a.tokens <= 16) return launch_few<T>(a, s);
    switch (choose_tile(a)) {
        case 0: return launch_tile<T, 2, 1, 1, 2, 4, 4>(a, s);
        case 1: return launch_tile<T, 4, 1, 1, 2, 4, 2>(a, s);
        case 2: return launch_tile<T, 4, 1, 2, 4, 4, 2>(a, s);
        case 3: return launch_tile<T, 4, 1, 2, 4, 3, 1>(a, s);
        default:
            return launch_kernel(big_kernel<T>, (int64_t)((a.rows + kBigRows - 1) / kBigRows) *
                                                    ((a.tokens + kBigTokens - 1) / kBigTokens),
                                 a, s);
    }
}

}  // namespace

hipError_t launch_linear4(const Linear4Args &a, int dtype, hipStream_t s) {
    return dtype == TAS_F16 ? launch<_Float16>(a, s) : launch<__bf16>(a, s);
}

}  // namespace tas_step_impl
