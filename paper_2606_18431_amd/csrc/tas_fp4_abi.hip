// tas_fp4_abi.hip - host side of the C ABI declared in include/tas_fp4.h: checks of the
// arguments, and the launches.
#include <hip/hip_runtime.h>

#include <cmath>

#include "tas_fp4.h"
#include "tas_fp4_internal.h"
#include "tas_step_host.h"

using namespace tas_step_impl;

namespace {

// Places are compared in units of two bytes, which divide every row, stride and address.
int64_t place(const void *p) { return (int64_t)((uintptr_t)p / 2); }

Region region_of(const tas_rows &r, int64_t n0, int64_t n1, int64_t n2, int64_t row) {
    return {place(r.p), row / 2, {r.stride[0] / 2, r.stride[1] / 2, r.stride[2] / 2},
            {n0, n1, n2}};
}
// Rows of n tokens, stride and length in 16-bit elements.
Region tokens_of(const void *p, int64_t stride, int64_t row, int64_t n) {
    return {place(p), row, {stride, 0, 0}, {n, 1, 1}};
}
Region bytes_of(const void *p, int64_t bytes) {
    return {place(p), (bytes + 1) / 2, {0, 0, 0}, {1, 1, 1}};
}

struct CacheShape {
    int64_t n_blocks, kv_heads, block_tokens, head_dim;
};
CacheShape shape_of(const tas_step *s) {
    return {s->n_blocks, s->kv_heads, int64_t(1) << s->blk_shift, s->head_dim};
}
bool valid_rows4(const tas_rows &r, int64_t align) {
    if (!r.p || (uintptr_t)r.p % align) return false;
    for (int i = 0; i < 3; i++)
        if (r.stride[i] < 0 || r.stride[i] % align ||
            r.stride[i] > (i == 2 ? kMaxTokenStride : kMaxStride))
            return false;
    return true;
}
bool valid_cache4(const tas_cache_fp4 &c, int64_t head_dim) {
    return valid_rows4(c.k, 16) && valid_rows4(c.v, 16) &&
           valid_rows4(c.k_scale, head_dim / 32) && valid_rows4(c.v_scale, head_dim / 32);
}
struct CacheRegions {
    Region r[4];
    CacheRegions(const tas_cache_fp4 &c, const CacheShape &s) {
        const tas_rows *rows[4] = {&c.k, &c.v, &c.k_scale, &c.v_scale};
        for (int i = 0; i < 4; i++)
            r[i] = region_of(*rows[i], s.n_blocks, s.kv_heads, s.block_tokens,
                             s.head_dim / (i < 2 ? 2 : 32));
    }
    bool meets(const Region &x) const {
        Overlap overlap;
        for (const Region &y : r)
            if (overlap(x, y)) return true;
        return false;
    }
};
// No byte of the pool is in two places of it.
bool disjoint(const tas_cache_fp4 &c, const CacheShape &s, const CacheRegions &regions) {
    const tas_rows *rows[4] = {&c.k, &c.v, &c.k_scale, &c.v_scale};
    for (int i = 0; i < 4; i++) {
        if (!disjoint_slots(rows[i]->stride[0], rows[i]->stride[1], rows[i]->stride[2], s.n_blocks,
                            s.kv_heads, s.block_tokens, s.head_dim / (i < 2 ? 2 : 32)))
            return false;
        for (int j = 0; j < i; j++)
            if (Overlap()(regions.r[i], regions.r[j])) return false;
    }
    return true;
}
bool valid_dtype(int32_t dtype) { return dtype == TAS_F16 || dtype == TAS_BF16; }
int done(hipError_t e) { return e == hipSuccess ? TAS_OK : TAS_EHIP; }

// A tensor's rows, and what its sides have in common; the stride of a dimension of one says
// nothing.
bool valid_tensor(const tas_tensor_fp4 *from, tas_tensor_fp4 *a, int64_t &rows) {
    if (!from) return false;
    *a = *from;
    if (!valid_dtype(a->dtype) || a->reserved) return false;
    if (a->cols < 32 || a->cols % 32) return false;
    rows = 1;
    int64_t most = kMaxGroups * 256 * 8 / a->cols;  // (a thread has eight elements)
    for (int64_t n : a->n) {
        if (n < 0 || n > most) return false;
        rows *= n;
        if (n) most /= n;
    }
    if (!rows) return true;
    auto strides = [&](tas_rows &r, int64_t align) {
        if (!r.p || (uintptr_t)r.p % align) return false;
        for (int i = 0; i < 3; i++) {  // (places stay far below 2^63)
            if (a->n[i] == 1) r.stride[i] = 0;
            if (r.stride[i] < 0 || r.stride[i] % align ||
                r.stride[i] > (int64_t(1) << 50) / a->n[i])
                return false;
        }
        return true;
    };
    return strides(a->x, 16) && strides(a->codes, 4) && strides(a->scales, 1);
}
Tensor4Args tensor_args(const tas_tensor_fp4 *a, int64_t rows) {
    Tensor4Args k{};
    k.x = a->x;
    k.codes = a->codes;
    k.scales = a->scales;
    k.per_row = (uint32_t)(a->cols / 8);
    k.units = (uint32_t)(rows * (a->cols / 8));
    k.n1 = (uint32_t)a->n[1];
    k.n2 = (uint32_t)a->n[2];
    return k;
}
// (scales' rows may have any length and place: their units are bytes, as all the others are
// here then)
Region byte_region(const tas_rows &r, const int64_t (&n)[3], int64_t row) {
    return {(int64_t)(uintptr_t)r.p, row, {r.stride[0], r.stride[1], r.stride[2]},
            {n[0], n[1], n[2]}};
}

}  // namespace

extern "C" {

int tas_fp4_append(tas_step *s, const tas_append_fp4 *a, void *stream) {
    if (!s || !a || !s->appendable) return TAS_EINVAL;
    if (!s->ws) return TAS_ESTATE;
    const int64_t D = s->head_dim;
    if (!valid_dtype(a->dtype)) return TAS_EINVAL;
    if (a->rot_dim < 0 || a->rot_dim > D || a->rot_dim % 16) return TAS_EINVAL;
    if (a->interleaved != 0 && a->interleaved != 1) return TAS_EINVAL;
    if (!(a->eps >= 0) || std::isinf(a->eps)) return TAS_EINVAL;
    if (!a->q_weight != !a->k_weight) return TAS_EINVAL;
    if (a->q_weight && (!aligned16(a->q_weight) || !aligned16(a->k_weight))) return TAS_EINVAL;
    if (a->rot_dim &&
        (!aligned16(a->cos) || !aligned16(a->sin) || a->positions < s->max_pos))
        return TAS_EINVAL;
    if (!valid_cache4(a->cache, D)) return TAS_EINVAL;
    const CacheShape shape = shape_of(s);
    const CacheRegions cache(a->cache, shape);
    if (!disjoint(a->cache, shape, cache)) return TAS_EINVAL;
    const int64_t T = s->head.n_tok;
    if (T == 0) return TAS_OK;
    const int64_t in_row = (s->heads + 2 * s->kv_heads) * D, out_row = s->heads * D;
    if (!valid_rows(a->qkv, a->qkv_stride, in_row) ||
        !valid_rows(a->q_out, a->q_out_stride, out_row))
        return TAS_EINVAL;
    const Region in = tokens_of(a->qkv, a->qkv_stride, in_row, T);
    const Region out = tokens_of(a->q_out, a->q_out_stride, out_row, T);
    // (a token's row is read before it is written)
    const bool in_place = a->q_out == a->qkv && (a->q_out_stride == a->qkv_stride || T == 1);
    if (cache.meets(in) || cache.meets(out) || (!in_place && Overlap()(in, out)))
        return TAS_EINVAL;
    auto safe = [&](const Region &r) { return !cache.meets(r) && !Overlap()(r, out); };
    if (a->q_weight && !(safe(bytes_of(a->q_weight, D * 2)) && safe(bytes_of(a->k_weight, D * 2))))
        return TAS_EINVAL;
    if (a->rot_dim) {
        const int64_t bytes = s->max_pos * a->rot_dim * 2;
        if (!safe(bytes_of(a->cos, bytes)) || !safe(bytes_of(a->sin, bytes))) return TAS_EINVAL;
    }
    Append4Args k{};
    k.reqs = (const Req *)(s->ws + s->head.req);
    k.tok_req = (const int32_t *)(s->ws + s->head.tok_req);
    k.tables = (const int32_t *)(s->ws + s->head.tables);
    k.qkv = a->qkv;
    k.q_out = a->q_out;
    k.q_weight = a->q_weight;
    k.k_weight = a->k_weight;
    k.cos = a->cos;
    k.sin = a->sin;
    k.qkv_stride = a->qkv_stride;
    k.q_out_stride = a->q_out_stride;
    k.f = a->cache;
    k.n_tok = s->head.n_tok;
    k.heads = s->heads;
    k.kv_heads = s->kv_heads;
    k.rot = a->rot_dim;
    k.interleaved = a->interleaved;
    k.blk_shift = s->blk_shift;
    k.eps = a->eps;
    return done(launch_append4(k, a->dtype, s->head_dim, (hipStream_t)stream));
}

int tas_fp4_attention(tas_step *s, const tas_attention_fp4 *a, void *stream) {
    if (!s || !a) return TAS_EINVAL;
    if (!s->ws) return TAS_ESTATE;
    if (!valid_dtype(a->dtype)) return TAS_EINVAL;
    const float scale2 = a->scale * 1.4426950408889634f;
    if (!(a->scale > 0) || std::isinf(scale2)) return TAS_EINVAL;
    if (!valid_cache4(a->cache, s->head_dim)) return TAS_EINVAL;
    const int64_t T = s->head.n_tok;
    if (T == 0) return TAS_OK;
    const int64_t row = (int64_t)s->heads * s->head_dim;
    if (!valid_rows(a->q, a->q_stride, row) || !valid_rows(a->out, a->out_stride, row))
        return TAS_EINVAL;
    if ((uintptr_t)a->lse % 4) return TAS_EINVAL;
    const CacheRegions cache(a->cache, shape_of(s));
    const Region in = tokens_of(a->q, a->q_stride, row, T);
    const Region out = tokens_of(a->out, a->out_stride, row, T);
    // (an item reads its rows before it writes them, and no others)
    const bool in_place = a->out == a->q && (a->out_stride == a->q_stride || T == 1);
    if (cache.meets(out) || (!in_place && Overlap()(in, out))) return TAS_EINVAL;
    if (a->lse) {
        const Region lse = bytes_of(a->lse, T * s->heads * 4);
        if (cache.meets(lse) || Overlap()(lse, in) || Overlap()(lse, out)) return TAS_EINVAL;
    }
    Attn4Args k{};
    k.tables = (const int32_t *)(s->ws + s->head.tables);
    k.tok_own = (const Own *)(s->ws + s->head.tok_own);
    k.items = (const Item *)(s->ws + s->head.items);
    k.units = (const Unit *)(s->ws + s->head.units);
    k.merge = k.units + s->head.n_join;
    k.done = (uint32_t *)(s->ws + s->head.done);
    k.q = a->q;
    k.out = a->out;
    k.lse = a->lse;
    k.part_o = (float *)(s->ws + s->part_o());
    k.part_lse = (float *)(s->ws + s->part_lse());
    k.q_stride = a->q_stride;
    k.out_stride = a->out_stride;
    k.f = a->cache;
    k.group = s->heads / s->kv_heads;
    k.heads = s->heads;
    k.sub_shift = s->blk_shift - 4;
    k.scale2 = scale2;
    k.n_wide = s->head.n_wide;
    return done(launch_attention4(k, s->head.n_wide + s->head.n_thin, s->head.n_merge, a->dtype,
                                  s->head_dim, (hipStream_t)stream));
}

int tas_fp4_pack(const tas_tensor_fp4 *from, void *stream) {
    tas_tensor_fp4 tensor, *const a = &tensor;
    int64_t rows;
    if (!valid_tensor(from, a, rows)) return TAS_EINVAL;
    if (!rows) return TAS_OK;
    const int64_t(&n)[3] = a->n;
    const int64_t cb = a->cols / 2, sb = a->cols / 32;
    if (!disjoint_slots(a->codes.stride[0], a->codes.stride[1], a->codes.stride[2], n[0], n[1],
                        n[2], cb) ||
        !disjoint_slots(a->scales.stride[0], a->scales.stride[1], a->scales.stride[2], n[0], n[1],
                        n[2], sb))
        return TAS_EINVAL;
    const Region x = byte_region(a->x, n, a->cols * 2), codes = byte_region(a->codes, n, cb);
    const Region scales = byte_region(a->scales, n, sb);
    if (Overlap()(x, codes) || Overlap()(x, scales) || Overlap()(codes, scales)) return TAS_EINVAL;
    return done(launch_pack4(tensor_args(a, rows), a->dtype, (hipStream_t)stream));
}

// What a call that gives values refuses, besides; its kernel's arguments.
static bool values_args(const tas_tensor_fp4 *from, Tensor4Args &k, int64_t &rows) {
    tas_tensor_fp4 tensor, *const a = &tensor;
    if (!valid_tensor(from, a, rows)) return false;
    if (!rows) return true;
    const int64_t(&n)[3] = a->n;
    if (!disjoint_slots(a->x.stride[0], a->x.stride[1], a->x.stride[2], n[0], n[1], n[2],
                        a->cols * 2))
        return false;
    const Region x = byte_region(a->x, n, a->cols * 2);
    if (Overlap()(x, byte_region(a->codes, n, a->cols / 2)) ||
        Overlap()(x, byte_region(a->scales, n, a->cols / 32)))
        return false;
    k = tensor_args(a, rows);
    return true;
}

int tas_fp4_values(const tas_tensor_fp4 *a, void *stream) {
    Values4Args k{};
    int64_t rows;
    if (!values_args(a, k.t[0], rows)) return TAS_EINVAL;
    if (!rows) return TAS_OK;
    return done(launch_values4(k, 1, a->dtype, (hipStream_t)stream));
}

int tas_fp4_cache_values(const tas_cache_values_fp4 *a, void *stream) {
    if (!a || (a->head_dim != 64 && a->head_dim != 128)) return TAS_EINVAL;
    tas_tensor_fp4 t[2]{};
    Values4Args k{};
    int64_t rows = 0;
    for (int i = 0; i < 2; i++) {
        const int64_t row = a->head_dim * 2;
        t[i].dtype = a->dtype;
        t[i].n[0] = a->n_blocks;
        t[i].n[1] = a->kv_heads;
        t[i].n[2] = a->block_tokens;
        t[i].cols = a->head_dim;
        for (int64_t n : t[i].n)
            if (n < 0 || n > INT32_MAX) return TAS_EINVAL;
        if (a->kv_heads * a->block_tokens > INT32_MAX) return TAS_EINVAL;
        t[i].x = {i ? a->v : a->k,
                  {a->kv_heads * a->block_tokens * row, a->block_tokens * row, row}};
        t[i].codes = i ? a->cache.v : a->cache.k;
        t[i].scales = i ? a->cache.v_scale : a->cache.k_scale;
        if (!values_args(&t[i], k.t[i], rows)) return TAS_EINVAL;
    }
    if (!rows) return TAS_OK;
    for (int i = 0; i < 2; i++) {  // an output over the other tensor's sides
        const Region x = byte_region(t[i].x, t[i].n, t[i].cols * 2);
        const tas_tensor_fp4 &y = t[1 - i];
        if (Overlap()(x, byte_region(y.x, y.n, y.cols * 2)) ||
            Overlap()(x, byte_region(y.codes, y.n, y.cols / 2)) ||
            Overlap()(x, byte_region(y.scales, y.n, y.cols / 32)))
            return TAS_EINVAL;
    }
    return done(launch_values4(k, 2, a->dtype, (hipStream_t)stream));
}

static bool valid_matrix(int64_t rows, int64_t cols) {
    return rows >= 1 && rows <= (int64_t(1) << 24) && cols >= 32 && cols % 32 == 0 &&
           cols <= (int64_t(1) << 20);
}

size_t tas_fp4_weights_bytes(int64_t rows, int64_t cols) {
    if (!valid_matrix(rows, cols)) return 0;
    const WeightsShape w = weights_shape(rows, cols);
    return (w.tiles_n * w.tiles_k + 3) / 4 > kMaxGroups ? 0 : (size_t)w.bytes;
}

int tas_fp4_weights(int64_t rows, int64_t cols, const void *codes, int64_t codes_stride,
                    const void *scales, int64_t scales_stride, void *d_weights, void *stream) {
    const size_t bytes = tas_fp4_weights_bytes(rows, cols);
    if (!bytes || !aligned16(codes) || !scales || !d_weights || (uintptr_t)d_weights & 255)
        return TAS_EINVAL;
    const int64_t most = int64_t(1) << 31;
    if (codes_stride < 0 || codes_stride % 16 || codes_stride > most || scales_stride < 0 ||
        scales_stride > most)
        return TAS_EINVAL;
    const int64_t n[3] = {1, 1, rows}, one[3] = {1, 1, 1};
    const Region out = byte_region({d_weights, {0, 0, 0}}, one, (int64_t)bytes);
    if (Overlap()(out, byte_region({(void *)codes, {0, 0, codes_stride}}, n, cols / 2)) ||
        Overlap()(out, byte_region({(void *)scales, {0, 0, scales_stride}}, n, cols / 32)))
        return TAS_EINVAL;
    Weights4Args k{};
    k.codes = (const char *)codes;
    k.scales = (const char *)scales;
    k.out = (char *)d_weights;
    k.codes_stride = codes_stride;
    k.scales_stride = scales_stride;
    k.rows = rows;
    k.blocks = cols / 32;
    k.w = weights_shape(rows, cols);
    return done(launch_weights4(k, (hipStream_t)stream));
}

// The sizes of a product, of a matrix that there can be.
static bool valid_product(int64_t tokens, int64_t rows) {
    if (tokens < 0 || tokens > (int64_t(1) << 24)) return false;
    // (smaller tiles are not taken where there are many)
    return ceil_div(rows, 64) * ceil_div(tokens, 64) <= kMaxGroups / 8;
}
static Linear4Args linear_sizes(int64_t tokens, int64_t rows, int64_t cols) {
    const WeightsShape w = weights_shape(rows, cols);
    Linear4Args k{};
    k.tokens = (int32_t)tokens;
    k.rows = (int32_t)rows;
    k.blocks = (int32_t)(cols / 32);
    k.tiles_n = (int32_t)w.tiles_n;
    k.tiles_k = (int32_t)w.tiles_k;
    return k;
}

int tas_fp4_linear_kernel(int64_t tokens, int64_t rows, int64_t cols) {
    if (!tas_fp4_weights_bytes(rows, cols) || tokens < 1 || !valid_product(tokens, rows))
        return TAS_EINVAL;
    return linear4_kernel(linear_sizes(tokens, rows, cols));
}

int tas_fp4_linear(const tas_linear_fp4 *a, void *stream) {
    if (!a || !valid_dtype(a->dtype) || a->reserved) return TAS_EINVAL;
    const size_t bytes = tas_fp4_weights_bytes(a->rows, a->cols);
    if (!bytes || !a->weights || (uintptr_t)a->weights & 255) return TAS_EINVAL;
    if (!valid_product(a->tokens, a->rows)) return TAS_EINVAL;
    if (!a->tokens) return TAS_OK;
    if (!valid_rows(a->x, a->x_stride, a->cols) || a->x_stride > kMaxTokenStride)
        return TAS_EINVAL;
    if (!a->y || (uintptr_t)a->y % 2 || a->y_stride < a->rows ||
        a->y_stride >= int64_t(1) << 31)
        return TAS_EINVAL;
    const Region y = tokens_of(a->y, a->y_stride, a->rows, a->tokens);
    if (Overlap()(y, tokens_of(a->x, a->x_stride, a->cols, a->tokens)) ||
        Overlap()(y, bytes_of(a->weights, (int64_t)bytes)))
        return TAS_EINVAL;
    Linear4Args k = linear_sizes(a->tokens, a->rows, a->cols);
    k.x = a->x;
    k.codes = (const char *)a->weights;
    k.scales = (const char *)a->weights + weights_shape(a->rows, a->cols).scales_at;
    k.y = a->y;
    k.x_stride = a->x_stride;
    k.y_stride = a->y_stride;
    k.y_fours = a->rows % 4 == 0 && a->y_stride % 4 == 0 && (uintptr_t)a->y % 8 == 0;
    k.x_much = a->tokens / 4 > a->rows;  // (an element of x has four times the bits)
    return done(launch_linear4(k, a->dtype, (hipStream_t)stream));
}

}  // extern "C"
