// tas_step_host.h - a step as the host holds it, and the checks of arguments that the
// entry points share (host only).
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <vector>

#include "tas_step.h"
#include "tas_step_internal.h"
#include "tas_step_overlap.h"

namespace tas_step_impl {

constexpr int64_t kMaxStride = (int64_t(1) << 31) - 8;      // of a block or head, elements
constexpr int64_t kMaxTokenStride = int64_t(1) << 24;       // of a token in a block
constexpr int64_t kMaxGroups = (int64_t(1) << 24) - 1;      // of a launch: 2^32 threads

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

inline bool aligned16(const void *p) { return p && ((uintptr_t)p & 15) == 0; }

inline bool valid_cache(const tas_cache &c) {
    if (!aligned16(c.k) || !aligned16(c.v)) return false;
    const int64_t s[6] = {c.k_block, c.v_block, c.k_head, c.v_head, c.k_token, c.v_token};
    for (int i = 0; i < 6; i++) {
        if (s[i] < 0 || s[i] % 8) return false;
        if (s[i] > (i >= 4 ? kMaxTokenStride : kMaxStride)) return false;
    }
    return true;
}

// No two slots of K, or of V, share an element, so that the new tokens' writes do not
// race: in the order of the strides, each is at least what the shorter ones span.
inline bool disjoint_slots(int64_t block, int64_t head, int64_t token, int64_t n_blocks,
                           int64_t kv_heads, int64_t block_tokens, int64_t head_dim) {
    struct Axis {
        int64_t stride, n;
    } axes[3] = {{token, block_tokens}, {head, kv_heads}, {block, n_blocks}};
    std::sort(axes, axes + 3, [](const Axis &x, const Axis &y) { return x.stride < y.stride; });
    int64_t span = head_dim;
    for (const Axis &x : axes) {
        if (x.n == 1) continue;  // its stride says nothing
        if (x.stride < span) return false;
        span += (x.n - 1) * x.stride;
    }
    return true;
}

// The memory of one of a cache's tensors (aligned, strides in elements).
inline Region region_of(const void *p, int64_t block, int64_t head, int64_t token,
                        int64_t n_blocks, int64_t kv_heads, int64_t block_tokens,
                        int64_t head_dim) {
    return {(int64_t)((uintptr_t)p / 16), head_dim / 8, {block / 8, head / 8, token / 8},
            {n_blocks, kv_heads, block_tokens}};
}

// The rows of n_tok tokens (aligned, the stride in elements).
inline Region region_of(const void *p, int64_t stride, int64_t row, int64_t n_tok) {
    return {(int64_t)((uintptr_t)p / 16), row / 8, {stride / 8, 0, 0}, {n_tok, 1, 1}};
}

// Whether an output's rows are in memory that is read or written besides. They may be the
// input's own rows: a row is read before it is written.
inline bool clash(const void *out, int64_t out_stride, int64_t out_row, const void *in,
                  int64_t in_stride, int64_t in_row, int64_t n_tok, const Region &k,
                  const Region &v) {
    const Region o = region_of(out, out_stride, out_row, n_tok);
    Overlap overlap;
    const bool in_place = out == in && (out_stride == in_stride || n_tok == 1);
    return (!in_place && overlap(o, region_of(in, in_stride, in_row, n_tok))) || overlap(o, k) ||
           overlap(o, v);
}

inline bool valid_rows(const void *p, int64_t stride, int64_t row) {
    return aligned16(p) && stride >= row && stride % 8 == 0;
}

}  // namespace tas_step_impl

struct tas_step {
    std::vector<char> blob;  // the plan
    tas_step_impl::PlanHead head{};
    int32_t heads = 0, kv_heads = 0, head_dim = 0, blk_shift = 0, n_blocks = 0;
    int64_t max_pos = 0;
    bool appendable = false;
    char *ws = nullptr;  // null: not bound
    size_t part_o() const { return blob.size(); }
    size_t part_lse() const {
        return part_o() + tas_step_impl::align256((size_t)head.part_rows * head_dim * 4);
    }
    size_t bytes() const { return part_lse() + tas_step_impl::align256((size_t)head.part_rows * 4); }
};
