// tas_step_internal.h - the plan of a step as the host writes it and the
// kernels read it, and the launchers of the kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tas_step.h"

namespace tas_step_impl {

// Rows of a key head are (token, query head of its group), token-major. A
// segment is a run of tokens with one list of keys: a request with its own
// context, or a prefix group's tokens with the prefix.
constexpr int kThinRows = 16;   // rows of a thin item (all rows of its segment)
constexpr int kThinKeys = 32;   // keys of one wave's step
constexpr int kWideRows = 128;  // rows of a wide item
constexpr int kWideKeys = 64;   // keys of one step of a wide item
constexpr int kJoinRows = 16;   // rows of a join

struct Req {
    int32_t t0, n_new, kv_len, table;   // first token; pages at tables[table]
    int32_t prefix_len, own_seg, pre_seg, pad;  // segments, -1: none
};
struct Seg {
    int32_t t0, n_tok;    // tokens
    int32_t kv_len;       // keys
    int32_t lim0;         // token j sees the keys below min(kv_len, lim0 + j)
    int32_t table;        // pages at tables[table]
    int32_t nsplit;       // pieces of the keys, each with a partial result
    int32_t part;         // partial row of (key head 0, piece 0, row 0), -1: none,
                          // results go to the output
    int32_t rows;         // n_tok * heads / kv_heads
};
// Rows row0.. of one key head of a segment against its keys k0 .. k1 - 1. (The segment
// is held here, not pointed to: a workgroup's first loads wait for it.)
struct Item {
    Seg s;
    int32_t seg, hk, row0, k0, k1;
    int32_t part;  // partial row of row0, -1: output
    int32_t unit;  // the join that waits for this item, -1: none
    int32_t pad;
};
// Rows row0 .. row0 + rows - 1 of one key head of a segment, the results of which are
// partial ones; of a prefix's rows, the parts of the tokens' own segments too. Rows of
// a thin segment are joined by the last of the `items` items that have a part of them,
// those of a wide one by a second kernel.
struct Unit {
    Seg s;
    int32_t seg, hk, row0, rows, items, prefix, pad[2];
};
// Of a token under a prefix: where the parts of its own segment lie (nsplit 0: none).
struct Own {
    int32_t part, nsplit, rows, t0;
};
struct PlanHead {
    int64_t bytes;      // of the blob
    int64_t part_rows;  // partial rows
    int32_t n_req, n_tok, n_seg, n_thin, n_wide, n_join, n_merge, n_table;
    // byte offsets in the blob; the items as the workgroups take them; the units those of thin segments (join), then the others (merge); done holds a
    // counter for each of the first, zero between launches
    int64_t req, seg, items, units, tables, tok_req, tok_own, done;
};

struct AppendArgs {
    const Req *reqs;
    const int32_t *tok_req, *tables;
    const void *qkv;
    void *q_out;
    const void *q_weight, *k_weight;
    const float *cos, *sin;
    int64_t qkv_stride, q_out_stride;
    tas_cache c;
    int32_t n_tok, heads, kv_heads, rot, interleaved;
    int32_t blk_shift;  // log2(block_tokens)
    float eps;
};

constexpr int heads_of_wave(int head_dim) { return 1024 / head_dim; }  // 16 elements a lane
// Workgroups of an append: four waves, each for some heads of one token.
inline int64_t append_groups(int64_t n_tok, int heads, int kv_heads, int head_dim) {
    const int n = heads_of_wave(head_dim);
    return (n_tok * ((heads + 2 * kv_heads + n - 1) / n) + 3) / 4;
}

struct AttnArgs {
    const Item *items;
    const int32_t *tables;
    const Unit *units, *merge;
    const Own *tok_own;
    uint32_t *done;
    const void *q;
    void *out;
    float *lse;
    float *part_o;    // [part_rows][head_dim], normalised
    float *part_lse;  // [part_rows], base 2
    int64_t q_stride, out_stride;
    tas_cache c;
    int32_t n_wide;  // items
    int32_t group, heads;
    int32_t sub_shift;  // log2(block_tokens / 16)
    float scale2;       // scale * log2(e)
};

// Launches n workgroups of 256; the launch's own error. (hipGetLastError would also
// return one that an earlier call of the program left.)
template <typename Args>
hipError_t launch_kernel(void (*kernel)(Args), int64_t n, const Args &a, hipStream_t s) {
    Args copy = a;
    void *args[] = {&copy};
    return hipLaunchKernel((const void *)kernel, dim3((uint32_t)n), dim3(256), args, 0, s);
}

// Return hipSuccess or the launch's error.
hipError_t launch_append(const AppendArgs &a, int dtype, int head_dim, hipStream_t s);
hipError_t launch_attention(const AttnArgs &a, int n_items, int n_merge, int dtype, int head_dim,
                            hipStream_t s);

}  // namespace tas_step_impl
