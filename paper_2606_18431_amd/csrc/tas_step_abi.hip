// tas_step_abi.hip - host side of the C ABI declared in include/tas_step.h.
//
// tas_step_create validates a batch on the host (every block number that a
// kernel will follow is checked here) and cuts its attention into items of work;
// tas_step_bind copies that plan into the caller's workspace. tas_step_append
// and tas_step_attention only enqueue kernels.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "tas_step.h"
#include "tas_step_internal.h"
#include "tas_step_overlap.h"

using namespace tas_step_impl;

namespace {

constexpr int64_t kMaxTokens = int64_t(1) << 24;     // of a batch
constexpr int64_t kMaxPartRows = int64_t(1) << 28;
constexpr int64_t kMaxStride = (int64_t(1) << 31) - 8;      // of a block or head, elements
constexpr int64_t kMaxTokenStride = int64_t(1) << 24;       // of a token in a block
constexpr int64_t kMaxGroups = (int64_t(1) << 24) - 1;      // of a launch: 2^32 threads
constexpr int64_t kUnits = 256;                      // compute units
// By registers a compute unit holds two wide or three thin items of head size 128, and
// three or four of head size 64; the numbers below are those of 128 for both.
constexpr int64_t kSlots = 2 * kUnits;               // wide items taken to run at once
constexpr int32_t kThinItems = 768;                  // thin items wanted

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

struct Plan {
    PlanHead head{};
    std::vector<Req> reqs;
    std::vector<Seg> segs;
    std::vector<Item> thin, wide, items;
    std::vector<Unit> join, merge;
    std::vector<int32_t> tables, tok_req;
    std::vector<Own> tok_own;  // empty without prefixes
    int64_t max_pos = 0;  // largest position of a new token + 1
    bool appendable = true;
};

bool is_thin(const Seg &s) { return s.rows <= kThinRows; }
int32_t tile_rows(const Seg &s) { return is_thin(s) ? kThinRows : kWideRows; }
int32_t tiles_of(const Seg &s) { return (s.rows + tile_rows(s) - 1) / tile_rows(s); }

// The longest items first: those that start last are short ones. (Items of one
// length keep their order, which has the key heads innermost: workgroups go round
// the chip's 8 dies, so with 8 key heads or a divisor of it the items that share
// keys share a die's cache.)
void longest_first(std::vector<Item> &items, int32_t unit) {
    int32_t most = 0;
    for (const Item &it : items) most = std::max(most, (it.k1 - it.k0 + unit - 1) / unit);
    std::vector<size_t> at(most + 2, 0);
    auto slot = [&](const Item &it) { return most - (it.k1 - it.k0 + unit - 1) / unit; };
    for (const Item &it : items) at[slot(it) + 1]++;
    for (int32_t i = 0; i <= most; i++) at[i + 1] += at[i];
    std::vector<Item> to(items.size());
    for (const Item &it : items) to[at[slot(it)]++] = it;
    items.swap(to);
}

bool valid_shape(const tas_batch *b) {
    if (!b || b->kv_heads < 1 || b->heads < 1 || b->heads > 1024 || b->heads % b->kv_heads)
        return false;
    if (b->head_dim != 64 && b->head_dim != 128) return false;
    if (b->block_tokens < 16 || b->block_tokens > 4096 ||
        (b->block_tokens & (b->block_tokens - 1)))
        return false;
    if (b->n_req < 1 || b->n_blocks < 1 || b->n_prefix < 0) return false;
    if (b->causal != 0 && b->causal != 1) return false;
    if (!b->n_new || !b->kv_len || b->blocks_stride < 0) return false;
    if (b->n_prefix && (!b->prefix_first || !b->prefix_len || b->prefix_stride < 0)) return false;
    return true;
}

// Appends the pages of `len` keys to the tables; the table's offset, or -1.
int64_t add_table(const tas_batch *b, const int32_t *pages, int64_t stride, int64_t len, Plan &p) {
    const int64_t n = ceil_div(len, b->block_tokens);
    if (n > stride || (n && !pages)) return -1;
    const int64_t at = (int64_t)p.tables.size();
    if (at + n > INT32_MAX) return -1;
    for (int64_t i = 0; i < n; i++)
        if (pages[i] < 0 || pages[i] >= b->n_blocks) return -1;
    p.tables.insert(p.tables.end(), pages, pages + n);
    return at;
}

// Two new tokens appended to one slot would race: the blocks that new tokens go to are
// distinct, over all requests and within one (a block has one request that fills it).
bool distinct_slots(const tas_batch *b, const Plan &p) {
    std::vector<int32_t> written;
    for (const Req &r : p.reqs) {
        if (!r.n_new || r.n_new > r.kv_len) continue;
        const int32_t first = (r.kv_len - r.n_new) / b->block_tokens;
        const int32_t last = (r.kv_len - 1) / b->block_tokens;
        for (int32_t i = first; i <= last; i++) written.push_back(p.tables[r.table + i]);
    }
    std::sort(written.begin(), written.end());
    return std::adjacent_find(written.begin(), written.end()) == written.end();
}

// Pieces of a thin segment's keys: as many as give every slot its share of the batch,
// but no more than pay. I steps of 128 keys in n pieces take about 0.9 I / n us, and
// joining the n parts 2.2 us for every eight, in each of the sets of rows that a join
// has threads for: that is least at n = 1.8 sqrt(I sets). A join as such costs some
// 2 us, what three steps take. (One decode of 32/8 heads of 128: context 777 in pieces
// of 256 keys 9.3 us, of 128 8.6; 32000 in 125 pieces 49 us, in 57 35.) Parts that the
// merge kernel joins are one set, and two steps long at least.
int64_t thin_pieces(const Seg &s, int64_t share, bool merged) {
    const int64_t step = 4 * kThinKeys, steps = ceil_div(s.kv_len, step);
    if (steps <= 3 && !merged) return 1;
    int sets = 1;
    while (!merged && sets * 2 * s.rows <= kJoinRows) sets *= 2;
    const int64_t pay = (int64_t)(1.8 * std::sqrt((double)steps * sets));
    const int64_t piece = merged ? std::max(share, 2 * step) : share;
    return std::min(ceil_div(s.kv_len, piece), pay);
}

// Keys of a piece of the thin segments: the share of all keys that makes kThinItems. As
// every segment has a last piece that is shorter, these are somewhat more items than that:
// where a piece that is longer by a third at most makes that many, or a sixteenth fewer,
// that one. At head size 128 the rest would take a round of its own (32/8 heads, 64
// contexts of about 1200: 928 items 66 us, 760 items 64; with more slots left empty it
// loses: 16/2 heads, 28 of about 14830: 786 items 77 us, 694 items 82). At 64, where
// either number runs at once, the fewer items measured faster too (16/16 heads, 8 contexts
// of about 20039: 816 items 136 us, 752 items 121).
int64_t choose_thin_piece(const Plan &p, const std::vector<char> &joined, int64_t kv_heads,
                          int64_t keys, bool any_wide) {
    const int64_t step = 4 * kThinKeys;
    const int64_t share = ceil_div(ceil_div(keys, kThinItems), step) * step;
    if (any_wide || (int64_t)p.segs.size() * kv_heads > kThinItems) return share;
    for (int64_t piece = share; piece <= share + share / 3; piece += step) {
        int64_t items = 0;
        for (size_t i = 0; i < p.segs.size(); i++)
            items += kv_heads *
                     std::max<int64_t>(1, thin_pieces(p.segs[i], piece, joined[i]));
        if (items <= kThinItems)
            return items >= kThinItems - kThinItems / 16 ? piece : share;
    }
    return share;
}

// Pieces of a wide segment's keys, each of `piece` steps, but (as above, with one set
// and 1 us for a step) no more than pay.
int64_t wide_pieces(const Seg &s, int64_t piece) {
    const int64_t steps = ceil_div(s.kv_len, kWideKeys);
    return std::max<int64_t>(
        1, std::min(ceil_div(steps, piece), (int64_t)(1.9 * std::sqrt((double)steps))));
}

// Steps of a piece of the wide segments' keys, by what the batch then takes. Measured: a
// step of 64 keys lasts 1.16 us where a compute unit has one item, 2.06 us where it has
// two (head size 64: 0.80, 1.34; three are not taken into account); the thin items' keys
// stream at 6 TB/s beside that; a merge takes 2 us, 2.2 for every eight parts of a row,
// and the time to write and read the parts at 10 TB/s (they stay in caches for the most
// part). (One chunk of 1024, 32/8 heads of 128, nothing before it: whole 25 us, in two
// pieces 32; 16/16 heads of 64 over 4096 keys: whole 56 us, in four 33.)
int64_t choose_wide_piece(const tas_batch *b, const Plan &p, const std::vector<char> &joined,
                          int64_t thin_keys) {
    const int64_t Hk = b->kv_heads;
    const double step_us[2] = {b->head_dim == 64 ? 0.80 : 1.16, b->head_dim == 64 ? 1.34 : 2.06};
    const double thin_us = (double)thin_keys * b->head_dim * 4 / 6e6;
    int64_t most = 0, n_thin = 0;
    for (const Seg &s : p.segs) {
        if (is_thin(s))
            n_thin += Hk;
        else
            most = std::max(most, ceil_div(s.kv_len, kWideKeys));
    }
    int64_t best = 1;
    double least = 0;
    for (int64_t n : {1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 15, 20, 24, 32, 48, 64}) {
        const int64_t piece = std::max<int64_t>(1, ceil_div(most, n));
        int64_t items = n_thin, longest = 0, parts = 0;
        double steps = 0, part_bytes = 0;
        for (size_t i = 0; i < p.segs.size(); i++) {
            const Seg &s = p.segs[i];
            if (is_thin(s)) continue;
            const int64_t all = ceil_div(s.kv_len, kWideKeys), k = wide_pieces(s, piece);
            items += tiles_of(s) * Hk * k;
            steps += (double)(tiles_of(s) * Hk * all);
            longest = std::max(longest, ceil_div(all, k));
            if (k > 1 || joined[i]) {
                parts = std::max(parts, k + joined[i]);  // (and of the own keys)
                part_bytes += (double)(s.rows * Hk * k) * b->head_dim * 4;
            }
        }
        double us = std::max(longest * step_us[items > kUnits],
                             steps * step_us[1] / kSlots + thin_us);
        if (parts) us += 2 + 2.2 * ceil_div(parts, 8) + part_bytes * 2 / 10e6;
        if (n == 1 || us < least) least = us, best = piece;
        if (piece == 1) break;
    }
    return best;
}

// Cuts the keys of the segments into items. A segment's keys are split into
// nsplit pieces (the last ones shorter, or empty); every tile of its rows has an
// item for each piece, an empty one where causality leaves nothing, so that a join
// finds nsplit partial results for every row.
int make_items(const tas_batch *b, Plan &p) {
    const int32_t G = b->heads / b->kv_heads, Hk = b->kv_heads;
    int64_t thin_keys = 0, wide_steps = 0;
    for (const Seg &s : p.segs) {
        if (is_thin(s))
            thin_keys += (int64_t)s.kv_len * Hk;
        else
            wide_steps += (int64_t)tiles_of(s) * Hk * ceil_div(s.kv_len, kWideKeys);
    }
    const int64_t step = 4 * kThinKeys;
    // whose parts the merge kernel joins though they are not split
    std::vector<char> joined(p.segs.size(), 0);
    for (const Req &r : p.reqs)
        if (r.pre_seg >= 0 && !is_thin(p.segs[r.pre_seg])) {
            joined[r.pre_seg] = 1;
            if (r.own_seg >= 0) joined[r.own_seg] = 1;
        }
    const int64_t thin_piece = choose_thin_piece(p, joined, Hk, thin_keys, wide_steps > 0);
    const int64_t wide_piece = wide_steps ? choose_wide_piece(b, p, joined, thin_keys) : 1;
    for (size_t i = 0; i < p.segs.size(); i++) {
        Seg &s = p.segs[i];
        s.nsplit = (int32_t)std::max<int64_t>(
            1, is_thin(s) ? thin_pieces(s, thin_piece, joined[i])
                          : wide_pieces(s, wide_piece));
        s.part = -1;
    }
    // a result goes straight to the output where it has one part only
    int64_t part_rows = 0;
    std::vector<int32_t> unit0(p.segs.size(), -1);  // join of a thin segment's key head 0
    std::vector<int32_t> is_prefix(p.segs.size(), 0);
    for (const Req &r : p.reqs)
        if (r.pre_seg >= 0) is_prefix[r.pre_seg] = 1;
    auto partial = [&](int32_t seg, bool joins) {
        Seg &s = p.segs[seg];
        s.part = (int32_t)part_rows;
        part_rows += (int64_t)Hk * s.nsplit * s.rows;
        if (part_rows > kMaxPartRows) return false;
        if (!joins) return true;
        if (is_thin(s))
            unit0[seg] = (int32_t)p.join.size();
        else if ((int64_t)p.merge.size() + Hk * ceil_div(s.rows, kJoinRows) > kMaxGroups)
            return false;
        for (int32_t hk = 0; hk < Hk; hk++)
            for (int32_t row0 = 0; row0 < s.rows; row0 += kJoinRows)
                (is_thin(s) ? p.join : p.merge)
                    .push_back({s, seg, hk, row0, std::min(kJoinRows, s.rows - row0), 0,
                                is_prefix[seg], {0, 0}});
        return true;
    };
    std::vector<int32_t> shared(p.segs.size(), -1);  // the prefix that an own segment joins
    for (const Req &r : p.reqs) {
        if (r.pre_seg >= 0 && p.segs[r.pre_seg].part < 0 && !partial(r.pre_seg, true))
            return TAS_EINVAL;
        if (r.own_seg < 0) continue;
        shared[r.own_seg] = r.pre_seg;
        if ((r.pre_seg >= 0 || p.segs[r.own_seg].nsplit > 1) &&
            !partial(r.own_seg, r.pre_seg < 0))
            return TAS_EINVAL;
    }
    if (b->n_prefix) {
        p.tok_own.reserve(p.tok_req.size());
        for (const Req &r : p.reqs) {
            Own own{};
            if (r.own_seg >= 0) {
                const Seg &s = p.segs[r.own_seg];
                own = {s.part, s.nsplit, s.rows, s.t0};
            }
            p.tok_own.insert(p.tok_own.end(), (size_t)r.n_new, own);
        }
    }
    int64_t n_items = 0;
    for (const Seg &s : p.segs) n_items += (int64_t)Hk * tiles_of(s) * s.nsplit;
    if (n_items > kMaxGroups) return TAS_EINVAL;
    for (size_t i = 0; i < p.segs.size(); i++) {
        const Seg &s = p.segs[i];
        const int32_t tile = tile_rows(s);
        const int64_t unit = is_thin(s) ? step : kWideKeys;
        const int64_t piece = ceil_div(ceil_div(s.kv_len, s.nsplit), unit) * unit;
        std::vector<Item> &to = is_thin(s) ? p.thin : p.wide;
        const int32_t unit_of = unit0[shared[i] >= 0 ? shared[i] : (int32_t)i];
        for (int32_t row0 = 0; row0 < s.rows; row0 += tile) {
            const int32_t rows = std::min(tile, s.rows - row0);
            const int64_t lim = std::max<int64_t>(
                0, std::min<int64_t>(s.kv_len, (int64_t)s.lim0 + (row0 + rows - 1) / G));
            for (int32_t n = 0; n < s.nsplit; n++)
                for (int32_t hk = 0; hk < Hk; hk++) {
                    Item it{};
                    it.s = s;
                    it.seg = (int32_t)i;
                    it.hk = hk;
                    it.row0 = row0;
                    it.k0 = (int32_t)std::min<int64_t>(n * piece, lim);
                    it.k1 = (int32_t)std::min<int64_t>((n + 1) * piece, lim);
                    it.part = it.unit = -1;
                    if (s.part >= 0) {
                        it.part =
                            (int32_t)(s.part + ((int64_t)hk * s.nsplit + n) * s.rows + row0);
                        if (unit_of >= 0) {
                            it.unit = unit_of + hk;
                            p.join[it.unit].items++;
                        }
                    }
                    to.push_back(it);
                }
        }
    }
    longest_first(p.thin, (int32_t)step);
    longest_first(p.wide, kWideKeys);
    // A wide item keeps the matrix cores busy and a thin one the memory, so that a compute
    // unit is to have one of each as long as there are both: either kind has half of the
    // slots, or what the other leaves, and the items are listed as those slots come free
    // (the work of the kind before an item, over its slots; in steps of a wide item, of
    // which a thin item's last 1.5, and one for the start). (60 decodes and 4 chunks, 28/4
    // heads of 128: 130 us; 256 of each alternately 136, all the wide items first 146.)
    struct Kind {
        const std::vector<Item> &items;
        double step, slots;  // keys of a step's time
        size_t next = 0;
        double before = 0;
        double start() const { return next < slots ? 0 : before / slots; }
    };
    const double n_wide = (double)p.wide.size(), n_thin = (double)p.thin.size();
    Kind wide{p.wide, kWideKeys, kSlots - std::min<double>(n_thin, kUnits)};
    Kind thin{p.thin, (double)step / 1.5, kSlots - std::min<double>(n_wide, kUnits)};
    p.items.reserve(p.wide.size() + p.thin.size());
    while (p.items.size() < p.wide.size() + p.thin.size()) {
        const bool w = wide.next < p.wide.size() &&
                       (thin.next == p.thin.size() || wide.start() <= thin.start());
        Kind &from = w ? wide : thin;
        const Item &it = from.items[from.next++];
        from.before += (it.k1 - it.k0) / from.step + 1;
        p.items.push_back(it);
    }
    p.head.part_rows = part_rows;
    return TAS_OK;
}

int make_plan(const tas_batch *b, Plan &p) {
    if (!valid_shape(b)) return TAS_EINVAL;
    const int32_t G = b->heads / b->kv_heads;
    std::vector<int64_t> prefix_table(b->n_prefix);
    for (int32_t g = 0; g < b->n_prefix; g++) {
        const int32_t lo = b->prefix_first[g], hi = b->prefix_first[g + 1];
        if (lo < 0 || hi < lo || hi > b->n_req || (g == 0 && lo != 0)) return TAS_EINVAL;
        if (g == b->n_prefix - 1 && hi != b->n_req) return TAS_EINVAL;
        if (b->prefix_len[g] < 0) return TAS_EINVAL;
    }
    for (int32_t g = 0; g < b->n_prefix; g++) {
        prefix_table[g] =
            add_table(b, b->prefix_blocks ? b->prefix_blocks + g * b->prefix_stride : nullptr,
                      b->prefix_stride, b->prefix_len[g], p);
        if (prefix_table[g] < 0) return TAS_EINVAL;
    }
    int64_t t = 0;
    int32_t g = 0, group_seg = -1;
    p.reqs.reserve(b->n_req);
    for (int32_t i = 0; i < b->n_req; i++) {
        while (g < b->n_prefix && i >= b->prefix_first[g + 1]) g++, group_seg = -1;
        const int64_t n = b->n_new[i], kv = b->kv_len[i];
        const int64_t pre = b->n_prefix ? b->prefix_len[g] : 0;
        if (n < 0 || kv < 0 || pre + kv > INT32_MAX / 2 || t + n > kMaxTokens) return TAS_EINVAL;
        Req r{};
        r.t0 = (int32_t)t;
        r.n_new = (int32_t)n;
        r.kv_len = (int32_t)kv;
        r.prefix_len = (int32_t)pre;
        r.own_seg = r.pre_seg = -1;
        const int64_t at = add_table(b, b->blocks ? b->blocks + i * b->blocks_stride : nullptr,
                                     b->blocks_stride, kv, p);
        if (at < 0) return TAS_EINVAL;
        r.table = (int32_t)at;
        if (n) {
            if (kv < n) p.appendable = false;
            p.max_pos = std::max(p.max_pos, pre + kv);
            if (kv || !pre) {  // without any key an empty item writes the zeros
                Seg s{};
                s.t0 = r.t0;
                s.n_tok = r.n_new;
                s.kv_len = r.kv_len;
                s.lim0 = b->causal ? (int32_t)(kv - n + 1) : r.kv_len;
                s.table = r.table;
                s.rows = (int32_t)(n * G);
                r.own_seg = (int32_t)p.segs.size();
                p.segs.push_back(s);
            }
            if (pre) {
                if (group_seg < 0) {
                    Seg s{};
                    s.t0 = r.t0;
                    s.kv_len = s.lim0 = (int32_t)pre;
                    s.table = (int32_t)prefix_table[g];
                    group_seg = (int32_t)p.segs.size();
                    p.segs.push_back(s);
                }
                // the group's tokens follow one another: requests without new
                // ones in between add none
                p.segs[group_seg].n_tok += (int32_t)n;
                p.segs[group_seg].rows += (int32_t)(n * G);
                r.pre_seg = group_seg;
            }
        }
        p.tok_req.insert(p.tok_req.end(), (size_t)n, i);
        p.reqs.push_back(r);
        t += n;
    }
    // rows and heads of the batch are counted in 32 bits
    if (t * (b->heads + 2 * b->kv_heads) > INT32_MAX / 2) return TAS_EINVAL;
    if (append_groups(t, b->heads, b->kv_heads, b->head_dim) > kMaxGroups) return TAS_EINVAL;
    if (p.appendable && !distinct_slots(b, p)) {
        // A causal batch's new tokens are the last ones of contexts of their own: a block
        // that two of them end in is an error of the tables. Without causality they may
        // be queries over any pages, and only append would race.
        if (b->causal) return TAS_EINVAL;
        p.appendable = false;
    }
    const int rc = make_items(b, p);
    if (rc != TAS_OK) return rc;
    PlanHead &h = p.head;
    size_t at = align256(sizeof(PlanHead));
    auto place = [&](int64_t &off, size_t bytes) { off = (int64_t)at, at += align256(bytes); };
    h.n_req = b->n_req;
    h.n_tok = (int32_t)t;
    h.n_seg = (int32_t)p.segs.size();
    h.n_thin = (int32_t)p.thin.size();
    h.n_wide = (int32_t)p.wide.size();
    h.n_join = (int32_t)p.join.size();
    h.n_merge = (int32_t)p.merge.size();
    h.n_table = (int32_t)p.tables.size();
    place(h.req, p.reqs.size() * sizeof(Req));
    place(h.seg, p.segs.size() * sizeof(Seg));
    place(h.items, p.items.size() * sizeof(Item));
    place(h.units, (p.join.size() + p.merge.size()) * sizeof(Unit));
    place(h.tables, p.tables.size() * 4);
    place(h.tok_req, p.tok_req.size() * 4);
    place(h.tok_own, p.tok_own.size() * sizeof(Own));
    place(h.done, p.join.size() * 4);
    h.bytes = (int64_t)at;
    return TAS_OK;
}

void write_blob(const Plan &p, char *to) {
    const PlanHead &h = p.head;
    memcpy(to, &h, sizeof(h));
    auto put = [&](int64_t off, const void *from, size_t bytes) {
        if (bytes) memcpy(to + off, from, bytes);
    };
    put(h.req, p.reqs.data(), p.reqs.size() * sizeof(Req));
    put(h.seg, p.segs.data(), p.segs.size() * sizeof(Seg));
    put(h.items, p.items.data(), p.items.size() * sizeof(Item));
    put(h.units, p.join.data(), p.join.size() * sizeof(Unit));
    put(h.units + p.join.size() * sizeof(Unit), p.merge.data(), p.merge.size() * sizeof(Unit));
    put(h.tables, p.tables.data(), p.tables.size() * 4);
    put(h.tok_req, p.tok_req.data(), p.tok_req.size() * 4);
    put(h.tok_own, p.tok_own.data(), p.tok_own.size() * sizeof(Own));
}


bool aligned16(const void *p) { return p && ((uintptr_t)p & 15) == 0; }

bool valid_cache(const tas_cache &c) {
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
bool disjoint_slots(int64_t block, int64_t head, int64_t token, int64_t n_blocks,
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
Region region_of(const void *p, int64_t block, int64_t head, int64_t token, int64_t n_blocks,
                 int64_t kv_heads, int64_t block_tokens, int64_t head_dim) {
    return {(int64_t)((uintptr_t)p / 16), head_dim / 8, {block / 8, head / 8, token / 8},
            {n_blocks, kv_heads, block_tokens}};
}

// The rows of n_tok tokens (aligned, the stride in elements).
Region region_of(const void *p, int64_t stride, int64_t row, int64_t n_tok) {
    return {(int64_t)((uintptr_t)p / 16), row / 8, {stride / 8, 0, 0}, {n_tok, 1, 1}};
}

// Whether an output's rows are in memory that is read or written besides. They may be the
// input's own rows: a row is read before it is written.
bool clash(const void *out, int64_t out_stride, int64_t out_row, const void *in,
           int64_t in_stride, int64_t in_row, int64_t n_tok, const Region &k, const Region &v) {
    const Region o = region_of(out, out_stride, out_row, n_tok);
    Overlap overlap;
    const bool in_place = out == in && (out_stride == in_stride || n_tok == 1);
    return (!in_place && overlap(o, region_of(in, in_stride, in_row, n_tok))) || overlap(o, k) ||
           overlap(o, v);
}

bool valid_rows(const void *p, int64_t stride, int64_t row) {
    return aligned16(p) && stride >= row && stride % 8 == 0;
}

}  // namespace

struct tas_step {
    std::vector<char> blob;  // the plan
    PlanHead head{};
    int32_t heads = 0, kv_heads = 0, head_dim = 0, blk_shift = 0, n_blocks = 0;
    int64_t max_pos = 0;
    bool appendable = false;
    char *ws = nullptr;  // null: not bound
    size_t part_o() const { return blob.size(); }
    size_t part_lse() const {
        return part_o() + align256((size_t)head.part_rows * head_dim * 4);
    }
    size_t bytes() const { return part_lse() + align256((size_t)head.part_rows * 4); }
};

static int valid_workspace(const tas_step *s, const void *d_ws, size_t ws_bytes) {
    if (!s || !d_ws || ((uintptr_t)d_ws & 255)) return TAS_EINVAL;
    return ws_bytes < s->bytes() ? TAS_ENOMEM : TAS_OK;
}

extern "C" {

int tas_step_create(const tas_batch *b, tas_step **out) try {
    if (!out) return TAS_EINVAL;
    *out = nullptr;
    Plan p;
    const int rc = make_plan(b, p);
    if (rc != TAS_OK) return rc;
    std::vector<char> blob((size_t)p.head.bytes);
    write_blob(p, blob.data());
    tas_step *s = new tas_step;
    s->blob.swap(blob);
    s->head = p.head;
    s->heads = b->heads;
    s->kv_heads = b->kv_heads;
    s->head_dim = b->head_dim;
    s->n_blocks = b->n_blocks;
    while ((1 << s->blk_shift) < b->block_tokens) s->blk_shift++;
    s->max_pos = p.max_pos;
    s->appendable = p.appendable;
    *out = s;
    return TAS_OK;
} catch (...) {
    return TAS_ENOMEM;
}

size_t tas_step_bytes(const tas_step *s) { return s ? s->bytes() : 0; }

int tas_step_bind(tas_step *s, void *d_ws, size_t ws_bytes, void *stream) {
    const int rc = valid_workspace(s, d_ws, ws_bytes);
    if (rc != TAS_OK) return rc;
    const hipStream_t st = (hipStream_t)stream;
    if (hipMemcpyAsync(d_ws, s->blob.data(), s->blob.size(), hipMemcpyHostToDevice, st) !=
            hipSuccess ||
        hipStreamSynchronize(st) != hipSuccess)
        return TAS_EHIP;
    s->ws = (char *)d_ws;
    return TAS_OK;
}

int tas_step_attach(tas_step *s, void *d_ws, size_t ws_bytes) {
    const int rc = valid_workspace(s, d_ws, ws_bytes);
    if (rc == TAS_OK) s->ws = (char *)d_ws;
    return rc;
}

void tas_step_destroy(tas_step *s) { delete s; }

int64_t tas_step_tokens(const tas_step *s) { return s ? s->head.n_tok : -1; }

int tas_step_plan(const tas_step *s, void *buf, size_t buf_bytes, size_t *bytes) {
    if (!s || !bytes) return TAS_EINVAL;
    *bytes = s->blob.size();
    if (!buf) return TAS_OK;
    if (buf_bytes < s->blob.size()) return TAS_ENOMEM;
    memcpy(buf, s->blob.data(), s->blob.size());
    return TAS_OK;
}

int tas_step_append(tas_step *s, const tas_append *a, void *stream) {
    if (!s || !a || !s->appendable) return TAS_EINVAL;
    if (!s->ws) return TAS_ESTATE;
    const int64_t D = s->head_dim;
    if (a->dtype != TAS_F16 && a->dtype != TAS_BF16) return TAS_EINVAL;
    if (a->rot_dim < 0 || a->rot_dim > D || a->rot_dim % 16) return TAS_EINVAL;
    if (a->interleaved != 0 && a->interleaved != 1) return TAS_EINVAL;
    if (!(a->eps >= 0) || std::isinf(a->eps)) return TAS_EINVAL;
    if (!a->q_weight != !a->k_weight) return TAS_EINVAL;
    if (a->q_weight && (!aligned16(a->q_weight) || !aligned16(a->k_weight))) return TAS_EINVAL;
    if (a->rot_dim &&
        (!aligned16(a->cos) || !aligned16(a->sin) || a->positions < s->max_pos))
        return TAS_EINVAL;
    if (!valid_cache(a->cache)) return TAS_EINVAL;
    const tas_cache &c = a->cache;
    const int64_t bt = int64_t(1) << s->blk_shift;
    if (!disjoint_slots(c.k_block, c.k_head, c.k_token, s->n_blocks, s->kv_heads, bt, D) ||
        !disjoint_slots(c.v_block, c.v_head, c.v_token, s->n_blocks, s->kv_heads, bt, D))
        return TAS_EINVAL;
    const Region kr =
        region_of(c.k, c.k_block, c.k_head, c.k_token, s->n_blocks, s->kv_heads, bt, D);
    const Region vr =
        region_of(c.v, c.v_block, c.v_head, c.v_token, s->n_blocks, s->kv_heads, bt, D);
    if (Overlap()(kr, vr)) return TAS_EINVAL;  // (K of a token and V of another would race)
    if (s->head.n_tok == 0) return TAS_OK;
    const int64_t in_row = (s->heads + 2 * s->kv_heads) * D, out_row = s->heads * D;
    if (!valid_rows(a->qkv, a->qkv_stride, in_row) ||
        !valid_rows(a->q_out, a->q_out_stride, out_row))
        return TAS_EINVAL;
    const Region in = region_of(a->qkv, a->qkv_stride, in_row, s->head.n_tok);
    if (clash(a->q_out, a->q_out_stride, out_row, a->qkv, a->qkv_stride, in_row, s->head.n_tok, kr,
              vr) ||
        Overlap()(in, kr) || Overlap()(in, vr))
        return TAS_EINVAL;
    AppendArgs k{};
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
    k.c = a->cache;
    k.n_tok = s->head.n_tok;
    k.heads = s->heads;
    k.kv_heads = s->kv_heads;
    k.rot = a->rot_dim;
    k.interleaved = a->interleaved;
    k.blk_shift = s->blk_shift;
    k.eps = a->eps;
    return launch_append(k, a->dtype, s->head_dim, (hipStream_t)stream) == hipSuccess ? TAS_OK
                                                                                     : TAS_EHIP;
}

int tas_step_attention(tas_step *s, const tas_attention *a, void *stream) {
    if (!s || !a) return TAS_EINVAL;
    if (!s->ws) return TAS_ESTATE;
    if (a->dtype != TAS_F16 && a->dtype != TAS_BF16) return TAS_EINVAL;
    const float scale2 = a->scale * 1.4426950408889634f;
    if (!(a->scale > 0) || std::isinf(scale2)) return TAS_EINVAL;
    if (!valid_cache(a->cache)) return TAS_EINVAL;
    if (s->head.n_tok == 0) return TAS_OK;
    const int64_t row = (int64_t)s->heads * s->head_dim;
    if (!valid_rows(a->q, a->q_stride, row) || !valid_rows(a->out, a->out_stride, row))
        return TAS_EINVAL;
    const tas_cache &c = a->cache;
    const int64_t bt = int64_t(1) << s->blk_shift, D = s->head_dim;
    if (clash(a->out, a->out_stride, row, a->q, a->q_stride, row, s->head.n_tok,
              region_of(c.k, c.k_block, c.k_head, c.k_token, s->n_blocks, s->kv_heads, bt, D),
              region_of(c.v, c.v_block, c.v_head, c.v_token, s->n_blocks, s->kv_heads, bt, D)))
        return TAS_EINVAL;
    AttnArgs k{};
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
    k.c = a->cache;
    k.group = s->heads / s->kv_heads;
    k.heads = s->heads;
    k.sub_shift = s->blk_shift - 4;
    k.scale2 = scale2;
    k.n_wide = s->head.n_wide;
    return launch_attention(k, s->head.n_wide + s->head.n_thin, s->head.n_merge, a->dtype,
                            s->head_dim, (hipStream_t)stream) == hipSuccess
               ? TAS_OK
               : TAS_EHIP;
}

}  // extern "C"
