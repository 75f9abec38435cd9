"""The plan of a step on the host (no GPU): what tas_step_create would copy to
the device covers every visible key of every row once, follows the right pages,
gives partial results disjoint places, and invalid batches are refused."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest

from paper_2606_18431_amd import step, tas

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

REQ = np.dtype([(f, np.int32) for f in ("t0", "n_new", "kv_len", "table", "prefix_len", "own_seg",
                                        "pre_seg", "pad")])
SEG = np.dtype([(f, np.int32) for f in ("t0", "n_tok", "kv_len", "lim0", "table", "nsplit", "part",
                                        "rows")])
ITEM = np.dtype([("s", SEG)] + [(f, np.int32) for f in ("seg", "hk", "row0", "k0", "k1", "part",
                                                        "unit", "pad")])
UNIT = np.dtype([("s", SEG)] + [(f, np.int32) for f in ("seg", "hk", "row0", "rows", "items",
                                                        "prefix", "pad0", "pad1")])
OWN = np.dtype([(f, np.int32) for f in ("part", "nsplit", "rows", "t0")])
HEAD = np.dtype([("bytes", np.int64), ("part_rows", np.int64)]
                + [(f, np.int32) for f in ("n_req", "n_tok", "n_seg", "n_thin", "n_wide",
                                           "n_join", "n_merge", "n_table")]
                + [(f, np.int64) for f in ("req", "seg", "items", "units", "tables", "tok_req",
                                           "tok_own", "done")])
THIN_ROWS, WIDE_ROWS, JOIN_ROWS = 16, 128, 16


def plan(b):
    """The parsed plan of a tas_batch."""
    ctx = step.tas_step_create(b)
    try:
        blob = step.tas_step_plan(ctx)
        h = np.frombuffer(blob, HEAD, 1)[0]
        assert h["bytes"] == len(blob) and step.tas_step_tokens(ctx) == h["n_tok"]
        assert step.tas_step_bytes(ctx) >= len(blob) + h["part_rows"] * (b.head_dim + 1) * 4
    finally:
        step.tas_step_destroy(ctx)

    def at(off, dtype, n):
        return np.frombuffer(blob, dtype, int(n), int(off))

    items = at(h["items"], ITEM, h["n_wide"] + h["n_thin"])
    segs = at(h["seg"], SEG, h["n_seg"])
    wide = segs["rows"][items["seg"]] > THIN_ROWS
    assert int(wide.sum()) == h["n_wide"]
    return dict(head=h, reqs=at(h["req"], REQ, h["n_req"]), segs=segs,
                wide=items[wide], thin=items[~wide],
                units=at(h["units"], UNIT, h["n_join"] + h["n_merge"]),
                tables=at(h["tables"], np.int32, h["n_table"]),
                tok_req=at(h["tok_req"], np.int32, h["n_tok"]),
                tok_own=at(h["tok_own"], OWN, h["n_tok"] if b.n_prefix else 0),
                done=at(h["done"], np.int32, h["n_join"]))


def batch(seed, n_req, max_new, max_ctx, heads, kv_heads, block, groups=0, causal=True,
          some_empty=False):
    rng = np.random.default_rng(seed)
    n = rng.integers(0 if some_empty else 1, max_new + 1, n_req)
    kv = np.maximum(n, rng.integers(1, max_ctx + 1, n_req)) * (1 if not some_empty
                                                             else rng.integers(0, 2, n_req))
    if causal:
        kv = np.maximum(kv, n)
    width = int(max(1, (-(-kv // block)).max()))
    pre = rng.integers(0, 3 * block, groups)
    pwidth = int(max(1, (-(-pre // block)).max())) if groups else 0
    n_blocks = n_req * width + groups * pwidth + 3
    ids = rng.permutation(n_blocks).astype(np.int32)
    blocks = ids[:n_req * width].reshape(n_req, width)
    kw = dict(heads=heads, kv_heads=kv_heads, head_dim=64, block_tokens=block, n_blocks=n_blocks,
              causal=causal)
    if groups:
        cuts = np.sort(rng.integers(0, n_req + 1, groups - 1))
        kw.update(prefix_first=np.concatenate([[0], cuts, [n_req]]), prefix_len=pre,
                  prefix_blocks=ids[n_req * width:n_req * width + groups * pwidth]
                  .reshape(groups, pwidth))
    return n, kv, blocks, kw


CASES = [dict(seed=1, n_req=1, max_new=1, max_ctx=1, heads=8, kv_heads=8, block=16),
         dict(seed=2, n_req=70, max_new=1, max_ctx=9000, heads=32, kv_heads=8, block=16),
         dict(seed=3, n_req=5, max_new=300, max_ctx=700, heads=7, kv_heads=1, block=32),
         dict(seed=4, n_req=9, max_new=6, max_ctx=40, heads=12, kv_heads=4, block=16, groups=3),
         dict(seed=5, n_req=40, max_new=2, max_ctx=500, heads=64, kv_heads=2, block=64, groups=2,
              some_empty=True),
         dict(seed=6, n_req=12, max_new=40, max_ctx=100, heads=4, kv_heads=2, block=16,
              causal=False, some_empty=True),
         dict(seed=7, n_req=3, max_new=1000, max_ctx=9000, heads=16, kv_heads=2, block=16,
              groups=1)]


@pytest.mark.parametrize("case", CASES, ids=lambda c: str(c["seed"]))
def test_plan_covers_every_visible_key_once(case):
    n, kv, blocks, kw = batch(**case)
    b, keep = step.make_batch(n, kv, blocks, **kw)
    p = plan(b)
    Hk, G, bt = kw["kv_heads"], kw["heads"] // kw["kv_heads"], kw["block_tokens"]
    T = int(n.sum())
    assert p["head"]["n_tok"] == T and p["head"]["n_req"] == len(n)
    assert np.array_equal(p["tok_req"], np.repeat(np.arange(len(n)), n))
    first = kw.get("prefix_first")
    used = np.zeros(int(p["head"]["part_rows"]), np.int32)
    n_join = int(p["head"]["n_join"])
    counted = np.zeros(n_join, np.int64)
    covered = {}  # (seg, hk) -> per row, the pieces that saw it
    for kind, tile in (("thin", THIN_ROWS), ("wide", WIDE_ROWS)):
        for it in p[kind]:
            s = p["segs"][it["seg"]]
            assert s == it["s"]
            assert (s["rows"] <= THIN_ROWS) == (kind == "thin")
            assert 0 <= it["hk"] < Hk and it["row0"] % tile == 0 and it["row0"] < s["rows"]
            rows = min(tile, s["rows"] - it["row0"])
            assert 0 <= it["k0"] <= it["k1"] <= s["kv_len"]
            assert it["k0"] % 32 == 0 or it["k0"] == it["k1"]
            assert (it["part"] >= 0) == (s["part"] >= 0)
            if it["part"] >= 0:
                used[it["part"]:it["part"] + rows] += 1
            if it["unit"] >= 0:  # a thin item of the unit's rows
                assert kind == "thin" and it["part"] >= 0
                counted[it["unit"]] += 1
                un = p["units"][it["unit"]]
                shift = (int(s["t0"]) - int(p["segs"][un["seg"]]["t0"])) * G + it["row0"]
                assert un["hk"] == it["hk"] and un["row0"] <= shift
                assert shift + rows <= un["row0"] + un["rows"]
            for r in range(it["row0"], it["row0"] + rows):
                covered.setdefault((int(it["seg"]), int(it["hk"]), r), []).append(it)
    assert (used == 1).all()  # every partial row is written, by one item
    # a join waits for its items, which are all that have parts of its rows
    assert np.array_equal(counted, p["units"]["items"][:n_join]) and not p["done"].any()
    joined = {}
    for u, un in enumerate(p["units"]):
        s = p["segs"][un["seg"]]
        assert s == un["s"]
        assert un["row0"] % JOIN_ROWS == 0 and un["row0"] + un["rows"] <= s["rows"]
        assert un["rows"] == min(JOIN_ROWS, s["rows"] - un["row0"])
        assert (u < n_join) == (s["rows"] <= THIN_ROWS)
        own = set()
        for r in range(un["row0"], un["row0"] + un["rows"]):
            rq = p["reqs"][p["tok_req"][s["t0"] + r // G]]
            assert un["seg"] == (rq["pre_seg"] if un["prefix"] else rq["own_seg"])
            assert un["prefix"] or rq["pre_seg"] < 0
            own.add(int(rq["own_seg"]))
            key = (int(s["t0"]) + r // G, int(un["hk"]), r % G)
            assert key not in joined
            joined[key] = u
        if u < n_join:
            parts = sum(int(p["segs"][x]["nsplit"]) for x in own if x >= 0)
            assert un["items"] == parts + (int(s["nsplit"]) if un["prefix"] else 0)
    for i, s in enumerate(p["segs"]):
        assert s["rows"] == s["n_tok"] * G
        for hk in range(Hk):
            for r in range(0, s["rows"], max(1, s["rows"] // 50)):
                its = sorted(covered[i, hk, r], key=lambda x: (x["k0"], x["k1"]))
                assert len(its) == s["nsplit"] and (s["part"] >= 0 or len(its) == 1)
                lim = max(0, min(s["kv_len"], s["lim0"] + r // G))
                at = 0
                for it in its:
                    assert it["k0"] == at or it["k0"] == it["k1"]
                    at = max(at, int(it["k1"]))
                assert at >= lim
                if s["part"] >= 0:
                    assert sorted(x["part"] + r - x["row0"] for x in its) == \
                        [s["part"] + (hk * s["nsplit"] + m) * s["rows"] + r
                         for m in range(s["nsplit"])]
    t = 0
    for i, r in enumerate(p["reqs"]):
        assert (r["t0"], r["n_new"], r["kv_len"]) == (t, n[i], kv[i])
        pages = -(-int(kv[i]) // bt)
        assert np.array_equal(p["tables"][r["table"]:r["table"] + pages], blocks[i, :pages])
        g = None if first is None else int(np.searchsorted(first, i, side="right") - 1)
        pre = 0 if g is None else int(kw["prefix_len"][g])
        assert r["prefix_len"] == pre
        if n[i]:
            own, shared = r["own_seg"], r["pre_seg"]
            assert (shared >= 0) == (pre > 0) and (own >= 0 or pre > 0)
            if own >= 0:
                s = p["segs"][own]
                assert (s["t0"], s["n_tok"], s["kv_len"], s["table"]) == (t, n[i], kv[i],
                                                                        r["table"])
                assert s["lim0"] == (kv[i] - n[i] + 1 if kw["causal"] else kv[i])
            if shared >= 0:
                s = p["segs"][shared]
                assert s["t0"] <= t and t + n[i] <= s["t0"] + s["n_tok"]
                assert s["kv_len"] == s["lim0"] == pre and s["part"] >= 0
                q = -(-pre // bt)
                assert np.array_equal(p["tables"][s["table"]:s["table"] + q],
                                      np.asarray(kw["prefix_blocks"])[g, :q])
            parts = shared >= 0 or p["segs"][own]["part"] >= 0
            for j in range(t, t + n[i]):
                for hk in range(Hk):
                    assert all(((j, hk, x) in joined) == parts for x in range(G))
        for own in p["tok_own"][t:t + n[i]]:
            if r["own_seg"] < 0:
                assert own["nsplit"] == 0
            else:
                assert all(own[f] == p["segs"][r["own_seg"]][f] for f in OWN.names)
        t += int(n[i])


def refused(n, kv, blocks, **kw):
    base = dict(heads=8, kv_heads=2, head_dim=64, block_tokens=16, n_blocks=8)
    b, keep = step.make_batch(n, kv, blocks, **{**base, **kw})
    ctx = ctypes.c_void_p(1)
    rc = step.lib().tas_step_create(ctypes.byref(b), ctypes.byref(ctx))
    assert (rc == 0) == bool(ctx.value)
    step.tas_step_destroy(ctx.value)
    return rc == tas.TAS_EINVAL


def test_refused_batches():
    pages = [[0, 1], [2, 3]]
    assert not refused([1, 2], [20, 32], pages)
    assert not refused([0, 0], [0, 0], pages)
    for bad in (dict(heads=0), dict(heads=7), dict(kv_heads=0), dict(heads=2048, kv_heads=2),
                dict(head_dim=96), dict(head_dim=0), dict(block_tokens=8),
                dict(block_tokens=48), dict(block_tokens=8192), dict(n_blocks=0),
                dict(n_blocks=3)):
        assert refused([1, 2], [20, 32], pages, **bad), bad
    assert refused([-1, 2], [20, 32], pages)
    assert refused([1, 2], [-1, 32], pages)
    assert refused([1, 2], [33, 32], pages)          # three blocks of a table of two
    assert refused([1, 2], [20, 32], [[0, 8], [2, 3]])
    assert refused([1, 2], [20, 32], [[-1, 1], [2, 3]])
    assert not refused([1, 2], [16, 32], [[0, -1], [2, 3]])   # not reached
    assert refused([1, 1], [20, 32], [[0, 1], [2, 1]])        # one slot's block twice
    assert not refused([1, 1], [20, 32], [[0, 1], [0, 3]])    # read by both, written by neither
    assert refused([20, 1], [20, 1], [[5, 5], [2, 3]])
    assert refused([1 << 25, 1], [1 << 25, 1], pages)
    many = np.arange(1 << 16).reshape(1, -1)
    assert not refused([1 << 19], [1 << 19], many, n_blocks=1 << 16, heads=32)
    assert refused([1 << 20], [1 << 20], many, n_blocks=1 << 16, heads=1024, kv_heads=1024)


def test_refused_prefixes():
    pages = [[0, 1], [2, 3]]
    good = dict(prefix_first=[0, 1, 2], prefix_len=[20, 0], prefix_blocks=[[4, 5], [6, 7]])
    assert not refused([1, 2], [20, 32], pages, **good)
    for bad in (dict(prefix_first=[0, 1, 1]), dict(prefix_first=[1, 1, 2]),
                dict(prefix_first=[0, 2, 1]), dict(prefix_first=[0, 3, 2]),
                dict(prefix_len=[-1, 0]), dict(prefix_len=[33, 0]),
                dict(prefix_blocks=[[4, 8], [6, 7]]), dict(prefix_blocks=[[4, -1], [6, 7]])):
        assert refused([1, 2], [20, 32], pages, **{**good, **bad}), bad
    with pytest.raises(ValueError):
        step.make_batch([1], [1], [[0]], heads=1, kv_heads=1, head_dim=64, block_tokens=16,
                        n_blocks=1, prefix_first=[0, 1], prefix_len=[1, 2], prefix_blocks=[[0]])
    with pytest.raises(ValueError):
        step.make_batch([1, 2], [1], [[0]], heads=1, kv_heads=1, head_dim=64, block_tokens=16,
                        n_blocks=1)


def test_refused_values():
    """Nothing is cut to 32 bits or rounded on the way to the C structs."""
    kw = dict(heads=1, kv_heads=1, head_dim=64, block_tokens=16, n_blocks=4)
    step.make_batch(np.array([1], np.int64), np.array([1], np.uint8), [[0]], **kw)
    for n, kv, bl in (([1], [2 ** 32 + 1], [[0]]), ([2 ** 31], [1], [[0]]),
                      ([1], [1], [[-2 ** 31 - 1]]), ([1.5], [1], [[0]]), ([1], [1], [[0.0]]),
                      ([True], [1], [[0]])):
        with pytest.raises(ValueError):
            step.make_batch(n, kv, bl, **kw)


def test_null_arguments_and_unbound_steps():
    L = step.lib()
    assert L.tas_step_bytes(None) == 0 and L.tas_step_tokens(None) == -1
    assert L.tas_step_create(None, None) == tas.TAS_EINVAL
    assert L.tas_step_bind(None, None, 0, None) == tas.TAS_EINVAL
    assert L.tas_step_append(None, None, None) == tas.TAS_EINVAL
    assert L.tas_step_attention(None, None, None) == tas.TAS_EINVAL
    assert L.tas_step_plan(None, None, 0, None) == tas.TAS_EINVAL
    L.tas_step_destroy(None)
    b, keep = step.make_batch([1, 1], [1, 1], [[0], [1]], heads=1, kv_heads=1, head_dim=64,
                              block_tokens=16, n_blocks=2)
    ctx = step.tas_step_create(b)
    need, n = step.tas_step_bytes(ctx), ctypes.c_size_t()
    # refused before the address is used
    assert L.tas_step_bind(ctx, 1 << 40, need - 1, None) == tas.TAS_ENOMEM
    assert L.tas_step_bind(ctx, (1 << 40) + 16, need, None) == tas.TAS_EINVAL
    assert L.tas_step_bind(ctx, None, need, None) == tas.TAS_EINVAL
    assert L.tas_step_append(ctx, ctypes.byref(step.tas_append()), None) == tas.TAS_ESTATE
    assert L.tas_step_attention(ctx, ctypes.byref(step.tas_attention()), None) == tas.TAS_ESTATE
    buf = ctypes.create_string_buffer(8)
    assert L.tas_step_plan(ctx, buf, 8, ctypes.byref(n)) == tas.TAS_ENOMEM
    step.tas_step_destroy(ctx)
    b.blocks = None
    with pytest.raises(tas.TasError):
        step.tas_step_create(b)


def test_library_exports_every_declared_symbol():
    src = open(os.path.join(ROOT, "include", "tas_step.h")).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    names = sorted(set(re.findall(r"\b(tas_step_[a-z_]+)\s*\(", src)))
    assert names == sorted(step.EXPORTS)
    for n in names:
        assert hasattr(step.lib(), n), n


def test_struct_layouts_match_header(tmp_path):
    structs = [step.tas_batch, step.tas_cache, step.tas_append, step.tas_attention]
    lines = ['#include <stddef.h>', '#include <stdio.h>', '#include "tas_step.h"',
             'int main(void) {']
    for st in structs:
        n = st.__name__
        lines.append(f'printf("{n} %zu\\n", sizeof({n}));')
        for f, _ in st._fields_:
            lines.append(f'printf("{n}.{f} %zu\\n", offsetof({n}, {f}));')
    lines.append('return 0; }')
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines))
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), "-o", str(exe),
                           str(src)])
    got = dict(x.split() for x in subprocess.check_output([str(exe)], text=True).splitlines())
    for st in structs:
        assert int(got[st.__name__]) == ctypes.sizeof(st)
        for f, _ in st._fields_:
            assert int(got[f"{st.__name__}.{f}"]) == getattr(st, f).offset, f


@pytest.mark.parametrize("left_out", ["prefix_first", "prefix_len", "prefix_blocks"])
def test_prefix_arguments_go_together(left_out):
    """A prefix that is only half described is refused, not left out."""
    kw = dict(heads=1, kv_heads=1, head_dim=64, block_tokens=16, n_blocks=4)
    prefix = dict(prefix_first=[0, 1], prefix_len=[20], prefix_blocks=[[1, 2]])
    b, keep = step.make_batch([1], [1], [[0]], **kw, **prefix)
    assert b.n_prefix == 1
    del prefix[left_out]
    with pytest.raises(ValueError):
        step.make_batch([1], [1], [[0]], **kw, **prefix)
    for name, value in prefix.items():
        with pytest.raises(ValueError):
            step.make_batch([1], [1], [[0]], **kw, **{name: value})


@pytest.mark.parametrize("name", ["heads", "kv_heads", "head_dim", "block_tokens", "n_blocks"])
def test_refused_sizes(name):
    """No size is cut to 32 bits on the way to the C struct either."""
    kw = dict(heads=1, kv_heads=1, head_dim=64, block_tokens=16, n_blocks=4)
    b, keep = step.make_batch([1], [1], [[0]], **{**kw, name: np.int64(kw[name])})
    assert getattr(b, name) == kw[name]
    for value in (2 ** 32 + kw[name], 2 ** 31, -2 ** 31 - 1, -2 ** 32 + kw[name]):
        with pytest.raises(ValueError):
            step.make_batch([1], [1], [[0]], **{**kw, name: value})
    for value in (float(kw[name]), str(kw[name]), None):
        with pytest.raises(TypeError):
            step.make_batch([1], [1], [[0]], **{**kw, name: value})


def test_new_tokens_in_one_block_without_causality():
    """Without causality new tokens may be queries over any pages, shared ones too: the
    batch is planned. Only append would race; a causal batch stays refused."""
    pages = [[0, 1], [0, 1]]
    assert not refused([1, 1], [20, 20], pages, causal=False)
    assert not refused([1, 2], [20, 32], pages, causal=False)
    assert not refused([20], [20], [[5, 5]], causal=False)
    assert refused([1, 1], [20, 20], pages)
    assert refused([1, 2], [20, 32], pages)


def test_batches_of_more_workgroups_than_a_launch_takes():
    """A launch has fewer than 2^32 threads, 2^24 workgroups of 256: batches beyond that
    are refused when they are planned, not after append has written the cache."""
    # as many items: one for each request and key head
    n = 1 << 15
    one = np.arange(n).reshape(n, 1)
    assert refused(np.ones(n, int), np.ones(n, int), one, n_blocks=n, heads=512, kv_heads=512)
    # as many groups of 16 rows whose parts of a prefix are merged
    assert refused([1 << 22], [0], [[0]], heads=64, kv_heads=64, causal=False,
                   prefix_first=[0, 1], prefix_len=[16], prefix_blocks=[[1]])
    # tokens and heads to append, at 8 heads of a token to a wave
    n = 1 << 21
    kw = dict(heads=128, kv_heads=128, head_dim=128, block_tokens=4096, n_blocks=512)
    assert refused([n], [n], np.arange(512).reshape(1, -1), **kw)
    assert not refused([n // 8], [n // 8], np.arange(512).reshape(1, -1), **kw)


def test_workspace_of_the_callers_own_copy():
    """tas_step_attach takes what tas_step_bind takes, and copies nothing (host only)."""
    L = step.lib()
    b, keep = step.make_batch([1, 1], [1, 1], [[0], [1]], heads=1, kv_heads=1, head_dim=64,
                              block_tokens=16, n_blocks=2)
    ctx = step.tas_step_create(b)
    need = step.tas_step_bytes(ctx)
    assert L.tas_step_attach(None, 1 << 40, need) == tas.TAS_EINVAL
    assert L.tas_step_attach(ctx, None, need) == tas.TAS_EINVAL
    assert L.tas_step_attach(ctx, (1 << 40) + 16, need) == tas.TAS_EINVAL
    assert L.tas_step_attach(ctx, 1 << 40, need - 1) == tas.TAS_ENOMEM
    assert L.tas_step_append(ctx, ctypes.byref(step.tas_append()), None) == tas.TAS_ESTATE
    step.tas_step_attach(ctx, 1 << 40, need)  # (an address that nothing here uses)
    a = step.tas_append(dtype=7)
    assert L.tas_step_append(ctx, ctypes.byref(a), None) == tas.TAS_EINVAL  # bound: checked
    step.tas_step_destroy(ctx)
