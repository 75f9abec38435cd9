"""The operators of a serving iteration against their formulas in 64 bits on the
CPU, at the sizes where a kernel can go wrong: contexts that end inside a block, a
tile or a piece, one token, no key at all, groups of heads of every size, shared
prefixes, strided tensors, slots that nobody may read, other streams and graphs."""
import math

import numpy as np
import pytest

from paper_2606_18431_amd import step, tas

pytestmark = pytest.mark.gpu

# unit roundoffs; a result is rounded once, the softmax's weights once before
ROUND = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


@pytest.fixture(scope="module")
def torch():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def dtype_of(torch, name):
    return {"bf16": torch.bfloat16, "f16": torch.float16}[name]


class Batch:
    """A batch's host arrays, with pages taken from a shuffled pool."""

    def __init__(self, seed, n_new, kv_len, heads, kv_heads, size, block=16, first=None,
                 prefix=None, causal=True, extra=2):
        rng = np.random.default_rng(seed)
        self.n, self.kv = np.asarray(n_new), np.asarray(kv_len)
        self.heads, self.kv_heads, self.size, self.block = heads, kv_heads, size, block
        self.causal, self.first, self.prefix = causal, first, prefix
        need = [-(-int(k) // block) for k in self.kv]
        pre = [-(-p // block) for p in (prefix or [])]
        self.n_blocks = sum(need) + sum(pre) + extra
        ids = rng.permutation(self.n_blocks).astype(np.int32)
        self.blocks = np.full((len(self.n), max(need + [1])), -1, np.int32)
        at = 0
        for i, m in enumerate(need):
            self.blocks[i, :m] = ids[at:at + m]
            at += m
        self.prefix_blocks = None
        if prefix:
            self.prefix_blocks = np.full((len(pre), max(pre + [1])), -1, np.int32)
            for i, m in enumerate(pre):
                self.prefix_blocks[i, :m] = ids[at:at + m]
                at += m
        self.T = int(self.n.sum())

    def step(self):
        return step.Step(self.n, self.kv, self.blocks, heads=self.heads, kv_heads=self.kv_heads,
                         head_dim=self.size, block_tokens=self.block, n_blocks=self.n_blocks,
                         prefix_first=self.first, prefix_len=self.prefix,
                         prefix_blocks=self.prefix_blocks, causal=self.causal)

    def group(self, i):
        return int(np.searchsorted(self.first, i, side="right") - 1) if self.prefix else None

    def slots(self, i):
        """(block, offset) of every key that request i may read: prefix, own."""
        b = self.block
        out = []
        if self.prefix:
            g = self.group(i)
            out += [(self.prefix_blocks[g, y // b], y % b) for y in range(self.prefix[g])]
        out += [(self.blocks[i, y // b], y % b) for y in range(int(self.kv[i]))]
        return np.asarray(out, np.int64).reshape(-1, 2)

    def positions(self):
        pre = [self.prefix[self.group(i)] if self.prefix else 0 for i in range(len(self.n))]
        return np.concatenate([np.arange(p + k - n, p + k)
                               for p, n, k in zip(pre, self.n, self.kv)])


def reference(torch, b, q, k_cache, v_cache, scale, u):
    """(out, lse, tolerance of out, tolerance of lse) in float64."""
    q, G = q.double().cpu(), b.heads // b.kv_heads
    k_cache, v_cache = k_cache.double().cpu(), v_cache.double().cpu()
    out = torch.zeros((b.T, b.heads, b.size), dtype=torch.float64)
    lse = torch.full((b.T, b.heads), -math.inf, dtype=torch.float64)
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    t = 0
    for i in range(len(b.n)):
        n, kv = int(b.n[i]), int(b.kv[i])
        sl = b.slots(i)
        pre = len(sl) - kv
        if len(sl):
            k = k_cache[sl[:, 0], :, sl[:, 1]]  # [keys, Hk, D]
            v = v_cache[sl[:, 0], :, sl[:, 1]]
        for j in range(n):
            seen = pre + (max(0, min(kv, kv - n + 1 + j)) if b.causal else kv)
            if not seen:
                continue
            for h in range(b.kv_heads):
                qs = q[t + j, h * G:(h + 1) * G]
                kk, vv = k[:seen, h], v[:seen, h]
                s = scale * qs @ kk.T
                m = s.max(-1, keepdim=True).values
                w = torch.exp(s - m)
                l = w.sum(-1, keepdim=True)
                out[t + j, h * G:(h + 1) * G] = w @ vv / l
                lse[t + j, h * G:(h + 1) * G] = (m + l.log())[:, 0]
                # a score: size + 1 products and sums in 32 bits, then the scaled
                # difference's rounding; it moves a weight by as much
                d = 2.0 ** -24 * ((b.size + 4) * (scale * qs.abs() @ kk.abs().T).amax(-1)
                                  + 4 * s.abs().amax(-1)) + 2.0 ** -20
                mean = w @ vv.abs() / l
                # 16-bit floats: a weight below 2^-14 keeps 2^-25; sums of them in 32 bits
                small = seen * 2.0 ** -25 * vv.abs().amax(0) * (u == 2.0 ** -11)
                tol[t + j, h * G:(h + 1) * G] = \
                    (u * (out[t + j, h * G:(h + 1) * G].abs() + 1.01 * mean)
                     + (2 * d[:, None] + 2.0 ** -20) * mean + small + 2.0 ** -24)
                ltol[t + j, h * G:(h + 1) * G] = \
                    d + 2.0 ** -21 * (1 + lse[t + j, h * G:(h + 1) * G].abs())
        t += n
    return out, lse, tol, ltol


def caches(torch, b, dtype, seed, order="head", poison=True):
    """K and V of a pool whose slots nobody may read are NaN; views of the shape
    [blocks, kv_heads, block, size] in the given order of memory."""
    g = torch.Generator().manual_seed(seed)
    got = []
    both = torch.zeros((b.n_blocks, 2, b.kv_heads, b.block, b.size), dtype=dtype, device="cuda")
    for x in range(2):
        val = torch.randn((b.n_blocks, b.kv_heads, b.block, b.size), generator=g).to(dtype)
        if poison:
            seen = torch.zeros((b.n_blocks, b.block), dtype=torch.bool)
            for i in range(len(b.n)):
                sl = b.slots(i)
                seen[sl[:, 0], sl[:, 1]] = True
            val = torch.where(seen[:, None, :, None], val, torch.full_like(val, math.nan))
        if order == "head":
            c = val.cuda()
        elif order == "token":
            c = val.permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3)
        else:  # K and V of a block beside each other
            both[:, x] = val.cuda()
            c = both[:, x]
        got.append(c)
    return got


def near(got, want, tol, what):
    got = got.double().cpu()
    assert got.shape == want.shape
    ok = (got == want) | ((got - want).abs() <= tol)
    if not bool(ok.all()):
        at = (~ok).nonzero()[0].tolist()
        raise AssertionError(f"{what}: {int((~ok).sum())} of {ok.numel()} off, first at {at}: "
                             f"{got[tuple(at)]} for {want[tuple(at)]}, tolerance {tol[tuple(at)]}")


def check_attention(torch, b, name, seed=1, order="head", scale=None):
    print(f"[gpu] attention {name} n={b.n.tolist()[:8]} kv={b.kv.tolist()[:8]} heads="
          f"{b.heads}/{b.kv_heads}x{b.size} block={b.block} prefix={b.prefix}", flush=True)
    dt = dtype_of(torch, name)
    k, v = caches(torch, b, dt, seed, order)
    g = torch.Generator().manual_seed(seed + 100)
    q = (2 * torch.randn((b.T, b.heads, b.size), generator=g)).to(dt)
    sc = scale if scale is not None else b.size ** -0.5
    want, wlse, tol, ltol = reference(torch, b, q, k, v, sc, ROUND[name])
    s = b.step()
    lse = torch.full((b.T, b.heads), 7.0, device="cuda")
    out = s.attention(q.cuda(), k, v, scale=scale, lse=lse)
    torch.cuda.synchronize()
    near(out, want, tol, "out")
    near(lse, wlse, ltol, "lse")


EDGES = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 1000]


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("size", [64, 128])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (6, 2), (7, 1), (16, 1), (20, 4), (64, 2)])
def test_decode(torch, name, size, heads, kv_heads):
    check_attention(torch, Batch(3, [1] * len(EDGES), EDGES, heads, kv_heads, size), name)


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("size", [64, 128])
@pytest.mark.parametrize("block", [16, 64, 256])
def test_mixed_batch(torch, name, size, block):
    n = [1, 3, 0, 40, 130, 1, 257, 5]
    kv = [300, 3, 70, 41, 130, 1, 600, 90]
    check_attention(torch, Batch(4, n, kv, 12, 4, size, block), name)


@pytest.mark.parametrize("n,kv", [(1, 5000), (1, 33000), (16, 4111), (129, 2050)])
def test_few_rows_over_a_long_context(torch, n, kv):
    """One request: its keys are cut into pieces and the partial results joined."""
    check_attention(torch, Batch(5, [n], [kv], 2, 1, 128), "bf16")
    check_attention(torch, Batch(5, [n], [kv], 3, 3, 64), "f16")


@pytest.mark.parametrize("n,kv", [(17, 17), (64, 64), (65, 200), (128, 128), (127, 129)])
@pytest.mark.parametrize("group", [1, 5, 8])
def test_chunk_edges(torch, n, kv, group):
    check_attention(torch, Batch(6, [n], [kv], 2 * group, 2, 128), "bf16")


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("prefix", [[1], [15], [16], [100], [700]])
def test_shared_prefix(torch, name, prefix):
    n = [1] * 9
    kv = [1, 5, 16, 17, 300, 2, 64, 90, 33]
    check_attention(torch, Batch(7, n, kv, 16, 4, 128, first=[0, 9], prefix=prefix), name)
    n = [3, 1, 5, 2, 0, 40, 1, 1, 4]
    kv = [3, 5, 16, 17, 20, 44, 64, 90, 33]
    check_attention(torch, Batch(8, n, kv, 8, 2, 64, first=[0, 9], prefix=prefix), name)


def test_prefix_groups(torch):
    """Groups of different lengths, one without a prefix, one without requests, one
    whose requests have no new tokens, one request with nothing but its prefix."""
    n = [1, 2, 1, 0, 0, 3, 1, 30, 1, 1]
    kv = [40, 2, 300, 4, 9, 3, 1, 31, 200, 0]
    b = Batch(9, n, kv, 6, 2, 128, first=[0, 3, 3, 5, 7, 10], prefix=[50, 16, 7, 0, 130],
              causal=False)
    check_attention(torch, b, "bf16")
    kv[-1] = 1
    b = Batch(9, n, kv, 6, 2, 128, first=[0, 3, 3, 5, 7, 10], prefix=[50, 16, 7, 0, 130])
    check_attention(torch, b, "f16")


@pytest.mark.parametrize("causal", [True, False])
def test_rows_without_keys(torch, causal):
    """More new tokens than keys: the first rows see nothing (causal); requests
    without any key give zeros and -inf, in thin and wide items."""
    n = [1, 5, 40, 200, 2, 1]
    kv = [0, 2, 0, 150, 90, 0]
    check_attention(torch, Batch(10, n, kv, 4, 2, 64, causal=causal), "bf16")
    check_attention(torch, Batch(10, n, kv, 4, 1, 128, causal=causal), "f16")


@pytest.mark.parametrize("order", ["token", "beside"])
def test_other_cache_orders(torch, order):
    n, kv = [1, 40, 1, 300], [100, 90, 17, 400]
    check_attention(torch, Batch(11, n, kv, 8, 2, 128, block=32), "bf16", order=order)


def test_scale_and_large_scores(torch):
    """Scores of some hundreds: only differences to the maximum reach the exponent."""
    check_attention(torch, Batch(12, [1, 33], [200, 333], 4, 2, 64), "f16", scale=4.0)
    check_attention(torch, Batch(12, [1, 33], [200, 333], 4, 2, 64), "bf16", scale=1e-4)


def test_infinite_and_nan_keys_stay_with_their_rows(torch):
    """A non-finite value in one request's context reaches its rows and no others;
    a score of -inf is a weight of 0."""
    b = Batch(13, [1, 1, 20], [50, 70, 90], 4, 2, 128)
    k, v = caches(torch, b, torch.bfloat16, 3)
    q = torch.randn((b.T, 4, 128)).to(torch.bfloat16).abs().cuda()
    s = b.step()
    clean = s.attention(q, k, v)
    k2, v2 = k.clone(), v.clone()
    v2[b.blocks[1, 1], 0, 3, 5] = math.nan     # request 1, key 19, key head 0
    k2[b.blocks[0, 0], 1, 2] = -math.inf       # request 0, key 2, key head 1: weight 0
    got = s.attention(q, k2, v2)
    assert torch.isnan(got[1, :2, 5]).all() and torch.isfinite(got[0]).all()
    same = torch.ones_like(clean, dtype=torch.bool)
    same[1, :2, 5] = False
    same[0, 2:] = False
    assert torch.equal(got[same], clean[same])
    v3 = v.clone()
    v3[b.blocks[0, 0], 1, 2] = 0
    k3 = k.clone()
    k3[b.blocks[0, 0], 1, 2] = -1000           # as good as -inf
    want = s.attention(q, k3, v3)
    assert torch.equal(got[0, 2:], want[0, 2:])


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("size", [64, 128])
@pytest.mark.parametrize("n,kv,heads", [(5, 40, 2), (3, 90, 10), (70, 70, 1), (200, 333, 2),
                                        (150, 160, 8)])
def test_values_after_a_token_do_not_reach_it(torch, name, size, n, kv, heads):
    """A new token's V that is infinite or NaN makes the tokens from it on NaN (a row as
    a whole, or the element) and leaves those before it as they were."""
    b = Batch(33, [n], [kv], heads, 1, size)
    k, v = caches(torch, b, dtype_of(torch, name), 3)
    q = torch.randn((n, heads, size)).to(k.dtype).cuda()
    s = b.step()
    clean = s.attention(q, k, v)
    for bad in (n - 1, n // 2, n // 3):
        for value in (math.nan, math.inf, -math.inf):
            y = kv - n + bad
            v2 = v.clone()
            v2[b.blocks[0, y // 16], 0, y % 16, 7] = value
            got = s.attention(q, k, v2)
            assert torch.equal(got[:bad], clean[:bad])
            assert not torch.isfinite(got[bad:, :, 7]).any()
            k2 = k.clone()
            k2[b.blocks[0, y // 16], 0, y % 16] = value
            assert torch.equal(s.attention(q, k2, v)[:bad], clean[:bad])


def test_strided_queries_output_in_place_and_determinism(torch):
    b = Batch(14, [1, 60, 3], [3000, 80, 700], 8, 2, 128)
    k, v = caches(torch, b, torch.bfloat16, 4)
    qkv = torch.randn((b.T, 12, 128), device="cuda").to(torch.bfloat16)
    q = qkv[:, :8]
    s = b.step()
    want = s.attention(q.contiguous(), k, v)
    assert torch.equal(s.attention(q, k, v), want)          # rows apart
    wide = torch.full((b.T, 10, 128), 3.0, device="cuda", dtype=torch.bfloat16)
    s.attention(q, k, v, out=wide[:, 1:9])
    assert torch.equal(wide[:, 1:9], want)
    assert bool((wide[:, 0] == 3).all()) and bool((wide[:, 9] == 3).all())
    assert s.attention(q, k, v, out=q).data_ptr() == qkv.data_ptr()
    assert torch.equal(q, want)


def test_other_streams_and_graphs(torch):
    b = Batch(15, [1, 1, 50], [2000, 17, 400], 8, 2, 64)
    k, v = caches(torch, b, torch.float16, 5)
    s = b.step()
    q = torch.randn((b.T, 8, 64), device="cuda").half()
    want = s.attention(q, k, v)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = s.attention(q, k, v, stream=side)
    with torch.cuda.stream(side):
        again = s.attention(q, k, v)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want) and torch.equal(again, want)
    # a graph replayed on new contents of its inputs, with other work in between
    qkv = torch.empty((b.T, 12, 64), device="cuda", dtype=torch.float16)
    cos, sin = torch.rand((2100, 32), device="cuda"), torch.rand((2100, 32), device="cuda")
    out = torch.empty_like(q)
    kg, vg = k.clone(), v.clone()

    def body():
        x = s.append(qkv, kg, vg, cos, sin)
        s.attention(x, kg, vg, out=out)

    qkv.normal_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        body()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        body()
    for i in range(4):
        qkv.normal_()
        graph.replay()
        torch.cuda.synchronize()
        ke, ve = k.clone(), v.clone()
        x = s.append(qkv, ke, ve, cos, sin)
        assert torch.equal(out, s.attention(x, ke, ve)), i
        assert torch.equal(ke.nan_to_num(), kg.nan_to_num())
        torch.cuda.synchronize()


def test_blocks_beyond_four_gigabytes(torch):
    """Offsets that pass 32 bits: the pages lie at the far end of a pool of 9 GB."""
    n_blocks, shape = 1 << 17, (1 << 17, 8, 16, 128)
    k = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    v = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    kv = [100, 700]
    small = Batch(16, [1, 70], kv, 8, 8, 128)
    ks, vs = caches(torch, small, torch.bfloat16, 6)
    far = np.where(small.blocks >= 0, n_blocks - 1 - small.blocks, -1)
    order = torch.arange(small.n_blocks)
    k[(n_blocks - 1 - order).cuda()] = ks
    v[(n_blocks - 1 - order).cuda()] = vs
    s = step.Step(small.n, small.kv, far, heads=8, kv_heads=8, head_dim=128, block_tokens=16,
                  n_blocks=n_blocks)
    qkv = torch.randn((71, 24, 128), device="cuda").to(torch.bfloat16)
    q1 = small.step().append(qkv, ks, vs)
    q2 = s.append(qkv, k, v)
    assert torch.equal(q1, q2)
    back = (n_blocks - 1 - order).cuda()
    assert torch.equal(k[back].nan_to_num(), ks.nan_to_num())
    assert torch.equal(v[back].nan_to_num(), vs.nan_to_num())
    assert torch.equal(s.attention(q2, k, v), small.step().attention(q1, ks, vs))


# ------------------------------------------------------------------ append


def append_reference(torch, b, qkv, cos, sin, qw, kw, eps, interleaved):
    """(values of all heads, tolerance before rounding) in float64."""
    x = qkv.double().cpu()
    H, Hk, D = b.heads, b.kv_heads, b.size
    y, tol = x.clone(), torch.zeros_like(x)
    pos = b.positions()
    for h in range(H + Hk):
        u = x[:, h]
        if qw is not None:
            w = (qw if h < H else kw).double().cpu()
            u = u / torch.sqrt((u * u).mean(-1, keepdim=True) + eps) * w
        z, size = u.clone(), u.abs()
        if cos is not None:
            R = 2 * cos.shape[1]
            c, s = cos.double().cpu()[pos], sin.double().cpu()[pos]
            first = np.arange(0, R, 2) if interleaved else np.arange(R // 2)
            second = first + 1 if interleaved else first + R // 2
            z[:, first] = u[:, first] * c - u[:, second] * s
            z[:, second] = u[:, second] * c + u[:, first] * s
            size = size.clone()
            size[:, first] = u[:, first].abs() * c.abs() + u[:, second].abs() * s.abs()
            size[:, second] = u[:, second].abs() * c.abs() + u[:, first].abs() * s.abs()
        y[:, h], tol[:, h] = z, size
    # the norm: D squares and sums, a root, a division, two products; the rotation: three
    return y, tol * (D + 12) * 2.0 ** -24


def check_append(torch, b, name, rot, interleaved, norm, order="head"):
    print(f"[gpu] append {name} n={b.n.tolist()[:8]} heads={b.heads}/{b.kv_heads}x{b.size} "
          f"block={b.block} rot={rot} interleaved={interleaved} norm={norm}", flush=True)
    dt = dtype_of(torch, name)
    k, v = caches(torch, b, dt, 8, order, poison=False)
    k0, v0 = k.clone(), v.clone()
    g = torch.Generator().manual_seed(77)
    H, Hk, D = b.heads, b.kv_heads, b.size
    qkv = torch.randn((b.T, H + 2 * Hk, D), generator=g).to(dt).cuda()
    qkv[-1, 0] = 0  # a head of zeros
    cos = sin = qw = kw = None
    if rot:
        a = torch.rand((int(b.positions().max()) + 1, rot // 2), generator=g) * 6.3
        cos, sin = a.cos().cuda(), a.sin().cuda()
    if norm:
        qw, kw = (1 + 0.2 * torch.randn((2, D), generator=g)).to(dt).cuda()
    want, tol = append_reference(torch, b, qkv, cos, sin, qw, kw, 1e-5, interleaved)
    s = b.step()
    q = s.append(qkv, k, v, cos, sin, q_weight=qw, k_weight=kw, eps=1e-5,
                 interleaved=interleaved)
    torch.cuda.synchronize()
    # below the smallest normal number a 16-bit float keeps 2^-25
    tol = tol + ROUND[name] * want.abs() * 1.01 + (2.0 ** -25 if name == "f16" else 2.0 ** -140)
    near(q, want[:, :H], tol[:, :H], "queries")
    t = 0
    for i in range(len(b.n)):
        sl = b.slots(i)[len(b.slots(i)) - int(b.n[i]):]
        for (page, at) in sl:
            near(k[page, :, at], want[t, H:H + Hk], tol[t, H:H + Hk], "keys")
            assert torch.equal(v[page, :, at], qkv[t, H + Hk:])
            k0[page, :, at], v0[page, :, at] = k[page, :, at], v[page, :, at]
            t += 1
    assert torch.equal(k, k0) and torch.equal(v, v0)  # nothing else was written


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("size,rot", [(64, 64), (64, 32), (64, 16), (128, 128), (128, 64),
                                      (128, 96), (128, 0)])
def test_append(torch, name, size, rot, interleaved):
    n, kv = [1, 5, 0, 37, 1], [33, 5, 9, 100, 1]
    check_append(torch, Batch(20, n, kv, 6, 2, size), name, rot, interleaved, norm=rot != 32)
    check_append(torch, Batch(21, n, kv, 7, 7, size, block=32, first=[0, 2, 5], prefix=[20, 7]),
                 name, rot, interleaved, norm=rot == 32, order="token")


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (8, 1), (33, 3)])
def test_append_heads(torch, heads, kv_heads):
    check_append(torch, Batch(22, [1, 3], [1, 60], heads, kv_heads, 128), "bf16", 128, False, True)
    check_append(torch, Batch(22, [1, 3], [1, 60], heads, kv_heads, 64), "f16", 64, True, True,
                 order="beside")


# ------------------------------------------------------------------ refusals


def test_refused_arguments(torch):
    b = Batch(30, [1, 4], [30, 20], 4, 2, 64)
    k, v = caches(torch, b, torch.bfloat16, 9)
    s = b.step()
    assert s.tokens == 5
    q = torch.zeros((5, 4, 64), device="cuda", dtype=torch.bfloat16)
    qkv = torch.zeros((5, 8, 64), device="cuda", dtype=torch.bfloat16)
    cos = torch.zeros((30, 32), device="cuda")
    s.attention(q, k, v)
    s.append(qkv, k, v, cos, cos)
    for bad in (q.float(), q.half(), q[:4], q[:, :3], q.cpu(), q.transpose(0, 1).contiguous(),
                torch.zeros((5, 4, 128), device="cuda", dtype=torch.bfloat16)[..., ::2]):
        with pytest.raises(ValueError):
            s.attention(bad, k, v)
    for bk in (k[1:], k.half(), k.cpu(), k.transpose(2, 3), k[:, :1]):
        with pytest.raises(ValueError):
            s.attention(q, bk, v)
        with pytest.raises(ValueError):
            s.append(qkv, k, bk)
    for kw in (dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan)):
        with pytest.raises(tas.TasError) as e:
            s.attention(q, k, v, **kw)
        assert e.value.code == tas.TAS_EINVAL
    for lse in (torch.zeros((5, 4)), torch.zeros((4, 5), device="cuda"),
                torch.zeros((5, 4), device="cuda", dtype=torch.float64)):
        with pytest.raises(ValueError):
            s.attention(q, k, v, lse=lse)
    odd = torch.zeros(5 * 4 * 64 + 4, device="cuda", dtype=torch.bfloat16)[4:].view(5, 4, 64)
    with pytest.raises(tas.TasError):  # 8-byte aligned
        s.attention(odd, k, v)
    apart = torch.zeros((5, 4 * 64 + 4), device="cuda", dtype=torch.bfloat16)
    with pytest.raises(tas.TasError):  # tokens 4 elements off the 16 bytes
        s.attention(apart[:, :256].view(5, 4, 64), k, v)
    for c, sn in ((cos[:29], cos[:29]), (cos[:, :4].contiguous(), cos[:, :4].contiguous()),
                  (torch.zeros((30, 40), device="cuda"),) * 2):
        with pytest.raises(tas.TasError):
            s.append(qkv, k, v, c, sn)
    for c, sn in ((cos, None), (cos, cos[:20]), (cos.half(), cos.half()), (cos.cpu(), cos.cpu()),
                  (cos.T, cos.T)):
        with pytest.raises(ValueError):
            s.append(qkv, k, v, c, sn)
    w = torch.ones(64, device="cuda", dtype=torch.bfloat16)
    for qw, kw in ((w, None), (w.float(), w.float()), (w[:32], w[:32])):
        with pytest.raises(ValueError):
            s.append(qkv, k, v, q_weight=qw, k_weight=kw)
    for eps in (-1.0, math.nan, math.inf):
        with pytest.raises(tas.TasError):
            s.append(qkv, k, v, q_weight=w, k_weight=w, eps=eps)
    # more new tokens than context: attention only
    few = Batch(31, [3], [2], 4, 2, 64)
    k2, v2 = caches(torch, few, torch.bfloat16, 9)
    f = few.step()
    f.attention(q[:3], k2, v2)
    with pytest.raises(tas.TasError):
        f.append(qkv[:3], k2, v2)
    s.close()
    with pytest.raises(ValueError):
        s.attention(q, k, v)
    with pytest.raises(tas.TasError):
        step.Step([1], [17], [[0]], heads=4, kv_heads=2, head_dim=64, block_tokens=16, n_blocks=4)


def test_batch_without_new_tokens(torch):
    b = Batch(32, [0, 0], [5, 0], 4, 2, 64)
    k, v = caches(torch, b, torch.float16, 9)
    s = b.step()
    q = torch.empty((0, 4, 64), device="cuda", dtype=torch.float16)
    assert s.attention(q, k, v).shape == (0, 4, 64)
    assert s.append(torch.empty((0, 8, 64), device="cuda", dtype=torch.float16), k, v).shape == \
        (0, 4, 64)


@pytest.mark.parametrize("shared", ["block", "head", "token", "half a token", "k is v"])
def test_append_refuses_slots_that_share_elements(torch, shared):
    """A broadcast cache can be attended to; its slots cannot be written."""
    b = Batch(33, [1, 4], [30, 20], 4, 2, 64)
    k, v = caches(torch, b, torch.bfloat16, 9, poison=False)
    s = b.step()
    qkv = torch.zeros((5, 8, 64), device="cuda", dtype=torch.bfloat16)
    bk, bv = {
        "block": (k[:1].expand_as(k), v),
        "head": (k, v[:, :1].expand_as(v)),
        "token": (k[:, :, :1].expand_as(k), v),
        "half a token": (k, v.as_strided(v.shape, (v.stride(0), v.stride(1), 32, 1))),
        "k is v": (k, k),
    }[shared]
    before = k.clone(), v.clone()
    with pytest.raises(tas.TasError) as e:
        s.append(qkv, bk, bv)
    assert e.value.code == tas.TAS_EINVAL
    assert torch.equal(k, before[0]) and torch.equal(v, before[1])
    s.attention(qkv[:, :4].contiguous(), bk, bv)
    s.append(qkv, k, v)


def test_append_takes_any_order_of_disjoint_slots(torch):
    """One block and one key head: their strides say nothing."""
    s = step.Step([2], [9], [[0]], heads=2, kv_heads=1, head_dim=64, block_tokens=16, n_blocks=1)
    qkv = torch.randn((2, 4, 64), device="cuda", dtype=torch.float16)
    k, v = torch.zeros((2, 16, 64), device="cuda", dtype=torch.float16)
    s.append(qkv, k.as_strided((1, 1, 16, 64), (0, 0, 64, 1)),
             v.as_strided((1, 1, 16, 64), (8, 8, 64, 1)))
    assert torch.equal(k[7:9], qkv[:, 2]) and torch.equal(v[7:9], qkv[:, 3])


def test_requests_over_the_same_pages(torch):
    """Queries of two requests over one context (no causality): attended as each by
    itself, and not appended, which would race."""
    kv, pages = [40, 40, 33], [[3, 1, 4], [3, 1, 4], [3, 1, 4]]
    kw = dict(heads=4, kv_heads=2, head_dim=64, block_tokens=16, n_blocks=5, causal=False)
    k, v = torch.randn((2, 5, 2, 16, 64), device="cuda", dtype=torch.bfloat16)
    q = torch.randn((23, 4, 64), device="cuda", dtype=torch.bfloat16)
    n = [1, 20, 2]
    s = step.Step(n, kv, pages, **kw)
    got = s.attention(q, k, v)
    t = 0
    for i in range(3):
        one = step.Step([n[i]], [kv[i]], [pages[i]], **kw)
        assert torch.equal(got[t:t + n[i]], one.attention(q[t:t + n[i]], k, v)), i
        t += n[i]
    with pytest.raises(tas.TasError) as e:
        s.append(torch.zeros((23, 8, 64), device="cuda", dtype=torch.bfloat16), k, v)
    assert e.value.code == tas.TAS_EINVAL


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("size", [64, 128])
@pytest.mark.parametrize("n,group", [(1, 4), (3, 8)])
def test_many_small_weights(torch, name, size, n, group):
    """One key has nearly all of the weight, and 8000 others 2^-25.5 of its each, which a
    16-bit float cannot hold beside 1: what they add to the row is not lost. (96 requests
    over the same pages, so that the keys of a row stay in one piece.)"""
    dt, keys, heads = dtype_of(torch, name), 8000, 8
    g = torch.Generator().manual_seed(5)
    k, v = torch.zeros((2, 500, heads, 16, size), dtype=dt)
    k[0, :, 0, 3] = 4.41796875                  # scores 17.67 = 25.5 log(2), and 0
    v[:] = (50 + 100 * torch.rand(v.shape, generator=g)).to(dt)
    v[0, :, 0] = 0
    q = torch.zeros((96 * n, heads * group, size), dtype=dt)
    q[..., 3] = 4
    s = step.Step([n] * 96, [keys] * 96, np.tile(np.arange(500), (96, 1)), heads=heads * group,
                  kv_heads=heads, head_dim=size, block_tokens=16, n_blocks=500, causal=False)
    got = s.attention(q.cuda(), k.cuda(), v.cuda(), scale=1.0)
    w = math.exp(-4 * float(k[0, 0, 0, 3]))
    flat = v.double().permute(1, 0, 2, 3).reshape(heads, keys, size)
    want = w * flat.sum(1) / (1 + w * (keys - 1))
    want = want.repeat_interleave(group, 0).expand(96 * n, -1, -1)
    # rounding of the result and of the weights; 16-bit floats keep weights of 2^7 down
    # to 2^-25, with an error of 2^-32 of the largest
    u = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}[name]
    tol = 2.01 * u * want + 2.0 ** -15 * want + (keys * 2.0 ** -32 * 150 if name == "f16" else 0)
    near(got, want, tol, "out")


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("n,heads", [(5, 2), (40, 1)])
def test_value_under_a_weight_of_zero(torch, name, n, heads):
    """A key of -inf (score -inf, weight 0) does not hide its value from the rows that see
    it: 0 times NaN is NaN."""
    b = Batch(34, [n], [n + 50], heads, 1, 64)
    k, v = caches(torch, b, dtype_of(torch, name), 3)
    q = (torch.rand((n, heads, 64)) + 0.1).to(k.dtype).cuda()
    s = b.step()
    clean = s.attention(q, k, v)
    bad = n // 2
    page, at = b.blocks[0, (50 + bad) // 16], (50 + bad) % 16
    k[page, 0, at] = -math.inf
    v[page, 0, at, 7] = math.nan
    got = s.attention(q, k, v)
    assert torch.equal(got[:bad], clean[:bad])
    assert not torch.isfinite(got[bad:, :, 7]).any()


def test_error_of_an_earlier_call_is_not_reported(torch):
    """A call that failed before, and whose error nobody took, is not this one's."""
    b = Batch(35, [1, 20], [30, 40], 4, 2, 64)
    k, v = caches(torch, b, torch.bfloat16, 9)
    s = b.step()
    qkv = torch.randn((21, 8, 64), device="cuda", dtype=torch.bfloat16)
    q, out = torch.empty((2, 21, 4, 64), device="cuda", dtype=torch.bfloat16)
    L = step.lib()
    try:
        assert L.hipSetDevice(1 << 20) != 0
        s.append(qkv, k, v, out=q)
        s.attention(q, k, v, out=out)
    finally:
        L.hipGetLastError()
    torch.cuda.synchronize()


def test_scale_beyond_the_exponent(torch):
    """A scale that is finite itself, but not in the base 2 of the kernels: refused, where
    every row would be NaN."""
    b = Batch(37, [1, 20], [30, 40], 4, 2, 64)
    k, v = caches(torch, b, torch.bfloat16, 9)
    q = torch.randn((21, 4, 64), device="cuda", dtype=torch.bfloat16)
    s = b.step()
    s.attention(q, k, v, scale=2.3e38)
    for scale in (2.4e38, 3e38, 3.4e38):
        with pytest.raises(tas.TasError) as e:
            s.attention(q, k, v, scale=scale)
        assert e.value.code == tas.TAS_EINVAL


def test_append_refuses_k_and_v_in_one_place(torch):
    """K and V that are parts of one pool: a block further on their slots are the same
    memory, which new keys and values would race for; beside each other they are not."""
    b = Batch(39, [1, 4], [30, 20], 4, 2, 64)
    n = b.n_blocks
    s = b.step()
    qkv = torch.randn((5, 8, 64), device="cuda", dtype=torch.bfloat16)
    pool = torch.zeros((2 * n, 2, 16, 64), device="cuda", dtype=torch.bfloat16)
    for k, v in ((pool[:n], pool[1:n + 1]), (pool[1:n + 1], pool[:n]), (pool[:n], pool[:n]),
                 (pool.flatten()[8:8 + pool[:n].numel()].view_as(pool[:n]), pool[n:])):
        with pytest.raises(tas.TasError) as e:
            s.append(qkv, k, v)
        assert e.value.code == tas.TAS_EINVAL
        assert not pool.any()
    wide = torch.zeros((n, 2, 16, 128), device="cuda", dtype=torch.bfloat16)
    beside = torch.zeros((n, 2, 2, 16, 64), device="cuda", dtype=torch.bfloat16)
    last = torch.zeros((n, 2, 16, 2, 64), device="cuda", dtype=torch.bfloat16)
    want = None
    for k, v in ((pool[:n], pool[n:]), (pool[::2], pool[1::2]), (wide[..., :64], wide[..., 64:]),
                 (beside[:, 1], beside[:, 0]), (last[:, :, :, 0], last[:, :, :, 1])):
        k.zero_(), v.zero_()
        s.append(qkv, k, v)
        want = want or (k.clone(), v.clone())
        assert torch.equal(k, want[0]) and torch.equal(v, want[1])


def test_outputs_over_other_tensors(torch):
    """An output may be its input's own rows, or lie between rows; over other rows, heads
    or the cache it is refused, and nothing is written."""
    b = Batch(40, [1, 4, 60], [300, 20, 90], 4, 2, 64)
    k, v = caches(torch, b, torch.bfloat16, 9, poison=False)
    s = b.step()
    T = b.T
    buf = torch.randn((T + 1, 16, 64), device="cuda", dtype=torch.bfloat16)
    qkv = buf[:T, :8]
    ke, ve = k.clone(), v.clone()
    cos, sin = torch.rand((2, 300, 32), device="cuda")
    want_q = s.append(qkv.contiguous(), ke, ve, cos, sin)
    want = s.attention(want_q, ke, ve)
    first = buf.clone(), k.clone(), v.clone()
    flat = k.flatten()[:T * 4 * 64].view(T, 4, 64)
    for out in (qkv[:, 1:5], qkv[:, 4:8], buf[1:, :4], buf[:T, 6:10], flat,
                buf.flatten()[8:].as_strided((T, 4, 64), (1024, 64, 1)),
                buf.flatten()[:T * 256].view(T, 4, 64)):
        with pytest.raises(tas.TasError) as e:
            s.append(qkv, k, v, cos, sin, out=out)
        assert e.value.code == tas.TAS_EINVAL
    inside = v.flatten()[:T * 8 * 64].view(T, 8, 64)
    with pytest.raises(tas.TasError):
        s.append(inside, k, v, cos, sin)
    assert all(torch.equal(x, y) for x, y in zip(first, (buf, k, v)))
    k1, v1 = k.clone(), v.clone()
    s.append(qkv, k1, v1, cos, sin, out=buf[:T, 8:12])
    assert torch.equal(buf[:T, 8:12], want_q) and torch.equal(k1, ke) and torch.equal(v1, ve)
    k1, v1 = k.clone(), v.clone()
    s.append(qkv, k1, v1, cos, sin, out=qkv[:, :4])  # in place
    assert torch.equal(qkv[:, :4], want_q) and torch.equal(k1, ke) and torch.equal(v1, ve)
    assert torch.equal(buf[:T, 4:8], first[0][:T, 4:8])

    q, first = buf[:T, :4], buf.clone()
    for out in (buf[1:, :4], buf[:T, 1:5], ke.flatten()[:T * 256].view(T, 4, 64),
                buf.flatten()[:T * 256].view(T, 4, 64)):
        with pytest.raises(tas.TasError) as e:
            s.attention(q, ke, ve, out=out)
        assert e.value.code == tas.TAS_EINVAL
    assert torch.equal(buf, first) and torch.equal(k1, ke)
    s.attention(q, ke, ve, out=buf[:T, 4:8])
    assert torch.equal(buf[:T, 4:8], want)
    s.attention(q, ke, ve, out=q)
    assert torch.equal(q, want)


def test_tensors_dropped_while_another_stream_uses_them(torch):
    """Memory of a call's tensors is not reused before the call on its stream is done."""
    b = Batch(41, [1, 40], [300, 90], 4, 2, 64)
    k, v = caches(torch, b, torch.bfloat16, 9, poison=False)
    s = b.step()
    qkv = torch.randn((b.T, 8, 64), device="cuda", dtype=torch.bfloat16)
    cos, sin = torch.rand((2, 300, 32), device="cuda")
    ke, ve = k.clone(), v.clone()
    want_q = s.append(qkv, ke, ve, cos, sin)
    want = s.attention(want_q, ke, ve)
    a = torch.randn((8192, 8192), device="cuda", dtype=torch.bfloat16)
    a @ a
    side = torch.cuda.Stream()

    def busy():
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for _ in range(250):
                torch.mm(a, a)

    def dropped(call, tensors):
        """The call's result on the busy stream; the tensors' memory asked for again."""
        torch.cuda.synchronize()
        tensors = [t.clone() for t in tensors]
        busy()
        out = call(*tensors)
        places = {t.data_ptr() for t in tensors}
        sizes = [t.numel() * t.element_size() for t in tensors]
        del tensors
        again = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes]
        assert not places & {t.data_ptr() for t in again}
        side.synchronize()
        return out

    got = dropped(lambda *t: s.append(*t, stream=side), [qkv, k, v, cos, sin])
    assert torch.equal(got, want_q)
    got = dropped(lambda *t: s.attention(*t, stream=side), [want_q, ke, ve])
    assert torch.equal(got, want)


def test_planning_does_not_wait_for_the_device(torch):
    """A step is made while the device still works on what came before; its calls come
    after that, and its workspace is not one that the work before still uses."""
    b = Batch(36, [1, 20], [30, 40], 4, 2, 64)
    k, v = caches(torch, b, torch.bfloat16, 9, poison=False)
    q = torch.randn((21, 4, 64), device="cuda", dtype=torch.bfloat16)
    want = b.step().attention(q, k, v)
    a = torch.randn((8192, 8192), device="cuda", dtype=torch.bfloat16)
    a @ a
    torch.cuda.synchronize()
    done = torch.cuda.Event()
    for _ in range(250):
        a @ a
    done.record()
    got = [b.step().attention(q, k, v) for _ in range(5)]
    assert not done.query()
    assert all(torch.equal(x, want) for x in got)


def test_a_backward_pass_is_refused(torch):
    """An input's gradient is not lost without a word; values are those without one."""
    b = Batch(38, [1, 20], [30, 40], 4, 2, 64)
    k, v = caches(torch, b, torch.bfloat16, 9)
    s = b.step()
    q = torch.randn((21, 4, 64), device="cuda", dtype=torch.bfloat16)
    qkv = torch.randn((21, 8, 64), device="cuda", dtype=torch.bfloat16)
    w = torch.ones(64, device="cuda", dtype=torch.bfloat16)
    cos = torch.rand((40, 32), device="cuda")
    want = s.attention(q, k, v)
    assert not want.requires_grad

    def grad(t):
        return t.detach().clone().requires_grad_()

    for args in ((grad(q), k, v), (q, grad(k), v), (q, k, grad(v))):
        out = s.attention(*args)
        assert out.requires_grad and torch.equal(out, want)
        with pytest.raises(NotImplementedError):
            out.float().sum().backward()
        given = torch.empty_like(q)
        assert s.attention(*args, out=given).data_ptr() == given.data_ptr()
        assert torch.equal(given, want) and not given.requires_grad
        with torch.no_grad():
            assert not s.attention(*args).requires_grad
        with torch.inference_mode():
            assert torch.equal(s.attention(*args), want)
    x = s.append(qkv, k, v, cos, cos, q_weight=w, k_weight=w)
    assert not x.requires_grad
    for args in ((grad(qkv), cos, cos, w, w), (qkv, grad(cos), cos, w, w),
                 (qkv, cos, grad(cos), w, w), (qkv, cos, cos, grad(w), w),
                 (qkv, cos, cos, w, grad(w))):
        out = s.append(args[0], k, v, args[1], args[2], q_weight=args[3], k_weight=args[4])
        assert out.requires_grad and torch.equal(out, x)
        with pytest.raises(NotImplementedError):
            out.float().sum().backward()
        with torch.no_grad():
            assert not s.append(args[0], k, v, args[1], args[2], q_weight=args[3],
                                k_weight=args[4]).requires_grad
    assert not s.append(grad(qkv).detach(), k, v).requires_grad


def test_plan_under_way(torch):
    """While a step's plan waits behind the device's work, calls on other streams wait for
    it, and a capture, whose replays would not, is refused."""
    b = Batch(42, [1, 20], [30, 40], 4, 2, 64)
    k, v = caches(torch, b, torch.bfloat16, 9, poison=False)
    q = torch.randn((21, 4, 64), device="cuda", dtype=torch.bfloat16)
    want = b.step().attention(q, k, v)
    a = torch.randn((8192, 8192), device="cuda", dtype=torch.bfloat16)
    a @ a
    other, side = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(250):
        a @ a
    s = b.step()                      # its copy is behind the products
    with torch.cuda.stream(other):
        x = s.attention(q, k, v)
    y = s.attention(q, k, v, stream=side)
    z = s.attention(q, k, v)
    graph = torch.cuda.CUDAGraph()
    out = torch.empty_like(q)
    with torch.cuda.stream(other):
        graph.capture_begin()
        out.zero_()
        refused = False
        try:
            s.attention(q, k, v, out=out)
        except ValueError:
            refused = True
        graph.capture_end()
    late = s._copied.query()
    torch.cuda.synchronize()
    assert refused and not late
    assert all(torch.equal(t, want) for t in (x, y, z))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):     # (it synchronizes first)
        s.attention(q, k, v, out=out)
        with pytest.raises(ValueError):
            b.step()
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
