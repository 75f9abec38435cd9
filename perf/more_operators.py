"""A serving iteration in four bits, as cases to be timed.

Three operators of one iteration, for an engine whose KV cache and weights are held in
four bits (so that a pool of the same memory has 3.8 times the blocks that the simulator
counts, and a decode step reads that much less):

- "append": the new tokens' queries and keys are normed and rotated; keys and values are
  rounded to four bits and go to their slots of the paged cache;
- "attention": every new token attends to its request's pages there, which may begin with
  pages that a group of requests shares;
- "linear": the product of the tokens' activations with a weight matrix in four bits.

Four bits: 32 adjacent elements of a row are a block with one scale, a power of two 2^e
held as the byte e + 127 (255: the block is NaN). An element is a sign and one of
0, 0.5, 1, 1.5, 2, 3, 4, 6, times the scale; the even one of two is in the low half of its
byte. Values are rounded to the nearest of these, halves to the even code, at the smallest
scale with max |x| < 7 * 2^e (within the exponents that the tensors' 16-bit type holds;
beyond the largest value they become that).

A case fixes the sizes; values, and which blocks of the pool the pages are, come from the
seed. The plan of a batch (``Step``) and the weights' layout (``Weights``) are made in
``prepare``: a serving program makes one an iteration and the other once.

With ``own`` false the operators are computed by elementary torch operations in 32 bits
(keys in 64: a value next to the border of two codes); with ``own`` true by the package's
entry points. What is held in four bits is returned as the values it stands for, the
cache after an append by the package's ``Cache.values``.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
# exponents of a scale at which the 16-bit type holds every value
EXPONENTS = {torch.bfloat16: (-125, 125), torch.float16: (-23, 13)}
MAGNITUDES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
BORDERS = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]  # between them; each goes to the even code
EPS = 1e-6


def listed():
    return [
        # a decode iteration of a full batch of 64: the call that runs most often
        dict(name="append decode 64", op="append", type="bf16", heads=32, kv_heads=8, size=128,
             rot=128, pairs="halves", norm=True, block=16, requests=64, new=1, chunks=0, chunk=0,
             context=900, spread=1.0, longest=8192, groups=0, prefix=0, mix=1),
        # decodes with three prefill chunks beside them; half of each head rotated
        dict(name="append mixed", op="append", type="f16", heads=16, kv_heads=16, size=64, rot=32,
             pairs="interleaved", norm=False, block=16, requests=48, new=1, chunks=3, chunk=1024,
             context=900, spread=1.0, longest=8192, groups=0, prefix=0, mix=2),
        # most of the large sweep's token budget taken by prefill chunks
        dict(name="append full budget", op="append", type="bf16", heads=32, kv_heads=8, size=128,
             rot=128, pairs="halves", norm=True, block=16, requests=16, new=1, chunks=16,
             chunk=1024, context=2000, spread=1.0, longest=8192, groups=0, prefix=0, mix=3),
        # an idle server with one short conversation: nothing but latency
        dict(name="attention one decode", op="attention", type="bf16", heads=32, kv_heads=8,
             size=128, block=16, requests=1, new=1, chunks=0, chunk=0, context=777, spread=0.0,
             longest=777, groups=0, prefix=0, mix=4),
        # the large sweep's 256 sequences with heavy-tailed contexts, the pool nearly full
        dict(name="attention decode 256", op="attention", type="f16", heads=32, kv_heads=8,
             size=128, block=16, requests=256, new=1, chunks=0, chunk=0, context=1000, spread=1.2,
             longest=16384, groups=0, prefix=0, mix=6),
        # decodes and prefill chunks in one iteration; seven query heads to a key head
        dict(name="attention mixed", op="attention", type="bf16", heads=28, kv_heads=4, size=128,
             block=16, requests=64, new=1, chunks=4, chunk=1024, context=1500, spread=1.0,
             longest=8192, groups=0, prefix=0, mix=7),
        # most of the large sweep's token budget taken by chunks of long prompts
        dict(name="attention full budget", op="attention", type="bf16", heads=32, kv_heads=8,
             size=128, block=16, requests=16, new=1, chunks=16, chunk=1024, context=4000,
             spread=0.8, longest=16384, groups=0, prefix=0, mix=9),
        # three tenants' prompts that end inside a block, one to five new tokens a request
        dict(name="attention prefix groups", op="attention", type="f16", heads=16, kv_heads=2,
             size=64, block=16, requests=48, new=5, chunks=0, chunk=0, context=300, spread=1.0,
             longest=4096, groups=3, prefix=1500, mix=12),
        # one decode's queries, keys and values: 32 + 2 * 8 heads of 128 from a state of 4096
        dict(name="linear one token", op="linear", type="bf16", tokens=1, rows=6144, cols=4096),
        # a few decodes, sizes that end inside every tile
        dict(name="linear odd sizes", op="linear", type="f16", tokens=13, rows=5003, cols=4128),
        # 64 decodes through the wide matrix of a layer's second half
        dict(name="linear decode 64", op="linear", type="bf16", tokens=64, rows=16384, cols=4096),
        # a prefill-heavy iteration through the heads' matrix
        dict(name="linear full budget", op="linear", type="bf16", tokens=8192, rows=6144,
             cols=4096),
    ]


LARGEST_FLOPS = 8e11  # of a drawn case; the listed ones go to 0.88e12
LARGEST_LINEAR = 4e11  # of a drawn product; the listed ones go to 4.1e11
LARGEST_BYTES = 5e8
LARGEST_TOKENS = 400_000  # context of a drawn batch
LARGEST_PADDED = 3_000_000  # requests times the longest context


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["append", "attention", "attention", "prefix", "linear", "linear"])
        if op == "linear":
            case = dict(op="linear", type=rng.choice(["bf16", "f16"]), tokens=_log(rng, 1, 8192),
                        rows=_log(rng, 1, 32768), cols=32 * _log(rng, 1, 512))
            w = work(case)
            if w["flops"] <= LARGEST_LINEAR and w["bytes"] <= LARGEST_BYTES:
                return case
            continue
        heads, kv_heads = rng.choice([(32, 8), (64, 8), (28, 4), (8, 1), (16, 16), (16, 2), (20, 4)])
        size = rng.choice([64, 128, 128])
        case = dict(op="attention" if op == "prefix" else op, type=rng.choice(["bf16", "f16"]),
                    heads=heads, kv_heads=kv_heads, size=size, block=rng.choice([16, 16, 32, 64]))
        requests = _log(rng, 1, 256)
        chunks = rng.choice([0, 0, 1, 4, requests])
        case |= dict(requests=requests, new=rng.choice([1, 1, 1, 2, 5]),
                     chunks=min(chunks, requests), chunk=_log(rng, 16, 1024),
                     context=_log(rng, 1, 32768), spread=rng.choice([0.0, 0.5, 1.0]),
                     longest=32768, groups=0, prefix=0, mix=rng.randrange(1 << 30))
        if op == "append":
            case |= dict(rot=rng.choice([size, size, size // 2]),
                         pairs=rng.choice(["halves", "interleaved"]),
                         norm=rng.choice([True, False]))
        if op == "prefix":
            case |= dict(groups=min(requests, rng.choice([1, 1, 2, 3])),
                         prefix=_log(rng, 64, 16384))
        n_new, kv_len, _ = _lengths(case)
        w = work(case)
        if (n_new.sum() <= 16384 and kv_len.sum() <= LARGEST_TOKENS
                and w["flops"] <= LARGEST_FLOPS and w["bytes"] <= LARGEST_BYTES
                and requests * (int(kv_len.max()) + case["prefix"]) <= LARGEST_PADDED):
            return case


def _lengths(case):
    """New tokens and own context (new tokens among them) of every request, and the
    first request of every prefix group (and the end)."""
    rng = np.random.default_rng([23, case["mix"]])
    n = case["requests"]
    z = rng.standard_normal(n)
    context = np.rint(case["context"] * np.exp(case["spread"] * z))
    context = np.clip(context, 1, case["longest"]).astype(np.int64)
    n_new = rng.integers(1, case["new"] + 1, n)
    if case["chunks"]:
        # the chunks come last, as the scheduler adds them to the running decodes; all
        # but the first of them may be the shorter end of a prompt
        part = rng.integers(max(1, case["chunk"] // 2), case["chunk"] + 1, case["chunks"])
        part[0] = case["chunk"]
        n_new[n - case["chunks"]:] = part
    kv_len = np.maximum(context, n_new)
    first = np.linspace(0, n, case["groups"] + 1).astype(np.int64) if case["groups"] else None
    return n_new, kv_len, first


def _pool(case, rng):
    """Block numbers of the pages, of the shared prefixes, and the blocks of the pool. After
    long use the pages of a request lie anywhere in it. For append only blocks that new
    tokens go to have to be there."""
    b = case["block"]
    n_new, kv_len, _ = _lengths(case)
    end = -(-kv_len // b)
    need = end - (kv_len - n_new) // b if case["op"] == "append" else end
    pre = -(-case["prefix"] // b)
    used = int(need.sum()) + pre * case["groups"]
    n_blocks = used + used // 16 + 1
    order = rng.permutation(n_blocks).astype(np.int32)
    blocks = np.zeros((len(n_new), int(end.max())), np.int32)
    at = 0
    for i, m in enumerate(need):
        blocks[i, int(end[i]) - m:int(end[i])] = order[at:at + m]
        at += m
    shared = order[at:at + pre * case["groups"]].reshape(case["groups"], pre)
    return blocks, shared if case["groups"] else None, n_blocks


def _angles(positions, rot, device):
    f = 1.0 / 10000.0 ** (torch.arange(0, rot, 2, device=device, dtype=torch.float64) / rot)
    a = torch.arange(positions, device=device, dtype=torch.float64)[:, None] * f
    return a.cos().float(), a.sin().float()


def _inputs(case, seed):
    """The inputs, from the case and the seed alone."""
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    dtype = DTYPES[case["type"]]

    def normal(*shape, dtype=dtype):
        return torch.randn(shape, generator=g, device=dev, dtype=dtype)

    if case["op"] == "linear":
        n, k = case["rows"], case["cols"]
        codes, scales = _round4(normal(n, k, dtype=torch.float32) * k ** -0.5, EXPONENTS[dtype])
        return dict(case=case, x=normal(case["tokens"], k), codes=codes, scales=scales)
    Hq, Hk, D, b = case["heads"], case["kv_heads"], case["size"], case["block"]
    n_new, kv_len, first = _lengths(case)
    blocks, shared, n_blocks = _pool(case, np.random.default_rng([29, int(seed)]))
    T = int(n_new.sum())
    s = dict(case=case, n_new=n_new, kv_len=kv_len, blocks=blocks, first=first, shared=shared,
             n_blocks=n_blocks)
    for name in ("k", "v"):
        s[name], s[name + "_scale"] = _round4(normal(n_blocks, Hk, b, D), EXPONENTS[dtype])
    if case["op"] == "append":
        s["qkv"] = normal(T, Hq + 2 * Hk, D)
        s["cos"], s["sin"] = _angles(int(kv_len.max()), case["rot"], dev)
        s["q_weight"] = s["k_weight"] = None
        if case["norm"]:
            s["q_weight"] = (1 + 0.1 * normal(D, dtype=torch.float32)).to(dtype)
            s["k_weight"] = (1 + 0.1 * normal(D, dtype=torch.float32)).to(dtype)
    else:
        # 1.5: scores spread as trained heads have them, not nearly equal ones
        s["q"] = (1.5 * normal(T, Hq, D, dtype=torch.float32)).to(dtype)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2606_18431_amd import fp4, step
    if case["op"] == "linear":
        if own:
            s["weights"] = fp4.Weights(s["codes"], s["scales"])
        return s
    dev = s["k"].device
    b = case["block"]
    n_new, kv_len = s["n_new"], s["kv_len"]
    request = np.repeat(np.arange(len(n_new)), n_new)
    own_pos = np.concatenate([np.arange(k - n, k) for n, k in zip(n_new, kv_len)])
    if case["op"] == "append":
        s["pos"] = torch.from_numpy(own_pos).to(dev)
        s["slot_block"] = torch.from_numpy(s["blocks"][request, own_pos // b].astype(np.int64)).to(dev)
        s["slot_at"] = torch.from_numpy(own_pos % b).to(dev)
    else:
        s["table"] = torch.from_numpy(s["blocks"].astype(np.int64)).to(dev)
        s["kv_len_d"] = torch.from_numpy(kv_len).to(dev)
        if case["groups"]:
            group = np.searchsorted(s["first"], np.arange(len(n_new)), side="right") - 1
            s["group"] = torch.from_numpy(group).to(dev)
            s["shared_table"] = torch.from_numpy(s["shared"].astype(np.int64)).to(dev)
        # single tokens lie first in the batch, then one request after another
        s["singles"] = int((np.cumsum(n_new != 1) == 0).sum())
    if own:
        s["cache"] = fp4.Cache(s["k"], s["v"], s["k_scale"], s["v_scale"])
        s["step"] = step.Step(
            n_new, kv_len, s["blocks"], heads=case["heads"], kv_heads=case["kv_heads"],
            head_dim=case["size"], block_tokens=b, n_blocks=s["n_blocks"],
            prefix_first=s["first"], prefix_blocks=s["shared"],
            prefix_len=[case["prefix"]] * case["groups"] if case["groups"] else None, device=dev)
    return s


def run(s):
    op = s["case"]["op"]
    if own:
        from paper_2606_18431_amd import fp4

        if op == "linear":
            return fp4.linear(s["x"], s["weights"])
        if op == "append":
            q = s["step"].append_fp4(s["qkv"], s["cache"], s["cos"], s["sin"],
                                     q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS,
                                     interleaved=s["case"]["pairs"] == "interleaved")
            k, v = s["cache"].values(q.dtype)
            return q, k, v
        return s["step"].attention_fp4(s["q"], s["cache"])
    if op == "linear":
        return (s["x"].float() @ _values4(s["codes"], s["scales"]).T).to(s["x"].dtype)
    if op == "append":
        return _plain_append(s)
    return _plain_attention(s)


# ------------------------------------------------------------ the plain forms


def _scale4(x, exponents):
    """Exponents of the scales of x [..., 32]; which blocks are finite."""
    most = x.abs().amax(-1)
    e = torch.frexp(most).exponent - 3
    e = e + (most >= torch.ldexp(torch.full_like(most, 7), e))
    e = torch.where(most > 0, e, exponents[0]).clamp(*exponents)
    return e, torch.isfinite(most)


def _code4(x, e):
    """Codes of the elements of x [..., 32] at the scales 2^e."""
    t = torch.ldexp(x.abs(), -e[..., None])
    code = torch.zeros(x.shape, dtype=torch.uint8, device=x.device)
    for i, border in enumerate(BORDERS):
        code += t > border if i % 2 == 0 else t >= border
    return code + 8 * torch.signbit(x).to(torch.uint8)


def _round4(x, exponents):
    """(codes [..., n / 2], scales [..., n / 32]) of x [..., n]."""
    blocks = x.unflatten(-1, (-1, 32))
    if blocks.dtype != torch.float64:
        blocks = blocks.float()
    e, finite = _scale4(blocks, exponents)
    code = (_code4(blocks, e) * finite[..., None]).flatten(-2)
    scale = torch.where(finite, e + 127, 255).to(torch.uint8)
    return code[..., ::2] | code[..., 1::2] << 4, scale


def _values4(codes, scales):
    """The values in 32 bits."""
    m = torch.tensor(MAGNITUDES, device=codes.device)
    m = torch.cat([m, -m])
    pair = torch.stack([m.repeat(16), m.repeat_interleave(16)], -1)  # of every byte
    x = pair[codes.int()].flatten(-2).unflatten(-1, (-1, 32))
    e = scales.int() - 127
    f = torch.where(e < 128, torch.ldexp(torch.ones_like(e, dtype=torch.float32), e), math.nan)
    return (x * f[..., None]).flatten(-2)


def _plain_append(s):
    case = s["case"]
    Hq, Hk, R = case["heads"], case["kv_heads"], case["rot"]
    dtype = s["qkv"].dtype

    def normed_and_turned(x, weight):
        if weight is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.to(x.dtype)
        c, t = (a[s["pos"]][:, None].to(x.dtype) for a in (s["cos"], s["sin"]))
        if case["pairs"] == "halves":
            a, b = x[..., :R // 2], x[..., R // 2:R]
            return torch.cat([a * c - b * t, b * c + a * t, x[..., R:]], -1)
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        return torch.cat([torch.stack([a * c - b * t, b * c + a * t], -1).flatten(-2),
                          x[..., R:]], -1)

    q = normed_and_turned(s["qkv"][:, :Hq].float(), s["q_weight"]).to(dtype)
    # in 64 bits: which code a key's element gets
    k = normed_and_turned(s["qkv"][:, Hq:Hq + Hk].double(), s["k_weight"])
    caches = []
    for name, new in (("k", k), ("v", s["qkv"][:, Hq + Hk:])):
        cache = _values4(s[name], s[name + "_scale"])
        cache[s["slot_block"], :, s["slot_at"]] = _values4(*_round4(new, EXPONENTS[dtype]))
        caches.append(cache.to(dtype))
    return q, *caches


def _pages(s, name, table):
    """[..., pages] block numbers -> [..., Hk, pages * block, D] in 32 bits."""
    x = _values4(s[name][table], s[name + "_scale"][table])  # [..., pages, Hk, block, D]
    return x.movedim(-3, -4).flatten(-3, -2)


def _softmax_product(scores, v):
    m = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - m)
    return (p @ v) / p.sum(-1, keepdim=True)


def _plain_attention(s):
    """All requests with one new token at once, padded to the longest; then each of the
    others by itself."""
    case = s["case"]
    Hk, D, b = case["kv_heads"], case["size"], case["block"]
    G = case["heads"] // Hk
    scale = D ** -0.5
    q = s["q"].float()
    out = torch.empty_like(q)
    p = case["prefix"]
    n1 = s["singles"]
    if n1:
        k, v = _pages(s, "k", s["table"][:n1]), _pages(s, "v", s["table"][:n1])
        at = torch.arange(k.shape[2], device=k.device)
        hide = (at >= s["kv_len_d"][:n1, None])[:, None, None, :]
        qs = q[:n1].view(n1, Hk, G, D) * scale
        scores = (qs @ k.transpose(-1, -2)).masked_fill(hide, -math.inf)
        v = v.masked_fill(hide.transpose(-1, -2), 0)
        if case["groups"]:
            table = s["shared_table"][s["group"][:n1]]
            kp, vp = _pages(s, "k", table)[:, :, :p], _pages(s, "v", table)[:, :, :p]
            scores = torch.cat([qs @ kp.transpose(-1, -2), scores], -1)
            v = torch.cat([vp, v], -2)
        out[:n1] = _softmax_product(scores, v).reshape(n1, Hk * G, D)
    t = n1
    for i in range(n1, len(s["n_new"])):
        n, m = int(s["n_new"][i]), int(s["kv_len"][i])
        pages = -(-m // b)
        k = _pages(s, "k", s["table"][i, :pages])[:, :m]
        v = _pages(s, "v", s["table"][i, :pages])[:, :m]
        if case["groups"]:
            table = s["shared_table"][s["group"][i]]
            k = torch.cat([_pages(s, "k", table)[:, :p], k], 1)
            v = torch.cat([_pages(s, "v", table)[:, :p], v], 1)
        qs = q[t:t + n].view(n, Hk, G, D).permute(1, 2, 0, 3) * scale  # [Hk, G, n, D]
        scores = qs.reshape(Hk, G * n, D) @ k.transpose(-1, -2)
        pos = torch.arange(m - n, m, device=k.device) + k.shape[1] - m
        hide = torch.arange(k.shape[1], device=k.device)[None] > pos[:, None]
        scores.view(Hk, G, n, -1).masked_fill_(hide, -math.inf)
        o = _softmax_product(scores, v)
        out[t:t + n] = o.view(Hk, G, n, D).permute(2, 0, 1, 3).reshape(n, Hk * G, D)
        t += n
    return out.to(s["q"].dtype)


# ------------------------------------------------------------ in 64 bits


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "linear":
        return s["x"].double() @ _exact_values(s["codes"], s["scales"]).T
    return _exact_append(s) if case["op"] == "append" else _exact_attention(s)


def _exact_values(codes, scales):
    m = torch.tensor(MAGNITUDES, device=codes.device, dtype=torch.float64)
    out = torch.empty((*codes.shape[:-1], 2 * codes.shape[-1]), device=codes.device,
                      dtype=torch.float64)
    for half in (0, 1):
        c = (codes >> 4 * half & 15).long()
        out[..., half::2] = m[c % 8] * (1 - 2 * (c // 8))
    f = 2.0 ** (scales.double() - 127)
    f[scales == 255] = math.nan
    return out * f.repeat_interleave(32, -1)


def _exact_rounded(x, exponents):
    """x [..., n] in 64 bits, rounded to four."""
    y = x.reshape(*x.shape[:-1], -1, 32)
    most = y.abs().amax(-1, keepdim=True)
    e = torch.full_like(most, exponents[0])
    for _ in range(exponents[1] - exponents[0]):  # the smallest that holds the largest
        small = most >= 7 * 2.0 ** e
        if not bool(small.any()):
            break
        e = torch.where(small & (e < exponents[1]), e + 1, e)
    t = y.abs() / 2.0 ** e
    part = torch.where(t < 2, 0.5, torch.where(t < 4, 1.0, 2.0))  # between adjacent values
    r = torch.clamp(torch.round(t / part) * part, max=6.0) * torch.sign(y) * 2.0 ** e
    return r.reshape(x.shape)


def _exact_append(s):
    case = s["case"]
    Hq, Hk, D, R, b = (case[x] for x in ("heads", "kv_heads", "size", "rot", "block"))
    n_new, kv_len, dev = s["n_new"], s["kv_len"], s["qkv"].device
    x = s["qkv"].double()
    m = R // 2
    if case["pairs"] == "halves":
        first, second = list(range(m)), list(range(m, R))
    else:
        first, second = list(range(0, R, 2)), list(range(1, R, 2))
    pos = torch.cat([torch.arange(int(k - n), int(k)) for n, k in zip(n_new, kv_len)]).to(dev)
    c, t = s["cos"].double()[pos], s["sin"].double()[pos]
    out = x.clone()
    for h in range(Hq + Hk):
        u = x[:, h]
        if case["norm"]:
            w = s["q_weight"] if h < Hq else s["k_weight"]
            u = u / torch.sqrt((u ** 2).sum(-1, keepdim=True) / D + EPS) * w.double()
        y = u.clone()
        y[:, first] = u[:, first] * c - u[:, second] * t
        y[:, second] = u[:, second] * c + u[:, first] * t
        out[:, h] = y
    new = _exact_rounded(out[:, Hq:], EXPONENTS[s["qkv"].dtype])
    k_cache, v_cache = (_exact_values(s[n], s[n + "_scale"]) for n in ("k", "v"))
    at = 0
    for i in range(len(n_new)):
        n, k = int(n_new[i]), int(kv_len[i])
        own_pos = np.arange(k - n, k)
        page = torch.from_numpy(s["blocks"][i, own_pos // b].astype(np.int64)).to(dev)
        off = torch.from_numpy(own_pos % b).to(dev)
        k_cache[page, :, off] = new[at:at + n, :Hk]
        v_cache[page, :, off] = new[at:at + n, Hk:]
        at += n
    return out[:, :Hq].contiguous(), k_cache, v_cache


def _exact_attention(s):
    case = s["case"]
    Hq, Hk, D, b = (case[x] for x in ("heads", "kv_heads", "size", "block"))
    n_new, kv_len, dev = s["n_new"], s["kv_len"], s["q"].device
    q = s["q"].double()
    out = torch.empty_like(q)
    G = Hq // Hk
    t = 0
    for i in range(len(n_new)):
        n, m = int(n_new[i]), int(kv_len[i])
        y = np.arange(m)
        rows = s["blocks"][i, y // b].astype(np.int64) * b + y % b
        if case["groups"]:
            g = int(np.nonzero(s["first"] <= i)[0][-1])
            y = np.arange(case["prefix"])
            rows = np.concatenate([s["shared"][g, y // b].astype(np.int64) * b + y % b, rows])
        rows = torch.from_numpy(rows).to(dev)
        total = len(rows)
        seen = torch.arange(total, device=dev)[None, :] <= \
            torch.arange(total - n, total, device=dev)[:, None]
        for h in range(Hk):
            k, v = (_exact_values(s[x][rows // b, h, rows % b], s[x + "_scale"][rows // b, h, rows % b])
                    for x in ("k", "v"))
            for j in range(h * G, (h + 1) * G):
                e = (q[t:t + n, j] @ k.T) / math.sqrt(D)
                e = torch.where(seen, e, torch.full_like(e, -math.inf))
                e = torch.exp(e - e.max(-1, keepdim=True).values)
                out[t:t + n, j] = (e / e.sum(-1, keepdim=True)) @ v
        t += n
    return out


# ------------------------------------------------------------ what a pass cannot do without


FOUR = 0.5 + 1 / 32  # bytes of an element with its share of the scale


def work(case):
    if case["op"] == "linear":
        t, n, k = case["tokens"], case["rows"], case["cols"]
        return {"bytes": 2.0 * t * (k + n) + FOUR * n * k, "flops": 2.0 * t * n * k}
    n_new, kv_len, first = _lengths(case)
    Hq, Hk, D = case["heads"], case["kv_heads"], case["size"]
    T = int(n_new.sum())
    if case["op"] == "append":
        positions = len(np.unique(np.concatenate([np.arange(k - n, k)
                                                  for n, k in zip(n_new, kv_len)])))
        pool = 2.0 * _pool(case, np.random.default_rng(0))[2] * case["block"] * Hk * D
        # queries, keys and values in, queries out, keys and values to the cache, the angles
        # of the positions that occur; then the pool's codes in and its values out. A norm
        # takes 4 operations a value, the rotation 3, rounding 2
        return {"bytes": 2.0 * T * (2 * Hq + 2 * Hk) * D + FOUR * T * 2 * Hk * D
                + positions * case["rot"] * 4.0 + pool * (FOUR + 2),
                "flops": float(T * ((Hq + Hk) * (3 * case["rot"] + (4 * D if case["norm"] else 0))
                                    + 4 * Hk * D))}
    # a key is read once for all the rows that see it, a shared one once a group
    keys = int(kv_len.sum()) + case["prefix"] * case["groups"]
    pairs = float((n_new * (kv_len - n_new) + n_new * (n_new + 1) // 2).sum()) \
        + float(T) * case["prefix"]
    return {"bytes": 2.0 * 2 * T * Hq * D + 2.0 * FOUR * keys * Hk * D, "flops": 4.0 * pairs * Hq * D}
