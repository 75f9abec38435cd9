"""The attention part of a serving iteration, as cases to be timed.

The simulator prices an iteration by integers; these operators are what such an
iteration does with the batch that the scheduler formed: the new tokens' queries,
keys and values are normed and rotated, keys and values go to the paged cache
("append"), and every new token attends to its request's pages ("attention"), which
may begin with pages shared by a group of requests ("prefix": the simulator's
prefix-cache hits).

A case fixes the batch: how many requests, how many new tokens and how much context
each has. The values of the tensors, and which blocks of the pool the pages are, come
from the seed. The plan of a batch (``Step``) is made in ``prepare``: a serving
program makes it once an iteration, when the scheduler has formed the batch, and uses
it for every layer of the model.

With ``own`` false the operators are computed by elementary torch operations in
32 bits; with ``own`` true by the package's entry points.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
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
        # chat traffic: 64 decodes
        dict(name="attention decode 64", op="attention", type="bf16", heads=32, kv_heads=8,
             size=128, block=16, requests=64, new=1, chunks=0, chunk=0, context=900, spread=1.0,
             longest=8192, groups=0, prefix=0, mix=5),
        # the large sweep's 256 sequences with heavy-tailed contexts, the pool nearly full
        dict(name="attention decode 256", op="attention", type="f16", heads=32, kv_heads=8,
             size=128, block=16, requests=256, new=1, chunks=0, chunk=0, context=1000, spread=1.2,
             longest=16384, groups=0, prefix=0, mix=6),
        # decodes and prefill chunks in one iteration; seven query heads to a key head
        dict(name="attention mixed", op="attention", type="bf16", heads=28, kv_heads=4, size=128,
             block=16, requests=64, new=1, chunks=4, chunk=1024, context=1500, spread=1.0,
             longest=8192, groups=0, prefix=0, mix=7),
        # one prefill chunk, a key head to each query head
        dict(name="attention one chunk", op="attention", type="f16", heads=16, kv_heads=16,
             size=64, block=16, requests=1, new=1, chunks=1, chunk=1024, context=4096, spread=0.0,
             longest=4096, groups=0, prefix=0, mix=8),
        # most of the large sweep's token budget taken by chunks of long prompts
        dict(name="attention full budget", op="attention", type="bf16", heads=32, kv_heads=8,
             size=128, block=16, requests=16, new=1, chunks=16, chunk=1024, context=4000,
             spread=0.8, longest=16384, groups=0, prefix=0, mix=9),
        # 64 decodes under one system prompt
        dict(name="prefix decode 64", op="attention", type="bf16", heads=32, kv_heads=8, size=128,
             block=16, requests=64, new=1, chunks=0, chunk=0, context=150, spread=1.0,
             longest=4096, groups=1, prefix=2048, mix=10),
        # 256 answers sampled from one long document
        dict(name="prefix decode 256", op="attention", type="bf16", heads=64, kv_heads=8, size=128,
             block=16, requests=256, new=1, chunks=0, chunk=0, context=500, spread=1.0,
             longest=4096, groups=1, prefix=8192, mix=11),
        # three tenants' prompts that end inside a block, one to five new tokens a request
        dict(name="prefix groups", op="attention", type="f16", heads=16, kv_heads=2, size=64,
             block=16, requests=48, new=5, chunks=0, chunk=0, context=300, spread=1.0,
             longest=4096, groups=3, prefix=1500, mix=12),
    ]


LARGEST_FLOPS = 8e11  # of a drawn case; the listed ones go to 0.88e12 and 1.84e9
LARGEST_BYTES = 1.8e9
LARGEST_TOKENS = 400_000  # context of a drawn batch
LARGEST_PADDED = 3_000_000  # requests times the longest context


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["append", "attention", "attention", "prefix"])
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
        tokens, w = int(kv_len.sum()), work(case)
        if (n_new.sum() <= 16384 and tokens <= LARGEST_TOKENS and w["flops"] <= LARGEST_FLOPS
                and w["bytes"] <= LARGEST_BYTES
                and requests * (int(kv_len.max()) + case["prefix"]) <= LARGEST_PADDED):
            return case


def _lengths(case):
    """New tokens and own context (new tokens among them) of every request, and the
    first request of every prefix group (and the end)."""
    rng = np.random.default_rng([17, case["mix"]])
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
    Hq, Hk, D, b = case["heads"], case["kv_heads"], case["size"], case["block"]
    n_new, kv_len, first = _lengths(case)
    # the pool after long use: the pages of a request lie anywhere in it
    need = -(-kv_len // b)
    pre = -(-case["prefix"] // b)
    used = int(need.sum()) + pre * case["groups"]
    n_blocks = used + used // 16 + 1
    if case["op"] == "append":
        # only blocks that new tokens go to have to be there
        need = need - (kv_len - n_new) // b
        n_blocks = int(need.sum()) + int(need.sum()) // 16 + 1
    order = np.random.default_rng([19, int(seed)]).permutation(n_blocks).astype(np.int32)
    width = int((-(-kv_len // b)).max())
    blocks = np.zeros((len(n_new), width), np.int32)
    at = 0
    for i, m in enumerate(need):
        end = -(-int(kv_len[i]) // b)
        blocks[i, end - m:end] = order[at:at + m]
        at += m
    prefix_blocks = None
    if case["groups"]:
        prefix_blocks = order[at:at + pre * case["groups"]].reshape(case["groups"], pre)
    T = int(n_new.sum())
    shape = (n_blocks, Hk, b, D)
    k_cache = torch.randn(shape, generator=g, device=dev, dtype=dtype)
    v_cache = torch.randn(shape, generator=g, device=dev, dtype=dtype)
    s = dict(case=case, n_new=n_new, kv_len=kv_len, blocks=blocks, first=first,
             prefix_blocks=prefix_blocks, n_blocks=n_blocks, k_cache=k_cache, v_cache=v_cache)
    if case["op"] == "append":
        s["qkv"] = torch.randn((T, Hq + 2 * Hk, D), generator=g, device=dev, dtype=dtype)
        s["cos"], s["sin"] = _angles(int(kv_len.max()), case["rot"], dev)
        s["q_weight"] = s["k_weight"] = None
        if case["norm"]:
            s["q_weight"] = 1 + 0.1 * torch.randn(D, generator=g, device=dev)
            s["k_weight"] = 1 + 0.1 * torch.randn(D, generator=g, device=dev)
            s["q_weight"], s["k_weight"] = s["q_weight"].to(dtype), s["k_weight"].to(dtype)
    else:
        # 1.5: scores spread as trained heads have them, not nearly equal ones
        s["q"] = (1.5 * torch.randn((T, Hq, D), generator=g, device=dev)).to(dtype)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    dev = s["k_cache"].device
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
            s["prefix_table"] = torch.from_numpy(s["prefix_blocks"].astype(np.int64)).to(dev)
        # single tokens lie first in the batch, then one request after another
        s["singles"] = int((np.cumsum(n_new != 1) == 0).sum())
    if own:
        from paper_2606_18431_amd import step

        s["step"] = step.Step(
            n_new, kv_len, s["blocks"], heads=case["heads"], kv_heads=case["kv_heads"],
            head_dim=case["size"], block_tokens=b, n_blocks=s["n_blocks"],
            prefix_first=s["first"], prefix_blocks=s["prefix_blocks"],
            prefix_len=[case["prefix"]] * case["groups"] if case["groups"] else None, device=dev)
    return s


def run(s):
    if own:
        if s["case"]["op"] == "append":
            q = s["step"].append(s["qkv"], s["k_cache"], s["v_cache"], s["cos"], s["sin"],
                                 q_weight=s["q_weight"], k_weight=s["k_weight"], eps=EPS,
                                 interleaved=s["case"]["pairs"] == "interleaved")
            return q, s["k_cache"], s["v_cache"]
        return s["step"].attention(s["q"], s["k_cache"], s["v_cache"])
    if s["case"]["op"] == "append":
        return _plain_append(s)
    return _plain_attention(s)


# ------------------------------------------------------------ the plain forms


def _plain_append(s):
    case = s["case"]
    Hq, Hk, R = case["heads"], case["kv_heads"], case["rot"]
    x = s["qkv"].float()
    qk, v = x[:, :Hq + Hk], s["qkv"][:, Hq + Hk:]
    if case["norm"]:
        r = torch.rsqrt((qk * qk).mean(-1, keepdim=True) + EPS)
        w = torch.cat([s["q_weight"].float().expand(Hq, -1), s["k_weight"].float().expand(Hk, -1)])
        qk = qk * r * w
    c, t = s["cos"][s["pos"]][:, None], s["sin"][s["pos"]][:, None]
    if case["pairs"] == "halves":
        a, b = qk[..., :R // 2], qk[..., R // 2:R]
        turned = torch.cat([a * c - b * t, b * c + a * t, qk[..., R:]], -1)
    else:
        a, b = qk[..., 0:R:2], qk[..., 1:R:2]
        turned = torch.cat([torch.stack([a * c - b * t, b * c + a * t], -1).flatten(-2),
                            qk[..., R:]], -1)
    turned = turned.to(s["qkv"].dtype)
    s["k_cache"][s["slot_block"], :, s["slot_at"]] = turned[:, Hq:]
    s["v_cache"][s["slot_block"], :, s["slot_at"]] = v
    return turned[:, :Hq].contiguous(), s["k_cache"], s["v_cache"]


def _pages(cache, table):
    """[..., pages] block numbers -> [..., Hk, pages * block, D] in 32 bits."""
    x = cache[table].float()  # [..., pages, Hk, block, D]
    x = x.movedim(-3, -4)
    return x.flatten(-3, -2)


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
        k, v = _pages(s["k_cache"], s["table"][:n1]), _pages(s["v_cache"], s["table"][:n1])
        at = torch.arange(k.shape[2], device=k.device)
        hide = (at >= s["kv_len_d"][:n1, None])[:, None, None, :]
        qs = q[:n1].view(n1, Hk, G, D) * scale
        scores = (qs @ k.transpose(-1, -2)).masked_fill(hide, -math.inf)
        v = v.masked_fill(hide.transpose(-1, -2), 0)
        if case["groups"]:
            table = s["prefix_table"][s["group"][:n1]]
            kp = _pages(s["k_cache"], table)[:, :, :p]
            vp = _pages(s["v_cache"], table)[:, :, :p]
            scores = torch.cat([qs @ kp.transpose(-1, -2), scores], -1)
            v = torch.cat([vp, v], -2)
        out[:n1] = _softmax_product(scores, v).reshape(n1, Hk * G, D)
    t = n1
    for i in range(n1, len(s["n_new"])):
        n, m = int(s["n_new"][i]), int(s["kv_len"][i])
        pages = -(-m // b)
        k = _pages(s["k_cache"], s["table"][i, :pages])[:, :m]
        v = _pages(s["v_cache"], s["table"][i, :pages])[:, :m]
        if case["groups"]:
            table = s["prefix_table"][s["group"][i]]
            k = torch.cat([_pages(s["k_cache"], table)[:, :p], k], 1)
            v = torch.cat([_pages(s["v_cache"], table)[:, :p], v], 1)
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
    return _exact_append(s) if case["op"] == "append" else _exact_attention(s)


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
    k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
    at = 0
    for i in range(len(n_new)):
        n, k = int(n_new[i]), int(kv_len[i])
        own_pos = np.arange(k - n, k)
        page = torch.from_numpy(s["blocks"][i, own_pos // b].astype(np.int64)).to(dev)
        off = torch.from_numpy(own_pos % b).to(dev)
        k_cache[page, :, off] = out[at:at + n, Hq:Hq + Hk]
        v_cache[page, :, off] = x[at:at + n, Hq + Hk:]
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
        rows = [s["blocks"][i, y // b] * b + y % b for y in range(0, m)]
        if case["groups"]:
            g = int(np.nonzero(s["first"] <= i)[0][-1])
            shared = [s["prefix_blocks"][g, y // b] * b + y % b for y in range(case["prefix"])]
            rows = shared + rows
        rows = torch.tensor(np.asarray(rows, np.int64), device=dev)
        total = len(rows)
        seen = torch.arange(total, device=dev)[None, :] <= \
            torch.arange(total - n, total, device=dev)[:, None]
        for h in range(Hk):
            k = s["k_cache"][rows // b, h, rows % b].double()
            v = s["v_cache"][rows // b, h, rows % b].double()
            for j in range(h * G, (h + 1) * G):
                e = (q[t:t + n, j] @ k.T) / math.sqrt(D)
                e = torch.where(seen, e, torch.full_like(e, -math.inf))
                e = torch.exp(e - e.max(-1, keepdim=True).values)
                out[t:t + n, j] = (e / e.sum(-1, keepdim=True)) @ v
        t += n
    return out


# ------------------------------------------------------------ what a pass cannot do without


def work(case):
    n_new, kv_len, first = _lengths(case)
    Hq, Hk, D = case["heads"], case["kv_heads"], case["size"]
    T = int(n_new.sum())
    if case["op"] == "append":
        heads = Hq + 2 * Hk
        positions = len(np.unique(np.concatenate([np.arange(k - n, k)
                                                  for n, k in zip(n_new, kv_len)])))
        # queries, keys and values in and out, the angles of the positions that occur;
        # a norm takes 4 operations a value, the rotation 3
        return {"bytes": 2.0 * T * heads * D * 2 + positions * case["rot"] * 4.0,
                "flops": float(T * (Hq + Hk) * (3 * case["rot"] + (4 * D if case["norm"] else 0)))}
    # a key is read once for all the rows that see it, a shared one once a group
    keys = int(kv_len.sum()) + case["prefix"] * case["groups"]
    pairs = float((n_new * (kv_len - n_new) + n_new * (n_new + 1) // 2).sum()) \
        + float(T) * case["prefix"]
    return {"bytes": 2.0 * 2 * T * Hq * D + 2.0 * 2 * keys * Hk * D, "flops": 4.0 * pairs * Hq * D}
