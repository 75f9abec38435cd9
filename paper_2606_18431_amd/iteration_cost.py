"""What an iteration's attention costs on this GPU, in the cost model's terms.

The simulator prices an iteration as base + tok * sum(n) + sum(ctx) / div
microseconds (``workloads.Engine``). This command forms iterations of a workload
as its scheduler would have them in progress, runs their attention part on the
GPU as a model's layers do (``step.Step``: norm, rotate and append the new tokens,
then attend over the pages) and fits the three coefficients to the times:

    python -m paper_2606_18431_amd.iteration_cost --cfg 4 --layers 32
    python -m paper_2606_18431_amd.iteration_cost --cfg 4 --layers 32 --cache-bits 4 --hidden 4096

``--prefix N`` puts N shared tokens (a system prompt, computed once) before every
request's own context. In an iteration's context they count once, as they are read
(each new token's work on them is in tok). The times hold the layers' two calls, made
from the host one layer after another. ``--cache-bits 4`` holds the caches in four bits
(``fp4.Cache``); their blocks take 3.8 times less memory. ``--hidden N`` adds the products
with a layer's weights, held in four bits (``fp4.Weights``): of a state of N to the heads,
from the heads back, and to ``--ffn`` (4 N) and back; the norms and the activation between
them are not in the times. Without it the weights' part of an iteration is not in them
(add it to base and tok from the model's own measurements). Never in them is the plan of
the batch, which the host makes once an iteration and which is printed by itself (an engine
that plans while the GPU works does not wait for it; one that plans in between adds it to
base).
"""
from __future__ import annotations

import argparse
import dataclasses
import math
import time

import numpy as np

from . import workloads as W


@dataclasses.dataclass
class Iteration:
    """One iteration's batch: new tokens and context of every request in it (the
    new ones included), and the blocks that hold the contexts."""

    n_new: np.ndarray
    kv_len: np.ndarray
    blocks: np.ndarray  # [requests, pages], -1 beyond a context

    @property
    def tokens(self) -> int:
        return int(self.n_new.sum())

    @property
    def context(self) -> int:
        return int(self.kv_len.sum())


def form_iteration(w: W.Workload, trace: int, first: int, rng, prefix_blocks: int = 0) -> Iteration:
    """An iteration in the middle of a run: requests from ``first`` on, each somewhere
    in its life (every one of its prefill chunks and decode steps is equally likely),
    admitted while the engine's sequence cap, token budget and KV blocks last.
    ``prefix_blocks`` of the pool are taken by shared tokens."""
    e = w.engine
    n_new, kv_len = [], []
    used = prefix_blocks
    budget = e.max_tokens
    for i in range(first, first + 4 * e.max_seqs):
        p, d = int(w.prompt[trace, i % w.n_req]), int(w.decode[trace, i % w.n_req])
        chunks = -(-p // e.chunk)
        at = int(rng.integers(0, chunks + d - 1)) if chunks + d > 1 else 0
        if at < chunks:
            kv = min((at + 1) * e.chunk, p)
            n = kv - at * e.chunk
        else:
            kv, n = p + at - chunks + 1, 1
        n_pages = -(-kv // e.block_tokens)
        if n > budget or used + n_pages > e.kv_blocks or len(n_new) == e.max_seqs:
            break
        n_new.append(n)
        kv_len.append(kv)
        used += n_pages
        budget -= n
    if not n_new:
        raise ValueError("no request fits the engine's budgets")
    n_new, kv_len = np.asarray(n_new), np.asarray(kv_len)
    pages = -(-kv_len // e.block_tokens)
    ids = prefix_blocks + rng.permutation(e.kv_blocks - prefix_blocks)
    blocks = np.full((len(n_new), int(pages.max())), -1, np.int32)
    at = 0
    for i, n in enumerate(pages):
        blocks[i, :n] = ids[at:at + n]
        at += n
    return Iteration(n_new, kv_len, blocks)


class Layers:
    """The layers' caches, one of each layer's own as in a model (as many as the memory
    holds, in turn), and the inputs of their attention; random values. ``hidden`` and
    ``ffn``: with the layers' weights, in four bits, each layer's own as well."""

    def __init__(self, e: W.Engine, layers, heads, kv_heads, head_dim, dtype, device, positions,
                 cache_bits=16, hidden=0, ffn=0):
        import torch

        if cache_bits not in (4, 16):
            raise ValueError(f"caches of {cache_bits} bits: 4 or 16")
        if hidden < 0 or hidden % 32 or ffn < 0 or ffn % 32 or (ffn and not hidden):
            raise ValueError(f"hidden {hidden}, ffn {ffn}: multiples of 32, ffn with hidden")
        self.torch, self.cache_bits = torch, cache_bits
        shape = (e.kv_blocks, kv_heads, e.block_tokens, head_dim)
        g = torch.Generator(device=device)
        g.manual_seed(0)

        def random(*shape):
            return torch.randn(shape, generator=g, device=device, dtype=dtype)

        def random_fp4(*shape, scale=0):
            """Codes, and scales of 2^scale."""
            *lead, n = shape
            codes = torch.randint(0, 256, (*lead, n // 2), generator=g, device=device,
                                  dtype=torch.uint8)
            return codes, torch.full((*lead, n // 32), 127 + scale, device=device,
                                     dtype=torch.uint8)

        def cache():
            if cache_bits == 16:
                return random(*shape), random(*shape)
            from . import fp4

            (k, k_scale), (v, v_scale) = random_fp4(*shape), random_fp4(*shape)
            return fp4.Cache(k, v, k_scale, v_scale)

        self.layers = layers
        self.weights = []
        if hidden:
            from . import fp4

            ffn = ffn or 4 * hidden
            rows = (heads + 2 * kv_heads) * head_dim
            sizes = ((rows, hidden), (hidden, heads * head_dim), (ffn, hidden), (hidden, ffn))
            # values of some 2 * 2^scale: about 1 / sqrt(cols), so that the states stay near 1
            self.weights = [[fp4.Weights(*random_fp4(n, k, scale=-round(math.log2(3 * k ** 0.5))))
                             for n, k in sizes] for _ in range(layers)]
            self.x = random(e.max_tokens, hidden)
        caches = layers
        if torch.device(device).type == "cuda":
            per_value = 2.0 if cache_bits == 16 else 0.5 + 1 / 32
            layer_bytes = int(2 * per_value * math.prod(shape))
            caches = min(layers, max(1, torch.cuda.mem_get_info(device)[0] * 3 // 4 // layer_bytes))
        self.caches = [cache() for _ in range(caches)]
        self.qkv = random(e.max_tokens, heads + 2 * kv_heads, head_dim)
        self.weight = torch.ones(head_dim, device=device, dtype=dtype)
        freq = 1e4 ** (-torch.arange(0, head_dim, 2, device=device, dtype=torch.float64) / head_dim)
        angle = torch.arange(positions, device=device, dtype=torch.float64)[:, None] * freq
        self.cos, self.sin = angle.cos().float(), angle.sin().float()

    def run(self, step):
        """All layers, one after another, for the step's batch."""
        qkv = self.qkv[:step.tokens]
        for i in range(self.layers):
            cache = self.caches[i % len(self.caches)]
            if self.weights:
                from .fp4 import linear

                of_heads, from_heads, up, down = self.weights[i]
                qkv = linear(self.x[:step.tokens], of_heads).view(qkv.shape)
            turn = (self.cos, self.sin)
            norm = dict(q_weight=self.weight, k_weight=self.weight)
            if self.cache_bits == 16:
                k_cache, v_cache = cache
                q = step.append(qkv, k_cache, v_cache, *turn, **norm)
                o = step.attention(q, k_cache, v_cache)
            else:
                q = step.append_fp4(qkv, cache, *turn, **norm)
                o = step.attention_fp4(q, cache)
            if self.weights:
                linear(linear(linear(o.flatten(1), from_heads), up), down)

    def time_us(self, step, repeats: int = 3) -> float:
        """Microseconds of the layers, the median of some passes."""
        torch = self.torch
        self.run(step)
        times = []
        for _ in range(repeats):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            self.run(step)
            b.record()
            b.synchronize()
            times.append(a.elapsed_time(b) * 1e3)
        return float(np.median(times))


def context_read(it: Iteration, prefix: int) -> int:
    """Tokens of context that an iteration's attention reads: shared ones once."""
    return it.context + prefix


def _nonnegative(x, y):
    """Least squares with no coefficient below zero."""
    keep = list(range(x.shape[1]))
    while keep:
        c, *_ = np.linalg.lstsq(x[:, keep], y, rcond=None)
        if (c >= 0).all():
            break
        keep.remove(keep[int(np.argmin(c))])
    full = np.zeros(x.shape[1])
    if keep:
        full[keep] = c
    return full


def fit(tokens, context, us):
    """(base, tok, div, share of the variance explained) of us = base + tok * tokens
    + context / div, by least squares with no coefficient below zero."""
    x = np.stack([np.ones(len(us)), np.asarray(tokens, float), np.asarray(context, float)], 1)
    y = np.asarray(us, float)
    c = _nonnegative(x, y)
    left = ((y - x @ c) ** 2).sum()
    var = ((y - y.mean()) ** 2).sum()
    return c[0], c[1], (1 / c[2] if c[2] > 0 else float("inf")), 1 - left / var if var > 0 else 1.0


NO_PRICE = 2 ** 31 - 1  # the divisor of a context without a price


def whole_terms(tokens, context, us):
    """(base, tok, div) as the engine holds them, whole numbers: for either neighbour of
    the fitted tok the base and div that fit what is left, the closer of the two."""
    tokens, context, y = (np.asarray(a, float) for a in (tokens, context, us))
    x = np.stack([np.ones(len(y)), context], 1)
    low = int(fit(tokens, context, us)[1])
    best = None
    for tok in (low, low + 1):
        base, slope = _nonnegative(x, y - tok * tokens)
        base = round(base)
        div = min(NO_PRICE, max(1, round(1 / slope))) if slope > 0 else NO_PRICE
        off = ((y - base - tok * tokens - context / div) ** 2).sum()
        if best is None or off < best[0]:
            best = (off, (base, tok, div))
    return best[1]


def measure(w: W.Workload, *, iterations=24, layers=32, heads=32, kv_heads=8, head_dim=128,
            dtype="bf16", prefix=0, seed=0, device="cuda", say=lambda line: None, plans=None,
            cache_bits=16, hidden=0, ffn=0):
    """Times of ``iterations`` iterations of the workload; a list of (requests, tokens,
    context, microseconds), the prefix once in the context. ``plans``: a list that
    receives the microseconds that the host took for each iteration's plan."""
    import torch

    from . import step as S

    e = w.engine
    rng = np.random.default_rng([seed, 31])
    prefix_pages = -(-prefix // e.block_tokens)
    positions = prefix + int((w.prompt.astype(np.int64) + w.decode).max())
    model = Layers(e, layers, heads, kv_heads, head_dim,
                   {"bf16": torch.bfloat16, "f16": torch.float16}[dtype], device, positions,
                   cache_bits, hidden, ffn)
    rows = []
    for i in range(iterations):
        it = form_iteration(w, int(rng.integers(0, w.n_traces)), int(rng.integers(0, w.n_req)), rng,
                            prefix_pages)
        shared = dict(prefix_first=[0, len(it.n_new)], prefix_len=[prefix],
                      prefix_blocks=np.arange(prefix_pages)[None]) if prefix else {}
        start = time.perf_counter()
        step = S.Step(it.n_new, it.kv_len, it.blocks, heads=heads, kv_heads=kv_heads,
                      head_dim=head_dim, block_tokens=e.block_tokens, n_blocks=e.kv_blocks,
                      device=device, **shared)
        plan_us = (time.perf_counter() - start) * 1e6
        if plans is not None:
            plans.append(plan_us)
        us = model.time_us(step)
        step.close()
        rows.append((len(it.n_new), it.tokens, context_read(it, prefix), us))
        say(f"{rows[-1][0]:4d} requests {rows[-1][1]:6d} tokens {rows[-1][2]:8d} context "
            f"{us:10.1f} us, plan {plan_us:6.1f}")
    return rows


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--cfg", type=int, default=4, help="workload (0 to 5)")
    p.add_argument("--iterations", type=int, default=24)
    p.add_argument("--layers", type=int, default=32)
    p.add_argument("--heads", type=int, default=32)
    p.add_argument("--kv-heads", type=int, default=8)
    p.add_argument("--head-dim", type=int, default=128)
    p.add_argument("--dtype", choices=["bf16", "f16"], default="bf16")
    p.add_argument("--cache-bits", type=int, choices=[16, 4], default=16)
    p.add_argument("--hidden", type=int, default=0,
                   help="with the products with a layer's weights in four bits, of a state of so many")
    p.add_argument("--ffn", type=int, default=0, help="of the layer's second half (4 * hidden)")
    p.add_argument("--prefix", type=int, default=0, help="shared tokens before every request")
    p.add_argument("--seed", type=int, default=0)
    a = p.parse_args(argv)
    w = W.make(a.cfg, n_traces=1, n_settings=4 if a.cfg != 0 else None)
    plans = []
    rows = measure(w, plans=plans, iterations=a.iterations, layers=a.layers, heads=a.heads,
                   kv_heads=a.kv_heads, head_dim=a.head_dim, dtype=a.dtype, prefix=a.prefix,
                   seed=a.seed, cache_bits=a.cache_bits, hidden=a.hidden, ffn=a.ffn,
                   say=lambda line: print(line, flush=True))
    _, tokens, context, us = zip(*rows)
    base, tok, div, r2 = fit(tokens, context, us)
    print(f"{w.name}, {a.layers} layers of {a.heads}/{a.kv_heads} heads of {a.head_dim}, "
          f"{a.dtype}, cache of {a.cache_bits} bits: {'attention and products' if a.hidden else 'attention'}"
          f" of an iteration = {base:.0f} + {tok:.4f} * tokens + context / "
          f"{div:.1f} us ({100 * r2:.1f}% of the variance)")
    whole = whole_terms(tokens, context, us)
    print("in whole numbers, for Engine(iter_base_us, iter_tok_us, iter_ctx_div): %d, %d, %d" % whole)
    print(f"the host plans an iteration in {np.median(plans):.0f} us (median), beside the GPU's "
          "work or before it")
    e = w.engine
    print(f"the workload's engine prices the whole iteration at {e.iter_base_us} + "
          f"{e.iter_tok_us} * tokens + context / {e.iter_ctx_div} us")


if __name__ == "__main__":
    main()
