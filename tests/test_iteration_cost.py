"""Iterations formed from a workload keep the engine's budgets, and the fit returns
the coefficients that made its data (no GPU); on a GPU, a short measurement."""
import numpy as np
import pytest

from paper_2606_18431_amd import iteration_cost as C
from paper_2606_18431_amd import workloads as W


@pytest.mark.parametrize("cfg", [0, 2, 4, 5])
@pytest.mark.parametrize("prefix_blocks", [0, 33])
def test_iterations_keep_the_budgets(cfg, prefix_blocks):
    w = W.make(cfg, n_traces=1, n_req=400)
    e = w.engine
    rng = np.random.default_rng(5)
    mixed = 0
    for first in (0, 17, 390):
        it = C.form_iteration(w, 0, first, rng, prefix_blocks)
        assert 1 <= len(it.n_new) <= e.max_seqs
        assert it.tokens <= e.max_tokens and (it.n_new >= 1).all() and (it.n_new <= e.chunk).all()
        assert (it.kv_len >= it.n_new).all()
        used = it.blocks[it.blocks >= 0]
        assert len(used) == len(set(used.tolist())) == (-(-it.kv_len // e.block_tokens)).sum()
        assert len(used) + prefix_blocks <= e.kv_blocks
        assert used.min() >= prefix_blocks and used.max() < e.kv_blocks
        for i, kv in enumerate(it.kv_len):
            r = (first + i) % w.n_req
            p, d = int(w.prompt[0, r]), int(w.decode[0, r])
            # a chunk of the prompt, or a decode step that is not the last token's
            assert (it.n_new[i] == 1 and p < kv <= p + d - 1) or \
                (kv <= p and (kv == p or kv % e.chunk == 0)
                 and it.n_new[i] == kv - (kv - 1) // e.chunk * e.chunk)
            mixed |= 1 if it.n_new[i] == 1 else 2
    assert mixed & 1


def test_fit_returns_the_coefficients():
    rng = np.random.default_rng(1)
    tokens, context = rng.integers(1, 8192, 40), rng.integers(1, 400_000, 40)
    base, tok, div, r2 = C.fit(tokens, context, 300 + 0.5 * tokens + context / 64)
    assert abs(base - 300) < 1e-6 and abs(tok - 0.5) < 1e-9 and abs(div - 64) < 1e-6 and r2 > 1 - 1e-9
    base, tok, div, r2 = C.fit(tokens, context, 100 - 0.001 * tokens + context / 50)
    assert tok == 0 and base > 0 and abs(div - 50) < 2 and r2 > 0.9


@pytest.mark.gpu
@pytest.mark.parametrize("prefix", [0, 100])
def test_measure_runs_the_operators(prefix):
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    w = W.make(1, n_traces=1, n_settings=4, n_req=200)
    rows = C.measure(w, iterations=4, layers=2, heads=8, kv_heads=2, head_dim=64, dtype="f16",
                     prefix=prefix)
    assert len(rows) == 4
    for n, tokens, context, us in rows:
        assert n >= 1 and tokens >= n and context >= tokens and 0 < us < 1e6


class FakeStep:
    """A step that notes the caches of its calls."""

    tokens = 3

    def __init__(self):
        self.calls = []

    def append(self, qkv, k_cache, v_cache, *args, **kw):
        assert qkv.shape[0] == self.tokens
        self.calls.append(("append", k_cache.data_ptr(), v_cache.data_ptr()))
        return "queries"

    def attention(self, q, k_cache, v_cache):
        assert q == "queries"
        self.calls.append(("attention", k_cache.data_ptr(), v_cache.data_ptr()))


def test_every_layer_has_a_cache_of_its_own():
    """As a model's layers have: what a layer reads was not read by the one before it, and
    is not in the caches of the chip for that."""
    torch = pytest.importorskip("torch")
    e = W.Engine(kv_blocks=4, max_tokens=64)
    m = C.Layers(e, 5, heads=2, kv_heads=1, head_dim=64, dtype=torch.float16, device="cpu",
                 positions=10)
    s = FakeStep()
    m.run(s)
    assert [c[0] for c in s.calls] == ["append", "attention"] * 5
    assert all(s.calls[i][1:] == s.calls[i + 1][1:] for i in range(0, 10, 2))
    assert len({p for c in s.calls for p in c[1:]}) == 10


@pytest.mark.gpu
def test_measure_gives_the_times_of_the_plans():
    """Each iteration's plan is timed too: it is made once an iteration, by the host."""
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    w = W.make(1, n_traces=1, n_settings=4, n_req=200)
    plans = []
    rows = C.measure(w, iterations=4, layers=2, heads=8, kv_heads=2, head_dim=64, dtype="f16",
                     plans=plans)
    assert len(plans) == len(rows) == 4 and all(0 < us < 1e6 for us in plans)


def test_a_shared_prefix_is_read_once():
    """The context that a batch costs: its requests' own, and the shared tokens once."""
    it = C.Iteration(np.array([1, 1, 40]), np.array([100, 7, 40]), np.zeros((3, 7), np.int32))
    assert it.context == 147
    assert C.context_read(it, 0) == 147 and C.context_read(it, 2048) == 147 + 2048


def test_whole_terms_fit_the_engine():
    """The engine's terms are whole numbers: the ones that fit best with the tokens' price
    rounded, not each rounded by itself."""
    rng = np.random.default_rng(2)
    tokens, context = rng.integers(1, 8192, 60), rng.integers(1, 400_000, 60)
    assert C.whole_terms(tokens, context, 300 + 2 * tokens + context / 64) == (300, 2, 64)
    us = 100 + 0.66 * tokens + context / 46
    base, tok, div = C.whole_terms(tokens, context, us)
    assert (tok, type(base), type(tok), type(div)) == (1, int, int, int)
    assert base >= 0 and div >= 1
    W.Engine(iter_base_us=base, iter_tok_us=tok, iter_ctx_div=div)

    def off(b, t, d):
        return ((us - b - t * tokens - context / d) ** 2).sum()

    for t in (0, 1):
        for b in (0, 100, base - 50, base + 50):
            for d in (46, div - 2, div + 2):
                assert b < 0 or off(base, tok, div) <= off(b, t, d)
    base, tok, div = C.whole_terms(tokens, context, 5.0 * tokens)  # no price of context
    assert (base, tok) == (0, 5) and div == 2 ** 31 - 1


def test_layers_refuse_what_they_would_not_run():
    """Other bits of a cache, and a second half of a layer without its first."""
    torch = pytest.importorskip("torch")
    for kw in (dict(cache_bits=8), dict(cache_bits=0), dict(ffn=64), dict(hidden=48),
               dict(hidden=-32), dict(hidden=64, ffn=100), dict(hidden=64, ffn=-64)):
        with pytest.raises(ValueError):
            C.Layers(W.Engine(kv_blocks=4, max_tokens=64), 1, heads=2, kv_heads=1, head_dim=64,
                     dtype=torch.float16, device="cpu", positions=10, **kw)
