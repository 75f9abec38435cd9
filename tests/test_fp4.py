"""The C ABI of the operators in four bits, without a GPU: declared symbols, struct layouts,
and arguments that are refused before any address is used."""
import ctypes
import os
import re
import subprocess

import pytest

from paper_2606_18431_amd import fp4, step, tas

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
AT = 1 << 40  # an address that nothing here uses


def test_library_exports_every_declared_symbol():
    src = open(os.path.join(ROOT, "include", "tas_fp4.h")).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    names = sorted(set(re.findall(r"\b(tas_fp4_[a-z_]+)\s*\(", src)))
    assert names == sorted(fp4.EXPORTS)
    for n in names:
        assert hasattr(step.lib(), n), n


def test_struct_layouts_match_header(tmp_path):
    structs = [fp4.tas_rows, fp4.tas_cache_fp4, fp4.tas_append_fp4, fp4.tas_attention_fp4,
               fp4.tas_tensor_fp4, fp4.tas_cache_values_fp4, fp4.tas_linear_fp4]
    lines = ['#include <stddef.h>', '#include <stdio.h>', '#include "tas_fp4.h"',
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
    assert step._APPEND_FP4.size == ctypes.sizeof(fp4.tas_append_fp4)
    assert step._ATTENTION_FP4.size == ctypes.sizeof(fp4.tas_attention_fp4)


def rows(p, *stride):
    return fp4.tas_rows(p, (ctypes.c_int64 * 3)(*stride))


@pytest.fixture
def bound():
    b, keep = step.make_batch([1, 3], [20, 3], [[0, 1], [2, 3]], heads=4, kv_heads=2, head_dim=64,
                              block_tokens=16, n_blocks=4)
    ctx = step.tas_step_create(b)
    step.tas_step_attach(ctx, AT, step.tas_step_bytes(ctx))
    yield ctx
    step.tas_step_destroy(ctx)


def cache(**kw):
    """Blocks of 2 heads of 16 tokens of 64: 32 bytes of codes and 2 of scales a row."""
    c = dict(k=rows(AT + (1 << 20), 1024, 512, 32), v=rows(AT + (2 << 20), 1024, 512, 32),
             k_scale=rows(AT + (3 << 20), 64, 32, 2), v_scale=rows(AT + (4 << 20), 64, 32, 2))
    c.update(kw)
    return fp4.tas_cache_fp4(*(c[n] for n in ("k", "v", "k_scale", "v_scale")))


def refused(call, ctx, args):
    return call(ctx, ctypes.byref(args), None) == tas.TAS_EINVAL


BAD_CACHES = [dict(k=rows(AT + 8, 1024, 512, 32)), dict(k=rows(None, 1024, 512, 32)),
              dict(v=rows(AT + (2 << 20), 1024, 512, 24)), dict(v=rows(AT, -1024, 512, 32)),
              dict(v=rows(AT, 1 << 31, 512, 32)), dict(v=rows(AT, 1024, 512, (1 << 24) + 16)),
              dict(k_scale=rows(AT + 1, 64, 32, 2)), dict(v_scale=rows(AT, 64, 31, 2)),
              dict(v_scale=rows(None, 64, 32, 2))]


def test_refused_attention(bound):
    """(The last argument that is looked at is refused in each: nothing is launched.)"""
    L = step.lib()

    def args(**kw):
        a = dict(dtype=1, scale=0.125, q=AT + (8 << 20), q_stride=256, out=AT + (9 << 20),
                 out_stride=256, lse=AT + (9 << 20), cache=cache())  # lse over out
        a.update(kw)
        return fp4.tas_attention_fp4(**a)

    assert L.tas_fp4_attention(None, None, None) == tas.TAS_EINVAL
    assert refused(L.tas_fp4_attention, bound, args())
    for kw in [dict(dtype=2), dict(scale=0), dict(scale=float("nan")), dict(scale=3e38),
               dict(q=AT + 8), dict(q=None), dict(q_stride=255), dict(q_stride=260),
               dict(out=None), dict(out_stride=248), dict(lse=AT + (10 << 20) + 2),
               dict(lse=AT + (1 << 20)), dict(lse=AT + (4 << 20)), dict(lse=AT + (8 << 20)),
               dict(out=AT + (8 << 20) + 16, lse=None), dict(out=AT + (2 << 20), lse=None),
               dict(out=AT + (4 << 20), lse=None)] + [dict(cache=cache(**c), lse=None)
                                                     for c in BAD_CACHES]:
        assert refused(L.tas_fp4_attention, bound, args(**kw)), kw


def test_refused_append(bound):
    L = step.lib()

    def args(**kw):
        a = dict(dtype=0, rot_dim=32, interleaved=0, eps=1e-6, qkv=AT + (8 << 20), qkv_stride=512,
                 q_out=AT + (9 << 20), q_out_stride=256, q_weight=AT + (10 << 20),
                 k_weight=AT + (11 << 20), cos=AT + (12 << 20), sin=AT + (9 << 20) + 1024,
                 positions=20, cache=cache())  # sin over q_out
        a.update(kw)
        return fp4.tas_append_fp4(**a)

    assert L.tas_fp4_append(None, None, None) == tas.TAS_EINVAL
    assert refused(L.tas_fp4_append, bound, args())
    apart = dict(sin=AT + (13 << 20))
    for kw in [dict(dtype=2), dict(rot_dim=24), dict(rot_dim=80), dict(interleaved=2),
               dict(eps=-1), dict(k_weight=None), dict(q_weight=AT + 8), dict(cos=None),
               dict(positions=19), dict(qkv=None), dict(qkv_stride=504), dict(q_out_stride=252),
               dict(qkv=AT + (9 << 20)), dict(q_out=AT + (8 << 20) + 512),
               dict(q_out=AT + (3 << 20)), dict(qkv=AT + (2 << 20)),
               dict(q_weight=AT + (9 << 20) + 256), dict(k_weight=AT + (1 << 20)),
               dict(cos=AT + (4 << 20))]:
        assert refused(L.tas_fp4_append, bound, args(**{**apart, **kw})), kw
    for c in BAD_CACHES + [dict(k=rows(AT + (1 << 20), 0, 512, 32)),
                           dict(k=rows(AT + (1 << 20), 1024, 256, 32)),
                           dict(k=rows(AT + (1 << 20), 1024, 512, 16)),
                           dict(v_scale=rows(AT + (4 << 20), 64, 0, 2)),
                           dict(k=rows(AT + (2 << 20) + 512, 1024, 512, 32)),
                           dict(k_scale=rows(AT + (4 << 20) + 64, 64, 32, 2)),
                           dict(k_scale=rows(AT + (1 << 20) + 64, 64, 32, 2))]:
        assert refused(L.tas_fp4_append, bound, args(**apart, cache=cache(**c))), c


def test_refused_strides_beyond_memory():
    """Token strides whose places pass 64 bits, where two rows would be one (nothing runs: the
    stride is refused before any launch); over 16-bit caches too."""
    L = step.lib()
    b, keep = step.make_batch([5], [20], [[0, 1]], heads=4, kv_heads=2, head_dim=64,
                              block_tokens=16, n_blocks=4)
    ctx = step.tas_step_create(b)
    step.tas_step_attach(ctx, AT, step.tas_step_bytes(ctx))
    wide = step.tas_cache(AT + (1 << 20), AT + (2 << 20), 2048, 1024, 64, 2048, 1024, 64)
    rows_ = dict(q=AT + (8 << 20), q_stride=256, out=AT + (9 << 20), out_stride=256)
    turn = dict(eps=1e-6, qkv=AT + (8 << 20), qkv_stride=512, q_out=AT + (9 << 20),
                q_out_stride=256)
    for stride in (1 << 62, (1 << 61) + 8, (1 << 63) - 8):
        for kw in (dict(q_stride=stride), dict(out_stride=stride),
                   dict(q_stride=stride, out_stride=stride, out=rows_["q"])):
            a = dict(dtype=1, scale=0.125, **{**rows_, **kw})
            assert refused(L.tas_fp4_attention, ctx, fp4.tas_attention_fp4(cache=cache(), **a)), kw
            assert refused(L.tas_step_attention, ctx, step.tas_attention(cache=wide, **a)), kw
        for kw in (dict(qkv_stride=stride), dict(q_out_stride=stride),
                   dict(qkv_stride=stride, q_out_stride=stride, q_out=turn["qkv"])):
            a = dict(dtype=1, **{**turn, **kw})
            assert refused(L.tas_fp4_append, ctx, fp4.tas_append_fp4(cache=cache(), **a)), kw
            assert refused(L.tas_step_append, ctx, step.tas_append(cache=wide, **a)), kw
    step.tas_step_destroy(ctx)


def test_unbound_steps_and_batches_that_cannot_be_appended():
    L = step.lib()
    b, keep = step.make_batch([1], [1], [[0]], heads=1, kv_heads=1, head_dim=64, block_tokens=16,
                              n_blocks=1)
    ctx = step.tas_step_create(b)
    assert L.tas_fp4_append(ctx, ctypes.byref(fp4.tas_append_fp4()), None) == tas.TAS_ESTATE
    assert L.tas_fp4_attention(ctx, ctypes.byref(fp4.tas_attention_fp4()), None) == tas.TAS_ESTATE
    step.tas_step_destroy(ctx)
    b, keep = step.make_batch([3], [2], [[0]], heads=1, kv_heads=1, head_dim=64, block_tokens=16,
                              n_blocks=1)
    ctx = step.tas_step_create(b)
    assert L.tas_fp4_append(ctx, ctypes.byref(fp4.tas_append_fp4()), None) == tas.TAS_EINVAL
    step.tas_step_destroy(ctx)


def test_refused_tensors():
    L = step.lib()

    def tensor(**kw):
        t = dict(dtype=1, reserved=0, n=(2, 3, 5), cols=64, x=rows(AT, 1920, 640, 128),
                 codes=rows(AT + (1 << 20), 480, 160, 32), scales=rows(AT + (1 << 20), 30, 10, 2))
        t.update(kw)
        t["n"] = (ctypes.c_int64 * 3)(*t["n"])
        return ctypes.byref(fp4.tas_tensor_fp4(**t))  # scales over codes

    apart = dict(scales=rows(AT + (2 << 20), 30, 10, 2))
    assert L.tas_fp4_pack(None, None) == L.tas_fp4_values(None, None) == tas.TAS_EINVAL
    assert L.tas_fp4_pack(tensor(), None) == tas.TAS_EINVAL
    assert L.tas_fp4_pack(tensor(n=(2, 0, 5)), None) == 0
    both = [dict(dtype=2), dict(reserved=1), dict(cols=48), dict(cols=0), dict(cols=-32),
            dict(n=(-1, 3, 5)), dict(n=(1 << 20, 1 << 20, 1)), dict(n=(1 << 62, 1 << 62, 4)), dict(n=(1 << 24, 1 << 5, 1)),
            dict(n=(1, 1 << 29, 1)),
            dict(cols=1 << 36), dict(x=rows(AT + 8, 1920, 640, 128)),
            dict(x=rows(AT, 1920, 640, 136)), dict(x=rows(AT, -1920, 640, 128)),
            dict(x=rows(None, 1920, 640, 128)), dict(codes=rows(AT + 2, 480, 160, 32)),
            dict(codes=rows(AT + (1 << 20), 480, 1 << 50, 32)), dict(scales=rows(None, 30, 10, 2)),
            dict(codes=rows(AT + 1900, 480, 160, 32)), dict(scales=rows(AT + 3800, 30, 10, 2))]
    for kw in both:
        assert L.tas_fp4_pack(tensor(**{**apart, **kw}), None) == tas.TAS_EINVAL, kw
        assert L.tas_fp4_values(tensor(**{**apart, **kw}), None) == tas.TAS_EINVAL, kw
    for kw in (dict(codes=rows(AT + (1 << 20), 480, 160, 16)), dict(scales=rows(AT + (2 << 20), 30, 0, 2)),
               dict(scales=rows(AT + (1 << 20) + 957, 30, 10, 2))):
        assert L.tas_fp4_pack(tensor(**{**apart, **kw}), None) == tas.TAS_EINVAL, kw
    assert L.tas_fp4_values(tensor(**apart, x=rows(AT, 1920, 0, 128)), None) == tas.TAS_EINVAL


def test_refused_cache_values():
    L = step.lib()

    def call(**kw):
        a = dict(dtype=1, head_dim=64, n_blocks=4, kv_heads=2, block_tokens=16, cache=cache(),
                 k=AT + (8 << 20), v=AT + (8 << 20) + 4096)  # v over the end of k
        a.update(kw)
        return L.tas_fp4_cache_values(ctypes.byref(fp4.tas_cache_values_fp4(**a)), None)

    assert L.tas_fp4_cache_values(None, None) == tas.TAS_EINVAL
    assert call() == tas.TAS_EINVAL
    apart = dict(v=AT + (9 << 20))
    assert call(**apart, n_blocks=0) == 0
    for kw in [dict(dtype=2), dict(head_dim=96), dict(n_blocks=-1), dict(kv_heads=1 << 32),
               dict(n_blocks=1 << 30, kv_heads=1 << 10), dict(kv_heads=1 << 20, block_tokens=1 << 20),
               dict(k=None), dict(k=AT + 8), dict(v=AT + (9 << 20) + 2), dict(k=AT + (2 << 20)),
               dict(v=AT + (3 << 20)), dict(v=AT + (1 << 20)), dict(k=AT + (4 << 20) + 128),
               dict(cache=cache(k=rows(AT + 2, 1024, 512, 32))),
               dict(cache=cache(v_scale=rows(None, 64, 32, 2)))]:
        assert call(**{**apart, **kw}) == tas.TAS_EINVAL, kw


def test_weights_bytes():
    L = step.lib()
    assert L.tas_fp4_weights_bytes(1, 32) == 1024 + 64
    assert L.tas_fp4_weights_bytes(17, 160) == 4 * (1024 + 64)
    assert L.tas_fp4_weights_bytes(4096, 4096) == 4096 * 4096 * 17 // 32
    for bad in ((0, 32), (-1, 32), (1, 0), (1, 16), (1, 48), (1, -32), (1 << 25, 32),
                (1, (1 << 20) + 32), (1 << 24, 1 << 20)):
        assert L.tas_fp4_weights_bytes(*bad) == 0, bad


# Sizes (tokens, rows, columns) for each of the product's kernels, by its number: columns that end
# inside a tile and that do not, that leave steps and groups of waves whole, in part or empty.
KERNEL_SHAPES = {
    0: [(1, 130, 1120), (8, 4090, 4192), (5, 100, 96)],
    1: [(8, 4100, 1184), (3, 8200, 96)],
    2: [(16, 100, 1120), (9, 4090, 4192)],
    3: [(16, 4100, 2144), (12, 16400, 4384)],
    4: [(16, 16400, 1120), (9, 16390, 4064), (12, 33000, 96), (16, 16390, 128), (13, 16390, 2080)],
    5: [(17, 5, 96), (32, 1000, 8224), (200, 100, 1120)],
    6: [(17, 4100, 1120), (31, 4100, 4192), (20, 16390, 544)],
    7: [(33, 4100, 1184), (17, 4100, 288), (127, 4090, 2144)],
    8: [(130, 5000, 1120), (33, 10000, 2144), (64, 10000, 4384)],
    9: [(17, 26000, 544), (25, 26000, 1184), (20, 16390, 4384), (32, 33000, 2080), (17, 26000, 2176)],
    10: [(33, 16390, 4128), (64, 16390, 4384), (200, 8100, 4384), (50, 16390, 8288)],
    11: [(33, 16390, 1120), (180, 10000, 96), (33, 26000, 160), (1030, 4090, 1184),
         (33, 33000, 4128)],
    12: [(33, 33000, 1120), (130, 33000, 544), (2040, 4090, 1120), (400, 33000, 288),
         (2000, 4000, 2080)],
    13: [(70, 26000, 96), (200, 26000, 544), (600, 20000, 1120), (2100, 8201, 288),
         (4090, 4100, 160)]}


def test_every_kernel_of_the_product_has_sizes():
    """Whatever the rule that chooses: the tests on a GPU reach each of its kernels."""
    header = open(os.path.join(ROOT, "include", "tas_fp4.h")).read()
    assert f"TAS_FP4_LINEAR_KERNELS = {fp4.LINEAR_KERNELS} " in header
    assert sorted(KERNEL_SHAPES) == list(range(fp4.LINEAR_KERNELS))
    number = step.lib().tas_fp4_linear_kernel
    for kernel, shapes in KERNEL_SHAPES.items():
        assert any(cols % 128 for _, _, cols in shapes)
        for shape in shapes:
            assert number(*shape) == kernel, shape


def test_kernel_of_refused_products():
    number = step.lib().tas_fp4_linear_kernel
    for bad in ((0, 40, 64), (-1, 40, 64), ((1 << 24) + 1, 40, 64), (3, 0, 64), (3, 40, 48),
                (3, (1 << 24) + 1, 64), (1 << 24, 1 << 24, 64)):
        assert number(*bad) == tas.TAS_EINVAL, bad


def test_refused_weights_and_products():
    L = step.lib()
    ok = [40, 64, AT, 32, AT + (1 << 20), 2, AT + (1 << 20)]  # (onto the scales)
    assert L.tas_fp4_weights(*ok, None) == tas.TAS_EINVAL
    for i, bad in ((0, 0), (1, 48), (2, None), (2, AT + 8), (3, 24), (3, -32), (3, (1 << 31) + 16),
                   (4, None), (5, -1), (6, None), (6, AT + 128), (6, AT)):
        args = ok[:6] + [AT + (2 << 20)]
        args[i] = bad
        assert L.tas_fp4_weights(*args, None) == tas.TAS_EINVAL, (i, bad)

    def linear(**kw):
        a = dict(dtype=1, reserved=0, tokens=3, rows=40, cols=64, x=AT, x_stride=64,
                 weights=AT + (1 << 20), y=AT + 128, y_stride=40)  # y over x
        a.update(kw)
        return L.tas_fp4_linear(ctypes.byref(fp4.tas_linear_fp4(**a)), None)

    assert L.tas_fp4_linear(None, None) == tas.TAS_EINVAL
    assert linear() == tas.TAS_EINVAL
    assert linear(tokens=0, x=None, y=None) == 0
    apart = dict(y=AT + (3 << 20))
    for kw in (dict(dtype=2), dict(reserved=1), dict(tokens=-1), dict(tokens=1 << 25),
               dict(rows=0), dict(cols=48), dict(x=None), dict(x=AT + 8), dict(x_stride=56),
               dict(x_stride=68), dict(x_stride=(1 << 24) + 8), dict(weights=None),
               dict(weights=AT + 128), dict(y=None), dict(y=AT + (3 << 20) + 1),
               dict(y_stride=39), dict(y_stride=1 << 31), dict(y=AT + (1 << 20) + 3000)):
        assert linear(**{**apart, **kw}) == tas.TAS_EINVAL, kw


def test_every_layer_has_a_cache_of_its_own():
    """As with caches of 16 bits: what a layer reads was not read by the one before it."""
    torch = pytest.importorskip("torch")
    from paper_2606_18431_amd import iteration_cost as C
    from paper_2606_18431_amd import workloads as W

    class Step:
        tokens = 3
        calls = []

        def append_fp4(self, qkv, cache, *args, **kw):
            assert qkv.shape[0] == self.tokens and isinstance(cache, fp4.Cache)
            self.calls.append(("append", *(t.data_ptr() for t in cache)))
            return "queries"

        def attention_fp4(self, q, cache):
            assert q == "queries"
            self.calls.append(("attention", *(t.data_ptr() for t in cache)))

    m = C.Layers(W.Engine(kv_blocks=4, max_tokens=64), 5, heads=2, kv_heads=1, head_dim=64,
                 dtype=torch.float16, device="cpu", positions=10, cache_bits=4)
    s = Step()
    m.run(s)
    assert [c[0] for c in s.calls] == ["append", "attention"] * 5
    assert all(s.calls[i][1:] == s.calls[i + 1][1:] for i in range(0, 10, 2))
    assert len({p for c in s.calls for p in c[1:]}) == 20


def test_a_layer_gives_each_product_the_result_before(monkeypatch):
    """Of a layer's run with its weights: the state through the heads' matrix to the append, the
    queries to the attention, its result back from the heads, up and down; each layer with its
    own matrices and cache."""
    torch = pytest.importorskip("torch")
    from paper_2606_18431_amd import iteration_cost as C
    from paper_2606_18431_amd import workloads as W

    calls = []

    class Weights:
        def __init__(self, codes, scales):
            assert scales.shape == (codes.shape[0], codes.shape[1] // 16)
            self.shape = codes.shape[0], 2 * codes.shape[1]

    def linear(x, w):
        assert x.shape == (3, w.shape[1])
        y = torch.empty((3, w.shape[0]), dtype=x.dtype)
        calls.append(("linear", x, w, y))
        return y

    class Step:
        tokens = 3

        def append_fp4(self, qkv, cache, *args, **kw):
            assert qkv.shape == (3, 8, 64)
            calls.append(("append", qkv, cache, torch.empty((3, 4, 64))))
            return calls[-1][-1]

        def attention_fp4(self, q, cache):
            calls.append(("attention", q, cache, torch.empty((3, 4, 64))))
            return calls[-1][-1]

    monkeypatch.setattr(fp4, "Weights", Weights)
    monkeypatch.setattr(fp4, "linear", linear)
    m = C.Layers(W.Engine(kv_blocks=4, max_tokens=64), 2, heads=4, kv_heads=2, head_dim=64,
                 dtype=torch.float16, device="cpu", positions=10, cache_bits=4, hidden=128, ffn=160)
    m.run(Step())
    assert [c[0] for c in calls] == \
        ["linear", "append", "attention", "linear", "linear", "linear"] * 2
    for layer in range(2):
        part = calls[6 * layer:6 * layer + 6]
        assert part[0][1].data_ptr() == m.x.data_ptr()
        for before, after in zip(part, part[1:]):
            assert after[1].data_ptr() == before[-1].data_ptr()
        products = [c[2] for c in part if c[0] == "linear"]
        assert [w.shape for w in products] == [(512, 128), (128, 256), (160, 128), (128, 160)]
        assert all(x is y for x, y in zip(products, m.weights[layer]))
        assert part[1][2] is part[2][2] is m.caches[layer]
