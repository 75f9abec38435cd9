"""A serving iteration in four bits against its formulas in 64 bits on the CPU: rounding to
four bits and back, append and attention over a paged cache in four bits, products with
weights in four bits; at the sizes where a kernel can go wrong, strided tensors, slots that
nobody may read, other streams and graphs."""
import math

import numpy as np
import pytest

from paper_2606_18431_amd import fp4, step, tas
from test_gpu_step import EDGES, ROUND, Batch, append_reference, dtype_of, near, reference

pytestmark = pytest.mark.gpu

MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
EXPONENTS = {"bf16": (-125, 125), "f16": (-23, 13)}


@pytest.fixture(scope="module")
def torch():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def stand_for(torch, codes, scales):
    """The values in float64, on the CPU."""
    c = codes.cpu().long()
    c = torch.stack([c & 15, c >> 4], -1).flatten(-2)
    m = torch.tensor(MAGNITUDES + tuple(-x for x in MAGNITUDES), dtype=torch.float64)
    f = 2.0 ** (scales.cpu().double() - 127)
    f[scales.cpu() == 255] = math.nan
    return m[c] * f.repeat_interleave(32, -1)


def rounded(torch, x, name):
    """float64 x [..., n] rounded to four bits, the nearest of the eight by search, the even
    code of two as near; and how far, relatively, each is from a border of two codes or its
    block's largest from one of two scales."""
    lo, hi = EXPONENTS[name]
    y = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    most = y.abs().amax(-1)
    e = torch.full_like(most, lo)
    for k in range(lo, hi):
        e = torch.where(most >= 7 * 2.0 ** k, torch.full_like(e, k + 1), e)
    t = y.abs() / 2.0 ** e[..., None]
    m = torch.tensor(MAGNITUDES, dtype=torch.float64)
    off = (t[..., None] - m).abs()
    even_first = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7])
    code = even_first[off[..., even_first].argmin(-1)]
    borders = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float64)
    near_code = ((t[..., None] - borders).abs() / borders).amin(-1)
    near_scale = ((most / 2.0 ** e) / 3.5 - 1).abs().minimum(((most / 2.0 ** e) / 7 - 1).abs())
    value = m[code] * torch.where(torch.signbit(y), -1.0, 1.0) * 2.0 ** e[..., None]
    bad = ~torch.isfinite(most)
    value[bad] = math.nan
    # (a zero is at no border of a scale)
    near_scale[most == 0] = 1
    close = near_code.minimum(near_scale[..., None])
    return value.reshape(x.shape), close.reshape(x.shape)


def same(got, want):
    return bool(((got == want) | (got.isnan() & want.isnan())).all())


# ------------------------------------------------------------------ to four bits and back


@pytest.mark.parametrize("name", ["bf16", "f16"])
def test_values_of_every_code_and_scale(torch, name):
    """All 256 bytes of codes at all 256 scales: exact where the 16-bit type has the value,
    rounded as it rounds elsewhere, NaN at 255."""
    codes = torch.arange(256, dtype=torch.uint8).repeat(256, 1)
    scales = torch.arange(256, dtype=torch.uint8)[:, None].repeat(1, 16)
    got = fp4.values(codes.cuda(), scales.cuda(), dtype_of(torch, name))
    want = stand_for(torch, codes, scales).to(dtype_of(torch, name)).double()
    assert same(got.double().cpu(), want)


@pytest.mark.parametrize("name", ["bf16", "f16"])
def test_pack_every_border(torch, name):
    """Values at, just below and just above every border, at many exponents: at the ends of
    the range, among the type's subnormal numbers, with zeros of both signs."""
    dt = dtype_of(torch, name)
    lo, hi = (-133, 127) if name == "bf16" else (-24, 15)
    rows = []
    for e in list(range(lo, lo + 14)) + list(range(-8, 9)) + list(range(hi - 6, hi + 1)):
        b = torch.tensor([0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7, 0],
                         dtype=torch.float64) * 2.0 ** e
        for most in (4, 5, 6, 6.9, 7, 7.9):
            x = torch.cat([b[b.abs() <= most * 2.0 ** e], torch.zeros(32, dtype=torch.float64)])[:32]
            x[31] = most * 2.0 ** e
            for f in (1, 1 + 2.0 ** -7, 1 - 2.0 ** -8, -1):
                y = (x * f).to(dt)
                rows.append(torch.where(y.isinf(), torch.zeros_like(y), y))
    x = torch.stack(rows)
    want, _ = rounded(torch, x.double(), name)
    codes, scales = fp4.pack(x.cuda())
    assert codes.shape == (len(x), 16) and scales.shape == (len(x), 1)
    assert same(stand_for(torch, codes, scales), want)
    assert same(fp4.values(codes, scales, dt).double().cpu(), want)  # each is one of the type
    assert torch.equal(torch.signbit(fp4.values(codes, scales, dt)).cpu(), torch.signbit(x))


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("shape", [(32,), (1, 64), (7, 96), (3, 5, 128), (2, 3, 17, 64), (2, 4128),
                                   (1000, 32), (0, 64), (3, 0, 32)])
def test_pack_and_values(torch, name, shape):
    g = torch.Generator().manual_seed(3)
    dt = dtype_of(torch, name)
    x = (torch.randn(shape, generator=g) * torch.exp(3 * torch.randn(shape, generator=g))).to(dt)
    want, _ = rounded(torch, x.double(), name)
    codes, scales = fp4.pack(x.cuda())
    assert codes.shape == (*shape[:-1], shape[-1] // 2)
    assert scales.shape == (*shape[:-1], shape[-1] // 32)
    assert same(stand_for(torch, codes, scales), want)
    assert same(fp4.values(codes, scales, dt).double().cpu(), want)


def test_pack_blocks_with_infinities(torch):
    """A value that is not finite makes its block NaN, and no other."""
    x = torch.randn((6, 96), dtype=torch.bfloat16)
    for i, bad in enumerate((math.nan, math.inf, -math.inf)):
        x[i, 32 + 7 * i] = bad
    x[4, 0] = 3.3e38
    codes, scales = fp4.pack(x.cuda())
    v = fp4.values(codes, scales, torch.bfloat16).cpu()
    want, _ = rounded(torch, x.double(), "bf16")
    assert same(v.double(), want)
    assert bool(v[:3, 32:64].isnan().all()) and not bool(v[3:].isnan().any())
    assert bool((scales[:3, 1] == 255).all()) and not bool(codes[:3, 16:32].any())


def test_strided_tensors(torch):
    """Rows apart, permuted and broadcast dimensions."""
    big = torch.randn((5, 7, 3, 160), device="cuda", dtype=torch.float16)
    for x in (big[:, :, :, 32:96], big.permute(2, 0, 1, 3), big[::2, 1:, 1], big[0, 0, :1].expand(9, 160),
              big[1, 2, 1]):
        codes, scales = fp4.pack(x)
        ref = fp4.pack(x.contiguous())
        assert torch.equal(codes, ref[0]) and torch.equal(scales, ref[1])
    codes, scales = fp4.pack(big)
    want = fp4.values(codes, scales, torch.float16)
    for p in ((0, 1, 2, 3), (2, 1, 0, 3), (1, 2, 0, 3)):
        assert torch.equal(fp4.values(codes.permute(p), scales.permute(p), torch.float16),
                           want.permute(p))
    assert torch.equal(fp4.values(codes[:, :, :, 16:48], scales[..., 1:3], torch.float16),
                       want[..., 32:96])


# ------------------------------------------------------------------ append


def cache_of(torch, b, seed, order="head", poison=True):
    """A cache of random codes and scales around 1 in the given order of memory; slots that
    nobody may read are NaN. With its values in float64."""
    g = torch.Generator().manual_seed(seed)
    seen = torch.zeros((b.n_blocks, b.block), dtype=torch.bool)
    for i in range(len(b.n)):
        sl = b.slots(i)
        seen[sl[:, 0], sl[:, 1]] = True
    tensors, vals = [], []
    for _ in range(2):
        shape = (b.n_blocks, b.kv_heads, b.block)
        c = torch.randint(0, 256, (*shape, b.size // 2), generator=g, dtype=torch.uint8)
        s = torch.randint(123, 128, (*shape, b.size // 32), generator=g, dtype=torch.uint8)
        if poison:
            s = torch.where(seen[:, None, :, None], s, torch.full_like(s, 255))
        vals.append(stand_for(torch, c, s))
        tensors += [c, s]
    k, ks, v, vs = tensors
    if order == "head":
        got = [t.cuda() for t in (k, v, ks, vs)]
    elif order == "token":
        got = [t.permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3) for t in (k, v, ks, vs)]
    else:  # K and V of a block beside each other, codes and scales apart
        cc = torch.stack([k, v], 1).cuda()
        ss = torch.stack([ks, vs], -2).cuda()
        got = [cc[:, 0], cc[:, 1], ss[..., 0, :], ss[..., 1, :]]
    return fp4.Cache(*got), vals


@pytest.mark.parametrize("size", [64, 128])
@pytest.mark.parametrize("order", ["head", "token", "beside"])
def test_cache_values(torch, size, order):
    """Keys and values at once, as ``values`` gives each; an empty pool."""
    b = Batch(25, [3, 1], [50, 20], 6, 3, size, block=32)
    cache, (k, v) = cache_of(torch, b, 4, order)
    for dt in (torch.bfloat16, torch.float16):
        got = cache.values(dt)
        assert got[0].shape == (b.n_blocks, 3, 32, size) and got[0].dtype == dt
        assert same(got[0].double().cpu(), k) and same(got[1].double().cpu(), v)
    assert fp4.Cache(*(t[:0] for t in cache)).values(torch.float16)[1].shape == (0, 3, 32, size)
    for i, t in enumerate(cache):
        for bad in (t[1:], t.char(), t.cpu(), t[..., ::2]):
            with pytest.raises(ValueError):
                fp4.Cache(*(bad if j == i else u for j, u in enumerate(cache))).values(torch.float16)
    with pytest.raises(ValueError):
        cache.values(torch.float32)


def check_append(torch, b, name, rot, interleaved, norm, order="head"):
    print(f"[gpu] append_fp4 {name} n={b.n.tolist()[:8]} heads={b.heads}/{b.kv_heads}x{b.size} "
          f"block={b.block} rot={rot} interleaved={interleaved} norm={norm}", flush=True)
    dt = dtype_of(torch, name)
    cache, _ = cache_of(torch, b, 8, order, poison=False)
    before = [t.clone() for t in cache]
    g = torch.Generator().manual_seed(77)
    H, Hk, D = b.heads, b.kv_heads, b.size
    qkv = torch.randn((b.T, H + 2 * Hk, D), generator=g).to(dt).cuda()
    qkv[-1, 0] = 0  # a head of zeros
    qkv[-1, -1] = 0
    cos = sin = qw = kw = None
    if rot:
        a = torch.rand((int(b.positions().max()) + 1, rot // 2), generator=g) * 6.3
        cos, sin = a.cos().cuda(), a.sin().cuda()
    if norm:
        qw, kw = (1 + 0.2 * torch.randn((2, D), generator=g)).to(dt).cuda()
    want, tol = append_reference(torch, b, qkv, cos, sin, qw, kw, 1e-5, interleaved)
    s = b.step()
    q = s.append_fp4(qkv, cache, cos, sin, q_weight=qw, k_weight=kw, eps=1e-5,
                     interleaved=interleaved)
    torch.cuda.synchronize()
    # below the smallest normal number a 16-bit float keeps 2^-25
    qtol = tol + ROUND[name] * want.abs() * 1.01 + (2.0 ** -25 if name == "f16" else 2.0 ** -140)
    near(q, want[:, :H], qtol[:, :H], "queries")
    keys, close = rounded(torch, want[:, H:H + Hk], name)
    vals, _ = rounded(torch, qkv[:, H + Hk:].double().cpu(), name)
    # The reference and the kernel each work keys out in 64 bits: some 150 roundings of
    # 2^-53, on terms a few times the result (2^-40 is a thousand times that). Only keys
    # nearer to a border than that may differ.
    k, v = (stand_for(torch, c, e) for c, e in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)))
    t = 0
    for i in range(len(b.n)):
        sl = b.slots(i)[len(b.slots(i)) - int(b.n[i]):]
        for (page, at) in sl:
            ok = (k[page, :, at] == keys[t]) | (close[t] < 2.0 ** -40)
            assert bool(ok.all()), ("keys", i, t)
            assert torch.equal(v[page, :, at], vals[t]), ("values", i, t)
            for x, y in zip(cache, before):
                y[page, :, at] = x[page, :, at]
            t += 1
    assert all(torch.equal(x, y) for x, y in zip(cache, before))  # nothing else was written
    assert float((close < 2.0 ** -40).double().mean()) < 0.01


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("size,rot", [(64, 64), (64, 32), (64, 16), (128, 128), (128, 64),
                                      (128, 96), (128, 16)])
def test_append(torch, name, size, rot, interleaved):
    n, kv = [1, 5, 0, 37, 1], [33, 5, 9, 100, 1]
    check_append(torch, Batch(20, n, kv, 6, 2, size), name, rot, interleaved, norm=rot != 32)
    check_append(torch, Batch(21, n, kv, 7, 7, size, block=32, first=[0, 2, 5], prefix=[20, 7]),
                 name, rot, interleaved, norm=True, order="token")


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (8, 1), (33, 3)])
def test_append_heads(torch, heads, kv_heads):
    check_append(torch, Batch(22, [1, 3], [1, 60], heads, kv_heads, 128), "bf16", 128, False, True)
    check_append(torch, Batch(22, [1, 3], [1, 60], heads, kv_heads, 64), "f16", 64, True, True,
                 order="beside")


@pytest.mark.parametrize("name", ["bf16", "f16"])
def test_append_without_norm_and_rotation_is_pack(torch, name):
    """Keys and values as they are: what ``pack`` makes of them, infinities among them."""
    dt = dtype_of(torch, name)
    b = Batch(23, [4, 30], [4, 60], 2, 2, 64)
    cache, _ = cache_of(torch, b, 3, poison=False)
    qkv = (torch.randn((b.T, 6, 64)) * torch.exp(4 * torch.randn((b.T, 6, 1)))).to(dt).cuda()
    qkv[3, 2, 5], qkv[7, 3, 40], qkv[9, 4, 2], qkv[9, 5, 33] = math.inf, math.nan, -math.inf, math.nan
    q = b.step().append_fp4(qkv, cache)
    assert torch.equal(q, qkv[:, :2])
    codes, scales = fp4.pack(qkv)
    t = 0
    for i in range(2):
        for (page, at) in b.slots(i)[len(b.slots(i)) - int(b.n[i]):]:
            assert torch.equal(cache.k[page, :, at], codes[t, 2:4])
            assert torch.equal(cache.k_scale[page, :, at], scales[t, 2:4])
            assert torch.equal(cache.v[page, :, at], codes[t, 4:])
            assert torch.equal(cache.v_scale[page, :, at], scales[t, 4:])
            t += 1


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("scale", [1.0, 2.0 ** -10, 2.0 ** 14, 2.0 ** -70, 2.0 ** 62])
def test_append_keys_at_borders(torch, name, scale):
    """Two million keys, some of which lie within a rounding error of 32 bits of the border
    of two codes or scales: each has the code of the formula in 64 bits. Also where squares
    leave the range of 32 bits."""
    if name == "f16" and not 2.0 ** -12 < scale < 2.0 ** 12:
        pytest.skip("beyond the type")
    dt, T = dtype_of(torch, name), 2000
    b = Batch(24, [T], [T], 8, 8, 128)
    cache = fp4.Cache.zeros(b.n_blocks, 8, 16, 128)
    g = torch.Generator().manual_seed(12)
    qkv = (scale * torch.randn((T, 24, 128), generator=g)).to(dt)
    qkv[::3, 8:16] = qkv[::3, 8:16].sign() * scale                   # norms that are powers of two
    qkv[1::3, 8:16, 32:64] *= 2.0 ** -6
    a = torch.rand((T, 64), generator=g) * 6.3
    a[::2] = torch.randint(0, 9, (T // 2, 64), generator=g) * (math.pi / 4)
    cos, sin = a.cos(), a.sin()
    qw, kw = (torch.randint(1, 9, (2, 128), generator=g) / 4).to(dt)
    want, _ = append_reference(torch, b, qkv, cos, sin, qw, kw, 0.0, False)
    b.step().append_fp4(qkv.cuda(), cache, cos.cuda(), sin.cuda(), q_weight=qw.cuda(),
                        k_weight=kw.cuda(), eps=0.0)
    k, _ = cache.values(dt)
    page = torch.from_numpy(b.blocks[0]).long()[torch.arange(T) // 16]
    got = k.double().cpu()[page, :, torch.arange(T) % 16]
    keys, close = rounded(torch, want[:, 8:16], name)
    # 64 bits: some 150 roundings of 2^-53, on terms a few times the result
    assert bool(((got == keys) | (close < 2.0 ** -40)).all())
    assert bool((close < 2.0 ** -22).any())


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rot", [0, 64, 128])
@pytest.mark.parametrize("size,weight", [(40, -98), (55, -99), (58, -60), (-10, 118), (-10, 121),
                                         (-40, 90), (0, -126), (0, 121)])
def test_append_weights_at_the_ends(torch, size, weight, rot, interleaved):
    """Heads and norm weights of opposite sizes, whose quotient leaves the range of 32 bits
    though the result does not; zeros among the elements. Keys have the codes of the formula
    in 64 bits, queries its value within the roundings of 32."""
    T = 150
    b = Batch(24, [T], [T], 4, 2, 128)
    cache = fp4.Cache.zeros(b.n_blocks, 2, 16, 128)
    g = torch.Generator().manual_seed(14)
    qkv = (2.0 ** size * torch.randn((T, 8, 128), generator=g)).bfloat16()
    qkv[:, :, ::5] = 0
    qkv[::2, :, 3::4] = 0  # whole rotated pairs, of both kinds, among them
    qkv[::2, :, 2::4] = 0
    w = torch.randint(1, 9, (2, 128), generator=g) / 4
    w[:, 32:64] *= 2.0 ** weight
    w[:, 96:] *= 2.0 ** weight
    qw, kw = w.bfloat16()
    cos = sin = None
    if rot:
        a = torch.rand((T, rot // 2), generator=g) * 6.3
        a[::2] = torch.randint(0, 9, (T // 2, rot // 2), generator=g) * (math.pi / 4)
        cos, sin = a.cos().cuda(), a.sin().cuda()
    want, tol = append_reference(torch, b, qkv, cos, sin, qw, kw, 0.0, interleaved)
    assert torch.isfinite(want).all()
    q = b.step().append_fp4(qkv.cuda(), cache, cos, sin, q_weight=qw.cuda(), k_weight=kw.cuda(),
                            eps=0.0, interleaved=interleaved)
    k, _ = cache.values(torch.bfloat16)
    page = torch.from_numpy(b.blocks[0]).long()[torch.arange(T) // 16]
    got = k.double().cpu()[page, :, torch.arange(T) % 16]
    keys, close = rounded(torch, want[:, 4:6], "bf16")
    # 64 bits: some 150 roundings of 2^-53, on terms a few times the result
    assert bool(((got == keys) | (close < 2.0 ** -40)).all())
    # a bfloat16 is a multiple of 2^-133, and 32 bits of 2^-149
    near(q, want[:, :4], tol[:, :4] + ROUND["bf16"] * want[:, :4].abs() * 1.01 + 2.0 ** -133,
         "queries")


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("small,weight,turn", [(-133, 110, 0), (-125, 40, 60), (-100, 0, 100),
                                               (-133, 127, 20), (-120, 60, 0)])
def test_append_keys_lost_in_32_bits(torch, small, weight, turn, interleaved):
    """Keys of which 32 bits keep a part or nothing at a stage, brought back by weights or
    angles: the codes of the formula in 64 bits."""
    T = 150
    b = Batch(24, [T], [T], 2, 2, 128)
    cache = fp4.Cache.zeros(b.n_blocks, 2, 16, 128)
    g = torch.Generator().manual_seed(15)
    qkv = torch.randn((T, 6, 128), generator=g, dtype=torch.float64)
    w = (torch.randint(1, 9, (128,), generator=g) / 4).double()
    for at in (slice(32, 64), slice(96, 128)):  # rotated with one another, or by themselves
        qkv[:, :, at] *= 2.0 ** small
        w[at] *= 2.0 ** min(weight, 126)
    qkv[:, :, :32] *= 2.0 ** 55
    qkv, w = qkv.bfloat16(), w.bfloat16()
    a = torch.rand((T, 64), generator=g) * 6.3
    cos, sin = 2.0 ** turn * a.cos(), 2.0 ** turn * a.sin()
    want, _ = append_reference(torch, b, qkv, cos, sin, w, w, 0.0, interleaved)
    assert torch.isfinite(want.float()).all()
    b.step().append_fp4(qkv.cuda(), cache, cos.cuda(), sin.cuda(), q_weight=w.cuda(),
                        k_weight=w.cuda(), eps=0.0, interleaved=interleaved)
    k, _ = cache.values(torch.bfloat16)
    page = torch.from_numpy(b.blocks[0]).long()[torch.arange(T) // 16]
    got = k.double().cpu()[page, :, torch.arange(T) % 16]
    keys, close = rounded(torch, want[:, 2:4], "bf16")
    # 64 bits: some 150 roundings of 2^-53, on terms a few times the result
    assert bool(((got == keys) | (close < 2.0 ** -40)).all())
    assert (got[..., 32:64] != 0).any()  # (not all below the smallest scale's codes)



@pytest.mark.parametrize("size", [64, 128])
def test_append_in_place(torch, size):
    """The queries over their own rows of queries, keys and values, the others as they were."""
    b = Batch(26, [1, 7, 0, 40], [33, 9, 5, 90], 8, 2, size)
    qkv = torch.randn((48, 12, size), device="cuda", dtype=torch.bfloat16)
    cos, sin = torch.rand((2, 100, size // 2), device="cuda")
    w = torch.rand(size, device="cuda").bfloat16()
    one, two = (fp4.Cache.zeros(b.n_blocks, 2, 16, size) for _ in range(2))
    s, x = b.step(), qkv.clone()
    want = s.append_fp4(qkv, one, cos, sin, q_weight=w, k_weight=w)
    got = s.append_fp4(x, two, cos, sin, q_weight=w, k_weight=w, out=x[:, :8])
    assert got.data_ptr() == x.data_ptr() and torch.equal(got, want)
    assert torch.equal(x[:, 8:], qkv[:, 8:])
    assert all(torch.equal(t, u) for t, u in zip(one, two))

# ------------------------------------------------------------------ attention


def check_attention(torch, b, name, seed=1, order="head", scale=None):
    print(f"[gpu] attention_fp4 {name} n={b.n.tolist()[:8]} kv={b.kv.tolist()[:8]} heads="
          f"{b.heads}/{b.kv_heads}x{b.size} block={b.block} prefix={b.prefix}", flush=True)
    dt = dtype_of(torch, name)
    cache, (k, v) = cache_of(torch, b, seed, order)
    g = torch.Generator().manual_seed(seed + 100)
    q = torch.randn((b.T, b.heads, b.size), generator=g).to(dt)
    sc = scale if scale is not None else b.size ** -0.5
    want, wlse, tol, ltol = reference(torch, b, q, k, v, sc, ROUND[name])
    s = b.step()
    lse = torch.full((b.T, b.heads), 7.0, device="cuda")
    out = s.attention_fp4(q.cuda(), cache, scale=scale, lse=lse)
    torch.cuda.synchronize()
    near(out, want, tol, "out")
    near(lse, wlse, ltol, "lse")


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
    check_attention(torch, Batch(6, [n], [kv], 2 * group, 2, 64), "f16")


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


@pytest.mark.parametrize("causal", [True, False])
def test_rows_without_keys(torch, causal):
    """More new tokens than keys: the first rows see nothing (causal); requests
    without any key give zeros and -inf, in thin and wide items."""
    n = [1, 5, 40, 200, 2, 1]
    kv = [0, 2, 0, 150, 90, 0]
    check_attention(torch, Batch(10, n, kv, 4, 2, 64, causal=causal), "bf16")
    check_attention(torch, Batch(10, n, kv, 4, 1, 128, causal=causal), "f16")


@pytest.mark.parametrize("order", ["token", "beside"])
@pytest.mark.parametrize("size", [64, 128])
def test_other_cache_orders(torch, order, size):
    n, kv = [1, 40, 1, 300], [100, 90, 17, 400]
    check_attention(torch, Batch(11, n, kv, 8, 2, size, block=32), "bf16", order=order)


def test_scale_and_large_scores(torch):
    """Scores of some hundreds: only differences to the maximum reach the exponent."""
    check_attention(torch, Batch(12, [1, 33], [200, 333], 4, 2, 64), "f16", scale=4.0)
    check_attention(torch, Batch(12, [1, 33], [200, 333], 4, 2, 64), "bf16", scale=1e-4)


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("size", [64, 128])
@pytest.mark.parametrize("n,kv,heads", [(1, 90, 4), (5, 40, 2), (3, 90, 10), (70, 70, 1),
                                        (200, 333, 2), (150, 160, 8)])
def test_values_after_a_token_do_not_reach_it(torch, name, size, n, kv, heads):
    """A new token's block of V that is NaN makes the tokens from it on NaN (a row as a
    whole, or the block's elements) and leaves those before it as they were; so its keys."""
    b = Batch(33, [n], [kv], heads, 1, size)
    cache, _ = cache_of(torch, b, 3)
    q = torch.randn((n, heads, size)).to(dtype_of(torch, name)).cuda()
    s = b.step()
    clean = s.attention_fp4(q, cache)
    for bad in {n - 1, n // 2, n // 3}:
        y = kv - n + bad
        for scales in (cache.v_scale, cache.k_scale):
            at = (b.blocks[0, y // 16], 0, y % 16, 1)
            old = int(scales[at])
            scales[at] = 255
            got = s.attention_fp4(q, cache)
            scales[at] = old
            assert torch.equal(got[:bad], clean[:bad])
            assert not torch.isfinite(got[bad:, :, 32:64]).any()
    assert torch.equal(s.attention_fp4(q, cache), clean)


def test_strided_queries_output_in_place_and_determinism(torch):
    b = Batch(14, [1, 60, 3], [3000, 80, 700], 8, 2, 128)
    cache, _ = cache_of(torch, b, 4)
    qkv = torch.randn((b.T, 12, 128), device="cuda").to(torch.bfloat16)
    q = qkv[:, :8]
    s = b.step()
    want = s.attention_fp4(q.contiguous(), cache)
    assert torch.equal(s.attention_fp4(q, cache), want)          # rows apart
    wide = torch.full((b.T, 10, 128), 3.0, device="cuda", dtype=torch.bfloat16)
    s.attention_fp4(q, cache, out=wide[:, 1:9])
    assert torch.equal(wide[:, 1:9], want)
    assert bool((wide[:, 0] == 3).all()) and bool((wide[:, 9] == 3).all())
    assert s.attention_fp4(q, cache, out=q).data_ptr() == qkv.data_ptr()
    assert torch.equal(q, want)


def test_blocks_beyond_four_gigabytes(torch):
    """Offsets that pass 32 bits: the pages lie at the far end of pools of 5 GB."""
    n_blocks = 5 << 16
    small = Batch(16, [1, 70], [100, 700], 16, 16, 128)
    cs, _ = cache_of(torch, small, 6)
    far = np.where(small.blocks >= 0, n_blocks - 1 - small.blocks, -1)
    back = (n_blocks - 1 - torch.arange(small.n_blocks)).cuda()
    big = fp4.Cache(*(torch.empty((n_blocks, *t.shape[1:]), dtype=torch.uint8, device="cuda")
                      for t in cs))
    for t, u in zip(big, cs):
        t[back] = u
    assert big.k.numel() > 4 << 30
    s = step.Step(small.n, small.kv, far, heads=16, kv_heads=16, head_dim=128, block_tokens=16,
                  n_blocks=n_blocks)
    qkv = torch.randn((71, 48, 128), device="cuda").to(torch.bfloat16)
    q1 = small.step().append_fp4(qkv, cs)
    q2 = s.append_fp4(qkv, big)
    assert torch.equal(q1, q2)
    assert all(torch.equal(t[back], u) for t, u in zip(big, cs))
    assert torch.equal(s.attention_fp4(q2, big), small.step().attention_fp4(q1, cs))


# ------------------------------------------------------------------ products


def check_linear(torch, tokens, rows, cols, name, x=None, scales=None):
    print(f"[gpu] linear {name} {tokens} x {rows} x {cols}", flush=True)
    dt = dtype_of(torch, name)
    g = torch.Generator().manual_seed(tokens + 7 * rows + cols)
    codes = torch.randint(0, 256, (rows, cols // 2), generator=g, dtype=torch.uint8)
    if scales is None:
        scales = torch.randint(118, 124, (rows, cols // 32), generator=g, dtype=torch.uint8)
    if x is None:
        x = torch.randn((tokens, cols), generator=g).to(dt)
    w = stand_for(torch, codes, scales)
    want = x.double() @ w.T
    # Each product is exact in 32 bits; it goes through at most the 32 sums of its matrix
    # instruction, one for each later instruction and the join of the parts.
    tol = ROUND[name] * want.abs() * 1.01 + (cols / 32 + 48) * 2.0 ** -23 * (x.double().abs() @ w.T.abs()) \
        + (2.0 ** -25 if name == "f16" else 2.0 ** -133)
    got = fp4.linear(x.cuda(), fp4.Weights(codes.cuda(), scales.cuda()))
    assert got.shape == (tokens, rows)
    near(got, want, tol, "y")


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("tokens", [1, 2, 15, 16, 17, 31, 33, 64, 65, 127, 129, 300])
def test_linear_tokens(torch, name, tokens):
    check_linear(torch, tokens, 80, 544, name)


@pytest.mark.parametrize("tokens", [1, 20, 50, 200])
@pytest.mark.parametrize("rows", [1, 3, 15, 17, 63, 255, 257, 1000])
def test_linear_rows(torch, tokens, rows):
    check_linear(torch, tokens, rows, 256, "bf16")


@pytest.mark.parametrize("tokens", [1, 40, 130])
@pytest.mark.parametrize("cols", [32, 64, 96, 128, 160, 480, 512, 544, 2080, 4096, 4128, 8224])
def test_linear_cols(torch, tokens, cols):
    check_linear(torch, tokens, 130, cols, "f16")


@pytest.mark.parametrize("tokens,rows", [(5, 8200), (5, 16400), (33, 8200), (40, 16400), (90, 8200)])
def test_linear_many_rows(torch, tokens, rows):
    check_linear(torch, tokens, rows, 160, "bf16")


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("tokens,rows,cols", [(4090, 4100, 160), (4096, 4096, 32), (2100, 8201, 288)])
def test_linear_many_of_both(torch, name, tokens, rows, cols):
    """As many tiles as the largest kernel is taken for, some of them beyond the matrix."""
    check_linear(torch, tokens, rows, cols, name)


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("tokens,rows,cols", [
    (8, 4100, 4384), (16, 4100, 4384), (9, 100, 8224), (7, 100, 16512), (12, 16400, 4384),
    (3, 32800, 160), (32, 1000, 8224), (20, 4100, 4384), (40, 4200, 4384), (64, 8200, 4384),
    (63, 8200, 96), (100, 16400, 1120), (200, 8100, 1120), (200, 8100, 4384), (250, 8200, 4384),
    (2040, 4090, 1120), (8190, 100, 4384), (1870, 300, 1120), (1700, 3, 64)])
def test_linear_every_kernel(torch, name, tokens, rows, cols):
    """Rows enough for each number of them to a workgroup, columns that leave units of a wave
    whole, in part and empty."""
    check_linear(torch, tokens, rows, cols, name)


def test_linear_extremes(torch):
    """Weights at the ends of their exponents."""
    for name, bytes_ in (("bf16", (2, 30, 127, 200)), ("f16", (104, 127, 136))):
        for byte in bytes_:
            dt = dtype_of(torch, name)
            most = 100 if name == "bf16" else 10  # (a power at which the type holds x)
            x = (torch.randn((3, 64)) * 2.0 ** min(most, max(-most, 127 - byte)) * 2.0 ** -4).to(dt)
            check_linear(torch, 3, 20, 64, name, x=x,
                         scales=torch.full((20, 2), byte, dtype=torch.uint8))


@pytest.mark.parametrize("tokens", [3, 40, 200])
def test_linear_values_that_are_not_finite(torch, tokens):
    """NaN in a block of W reaches its row of the matrix in every token; in x its token;
    columns beyond the matrix, where a block of a tile ends, do not reach anything."""
    rows, cols = 100, 96
    codes, scales = fp4.pack(torch.randn((rows, cols), device="cuda", dtype=torch.bfloat16))
    big = torch.full((tokens, 256), math.nan, device="cuda", dtype=torch.bfloat16)
    big[:, :cols] = torch.randn((tokens, cols))
    x = big[:, :cols]
    clean = fp4.linear(x, fp4.Weights(codes, scales))
    assert torch.isfinite(clean).all()
    assert torch.equal(clean, fp4.linear(x.contiguous(), fp4.Weights(codes, scales)))
    bad = scales.clone()
    bad[17, 1] = 255
    got = fp4.linear(x, fp4.Weights(codes, bad))
    assert torch.isnan(got[:, 17]).all()
    got[:, 17] = clean[:, 17]
    assert torch.equal(got, clean)
    x[1, 40] = math.inf
    got = fp4.linear(x, fp4.Weights(codes, scales))
    assert not torch.isfinite(got[1]).any()
    got[1] = clean[1]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("tokens", [3, 40, 200])
@pytest.mark.parametrize("cols", [96, 160, 1120])
def test_linear_infinite_weights(torch, name, tokens, cols):
    """A scale that the 16-bit type has not makes a weight infinite, and its products with
    positive values, in whichever block: infinite, not NaN."""
    dt = dtype_of(torch, name)
    codes, scales = fp4.pack(torch.randn((50, cols), device="cuda").to(dt))
    x = (torch.rand((tokens, cols), device="cuda") + 0.5).to(dt)
    clean = fp4.linear(x, fp4.Weights(codes, scales))
    blocks = cols // 32
    for row, block in ((0, 0), (17, blocks // 2), (49, blocks - 1)):
        codes[row, block * 16:block * 16 + 16] = 0x77  # all 6
        scales[row, block] = 254
        clean[:, row] = math.inf
    assert torch.equal(fp4.linear(x, fp4.Weights(codes, scales)), clean)


def test_linear_strided_tensors(torch):
    x = torch.randn((70, 300), device="cuda", dtype=torch.float16)[:, 8:264]
    x = torch.empty((70, 304), device="cuda", dtype=torch.float16)[:, 8:264].copy_(x)
    codes, scales = fp4.pack(torch.randn((50, 512), device="cuda", dtype=torch.float16))
    w = fp4.Weights(codes[:, 64:192], scales[:, 4:12])
    v = fp4.Weights(codes[:, 64:192].contiguous(), scales[:, 4:12].contiguous())
    for t in (70, 60, 30, 9, 1):
        want = fp4.linear(x[:t].contiguous(), v)
        assert torch.equal(fp4.linear(x[:t], w), want)
        wide = torch.full((t, 61), 3.0, device="cuda", dtype=torch.float16)
        assert fp4.linear(x[:t], w, out=wide[:, 3:53]).data_ptr() == wide[:, 3:53].data_ptr()
        assert torch.equal(wide[:, 3:53], want)
        assert bool((wide[:, :3] == 3).all()) and bool((wide[:, 53:] == 3).all())
    assert fp4.linear(x[:0], w).shape == (0, 50)


# ------------------------------------------------------------------ together


def test_a_layer(torch):
    """Products, append, attention and products, as a layer has them, against the formulas
    from each step's own inputs."""
    b = Batch(50, [1, 20, 3], [100, 41, 3], 8, 2, 64)
    g = torch.Generator().manual_seed(1)
    hidden = 160

    def matrix(rows, cols):
        c, e = fp4.pack((torch.randn((rows, cols), generator=g) * cols ** -0.5).bfloat16().cuda())
        return fp4.Weights(c, e), stand_for(torch, c, e)

    wqkv, mqkv = matrix(12 * 64, hidden)
    wout, mout = matrix(hidden, 8 * 64)
    cache, _ = cache_of(torch, b, 9)
    x = torch.randn((b.T, hidden), generator=g).bfloat16().cuda()
    a = torch.rand((int(b.positions().max()) + 1, 32), generator=g) * 6.3
    s = b.step()
    qkv = fp4.linear(x, wqkv).view(b.T, 12, 64)
    q = s.append_fp4(qkv, cache, a.cos().cuda(), a.sin().cuda())
    o = s.attention_fp4(q, cache)
    y = fp4.linear(o.flatten(1), wout)

    def tolerance(t, m):
        t = t.double().cpu()
        return 1.01 * ROUND["bf16"] * (t @ m.T).abs() + 60 * 2.0 ** -23 * (t.abs() @ m.T.abs())

    near(qkv.flatten(1), x.double().cpu() @ mqkv.T, tolerance(x, mqkv), "qkv")
    want, tol = append_reference(torch, b, qkv, a.cos(), a.sin(), None, None, 0, False)
    near(q, want[:, :8], tol[:, :8] + 1.01 * ROUND["bf16"] * want[:, :8].abs(), "q")
    k, v = cache.values(torch.bfloat16)
    want, _, tol, _ = reference(torch, b, q, k, v, 64 ** -0.5, ROUND["bf16"])
    near(o, want, tol, "o")
    near(y, o.flatten(1).double().cpu() @ mout.T, tolerance(o.flatten(1), mout), "y")


def test_other_streams_and_graphs(torch):
    b = Batch(15, [1, 1, 50], [2000, 17, 400], 8, 2, 64)
    cache, _ = cache_of(torch, b, 5, poison=False)
    s = b.step()
    codes, scales = fp4.pack(torch.randn((12 * 64, 96), device="cuda").half())
    w = fp4.Weights(codes, scales)
    x = torch.randn((b.T, 96), device="cuda").half()
    cos, sin = torch.rand((2, 2100, 32), device="cuda")

    def body(x, cache, out=None, **kw):
        qkv = fp4.linear(x, w, **kw).view(b.T, 12, 64)
        q = s.append_fp4(qkv, cache, cos, sin, **kw)
        return s.attention_fp4(q, cache, out=out, **kw)

    one = fp4.Cache(*(t.clone() for t in cache))
    want = body(x, one)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    two = fp4.Cache(*(t.clone() for t in cache))
    side.wait_stream(torch.cuda.current_stream())
    got = body(x, two, stream=side)
    with torch.cuda.stream(side):
        again = body(x, two)
        third = fp4.Weights(codes, scales, stream=side)
        y = fp4.linear(x, third)
        back = fp4.values(*fp4.pack(x), torch.float16)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want) and torch.equal(again, want)
    assert torch.equal(y, fp4.linear(x, w))
    assert torch.equal(back, fp4.values(*fp4.pack(x), torch.float16))
    assert all(torch.equal(t, u) for t, u in zip(one, two))
    # a graph replayed on new contents of its inputs, with other work in between
    xg, out = torch.empty_like(x), torch.empty((b.T, 8, 64), device="cuda", dtype=torch.float16)
    kg = fp4.Cache(*(t.clone() for t in cache))
    xg.normal_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        body(xg, kg, out)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        body(xg, kg, out)
        vals = kg.values(torch.float16)
    for i in range(4):
        xg.normal_()
        graph.replay()
        torch.cuda.synchronize()
        ke = fp4.Cache(*(t.clone() for t in cache))
        assert torch.equal(out, body(xg, ke)), i
        assert all(torch.equal(t, u) for t, u in zip(ke, kg))
        assert all(torch.equal(t, u) for t, u in zip(vals, ke.values(torch.float16)))
        torch.cuda.synchronize()


def test_a_step_and_weights_of_two_graphs_and_both_kinds_of_cache(torch):
    """Calls of both kinds in turn share a step's workspace, and so do two graphs' replays;
    two threads share weights."""
    from concurrent.futures import ThreadPoolExecutor

    b = Batch(23, [1, 1, 70], [5000, 17, 900], 8, 2, 128)
    caches = [cache_of(torch, b, seed, poison=False)[0] for seed in (4, 5)]
    qs = [torch.randn((b.T, 8, 128), device="cuda").bfloat16() for _ in range(2)]
    wide = caches[0].values(torch.bfloat16)
    w = fp4.Weights(*fp4.pack(torch.randn((96, 1024), device="cuda").bfloat16()))
    torch.cuda.synchronize()
    want = [b.step().attention_fp4(q, c) for q, c in zip(qs, caches)]
    want_wide = b.step().attention(qs[1], *wide)
    want_y = [fp4.linear(o.flatten(1), w) for o in want]
    s = b.step()
    for _ in range(3):
        assert torch.equal(s.attention_fp4(qs[0], caches[0]), want[0])
        assert torch.equal(s.attention(qs[1], *wide), want_wide)
        assert torch.equal(s.attention_fp4(qs[1], caches[1]), want[1])
    torch.cuda.synchronize()
    graphs, outs = [], []
    for q, c in zip(qs, caches):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            o = s.attention_fp4(q, c)
            outs.append((o, fp4.linear(o.flatten(1), w)))
        graphs.append(graph)
    for i in (0, 1, 1, 0, 1, 0, 0):
        for t in outs[i]:
            t.zero_()
        graphs[i].replay()
        assert torch.equal(s.attention(qs[1], *wide), want_wide)
        torch.cuda.synchronize()
        assert torch.equal(outs[i][0], want[i]) and torch.equal(outs[i][1], want_y[i])

    def calls(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            got = [fp4.linear(want[i].flatten(1), w) for _ in range(50)]
            torch.cuda.current_stream().synchronize()
        return all(torch.equal(y, want_y[i]) for y in got)

    with ThreadPoolExecutor(2) as pool:
        assert all(pool.map(calls, (0, 1)))


def test_tensors_dropped_while_another_stream_uses_them(torch):
    """Memory of a call's tensors is not reused before the call on its stream is done."""
    b = Batch(41, [1, 40], [300, 90], 4, 2, 64)
    cache, _ = cache_of(torch, b, 9, poison=False)
    s = b.step()
    qkv = torch.randn((b.T, 8, 64), device="cuda", dtype=torch.bfloat16)
    codes, scales = fp4.pack(torch.randn((64, 512), device="cuda", dtype=torch.bfloat16))
    one = fp4.Cache(*(t.clone() for t in cache))
    want_q = s.append_fp4(qkv, one)
    want = s.attention_fp4(want_q, one)
    want_y = fp4.linear(qkv.flatten(1), fp4.Weights(codes, scales))
    want_c, want_s = fp4.pack(qkv)
    a = torch.randn((8192, 8192), device="cuda", dtype=torch.bfloat16)
    a @ a
    side = torch.cuda.Stream()

    def dropped(call, tensors):
        """The call's result on the busy stream; the tensors' memory asked for again."""
        torch.cuda.synchronize()
        tensors = [t.clone() for t in tensors]
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            for _ in range(250):
                torch.mm(a, a)
        out = call(*tensors)
        places = {t.data_ptr() for t in tensors}
        sizes = [t.numel() * t.element_size() for t in tensors]
        del tensors
        again = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes]
        assert not places & {t.data_ptr() for t in again}
        side.synchronize()
        return out

    got = dropped(lambda q, *c: s.append_fp4(q, fp4.Cache(*c), stream=side), [qkv, *cache])
    assert torch.equal(got, want_q)
    got = dropped(lambda q, *c: s.attention_fp4(q, fp4.Cache(*c), stream=side), [want_q, *one])
    assert torch.equal(got, want)
    # the weights are laid out on the busy stream and dropped
    got = dropped(lambda x, c, e: fp4.linear(x, fp4.Weights(c, e, stream=side), stream=side),
                  [qkv.flatten(1), codes, scales])
    assert torch.equal(got, want_y)
    got = dropped(lambda x: fp4.pack(x, stream=side), [qkv])
    assert torch.equal(got[0], want_c) and torch.equal(got[1], want_s)
    got = dropped(lambda c, e: fp4.values(c, e, torch.bfloat16, stream=side), [want_c, want_s])
    assert torch.equal(got, fp4.values(want_c, want_s, torch.bfloat16))


def test_weights_under_way(torch):
    """While weights wait to be laid out behind the device's work, products on other streams
    wait for it, and a capture, whose replays would not, is refused."""
    x = torch.randn((5, 512), device="cuda", dtype=torch.bfloat16)
    codes, scales = fp4.pack(torch.randn((64, 512), device="cuda", dtype=torch.bfloat16))
    want = fp4.linear(x, fp4.Weights(codes, scales))
    a = torch.randn((8192, 8192), device="cuda", dtype=torch.bfloat16)
    a @ a
    other, side = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(250):
        a @ a
    w = fp4.Weights(codes, scales)
    with torch.cuda.stream(other):
        y = fp4.linear(x, w)
    z = fp4.linear(x, w, stream=side)
    graph = torch.cuda.CUDAGraph()
    out = torch.empty_like(want)
    with torch.cuda.stream(other):
        graph.capture_begin()
        out.zero_()
        refused = False
        try:
            fp4.linear(x, w, out=out)
        except ValueError:
            refused = True
        graph.capture_end()
    late = w._laid.query()
    torch.cuda.synchronize()
    assert refused and not late
    assert torch.equal(y, want) and torch.equal(z, want) and torch.equal(fp4.linear(x, w), want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fp4.linear(x, w, out=out)
        with pytest.raises(ValueError):
            fp4.Weights(codes, scales)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_weights_of_another_stream_on_the_default_one(torch):
    """Products on the default stream wait for a layout under way on another, and its memory is
    not given away there before they are done."""
    x = torch.randn((5, 512), device="cuda", dtype=torch.bfloat16)
    codes, scales = fp4.pack(torch.randn((640, 512), device="cuda", dtype=torch.bfloat16))
    want = fp4.linear(x, fp4.Weights(codes, scales))
    a = torch.randn((8192, 8192), device="cuda", dtype=torch.bfloat16)
    side = torch.cuda.Stream()
    for s in (side, torch.cuda.current_stream()):
        with torch.cuda.stream(s):
            a @ a
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(250):
            torch.mm(a, a)
    w = fp4.Weights(codes, scales, stream=side)
    y, z = fp4.linear(x, w), fp4.linear(x, w, stream=torch.cuda.default_stream())
    assert not w._laid.query()
    torch.cuda.synchronize()
    assert torch.equal(y, want) and torch.equal(z, want)
    w = fp4.Weights(codes, scales, stream=side)
    torch.cuda.synchronize()
    for _ in range(250):
        torch.mm(a, a)
    y = fp4.linear(x, w)
    at, n = w._data.data_ptr(), w._data.numel()
    del w
    with torch.cuda.stream(side):
        again = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    assert again.data_ptr() != at
    torch.cuda.synchronize()
    assert torch.equal(y, want)


# ------------------------------------------------------------------ refusals


def einval(call, *args, **kw):
    with pytest.raises(tas.TasError) as e:
        call(*args, **kw)
    assert e.value.code == tas.TAS_EINVAL


def test_refused_step_arguments(torch):
    b = Batch(30, [1, 4], [30, 20], 4, 2, 64)
    cache, _ = cache_of(torch, b, 9, poison=False)
    s = b.step()
    q = torch.zeros((5, 4, 64), device="cuda", dtype=torch.bfloat16)
    qkv = torch.zeros((5, 8, 64), device="cuda", dtype=torch.bfloat16)
    cos = torch.zeros((30, 32), device="cuda")
    s.attention_fp4(q, cache)
    s.append_fp4(qkv, cache, cos, cos)
    for i, t in enumerate(cache):
        for bad in (t[1:], t.char(), t.cpu(), t.transpose(2, 3), t[:, :1], t[..., ::2], t[0]):
            c = fp4.Cache(*(bad if j == i else u for j, u in enumerate(cache)))
            with pytest.raises(ValueError):
                s.attention_fp4(q, c)
            with pytest.raises(ValueError):
                s.append_fp4(qkv, c)
    for bad in (q.float(), q[:4], q[:, :3], q.cpu()):
        with pytest.raises(ValueError):
            s.attention_fp4(bad, cache)
    for scale in (0.0, -1.0, math.inf, math.nan, 3e38):
        einval(s.attention_fp4, q, cache, scale=scale)
    einval(s.append_fp4, qkv, cache, cos[:29], cos[:29])
    for eps in (-1.0, math.nan, math.inf):
        einval(s.append_fp4, qkv, cache, eps=eps)
    # codes off the 16 bytes, scales off their row
    room = torch.zeros(cache.k.numel() + 64, device="cuda", dtype=torch.uint8)
    odd = cache._replace(k=room[8:8 + cache.k.numel()].view_as(cache.k))
    einval(s.attention_fp4, q, odd)
    odd = cache._replace(v_scale=room[1:1 + cache.v_scale.numel()].view_as(cache.v_scale))
    einval(s.attention_fp4, q, odd)
    # slots that share memory can be attended to, not appended to
    shared = (cache._replace(k=cache.k[:1].expand_as(cache.k)),
              cache._replace(v_scale=cache.v_scale[:, :1].expand_as(cache.v_scale)),
              cache._replace(v=cache.k), cache._replace(k_scale=cache.v_scale),
              cache._replace(k_scale=cache.k.flatten()[:cache.k_scale.numel()].view_as(cache.k_scale)))
    before = [t.clone() for t in cache]
    for c in shared:
        s.attention_fp4(q, c)
        einval(s.append_fp4, qkv, c)
    # outputs over other rows, the cache, the inputs
    buf = torch.zeros((6, 16, 64), device="cuda", dtype=torch.bfloat16)
    x = buf[:5, :8]
    for out in (x[:, 1:5], x[:, 4:8], buf[1:, :4], buf[:5, 6:10],
                cache.v.view(torch.bfloat16).flatten()[:1280].view(5, 4, 64)):
        einval(s.append_fp4, x, cache, out=out)
    x = buf[:5, :4]
    for out in (buf[1:, :4], buf[:5, 1:5],
                cache.k.view(torch.bfloat16).flatten()[:1280].view(5, 4, 64)):
        einval(s.attention_fp4, x, cache, out=out)
    out = torch.empty_like(q)
    for lse in (q.view(torch.float32).flatten()[:20].view(5, 4),
                out.view(torch.float32).flatten()[:20].view(5, 4),
                cache.v_scale.flatten()[:80].view(torch.float32).view(5, 4)):
        einval(s.attention_fp4, q, cache, out=out, lse=lse)
    w = torch.ones(64, device="cuda", dtype=torch.bfloat16)
    einval(s.append_fp4, qkv, cache, q_weight=out.flatten()[:64], k_weight=w, out=out)
    einval(s.append_fp4, qkv, cache, out.view(torch.float32).flatten()[:30 * 8].view(30, 8),
           cos[:, :8].contiguous(), out=out)
    assert all(torch.equal(t, u) for t, u in zip(cache, before))
    s.close()
    with pytest.raises(ValueError):
        s.attention_fp4(q, cache)


def test_refused_tensors(torch):
    x = torch.randn((6, 64), device="cuda", dtype=torch.bfloat16)
    codes, scales = fp4.pack(x)
    for bad in (x.float(), x.cpu(), x[:, :48], x[:, ::2], x[:, :0], x.T,
                torch.zeros((1, 1, 1, 1, 32), device="cuda", dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            fp4.pack(bad)
    odd = torch.zeros((6, 72), device="cuda", dtype=torch.bfloat16)
    einval(fp4.pack, odd[:, 4:68])      # 8-byte aligned
    einval(fp4.pack, torch.zeros((6, 68), device="cuda", dtype=torch.bfloat16)[:, :64])
    for c, e in ((codes, scales[:, :1]), (codes[:5], scales), (codes.char(), scales),
                 (codes, scales.cpu()), (codes[:, ::2], scales), (codes[:, :24], scales)):
        with pytest.raises(ValueError):
            fp4.values(c, e, torch.bfloat16)
        with pytest.raises(ValueError):
            fp4.Weights(c, e)
    with pytest.raises(ValueError):
        fp4.values(codes, scales, torch.float32)
    with pytest.raises(ValueError):
        fp4.Weights(codes[:0], scales[:0])
    w = fp4.Weights(codes, scales)
    for bad in (x.float(), x.cpu(), x[:, :32], x[0], x.T, odd[:, ::2]):
        with pytest.raises(ValueError):
            fp4.linear(bad, w)
    y = torch.zeros((6, 6), device="cuda", dtype=torch.bfloat16)
    for bad in (y.half(), y[:5], y[:, :5], y.T, y.cpu()):
        if bad is y.T or bad.is_contiguous() and bad.shape == y.shape and bad.dtype == y.dtype \
                and bad.is_cuda:
            continue
        with pytest.raises(ValueError):
            fp4.linear(x, w, out=bad)
    einval(fp4.linear, odd[:, 4:68], w)
    einval(fp4.linear, x, w, out=x.flatten()[:36].view(6, 6))
    einval(fp4.linear, x, w, out=w._data[256:256 + 72].view(torch.bfloat16).view(6, 6))


def test_a_backward_pass_is_refused(torch):
    b = Batch(38, [1, 20], [30, 40], 4, 2, 64)
    cache, _ = cache_of(torch, b, 9)
    s = b.step()

    def grad(t):
        return t.detach().clone().requires_grad_()

    q = torch.randn((21, 4, 64), device="cuda", dtype=torch.bfloat16)
    qkv = torch.randn((21, 8, 64), device="cuda", dtype=torch.bfloat16)
    w = fp4.Weights(*fp4.pack(torch.randn((6, 64), device="cuda", dtype=torch.bfloat16)))
    x = qkv[:, 0].contiguous()
    for call, arg in ((lambda t: s.attention_fp4(t, cache), q),
                      (lambda t: s.append_fp4(t, cache), qkv), (lambda t: fp4.linear(t, w), x)):
        want = call(arg)
        assert not want.requires_grad
        out = call(grad(arg))
        assert out.requires_grad and torch.equal(out, want)
        with pytest.raises(NotImplementedError):
            out.float().sum().backward()
        with torch.no_grad():
            assert not call(grad(arg)).requires_grad
    with pytest.raises(NotImplementedError):
        fp4.pack(grad(x))
    with torch.no_grad():
        fp4.pack(grad(x))


def test_forward_mode_is_refused(torch):
    """A dual tensor, whose tangent the result would not have, in every place of every call;
    nothing is written then. Within a level, tensors without a tangent go on as ever."""
    import torch.autograd.forward_ad as fwd

    b = Batch(38, [1, 20], [30, 40], 4, 2, 64)
    cache, _ = cache_of(torch, b, 9, poison=False)
    wide = cache.values(torch.bfloat16)
    s = b.step()
    qkv = torch.randn((21, 8, 64), device="cuda", dtype=torch.bfloat16)
    q, out = qkv[:, :4].contiguous(), torch.zeros((21, 4, 64), device="cuda", dtype=torch.bfloat16)
    cos, sin = torch.rand((2, 60, 32), device="cuda")
    w = torch.ones(64, device="cuda", dtype=torch.bfloat16)
    lse = torch.zeros((21, 4), device="cuda")
    m = fp4.Weights(*fp4.pack(torch.randn((6, 64), device="cuda", dtype=torch.bfloat16)))
    y = torch.zeros((21, 6), device="cuda", dtype=torch.bfloat16)
    norm = lambda c, n, qw, kw, o: dict(cos=c, sin=n, q_weight=qw, k_weight=kw, out=o)
    calls = [(lambda t, *a: s.append_fp4(t, cache, **norm(*a)), [qkv, cos, sin, w, w, out]),
             (lambda t, k, v, *a: s.append(t, k, v, **norm(*a)), [qkv, *wide, cos, sin, w, w, out]),
             (lambda t, o, l: s.attention_fp4(t, cache, out=o, lse=l), [q, out, lse]),
             (lambda t, k, v, o, l: s.attention(t, k, v, out=o, lse=l), [q, *wide, out, lse]),
             (lambda t, o: fp4.linear(t, m, out=o), [q[:, 0], y]), (fp4.pack, [qkv])]
    written = [*cache, *wide, out, lse, y]
    before = [t.clone() for t in written]
    for call, args in calls:
        with fwd.dual_level():
            for i, t in enumerate(args):
                dual = fwd.make_dual(t, torch.ones_like(t))
                with pytest.raises(NotImplementedError):
                    call(*args[:i], dual, *args[i + 1:])
                with torch.no_grad(), pytest.raises(NotImplementedError):
                    call(*args[:i], dual, *args[i + 1:])
    torch.cuda.synchronize()
    assert all(torch.equal(t, u) for t, u in zip(written, before))
    for call, args in calls:
        def run():
            got = call(*args)
            return [t.clone() for t in (got if isinstance(got, tuple) else (got,))]

        want = run()
        with fwd.dual_level():
            got = run()
        assert all(torch.equal(t, u) for t, u in zip(got, want))
    with pytest.raises((NotImplementedError, RuntimeError)):
        torch.func.jvp(lambda t: fp4.linear(t, m), (q[:, 0],), (q[:, 0],))


# ------------------------------------------------------------------ the command


@pytest.mark.parametrize("prefix", [0, 100])
def test_measure_in_four_bits(torch, prefix):
    """Iterations over caches in four bits, with the products of the weights."""
    from paper_2606_18431_amd import iteration_cost as C
    from paper_2606_18431_amd import workloads as W

    w = W.make(1, n_traces=1, n_settings=4, n_req=200)
    rows = C.measure(w, iterations=4, layers=2, heads=8, kv_heads=2, head_dim=64, dtype="f16",
                     prefix=prefix, cache_bits=4, hidden=256)
    assert len(rows) == 4
    for n, tokens, context, us in rows:
        assert n >= 1 and tokens >= n and context >= tokens and 0 < us < 1e6


def test_layers_run_the_operators_in_order(torch):
    """A layer's run: heads' product, append, attention, and three products from its result."""
    from paper_2606_18431_amd import iteration_cost as C
    from paper_2606_18431_amd import workloads as W

    e = W.Engine(kv_blocks=16, max_tokens=64)
    m = C.Layers(e, 1, heads=4, kv_heads=2, head_dim=64, dtype=torch.bfloat16, device="cuda",
                 positions=100, cache_bits=4, hidden=128, ffn=160)
    assert [(w.rows, w.cols) for w in m.weights[0]] == [(512, 128), (128, 256), (160, 128), (128, 160)]
    s = step.Step([1, 3], [40, 3], [[3, 1, 4], [0, 0, 0]], heads=4, kv_heads=2, head_dim=64,
                  block_tokens=e.block_tokens, n_blocks=16)
    qkv = fp4.linear(m.x[:4], m.weights[0][0]).view(4, 8, 64)
    cache = fp4.Cache(*(t.clone() for t in m.caches[0]))
    q = s.append_fp4(qkv, cache, m.cos, m.sin, q_weight=m.weight, k_weight=m.weight)
    m.run(s)
    assert all(torch.equal(t, u) for t, u in zip(cache, m.caches[0]))
    assert torch.isfinite(s.attention_fp4(q, cache)).all()
