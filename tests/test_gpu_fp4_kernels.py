"""Every kernel of the products with weights in four bits, at sizes that select it: against the
formula in 64 bits, and what lies beside the matrix and the tokens, values that are not finite,
rows apart."""
import math

import pytest

from paper_2606_18431_amd import fp4, step
from test_fp4 import KERNEL_SHAPES
from test_gpu_fp4 import check_linear
from test_gpu_step import dtype_of

pytestmark = pytest.mark.gpu

SHAPES = [(k, *shape) for k, shapes in KERNEL_SHAPES.items() for shape in shapes]
# whose columns end inside a tile of 128: the fewest and the most of each kernel's
RAGGED = [(k, *shape) for k, shapes in KERNEL_SHAPES.items() for ragged in
          [sorted((s for s in shapes if s[2] % 128), key=lambda s: s[2])]
          for shape in dict.fromkeys((ragged[0], ragged[-1]))]


@pytest.fixture(scope="module")
def torch():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def selects(kernel, *shape):
    assert step.lib().tas_fp4_linear_kernel(*shape) == kernel
    print(f"[gpu] kernel {kernel}: {shape}", flush=True)


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("kernel,tokens,rows,cols", SHAPES)
def test_products(torch, kernel, tokens, rows, cols, name):
    selects(kernel, tokens, rows, cols)
    check_linear(torch, tokens, rows, cols, name)


def operands(torch, name, tokens, rows, cols):
    """Tokens of 1/2 to 3/2 in the columns of wider rows, NaN beside them; codes and scales."""
    dt = dtype_of(torch, name)
    g = torch.Generator(device="cuda").manual_seed(tokens + rows + cols)
    big = torch.full((tokens, cols + 104), math.nan, device="cuda", dtype=dt)
    big[:, 8:8 + cols] = torch.rand((tokens, cols), generator=g, device="cuda") + 0.5
    codes = torch.randint(0, 256, (rows, cols // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.randint(118, 124, (rows, cols // 32), generator=g, device="cuda",
                           dtype=torch.uint8)
    return big[:, 8:8 + cols], codes, scales


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("kernel,tokens,rows,cols", RAGGED)
def test_rows_apart(torch, kernel, tokens, rows, cols, name):
    """Tokens and results as columns of wider tensors, of any alignment; what lies beside them
    is not read and not written."""
    selects(kernel, tokens, rows, cols)
    x, codes, scales = operands(torch, name, tokens, rows, cols)
    w = fp4.Weights(codes, scales)
    want = fp4.linear(x.contiguous(), w)
    assert torch.isfinite(want).all()
    assert torch.equal(fp4.linear(x, w), want)
    for before, after in ((3, 5), (4, 8 - rows % 4)):  # (in fours or not)
        wide = torch.full((tokens, before + rows + after), 7.0, device="cuda", dtype=x.dtype)
        out = wide[:, before:before + rows]
        assert fp4.linear(x, w, out=out).data_ptr() == out.data_ptr()
        assert torch.equal(out, want)
        assert bool((wide[:, :before] == 7).all()) and bool((wide[:, before + rows:] == 7).all())


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("kernel,tokens,rows,cols", RAGGED)
def test_values_that_are_not_finite(torch, kernel, tokens, rows, cols, name):
    """A NaN block of W reaches its row of the matrix, an infinite weight makes its row infinite,
    an infinite element its token (by the weights' signs, NaN at a weight of 0): in the first
    block, a middle one and those of the tile that ends beyond the matrix, whose rest is 0 times
    what is read for it."""
    selects(kernel, tokens, rows, cols)
    x, codes, scales = operands(torch, name, tokens, rows, cols)
    clean = fp4.linear(x, fp4.Weights(codes, scales))
    blocks = cols // 32
    some = sorted({0, blocks // 2, blocks // 4 * 4, blocks - 1})
    for i, block in enumerate(some):
        row = (rows - 1, 0, rows // 2, rows // 3)[i]
        bad, at = scales.clone(), codes.clone()
        bad[row, block] = 255
        got = fp4.linear(x, fp4.Weights(codes, bad))
        assert torch.isnan(got[:, row]).all()
        got[:, row] = clean[:, row]
        assert torch.equal(got, clean)
        bad[row, block] = 254
        at[row, block * 16:block * 16 + 16] = 0x77  # all 6
        got = fp4.linear(x, fp4.Weights(at, bad))
        assert bool((got[:, row] == math.inf).all())
        got[:, row] = clean[:, row]
        assert torch.equal(got, clean)
    w = fp4.Weights(codes, scales)
    m = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], device="cuda")
    for i, col in enumerate(sorted({b * 32 for b in some} | {cols - 1})):
        token = (tokens - 1, 0, tokens // 2, tokens // 3, 0)[i]
        y = x.clone(memory_format=torch.contiguous_format)
        y[token, col] = math.inf
        got = fp4.linear(y, w)
        code = (codes[:, col // 2] >> 4 * (col % 2) & 15).long()
        want = m[code % 8] * (1 - 2 * (code // 8)) * math.inf
        assert bool(((got[token] == want) | (got[token].isnan() & want.isnan())).all())
        got[token] = clean[token]
        assert torch.equal(got, clean)


def test_rows_as_far_apart_as_they_may_be(torch):
    """Strides of 2^24 elements, with which the last of a workgroup's rows lie beyond 4 GB, and
    results 2^31 - 1 and 2^31 - 4 elements apart."""
    big = torch.full((200, 1 << 24), math.nan, device="cuda", dtype=torch.bfloat16)
    for kernel, shapes in KERNEL_SHAPES.items():
        tokens, rows, cols = max(s for s in shapes if s[0] <= 200)
        selects(kernel, tokens, rows, cols)
        x, codes, scales = operands(torch, "bf16", tokens, rows, cols)
        w = fp4.Weights(codes, scales)
        far = big[:tokens, 8:8 + cols].copy_(x)
        assert torch.equal(fp4.linear(far, w), fp4.linear(x, w))
        far.fill_(math.nan)
    del big, far
    x, codes, scales = operands(torch, "bf16", 3, 100, 96)
    w = fp4.Weights(codes, scales)
    for stride in ((1 << 31) - 1, (1 << 31) - 4):
        out = torch.empty_strided((3, 100), (stride, 1), device="cuda", dtype=torch.bfloat16)
        fp4.linear(x, w, out=out)
        assert torch.equal(out, fp4.linear(x, w))
        del out
