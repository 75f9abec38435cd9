"""The host's test for tensors that share memory, compiled by itself and compared with
the places counted out (no GPU)."""
import itertools
import os
import random
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

MAIN = r"""
#include <stdio.h>
#include <chrono>
#include "tas_step_overlap.h"
using namespace tas_step_impl;
static bool get(Region &r) {
    long long v[8];
    for (long long &x : v)
        if (scanf("%lld", &x) != 1) return false;
    r = {v[0], v[1], {v[2], v[3], v[4]}, {v[5], v[6], v[7]}};
    return true;
}
int main() {
    Region a, b;
    while (get(a) && get(b)) {
        const auto t = std::chrono::steady_clock::now();
        const int x = Overlap()(a, b), y = Overlap()(b, a);
        const std::chrono::duration<double, std::micro> us = std::chrono::steady_clock::now() - t;
        printf("%d %d %g\n", x, y, us.count() / 2);
    }
}
"""


@pytest.fixture(scope="module")
def overlap(tmp_path_factory):
    """Answers for pairs of (base, row, strides, sizes), and the microseconds of one."""
    d = tmp_path_factory.mktemp("overlap")
    src, exe = d / "overlap.cpp", d / "overlap"
    src.write_text(MAIN)
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-Wall", "-Werror",
                           "-fsanitize=undefined", "-fno-sanitize-recover", "-I",
                           os.path.join(ROOT, "paper_2606_18431_amd", "csrc"), "-o", str(exe),
                           str(src)])

    def ask(pairs):
        flat = [[r[0], r[1], *r[2], *r[3]] for p in pairs for r in p]
        text = "\n".join(" ".join(map(str, x)) for x in flat)
        out = subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True)
        rows = [line.split() for line in out.stdout.splitlines()]
        assert len(rows) == len(pairs)
        return [(int(x), int(y), float(us)) for x, y, us in rows]

    return ask


def places(r):
    base, row, stride, n = r
    at = [np.arange(m) * s for s, m in zip(stride, n)]
    first = base + at[0][:, None, None] + at[1][:, None] + at[2]
    return set((first[..., None] + np.arange(row)).ravel().tolist())


def test_small_regions_counted_out(overlap):
    rng = random.Random(3)
    pairs = []
    for _ in range(6000):
        def region(like=None):
            stride = [rng.choice([0, 1, 2, 3, 4, 6, 8, 12, 16, 24, 40, 64]) for _ in range(3)]
            if like and rng.random() < 0.7:
                stride = list(like[2])
            n = [rng.choice([0, 1, 2, 3, 5]) if rng.random() < 0.1 else rng.choice([1, 2, 3, 4])
                 for _ in range(3)]
            return rng.randrange(60), rng.choice([1, 2, 3, 4, 8]), stride, n

        a = region()
        pairs.append((a, region(a)))
    want = [bool(places(a) & places(b)) for a, b in pairs]
    assert 1000 < sum(want) < 5000
    for p, w, (x, y, _) in zip(pairs, want, overlap(pairs)):
        assert x == y == w, p


def cache(base, n_blocks, heads, tokens, row, order, block=None):
    """A cache of this order of its axes in memory, from the longest stride on."""
    size = dict(b=n_blocks, h=heads, t=tokens)
    stride, span = {}, row
    for axis in reversed(order):
        stride[axis] = block if axis == "b" and block else span
        span *= size[axis]
    return base, row, [stride[x] for x in "bht"], [size[x] for x in "bht"]


def test_caches(overlap):
    """Full sizes: apart, beside each other in a block or a token, a block further on."""
    N, H, T, D = 1 << 17, 8, 16, 16
    block = H * T * D
    shapes = ["bht", "bth", "hbt", "htb", "tbh", "thb"]
    pairs, want = [], []
    for x, y in itertools.product(shapes, shapes):
        a = cache(1000, N, H, T, D, x)
        for base, answer in ((1000 + N * block, 0), (1000, 1), (1000 + N * block - 1, 1),
                             (1000 + 3 * block // 2, None)):
            pairs.append((a, cache(base, N, H, T, D, y)))
            want.append(answer)
    for x, y in itertools.product(["bht", "bth"], repeat=2):
        # K and V in the halves of a block of both; then V's begins inside K's half
        for base, answer in ((block, 0), (block - 1, 1), (2 * block, 1)):
            pairs.append((cache(0, N, H, T, D, x, 2 * block),
                          cache(base, N, H, T, D, y, 2 * block)))
            want.append(answer)
    # K and V in the halves of a token's row
    a = (0, D, [2 * block, 2 * T * D, 2 * D], [N, H, T])
    for base, answer in ((D, 0), (D - 1, 1), (D + 1, 1), (2 * block, 1), (2 * block + D, 0)):
        pairs.append((a, (base, *a[1:])))
        want.append(answer)
    # one pool, a block further on
    a = cache(0, N, H, T, D, "bht")
    pairs.append((a, (block, *a[1:])))
    want.append(1)
    # rows of one buffer: queries, keys and values, then the output, or over them
    qkv = (0, 12 * D, [28 * D, 0, 0], [4000, 1, 1])
    for base, answer in ((12 * D, 0), (20 * D, 0), (11 * D, 1), (21 * D, 1), (28 * D - 1, 1)):
        pairs.append((qkv, (base, 8 * D, [28 * D, 0, 0], [4000, 1, 1])))
        want.append(answer)
    for p, w, (x, y, us) in zip(pairs, want, overlap(pairs)):
        assert x == y and (w is None or x == w), (p, w)
        assert us < 20000, (p, us)
