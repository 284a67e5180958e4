"""A code of NaN in V (the writer makes none; a page may come from elsewhere) is the NaN of its element: the rows that see the token have it in
that column, wherever the token lies among the kernels' tiles, and nothing else changes by a bit."""
import numpy as np
import pytest
import torch

import codes_bounds as B
import test_gpu_kv_attention_codes as base
from paper_2608_25431_b200 import binding

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    c = binding.Ctx(64)
    yield c
    c.close()


def spoil(x, r, t, head, columns, codes=(0x7F, 0xFF)):
    heads, dim = x["heads"], x["q"].shape[2]
    token = x["pool"][x["table"][r, t // x["pt"]], t % x["pt"]]
    for k, c in enumerate(columns):
        token[heads * dim + head * dim + c] = codes[k % 2]


def expect(ctx, x, places, sees, **near):
    """places: (request, token, K/V head, columns); sees(request, row, token)."""
    want = base.call(ctx, x, **near)
    y = dict(x, pool=x["pool"].copy())
    nan = np.zeros(want[0].shape, bool)
    group = x["q"].shape[1] // x["heads"]
    first = np.concatenate([[0], np.cumsum(x["want"] - x["have"])])
    for r, t, head, columns in places:
        spoil(y, r, t, head, columns)
        for i in range(int(x["want"][r] - x["have"][r])):
            if sees(r, i, t):
                for c in columns:
                    nan[first[r] + i, head * group:(head + 1) * group, c] = True
    got = base.call(ctx, y, **near)
    assert np.array_equal(np.isnan(got[0]), nan)
    assert np.array_equal(got[0][~nan], want[0][~nan]) and all(np.array_equal(a, b) for a, b in zip(got[1:], want[1:]))


@pytest.mark.parametrize("dtype, dim, pt", [(BF, 128, 16), (HF, 64, 24), (BF, 64, 3)])
@pytest.mark.parametrize("group, new", [(1, 1), (1, 3), (2, 7), (1, 30), (4, 50)])
@pytest.mark.parametrize("window", [0, 37])
def test_rows_that_see_it_and_no_others(ctx, dtype, dim, pt, group, new, window):
    x = B.step(new, dtype, [200, 5, 64], [new, new, 1], 3, group, dim, pt)

    def sees(r, i, t):
        pos = int(x["have"][r]) + i
        return t <= pos and (not window or t > pos - window)

    for t in (0, 100, 163, 164, 170, 190, 199, 200, 200 + new - 1):          # whole tiles, a window's edge, the step's own
        expect(ctx, x, [(0, t, 1, [0, 9, dim - 1])], sees, window=window)
    expect(ctx, x, [(0, 180, 0, [3]), (0, 199, 2, [3, 40]), (1, 2, 1, [dim - 1]), (1, 5, 1, [1]), (2, 64, 2, [7])], sees, window=window)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new", [3, 14, 30, 60])
def test_trees(ctx, dim, new):
    x = B.step(new, HF, [70, 33], [new, new], 2, 2, dim, 16, tree=True)
    first = [0, new]

    def sees(r, i, t):
        j = t - int(x["have"][r])
        return j < 0 or bool(int(x["mask"][first[r] + i, j // 32]) >> (j % 32) & 1)

    for j in range(-2, new, 5):
        expect(ctx, x, [(0, 70 + j, 1, [0, 31, 32, dim - 1]), (1, 33 + j, 0, [5])], sees)


@pytest.mark.parametrize("new", [1, 3, 30])
def test_pieces_that_are_joined(ctx, new):
    """One request over many CTAs: the token lies in one piece of its rows."""
    x = B.step(7, BF, [9000], [new], 1, 4, 128, 16)
    for t in (10, 4567, 8990, 9000):
        expect(ctx, x, [(0, t, 0, [77])], lambda r, i, t: t <= 9000 + i)


def test_calls_behind_one_with_nan(ctx):
    """Nothing of it stays for the next piece or call: many items to a CTA."""
    rng = np.random.default_rng(0)
    for new in (1, 12, 40):
        have = rng.integers(3, 90, 40)
        x = B.step(new, HF, have, [new] * 40, 8, 1, 64, 16)
        expect(ctx, x, [(r, int(have[r]), r % 8, [r]) for r in range(0, 40, 3)], lambda r, i, t: t <= int(have[r]) + i)
