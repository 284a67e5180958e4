"""What becomes of a call over 8-bit pages whose waits run out: a short limit (gift_ctx_wait_limit) makes them, and it has to be met.

The waits are those of the kernel for many query rows; it must end with nothing of its own under way, so that the calls behind it are
right."""
import numpy as np
import pytest
import torch

import codes_bounds as B
import test_gpu_kv_attention_codes as base
from oracle import paged as P
from paper_2608_25431_b200 import binding

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16
LIMITS = [1, 200, 500, 1000, 2000, 4000, 8000, 30000]


@pytest.fixture(scope="module")
def ctx():
    c = binding.Ctx(64)
    yield c
    c.close()


# one tile of rows, several (two CTAs to a slice, odd last tiles shared by two heads), small pages, capped and windowed, biased
CASES = [(BF, 128, 4, 20, 16, {}), (HF, 64, 4, 70, 24, {}), (BF, 128, 2, 30, 3, {}), (HF, 128, 4, 100, 16, dict(softcap=2.0, window=300)),
         (BF, 64, 8, 5, 64, dict(sloped=True, window=90))]


def batch(dtype, dim, group, new, pt, near):
    x = B.step(51, dtype, [2500, 0, 700, 33, 64, 1200, 5], [new, 3, 0, new, new, 1, new], 3, group, dim, pt)
    near = dict(near)
    if near.pop("sloped", False):
        near["slopes"] = np.array([2.0 ** -(h % 8 + 1) for h in range(3 * group)], np.float32)
    return x, near


@pytest.mark.parametrize("dtype, dim, group, new, pt, near", CASES)
def test_a_stalled_request_says_so_and_calls_behind_it_are_right(ctx, dtype, dim, group, new, pt, near):
    x, near = batch(dtype, dim, group, new, pt, near)
    rows = x["want"] - x["have"]
    of_row = np.repeat(np.arange(len(rows)), rows)
    ctx.wait_limit(0)
    want = base.call(ctx, x, **near)
    assert not want[3].any()
    seen = set()
    try:
        for ns in LIMITS:
            for _ in range(3):
                ctx.wait_limit(ns)
                out, lse, who, st = base.call(ctx, x, **near)
                assert set(st.tolist()) <= {0, binding.ST_STALLED} and not st[rows == 0].any(), ns
                seen |= set(st[rows > 0].tolist())
                stalled = st[of_row] != 0
                assert not out[stalled].any() and np.isneginf(lse[stalled]).all() and (who[stalled] == P.CONFLICT).all(), ns
                for a, b in zip((out, lse, who), want):
                    assert np.array_equal(a[~stalled], b[~stalled]), ns
                ctx.wait_limit(0)
                for a, b in zip(base.call(ctx, x, **near), want):
                    assert np.array_equal(a, b), ns
    finally:
        ctx.wait_limit(0)
    assert seen == {0, binding.ST_STALLED}
