"""Attention over 8-bit pages where K's scales and the queries are far from one: every kernel multiplies them in an order that stays within 32
bits, as long as q . k is below 2^104.  Bounds: tests/codes_bounds.py."""
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


def far(seed, dtype, new, k_power, q_power, dim=64, tokens=None):
    """A step whose K scales (of all tokens, or of some) are 2^k_power larger and whose queries 2^q_power."""
    x = B.step(seed, dtype, [90, 0], [new, new], 2, 1, dim, 16)
    flat = x["pool"].reshape(-1, x["pool"].shape[-1])
    m = 2 * 2 * dim
    scales = np.ascontiguousarray(flat[:, m:m + 16]).view("<f4").reshape(-1, 2, 2).copy()
    at = np.arange(flat.shape[0]) if tokens is None else np.array([x["table"][0, t // 16] * 16 + t % 16 for t in tokens])
    scales[at, :, 0] *= np.float32(2.0 ** k_power)
    flat[:, m:m + 16] = scales.astype("<f4").reshape(-1, 4).view(np.uint8).reshape(-1, 16)
    x["q"] = (x["q"].double() * 2.0 ** q_power).to(dtype)
    return x


@pytest.mark.parametrize("new", [1, 14, 30, 130])
@pytest.mark.parametrize("k_power, q_power", [(118, -118), (108, -118), (118, -112), (-110, 110), (-118, 118), (60, -118)])
def test_keys_and_queries_of_opposite_size(ctx, new, k_power, q_power):
    x = far(40, BF, new, k_power, q_power)
    base.check(ctx, x)
    base.check(ctx, x, softcap=0.7)
    base.check(ctx, x, scale=-0.2, window=40)


@pytest.mark.parametrize("new", [1, 14, 30])
@pytest.mark.parametrize("dim", [64, 128])
def test_a_small_scale_for_large_scores(ctx, new, dim):
    x = far(41, HF, new, 90, 8, dim)
    base.check(ctx, x, scale=2.0 ** -101)
    x = far(42, BF, new, 80, 18, dim)
    base.check(ctx, x, scale=-2.0 ** -101, softcap=3.0)
    x = far(42, BF, new, 113, -15, dim)
    base.check(ctx, x, scale=2.0 ** -101)


@pytest.mark.parametrize("new", [1, 14, 30])
def test_one_key_far_from_the_others(ctx, new):
    """Queries so small that ordinary keys have scores of 0, and one token whose scores count."""
    base.check(ctx, far(43, BF, new, 118, -118, tokens=[70]))
    base.check(ctx, far(44, BF, new, 118, -118, tokens=[3, 66, 89]), softcap=2.0)


@pytest.mark.parametrize("new", [1, 14, 30])
def test_no_scale_at_all(ctx, new):
    """A scale of 0: every visible token weighs the same, however large the keys."""
    base.check(ctx, far(45, BF, new, 98, 0), scale=0.0)
    base.check(ctx, far(46, HF, new, 95, 2), scale=0.0, softcap=2.0)
