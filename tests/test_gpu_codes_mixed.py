"""Decode rows and a prompt of several tiles in one call over 8-bit pages: all its requests share a kernel, whichever the call's average of
rows picks.  Bounds: tests/codes_bounds.py."""
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


# averages of query rows: up to 8, up to 16, above
@pytest.mark.parametrize("decodes, prompt, group", [(50, 200, 1), (30, 330, 1), (6, 300, 1), (20, 150, 4)])
@pytest.mark.parametrize("near", [{}, dict(window=70, softcap=2.0)])
def test_decode_rows_and_a_prompt(ctx, decodes, prompt, group, near):
    rng = np.random.default_rng(decodes)
    have, new = rng.integers(0, 150, decodes + 1), np.ones(decodes + 1, np.int64)
    at = decodes // 3
    have[at], new[at] = 100, prompt
    base.check(ctx, B.step(decodes, BF, have, new, 2, group, 64, 16), **near)
    base.check(ctx, B.step(prompt, HF, have, new, 1, group, 128, 24), extra=40, **near)


def test_room_for_more_rows_than_there_are(ctx):
    """A padded step: the rows that exist are the same whatever kernel the room picks, up to its rounding."""
    x = B.step(3, HF, [60, 200, 9], [1, 1, 2], 2, 2, 128, 16)
    for extra in (0, 10, 60, 500):
        base.check(ctx, x, extra=extra)
