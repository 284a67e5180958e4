"""Codes of heads full of numbers that lie in the middle of two codes, and of heads of any size.

The scale is max * (1 / 448) and a code the e4m3 number nearest to x * (1 / scale), each factor and product rounded to 32 bits: four
roundings of 2^-24, so a scale is within 2^-23 of max / 448, and a code is the nearest to a number within 2^-22 of x * 448 / max.  In the
middle of two codes it may be either."""
import numpy as np
import pytest
import torch

from oracle import paged8 as E
from paper_2608_25431_b200 import binding

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    c = binding.Ctx(64)
    yield c
    c.close()


def check(ctx, k, v):
    rows, heads, dim = k.shape
    pool = torch.zeros((-(-rows // 16), 16, binding.kv8_token_bytes(heads, dim)), dtype=torch.uint8, device="cuda")
    st = torch.ones(rows, dtype=torch.int32, device="cuda")
    ctx.kv_write(pool, k.cuda(), v.cuda(), torch.arange(rows, device="cuda"), None, st)
    torch.cuda.synchronize()
    assert not st.any()
    codes, scales, _ = E.unpack(pool.view(-1, pool.shape[-1])[:rows].cpu().numpy(), heads, dim)
    for j, x in enumerate((k, v)):
        x = x.double().numpy()
        scale = np.maximum(np.abs(x).max(-1) / 448.0, E.LEAST)
        assert (np.abs(scales[..., j] - scale) <= scale * 2.0 ** -23).all()
        z = x / scale[..., None]
        slack = np.abs(z) * 2.0 ** -22
        assert (np.abs(codes[:, j] - z) <= E.step(np.abs(z) + slack) / 2 + slack).all()
        # where no middle is that near, it is the one number
        near = np.abs(np.abs(z) / E.step(z) % 1.0 - 0.5) * E.step(z) <= slack
        sure = torch.from_numpy(z).float().to(torch.float8_e4m3fn).double().numpy()
        assert np.array_equal(codes[:, j][~near], sure[~near])


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("rows, heads, dim", [(700, 8, 128), (5, 3, 64), (900, 2, 80), (400, 1, 256), (33, 5, 16)])
def test_random_heads(ctx, dtype, rows, heads, dim):
    rng = np.random.default_rng(rows)
    check(ctx, *(torch.from_numpy(rng.standard_normal((rows, heads, dim))).to(dtype) for _ in range(2)))


@pytest.mark.parametrize("power", [-80, -40, 30, 100, 126])
def test_heads_of_any_size(ctx, power):
    rng = np.random.default_rng(power + 200)
    check(ctx, *(torch.from_numpy(np.clip(rng.standard_normal((300, 4, 64)), -1.9, 1.9) * 2.0 ** power).to(BF) for _ in range(2)))


def test_every_largest_element_and_every_tie(ctx):
    """Heads whose largest element runs over a binade of bf16, the others over all of its numbers below: every quotient that 8 bits by 8 bits
    give."""
    tops = 1 + torch.arange(128) / 128.0
    below = torch.arange(1, 129) / 128.0
    head = torch.cat([tops[:, None, None].expand(128, 2, 1), torch.stack([below[:127] * tops[:, None], (below[:127] / 2).expand(128, 127)], 1)], -1)
    k = torch.cat([head, head * 2.0 ** -3], 0).to(BF)
    check(ctx, k, -k)


def test_tiny_heads(ctx):
    """Scales at and around the least one."""
    rng = np.random.default_rng(5)
    k = torch.from_numpy(rng.integers(-255, 256, (60, 2, 64)) * 2.0 ** -133).to(BF)
    check(ctx, k, k * 2)
