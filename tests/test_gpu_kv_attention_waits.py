"""What becomes of an attention call whose waits run out: a short limit (gift_ctx_wait_limit) makes them.

The waits are those of the kernel for many query rows; it must end with nothing of its own under way, so that the
calls behind it are right."""
import pytest
import torch

import test_gpu_kv_attention as base
from paper_2608_25431_b200 import binding

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16
LIMITS = [1, 200, 500, 1000, 2000, 4000, 8000, 30000]


@pytest.fixture(scope="module")
def ctx():
    c = binding.Ctx(64)
    yield c
    c.close()


# one tile of rows, several tiles (two CTAs to a slice), gathered tokens, heads of 64
CASES = [(BF, 128, 4, 20, 16), (HF, 128, 4, 64, 16), (BF, 128, 2, 30, 3), (HF, 64, 8, 5, 64)]


def batch(dtype, dim, group, new, pt):
    return base.make(51, dtype, [2500, 0, 700, 33, 64, 1200, 5], [new, 3, 0, new, new, 1, new], 4, group, dim, pt)


@pytest.mark.parametrize("dtype,dim,group,new,pt", CASES)
def test_calls_behind_one_whose_waits_ran_out(ctx, dtype, dim, group, new, pt):
    x = batch(dtype, dim, group, new, pt)
    ctx.wait_limit(0)
    want = base.call(ctx, x)
    assert not want[3].any()
    for ns in LIMITS:
        ctx.wait_limit(ns)
        for _ in range(3):
            base.call(ctx, x)
        ctx.wait_limit(0)
        got = base.call(ctx, x)
        for a, b in zip(want[:3], got[:3]):
            assert torch.equal(a, b), ns
        assert not got[3].any(), ns


def test_limits_out_of_range(ctx):
    with pytest.raises(binding.GiftError):
        ctx.wait_limit(10 ** 9 + 1)
    with pytest.raises(ValueError):
        ctx.wait_limit(-1)
    ctx.wait_limit(10 ** 9)
    ctx.wait_limit(0)


@pytest.mark.parametrize("dtype,dim,group,new,pt", CASES)
def test_a_stalled_request_says_so(ctx, dtype, dim, group, new, pt):
    # a CTA that gives up may hold any head and any tile of rows of a request
    x = batch(dtype, dim, group, new, pt)
    rows = torch.tensor([max(0, int(w) - int(h)) for h, w in zip(x["have"], x["want"])])
    of_row = torch.repeat_interleave(torch.arange(len(rows)), rows).cuda()
    ctx.wait_limit(0)
    want = base.call(ctx, x)
    seen = set()
    for ns in LIMITS:
        for _ in range(4):
            ctx.wait_limit(ns)
            out, lse, who, st = base.call(ctx, x)
            assert all(s in (0, binding.ST_STALLED) for s in st), (ns, st)
            seen |= set(int(s) for s, m in zip(st, rows) if m)
            assert not st[rows == 0].any()
            stalled = torch.from_numpy(st.astype("int64")).cuda()[of_row] != 0
            assert not out[stalled].any() and torch.isneginf(lse[stalled]).all() and (who[stalled] == binding.OWNER_CONFLICT).all(), ns
            for a, b in zip((out, lse, who), want[:3]):
                assert torch.equal(a[~stalled], b[~stalled]), ns
    ctx.wait_limit(0)
    assert seen == {0, binding.ST_STALLED}
