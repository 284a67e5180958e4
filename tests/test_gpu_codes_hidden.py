"""What lies before a window in an 8-bit cache does not reach a row: codes of NaN, scales that are NaN, infinite or huge, in tokens that
nobody sees and in tokens that only other rows of the request see.  Nor do the rows of other requests, not even in a result's last bit."""
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


def spoiled(x, tokens, seed):
    """The step with bad contents in these (request, token) places."""
    rng = np.random.default_rng(seed)
    heads, dim, pt = x["heads"], x["q"].shape[2], x["pt"]
    y = dict(x, pool=x["pool"].copy())
    m = 2 * heads * dim
    bad = np.array([[np.nan, np.inf], [1e38, -np.inf], [1e30, np.nan]], "<f4")
    for n, (r, t) in enumerate(tokens):
        token = y["pool"][x["table"][r, t // pt], t % pt]
        token[:m] = rng.integers(0, 256, m)
        token[:m:7] = 0x7F
        token[m:m + 8 * heads] = np.tile(bad[n % 3], heads).view(np.uint8)
    return y


@pytest.mark.parametrize("dtype, dim", [(BF, 128), (HF, 64)])
@pytest.mark.parametrize("pt", [3, 16, 24])
@pytest.mark.parametrize("group, new", [(1, 1), (1, 14), (2, 30), (1, 300)])
@pytest.mark.parametrize("window", [13, 75, 203])
def test_tokens_before_a_window(ctx, dtype, dim, pt, group, new, window):
    x = B.step(window + new, dtype, [270, 130], [new, 1], 2, group, dim, pt)
    near = dict(window=window)
    if pt == 16:
        near.update(softcap=4.0, slopes=np.array([2.0 ** -(h + 2) for h in range(2 * group)], np.float32))
    want = base.call(ctx, x, **near)
    # those that no row sees
    nobody = [(r, t) for r in range(2) for t in range(max(0, int(x["have"][r]) - window + 1))]
    got = base.call(ctx, spoiled(x, nobody, 1), **near)
    assert not want[3].any() and all(np.array_equal(a, b) for a, b in zip(got, want))
    # those that the first rows alone see: the later ones stay as they are
    for cut in {1, new // 2, new - 1} - {0}:
        low, first = max(0, 270 - window + 1), max(0, 270 + cut - window + 1)
        some = [(0, t) for t in range(low, min(first, 270 + cut))]
        got = base.call(ctx, spoiled(x, some, 2), **near)
        assert np.array_equal(got[3], want[3]) and np.array_equal(got[2], want[2])
        assert np.array_equal(got[0][cut:], want[0][cut:]) and np.array_equal(got[1][cut:], want[1][cut:])


@pytest.mark.parametrize("group, new, other", [(1, 20, 60), (5, 10, 7), (4, 6, 40), (1, 3, 3)])
@pytest.mark.parametrize("near", [dict(softcap=3.0), dict(softcap=3.0, window=50), {}])
def test_rows_of_another_request(ctx, group, new, other, near):
    """Whatever size the next request's queries have, this one's rows are the same, to the bit."""
    x = B.step(new, HF, [150, 70], [new, other], 2, group, 64, 16)
    x["q"][:new] *= 0.25                                   # scores far below the cap
    want = base.call(ctx, x, **near)
    y = dict(x, q=x["q"].clone())
    y["q"][new:] *= 50.0
    got = base.call(ctx, y, **near)
    assert np.array_equal(got[0][:new], want[0][:new]) and np.array_equal(got[1][:new], want[1][:new])


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("requests, have, new", [(2, 90, 3), (2, 90, 14), (2, 90, 60), (50, 700, 3), (50, 700, 8), (50, 700, 14), (12, 700, 30)])
@pytest.mark.parametrize("softcap", [0.0, 3.0])
def test_tokens_that_another_row_sees(ctx, dim, requests, have, new, softcap):
    """A drafted token with a large key and value that its own row alone sees: the other rows are the same, to the bit."""
    x = B.step(new, HF, [have] * requests, [new] * requests, 2, 1, dim, 16, tree=True)
    mine = np.arange(requests * new) % new == 1
    x["mask"][:, 0] &= ~np.uint32(2)
    x["mask"][mine, 0] |= np.uint32(2)
    m = 4 * dim

    def louder(x, t, by):
        for r in range(requests):
            token = x["pool"][x["table"][r, t // 16], t % 16]
            token[m:m + 16] = (np.ascontiguousarray(token[m:m + 16]).view("<f4") * np.float32(by)).astype("<f4").view(np.uint8)

    for t in range(have, have + new):                      # some new maxima among the step's own tokens
        louder(x, t, 1.4)
    want = base.call(ctx, x, softcap=softcap)
    y = dict(x, pool=x["pool"].copy())
    louder(y, have + 1, 60.0)
    got = base.call(ctx, y, softcap=softcap)
    assert not np.array_equal(got[0][mine], want[0][mine])
    assert np.array_equal(got[0][~mine], want[0][~mine]) and np.array_equal(got[1][~mine], want[1][~mine])
