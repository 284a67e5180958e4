"""More rows than the GPU has warps against the 64-bit oracle: sampled rows, every status, every page that is not written."""
import numpy as np
import pytest
import torch

import test_gpu_kv_write as base
from paper_2608_25431_b200 import binding

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    c = binding.Ctx(64)
    yield c
    c.close()


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("dtype, heads, q_heads, dim, paired, axes, norm", [(BF, 3, 5, 64, False, 1, True), (HF, 2, 2, 128, True, 3, False), (BF, 1, 2, 256, False, 2, True)])
def test_sampled_rows(ctx, monkeypatch, bits, dtype, heads, q_heads, dim, paired, axes, norm):
    rows, pt = 7001, 16
    x = base.make(9, dtype, rows, heads, q_heads, dim, pt, bits, paired=paired, axes=axes, norm=norm)
    x["slots"][::50] = -1
    x["slots"][7::501] = 10 ** 9
    x["owner"][3::97] = 6
    q_out, pool, st = base.call(ctx, x)
    some = np.unique(np.concatenate([np.arange(0, rows, 61), [rows - 1], np.arange(3, rows, 970), np.arange(7, rows, 501)]))
    # base.check on the sampled rows, with the whole call's results in place of one of its own
    y = dict(x, **{k: x[k][some] for k in ("all", "q", "k", "v", "slots", "owner")}, pos=x["pos"][:, some])
    before, after = (p.reshape(-1, *p.shape[2:]) for p in (x["pool"], pool))
    mine = np.zeros(before.shape[0], bool)
    mine[y["slots"][(y["slots"] >= 0) & (y["slots"] < len(mine))]] = True
    shown = before.clone()
    shown[mine] = after[mine]
    monkeypatch.setattr(base, "call", lambda *_: (q_out[some], shown.reshape(pool.shape), st[some]))
    base.check(ctx, y)
    # the other rows: statuses, and slots that nobody writes
    good = (x["slots"] >= 0) & (x["slots"] < before.shape[0]) & (x["owner"] == 5)
    assert np.array_equal(st == 0, good | (x["slots"] == -1))
    free = np.ones(before.shape[0], bool)
    free[x["slots"][good]] = False
    assert torch.equal(after[free], before[free]) and (q_out[~good] == 7).all()
