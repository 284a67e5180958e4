"""Attention under both kernels against the 64-bit values, within the bounds of kv_bounds: every type, head size and
scale, infinite scores, and calls replayed from a graph."""
import numpy as np
import pytest
import torch

import kv_bounds as B
import test_gpu_kv_attention as base
from paper_2608_25431_b200 import binding

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16
# query rows per K/V head: few (warp-level products), one tile of 128 and several (tcgen05)
ROWS = [([4, 2, 1], 2), ([40, 33, 5], 2), ([60, 70, 3], 4)]


@pytest.fixture(scope="module")
def ctx():
    c = binding.Ctx(64)
    yield c
    c.close()


def on_gpu(x):
    return dict(x, pool=x["pool"].cuda(), q=x["q"].cuda())


def check(ctx, x, scale):
    out, lse, who, st = base.call(ctx, on_gpu(x), scale=scale)
    r = B.bounds(x, x["q"].shape[2] ** -0.5 if scale is None else scale)
    assert not st.any()
    assert np.array_equal(np.isneginf(lse.cpu().numpy()), np.isneginf(r["lse"]))
    shown = np.isfinite(r["lse"])
    assert B.worst(out.double().cpu().numpy(), r["out"], r["out_tol"]) <= 1
    assert B.worst(lse.double().cpu().numpy()[shown], r["lse"][shown], r["lse_tol"][shown]) <= 1


@pytest.mark.parametrize("scale", [None, 0.0, 1.0, -0.2, 3.0, -1.5, 1e-30])
@pytest.mark.parametrize("new,group", ROWS)
@pytest.mark.parametrize("dtype,dim", [(BF, 64), (BF, 128), (HF, 64), (HF, 128)])
@pytest.mark.parametrize("tree", [True, False])
def test_scales(ctx, scale, new, group, dtype, dim, tree):
    check(ctx, B.step(71, dtype, [70, 3, 0], new, 2, group, dim, 16, tree), scale)


@pytest.mark.parametrize("scale", [None, -0.2, 0.0])
@pytest.mark.parametrize("new,group", [([3], 2), ([40], 2), ([70], 4)])
@pytest.mark.parametrize("dtype,dim", [(BF, 128), (HF, 64)])
def test_scales_of_a_request_cut_over_the_gpu(ctx, scale, new, group, dtype, dim):
    check(ctx, B.step(72, dtype, [4000], new, 1, group, dim, 16), scale)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("pt", [1, 16, 24])
@pytest.mark.parametrize("new,group", ROWS)
def test_types_and_pages(ctx, dtype, dim, pt, new, group):
    check(ctx, B.step(73, dtype, [200, 65, 31], new, 2, group, dim, pt), None)


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("new,group", [(1, 1), (3, 2), (40, 2), (64, 4)])
@pytest.mark.parametrize("dtype,dim", [(BF, 128), (HF, 64)])
@pytest.mark.parametrize("far", [10, 2000])
def test_infinite_scores(ctx, sign, new, group, dtype, dim, far):
    inf = float("inf")
    x = base.make(74, dtype, [far, 10, 10], [new] * 3, 1, group, dim, 16)
    x["q"] = torch.ones_like(x["q"])
    for r in range(3):
        pages = torch.from_numpy(x["table"][r][x["table"][r] >= 0]).long().cuda()
        x["pool"][pages, :, 0] = 1.0 if r != 1 else 0.0
    page = x["pool"][int(x["table"][0, 0])]
    page[3, 0, 0, 0] = -sign * inf                 # one score of minus infinity: weight 0
    pages = torch.from_numpy(x["table"][1][x["table"][1] >= 0]).long().cuda()
    x["pool"][pages, :, 0, 0, 0] = -sign * inf     # all of them: the rows count as seeing nothing
    page = x["pool"][int(x["table"][2, 0])]
    page[5, 0, 0, 2] = sign * inf                  # plus infinity: not a number
    out, lse = base.check(ctx, x, scale=sign * dim ** -0.5)
    assert torch.isfinite(out[:new]).all() and not out[new:2 * new].any() and torch.isneginf(lse[new:2 * new]).all()
    assert torch.isnan(out[2 * new:]).all()


@pytest.mark.parametrize("new,group", [(20, 2), (64, 4), (1, 2)])
def test_a_captured_call_follows_its_inputs(ctx, new, group):
    """The kernel for many rows with the one that joins its pieces, and both kinds of call in one graph."""
    x = base.make(75, BF, [3000, 20, 64], [new, max(1, new // 2), new], 2, group, 128, 16)
    y = base.make(76, BF, [2500, 7], [1, 1], 2, group, 128, 16, tree=False)
    base.call(ctx, x)
    calls = []
    for z in (x, y, x):
        heads, dim = z["q"].shape[1:]
        calls.append(dict(z=z, b=binding.Batch(base.dev(z["owner"]), base.dev(z["have"]), base.dev(z["want"]), base.dev(z["table"]), 16, z["pool"].shape[0]),
                          q=z["q"].contiguous(), out=torch.zeros((z["rows"], heads, dim), dtype=BF, device="cuda"),
                          lse=torch.zeros((z["rows"], heads), device="cuda"), who=torch.zeros(z["rows"], dtype=torch.int32, device="cuda"),
                          st=torch.full((len(z["owner"]),), 9, dtype=torch.int32, device="cuda"), label=base.dev(z["label"]),
                          mask=None if z["mask"] is None else torch.from_numpy(z["mask"].view(np.int32)).cuda()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for c in calls:
            ctx.kv_attention(c["b"], c["z"]["pool"], c["q"], c["out"], c["st"], tree_mask=c["mask"], lse=c["lse"], row_owner=c["who"], owner_map=c["label"])

    def same(rows):
        for c in calls:
            c["out"].zero_()
            c["lse"].zero_()
            c["st"].fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        got = [(c["out"].clone(), c["lse"].clone(), c["who"].clone(), c["st"].clone()) for c in calls]
        for c, g in zip(calls, got):
            want = base.call(ctx, c["z"])
            n = rows if c["z"] is x else c["z"]["rows"]
            for a, b in zip(g[:3], want[:3]):
                assert torch.equal(a[:n], b[:n])
            assert np.array_equal(g[3].cpu().numpy(), want[3])

    for _ in range(3):
        same(x["rows"])
    # new values, other lengths, a page that is not its request's: the same buffers
    x["q"].mul_(0.5)
    few = [max(1, new // 4), 0, max(1, new // 3)]
    x["have"] = np.array([100, 29, 64], np.int32)
    x["want"] = x["have"] + np.array(few, np.int32)
    x["label"][x["table"][2, 1]] = x["owner"][2] + 1
    for c in (calls[0], calls[2]):
        c["b"].tensors[1].copy_(base.dev(x["have"]))
        c["b"].tensors[2].copy_(base.dev(x["want"]))
        c["q"].copy_(x["q"])
        c["label"].copy_(base.dev(x["label"]))
    for _ in range(2):
        same(sum(few))
    assert calls[0]["st"].tolist() == [0, 0, binding.ST_OWNER_MISMATCH]
