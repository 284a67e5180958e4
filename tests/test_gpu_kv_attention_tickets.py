"""What an attention call leaves in its context's scratch for the next one: nothing.

Two calls of one context at once are against the rule, and their results are nobody's; they stay within their
arrays, and the calls behind them must be right."""
import pytest
import torch

import test_gpu_kv_attention as base
from paper_2608_25431_b200 import binding

pytestmark = pytest.mark.gpu


def captured(ctx, x, times):
    heads, dim = x["q"].shape[1:]
    b = binding.Batch(base.dev(x["owner"]), base.dev(x["have"]), base.dev(x["want"]), base.dev(x["table"]), x["pt"], x["pool"].shape[0])
    out = torch.zeros((x["rows"], heads, dim), dtype=x["q"].dtype, device="cuda")
    st = torch.zeros(len(x["owner"]), dtype=torch.int32, device="cuda")
    q = x["q"].contiguous()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(times):
            ctx.kv_attention(b, x["pool"], q, out, st)
    return graph, (b, out, st, q)


def test_calls_behind_two_that_ran_at_once():
    ctx = binding.Ctx(64)
    xs = [base.make(61, torch.bfloat16, have, [1] * len(have), heads, 1, dim, 16, tree=False)
          for have, heads, dim in (([9000], 1, 128), ([6000, 50, 2000], 2, 64), ([70, 20000], 1, 128))]
    want = [base.call(ctx, x) for x in xs]
    graphs = [captured(ctx, x, 30) for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    for _ in range(10):
        torch.cuda.synchronize()
        for s, (g, _) in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for x, w in zip(xs, want):
            for _ in range(2):
                got = base.call(ctx, x)
                assert all(torch.equal(a, b) for a, b in zip(w[:3], got[:3])) and not got[3].any()
    ctx.close()


def test_calls_of_every_kind_in_turn():
    # cut and whole items, idle CTAs, calls without rows and refused ones between one another, one context
    ctx = binding.Ctx(64)
    xs = [base.make(62, torch.bfloat16, have, new, heads, 1, dim, 16, tree=False)
          for have, new, heads, dim in (([9000], [1], 1, 128), ([0], [1], 1, 64), ([30] * 400, [1] * 400, 2, 128), ([9, 5], [0, 0], 1, 128),
                                        ([4000, 8], [8, 2], 2, 64), ([3000, 70], [40, 30], 2, 128))]
    want = [base.call(ctx, x) for x in xs[:3]] + [None] + [base.call(ctx, x) for x in xs[4:]]
    for _ in range(4):
        for x, w in zip(xs, want):
            if w is None:
                base.call(ctx, dict(x, rows=0, q=x["q"][:0]), extra=0)
                continue
            short = dict(x, q=x["q"][:-1], rows=x["rows"] - 1)
            if short["rows"]:
                assert (base.call(ctx, short)[3] == binding.ST_BAD_TABLE).all()
            got = base.call(ctx, x)
            assert all(torch.equal(a, b) for a, b in zip(w[:3], got[:3])) and not got[3].any()
    ctx.close()


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("mode", ["global", "relaxed"])
def test_the_first_call_of_a_context_is_refused_under_a_capture(new, mode):
    x = base.make(63, torch.bfloat16, [5000, 9], [new, new], 1, 1, 128, 16, tree=False)
    ctx = binding.Ctx(64)
    b = binding.Batch(base.dev(x["owner"]), base.dev(x["have"]), base.dev(x["want"]), base.dev(x["table"]), x["pt"], x["pool"].shape[0])
    q = x["q"].contiguous()
    out, st = torch.zeros_like(q), torch.zeros(2, dtype=torch.int32, device="cuda")
    refused = []
    with torch.cuda.graph(torch.cuda.CUDAGraph(), capture_error_mode=mode):
        out.zero_()
        try:
            ctx.kv_attention(b, x["pool"], q, out, st)
        except binding.GiftError as e:
            refused.append(e)
    assert len(refused) == 1
    base.check(ctx, x)                                 # outside it is served, and so is a capture from then on
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, capture_error_mode=mode):
        ctx.kv_attention(b, x["pool"], q, out, st)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, base.call(ctx, x)[0]) and not st.any()
    ctx.close()
