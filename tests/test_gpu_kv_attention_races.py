"""Attention while the block table is rewritten: whatever the timing, no row holds what a page held that is not its
request's.  The table may be the untrusted side's; all entries here are pages of the pool."""
import pytest
import torch

from paper_2608_25431_b200 import binding

pytestmark = pytest.mark.gpu


# one row and several per K/V head (warp-level products), many (tcgen05: runs of a page, gathered tokens)
@pytest.mark.parametrize("rows,pt", [(1, 16), (4, 16), (40, 16), (40, 64), (40, 4)])
def test_no_row_holds_another_users_page(rows, pt):
    heads, group, dim, tokens = 2, 2, 64, 2048
    blocks = tokens // pt
    ctx = binding.Ctx(4)
    # own pages hold V of 1, another user's V of 1000; K is the same, so that scores do not tell
    pool = torch.zeros((2 * blocks, pt, 2, heads, dim), dtype=torch.bfloat16, device="cuda")
    pool[:blocks, :, 1], pool[blocks:, :, 1] = 1.0, 1000.0
    label = torch.zeros(2 * blocks, dtype=torch.int32, device="cuda")
    label[blocks:] = 1
    own = torch.arange(blocks, dtype=torch.int32, device="cuda")[None].contiguous()
    # one entry changes: a call that looked all of them up while they were its own, and this one again while it
    # was not, would put the other's V beside its own K
    table, other = own.clone(), own.clone()
    other[0, blocks // 2] += blocks
    one = torch.ones(1, dtype=torch.int32, device="cuda")
    b = binding.Batch(one * 0, one * (tokens - rows), one * tokens, table, pt, 2 * blocks)
    q = torch.randn((rows, heads * group, dim), device="cuda").bfloat16()
    mask = torch.full((rows, 2), -1, dtype=torch.int32, device="cuda")
    n = 60
    outs, st = torch.zeros((n, rows, heads * group, dim), dtype=torch.bfloat16, device="cuda"), torch.zeros((n, 1), dtype=torch.int32, device="cuda")
    ctx.kv_attention(b, pool, q, outs[0], st[0], tree_mask=mask, owner_map=label)
    torch.cuda.synchronize()
    assert not st[0].any() and (outs[0] == 1).all()
    side, noise = torch.cuda.Stream(), torch.cuda.Stream()
    x = torch.zeros(1 << 26, device="cuda")        # something that runs through the SMs' first-level caches meanwhile
    y = torch.zeros_like(x)
    flips = torch.cuda.CUDAGraph()
    with torch.cuda.graph(flips):
        for _ in range(1000):
            table.copy_(other)
            table.copy_(own)
    for _ in range(20):
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            flips.replay()
        with torch.cuda.stream(noise):
            for _ in range(20):
                torch.add(x, 1.0, out=y)
        for k in range(n):
            ctx.kv_attention(b, pool, q, outs[k], st[k], tree_mask=mask, owner_map=label)
        torch.cuda.synchronize()
        # a (row, head) is from own pages alone or zero
        assert ((outs == 1) | (outs == 0)).all(), (float(outs.max()), int((outs.amax((1, 2, 3)) > 1).sum()))
        assert all(s in (0, binding.ST_OWNER_MISMATCH) for s in st.flatten().tolist())
    ctx.kv_attention(b, pool, q, outs[0], st[0], tree_mask=mask, owner_map=label)
    torch.cuda.synchronize()
    assert not st[0].any() and (outs[0] == 1).all()
    ctx.close()
