"""Block tables while stack and tables are rewritten (they may be the untrusted side's): labels follow the pages that
were checked.  And calls of more pages than a call keeps for itself between its stages."""
import numpy as np
import pytest
import torch

from oracle import paged as P
from paper_2608_25431_b200 import binding
from test_gpu_paged_tables import dev, run_tables, same_tables

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Ctx(64)
    yield c
    c.close()


@pytest.mark.parametrize("take", [True, False])
@pytest.mark.parametrize("layers", [1, 40])
def test_a_page_that_was_not_checked_keeps_its_owner(ctx, take, layers):
    # user 0 takes page 5 (free), or gives it back, while the entry that names it also says 7 (user 9's) at times
    pages = 16
    label0 = torch.full((layers, pages), P.NONE, dtype=torch.int32, device="cuda")
    label0[:, 7] = 9
    if not take:
        label0[:, 5] = 0
    table, free, n_free = (torch.full((1, 2), -1, dtype=torch.int32, device="cuda"), torch.zeros(pages, dtype=torch.int32, device="cuda"),
                           torch.zeros(1, dtype=torch.int32, device="cuda"))
    named = free[:1] if take else table[0, :1]
    mine, other = dev([5]), dev([7])
    b = binding.Batch(dev([0]), dev([0 if take else 3]), dev([3 if take else 0]), table, 16, pages)
    label, st = label0.clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
    after = P.NONE if not take else 0
    side, flips = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(flips):
        for _ in range(1500):
            named.copy_(other)
            named.copy_(mine)
    for _ in range(25):
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            flips.replay()
        seen = []
        for _ in range(20):
            label.copy_(label0)
            n_free.fill_(1 if take else 0)
            ctx.block_tables(b, free, n_free, label, st, layers=layers)
            seen.append((label.clone(), st.clone()))
        torch.cuda.synchronize()
        for lab, s in seen:
            s = int(s)
            assert s in (0, P.BAD_TABLE)
            want = label0.clone()
            if s == 0:
                want[:, 5] = after
            assert torch.equal(lab, want), (s, lab[:, [5, 7]].tolist())


@pytest.mark.parametrize("spoil", [False, True])
def test_more_pages_than_are_kept(ctx, spoil):
    # 200 000 pages of one token are taken and 150 000 given back in one call
    rng = np.random.default_rng(3)
    n_take, n_give, pages = 200000, 150000, 350010
    perm = rng.permutation(pages).astype(np.int32)
    owner, have, want = np.array([3, 8], np.int32), np.array([0, n_give + 5], np.int32), np.array([n_take, 5], np.int32)
    table = np.full((2, n_take), -1, np.int32)
    table[1, : n_give + 5] = perm[: n_give + 5]
    label = np.full((2, pages), P.NONE, np.int32)
    label[:, perm[: n_give + 5]] = 8
    free = np.full(pages, -1, np.int32)
    n_free = n_take + 3
    free[:n_free] = perm[n_give + 5: n_give + 5 + n_free]
    if spoil:
        free[4] = free[n_free - 1]                        # a page of the first round and one of the last are the same
    s = owner, have, want, table, free, n_free, label, pages
    got, ref = run_tables(ctx, s, 1), P.block_tables(owner, have, want, table, 1, pages, free, n_free, label)
    assert bool((ref[4] == P.BAD_TABLE).all()) == spoil
    same_tables(got, ref)


@pytest.mark.parametrize("heights", [(4, 1000), (1000, -3), (40, 30000)])
def test_a_height_that_changes(ctx, heights):
    # the number of free pages is read once by a CTA: whatever each of them saw, labels stay with their pages
    pages, n = 20000, 64
    label0 = torch.full((2, pages), P.NONE, dtype=torch.int32, device="cuda")
    label0[:, 1000:] = 9                                  # user 9's, and not on the stack
    free = torch.arange(pages, dtype=torch.int32, device="cuda")
    table = torch.full((n, 4), -1, dtype=torch.int32, device="cuda")
    n_free, label, st = dev([heights[0]]), label0.clone(), torch.zeros(n, dtype=torch.int32, device="cuda")
    zero = torch.zeros(n, dtype=torch.int32, device="cuda")
    b = binding.Batch(torch.arange(n, dtype=torch.int32, device="cuda") % 8, zero, zero + 60, table, 16, pages)
    one, other = dev([heights[0]]), dev([heights[1]])
    side, flips = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(flips):
        for _ in range(1000):
            n_free.copy_(other)
            n_free.copy_(one)
    for _ in range(15):
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            flips.replay()
        seen = []
        for _ in range(15):
            label.copy_(label0)
            ctx.block_tables(b, free, n_free, label, st, layers=2)
            seen.append(label.clone())
        torch.cuda.synchronize()
        for lab in seen:
            assert (lab[:, 1000:] == 9).all() and (lab[:, :1000] >= P.NONE).all() and (lab[:, :1000] < 8).all() and torch.equal(lab[0], lab[1])
    label.copy_(label0)
    n_free.fill_(1000)
    ctx.block_tables(b, free, n_free, label, st, layers=2)
    torch.cuda.synchronize()
    assert not st.any() and int((label[0, :1000] >= 0).sum()) == n * 4 and torch.equal(label[0], label[1])
