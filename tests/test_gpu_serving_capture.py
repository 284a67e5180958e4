"""A whole serving step in one graph: block tables, slots, appends, attention, the segment table of its new blocks.
The graph is replayed on other lengths, values and labels in the same buffers, on a stream of its own, and every
array is compared with the same calls made one by one (tables with the oracle)."""
import numpy as np
import pytest
import torch

from oracle import paged as P
from paper_2608_25431_b200 import binding, workloads as W

pytestmark = pytest.mark.gpu

LAYERS, PT, HEADS, DIM, PAGES, N = 3, 16, 2, 128, 60, 5


def dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


class Side:
    def __init__(self, rows, group):
        i32 = dict(dtype=torch.int32, device="cuda")
        rng = np.random.default_rng(11)
        self.owner, self.have, self.want = dev([3, 0, 4, 1, 2]), torch.zeros(N, **i32), torch.zeros(N, **i32)
        self.table, self.free, self.n_free = torch.full((N, 20), -1, **i32), dev(rng.permutation(PAGES)), dev([PAGES])
        self.label = torch.full((LAYERS, PAGES), P.NONE, **i32)
        self.pool = torch.zeros((LAYERS, PAGES, PT, 2, HEADS, DIM), dtype=torch.bfloat16, device="cuda")
        self.kv = torch.zeros((rows, 2 * HEADS, DIM), dtype=torch.bfloat16, device="cuda")
        self.q, self.out = (torch.zeros((rows, HEADS * group, DIM), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.slots, self.ints = torch.zeros(rows, dtype=torch.int64, device="cuda"), torch.zeros((4, rows), **i32)
        self.ptr, self.total = torch.zeros(N + 1, **i32), torch.zeros(2, dtype=torch.int64, device="cuda")
        self.st = torch.zeros((2, N), **i32)
        self.serial, self.segs, self.entry = dev(np.arange(7, 7 + N)), torch.zeros((200, 40), dtype=torch.uint8, device="cuda"), torch.zeros(200, **i32)
        self.b = binding.Batch(self.owner, self.have, self.want, self.table, PT, PAGES)

    def arrays(self):
        return [v for v in vars(self).values() if isinstance(v, torch.Tensor)]

    def step(self, ctx):
        ctx.block_tables(self.b, self.free, self.n_free, self.label, self.st[0], layers=LAYERS)
        ctx.slot_map(self.b, self.slots, row_req=self.ints[0], row_owner=self.ints[1], row_ptr=self.ptr, total=self.total[:1])
        for layer in range(LAYERS):
            ctx.kv_append(self.pool[layer], self.kv[:, :HEADS], self.kv[:, HEADS:], self.slots, self.ints[1], self.ints[2], owner_map=self.label[layer])
        ctx.kv_attention(self.b, self.pool[1], self.q, self.out, self.st[1], row_owner=self.ints[3], owner_map=self.label[1])
        ctx.kv_segments(self.b, self.serial, self.segs, self.entry, LAYERS, 2 * HEADS * DIM * 2, new_blocks=True, total=self.total[1:])


@pytest.mark.parametrize("rows,group", [(800, 4), (800, 1), (70, 1)])
def test_a_captured_step_with_its_tables(rows, group):
    ctx = binding.Ctx(8)
    a, e = Side(rows, group), Side(rows, group)
    e.step(ctx)                                           # nothing to do yet; the context's scratch
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        a.step(ctx)
    # prompts, a decode step, tokens given back and taken, more blocks than there are, growth and shrinking, all given
    # back; with 70 rows most of these are more rows than the call has
    steps = [([0] * N, [1, 100, 33, 16, 200]), ([1, 100, 33, 16, 200], [2, 101, 34, 17, 201]), ([2, 101, 34, 17, 201], [0, 140, 34, 3, 230]),
             ([0, 140, 34, 3, 230], [310, 140, 34, 320, 320]), ([310, 140, 34, 3, 230], [64, 160, 64, 64, 256]), ([64, 160, 64, 64, 256], [0] * N)]
    for k, (have, want) in enumerate(steps):
        g = torch.Generator(device="cuda").manual_seed(k)
        kv, q = torch.randn(a.kv.shape, generator=g, device="cuda"), torch.randn(a.q.shape, generator=g, device="cuda")
        kept = a.table[2, 1].clone()
        for s in (a, e):
            s.have.copy_(dev(have))
            s.want.copy_(dev(want))
            s.kv.copy_(kv)
            s.q.copy_(q)
            s.out.zero_()
            if k == 4:                                    # another user's page in a table
                s.table[2, 1] = s.table[1, 0]
        before = [x.cpu().numpy() for x in (a.owner, a.have, a.want, a.table)]
        ref = P.block_tables(*before, PT, PAGES, a.free.cpu().numpy(), int(a.n_free), a.label.cpu().numpy())
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.synchronize()
        e.step(ctx)
        torch.cuda.synchronize()
        for x, y in zip(a.arrays(), e.arrays()):
            assert torch.equal(x, y), k
        now = [x.cpu().numpy() for x in (a.owner, a.have, a.want, a.table)]
        assert np.array_equal(now[3], ref[0]) and int(a.n_free) == ref[2] and np.array_equal(a.label.cpu().numpy(), ref[3]), k
        assert np.array_equal(a.st[0].cpu().numpy().astype(np.uint32), ref[4]), k
        segs, entry, total = P.kv_segments(*now, PT, PAGES, a.serial.cpu().numpy(), LAYERS, 2 * HEADS * DIM * 2, 200, W.SEG_DTYPE, new_blocks=True)
        assert np.array_equal(a.segs.cpu().numpy().reshape(-1).view(W.SEG_DTYPE), segs) and np.array_equal(a.entry.cpu().numpy(), entry), k
        assert int(a.total[1]) == total
        if sum(max(0, w - h) for h, w in zip(have, want)) > rows:
            assert (a.st[1] == binding.ST_BAD_TABLE).all() and not a.out.any()
        elif k < 3:
            assert not a.st.any()
        if k == 3:
            assert ref[4].tolist() == [0, 0, 0, P.NO_BLOCKS, P.NO_BLOCKS]
        if k == 4 and rows > 70:
            assert a.st[1].tolist() == [0, 0, binding.ST_OWNER_MISMATCH, 0, 0]
        if k == 4:
            for s in (a, e):
                s.table[2, 1] = kept
    assert int(a.n_free) == PAGES and (a.label == P.NONE).all() and (a.table == -1).all()
    ctx.close()
