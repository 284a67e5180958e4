"""A serving run over the cache in 8 bits, as its calls are meant to follow one another: block tables, slots, rows with norms and
rotation into labelled pages, attention with capped scores and a window, a tree of drafted tokens, the cache read back, its export
under the owners' keys and the same attention on the other side; and whole steps in one graph."""
import gc

import numpy as np
import pytest
import torch

import codes_bounds as B
from oracle import gcm, paged as P, paged8 as E
from paper_2608_25431_b200 import binding, workloads as W

pytestmark = pytest.mark.gpu

LAYERS, PT, HEADS, GROUP, DIM, PAGES = 2, 16, 3, 4, 64, 96
TOKEN = binding.kv8_token_bytes(HEADS, DIM)
FREQ = torch.tensor([1e4 ** (-i / 16) for i in range(16)], dtype=torch.float32)


def dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def np_(t):
    return t.cpu().numpy()


class Cache:
    """One side's pages, labels, tables and free pages, and a layer's weights."""

    def __init__(self, ctx, owner, seed, dtype=torch.bfloat16):
        rng = np.random.default_rng(seed)
        n = len(owner)
        self.ctx, self.owner, self.dtype = ctx, owner, dtype
        self.pool = torch.full((LAYERS, PAGES, PT, TOKEN), 0x7F, dtype=torch.uint8, device="cuda")     # whatever was there before
        self.label = torch.full((LAYERS, PAGES), P.NONE, dtype=torch.int32, device="cuda")
        self.table = torch.full((n, 20), -1, dtype=torch.int32, device="cuda")
        self.free, self.n_free = dev(rng.permutation(PAGES)), dev([PAGES])
        self.status = torch.zeros(n, dtype=torch.int32, device="cuda")
        g = torch.Generator().manual_seed(9)
        self.q_norm, self.k_norm = (1 + 0.1 * torch.randn(2, DIM, generator=g)).to(dtype).cuda()
        self.freq = FREQ.cuda()

    def batch(self, have, want):
        return binding.Batch(dev(self.owner), dev(have), dev(want), self.table, PT, PAGES)

    def resize(self, have, want):
        self.ctx.block_tables(self.batch(have, want), self.free, self.n_free, self.label, self.status, layers=LAYERS)
        assert not self.status.any()

    def write(self, have, want, qkv, rel=None):
        """q [layers, rows, heads, dim], turned, of rows that are in the pages afterwards."""
        rows = qkv.shape[1]
        slots, ints = torch.zeros(rows, dtype=torch.int64, device="cuda"), torch.zeros((3, rows), dtype=torch.int32, device="cuda")
        self.ctx.slot_map(self.batch(have, want), slots, row_pos=ints[0], row_owner=ints[1], rel=None if rel is None else dev(rel))
        q = torch.zeros((LAYERS, rows, HEADS * GROUP, DIM), dtype=self.dtype, device="cuda")
        hq = HEADS * GROUP
        for layer in range(LAYERS):
            self.ctx.kv_write(self.pool[layer], qkv[layer, :, hq:hq + HEADS], qkv[layer, :, hq + HEADS:], slots, ints[1], ints[2], q=qkv[layer, :, :hq], q_out=q[layer],
                              q_norm=self.q_norm, k_norm=self.k_norm, pos=ints[0], freq=self.freq, owner_map=self.label[layer])
            assert not ints[2].any()
        return q

    def attend(self, layer, have, want, q, mask=None, **near):
        out, who = torch.zeros_like(q), torch.zeros(q.shape[0], dtype=torch.int32, device="cuda")
        st = torch.full((len(self.owner),), 9, dtype=torch.int32, device="cuda")
        self.ctx.kv_attention_codes(self.batch(have, want), self.pool[layer], HEADS, q, out, st, tree_mask=mask, row_owner=who, owner_map=self.label[layer], **near)
        if not st.any():
            x = dict(owner=self.owner, have=have, want=want, table=np_(self.table), pool=np_(self.pool[layer]), heads=HEADS, q=q.cpu(), mask=None if mask is None else np_(mask).view(np.uint32), pt=PT)
            b = B.bounds(x, float(np.float32(DIM ** -0.5)), **near)
            assert B.worst(np_(out.double()), b["out"], b["out_tol"]) <= 1
            assert np.array_equal(np_(who), np.repeat(self.owner, np.maximum(0, want - have)))
        return out, who, st


def projected(rows, seed, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((LAYERS, rows, HEADS * GROUP + 2 * HEADS, DIM), generator=g).to(dtype).cuda()


def test_a_run_from_lengths_to_the_other_side():
    rng = np.random.default_rng(7)
    n = 6
    owner = np.array([3, 0, 5, 1, 4, 2], dtype=np.int32)
    ctx = binding.Ctx(8)
    keys = rng.integers(0, 256, size=(8, 16), dtype=np.uint8)
    ctx.set_keys(np.arange(8, dtype=np.int32), keys)
    a = Cache(ctx, owner, 1)

    # prompts: many rows a head
    zero, have = np.zeros(n, np.int32), np.array([1, 16, 17, 200, 64, 33], dtype=np.int32)
    a.resize(zero, have)
    q = a.write(zero, have, projected(int(have.sum()), 1))
    a.attend(0, zero, have, q[0])
    a.attend(1, zero, have, q[1], softcap=4.0, window=40)

    # a tree of drafted tokens; the path to every request's last one is accepted
    new = np.array([5, 8, 1, 7, 0, 30], dtype=np.int32)
    want, total = have + new, int(new.sum())
    a.resize(have, want)
    qkv = projected(total, 2)
    q = a.write(have, want, qkv)
    mask, parent, t = np.zeros((total, 1), dtype=np.uint32), np.full(total, -1), 0
    rel, accepted = np.full(total, -1, dtype=np.int32), np.zeros(n, np.int32)
    for r in range(n):
        for i in range(new[r]):
            up = int(rng.integers(-1, i)) if i else -1
            parent[t + i] = up
            mask[t + i, 0] = (mask[t + up, 0] if up >= 0 else 0) | np.uint32(1 << i)
        i, path = int(new[r]) - 1, []
        while i >= 0:
            path.append(i)
            i = int(parent[t + i])
        for k, i in enumerate(reversed(path)):
            rel[t + i] = k
        accepted[r] = len(path)
        t += int(new[r])
    for layer in range(LAYERS):
        a.attend(layer, have, want, q[layer], dev(mask.view(np.int32)))
    a.write(have, want, qkv, rel)                          # the accepted rows once more, where (and turned as) they belong now
    now = have + accepted
    a.resize(want, now)

    # a decode step
    step = now + 1
    a.resize(now, step)
    q = a.write(now, step, projected(n, 3))
    there = [a.attend(layer, now, step, q[layer], softcap=9.0)[0] for layer in range(LAYERS)]

    # the whole cache of a layer back in 16 bits
    rows = int(step.sum())
    slots, who = torch.zeros(rows, dtype=torch.int64, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda")
    ctx.slot_map(a.batch(zero, step), slots, row_owner=who)
    k, v = (torch.zeros((rows, HEADS, DIM), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    st = torch.ones(rows, dtype=torch.int32, device="cuda")
    ctx.kv_read(a.pool[1], k, v, slots, who, st, owner_map=a.label[1])
    values = E.values(np_(a.pool[1]).reshape(PAGES * PT, TOKEN)[np_(slots)], HEADS, DIM)
    assert not st.any()
    for j, got in enumerate((k, v)):
        assert (np.abs(np_(got.double()) - values[:, j]) <= np.abs(values[:, j]) * (2.0 ** -8 + 2.0 ** -23)).all()
    who[5] = 7
    ctx.kv_read(a.pool[1], k, v, slots, who, st, owner_map=a.label[1])
    assert st.nonzero().flatten().tolist() == [5] and not k[5].any() and not v[5].any()

    # export every block's filled bytes under its owner's key, out of place: codes and scales are all that the other side needs
    blocks = int((-(-step // PT)).sum())
    segs, page_table = torch.zeros((blocks * LAYERS, 40), dtype=torch.uint8, device="cuda"), torch.zeros(blocks * LAYERS, dtype=torch.int32, device="cuda")
    ctx.kv_segments(a.batch(now, step), dev(np.arange(100, 100 + n)), segs, page_table, LAYERS, TOKEN)
    src = a.pool.view(-1)
    cipher, nseg = torch.zeros_like(src), segs.shape[0]
    tags, st = torch.zeros((nseg, 16), dtype=torch.uint8, device="cuda"), torch.full((nseg,), 9, dtype=torch.int32, device="cuda")
    where = dict(page_table=page_table, page_bytes=PT * TOKEN, unit_bytes=PT * TOKEN)
    ctx.seg_encrypt(src, cipher, segs, nseg, tags, st, owner_map=a.label.view(-1), **where)
    assert not st.any()
    ref = np.zeros_like(np_(cipher))
    ref_tags, ref_st = gcm.seg_encrypt(np_(src), ref, np_(segs).reshape(-1).view(W.SEG_DTYPE), np.arange(8, dtype=np.int32), keys, 8, np_(page_table),
                                       PT * TOKEN, np_(a.label.view(-1)), PT * TOKEN)
    assert np.array_equal(np_(tags), ref_tags) and not ref_st.any() and np.array_equal(np_(cipher), ref)
    b = Cache(ctx, owner, 2)
    b.table.copy_(a.table)
    ctx.seg_decrypt(cipher, b.pool.view(-1), segs, nseg, tags, st, owner_map=b.label.view(-1), **where)
    assert not st.any() and torch.equal(b.label, a.label)
    for layer in range(LAYERS):
        assert torch.equal(b.attend(layer, now, step, q[layer], softcap=9.0)[0], there[layer])

    # a tampered block: its pages are nobody's, and its request's rows do not come out
    tags[2, 0] ^= 1
    ctx.seg_decrypt(cipher, b.pool.view(-1), segs, nseg, tags, st, owner_map=b.label.view(-1), **where)
    assert int(st[2]) == binding.ST_TAG_MISMATCH
    victim = int(np.searchsorted(np.cumsum(-(-step // PT)), 2, side="right"))
    out, who, st = b.attend(0, now, step, q[0])
    assert st.nonzero().flatten().tolist() == [victim] and int(st[victim]) == binding.ST_UNOWNED and not out[victim].any()
    ctx.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("group_rows", [1, 3, 40])
def test_a_captured_step_replays_on_new_lengths(dtype, group_rows):
    """Slots, rows written, attention and rows read back, captured once with room for group_rows tokens a request, replayed as the
    lengths grow, by turns with the same calls made one by one on other buffers."""
    owner = np.array([1, 2, 3], dtype=np.int32)
    ctx = binding.Ctx(4)
    rows = 3 * group_rows
    sides = []
    for _ in range(2):
        c = Cache(ctx, owner, 3, dtype)
        c.resize(np.zeros(3, np.int32), np.full(3, 300, np.int32))
        i32 = dict(dtype=torch.int32, device="cuda")
        s = dict(c=c, have=torch.zeros(3, **i32), want=torch.zeros(3, **i32), slots=torch.zeros(rows, dtype=torch.int64, device="cuda"), ints=torch.zeros((4, rows), **i32),
                 qkv=torch.zeros((rows, HEADS * GROUP + 2 * HEADS, DIM), dtype=dtype, device="cuda"), st=torch.zeros(3, **i32),
                 q=torch.zeros((rows, HEADS * GROUP, DIM), dtype=dtype, device="cuda"), out=torch.zeros((rows, HEADS * GROUP, DIM), dtype=dtype, device="cuda"),
                 back=torch.zeros((2, rows, HEADS, DIM), dtype=dtype, device="cuda"))
        s["b"] = binding.Batch(dev(owner), s["have"], s["want"], c.table, PT, PAGES)
        sides.append(s)

    def step(s):
        c, hq = s["c"], HEADS * GROUP
        ctx.slot_map(s["b"], s["slots"], row_pos=s["ints"][0], row_owner=s["ints"][1])
        ctx.kv_write(c.pool[0], s["qkv"][:, hq:hq + HEADS], s["qkv"][:, hq + HEADS:], s["slots"], s["ints"][1], s["ints"][2], q=s["qkv"][:, :hq], q_out=s["q"], q_norm=c.q_norm,
                     k_norm=c.k_norm, pos=s["ints"][0], freq=c.freq, owner_map=c.label[0])
        ctx.kv_attention_codes(s["b"], c.pool[0], HEADS, s["q"], s["out"], s["st"], owner_map=c.label[0], window=50)
        ctx.kv_read(c.pool[0], s["back"][0], s["back"][1], s["slots"], s["ints"][1], s["ints"][3], owner_map=c.label[0])

    a, e = sides
    step(e)                                                # nothing to do yet; the context's scratch
    gc.collect()                                           # no other graph may be destroyed while this one is captured
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(a)
    have = np.zeros(3, np.int32)
    for k in range(6):
        grow = np.array([group_rows, max(1, group_rows - k), 0 if k % 2 else 1], np.int32)
        for s in (a, e):
            s["qkv"].copy_(torch.randn(s["qkv"].shape, generator=torch.Generator().manual_seed(k)))
            s["have"].copy_(dev(have))
            s["want"].copy_(dev(have + grow))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.synchronize()
        step(e)
        torch.cuda.synchronize()
        for name in ("slots", "ints", "q", "out", "back", "st"):
            assert torch.equal(a[name], e[name]), (k, name)
        assert torch.equal(a["c"].pool[0], e["c"].pool[0]) and not a["st"].any() and a["out"][: int(grow.sum())].isfinite().all()
        have = have + grow
    ctx.close()
