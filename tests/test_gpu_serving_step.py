"""A serving run through the paged cache, as its calls are meant to follow one another: prefill, a step with a
tree of drafted tokens, its accepted path, a decode step, export under the owners' keys, import, and the same
attention on the other side.  Tables and labels are compared with the oracle, rows with the 64-bit attention,
ciphertext with the segment oracle."""
import numpy as np
import pytest
import torch

from oracle import gcm, paged as P
from paper_2608_25431_b200 import binding, workloads as W

pytestmark = pytest.mark.gpu

LAYERS, PT, HEADS, GROUP, DIM, PAGES = 2, 16, 2, 4, 128, 96
TOKEN = 2 * HEADS * DIM * 2


def dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def np_(t):
    return t.cpu().numpy()


class Cache:
    """One side's pools, labels, tables and free pages."""

    def __init__(self, ctx, owner, seed):
        rng = np.random.default_rng(seed)
        n = len(owner)
        self.ctx, self.owner = ctx, owner
        self.pool = torch.zeros((LAYERS, PAGES, PT, 2, HEADS, DIM), dtype=torch.bfloat16, device="cuda")
        self.label = torch.full((LAYERS, PAGES), P.NONE, dtype=torch.int32, device="cuda")
        self.table = torch.full((n, 20), -1, dtype=torch.int32, device="cuda")
        self.free, self.n_free = dev(rng.permutation(PAGES)), dev([PAGES])
        self.status = torch.zeros(n, dtype=torch.int32, device="cuda")

    def batch(self, have, want):
        return binding.Batch(dev(self.owner), dev(have), dev(want), self.table, PT, PAGES)

    def resize(self, have, want):
        ref = P.block_tables(self.owner, have, want, np_(self.table), PT, PAGES, np_(self.free), int(self.n_free.item()), np_(self.label))
        self.ctx.block_tables(self.batch(have, want), self.free, self.n_free, self.label, self.status, layers=LAYERS)
        assert np.array_equal(np_(self.table), ref[0]) and int(self.n_free.item()) == ref[2]
        assert np.array_equal(np_(self.label), ref[3]) and np.array_equal(np_(self.status).astype(np.uint32), ref[4])

    def append(self, have, want, k, v, rel=None):
        rows = k.shape[1]
        slots = torch.zeros(rows, dtype=torch.int64, device="cuda")
        who = torch.zeros(rows, dtype=torch.int32, device="cuda")
        self.ctx.slot_map(self.batch(have, want), slots, row_owner=who, rel=None if rel is None else dev(rel))
        st = torch.full((rows,), 9, dtype=torch.int32, device="cuda")
        for layer in range(LAYERS):
            self.ctx.kv_append(self.pool[layer], k[layer], v[layer], slots, who, st, owner_map=self.label[layer])
            assert not st.any()
        return slots

    def attend(self, layer, have, want, q, mask=None):
        out = torch.zeros_like(q)
        who = torch.zeros(q.shape[0], dtype=torch.int32, device="cuda")
        st = torch.full((len(self.owner),), 9, dtype=torch.int32, device="cuda")
        self.ctx.kv_attention(self.batch(have, want), self.pool[layer], q, out, st, tree_mask=mask, row_owner=who, owner_map=self.label[layer])
        ref = P.attention(self.owner, have, want, np_(self.table), np_(self.pool[layer].double()), np_(q.double()), float(np.float32(DIM ** -0.5)),
                          None if mask is None else np_(mask).view(np.uint32), np_(self.label[layer]))
        assert np.array_equal(np_(st).astype(np.uint32), ref["status"]) and np.array_equal(np_(who), ref["row_owner"])
        # bf16: the result's and the weights' roundings, 2^-9 each relative to sums of at most max |v|
        vmax = float(self.pool[layer].abs().max())
        assert np.abs(np_(out.double()) - ref["out"]).max() <= 2.0 ** -8 * vmax * 1.1
        return out, who, st


def test_a_run_from_lengths_to_the_other_side():
    rng = np.random.default_rng(77)
    n = 6
    owner = np.array([3, 0, 5, 1, 4, 2], dtype=np.int32)
    ctx = binding.Ctx(8)
    keys = rng.integers(0, 256, size=(8, 16), dtype=np.uint8)
    ctx.set_keys(np.arange(8, dtype=np.int32), keys)
    a = Cache(ctx, owner, 1)

    def rows(t):
        return torch.randn((LAYERS, t, 3 * HEADS, DIM), device="cuda").bfloat16()

    # prefill
    zero, have = np.zeros(n, np.int32), np.array([1, 16, 17, 200, 64, 33], dtype=np.int32)
    a.resize(zero, have)
    kv = rows(int(have.sum()))
    a.append(zero, have, kv[:, :, :HEADS], kv[:, :, HEADS:2 * HEADS])
    q = torch.randn((int(have.sum()), HEADS * GROUP, DIM), device="cuda").bfloat16()
    a.attend(0, zero, have, q)                                            # the prompt's own causal attention

    # a tree of drafted tokens
    new = np.array([5, 8, 1, 7, 0, 30], dtype=np.int32)
    want = have + new
    a.resize(have, want)
    total = int(new.sum())
    kv = rows(total)
    a.append(have, want, kv[:, :, :HEADS], kv[:, :, HEADS:2 * HEADS])
    mask = np.zeros((total, 1), dtype=np.uint32)
    parent, t = np.full(total, -1), 0
    for r in range(n):
        for i in range(new[r]):
            up = int(rng.integers(-1, i)) if i else -1
            parent[t + i] = up
            mask[t + i, 0] = (mask[t + up, 0] if up >= 0 else 0) | np.uint32(1 << i)
        t += int(new[r])
    q = torch.randn((total, HEADS * GROUP, DIM), device="cuda").bfloat16()
    for layer in range(LAYERS):
        a.attend(layer, have, want, q, torch.from_numpy(mask.view(np.int32)).cuda())

    # the path to every request's last drafted token is accepted: its rows move up, the other blocks go back
    rel, accepted, t = np.full(total, -1, dtype=np.int32), np.zeros(n, np.int32), 0
    for r in range(n):
        i, path = int(new[r]) - 1, []
        while i >= 0:
            path.append(i)
            i = int(parent[t + i])
        for k, i in enumerate(reversed(path)):
            rel[t + i] = k
        accepted[r] = len(path)
        t += int(new[r])
    a.append(have, want, kv[:, :, :HEADS], kv[:, :, HEADS:2 * HEADS], rel)
    now = have + accepted
    a.resize(want, now)

    # one decode step
    step = now + 1
    a.resize(now, step)
    kv = rows(n)
    a.append(now, step, kv[:, :, :HEADS], kv[:, :, HEADS:2 * HEADS])
    q = torch.randn((n, HEADS * GROUP, DIM), device="cuda").bfloat16()
    there = [a.attend(layer, now, step, q)[0] for layer in range(LAYERS)]

    # export every block under its owner's key, out of place
    blocks = int((-(-step // PT)).sum())
    segs = torch.zeros((blocks * LAYERS, 40), dtype=torch.uint8, device="cuda")
    page_table = torch.zeros(blocks * LAYERS, dtype=torch.int32, device="cuda")
    serial = np.arange(100, 100 + n, dtype=np.int32)
    ctx.kv_segments(a.batch(now, step), dev(serial), segs, page_table, LAYERS, TOKEN)
    src = a.pool.view(torch.uint8).reshape(-1)
    cipher = torch.zeros_like(src)
    nseg = segs.shape[0]
    tags = torch.zeros((nseg, 16), dtype=torch.uint8, device="cuda")
    st = torch.full((nseg,), 9, dtype=torch.int32, device="cuda")
    ctx.seg_encrypt(src, cipher, segs, nseg, tags, st, page_table=page_table, page_bytes=PT * TOKEN, owner_map=a.label.view(-1),
                    unit_bytes=PT * TOKEN)
    assert not st.any()
    h_segs = np_(segs).reshape(-1).view(W.SEG_DTYPE)
    ref = np.zeros_like(np_(cipher))
    ref_tags, ref_st = gcm.seg_encrypt(np_(src), ref, h_segs, np.arange(8, dtype=np.int32), keys, 8, np_(page_table), PT * TOKEN,
                                       np_(a.label.view(-1)), PT * TOKEN)
    assert np.array_equal(np_(tags), ref_tags) and not ref_st.any() and np.array_equal(np_(cipher), ref)

    # the other side: same page numbers, fresh labels
    b = Cache(ctx, owner, 2)
    b.table.copy_(a.table)
    dst = b.pool.view(torch.uint8).reshape(-1)
    ctx.seg_decrypt(cipher, dst, segs, nseg, tags, st, page_table=page_table, page_bytes=PT * TOKEN, owner_map=b.label.view(-1),
                    unit_bytes=PT * TOKEN)
    assert not st.any() and torch.equal(b.label, a.label)
    for layer in range(LAYERS):
        assert torch.equal(b.attend(layer, now, step, q)[0], there[layer])

    # a tampered block: its pages are nobody's, and its request's rows do not come out
    victim = int(np.nonzero(h_segs["owner"][: blocks] == 1)[0][2])
    tags[victim, 0] ^= 1
    ctx.seg_decrypt(cipher, dst, segs, nseg, tags, st, page_table=page_table, page_bytes=PT * TOKEN, owner_map=b.label.view(-1),
                    unit_bytes=PT * TOKEN)
    assert int(st[victim]) == binding.ST_TAG_MISMATCH
    out, who, st = b.attend(0, now, step, q)
    assert st.tolist() == [0, 0, 0, binding.ST_UNOWNED, 0, 0] and not out[3].any() and int(who[3]) == P.CONFLICT
    # a block table that names another user's page
    b.table[0, 0] = b.table[1, 0]
    _, _, st = b.attend(1, now, step, q)
    assert int(st[0]) == binding.ST_OWNER_MISMATCH and not st[1:].any()
    ctx.close()


def test_a_captured_step_replays_on_new_lengths():
    """slot map, append and attention of a decode step, captured once and replayed as the lengths grow."""
    owner = np.array([1, 2, 3], dtype=np.int32)
    ctx = binding.Ctx(4)
    a, b = Cache(ctx, owner, 3), Cache(ctx, owner, 3)
    have = np.array([15, 30, 2], dtype=np.int32)
    for c in (a, b):
        torch.manual_seed(5)
        c.resize(np.zeros(3, np.int32), have + 20)
        kv = torch.randn((LAYERS, int(have.sum()), 2 * HEADS, DIM), device="cuda").bfloat16()
        c.append(np.zeros(3, np.int32), have, kv[:, :, :HEADS], kv[:, :, HEADS:])
    kv = torch.zeros((3, 2 * HEADS, DIM), dtype=torch.bfloat16, device="cuda")
    q, out = torch.zeros((3, HEADS * GROUP, DIM), dtype=torch.bfloat16, device="cuda"), torch.zeros((3, HEADS * GROUP, DIM), dtype=torch.bfloat16, device="cuda")
    slots, who, st = torch.zeros(3, dtype=torch.int64, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    batch = a.batch(have, have + 1)

    def step(c, bt):
        ctx.slot_map(bt, slots, row_owner=who)
        ctx.kv_append(c.pool[0], kv[:, :HEADS], kv[:, HEADS:], slots, who, st, owner_map=c.label[0])
        ctx.kv_attention(bt, c.pool[0], q, out, st, owner_map=c.label[0])

    step(a, batch)                                        # the first call allocates; repeated below on the same values
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a, batch)
    for k in range(6):
        kv.copy_(torch.randn(kv.shape, device="cuda"))
        q.copy_(torch.randn(q.shape, device="cuda"))
        batch.tensors[1].copy_(dev(have + k))
        batch.tensors[2].copy_(dev(have + k + 1))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        step(b, b.batch(have + k, have + k + 1))
        torch.cuda.synchronize()
        assert torch.equal(got, out) and torch.equal(a.pool[0], b.pool[0]) and not st.any()
    ctx.close()
