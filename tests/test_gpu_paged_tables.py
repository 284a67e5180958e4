"""Block tables, slot maps, segment tables and K/V appends on the GPU against the oracle, and a serving
step that runs them together with the segment cipher."""
import numpy as np
import pytest
import torch

from oracle import paged as P
from paper_2608_25431_b200 import binding, workloads as W

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Ctx(64)
    yield c
    c.close()


def dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def u32(t):
    return t.cpu().numpy().astype(np.uint32)


def state(rng, n, pt, hi, layers=3, spare=10, shrink=0.3, grow=40):
    """A consistent random step: lengths, tables, free stack, labels."""
    have = rng.integers(0, hi + 1, size=n).astype(np.int32)
    want = np.where(rng.random(n) < shrink, (have * rng.random(n)).astype(np.int32), have + rng.integers(0, grow + 1, size=n)).astype(np.int32)
    owner = rng.integers(0, 50, size=n).astype(np.int32)
    width = int(max(1, (-(-np.maximum(have, want) // pt)).max()))
    held = -(-have // pt)
    pages = int(held.sum()) + int(np.maximum(0, -(-want // pt) - held).sum()) + spare
    perm = rng.permutation(pages).astype(np.int32)
    table = np.full((n, width), -1, dtype=np.int32)
    label = np.full((layers, pages), P.NONE, dtype=np.int32)
    at = 0
    for r in range(n):
        table[r, : held[r]] = perm[at: at + held[r]]
        label[:, table[r, : held[r]]] = owner[r]
        at += int(held[r])
    free = np.full(pages + 3, -7, dtype=np.int32)
    free[: pages - at] = perm[at:]
    return owner, have, want, table, free, pages - at, label, pages


def run_tables(ctx, s, pt):
    owner, have, want, table, free, n_free, label, pages = s
    t, f, n, l = dev(table), dev(free), dev(np.array([n_free])), dev(label)
    st = torch.full((len(owner),), 0x55, dtype=torch.int32, device="cuda")
    b = binding.Batch(dev(owner), dev(have), dev(want), t, pt, pages)
    ctx.block_tables(b, f, n, l, st, layers=label.shape[0])
    torch.cuda.synchronize()
    return t.cpu().numpy(), f.cpu().numpy(), int(n.item()), l.cpu().numpy(), u32(st)


def same_tables(got, want):
    t, f, n, l, st = want
    assert np.array_equal(got[4], st)
    assert got[2] == n and np.array_equal(got[0], t) and np.array_equal(got[3], l)
    assert np.array_equal(got[1][:n], f[:n])                 # above its height the stack holds nothing
    return True


@pytest.mark.parametrize("n,pt,hi,layers,spare", [(1, 16, 0, 1, 0), (1, 1, 30, 2, 5), (3, 16, 100, 1, 0), (33, 7, 90, 4, 3), (256, 16, 500, 3, 100),
                                                  (700, 16, 60, 2, 50), (1500, 3, 9, 1, 9), (8192, 16, 40, 1, 100)])
@pytest.mark.parametrize("seed", [0, 1])
def test_block_tables_match_the_oracle(ctx, n, pt, hi, layers, spare, seed):
    rng = np.random.default_rng(100 * n + seed)
    s = state(rng, n, pt, hi, layers, spare)
    same_tables(run_tables(ctx, s, pt), P.block_tables(s[0], s[1], s[2], s[3], pt, s[7], s[4], s[5], s[6]))


def test_block_tables_of_one_long_request(ctx):
    rng = np.random.default_rng(4)
    s = list(state(rng, 2, 16, 0, layers=5, shrink=0.0, grow=60000))
    same_tables(run_tables(ctx, s, 16), P.block_tables(s[0], s[1], s[2], s[3], 16, s[7], s[4], s[5], s[6]))


@pytest.mark.parametrize("short", [1, 5, 40, 10 ** 6])
def test_block_tables_serve_in_order_when_pages_run_short(ctx, short):
    rng = np.random.default_rng(short)
    s = list(state(rng, 120, 4, 50, shrink=0.2))
    s[5] = max(0, s[5] - 10 - short)
    same_tables(run_tables(ctx, s, 4), P.block_tables(s[0], s[1], s[2], s[3], 4, s[7], s[4], s[5], s[6]))


@pytest.mark.parametrize("spoil", ["owner", "owner_big", "have", "want", "too_long", "page_high", "page_low", "given_twice", "stack_twice",
                                   "stack_and_table", "foreign", "param", "taken_owned", "other_layer", "none_ok", "height_low", "height_high",
                                   "room"])
def test_block_tables_with_malformed_inputs(ctx, spoil):
    rng = np.random.default_rng(8)
    owner, have, want, table, free, n_free, label, pages = state(rng, 60, 4, 40)
    grows = np.nonzero(-(-want // 4) > -(-have // 4))[0]
    gives = np.nonzero(-(-want // 4) < -(-have // 4))[0]
    r, e = gives[3], (gives[3], -(-have[gives[3]] // 4) - 1)          # an entry that is given back
    if spoil == "owner":
        owner[grows[2]] = -1
    elif spoil == "owner_big":
        owner[grows[2]] = 1 << 20
    elif spoil == "have":
        have[grows[1]] = -5
    elif spoil == "want":
        want[r] = -1
    elif spoil == "too_long":
        want[grows[0]] = 2 ** 31 - 1
    elif spoil == "page_high":
        table[e] = pages
    elif spoil == "page_low":
        table[e] = -1
    elif spoil == "given_twice":
        table[e] = table[gives[4], -(-have[gives[4]] // 4) - 1]
        owner[r] = owner[gives[4]]
        label[:, table[r][table[r] >= 0]] = owner[r]
    elif spoil == "stack_twice":
        free[n_free - 1] = free[n_free - 2]
    elif spoil == "stack_and_table":
        label[:, table[e]] = P.NONE
        free[n_free - 1] = table[e]
    elif spoil == "foreign":
        label[2, table[e]] = owner[r] + 1
    elif spoil == "param":
        label[0, table[e]] = P.PARAM
    elif spoil == "taken_owned":
        label[0, free[n_free - 2]] = 3
    elif spoil == "other_layer":
        label[2, free[n_free - 2]] = P.CONFLICT
    elif spoil == "none_ok":
        label[1, table[e]], label[2, table[e]] = P.NONE, P.CONFLICT      # a failed import: the page may still be given back
    elif spoil == "height_low":
        n_free = -1
    elif spoil == "height_high":
        n_free = len(free) + 1
    elif spoil == "room":
        want[:] = 0
        free = free[: n_free + 2].copy()
    s = (owner, have, want, table, free, n_free, label, pages)
    ref = P.block_tables(owner, have, want, table, 4, pages, free, n_free, label)
    assert (ref[4] == P.BAD_TABLE).all() == (spoil not in ("owner", "owner_big", "have", "want", "too_long", "none_ok"))
    same_tables(run_tables(ctx, s, 4), ref)


@pytest.mark.parametrize("n,pt,hi,extra", [(1, 16, 0, 0), (2, 1, 5, 3), (40, 7, 100, 0), (512, 16, 300, 77), (8192, 16, 20, 1)])
def test_slot_maps_match_the_oracle(ctx, n, pt, hi, extra):
    rng = np.random.default_rng(n)
    owner, have, want, table, _, _, label, pages = state(rng, n, pt, hi)
    full = np.where(table < 0, rng.integers(-1, pages + 1, size=table.shape), table).astype(np.int32)     # some entries out of range
    if n > 30:
        owner[5], have[9], want[11] = -2, -1, 2 ** 31 - 1                                                 # malformed requests
    rows = P.slot_map(owner, have, want, full, pt, pages, 0)["total"] + extra
    for rel in (None, rng.integers(-2, 45, size=rows).astype(np.int32)):
        for n_rows in sorted({rows, max(0, rows - extra - 1)}):
            use = None if rel is None else rel[:n_rows]
            ref = P.slot_map(owner, have, want, full, pt, pages, n_rows, use)
            b = binding.Batch(dev(owner), dev(have), dev(want), dev(full), pt, pages)
            slots = torch.full((n_rows,), 99, dtype=torch.int64, device="cuda")
            ints = torch.full((3, max(1, n_rows)), 99, dtype=torch.int32, device="cuda")
            ptr = torch.full((n + 1,), 99, dtype=torch.int32, device="cuda")
            total = torch.zeros(1, dtype=torch.int64, device="cuda")
            ctx.slot_map(b, slots, row_req=ints[0], row_pos=ints[1], row_owner=ints[2], row_ptr=ptr, total=total,
                         rel=None if use is None else dev(use))
            torch.cuda.synchronize()
            assert int(total.item()) == ref["total"] and np.array_equal(ptr.cpu().numpy(), ref["ptr"])
            assert np.array_equal(slots.cpu().numpy(), ref["slots"])
            got = ints[:, :n_rows].cpu().numpy()
            assert np.array_equal(got[0], ref["req"]) and np.array_equal(got[1], ref["pos"]) and np.array_equal(got[2], ref["owner"])


def test_slot_map_without_optional_outputs_and_without_rows(ctx):
    b = binding.Batch(dev([1]), dev([3]), dev([5]), dev([[4]]), 16, 8)
    slots = torch.zeros(2, dtype=torch.int64, device="cuda")
    ctx.slot_map(b, slots)
    assert slots.tolist() == [67, 68]
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    empty = binding.Batch(none, none, none, torch.zeros((0, 1), dtype=torch.int32, device="cuda"), 16, 8)
    ptr = torch.full((1,), 9, dtype=torch.int32, device="cuda")
    ctx.slot_map(empty, slots, row_ptr=ptr)
    assert slots.tolist() == [-1, -1] and ptr.tolist() == [0]
    with pytest.raises(ValueError):
        ctx.slot_map(b, slots.int())
    with pytest.raises(ValueError):
        ctx.slot_map(b, slots, row_req=ptr)


@pytest.mark.parametrize("n,pt,hi,layers,whole,new", [(1, 16, 0, 1, False, False), (5, 16, 90, 3, True, False), (33, 8, 60, 2, False, True),
                                                      (300, 16, 200, 4, False, False), (8192, 16, 20, 1, True, True)])
def test_segment_tables_match_the_oracle(ctx, n, pt, hi, layers, whole, new):
    rng = np.random.default_rng(n + layers)
    owner, have, want, table, _, _, label, pages = state(rng, n, pt, hi)
    full = np.where(table < 0, rng.integers(-1, pages + 1, size=table.shape), table).astype(np.int32)
    if n > 30:
        owner[5], have[9], want[11] = -2, -1, 2 ** 31 - 1
    serial = rng.integers(-2 ** 31, 2 ** 31, size=n).astype(np.int32)
    args = (owner, have, want, full, pt, pages, serial.view(np.uint32), layers, 112)
    need = P.kv_segments(*args, 0, W.SEG_DTYPE, whole, new)[2]
    for cap in sorted({need, need + 5, max(0, need - 1)}):
        segs, pt_ref, total_ref = P.kv_segments(*args, cap, W.SEG_DTYPE, whole, new)
        b = binding.Batch(dev(owner), dev(have), dev(want), dev(full), pt, pages)
        out = torch.full((cap + 1, 40), 0xEE, dtype=torch.uint8, device="cuda")
        table_out = torch.full((cap,), 77, dtype=torch.int32, device="cuda")
        total = torch.zeros(1, dtype=torch.int64, device="cuda")
        ctx.kv_segments(b, dev(serial), out, table_out, layers, 112, whole_pages=whole, new_blocks=new, total=total)
        torch.cuda.synchronize()
        got = out.cpu().numpy()
        assert int(total.item()) == total_ref == need
        assert np.array_equal(got[:cap].reshape(-1), segs.view(np.uint8).reshape(-1))
        assert np.array_equal(table_out.cpu().numpy(), pt_ref) and (got[cap] == 0xEE).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,dim,pt,rows", [(32, 128, 16, 37), (1, 8, 1, 1), (5, 64, 7, 300), (3, 24, 16, 1000), (8, 128, 64, 5), (40, 128, 16, 9)])
@pytest.mark.parametrize("labels", [True, False])
def test_appends_match_the_oracle(ctx, dtype, heads, dim, pt, rows, labels):
    rng = np.random.default_rng(rows + heads)
    pages = -(-rows // pt) + 6
    pool = torch.randn((pages, pt, 2, heads, dim), device="cuda").to(dtype)
    before = pool.clone()
    qkv = torch.randn((rows, 3 * heads + 1, dim + 8), device="cuda").to(dtype)[:, :, :dim]      # strided rows and heads
    k, v = qkv[:, heads:2 * heads], qkv[:, 2 * heads:3 * heads]
    slots = rng.permutation(pages * pt)[:rows].astype(np.int64)
    label = rng.choice([3, 3, 3, 4, P.PARAM, P.NONE, P.CONFLICT], size=pages).astype(np.int32)
    who = rng.choice([3, 4, P.PARAM], size=rows, p=[0.8, 0.1, 0.1]).astype(np.int32)
    for bad in (-1, -2, pages * pt, 2 ** 40, -2 ** 40):
        if rows > 30:
            slots[int(rng.integers(rows))] = bad
    st_ref, wrote = P.append_status(slots, who, label if labels else None, pages, pt)
    st = torch.full((rows,), 55, dtype=torch.int32, device="cuda")
    ctx.kv_append(pool, k, v, dev(slots, torch.int64), dev(who) if labels else None, st, owner_map=dev(label) if labels else None)
    torch.cuda.synchronize()
    assert np.array_equal(u32(st), st_ref)
    flat = before.view(pages * pt, 2, heads, dim)
    for t in np.nonzero(wrote)[0]:
        flat[int(slots[t]), 0] = k[t]
        flat[int(slots[t]), 1] = v[t]
    assert torch.equal(pool.view(torch.int16), before.view(torch.int16))


def test_append_of_one_head_and_broadcast_rows(ctx):
    pool = torch.zeros((4, 4, 2, 1, 64), dtype=torch.float16, device="cuda")
    k = torch.randn((1, 1, 64), device="cuda").half().expand(8, 1, 64)
    st = torch.zeros(8, dtype=torch.int32, device="cuda")
    ctx.kv_append(pool, k, -k[:1].expand(8, 1, 64), torch.arange(8, device="cuda"), None, st)
    assert torch.equal(pool.view(16, 2, 64)[:8, 0], k[:, 0]) and torch.equal(pool.view(16, 2, 64)[:8, 1], -k[:, 0])
    assert not pool.view(16, 2, 64)[8:].any() and not st.any()
    with pytest.raises(ValueError):
        ctx.kv_append(pool, k.float(), k, torch.arange(8, device="cuda"), None, st)
    with pytest.raises(ValueError):
        ctx.kv_append(pool, k, k[:7], torch.arange(8, device="cuda"), None, st)
    with pytest.raises(binding.GiftError):
        ctx.kv_append(pool, torch.zeros((8, 1, 65), dtype=torch.float16, device="cuda")[:, :, 1:], k, torch.arange(8, device="cuda"), None, st)


def test_appends_past_four_gib(ctx):
    # a pool of 5 GiB: the last slots lie past 32-bit byte and element offsets
    pages, pt, heads, dim = 20480, 16, 32, 128
    pool = torch.empty((pages, pt, 2, heads, dim), dtype=torch.bfloat16, device="cuda")
    rows = 64
    pool[-4:].zero_()
    pool[:1].zero_()
    k = torch.randn((rows, heads, dim), device="cuda").bfloat16()
    slots = torch.arange(pages * pt - rows, pages * pt, device="cuda")
    st = torch.zeros(rows, dtype=torch.int32, device="cuda")
    ctx.kv_append(pool, k, -k, slots, None, st)
    got = pool[-4:].view(rows, 2, heads, dim)
    assert torch.equal(got[:, 0], k) and torch.equal(got[:, 1], -k) and not pool[:1].any()


def test_block_tables_without_a_stack(ctx):
    # nothing free and no room: what needs nothing is left alone, what needs a page is told so
    label = torch.full((1, 4), 1, dtype=torch.int32, device="cuda")
    t, st = dev([[0, 1], [2, -1]]), torch.full((2,), 9, dtype=torch.int32, device="cuda")
    n_free = torch.zeros(1, dtype=torch.int32, device="cuda")
    b = binding.Batch(dev([1, 1]), dev([8, 4]), dev([8, 5]), t, 4, 4)
    ctx.block_tables(b, torch.zeros(0, dtype=torch.int32, device="cuda"), n_free, label, st)
    assert st.tolist() == [0, P.NO_BLOCKS] and t.tolist() == [[0, 1], [2, -1]] and (label == 1).all()


def test_entries_behind_the_last_segment_are_refused_by_the_cipher(ctx):
    ctx.set_keys(np.arange(4, dtype=np.int32), np.arange(64, dtype=np.uint8))
    b = binding.Batch(dev([1, 2]), dev([0, 0]), dev([3, 2]), dev([[1, 0], [3, -1]]), 2, 4)
    segs, table = torch.zeros((6, 40), dtype=torch.uint8, device="cuda"), torch.zeros(6, dtype=torch.int32, device="cuda")
    ctx.kv_segments(b, dev([7, 8]), segs, table, 1, 64)
    buf = torch.arange(512, device="cuda").to(torch.uint8)
    out = torch.zeros_like(buf)
    tags, st = torch.ones((6, 16), dtype=torch.uint8, device="cuda"), torch.zeros(6, dtype=torch.int32, device="cuda")
    ctx.seg_encrypt(buf, out, segs, 6, tags, st, page_table=table, page_bytes=128, owner_map=dev([1, 1, P.NONE, 2]), unit_bytes=128)
    assert st.tolist() == [0, 0, 0] + [binding.ST_BAD_DESC] * 3 and not tags[3:].any()
    assert not out[64:128].any() and not out[256:384].any()            # the part of a page that holds no token, an unused page
    assert out[:64].any() and out[128:256].any() and out[384:].any()
