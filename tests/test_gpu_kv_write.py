"""Rows into the labelled pages and out of them against the 64-bit oracle; tolerances: tests/codes_bounds.py."""
import numpy as np
import pytest
import torch

import codes_bounds as B
from oracle import paged as P, paged8 as E
from paper_2608_25431_b200 import binding

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    c = binding.Ctx(64)
    yield c
    c.close()


def dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def make(seed, dtype, rows, heads, q_heads, dim, pt, bits, pages=None, norm=True, n_freq=None, axes=1, paired=False, far=0):
    """Rows of one projection (heads of q, k, v next to one another, odd strides), pages all owned by user 5."""
    rng = np.random.default_rng(seed)
    pages = pages or -(-rows // pt) + 2
    x = dict(dtype=dtype, heads=heads, dim=dim, pt=pt, bits=bits, paired=paired, eps=1e-6)
    x["all"] = torch.from_numpy(rng.standard_normal((rows, q_heads + 2 * heads + 1, dim + 8))).to(dtype)
    x["q"], x["k"], x["v"] = (x["all"][:, a:b, :dim] for a, b in ((0, q_heads), (q_heads, q_heads + heads), (q_heads + heads, q_heads + 2 * heads)))
    x["q_norm"], x["k_norm"] = (torch.from_numpy(1 + 0.3 * rng.standard_normal(dim)).to(dtype) if norm else None for _ in range(2))
    n_freq = dim // 2 if n_freq is None else n_freq
    x["freq"] = np.array([1e4 ** (-j / max(1, n_freq)) for j in range(n_freq)], np.float32)
    x["sections"] = [n_freq - (axes - 1) * (n_freq // axes)] + [n_freq // axes] * (axes - 1)
    x["pos"] = (rng.integers(0, 5000, (axes, rows)) + far).astype(np.int32)
    x["slots"] = rng.permutation(pages * pt)[:rows].astype(np.int64)
    x["owner"] = np.full(rows, 5, np.int32)
    x["label"] = np.full(pages, 5, np.int32)
    shape = (pages, pt, binding.kv8_token_bytes(heads, dim)) if bits == 8 else (pages, pt, 2, heads, dim)
    x["pool"] = torch.full(shape, 0x55, dtype=torch.uint8) if bits == 8 else torch.full(shape, 3.0, dtype=dtype)
    return x


def call(ctx, x, with_q=True, labels=True, stream=None):
    """(q_out, pool, status) after the call; what must stay is 7 or as it was."""
    on = {k: x[k].cuda() for k in ("all", "pool")}
    hq, hk, dim = x["q"].shape[1], x["heads"], x["dim"]
    q, k, v = on["all"][:, :hq, :dim], on["all"][:, hq:hq + hk, :dim], on["all"][:, hq + hk:hq + 2 * hk, :dim]
    q_out = torch.full((q.shape[0], hq + 1, dim + 8), 7.0, dtype=x["dtype"], device="cuda")
    st = torch.full((q.shape[0],), 9, dtype=torch.int32, device="cuda")
    turn = len(x["freq"]) > 0
    ctx.kv_write(on["pool"], k, v, dev(x["slots"], torch.int64), dev(x["owner"]), st, q=q if with_q else None, q_out=q_out[:, :hq, :dim] if with_q else None,
                 q_norm=x["q_norm"].cuda() if with_q and x["q_norm"] is not None else None, k_norm=None if x["k_norm"] is None else x["k_norm"].cuda(),
                 eps=x["eps"], pos=dev(x["pos"]) if turn else None, freq=torch.from_numpy(x["freq"]).cuda() if turn else None,
                 sections=x["sections"] if turn else None, paired=x["paired"], owner_map=dev(x["label"]) if labels else None, stream=stream)
    torch.cuda.synchronize()
    assert (q_out[:, hq:] == 7).all() and (q_out[:, :, dim:] == 7).all()
    return q_out[:, :hq, :dim].cpu(), on["pool"].cpu(), st.cpu().numpy().astype(np.uint32)


def norm_error(x, head, weight):
    return (x["dim"] * B.U / 2 + 2.0 ** -21) if weight is not None else 0.0


def expected(x, t, head, weight):
    """One head as it should be written, and how far each element may be off before it is rounded."""
    w = None if weight is None else weight.double().numpy()
    pos = x["pos"][:, t]
    y = E.turned(head, w, x["eps"], pos, x["freq"], x["sections"] if len(x["freq"]) else None, x["paired"])
    plain = E.turned(head, w, x["eps"], None, x["freq"], None, x["paired"])
    err, n, n_freq = norm_error(x, head, weight) * np.abs(plain), norm_error(x, head, weight), len(x["freq"])
    for i in range(n_freq):
        a, b = (2 * i, 2 * i + 1) if x["paired"] else (i, n_freq + i)
        err[a] = err[b] = (abs(plain[a]) + abs(plain[b])) * (n + 2.0 ** -20)
    return y, err


def check(ctx, x, with_q=True, labels=True):
    q_out, pool, st = call(ctx, x, with_q, labels)
    ref_st, good = P.append_status(x["slots"], x["owner"], x["label"] if labels else None, len(x["label"]), x["pt"])
    assert np.array_equal(st, ref_st)
    e, heads, dim, least = B.half_step(x["dtype"]), x["heads"], x["dim"], B.smallest(x["dtype"])
    got_q, q, k, v = (z.double().numpy() for z in (q_out, x["q"], x["k"], x["v"]))
    flat, before = pool.reshape(len(x["label"]) * x["pt"], *pool.shape[2:]), x["pool"].reshape(len(x["label"]) * x["pt"], *pool.shape[2:])
    touched = np.zeros(flat.shape[0], bool)
    for t in range(q.shape[0]):
        if not good[t]:
            assert (got_q[t] == 7).all()
            continue
        slot = int(x["slots"][t])
        touched[slot] = True
        if with_q:
            for h in range(q.shape[1]):
                y, err = expected(x, t, q[t, h], x["q_norm"])
                assert (np.abs(got_q[t, h] - y) <= e * (np.abs(y) + err) + err + least).all(), (t, h)
        if x["bits"] == 8:
            codes, scales, pad = E.unpack(flat[slot].numpy(), heads, dim)
            assert not pad.any()
        for h in range(heads):
            for j, (head, weight) in enumerate(((k[t, h], x["k_norm"]), (v[t, h], None))):
                y, err = expected(x, t, head, weight) if j == 0 else (head, np.zeros(dim))
                if x["bits"] == 16:
                    assert (np.abs(flat[slot, j, h].double().numpy() - y) <= e * (np.abs(y) + err) + err + least * (j == 0)).all()
                    continue
                top = np.abs(y).max()
                s64, d = max(top / 448.0, E.LEAST), err.max() / max(top, E.LEAST)
                assert abs(scales[h, j] - s64) <= s64 * (2.0 ** -22 + d), (t, h, j)
                z = y / s64
                slack = err / s64 + np.abs(z) * (2.0 ** -22 + d)
                assert (np.abs(codes[j, h] - z) <= E.step(np.abs(z) + slack) / 2 + slack).all(), (t, h, j)
    assert torch.equal(flat[~touched], before[~touched])


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim, heads, q_heads, paired, n_freq, axes, norm", [
    (128, 2, 4, False, None, 1, True), (128, 1, 1, True, 48, 3, False), (64, 3, 6, False, 16, 2, True), (64, 5, 5, True, None, 1, True),
    (80, 3, 3, False, 20, 3, True), (80, 1, 4, True, 20, 1, False), (96, 2, 2, False, 24, 1, True), (192, 1, 2, False, 48, 4, True),
    (256, 1, 1, False, None, 1, True), (256, 2, 1, True, 4, 1, True), (16, 3, 7, False, 8, 1, True), (16, 9, 1, True, 4, 2, True), (128, 1, 2, False, 0, 1, True)])
def test_rows(ctx, bits, dtype, dim, heads, q_heads, paired, n_freq, axes, norm):
    check(ctx, make(dim + heads, dtype, 7, heads, q_heads, dim, 4, bits, norm=norm, n_freq=n_freq, axes=axes, paired=paired))


@pytest.mark.parametrize("rows", [1, 2, 33, 300])
@pytest.mark.parametrize("pt", [1, 16, 24])
def test_numbers_of_rows(ctx, rows, pt):
    check(ctx, make(rows, BF, rows, 2, 2, 64, pt, 8))


def test_many_rows_take_a_warp_each(ctx):
    """More rows than the GPU has warps: sampled ones are compared, all of them written."""
    x = make(3, BF, 6000, 3, 2, 64, 16, 8)
    q_out, pool, st = call(ctx, x)
    assert not st.any()
    for t in range(0, 6000, 617):
        y = {k: x[k][t:t + 1] for k in ("all", "q", "k", "v", "slots", "owner")}
        z = dict(x, **y, pos=x["pos"][:, t:t + 1])
        one_q, one_pool, _ = call(ctx, z)
        assert torch.equal(one_q[0], q_out[t])
        s = int(x["slots"][t])
        assert torch.equal(one_pool[s // 16, s % 16], pool[s // 16, s % 16])


def test_k_and_v_alone_and_without_labels(ctx):
    check(ctx, make(5, HF, 9, 2, 2, 128, 8, 8), with_q=False)
    check(ctx, make(6, BF, 9, 2, 2, 128, 8, 8), labels=False)


@pytest.mark.parametrize("far", [-3000, 1 << 20, 2147480000])
def test_far_positions(ctx, far):
    check(ctx, make(8, HF, 6, 1, 2, 64, 4, 16, far=far))


@pytest.mark.parametrize("bits", [8, 16])
def test_refused_and_padded_rows(ctx, bits):
    x = make(9, BF, 12, 2, 2, 64, 4, bits, pages=20)
    x["slots"] = np.array([0, 5, 11, 13, -1, 80, -2, 1 << 40, 79, 17, 21, 25], np.int64)
    x["label"][[1, 2, 3, 4, 5]] = [P.NONE, 9, P.PARAM, P.CONFLICT, 5]
    x["owner"][0], x["owner"][11] = 4, P.PARAM
    check(ctx, x, labels=True)
    st = call(ctx, x)[2]
    assert st.tolist() == [P.OWNER_MISMATCH, P.UNOWNED, P.OWNER_MISMATCH, P.OWNER_MISMATCH, 0, P.BAD_DESC, P.BAD_DESC, P.BAD_DESC, 0, P.UNOWNED, 0, P.OWNER_MISMATCH]


def test_values_that_are_not_finite_or_far_from_one(ctx):
    """An infinity or NaN makes its head NaN, and no other; scales of any size; zeros."""
    x = make(10, BF, 8, 3, 2, 64, 4, 8, norm=False, n_freq=0)
    x["k"][0, 0, 5], x["k"][1, 1, 9], x["v"][2, 2, 63], x["v"][3, 0, 0] = float("inf"), float("nan"), float("-inf"), float("nan")
    x["k"][4, 0] = 0.0
    x["v"][5, 1] *= 2.0 ** 100
    x["k"][6, 2] *= 2.0 ** -120
    q_out, pool, st = call(ctx, x)
    assert not st.any() and torch.equal(q_out, x["q"])
    got = E.values(pool.reshape(-1, pool.shape[-1])[x["slots"]].numpy(), 3, 64)
    nan = np.zeros((8, 2, 3), bool)
    for t, j, h in ((0, 0, 0), (1, 0, 1), (2, 1, 2), (3, 1, 0)):
        nan[t, j, h] = True
    assert np.array_equal(np.isnan(got).all(-1), nan) and np.array_equal(np.isnan(got).any(-1), nan)
    kv = torch.stack([x["k"], x["v"]], 1).double().numpy()
    top = np.abs(kv).max(-1, keepdims=True)
    fine = ~nan
    # half a step of the largest binade is 16 of 448
    assert (np.abs(got - kv)[fine] <= (top * (16 / 448 + 2.0 ** -20) + 448 * 2.0 ** -126)[fine]).all() and (got[4, 0, 0] == 0).all()


def test_norms_of_heads_that_are_not_finite(ctx):
    x = make(11, BF, 4, 2, 2, 64, 4, 8)
    x["k"][0, 0, 3], x["k"][1, 1, 3] = float("inf"), float("nan")
    _, pool, _ = call(ctx, x)
    got = E.values(pool.reshape(-1, pool.shape[-1])[x["slots"]].numpy(), 2, 64)
    assert np.isnan(got[0, 0, 0]).all() and np.isnan(got[1, 0, 1]).all() and np.isnan(got).sum() == 128


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("heads, q_heads, dim", [(1, 1, 128), (3, 5, 64), (2, 2, 256)])
def test_norms_of_heads_of_any_size(ctx, bits, heads, q_heads, dim):
    """Heads of zeros, of numbers whose squares leave 32 bits at either end, next to ordinary ones."""
    x = make(14, BF, 9, heads, q_heads, dim, 4, bits)
    for t, f in enumerate((0.0, 2.0 ** 70, 2.0 ** 120, 2.0 ** -70, 2.0 ** -110, 2.0 ** 62, 2.0 ** -52, 2.0 ** -131)):
        x["k"][t, 0] *= f
        x["q"][t, -1] *= f
    check(ctx, x)
    check(ctx, dict(x, eps=2.0 ** -60))
    x["q"][0, -1] = x["k"][0, 0] = 2.0 ** -60                 # 0 / 0 is another matter
    check(ctx, dict(x, eps=0.0))


def test_q_in_place_and_another_stream(ctx):
    x = make(12, HF, 40, 2, 4, 128, 16, 8)
    want, pool, _ = call(ctx, x)
    s = torch.cuda.Stream()
    on = x["all"].cuda()
    p2, st = x["pool"].cuda(), torch.zeros(40, dtype=torch.int32, device="cuda")
    args = (dev(x["slots"], torch.int64), dev(x["owner"]), st)
    kw = dict(q_norm=x["q_norm"].cuda(), k_norm=x["k_norm"].cuda(), pos=dev(x["pos"][0]), freq=torch.from_numpy(x["freq"]).cuda(), owner_map=dev(x["label"]))
    torch.cuda.synchronize()
    ctx.kv_write(p2, on[:, 4:6, :128], on[:, 6:8, :128], *args, q=on[:, :4, :128], q_out=on[:, :4, :128], stream=s.cuda_stream, **kw)
    s.synchronize()
    assert torch.equal(on[:, :4, :128].cpu(), want) and torch.equal(p2.cpu(), pool) and torch.equal(on[:, 4:].cpu(), x["all"][:, 4:])


# ------------------------------------------------------------------------------------------- reading

@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("heads, dim, pt, rows", [(1, 16, 1, 1), (2, 64, 16, 37), (3, 80, 24, 50), (8, 128, 8, 200), (32, 128, 16, 9), (5, 256, 3, 12), (1, 1024, 4, 5)])
def test_read(ctx, bits, dtype, heads, dim, pt, rows):
    rng = np.random.default_rng(dim + rows)
    pages = -(-rows // pt) + 3
    x = rng.standard_normal((pages, pt, 2, heads, dim)) * np.exp(rng.uniform(-5, 3, (pages, pt, 2, heads, 1)))
    pool = torch.from_numpy(B.pages_of(x)) if bits == 8 else torch.from_numpy(x).to(dtype)
    values = E.values(pool.numpy(), heads, dim) if bits == 8 else pool.double().numpy()
    label, owner = rng.choice([4, 4, 4, 4, 7, P.PARAM, P.NONE, P.CONFLICT], pages).astype(np.int32), np.full(rows, 4, np.int32)
    slots = rng.integers(0, pages * pt, rows)
    if rows > 8:
        slots[[0, 1, 2, 3]] = [-1, -5, pages * pt, 1 << 35]
        slots[5] = slots[6]                                              # the same one twice
    out = torch.full((2, rows, heads + 1, dim + 8), 7.0, dtype=dtype, device="cuda")
    k, v = out[0, :, :heads, :dim], out[1, :, :heads, :dim]
    st = torch.full((rows,), 9, dtype=torch.int32, device="cuda")
    ctx.kv_read(pool.cuda(), k, v, dev(slots, torch.int64), dev(owner), st, owner_map=dev(label))
    torch.cuda.synchronize()
    ref, good = E.read_status(slots, owner, label, pages, pt)
    assert np.array_equal(st.cpu().numpy().astype(np.uint32), ref) and (out[:, :, heads:] == 7).all() and (out[:, :, :, dim:] == 7).all()
    for j, got in enumerate((k, v)):
        got = got.double().cpu().numpy()
        for t in range(rows):
            if slots[t] == -1:
                assert (got[t] == 7).all()
            elif not good[t]:
                assert (got[t] == 0).all()
            else:
                want = values[slots[t] // pt, slots[t] % pt, j]
                tol = (np.abs(want) * (B.half_step(dtype) + 2.0 ** -23) + B.smallest(dtype)) if bits == 8 else 0 * want
                assert (np.abs(got[t] - want) <= tol).all()


def test_written_and_read_back(ctx):
    """Through the pages and back without labels: half a step of the head's largest element at most; NaN heads stay NaN."""
    x = make(20, HF, 64, 4, 4, 128, 16, 8, norm=False, n_freq=0)
    x["k"][7, 2, 1] = float("nan")
    _, pool, _ = call(ctx, x, labels=False)
    k, v = (torch.empty((64, 4, 128), dtype=HF, device="cuda") for _ in range(2))
    st = torch.ones(64, dtype=torch.int32, device="cuda")
    ctx.kv_read(pool.cuda(), k, v, dev(x["slots"], torch.int64), None, st)
    torch.cuda.synchronize()
    assert not st.any()
    for got, want in ((k, x["k"]), (v, x["v"])):
        got, want = got.double().cpu(), want.double()
        nan = torch.isnan(want).any(-1)
        assert torch.isnan(got[nan]).all()
        top = want.abs().amax(-1, keepdim=True)
        assert ((got - want).abs() <= top * (16 / 448 + 2.0 ** -10))[~nan].all()


def test_pages_past_4_gib(ctx):
    """Slots whose bytes lie past 32-bit offsets, written and read."""
    heads, dim, pt = 32, 128, 16
    pages = 2 ** 32 // (pt * binding.kv8_token_bytes(heads, dim)) + 200
    pool = torch.zeros((pages, pt, binding.kv8_token_bytes(heads, dim)), dtype=torch.uint8, device="cuda")
    slots = torch.tensor([3, pages * pt - 1, pages * pt - 17 * pt - 3, pages * pt // 2], device="cuda")
    k, v = (torch.randn((4, heads, dim), device="cuda").to(BF) for _ in range(2))
    st, who = torch.ones(4, dtype=torch.int32, device="cuda"), torch.full((4,), 2, dtype=torch.int32, device="cuda")
    label = torch.full((pages,), 2, dtype=torch.int32, device="cuda")
    ctx.kv_write(pool, k, v, slots, who, st, owner_map=label)
    assert not st.any() and int((pool.view(-1, pool.shape[-1]).amax(-1) > 0).sum()) == 4
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    ctx.kv_read(pool, k2, v2, slots, who, st, owner_map=label)
    for got, want in ((k2, k), (v2, v)):
        assert ((got.double() - want.double()).abs() <= want.double().abs().amax(-1, keepdim=True) * (16 / 448 + 2.0 ** -7)).all()
