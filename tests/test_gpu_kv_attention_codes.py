"""Attention over 8-bit pages against the 64-bit oracle, within the bounds of codes_bounds, under all its kernels: up to 8 query rows
per K/V head, up to 16 (warp-level products), more (tcgen05 products)."""
import numpy as np
import pytest
import torch

import codes_bounds as B
from oracle import paged as P, paged8 as E
from paper_2608_25431_b200 import binding

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16
ROWS = [1, 2, 5]                       # query rows of a K/V head are these times the group below: all kernels are met


@pytest.fixture(scope="module")
def ctx():
    c = binding.Ctx(64)
    yield c
    c.close()


def dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def call(ctx, x, scale=None, labels=True, extra=0, stream=None, **near):
    heads, dim = x["q"].shape[1:]
    n = x["rows"] + extra
    all_q = torch.zeros((n, heads + 3, dim + 8), dtype=x["q"].dtype)
    all_q[: x["rows"], 2:2 + heads, :dim] = x["q"]
    all_q[x["rows"]:] = float("nan")
    q = all_q.cuda()[:, 2:2 + heads, :dim]
    mask = None
    if x["mask"] is not None:
        mask = torch.cat([torch.from_numpy(x["mask"].view(np.int32)), torch.zeros((extra, x["mask"].shape[1]), dtype=torch.int32)]).cuda()
    out = torch.full((n, heads + 1, dim + 8), 7.0, dtype=x["q"].dtype, device="cuda")
    lse, who = torch.full((n, heads), 7.0, device="cuda"), torch.full((n,), 7, dtype=torch.int32, device="cuda")
    st = torch.full((len(x["owner"]),), 7, dtype=torch.int32, device="cuda")
    b = binding.Batch(dev(x["owner"]), dev(x["have"]), dev(x["want"]), dev(x["table"]), x["pt"], x["pool"].shape[0])
    if near.get("slopes") is not None:
        near = dict(near, slopes=torch.from_numpy(near["slopes"]).cuda())
    ctx.kv_attention_codes(b, torch.from_numpy(x["pool"]).cuda(), x["heads"], q, out[:, :heads, :dim], st, tree_mask=mask, lse=lse, row_owner=who,
                           owner_map=dev(x["label"]) if labels else None, scale=scale, stream=stream, **near)
    torch.cuda.synchronize()
    assert (out[:, heads:] == 7).all() and (out[:, :, dim:] == 7).all()
    return out[:, :heads, :dim].double().cpu().numpy(), lse.double().cpu().numpy(), who.cpu().numpy(), st.cpu().numpy().astype(np.uint32)


def check(ctx, x, scale=None, labels=True, extra=0, **near):
    """Every request served: within the bounds, and nothing else touched."""
    out, lse, who, st = call(ctx, x, scale, labels, extra, **near)
    n, d = x["rows"], x["q"].shape[2]
    b = B.bounds(x, float(np.float32(d ** -0.5 if scale is None else scale)), near.get("softcap", 0.0), near.get("window", 0), near.get("slopes"))
    assert not st.any()
    grows = np.repeat(x["owner"], np.maximum(0, x["want"] - x["have"]))
    assert np.array_equal(who[:n], grows) and (who[n:] == 7).all() and (out[n:] == 7).all() and (lse[n:] == 7).all()
    assert B.worst(out[:n], b["out"], b["out_tol"]) <= 1
    none = np.isinf(b["lse"])
    assert np.array_equal(lse[:n] == -np.inf, none) and (out[:n][none] == 0).all()
    assert B.worst(np.where(none, 0, lse[:n]), np.where(none, 0, b["lse"]), b["lse_tol"]) <= 1


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("pt", [1, 3, 8, 16, 24, 64, 100])
@pytest.mark.parametrize("group, new", [(1, 1), (4, 1), (5, 3), (8, 5), (2, 70)])
def test_pages_groups_rows(ctx, dtype, dim, pt, group, new):
    check(ctx, B.step(pt + new, dtype, [0, 1, 63, 150], [new, new, 1, new], 2, group, dim, pt))


@pytest.mark.parametrize("heads", [1, 3, 4, 8, 12])
@pytest.mark.parametrize("new", [1, 12, 20])
def test_numbers_of_heads(ctx, heads, new):
    check(ctx, B.step(heads, HF, [40, 7, 200], [new] * 3, heads, 1, 128, 16))


@pytest.mark.parametrize("new", [1, 9, 33])
@pytest.mark.parametrize("have", [15, 16, 17, 31, 32, 63, 64, 65, 127, 128, 129, 255, 256, 511])
def test_lengths_around_steps_and_tiles(ctx, have, new):
    check(ctx, B.step(have, BF, [have], [new], 1, 1, 128, 16))
    check(ctx, B.step(have, HF, [have], [new], 2, 1, 64, 16))


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("group, new", [(1, 4), (4, 4), (2, 40), (1, 65)])
def test_trees(ctx, dim, group, new):
    check(ctx, B.step(new, BF, [0, 30, 100], [new, 1, new], 2, group, dim, 16, tree=True))
    check(ctx, B.step(new, HF, [0, 30, 100], [new, 2, 1], 1, group, dim, 8, tree=True), softcap=3.0)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim, pt", [(64, 16), (128, 16), (128, 3), (64, 24)])
@pytest.mark.parametrize("group, new", [(1, 1), (4, 3), (4, 30)])
@pytest.mark.parametrize("window, softcap, sloped", [(0, 20.0, False), (1, 0.0, False), (17, 0.0, True), (64, 5.0, False), (100, 1.0, True), (0, 0.0, True), (1 << 30, 0.0, False)])
def test_capped_biased_windowed(ctx, dtype, dim, pt, group, new, window, softcap, sloped):
    slopes = np.array([2.0 ** -(h + 1) for h in range(2 * group)], np.float32) if sloped else None
    check(ctx, B.step(window % 97 + new, dtype, [0, 300, 70], [new, new, 1], 2, group, dim, pt), window=window, softcap=softcap, slopes=slopes)


@pytest.mark.parametrize("new", [1, 3, 30])
def test_long_contexts_cut_over_many_ctas(ctx, new):
    """Few items, many slices: every item is joined of many pieces; the same call gives the same bits."""
    x = B.step(4, BF, [9000, 3], [new, 1], 1, 4, 128, 16)
    check(ctx, x)
    first, again = call(ctx, x), call(ctx, x)
    assert all(np.array_equal(a, b) for a, b in zip(first, again))
    x = B.step(5, HF, [5000] * 3, [new] * 3, 8, 1, 64, 16)
    check(ctx, x, window=1500)


def test_many_requests(ctx):
    """More items than slices, none of whose heads share a CTA, and requests that do not grow."""
    rng = np.random.default_rng(1)
    have, new = rng.integers(0, 40, 59), rng.integers(0, 3, 59)
    check(ctx, B.step(6, HF, have, new, 8, 2, 64, 8))
    check(ctx, B.step(7, BF, have, new * 9, 2, 2, 128, 16))


@pytest.mark.parametrize("new", [1, 14, 30])
@pytest.mark.parametrize("scale", [0.0, -0.3, 3.0, 1e-30])
def test_scales(ctx, scale, new):
    x = B.step(8, BF, [50, 0], [new, new], 2, 1, 64, 16)
    check(ctx, x, scale=scale)
    check(ctx, x, scale=scale, softcap=2.0)


@pytest.mark.parametrize("new", [1, 14, 30])
def test_rows_that_see_nothing(ctx, new):
    x = B.step(9, BF, [0, 20], [new, new], 2, 1, 64, 16, tree=True)
    x["mask"][0] = 0                                       # no cached token, not itself either
    x["mask"][new] = 0                                     # the cached tokens alone
    check(ctx, x)


@pytest.mark.parametrize("new", [1, 5, 14, 30])
def test_rows_behind_the_last_are_left(ctx, new):
    check(ctx, B.step(10, HF, [20, 5], [new, 0], 2, 1, 128, 16), extra=3)
    x = B.step(11, HF, [20, 5], [new, 2], 2, 1, 128, 16)
    x["rows"] -= 1
    x["q"] = x["q"][:-1]
    out, lse, who, st = call(ctx, x)
    assert (st == P.BAD_TABLE).all() and (out == 7).all() and (lse == 7).all() and (who == 7).all()


def test_without_labels_and_optional_arrays(ctx):
    x = B.step(12, BF, [20, 5], [2, 2], 2, 1, 64, 16)
    x["label"][:] = P.CONFLICT
    check(ctx, x, labels=False)
    q = x["q"].cuda()
    out, st = torch.empty_like(q), torch.ones(2, dtype=torch.int32, device="cuda")
    b = binding.Batch(dev(x["owner"]), dev(x["have"]), dev(x["want"]), dev(x["table"]), 16, x["pool"].shape[0])
    ctx.kv_attention_codes(b, torch.from_numpy(x["pool"]).cuda(), 2, q, out, st)
    assert not st.any() and np.array_equal(out.double().cpu().numpy(), call(ctx, x, labels=False)[0])


@pytest.mark.parametrize("pt", [2, 16])
@pytest.mark.parametrize("new", [1, 14, 30])
def test_pages_of_others(ctx, new, pt):
    """Requests with a foreign, an unowned, a conflicting, a missing and a far page, a parameter's page, a malformed one: each its own status."""
    x = B.step(13, BF, [70] * 8, [new] * 8, 2, 1, 64, pt)
    at = 33 // pt
    x["label"][x["table"][0, at]] = 59
    x["label"][x["table"][1, at]] = P.NONE
    x["label"][x["table"][2, 0]], x["label"][x["table"][2, at]] = 59, P.CONFLICT
    x["table"][3, at] = -1
    x["table"][4, -(-int(x["want"][4]) // pt) - 1] = 1 << 30
    x["label"][x["table"][5, at]] = P.PARAM
    x["want"][6] = x["table"].shape[1] * pt + 1
    x["owner"][6] = 3
    x["rows"], keep = 7 * new, np.r_[0:6 * new, 7 * new:8 * new]
    x["q"] = x["q"][keep]
    out, lse, who, st = call(ctx, x)
    r = E.attention(x["owner"], x["have"], x["want"], x["table"], x["pool"], 2, x["q"].double().numpy(), 64 ** -0.5, None, x["label"])
    assert np.array_equal(st, r["status"]) and np.array_equal(who, r["row_owner"])
    assert st.tolist() == [P.OWNER_MISMATCH, P.UNOWNED, P.OWNER_MISMATCH | P.UNOWNED, P.BAD_DESC, P.BAD_DESC, 0, P.BAD_DESC, 0]
    refused = who == P.CONFLICT
    assert (out[refused] == 0).all() and (lse[refused] == -np.inf).all() and np.allclose(out[~refused], r["out"][~refused], rtol=0.02, atol=0.02)


@pytest.mark.parametrize("pt", [2, 16])
@pytest.mark.parametrize("new", [1, 14, 30])
def test_pages_behind_the_window_are_another_matter(ctx, new, pt):
    x = B.step(14, HF, [200, 200], [new, new], 2, 1, 64, pt)
    low = 200 - 50 + 1
    x["label"][x["table"][0, : low // pt]] = 59            # nobody sees a token of these
    x["table"][1, : low // pt - 1] = -1
    x["label"][x["table"][1, low // pt]] = 59              # a row sees the last tokens of this one
    out, lse, who, st = call(ctx, x, window=50)
    assert st.tolist() == [0, P.OWNER_MISMATCH] and (out[new:] == 0).all()
    y = dict(x, owner=x["owner"][:1], have=x["have"][:1], want=x["want"][:1], table=x["table"][:1], q=x["q"][:new], rows=new, label=x["label"])
    check(ctx, y, window=50)


@pytest.mark.parametrize("new", [3, 14, 30])
@pytest.mark.parametrize("dim", [64, 128])
def test_what_hidden_tokens_hold_does_not_matter(ctx, new, dim):
    """Codes of NaN, scales that are NaN, infinite or huge, in tokens that a mask or a window hides, and behind the context."""
    x = B.step(15, BF, [60, 33], [new, new], 2, 1, dim, 16, tree=True)
    rng = np.random.default_rng(0)
    bad = {int(p) for p in range(x["pool"].shape[0])}
    flat = x["pool"].reshape(-1, x["pool"].shape[-1])
    used = {int(x["table"][r, t // 16]) * 16 + t % 16 for r in range(2) for t in range(int(x["want"][r]))}
    hide = []
    for r in range(2):
        victim = int(x["have"][r]) + 1                     # step token 1: seen by nobody
        x["mask"][r * new:(r + 1) * new, 0] &= ~np.uint32(2)
        hide.append(int(x["table"][r, victim // 16]) * 16 + victim % 16)
    want = call(ctx, x)
    for k, s in enumerate([s for s in range(flat.shape[0]) if s not in used] + hide):
        m = 2 * 2 * dim
        flat[s, :m] = rng.integers(0, 256, m)
        flat[s, : m : 7] = 0x7F
        flat[s, m:m + 16] = np.frombuffer(np.array([np.nan, np.inf, 1e38, -np.inf] if k % 2 else [1e30, 1e38, np.nan, np.nan], "<f4").tobytes(), np.uint8)
    assert bad and all(np.array_equal(a, b) for a, b in zip(call(ctx, x), want))


@pytest.mark.parametrize("new", [1, 14, 30])
def test_what_seen_tokens_hold_does(ctx, new):
    """A NaN scale of K or V, or a code of NaN, in a token that a row sees makes its head NaN, and no other."""
    for kind in range(4):
        x = B.step(16, HF, [40], [new], 3, 1, 64, 16)
        t = 5 if kind < 3 else 40                          # the last kind in the step's own tokens
        token = x["pool"][x["table"][0, t // 16], t % 16]
        m = 2 * 3 * 64
        if kind < 2:
            token[m + 8 + 4 * kind: m + 12 + 4 * kind] = np.frombuffer(np.float32(np.nan).tobytes(), np.uint8)
        else:
            token[3 * 64 + 64 + 9] = 0x7F                  # V of head 1
        out = call(ctx, x)[0]
        nan = np.isnan(out)
        assert not nan[:, [0, 2]].any()
        assert nan[:, 1].all() if kind < 2 else nan[:, 1, 9].all()


@pytest.mark.parametrize("new", [1, 14, 30])
def test_tokens_of_very_different_size(ctx, new):
    """V's scales over 60 powers of two, with the weight on small ones; queries and keys far from one."""
    x = B.step(17, BF, [90], [new], 2, 1, 64, 16)
    rng = np.random.default_rng(2)
    flat = x["pool"].reshape(-1, x["pool"].shape[-1])
    m = 2 * 2 * 64
    scales = np.ascontiguousarray(flat[:, m:m + 16]).view("<f4").reshape(-1, 2, 2).copy()
    scales[..., 1] *= 2.0 ** rng.integers(-30, 30, scales[..., 1].shape)
    scales[..., 0] *= 2.0 ** 40
    flat[:, m:m + 16] = scales.astype("<f4").reshape(-1, 4).view(np.uint8).reshape(-1, 16)
    x["q"] = (x["q"].double() * 2.0 ** -38).to(BF)
    check(ctx, x)
    x["q"] *= 1e-6                                         # all scores alike: the largest V decides
    check(ctx, x)


def test_streams_and_two_contexts_at_once(ctx):
    other = binding.Ctx(8)
    a, b = B.step(18, BF, [3000, 10], [1, 1], 2, 1, 128, 16), B.step(19, BF, [2000, 10], [30, 1], 2, 1, 128, 16)
    want = call(ctx, a), call(ctx, b)
    for c in (ctx, other):
        call(c, a)                                         # the scratch, before anything runs at once
    s = [torch.cuda.Stream(), torch.cuda.Stream()]
    sides = []
    for c, x, st in ((ctx, a, s[0]), (other, b, s[1])):
        q = x["q"].cuda()
        sides.append(dict(c=c, stream=st, q=q, out=torch.zeros_like(q), st=torch.ones(2, dtype=torch.int32, device="cuda"), pool=torch.from_numpy(x["pool"]).cuda(), label=dev(x["label"]),
                          b=binding.Batch(dev(x["owner"]), dev(x["have"]), dev(x["want"]), dev(x["table"]), 16, x["pool"].shape[0])))
    torch.cuda.synchronize()
    for _ in range(20):
        for y in sides:
            y["c"].kv_attention_codes(y["b"], y["pool"], 2, y["q"], y["out"], y["st"], owner_map=y["label"], stream=y["stream"].cuda_stream)
    torch.cuda.synchronize()
    for y, w in zip(sides, want):
        assert not y["st"].any() and np.array_equal(y["out"].double().cpu().numpy(), w[0])
    other.close()


def test_first_call_under_a_capture_is_refused():
    c = binding.Ctx(8)
    x = B.step(20, BF, [30], [1], 1, 1, 64, 16)
    q = x["q"].cuda()
    out, st, pool = torch.zeros_like(q), torch.ones(1, dtype=torch.int32, device="cuda"), torch.from_numpy(x["pool"]).cuda()
    b = binding.Batch(dev(x["owner"]), dev(x["have"]), dev(x["want"]), dev(x["table"]), 16, x["pool"].shape[0])
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        with torch.cuda.graph(g, stream=s):
            with pytest.raises(binding.GiftError) as e:
                c.kv_attention_codes(b, pool, 1, q, out, st, stream=s.cuda_stream)
            out.zero_()
    assert e.value.code == binding.E_INVAL
    g.reset()                                              # here and now, not in some later capture
    c.kv_attention_codes(b, pool, 1, q, out, st)
    torch.cuda.synchronize()
    assert not st.any()
    c.close()


@pytest.mark.parametrize("ns", [1, 1000, 20000])
def test_waits_that_run_out(ctx, ns):
    """Under short limits a request is right to the bit or zero and STALLED; then all is as before."""
    x = B.step(21, BF, [700, 90, 2000], [30, 40, 35], 2, 2, 128, 16)
    want = call(ctx, x)
    ctx.wait_limit(ns)
    try:
        for _ in range(3):
            out, lse, who, st = call(ctx, x)
            t = 0
            for r in range(3):
                m = int(x["want"][r] - x["have"][r])
                at = slice(t, t + m)
                if st[r] == binding.ST_STALLED:
                    assert (out[at] == 0).all() and (lse[at] == -np.inf).all() and (who[at] == P.CONFLICT).all()
                else:
                    assert st[r] == 0 and all(np.array_equal(a[at], b[at]) for a, b in zip((out, lse, who), want))
                t += m
    finally:
        ctx.wait_limit(0)
    assert all(np.array_equal(a, b) for a, b in zip(call(ctx, x), want))


def test_cache_past_4_gib(ctx):
    heads, dim, pt = 32, 128, 16
    pages = 2 ** 32 // (pt * binding.kv8_token_bytes(heads, dim)) + 300
    x = B.step(22, BF, [150, 90], [1, 20], heads, 1, dim, pt)
    pool = torch.zeros((pages, pt, binding.kv8_token_bytes(heads, dim)), dtype=torch.uint8, device="cuda")
    small = x["pool"].shape[0]
    pool[pages - small:] = torch.from_numpy(x["pool"]).cuda()
    for r in ([0], [1]):
        y = dict(x, owner=x["owner"][r], have=x["have"][r], want=x["want"][r], table=x["table"][r], q=x["q"][:1] if r == [0] else x["q"][1:])
        y["rows"] = y["q"].shape[0]
        want = call(ctx, y, labels=False)[0]
        q = y["q"].cuda()
        out, st = torch.zeros_like(q), torch.ones(1, dtype=torch.int32, device="cuda")
        b = binding.Batch(dev(y["owner"]), dev(y["have"]), dev(y["want"]), dev(np.where(y["table"] >= 0, y["table"] + pages - small, -1)), pt, pages)
        ctx.kv_attention_codes(b, pool, heads, q, out, st)
        assert not st.any() and np.array_equal(out.double().cpu().numpy(), want)


@pytest.mark.parametrize("heads", [1, 2, 3, 4])
@pytest.mark.parametrize("window", [0, 90])
def test_prompts_of_several_tiles_of_rows(ctx, heads, window):
    """One, two, three and four tiles of 128 rows to a head, alone and among each other: odd last tiles share their tokens with the next head's."""
    check(ctx, B.step(30 + heads, HF, [0, 70, 3, 130], [260, 300, 129, 400], heads, 1, 64, 16), window=window)
    check(ctx, B.step(40 + heads, BF, [0, 200, 9], [65, 20, 97], heads, 4, 128, 24), window=window)
    check(ctx, B.step(50 + heads, BF, [5], [130], heads, 5, 64, 4), window=window)


def test_trees_of_several_tiles_of_rows(ctx):
    check(ctx, B.step(60, HF, [40, 0], [140, 50], 3, 2, 64, 16, tree=True))


@pytest.mark.parametrize("pt", [4, 16])
def test_a_prompt_is_refused_as_a_whole(ctx, pt):
    """A bad page that only the last rows see, or, under a window, only the first ones: no row of the request comes out."""
    for have, window, page in ((0, 0, -1), (300, 100, 201 // pt)):
        x = B.step(61, BF, [have, 20], [300, 300], 2, 1, 64, pt)
        last = -(-int(x["want"][0]) // pt) - 1
        x["label"][x["table"][0, last if page < 0 else page]] = 59
        out, lse, who, st = call(ctx, x, window=window)
        assert st.tolist() == [P.OWNER_MISMATCH, 0] and (out[:300] == 0).all() and (lse[:300] == -np.inf).all() and (who[:300] == P.CONFLICT).all()
        assert np.abs(out[300:]).min(axis=(1, 2)).max() > 0 and (who[300:] == x["owner"][1]).all()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new", [1, 3])
def test_more_heads_to_a_group_than_a_tile_has_rows(ctx, dim, new):
    check(ctx, B.step(31, BF, [70, 0, 300], [new, new, new], 1, 160, dim, 16))


@pytest.mark.parametrize("new", [1, 6, 20])
@pytest.mark.parametrize("shared", ["rows", "heads", "both"])
def test_rows_of_q_that_share_memory(ctx, new, shared):
    x = B.step(32, HF, [50, 9], [new, new], 2, 2, 64, 16)
    n, heads, dim = x["q"].shape
    base = x["q"][:1] if shared == "rows" else x["q"][:, :1] if shared == "heads" else x["q"][:1, :1]
    x["q"] = base.expand(n, heads, dim)
    q = base.cuda().expand(n, heads, dim)
    out, st = torch.zeros((n, heads, dim), dtype=HF, device="cuda"), torch.ones(2, dtype=torch.int32, device="cuda")
    b = binding.Batch(dev(x["owner"]), dev(x["have"]), dev(x["want"]), dev(x["table"]), 16, x["pool"].shape[0])
    ctx.kv_attention_codes(b, torch.from_numpy(x["pool"]).cuda(), 2, q, out, st, owner_map=dev(x["label"]))
    torch.cuda.synchronize()
    bound = B.bounds(x, float(np.float32(dim ** -0.5)), 0.0, 0, None)
    assert not st.any() and B.worst(out.double().cpu().numpy(), bound["out"], bound["out_tol"]) <= 1


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("new", [2, 14, 30])
def test_rows_of_q_that_are_not_finite(ctx, dtype, new):
    """They are NaN, and their neighbours are as good as ever."""
    x = B.step(33, dtype, [100], [new], 2, 2, 64, 16)
    bound = B.bounds(x, float(np.float32(64 ** -0.5)), 0.0, 0, None)
    x["q"][1, 0, 7], x["q"][0, 3, 9] = float("nan"), float("inf")
    out, lse, _, st = call(ctx, x)
    fine = np.ones(out.shape[:2], bool)
    fine[1, 0] = fine[0, 3] = False
    assert not st.any() and np.isnan(out[~fine]).all() and np.isnan(lse[~fine]).all()
    assert B.worst(out[fine], bound["out"][fine], bound["out_tol"][fine]) <= 1


def test_a_page_twice_in_a_table_and_in_two_requests(ctx):
    """Tables only say where to read: a page may stand for several stretches of a context."""
    for new in (1, 14, 30):
        x = B.step(34, BF, [100, 64], [new, new], 2, 1, 64, 16)
        x["table"][0, 3] = x["table"][0, 1]
        x["label"][x["table"][0, 1]] = P.PARAM
        x["table"][1, 0] = x["table"][0, 1]
        check(ctx, x)
