"""Attention over the labelled paged cache against the 64-bit oracle.

Tolerances, from the arithmetic alone (e = torch.finfo(type).eps / 2, the largest relative rounding):
the result is rounded once, e |o|; every weight p is rounded to the pool's type for the product with v, and
its exponent carries the score's error s and that of exp2 (2^-20 covers both it and the 32-bit sums' joins):
(e + 2 s + 2^-20 + n 2^-23) A with A = sum p |v| / sum p and n the number of tokens; the score is a
32-bit sum of D exact products, s = scale * D * 2^-23 * max sum |q k|.  fp16 weights below 2^-14 lose up to
2^-25 each: n 2^-25 max |v|; the smallest fp16 step of the result adds 2^-25."""
import numpy as np
import pytest
import torch

from oracle import paged as P
from paper_2608_25431_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = binding.Ctx(64)
    yield c
    c.close()


def dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def make(seed, dtype, have, new, heads, group, dim, pt, tree=True, spare=4, words=None):
    """Inputs of a step: have and new tokens per request; the pages of a request are scattered."""
    rng = np.random.default_rng(seed)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    have, new = np.array(have, dtype=np.int32), np.array(new, dtype=np.int32)
    n, want = len(have), (have + new).astype(np.int32)
    blocks = -(-want // pt)
    pages = int(blocks.sum()) + spare
    perm = rng.permutation(pages).astype(np.int32)
    table = np.full((n, int(max(1, blocks.max()))), -1, dtype=np.int32)
    owner = rng.integers(0, 60, size=n).astype(np.int32)
    label = np.full(pages, P.NONE, dtype=np.int32)
    at = 0
    for r in range(n):
        table[r, : blocks[r]] = perm[at: at + blocks[r]]
        label[table[r, : blocks[r]]] = owner[r]
        at += int(blocks[r])
    rows, most = int(new.sum()), int(new.max())
    pool = torch.randn((pages, pt, 2, heads, dim), generator=g, device="cuda").to(dtype)
    q = torch.randn((rows, heads * group + 3, dim + 8), generator=g, device="cuda").to(dtype)[:, 2:2 + heads * group, :dim]
    mask = None
    if tree:
        words = words or -(-most // 32)
        mask = np.zeros((rows, words), dtype=np.uint32)
        t = 0
        for r in range(n):
            for i in range(new[r]):
                up = int(rng.integers(-1, i)) if i else -1
                if up >= 0:
                    mask[t + i] = mask[t + up]
                mask[t + i, i // 32] |= np.uint32(1 << (i % 32))
            t += int(new[r])
    return dict(owner=owner, have=have, want=want, table=table, pool=pool, q=q, mask=mask, label=label, pt=pt, rows=rows)


def call(ctx, x, scale=None, labels=True, extra=0, out=None, stream=None):
    heads, dim = x["q"].shape[1], x["q"].shape[2]
    n = x["rows"] + extra
    q = x["q"]
    mask = None if x["mask"] is None else torch.from_numpy(x["mask"].view(np.int32)).cuda()
    if extra:
        q = torch.cat([q, q.new_zeros((extra, heads, dim))])
        mask = None if mask is None else torch.cat([mask, mask.new_zeros((extra, mask.shape[1]))])
    if out is None:
        out = torch.full((n, heads + 1, dim + 8), 7.0, dtype=q.dtype, device="cuda")[:, :heads, :dim]
    lse = torch.full((n, heads), 7.0, device="cuda")
    who = torch.full((n,), 7, dtype=torch.int32, device="cuda")
    st = torch.full((len(x["owner"]),), 7, dtype=torch.int32, device="cuda")
    b = binding.Batch(dev(x["owner"]), dev(x["have"]), dev(x["want"]), dev(x["table"]), x["pt"], x["pool"].shape[0])
    ctx.kv_attention(b, x["pool"], q, out, st, tree_mask=mask, lse=lse, row_owner=who, owner_map=dev(x["label"]) if labels else None,
                     scale=scale, stream=stream)
    torch.cuda.synchronize()
    return out, lse, who, st.cpu().numpy().astype(np.uint32)


def check(ctx, x, scale=None, labels=True, extra=0):
    out, lse, who, st = call(ctx, x, scale, labels, extra)
    d = x["q"].shape[2]
    sc = d ** -0.5 if scale is None else scale
    pool, q = x["pool"].double().cpu().numpy(), x["q"].double().cpu().numpy()
    ref = P.attention(x["owner"], x["have"], x["want"], x["table"], pool, q, float(np.float32(sc)), x["mask"], x["label"] if labels else None)
    assert np.array_equal(st, ref["status"])
    n = ref["total"]
    assert np.array_equal(who[:n].cpu().numpy(), ref["row_owner"]) and (who[n:] == 7).all()
    got, gl = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert (got[n:] == 7).all() and (gl[n:] == 7).all()
    mags = P.attention(x["owner"], x["have"], x["want"], x["table"], np.concatenate([pool[:, :, :1], np.abs(pool[:, :, 1:])], 2), q,
                       float(np.float32(sc)), x["mask"], x["label"] if labels else None)["out"]
    e = torch.finfo(x["q"].dtype).eps / 2
    tokens = int(x["want"].max())
    fin = np.abs(np.where(np.isfinite(pool), pool, 0))
    s = abs(sc) * d * 2.0 ** -23 * np.abs(q).max() * d * fin[:, :, 0].max()
    tol = e * np.abs(ref["out"]) + (e + 2 * s + 2.0 ** -20 + tokens * 2.0 ** -23) * mags
    if x["q"].dtype == torch.float16:
        tol = tol + tokens * 2.0 ** -25 * fin[:, :, 1].max() + 2.0 ** -25
    with np.errstate(invalid="ignore"):
        off = np.abs(got[:n] - ref["out"])
        same = (got[:n] == ref["out"]) | (np.isnan(got[:n]) & np.isnan(ref["out"]))
        assert (same | (off <= tol)).all(), (np.nanmax(off / np.maximum(tol, 1e-30)), np.argwhere(~(same | (off <= tol)))[:5])
        loff = np.abs(gl[:n] - ref["lse"])
        lsame = (gl[:n] == ref["lse"]) | (np.isnan(gl[:n]) & np.isnan(ref["lse"]))
        ltol = s + 2.0 ** -20 + tokens * 2.0 ** -24 + np.abs(ref["lse"]) * 2.0 ** -22
        assert (lsame | (loff <= ltol)).all(), np.nanmax(loff / ltol)
    return out, lse


BF, HF = torch.bfloat16, torch.float16


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,group", [(1, 1), (2, 4), (1, 5), (3, 1), (2, 8)])
def test_decode_rows_of_every_small_length(ctx, dtype, dim, heads, group):
    have = [0, 1, 2, 7, 8, 15, 16, 17, 31, 33, 63, 64, 65, 127, 200]
    check(ctx, make(1, dtype, have, [1] * len(have), heads, group, dim, 16, tree=False))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("pt", [1, 3, 8, 16, 24, 64, 300])
def test_pages_of_any_size(ctx, dtype, pt):
    check(ctx, make(2, dtype, [0, 5, 100, 299], [3, 9, 1, 17], 2, 2, 128, pt))


@pytest.mark.parametrize("dtype,dim", [(BF, 128), (HF, 64)])
@pytest.mark.parametrize("new", [2, 8, 15, 16, 17, 31, 33, 64, 65, 100])
@pytest.mark.parametrize("tree", [True, False])
def test_drafted_tokens_of_every_tile_size(ctx, dtype, dim, new, tree):
    check(ctx, make(3, dtype, [0, 40, 129], [new, max(1, new // 2), new], 2, 2, dim, 16, tree))


@pytest.mark.parametrize("dtype,dim", [(BF, 128), (HF, 64)])
@pytest.mark.parametrize("pt", [1, 2, 3, 8, 24, 32, 64, 100, 256])
def test_pages_of_any_size_under_many_rows(ctx, dtype, dim, pt):
    # runs of 8 to 64 tokens in one copy, shorter ones gathered
    check(ctx, make(21, dtype, [0, 70, 300, 63], [40, 24, 33, 65], 2, 2, dim, pt))


@pytest.mark.parametrize("heads,group,new", [(1, 3, 40), (3, 5, 40), (2, 7, 20), (1, 16, 16), (1, 100, 3), (2, 128, 2), (1, 160, 2), (3, 8, 33)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_groups_of_any_size_under_many_rows(ctx, dtype, heads, group, new):
    # tiles of whole tokens (125 rows for groups of 5), several tiles per head, groups wider than a tile
    check(ctx, make(22, dtype, [0, 200, 61], [new, 1, new], heads, group, 128 if group < 10 else 64, 16))


@pytest.mark.parametrize("heads", [1, 3, 4])
def test_tiles_of_query_rows_that_share_a_slice(ctx, heads):
    # two CTAs walk one slice; an odd number of items leaves one without a partner
    check(ctx, make(23, BF, [3000, 10, 700, 0], [70, 64, 3, 100], heads, 4, 128, 16), extra=3)


@pytest.mark.parametrize("new,tree", [(150, True), (300, False), (129, True)])
def test_more_step_tokens_than_a_tile_has_rows(ctx, new, tree):
    check(ctx, make(24, BF, [0, 100], [new, 5], 1, 1, 64, 16, tree))


def test_rows_of_q_that_share_memory(ctx):
    x = make(25, BF, [50, 0], [30, 30], 1, 2, 128, 16)
    x["q"] = x["q"][:1].expand(60, 2, 128)
    check(ctx, x)
    x = make(25, BF, [50, 0], [30, 30], 1, 4, 64, 16)
    x["q"] = x["q"][:, :1].expand(60, 4, 64)
    check(ctx, x)
    x = make(25, BF, [50, 0], [30, 30], 2, 2, 64, 16)
    x["q"] = x["q"].transpose(0, 1).contiguous().transpose(0, 1)          # heads outermost
    check(ctx, x)


@pytest.mark.parametrize("dtype,dim,group,new", [(BF, 128, 4, 20), (HF, 64, 8, 40)])
def test_refusals_under_many_rows(ctx, dtype, dim, group, new):
    x = make(26, dtype, [1500, 30, 2000, 5, 700], [new] * 5, 2, group, dim, 16)
    x["label"][x["table"][0, 60]] = x["owner"][0] + 1
    x["label"][x["table"][1, 0]] = P.CONFLICT
    x["label"][x["table"][2, 3]] = P.PARAM
    x["table"][3, 0] = -7
    x["label"][x["table"][4, 44]], x["label"][x["table"][4, 2]] = P.NONE, x["owner"][4] + 1
    out, _ = check(ctx, x)
    assert not out[:2 * new].any() and out[2 * new: 3 * new].any()
    check(ctx, x, labels=False)


@pytest.mark.parametrize("new", [1, 20])
def test_many_short_items_of_which_some_are_refused(ctx, new):
    # a handful of one-tile items per CTA: each must get its own verdict
    n = 400
    x = make(28, BF, [r % 23 for r in range(n)], [new] * n, 4, 1, 64, 8)
    for r in range(0, n, 3):
        x["label"][x["table"][r, 0]] = P.CONFLICT if r % 2 else x["owner"][r] + 1
    _, _ = check(ctx, x)


def test_what_pages_hold_past_the_context_does_not_matter(ctx):
    for pt in (8, 16, 64):
        x = make(27, HF, [37, 5, 64, 100], [20] * 4, 2, 2, 128, pt)
        want = call(ctx, x)
        for r in range(4):
            end = int(x["want"][r])
            page = x["pool"][int(x["table"][r, end // pt])] if end % pt else None
            if page is not None:
                page[end % pt:] = float("nan")
        got = call(ctx, x)
        for a, b in zip(want[:3], got[:3]):
            assert torch.equal(a, b)
        check(ctx, x)


@pytest.mark.parametrize("dtype,dim,group", [(BF, 128, 1), (HF, 128, 8), (BF, 64, 4)])
def test_ragged_batches_with_idle_requests(ctx, dtype, dim, group):
    rng = np.random.default_rng(9)
    have = rng.integers(0, 400, size=40)
    new = rng.integers(0, 12, size=40)
    x = make(4, dtype, have, new, 2, group, dim, 16)
    x["want"][3] = max(0, x["have"][3] - 1) if new[3] == 0 else x["want"][3]
    check(ctx, x, extra=5)


@pytest.mark.parametrize("dtype,dim,heads,group,new", [(BF, 128, 1, 1, 1), (BF, 128, 8, 4, 1), (HF, 128, 2, 1, 16), (BF, 64, 1, 2, 40), (BF, 128, 1, 4, 64)])
def test_one_long_request_is_cut_over_the_gpu(ctx, dtype, dim, heads, group, new):
    check(ctx, make(5, dtype, [9000], [new], heads, group, dim, 16))


@pytest.mark.parametrize("new,group", [(1, 1), (9, 1), (20, 4)])
def test_one_long_and_many_short_requests(ctx, new, group):
    have = [5000] + [3] * 50 + [700] + [0] * 5
    check(ctx, make(6, BF, have, [new] * len(have), 1, group, 128, 16))


@pytest.mark.parametrize("group,new", [(1, 6), (8, 6), (8, 30)])
def test_rows_that_see_nothing_and_masks_with_stray_bits(ctx, group, new):
    x = make(7, BF, [0, 0, 20], [new] * 3, 2, group, 64, 16, words=3)
    x["mask"][0] = 0                               # empty row of an empty context
    x["mask"][new + 2] = 0
    x["mask"][2 * new] = 0                         # sees the context alone
    x["mask"][:, 1] |= 0xFFFFFFFF if new <= 32 else 0
    x["mask"][:, 2] = 0xFFFFFFFF                   # bits of tokens that do not exist
    x["mask"][1, 0] |= 0x80000000
    out, lse = check(ctx, x)
    assert not out[0].any() and torch.isneginf(lse[0]).all()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("group,new", [(1, 5), (4, 12), (8, 24)])
def test_what_hidden_tokens_hold_does_not_matter(ctx, dtype, group, new):
    have = [37, 0, 64]
    x = make(8, dtype, have, [new] * 3, 2, group, 128, 16)
    t0 = 0
    for r in range(3):
        # a drafted token that only its own row sees holds what overflowed
        j = new - 1
        x["mask"][t0: t0 + new, j // 32] &= ~np.uint32(1 << (j % 32))
        p = have[r] + j
        page = x["pool"][int(x["table"][r, p // 16])]
        page[p % 16, 0] = float("nan") if r == 0 else float("inf")
        page[p % 16, 1] = float("inf") if r == 1 else float("nan")
        page[p % 16 + 1:] = float("nan")           # past the end of the context
        if r == 2:                                 # its own row does: NaN comes out there and nowhere else
            x["mask"][t0 + j, j // 32] |= np.uint32(1 << (j % 32))
        t0 += new
    out, _ = check(ctx, x)
    assert torch.isfinite(out[: 3 * new - 1]).all() and torch.isnan(out[3 * new - 1]).all()


def test_infinite_scores(ctx):
    x = make(9, BF, [10, 10], [1, 1], 1, 1, 64, 16, tree=False)
    x["q"][:] = 1.0
    page = x["pool"][int(x["table"][0, 0])]
    page[:, 0] = 1.0
    page[3, 0, 0, 0] = float("-inf")               # one score of minus infinity: weight 0
    page = x["pool"][int(x["table"][1, 0])]
    page[:, 0] = 0.0
    page[:, 0, 0, 0] = float("-inf")               # all of them: the row counts as seeing nothing
    out, lse = check(ctx, x)
    assert not out[1].any() and torch.isneginf(lse[1]).all()


@pytest.mark.parametrize("group,new,have", [(1, 1, 100), (1, 3, 5000), (8, 16, 100), (8, 16, 3000)])
def test_refused_requests(ctx, group, new, have):
    x = make(10, BF, [have] * 7, [new] * 7, 2, group, 128, 16)
    blocks = (have + new + 15) // 16
    x["label"][x["table"][0, blocks - 1]] = x["owner"][0] + 1          # another user's page
    x["label"][x["table"][1, 0]] = P.NONE
    x["label"][x["table"][2, 1]] = P.PARAM                             # a shared prefix may be read
    x["label"][x["table"][3, 2]], x["label"][x["table"][3, 3]] = P.CONFLICT, x["owner"][3] + 1
    x["table"][4, blocks // 2] = x["pool"].shape[0]
    x["table"][5, 1] = -1
    x["label"][x["table"][5, 0]] = P.NONE
    out, lse = check(ctx, x)
    for r in (0, 1, 3, 4, 5):
        assert not out[r * new:(r + 1) * new].any() and torch.isneginf(lse[r * new:(r + 1) * new]).all()
    check(ctx, x, labels=False)


def test_malformed_requests_and_steps(ctx):
    x = make(11, HF, [5, 6, 7, 8], [2, 2, 2, 2], 1, 1, 64, 16)
    x["owner"][1] = -1
    x["rows"] = 8
    check(ctx, x)
    x = make(11, HF, [5, 6, 7], [40, 2, 2], 1, 1, 64, 16)
    x["mask"] = x["mask"][:, :1].copy()                                # 40 tokens, 32 bits
    check(ctx, x)
    x = make(12, HF, [5, 6, 7], [4, 4, 4], 1, 1, 64, 16)
    x["rows"], x["q"], x["mask"] = 11, x["q"][:11], x["mask"][:11]
    out, lse, who, st = call(ctx, x)
    assert (st == P.BAD_TABLE).all() and (out == 7).all() and (lse == 7).all() and (who == 7).all()


@pytest.mark.parametrize("scale", [0.0, 1.0, -0.2, 3.0])
def test_scales(ctx, scale):
    check(ctx, make(13, BF, [70, 3], [4, 2], 2, 2, 64, 16), scale=scale)


def test_the_same_call_gives_the_same_bits_and_streams_are_kept_apart(ctx):
    x = make(14, BF, [3000, 20, 500], [5, 9, 1], 2, 4, 128, 16)
    first = call(ctx, x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = call(ctx, x, stream=side.cuda_stream)
    for a, b in zip(first[:3], again[:3]):
        assert torch.equal(a, b)


def test_two_contexts_on_two_streams_at_once(ctx):
    # kernels of two calls that share SMs, tensor memory and L2; each context has its own scratch
    other = binding.Ctx(4)
    xs = [make(30, BF, [3000, 500, 40], [30, 40, 50], 2, 4, 128, 16), make(31, HF, [2500, 900, 0], [33, 20, 60], 4, 2, 64, 8)]
    want = [call(c, x) for c, x in zip((ctx, other), xs)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    bufs = []
    for x in xs:
        heads, dim = x["q"].shape[1:]
        bufs.append(dict(b=binding.Batch(dev(x["owner"]), dev(x["have"]), dev(x["want"]), dev(x["table"]), x["pt"], x["pool"].shape[0]),
                         mask=torch.from_numpy(x["mask"].view(np.int32)).cuda(), label=dev(x["label"]),
                         out=torch.zeros((x["rows"], heads, dim), dtype=x["q"].dtype, device="cuda"),
                         lse=torch.zeros((x["rows"], heads), device="cuda"), st=torch.full((3,), 9, dtype=torch.int32, device="cuda")))
    torch.cuda.synchronize()
    for _ in range(20):
        for c, x, s, d in zip((ctx, other), xs, streams, bufs):
            c.kv_attention(d["b"], x["pool"], x["q"], d["out"], d["st"], tree_mask=d["mask"], lse=d["lse"], owner_map=d["label"],
                           stream=s.cuda_stream)
    torch.cuda.synchronize()
    for w, d in zip(want, bufs):
        assert torch.equal(w[0], d["out"]) and torch.equal(w[1], d["lse"]) and not d["st"].any()
    other.close()


def test_a_captured_call_follows_its_inputs(ctx):
    x = make(15, BF, [400, 20, 64], [6, 3, 9], 2, 2, 128, 16)
    want = call(ctx, x)
    heads, dim = x["q"].shape[1:]
    q, out = x["q"].contiguous(), torch.zeros((x["rows"], heads, dim), dtype=BF, device="cuda")
    lse, who = torch.zeros((x["rows"], heads), device="cuda"), torch.zeros(x["rows"], dtype=torch.int32, device="cuda")
    st = torch.zeros(3, dtype=torch.int32, device="cuda")
    mask, label = torch.from_numpy(x["mask"].view(np.int32)).cuda(), dev(x["label"])
    b = binding.Batch(dev(x["owner"]), dev(x["have"]), dev(x["want"]), dev(x["table"]), 16, x["pool"].shape[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.kv_attention(b, x["pool"], q, out, st, tree_mask=mask, lse=lse, row_owner=who, owner_map=label)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]) and torch.equal(who, want[2])
    x["q"].mul_(0.5)                               # new values and lengths in the same buffers
    x["have"], x["want"] = np.array([100, 29, 64], np.int32), np.array([101, 32, 70], np.int32)
    b.tensors[1].copy_(dev(x["have"]))
    b.tensors[2].copy_(dev(x["want"]))
    q.copy_(x["q"])
    graph.replay()
    torch.cuda.synchronize()
    want = call(ctx, x)
    assert torch.equal(out[:10], want[0][:10]) and torch.equal(lse[:10], want[1][:10])


@pytest.mark.parametrize("new,pt", [(2, 16), (20, 16), (20, 4)])
def test_a_cache_past_four_gib(ctx, new, pt):
    # the request's pages are the pool's last ones: past 32-bit byte offsets
    heads, dim, pages = 32, 128, 20480 * 16 // pt
    pool = torch.empty((pages, pt, 2, heads, dim), dtype=BF, device="cuda")
    x = make(16, BF, [50], [new], heads, 1, dim, pt)
    want, _, _, _ = call(ctx, x)
    n = int(x["table"].size)
    pool[pages - n:] = x["pool"][torch.from_numpy(x["table"][0]).long().cuda()]
    y = dict(x, pool=pool, table=np.arange(pages - n, pages, dtype=np.int32)[None], label=np.full(pages, x["owner"][0], np.int32))
    got, _, _, st = call(ctx, y)
    assert not st.any() and torch.equal(got, want)


@pytest.mark.parametrize("n,new", [(8192, 1), (900, 18)])
def test_as_many_requests_as_a_batch_holds(ctx, n, new):
    rng = np.random.default_rng(n)
    check(ctx, make(29, BF, rng.integers(0, 12, size=n), np.where(rng.random(n) < 0.1, 0, new), 1, 1, 64, 4))
    if n == 8192:
        x = make(29, BF, [1] * (n + 1), [1] * (n + 1), 1, 1, 64, 4)
        with pytest.raises(binding.GiftError):
            call(ctx, x)


def test_wrong_tensors_are_refused(ctx):
    x = make(17, BF, [5], [2], 2, 1, 128, 16)
    with pytest.raises(ValueError):
        call(ctx, dict(x, q=x["q"].half()))
    with pytest.raises(ValueError):
        call(ctx, dict(x, mask=np.zeros((3, 1), np.uint32)))
    with pytest.raises(ValueError):
        call(ctx, dict(x, mask=np.zeros((2, 0), np.uint32)))
    with pytest.raises(ValueError):
        call(ctx, dict(x, pool=x["pool"].float(), q=x["q"].float()))
    with pytest.raises(binding.GiftError):
        call(ctx, dict(x, q=x["q"][:, :1]))        # one query head, two K/V heads
    with pytest.raises(binding.GiftError):
        call(ctx, x, out=torch.empty((1, 2, 128), dtype=BF, device="cuda").expand(2, 2, 128))
