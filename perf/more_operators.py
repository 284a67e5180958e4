"""The operators around the paged cache in 8 bits, as they are measured.

write      a step's q, k and v rows: norms of the heads, rotary positions, q out, K and V into labelled pages of 8 (or 16) bits
read       rows out of labelled pages, in 16 bits
attention  the step's rows over the 8-bit cache: single tokens, drafted trees, prompts; capped scores, distance bias, window

A token of an 8-bit page: e4m3 codes of K [heads][dim], of V [heads][dim], a 32-bit scale of K and of V for each head
([heads][2]), zeros up to a multiple of 16 bytes.  Sizes are those of the package's own workloads (32 heads of 128, blocks of 16
tokens, 16 to 512 requests, prompts of 256 to 2048 tokens) and generic grouped heads.  Lengths are spread evenly over
their range and dealt to the requests by the seed.
"""
import math

import numpy as np
import torch

own = False

NONE, PARAM, CONFLICT = -2, -1, -3
BAD_DESC, OWNER_MISMATCH, UNOWNED = 16, 2, 4
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
E4M3 = torch.float8_e4m3fn
EPS = 1e-6
LEAST = 2.0 ** -126


def listed():
    return [
        # K and V of one decode step, with norms and rotation
        dict(name="write decode", op="write", dtype="bf16", bits=8, requests=256, heads=32, q_heads=32, dim=128, pt=16, lo=256, hi=1024, new_lo=1, new_hi=1,
             norm=True, rot=128, axes=1, paired=False, far=0),
        # prefill chunks of 64 requests, one layer
        dict(name="write prefill", op="write", dtype="bf16", bits=8, requests=64, heads=32, q_heads=32, dim=128, pt=16, lo=0, hi=333, new_lo=511, new_hi=512,
             norm=True, rot=128, axes=1, paired=False, far=0),
        # rows of images and video far into a context: three axes, part of a head turned, neighbours as pairs, 16-bit pages
        dict(name="write axes", op="write", dtype="fp16", bits=16, requests=10, heads=8, q_heads=32, dim=128, pt=16, lo=0, hi=100, new_lo=1, new_hi=1000,
             norm=False, rot=96, axes=3, paired=True, far=1000000),
        # one short request back in 16 bits, some of its pages another user's
        dict(name="read small", op="read", dtype="fp16", bits=8, requests=1, heads=8, dim=128, pt=16, lo=500, hi=500, bad=1),
        # a batch of prompts back in 16 bits
        dict(name="read large", op="read", dtype="bf16", bits=8, requests=64, heads=32, dim=128, pt=16, lo=256, hi=1024, bad=0),
        # one request, one token: latency
        dict(name="attention one token", op="attention", dtype="bf16", requests=1, heads=32, q_heads=32, dim=128, pt=16, lo=513, hi=513, new_lo=1, new_hi=1,
             tree=False, bad=0, cap=0.0, window=0, slopes=False),
        # a decode step of the handoff's batch sizes, ragged
        dict(name="attention decode", op="attention", dtype="bf16", requests=64, heads=32, q_heads=32, dim=128, pt=16, lo=256, hi=2048, new_lo=1, new_hi=1,
             tree=False, bad=1, cap=0.0, window=0, slopes=False),
        # a decode step over long contexts, grouped heads
        dict(name="attention long", op="attention", dtype="fp16", requests=16, heads=8, q_heads=32, dim=128, pt=16, lo=4096, hi=32768, new_lo=1, new_hi=1,
             tree=False, bad=0, cap=0.0, window=0, slopes=False),
        # a decode step of a layer with capped scores, a distance bias and a window
        dict(name="attention window", op="attention", dtype="bf16", requests=64, heads=16, q_heads=32, dim=64, pt=16, lo=1, hi=8192, new_lo=1, new_hi=2,
             tree=False, bad=0, cap=50.0, window=1024, slopes=True),
        # drafted trees over long ragged contexts, grouped heads
        dict(name="attention tree grouped", op="attention", dtype="fp16", requests=48, heads=8, q_heads=32, dim=128, pt=16, lo=1, hi=16384, new_lo=1, new_hi=64,
             tree=True, bad=2, cap=0.0, window=0, slopes=False),
        # drafted trees, all heads their own, the largest batch
        dict(name="attention tree large", op="attention", dtype="bf16", requests=64, heads=32, q_heads=32, dim=128, pt=16, lo=256, hi=8192, new_lo=16, new_hi=16,
             tree=True, bad=0, cap=0.0, window=0, slopes=False),
        # prompt chunks behind what is cached, capped scores
        dict(name="attention prompt", op="attention", dtype="bf16", requests=8, heads=8, q_heads=32, dim=128, pt=16, lo=0, hi=2048, new_lo=300, new_hi=512,
             tree=False, bad=0, cap=30.0, window=0, slopes=False),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("write", "read", "attention", "attention"))
    pt = rng.choice((1, 8, 16, 16, 24, 32, 64))
    dtype = rng.choice(("bf16", "fp16"))
    heads = rng.choice((1, 2, 3, 4, 8, 16, 32))
    if op == "write":
        dim = rng.choice((64, 64, 80, 96, 128, 128, 192, 256))
        new_hi, n = _log(rng, 1, 512), _log(rng, 1, 64)
        heads = min(heads, 32 * 128 // dim)
        group = rng.choice((1, 2, 4, 8))
        return dict(op=op, dtype=dtype, bits=rng.choice((8, 8, 16)), requests=n, heads=heads, q_heads=heads * min(group, max(1, 32 * 128 // (dim * heads))), dim=dim,
                    pt=pt, lo=0, hi=_log(rng, 1, 300), new_lo=rng.randint(1, new_hi), new_hi=new_hi, norm=rng.random() < 0.6,
                    rot=rng.choice((0, dim, dim, dim // 2)), axes=rng.choice((1, 1, 2, 3)), paired=rng.random() < 0.4, far=rng.choice((0, 0, 100000, 1000000)))
    if op == "read":
        hi = _log(rng, 1, 1024)
        return dict(op=op, dtype=dtype, bits=rng.choice((8, 8, 16)), requests=_log(rng, 1, 64), heads=heads, dim=rng.choice((64, 80, 128)), pt=pt,
                    lo=rng.randint(1, hi), hi=hi, bad=rng.choice((0, 0, 1)) if hi > 200 else 0)
    group = rng.choice((1, 2, 4, 5, 8))
    new_hi = rng.choice((1, 1, 2, _log(rng, 1, 64), _log(rng, 1, 512)))
    n = _log(rng, 1, 64)
    hi = min(_log(rng, 1, 32768), max(1, 64 * 4096 * 32 // (n * max(heads, heads * group * new_hi // 24, 2))))
    tree = new_hi <= 64 and rng.random() < 0.5
    near = not tree and rng.random() < 0.4
    return dict(op="attention", dtype=dtype, requests=n, heads=heads, q_heads=heads * group, dim=rng.choice((64, 128)), pt=pt, lo=rng.randint(0, hi), hi=hi,
                new_lo=rng.randint(1, new_hi), new_hi=new_hi, tree=tree, bad=rng.choice((0, 0, 1)) if n > 3 else 0, cap=rng.choice((0.0, 0.0, 20.0, 50.0)),
                window=_log(rng, 1, 4096) if near else 0, slopes=near and rng.random() < 0.5)


# ---------------------------------------------------------------------------------------- inputs

def _spread(n, lo, hi):
    """n whole numbers evenly over [lo, hi]."""
    return [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)]


def _lengths(case):
    """(have, want) before the seed deals them out."""
    n = case["requests"]
    have = np.array(_spread(n, case["lo"], case["hi"]), dtype=np.int64)
    if case["op"] == "read":
        return have * 0, have
    new = np.array(_spread(n, case["new_lo"], case["new_hi"]), dtype=np.int64)
    return have, have + new[np.random.RandomState(n).permutation(n)]


def _up(a, b):
    return -(-a // b)


def _cuda(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def _token_bytes(heads, dim):
    return _up(2 * heads * (dim + 4), 16) * 16


def _parts(pages, heads, dim):
    """Codes [..., 2, heads, dim] and scales [..., heads, 2] of tokens of an 8-bit cache, as views."""
    m = 2 * heads * dim
    return pages[..., :m].view(E4M3).unflatten(-1, (2, heads, dim)), pages[..., m:m + 8 * heads].view(torch.float32).unflatten(-1, (heads, 2))


def _quantised(x):
    """(codes, scales) of heads [..., dim] in 32 bits."""
    top = x.abs().amax(-1)
    scale = torch.clamp(top / 448.0, min=LEAST)
    fine = torch.isfinite(x).all(-1)
    codes = torch.where(fine[..., None], x / scale[..., None], 0.0).to(E4M3)
    return codes, torch.where(fine, scale, math.nan)


def _filled(g, n_pages, pt, heads, dim, dtype):
    """8-bit pages that hold keys and values of the type, quantised a part at a time."""
    pages = torch.zeros((n_pages * pt, _token_bytes(heads, dim)), dtype=torch.uint8, device="cuda")
    codes, scales = _parts(pages, heads, dim)
    step = max(1, (1 << 27) // (2 * heads * dim))
    for t in range(0, n_pages * pt, step):
        k = min(step, n_pages * pt - t)
        x = torch.randn((k, 2, heads, dim), generator=g, device="cuda", dtype=dtype).float()
        c, s = _quantised(x)
        codes[t:t + k].copy_(c)
        scales[t:t + k].copy_(s.transpose(1, 2))
    return pages.view(n_pages, pt, -1)


def prepare(case, seed):
    op = case["op"]
    rng = np.random.RandomState(seed % (1 << 31))
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    have, want = _lengths(case)
    n, pt, heads, dim, dt = case["requests"], case["pt"], case["heads"], case["dim"], TYPES[case["dtype"]]
    deal = rng.permutation(n)
    have, want = have[deal], want[deal]
    owner = rng.permutation(max(n, 16))[:n].astype(np.int64)
    held = _up(want, pt)
    width = max(1, int(held.max()))
    pages = int(held.sum()) + 8
    table = np.full((n, width), -1, dtype=np.int64)
    inside = np.arange(width)[None, :] < held[:, None]
    table[inside] = rng.permutation(pages)[: int(held.sum())]
    label = np.full(pages, NONE, dtype=np.int64)
    label[table[inside]] = np.broadcast_to(owner[:, None], table.shape)[inside]
    for r in rng.permutation(n)[: case.get("bad", 0)]:
        # block-table entries redirected to another request's page (or one that nobody owns)
        if want[r] > 0:
            table[r, int(rng.randint(held[r]))] = int(rng.choice(np.flatnonzero(label != owner[r])))
    s = dict(case=case, owner=_cuda(owner), have=_cuda(have), want=_cuda(want), table=_cuda(table), label=_cuda(label), pages=pages, width=width)
    m = np.maximum(0, want - have)
    rows = s["rows"] = int(m.sum())
    req = np.repeat(np.arange(n), m)
    i = np.arange(rows) - np.repeat(np.cumsum(m) - m, m)
    pos = have[req] + i
    if case.get("bits", 8) == 8:
        s["pool"] = _filled(g, pages, pt, heads, dim, dt)
    else:
        s["pool"] = torch.randn((pages, pt, 2, heads, dim), generator=g, device="cuda", dtype=dt)
    if op != "attention":
        s["slots"] = _cuda(table[req, pos // pt] * pt + pos % pt, torch.int64)
        s["row_owner"] = _cuda(owner[req])
        s["status"] = torch.empty(rows, dtype=torch.int32, device="cuda")
    if op == "read":
        s["k"], s["v"] = (torch.zeros((rows, heads, dim), device="cuda", dtype=dt) for _ in range(2))
        return s
    # q, k and v as one projection leaves them
    q_heads = case["q_heads"]
    s["qkv"] = torch.randn((rows, q_heads + 2 * heads, dim), generator=g, device="cuda", dtype=dt)
    if op == "write":
        s["q_out"] = torch.empty((rows, q_heads, dim), device="cuda", dtype=dt)
        s["q_norm"], s["k_norm"] = ((1 + 0.2 * torch.randn(dim, generator=g, device="cuda")).to(dt) if case["norm"] else None for _ in range(2))
        turns, axes = case["rot"] // 2, case["axes"]
        s["pos"] = s["freq"] = s["sections"] = None
        if turns:
            s["freq"] = torch.tensor([1e4 ** (-j / turns) for j in range(turns)], dtype=torch.float32, device="cuda")
            s["sections"] = [turns - (axes - 1) * (turns // axes)] + [turns // axes] * (axes - 1)
            # one axis counts tokens; further ones are places within a picture
            s["pos"] = _cuda(np.stack([pos + case["far"]] + [rng.randint(0, 64, size=rows) + case["far"] // 1000 for _ in range(axes - 1)]))
        return s
    s["most"] = int(m.max())
    s["out"] = torch.empty((rows, q_heads, dim), dtype=dt, device="cuda")
    s["lse"] = torch.empty((rows, q_heads), dtype=torch.float32, device="cuda")
    s["status"] = torch.empty(n, dtype=torch.int32, device="cuda")
    s["row_owner"] = torch.empty(rows, dtype=torch.int32, device="cuda")
    s["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / q_heads) for h in range(q_heads)], dtype=torch.float32, device="cuda") if case["slopes"] else None
    s["mask"] = None
    if case["tree"]:
        # every drafted token hangs on one before it, or on the last cached one
        most = s["most"]
        seen = np.zeros((n, most, most), dtype=bool)
        for j in range(most):
            up = rng.randint(-1, j, size=n) if j else np.full(n, -1)
            seen[:, j] = np.where((up >= 0)[:, None], seen[np.arange(n), up], False)
            seen[:, j, j] = True
        words = _up(most, 32)
        bits = np.zeros((n, most, words * 32), dtype=bool)
        bits[:, :, :most] = seen
        packed = np.packbits(bits, axis=2, bitorder="little").view("<u4").astype(np.int64)
        s["mask"] = torch.from_numpy(packed[req, i].astype(np.uint32).view(np.int32).reshape(rows, words)).cuda()
    return s


# ------------------------------------------------------------------------------------ plain forms

def _views(s):
    c = s["case"]
    return torch.split(s["qkv"], [c["q_heads"], c["heads"], c["heads"]], 1)


def _row_status(s, may_read):
    """What becomes of every row by its slot and its page's label."""
    slot, pt = s["slots"], s["case"]["pt"]
    inside = (slot >= 0) & (slot < s["pages"] * pt)
    label = s["label"][torch.where(inside, slot // pt, 0)]
    fine = (label == s["row_owner"]) | ((label == PARAM) & may_read)
    st = torch.where(fine, 0, torch.where(label <= NONE, UNOWNED, OWNER_MISMATCH))
    return torch.where(slot == -1, 0, torch.where(inside, st, BAD_DESC)), inside & fine


def _turned(s, x, weight):
    """Heads of rows [rows, heads, dim], normed and turned, in 32 bits."""
    c = s["case"]
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    half = c["rot"] // 2
    if half == 0:
        return x
    axis = torch.repeat_interleave(torch.arange(c["axes"], device="cuda"), torch.tensor(s["sections"], device="cuda"))
    angle = s["pos"].T[:, axis].double() * s["freq"].double()                 # far positions need 64 bits
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    head, rest = x[..., : c["rot"]], x[..., c["rot"]:]
    a, b = (head[..., 0::2], head[..., 1::2]) if c["paired"] else (head[..., :half], head[..., half:])
    u, v = a * cos - b * sin, b * cos + a * sin
    return torch.cat([torch.stack([u, v], -1).flatten(-2) if c["paired"] else torch.cat([u, v], -1), rest], -1)


def _write_plain(s):
    c = s["case"]
    q, k, v = _views(s)
    status, good = _row_status(s, False)
    s["status"].copy_(status)
    s["q_out"].copy_(torch.where(good[:, None, None], _turned(s, q, s["q_norm"]).to(q.dtype), s["q_out"]))
    kv = torch.stack([_turned(s, k, s["k_norm"]), v.float()], 1)
    at = s["slots"][good]
    if c["bits"] == 16:
        s["pool"].view(-1, 2, c["heads"], c["dim"])[at] = kv.to(k.dtype)[good]
        return [s["q_out"], s["pool"], s["status"]]
    codes, scales = _quantised(kv)
    row = torch.zeros((kv.shape[0], s["pool"].shape[-1]), dtype=torch.uint8, device="cuda")
    to_codes, to_scales = _parts(row, c["heads"], c["dim"])
    to_codes.copy_(codes)
    to_scales.copy_(scales.transpose(1, 2))
    s["pool"].view(-1, row.shape[1])[at] = row[good]
    return [s["q_out"], *_parts(s["pool"], c["heads"], c["dim"]), s["status"]]


def _read_plain(s):
    c = s["case"]
    status, good = _row_status(s, True)
    s["status"].copy_(status)
    at = torch.where(good, s["slots"], 0)
    if c["bits"] == 16:
        kv = s["pool"].view(-1, 2, c["heads"], c["dim"])[at].float()
    else:
        codes, scales = _parts(s["pool"].view(-1, s["pool"].shape[-1])[at], c["heads"], c["dim"])
        kv = codes.float() * scales.transpose(1, 2)[..., None]
    kv = torch.where(good[:, None, None, None], kv, 0.0)
    s["k"].copy_(kv[:, 0])
    s["v"].copy_(kv[:, 1])
    return [s["k"], s["v"], s["status"]]


def _attention_plain(s):
    c, pt, rows, most = s["case"], s["case"]["pt"], s["rows"], s["most"]
    n, hk, hq, d = c["requests"], c["heads"], c["q_heads"], c["dim"]
    group, width = hq // hk, s["width"]
    owner, have, want = s["owner"].long(), s["have"].long(), s["want"].long()
    ends = torch.cumsum(want - have, 0)
    t = torch.arange(rows, device="cuda")
    req = torch.searchsorted(ends, t, right=True)
    i = t - (ends - want + have)[req]
    pos = torch.arange(width * pt, device="cuda")[None, :]
    row_pos = have[:, None] + torch.arange(most, device="cuda")[None, :]       # [n, most]
    low = have - c["window"] + 1 if c["window"] else torch.zeros_like(have)    # the first position that any row sees
    low = torch.clamp(low, min=0)
    # pages that hold a token that some row may see
    first = torch.arange(width, device="cuda")[None, :] * pt
    used = (first < want[:, None]) & (first + pt > low[:, None])
    table = s["table"].long()
    inside = (table >= 0) & (table < s["pages"])
    label = s["label"].long()[torch.where(inside, table, 0)]
    bad = (used & ~inside).any(1)
    unowned = (used & inside & (label <= NONE)).any(1)
    foreign = (used & inside & (label >= 0) & (label != owner[:, None])).any(1)
    status = torch.where(bad, BAD_DESC, unowned * UNOWNED + foreign * OWNER_MISMATCH)
    # the context of every request, padded to the longest, and what of it each row sees
    codes, scales = _parts(s["pool"][torch.where(used & inside, table, 0)].view(n, width * pt, -1), hk, d)
    there = (pos < want[:, None]) & (pos >= low[:, None])
    key = torch.where(there[:, :, None, None], codes[:, :, 0].float() * scales[..., 0, None], 0)
    val = torch.where(there[:, :, None, None], codes[:, :, 1].float() * scales[..., 1, None], 0)
    at = req * most + i
    q = torch.zeros((n * most, hq, d), device="cuda")
    q[at] = _views(s)[0].float()
    j = pos - have[:, None]                                       # index among the step's own tokens
    if s["mask"] is None:
        seen = j[:, None, :] <= torch.arange(most, device="cuda")[None, :, None]
    else:
        words = torch.zeros((n * most, s["mask"].shape[1]), dtype=torch.int64, device="cuda")
        words[at] = s["mask"].long()
        jj = torch.clamp(j, 0, 32 * words.shape[1] - 1)[:, None, :].expand(n, most, width * pt)
        word = torch.gather(words.view(n, most, -1), 2, jj // 32)
        seen = ((word >> (jj % 32)) & 1).bool() | (j < 0)[:, None, :]
    seen = seen & there[:, None, :]
    away = pos[:, None, :] - row_pos[:, :, None]                  # [n, most, tokens]
    if c["window"]:
        seen = seen & (away > -c["window"])
    q = q.view(n, most, hk, group, d).permute(0, 2, 3, 1, 4).reshape(n, hk, group * most, d)
    sc = (torch.matmul(q, key.permute(0, 2, 3, 1)) * (1.0 / math.sqrt(d))).view(n, hk, group, most, -1)
    del key
    if c["cap"]:
        sc = c["cap"] * torch.tanh(sc / c["cap"])
    if s["slopes"] is not None:
        sc = sc + s["slopes"].view(1, hk, group, 1, 1) * away[:, None, None].float()
    sc = torch.where(seen[:, None, None], sc, -math.inf)
    top = sc.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(sc - top)
    del sc
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(n, hk, group * most, -1), val.permute(0, 2, 1, 3)).view(n, hk, group, most, d)
    o = torch.where(total > 0, o / total, 0.0)
    lse = top + torch.log(total)
    fine = (status == 0)[:, None, None, None, None]
    o = torch.where(fine, o, 0.0).permute(0, 3, 1, 2, 4).reshape(n * most, hq, d)[at]
    lse = torch.where(fine, lse, -math.inf).permute(0, 3, 1, 2, 4).reshape(n * most, hq)[at]
    s["out"].copy_(o)
    s["lse"].copy_(lse)
    s["status"].copy_(status)
    s["row_owner"].copy_(torch.where(status == 0, owner, CONFLICT)[req])
    return [s["out"], s["lse"], s["row_owner"], s["status"]]


# -------------------------------------------------------------------------------- the framework's

_handle = []


def _ctx():
    """The context that a program keeps for its whole life."""
    if not _handle:
        from paper_2608_25431_b200 import binding
        _handle.extend([binding, binding.Ctx(1024)])
    return _handle


def _own(s):
    binding, ctx = _ctx()
    c, op = s["case"], s["case"]["op"]
    if op == "read":
        ctx.kv_read(s["pool"], s["k"], s["v"], s["slots"], s["row_owner"], s["status"], owner_map=s["label"])
        return [s["k"], s["v"], s["status"]]
    q, k, v = _views(s)
    if op == "write":
        ctx.kv_write(s["pool"], k, v, s["slots"], s["row_owner"], s["status"], q=q, q_out=s["q_out"], q_norm=s["q_norm"], k_norm=s["k_norm"], eps=EPS,
                     pos=s["pos"], freq=s["freq"], sections=s["sections"], paired=c["paired"], owner_map=s["label"])
        return [s["q_out"], s["pool"], s["status"]] if c["bits"] == 16 else [s["q_out"], *_parts(s["pool"], c["heads"], c["dim"]), s["status"]]
    b = binding.Batch(s["owner"], s["have"], s["want"], s["table"], c["pt"], s["pages"])
    ctx.kv_attention_codes(b, s["pool"], c["heads"], q, s["out"], s["status"], tree_mask=s["mask"], lse=s["lse"], row_owner=s["row_owner"], owner_map=s["label"],
                      softcap=c["cap"], window=c["window"], slopes=s["slopes"])
    return [s["out"], s["lse"], s["row_owner"], s["status"]]


def run(state):
    if own:
        return _own(state)
    return {"write": _write_plain, "read": _read_plain, "attention": _attention_plain}[state["case"]["op"]](state)


# --------------------------------------------------------------------------------- work and values

def work(case):
    have, want = _lengths(case)
    m = int((want - have).sum())
    heads, dim = case["heads"], case["dim"]
    token = 2 * heads * (dim + 4) if case.get("bits", 8) == 8 else 4 * heads * dim
    blocks = int(_up(want, case["pt"]).sum())
    if case["op"] == "read":
        return {"bytes": m * (token + 4 * heads * dim + 16) + 4 * blocks, "flops": 0}
    q = case["q_heads"] * dim * 2
    if case["op"] == "write":
        turn = 4 * case["axes"] if case["rot"] else 0
        return {"bytes": m * (2 * q + 4 * heads * dim + token + 16 + turn) + 4 * blocks, "flops": 0}
    low = np.maximum(0, have - case["window"] + 1) if case["window"] else 0 * have
    seen = want - have if case["tree"] else (want - have + 1) / 2.0            # of the step's tokens, per row
    span = np.minimum(have + seen, case["window"]) if case["window"] else have + seen
    return {"bytes": int((want - low).sum()) * token + 8 * int((_up(want, case["pt"]) - low // case["pt"]).sum()) + m * (2 * q + 4 * case["q_heads"] + 4)
            + 16 * case["requests"], "flops": 4.0 * float(((want - have) * span).sum()) * case["q_heads"] * dim}


def _nearest_code(x):
    """The e4m3 value nearest to x, ties to even, in 64 bits."""
    e = torch.clamp(torch.floor(torch.log2(torch.clamp(x.abs(), min=2.0 ** -20))), -6, 8)
    step = torch.exp2(e - 3)
    return torch.clamp(torch.round(x / step) * step, -448, 448)


def _exact_write(c, s):
    dim, turns = c["dim"], c["rot"] // 2
    q, k, v = (x.double() for x in _views(s))

    def turned(x, w):
        if w is not None:
            x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / dim + EPS) * w.double()
        y = x.clone()
        first = 0
        for axis, count in enumerate(s["sections"] or []):
            for f in range(first, first + count):
                a, b = (2 * f, 2 * f + 1) if c["paired"] else (f, f + turns)
                z = torch.polar(torch.ones(x.shape[0], dtype=torch.float64, device="cuda"), s["pos"][axis].double() * s["freq"][f].double())[:, None]
                z = torch.complex(x[..., a], x[..., b]) * z
                y[..., a], y[..., b] = z.real, z.imag
            first += count
        return y

    label = s["label"].tolist()
    good = [t for t, (slot, who) in enumerate(zip(s["slots"].tolist(), s["row_owner"].tolist())) if slot >= 0 and label[slot // c["pt"]] == who]
    good = torch.tensor(good, dtype=torch.int64, device="cuda")
    at = s["slots"][good]
    q, k, v = turned(q, s["q_norm"]), turned(k, s["k_norm"])[good], v[good]
    if c["bits"] == 16:
        pool = s["pool"].double()
        flat = pool.view(-1, 2, c["heads"], dim)
        flat[at, 0], flat[at, 1] = k, v
        return [q, pool, None]
    codes, scales = (x.double() for x in _parts(s["pool"], c["heads"], dim))
    for j, x in enumerate((k, v)):
        scale = torch.clamp(x.abs().max(-1).values / 448, min=LEAST)
        codes.view(-1, 2, c["heads"], dim)[at, j] = _nearest_code(x / scale[..., None])
        scales.view(-1, c["heads"], 2)[at, :, j] = scale
    return [q, codes, scales, None]


def exact(case, seed):
    """The values, one pair of elements, row or request at a time."""
    s = prepare(case, seed)
    if case["op"] == "write":
        return _exact_write(case, s)
    heads, d, pt = case["heads"], case["dim"], case["pt"]
    if case.get("bits", 8) == 16:
        keys, values = s["pool"].view(-1, 2, heads, d).unbind(1)
        one = torch.ones((), dtype=torch.float64, device="cuda")
        k_scale = v_scale = one.expand(keys.shape[0], heads)
    else:
        codes, scales = _parts(s["pool"].view(-1, s["pool"].shape[-1]), heads, d)
        (keys, values), (k_scale, v_scale) = codes.unbind(1), scales.double().unbind(2)
    owner, have, want, table, label = (s[x].tolist() for x in ("owner", "have", "want", "table", "label"))
    if case["op"] == "read":
        mine = torch.tensor([label[slot // pt] in (who, PARAM) for slot, who in zip(s["slots"].tolist(), s["row_owner"].tolist())], device="cuda")[:, None, None]
        at = s["slots"]
        return [keys[at].double() * k_scale[at][..., None] * mine, values[at].double() * v_scale[at][..., None] * mine, None]
    if float(((s["want"] - s["have"]).double() * s["want"].double()).sum()) * case["q_heads"] * d > 4e12:
        return None
    rows, hq = s["rows"], case["q_heads"]
    q, cap, window = _views(s)[0], case["cap"], case["window"]
    out = torch.zeros((rows, hq, d), dtype=torch.float64, device="cuda")
    lse = torch.full((rows, hq), -math.inf, dtype=torch.float64, device="cuda")
    t0 = 0
    for r in range(case["requests"]):
        m, low = want[r] - have[r], max(0, have[r] - window + 1) if window else 0
        mine = table[r][low // pt: -(-want[r] // pt)]
        if all(0 <= p < s["pages"] and label[p] in (owner[r], PARAM) for p in mine):
            places = torch.arange(low, want[r], device="cuda")
            at = s["table"][r].long()[places // pt] * pt + places % pt
            seen = torch.ones((m, want[r] - low), dtype=torch.bool, device="cuda")
            for i in range(m):
                if s["mask"] is None:
                    seen[i, have[r] + i + 1 - low:] = False
                    if window:
                        seen[i, : max(0, have[r] + i - window + 1 - low)] = False
                else:
                    bits = sum((w & 0xFFFFFFFF) << (32 * x) for x, w in enumerate(s["mask"][t0 + i].tolist()))
                    seen[i, have[r]:] = torch.tensor([bool(bits >> j & 1) for j in range(m)], device="cuda")
            for h in range(heads):
                g = slice(h * hq // heads, (h + 1) * hq // heads)
                key, value = keys[at, h].double() * k_scale[at, h, None], values[at, h].double() * v_scale[at, h, None]
                z = torch.einsum("tgd,ld->gtl", q[t0:t0 + m, g].double(), key) / math.sqrt(d)
                if cap:
                    z = cap * torch.tanh(z / cap)
                if s["slopes"] is not None:
                    z = z + s["slopes"][g].double()[:, None, None] * (places[None, None, :] - (have[r] + torch.arange(m, device="cuda"))[None, :, None])
                z = z.masked_fill(~seen[None], -math.inf)
                total = torch.logsumexp(z, -1)
                lse[t0:t0 + m, g] = total.T
                out[t0:t0 + m, g] = torch.einsum("gtl,ld->tgd", torch.exp(z - total[:, :, None]), value)
        t0 += m
    return [out, lse, None, None]
