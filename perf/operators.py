"""The operators of the paged cache between the boundary calls, as they are measured.

blocks    block tables from request lengths: pages taken from and given back to a free stack
slots     slot, position, request and owner label of every row of a step
segments  the segment table of a handoff, one segment per (layer, request, block)
append    the step's K and V rows written into labelled pages
attention the step's rows (a tree of drafted tokens, or one token) over the paged cache

Sizes are those of the package's own workloads (32 layers, 32 heads of 128, blocks of 16 tokens, 16 to
512 requests, prompts of 256 to 2048 tokens, mixed prefill and decode batches) and generic grouped heads.
Lengths are spread evenly over their range and dealt to the requests by the seed.
"""
import math

import numpy as np
import torch

own = False

NONE, PARAM, CONFLICT = -2, -1, -3
BAD_DESC, OWNER_MISMATCH, UNOWNED, NO_BLOCKS, BAD_TABLE = 16, 2, 4, 64, 128
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    return [
        # one decode step of a full batch: a request needs a new block every 16th step
        dict(name="blocks decode", op="blocks", requests=256, layers=32, pt=16, lo=256, hi=2048, new_lo=1, new_hi=1, every=0, back=0, spare=8),
        # a mixed batch: prefill chunks next to requests that give drafted tokens back, and a pool that runs short for the last few
        dict(name="blocks mixed", op="blocks", requests=512, layers=32, pt=16, lo=33, hi=4096, new_lo=1, new_hi=512, every=2, back=48, spare=-64),
        # rows of one decode step
        dict(name="slots decode", op="slots", requests=256, pt=16, lo=256, hi=2048, new_lo=1, new_hi=1, pad=0),
        # rows of a mixed batch of 512 requests, padded to a captured size
        dict(name="slots mixed", op="slots", requests=512, pt=16, lo=0, hi=4096, new_lo=1, new_hi=512, pad=1000),
        # handoff of one layer of a small batch
        dict(name="segments small", op="segments", requests=16, layers=1, pt=16, lo=256, hi=2048, whole=True),
        # handoff of a large batch, every layer
        dict(name="segments large", op="segments", requests=512, layers=32, pt=16, lo=1, hi=511, whole=False),
        # K and V of one decode step
        dict(name="append decode", op="append", dtype="bf16", requests=256, heads=32, q_heads=32, dim=128, pt=16, lo=256, hi=1024, new_lo=1, new_hi=1),
        # K and V of prefill chunks, one layer
        dict(name="append prefill", op="append", dtype="bf16", requests=64, heads=32, q_heads=32, dim=128, pt=16, lo=0, hi=333, new_lo=511, new_hi=512),
        # one request, one token: latency
        dict(name="attention one token", op="attention", dtype="bf16", requests=1, heads=32, q_heads=32, dim=128, pt=16, lo=513, hi=513, new_lo=1, new_hi=1, tree=False, bad=0),
        # a decode step of the handoff's batch sizes, ragged
        dict(name="attention decode", op="attention", dtype="bf16", requests=64, heads=32, q_heads=32, dim=128, pt=16, lo=256, hi=2048, new_lo=1, new_hi=1, tree=False, bad=1),
        # drafted trees over long ragged contexts, grouped heads
        dict(name="attention tree grouped", op="attention", dtype="fp16", requests=48, heads=8, q_heads=32, dim=128, pt=16, lo=1, hi=16384, new_lo=1, new_hi=64, tree=True, bad=2),
        # drafted trees, all heads their own, the largest batch
        dict(name="attention tree large", op="attention", dtype="bf16", requests=64, heads=32, q_heads=32, dim=128, pt=16, lo=256, hi=8192, new_lo=16, new_hi=16, tree=True, bad=0),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("blocks", "slots", "segments", "append", "attention", "attention"))
    pt = rng.choice((1, 8, 16, 16, 24, 32, 64))
    if op == "blocks":
        hi = _log(rng, pt, 4096)
        return dict(op=op, requests=_log(rng, 1, 512), layers=rng.randint(1, 32), pt=max(pt, 8), lo=rng.randint(0, hi), hi=hi, new_lo=rng.randint(0, 1),
                    new_hi=_log(rng, 1, 512), every=rng.choice((0, 2, 3, 5)), back=rng.randint(0, 64), spare=rng.choice((8, 100, -1)))
    if op == "slots":
        hi = _log(rng, 1, 4096)
        return dict(op=op, requests=_log(rng, 1, 512), pt=pt, lo=rng.randint(0, hi), hi=hi, new_lo=rng.randint(0, 1), new_hi=_log(rng, 1, 512), pad=rng.randint(1, 1500))
    if op == "segments":
        hi = _log(rng, 1, 512)
        return dict(op=op, requests=_log(rng, 1, 512), layers=rng.randint(1, 32), pt=max(pt, 16), lo=rng.randint(1, hi), hi=hi, whole=rng.random() < 0.5)
    heads = rng.choice((1, 2, 4, 8, 16, 32))
    if op == "append":
        new_hi = _log(rng, 1, 512)
        return dict(op=op, dtype=rng.choice(("bf16", "fp16")), requests=_log(rng, 1, 64), heads=heads, q_heads=32, dim=rng.choice((64, 128)), pt=pt,
                    lo=0, hi=_log(rng, 1, 300), new_lo=rng.randint(1, new_hi), new_hi=new_hi)
    group = rng.choice((1, 2, 4, 5, 8))
    new_hi = _log(rng, 1, 64)
    n = _log(rng, 1, 64)
    hi = min(_log(rng, 1, 32768), max(1, 64 * 4096 * 32 // (n * max(heads, heads * group * new_hi // 24, 2))))
    return dict(op=op, dtype=rng.choice(("bf16", "fp16")), requests=n, heads=heads, q_heads=heads * group, dim=rng.choice((64, 128)), pt=pt, lo=rng.randint(0, hi), hi=hi,
                new_lo=rng.randint(1, new_hi), new_hi=new_hi, tree=rng.random() < 0.7, bad=rng.choice((0, 0, 1)))


# ---------------------------------------------------------------------------------------- inputs

def _spread(n, lo, hi):
    """n whole numbers evenly over [lo, hi]."""
    return [lo + (hi - lo) * i // max(1, n - 1) for i in range(n)]


def _lengths(case):
    """(have, want) before the seed deals them out."""
    n = case["requests"]
    have = np.array(_spread(n, case["lo"], case["hi"]), dtype=np.int64)
    if case["op"] == "segments":
        return have * 0, have
    new = np.array(_spread(n, case["new_lo"], case["new_hi"]), dtype=np.int64)
    new = new[np.random.RandomState(n).permutation(n)]
    want = have + new
    if case["op"] == "blocks" and case["every"]:
        gives = np.arange(n) % case["every"] == 1
        want = np.where(gives, np.maximum(0, have - case["back"]), want)
    return have, want


def _up(a, b):
    return -(-a // b)


def _batch(case, seed):
    """owner, have, want on the host, the block table of what is held, and the pages' owners."""
    rng = np.random.RandomState(seed % (1 << 31))
    have, want = _lengths(case)
    n, pt = case["requests"], case["pt"]
    deal = rng.permutation(n)
    have, want = have[deal], want[deal]
    owner = rng.permutation(max(n, 16))[:n].astype(np.int64)
    held = _up(have if case["op"] == "blocks" else np.maximum(have, want), pt)
    width = max(1, int(_up(np.maximum(have, want), pt).max()))
    spare = max(0, int(np.maximum(0, _up(want, pt) - _up(have, pt)).sum()) + case.get("spare", 8))
    pages = int(held.sum()) + spare
    perm = rng.permutation(pages)
    table = np.full((n, width), -1, dtype=np.int64)
    col = np.arange(width)[None, :]
    inside = col < held[:, None]
    table[inside] = perm[: int(held.sum())]
    label = np.full(pages, NONE, dtype=np.int64)
    label[table[inside]] = np.broadcast_to(owner[:, None], table.shape)[inside]
    return owner, have, want, table, label, perm[int(held.sum()):], width, pages


def _cuda(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def prepare(case, seed):
    op = case["op"]
    owner, have, want, table, label, spare, width, pages = _batch(case, seed)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = dict(case=case, owner=_cuda(owner), have=_cuda(have), want=_cuda(want), pages=pages, width=width)
    if op == "blocks":
        free = np.full(pages, -1, dtype=np.int64)
        free[: spare.size] = spare
        start = np.concatenate([table.reshape(-1), free, [spare.size], np.tile(label, case["layers"]), np.zeros(case["requests"], dtype=np.int64)])
        s["start"] = _cuda(start)      # what the step begins with: every pass works on a copy, since the call changes it in place
        s["work"] = torch.empty_like(s["start"])
        return s
    s["table"] = _cuda(table)
    rows = int(np.maximum(0, want - have).sum())
    if op == "slots":
        n = rows + case["pad"]
        s["slots"] = torch.empty(n, dtype=torch.int64, device="cuda")
        s["ints"] = torch.empty((3, n), dtype=torch.int32, device="cuda")
        s["ptr"] = torch.empty(case["requests"] + 1, dtype=torch.int32, device="cuda")
        return s
    if op == "segments":
        total = int(_up(want, case["pt"]).sum()) * case["layers"]
        s["serial"] = torch.randint(0, 1 << 31, (case["requests"],), generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
        s["segs"] = torch.empty((max(1, total), 10), dtype=torch.int32, device="cuda")
        s["page_table"] = torch.empty(max(1, total), dtype=torch.int32, device="cuda")
        return s
    dt, heads, dim, pt = TYPES[case["dtype"]], case["heads"], case["dim"], case["pt"]
    if op == "attention" and case["bad"]:
        # block-table entries redirected to another request's page
        rng = np.random.RandomState(seed % (1 << 31) + 1)
        for r in rng.permutation(case["requests"])[: case["bad"]]:
            foreign = int(rng.randint(pages))
            if want[r] > 0 and label[foreign] != owner[r]:
                table[r, int(rng.randint(_up(int(want[r]), pt)))] = foreign
        s["table"] = _cuda(table)
    s["label"] = _cuda(label)
    s["pool"] = torch.randn((pages, pt, 2, heads, dim), generator=g, device="cuda", dtype=dt)
    # q, k and v as one projection leaves them
    s["qkv"] = torch.randn((max(1, rows), case["q_heads"] + 2 * heads, dim), generator=g, device="cuda", dtype=dt)
    m = np.maximum(0, want - have)
    req = np.repeat(np.arange(case["requests"]), m)
    if op == "append":
        pos = np.arange(rows) - np.repeat(np.cumsum(m) - m, m) + have[req]
        s["slots"] = _cuda(table[req, pos // pt] * pt + pos % pt, torch.int64)
        s["row_owner"] = _cuda(owner[req])
        s["status"] = torch.empty(rows, dtype=torch.int32, device="cuda")
        return s
    s["rows"], s["most"] = rows, int(m.max())
    s["out"] = torch.empty((max(1, rows), case["q_heads"], dim), dtype=dt, device="cuda")
    s["lse"] = torch.empty((max(1, rows), case["q_heads"]), dtype=torch.float32, device="cuda")
    s["status"] = torch.empty(case["requests"], dtype=torch.int32, device="cuda")
    s["row_owner"] = torch.empty(max(1, rows), dtype=torch.int32, device="cuda")
    s["mask"] = None
    if case["tree"]:
        # every drafted token hangs on one before it, or on the last cached one
        most = s["most"]
        rng = np.random.RandomState(seed % (1 << 31) + 2)
        seen = np.zeros((case["requests"], most, most), dtype=bool)
        for i in range(most):
            up = rng.randint(-1, i, size=case["requests"]) if i else np.full(case["requests"], -1)
            seen[:, i] = np.where((up >= 0)[:, None], seen[np.arange(case["requests"]), up], False)
            seen[:, i, i] = True
        words = _up(most, 32)
        bits = np.zeros((case["requests"], most, words * 32), dtype=bool)
        bits[:, :, :most] = seen
        packed = np.packbits(bits, axis=2, bitorder="little").view("<u4").astype(np.int64)
        i = np.arange(rows) - np.repeat(np.cumsum(m) - m, m)
        s["mask"] = torch.from_numpy(packed[req, i].astype(np.uint32).view(np.int32).reshape(rows, words)).cuda()
    return s


# ------------------------------------------------------------------------------------ plain forms

def _well_formed(s):
    pt, width = s["case"]["pt"], s["width"]
    owner, have, want = s["owner"].long(), s["have"].long(), s["want"].long()
    ok = (owner >= 0) & (have >= 0) & (want >= 0) & ((have + pt - 1) // pt <= width) & ((want + pt - 1) // pt <= width)
    return ok, owner, torch.where(ok, have, 0), torch.where(ok, want, 0)


def _parts(s):
    """The step's state in one buffer: table, free stack, its height, labels, status."""
    c, n = s["case"], s["case"]["requests"]
    w = s["work"]
    sizes = [n * s["width"], s["pages"], 1, c["layers"] * s["pages"], n]
    table, free, height, label, status = torch.split(w, sizes)
    return table.view(n, s["width"]), free, height, label.view(c["layers"], s["pages"]), status


def _blocks_plain(s):
    s["work"].copy_(s["start"])
    table, free, height, label, status = _parts(s)
    pt, pages, cap = s["case"]["pt"], s["pages"], free.numel()
    ok, owner, have, want = _well_formed(s)
    bh, bw = (have + pt - 1) // pt, (want + pt - 1) // pt
    f = height.long()
    need = torch.clamp(bw - bh, min=0)
    short = (need > 0) & (torch.cumsum(need, 0) > f)
    need = torch.where(short, 0, need)
    gives = torch.clamp(bh - bw, min=0)
    first, back = torch.cumsum(need, 0) - need, torch.cumsum(gives, 0) - gives
    taken, given = need.sum(), gives.sum()
    col = torch.arange(table.shape[1], device="cuda")[None, :]
    grow = (col >= bh[:, None]) & (col < bw[:, None]) & ~short[:, None]
    drop = (col >= bw[:, None]) & (col < bh[:, None])
    new = free[torch.clamp(f - 1 - (first[:, None] + col - bh[:, None]), 0, cap - 1)].long()
    page = torch.where(grow, new, table.long())
    used = grow | drop
    inside = (page >= 0) & (page < pages)
    at = torch.where(used & inside, page, pages)
    times = torch.zeros(pages + 1, dtype=torch.int64, device="cuda").scatter_add_(0, at.reshape(-1), torch.ones_like(at).reshape(-1))[:pages]
    here = torch.cat([label, torch.full_like(label[:, :1], NONE)], 1)[:, at].long()
    legal = torch.where(grow[None], here == NONE, (here == owner[None, :, None]) | (here == NONE) | (here == CONFLICT)).all(0)
    refused = (used & ~(inside & legal)).any() | (times > 1).any() | (f < 0).any() | (f - taken + given > cap).any()
    grow, drop = grow & ~refused, drop & ~refused
    status.copy_(torch.where(refused, BAD_TABLE, torch.where(~ok, BAD_DESC, torch.where(short, NO_BLOCKS, 0))))
    table.copy_(torch.where(grow, page, torch.where(drop, -1, table.long())))
    paint = torch.cat([label, torch.zeros_like(label[:, :1])], 1)
    value = torch.where(grow, owner[:, None], NONE).to(torch.int32)
    paint[:, torch.where(grow | drop, page, pages).reshape(-1)] = value.reshape(-1)
    label.copy_(paint[:, :pages])
    stack = torch.cat([free, torch.zeros_like(free[:1])])
    place = torch.where(drop, f - taken + back[:, None] + col - bw[:, None], cap)
    stack[place.reshape(-1)] = page.to(torch.int32).reshape(-1)
    free.copy_(stack[:cap])
    height.copy_(torch.where(refused, f, f - taken + given))
    return [table, free, height, label, status]


def _rows(s, n):
    """(request, index within it, held, inside) of rows 0 .. n-1, and the row pointers."""
    ok, owner, have, want = _well_formed(s)
    m = torch.clamp(want - have, min=0)
    ends = torch.cumsum(m, 0)
    t = torch.arange(n, device="cuda")
    req = torch.searchsorted(ends, t, right=True)
    inside = req < m.numel()
    req = torch.clamp(req, max=m.numel() - 1)
    i = t - (ends - m)[req]
    return owner, have, want, ends, req, i, inside


def _slots_plain(s):
    pt = s["case"]["pt"]
    owner, have, want, ends, req, i, inside = _rows(s, s["slots"].numel())
    pos = have[req] + i
    page = s["table"].long()[req, torch.clamp(pos // pt, 0, s["width"] - 1)]
    fits = inside & (page >= 0) & (page < s["pages"])
    s["slots"].copy_(torch.where(fits, page * pt + pos % pt, -1))
    s["ints"][0].copy_(torch.where(inside, req, -1))
    s["ints"][1].copy_(torch.where(inside, pos, -1))
    s["ints"][2].copy_(torch.where(inside, owner[req], NONE))
    s["ptr"][0].fill_(0)
    s["ptr"][1:].copy_(ends)
    return [s["slots"], s["ints"], s["ptr"]]


def _segments_plain(s):
    c, pt = s["case"], s["case"]["pt"]
    ok, owner, have, want = _well_formed(s)
    blocks = (want + pt - 1) // pt
    ends = torch.cumsum(blocks, 0)
    n = s["page_table"].numel()
    e = torch.arange(n, device="cuda")
    per = torch.clamp(ends[-1], min=1)
    layer, k = e // per, e % per
    inside = layer * (ends[-1] > 0) < c["layers"]
    req = torch.clamp(torch.searchsorted(ends, k, right=True), max=blocks.numel() - 1)
    b = k - (ends - blocks)[req]
    page = s["table"].long()[req, torch.clamp(b, 0, s["width"] - 1)]
    there = inside & (page >= 0) & (page < s["pages"])
    token = 2 * 32 * 128 * 2
    size = torch.full_like(b, pt * token) if c["whole"] else torch.clamp(want[req] - b * pt, max=pt) * token
    zero = torch.zeros_like(b)
    s["segs"].copy_(torch.stack([owner[req], zero, zero, zero, size, zero, s["serial"].long()[req], layer, b, e], 1))
    s["page_table"].copy_(torch.where(there, layer * s["pages"] + page, -1))
    return [s["segs"], s["page_table"]]


def _views(s):
    c = s["case"]
    q, k, v = torch.split(s["qkv"], [c["q_heads"], c["heads"], c["heads"]], 1)
    return q, k, v


def _append_plain(s):
    c = s["case"]
    _, k, v = _views(s)
    slot, who, pt = s["slots"], s["row_owner"], c["pt"]
    n = s["pages"] * pt
    inside = (slot >= 0) & (slot < n)
    label = s["label"][torch.where(inside, slot // pt, 0)]
    st = torch.where(label <= NONE, UNOWNED, torch.where(label != who, OWNER_MISMATCH, 0))
    s["status"].copy_(torch.where(slot == -1, 0, torch.where(inside, st, BAD_DESC)))
    good = inside & (st == 0)
    flat = s["pool"].view(n, 2, c["heads"], c["dim"])
    rows = slot.numel()
    flat[slot[good]] = torch.stack([k[:rows], v[:rows]], 1)[good]
    return [s["pool"], s["status"]]


def _attention_plain(s):
    c, pt, rows, most = s["case"], s["case"]["pt"], s["rows"], s["most"]
    n, hk, hq, d = c["requests"], c["heads"], c["q_heads"], c["dim"]
    group, width = hq // hk, s["width"]
    owner, have, want, ends, req, i, _ = _rows(s, rows)
    table = s["table"].long()
    used = torch.arange(width, device="cuda")[None, :] < ((want + pt - 1) // pt)[:, None]
    inside = (table >= 0) & (table < s["pages"])
    label = s["label"].long()[torch.where(inside, table, 0)]
    bad = (used & ~inside).any(1)
    unowned = (used & inside & (label <= NONE)).any(1)
    foreign = (used & inside & (label >= 0) & (label != owner[:, None])).any(1)
    status = torch.where(bad, BAD_DESC, unowned * UNOWNED + foreign * OWNER_MISMATCH)
    # the context of every request, padded to the longest, and what of it each row sees
    kv = s["pool"][torch.where(used & inside, table, 0)].view(n, width * pt, 2, hk, d)
    pos = torch.arange(width * pt, device="cuda")[None, :]
    there = pos < want[:, None]
    key = torch.where(there[:, :, None, None], kv[:, :, 0], 0).float()
    val = torch.where(there[:, :, None, None], kv[:, :, 1], 0).float()
    del kv
    at = req * most + i
    q = torch.zeros((n * most, hq, d), device="cuda")
    q[at] = _views(s)[0].float()[:rows]
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
    q = q.view(n, most, hk, group, d).permute(0, 2, 3, 1, 4).reshape(n, hk, group * most, d)
    sc = torch.matmul(q, key.permute(0, 2, 3, 1)) * (1.0 / math.sqrt(d))
    del key
    sc = torch.where(seen[:, None, None], sc.view(n, hk, group, most, -1), -math.inf)
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
    s["out"][:rows].copy_(o)
    s["lse"][:rows].copy_(lse)
    s["status"].copy_(status)
    s["row_owner"][:rows].copy_(torch.where(status == 0, owner, CONFLICT)[req])
    return [s["out"][:rows], s["lse"][:rows], s["row_owner"][:rows], s["status"]]


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
    if op == "blocks":
        s["work"].copy_(s["start"])
        table, free, height, label, status = _parts(s)
        b = binding.Batch(s["owner"], s["have"], s["want"], table, c["pt"], s["pages"])
        ctx.block_tables(b, free, height, label, status, layers=c["layers"])
        return [table, free, height, label, status]
    b = binding.Batch(s["owner"], s["have"], s["want"], s["table"], c["pt"], s["pages"])
    if op == "slots":
        ctx.slot_map(b, s["slots"], row_req=s["ints"][0], row_pos=s["ints"][1], row_owner=s["ints"][2], row_ptr=s["ptr"])
        return [s["slots"], s["ints"], s["ptr"]]
    if op == "segments":
        ctx.kv_segments(b, s["serial"], s["segs"], s["page_table"], layers=c["layers"], token_bytes=2 * 32 * 128 * 2, whole_pages=c["whole"])
        return [s["segs"], s["page_table"]]
    q, k, v = _views(s)
    if op == "append":
        n = s["slots"].numel()
        ctx.kv_append(s["pool"], k[:n], v[:n], s["slots"], s["row_owner"], s["status"], owner_map=s["label"])
        return [s["pool"], s["status"]]
    rows = s["rows"]
    ctx.kv_attention(b, s["pool"], q[:rows], s["out"][:rows], s["status"], tree_mask=s["mask"], lse=s["lse"][:rows], row_owner=s["row_owner"][:rows],
                     owner_map=s["label"])
    return [s["out"][:rows], s["lse"][:rows], s["row_owner"][:rows], s["status"]]


def run(state):
    if own:
        return _own(state)
    return {"blocks": _blocks_plain, "slots": _slots_plain, "segments": _segments_plain, "append": _append_plain, "attention": _attention_plain}[state["case"]["op"]](state)


# --------------------------------------------------------------------------------- work and values

def work(case):
    have, want = _lengths(case)
    n, pt, op = case["requests"], case["pt"], case["op"]
    m = int(np.maximum(0, want - have).sum())
    if op == "blocks":
        grow, drop = (int(np.maximum(0, x).sum()) for x in (_up(want, pt) - _up(have, pt), _up(have, pt) - _up(want, pt)))
        # lengths, owners, status; per page its stack and table entry and its label in every layer, read and written
        return {"bytes": 16 * n + 8 + 8 * (grow + drop) * (1 + case["layers"]), "flops": 0}
    if op == "slots":
        entries = int((_up(want, pt) - have // pt)[want > have].sum())
        return {"bytes": 16 * n + 4 * entries + 20 * (m + case["pad"]), "flops": 0}
    if op == "segments":
        blocks = int(_up(want, pt).sum())
        return {"bytes": 16 * n + 4 * blocks + 44 * blocks * case["layers"], "flops": 0}
    row = case["heads"] * case["dim"] * 2 * 2
    if op == "append":
        return {"bytes": m * (2 * row + 16) + 4 * int(_up(want, pt).sum()), "flops": 0}
    io = m * case["q_heads"] * (case["dim"] * 2 * 2 + 4) + m * 4
    return {"bytes": int(want.sum()) * row + 8 * int(_up(want, pt).sum()) + io + 16 * n,
            "flops": 4.0 * float(((want - have) * want).sum()) * case["q_heads"] * case["dim"]}


def exact(case, seed):
    """The attention's rows and the appended pool, one request or row at a time; the other operators give whole numbers."""
    if case["op"] not in ("append", "attention"):
        return None
    s = prepare(case, seed)
    q, k, v = _views(s)
    if case["op"] == "append":
        pool, pt = s["pool"].clone(), case["pt"]
        for t, (slot, who) in enumerate(zip(s["slots"].tolist(), s["row_owner"].tolist())):
            pool[slot // pt, slot % pt, 0] = k[t]
            pool[slot // pt, slot % pt, 1] = v[t]
        return [pool, None]
    owner, have, want, table, label = (s[x].tolist() for x in ("owner", "have", "want", "table", "label"))
    rows, hq, d, pt = s["rows"], case["q_heads"], case["dim"], case["pt"]
    out = torch.zeros((rows, hq, d), dtype=torch.float64, device="cuda")
    lse = torch.full((rows, hq), -math.inf, dtype=torch.float64, device="cuda")
    t0 = 0
    for r in range(case["requests"]):
        m = max(0, want[r] - have[r])
        mine = table[r][: -(-want[r] // pt)]
        if m and all(0 <= p < s["pages"] and label[p] in (owner[r], PARAM) for p in mine):
            ctx = s["pool"][torch.tensor(mine, device="cuda")].reshape(-1, 2, case["heads"], d)[: want[r]].double()
            seen = torch.ones((m, want[r]), dtype=torch.bool, device="cuda")
            for i in range(m):
                if s["mask"] is None:
                    seen[i, have[r] + i + 1:] = False
                else:
                    bits = sum((w & 0xFFFFFFFF) << (32 * x) for x, w in enumerate(s["mask"][t0 + i].tolist()))
                    seen[i, have[r]:] = torch.tensor([bool(bits >> j & 1) for j in range(m)], device="cuda")
            for h in range(case["heads"]):
                g = slice(h * hq // case["heads"], (h + 1) * hq // case["heads"])
                z = torch.einsum("tgd,ld->gtl", q[t0:t0 + m, g].double(), ctx[:, 0, h]) / math.sqrt(d)
                z = z.masked_fill(~seen[None], -math.inf)
                l = torch.logsumexp(z, -1)
                lse[t0:t0 + m, g] = l.T
                p = torch.exp(z - l[:, :, None])
                out[t0:t0 + m, g] = torch.einsum("gtl,ld->tgd", torch.nan_to_num(p, nan=0.0), ctx[:, 1, h])
        t0 += m
    return [out, lse, None, None]
