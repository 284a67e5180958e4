"""The paged cache's tables, appends and attention, one request, page and token at a time.

Test infrastructure only: plain Python loops and 64-bit numpy, written from the definitions
(paper sec. 4.2: a KV block is an ownership record; sec. 4.3 step 5: the attention rule joins the
labels of the blocks that a request's block table names; sec. 4.5: index tables).
"""
from __future__ import annotations

import math

import numpy as np

PARAM, NONE, CONFLICT = -1, -2, -3
OWNER_MISMATCH, UNOWNED, BAD_DESC, NO_BLOCKS, BAD_TABLE = 2, 4, 16, 64, 128
MAX_OWNER = 1 << 20


def shape(owner, have, want, page_tokens, max_blocks):
    """(well formed, have, want, blocks before, blocks after) of one request."""
    owner, have, want = int(owner), int(have), int(want)
    ok = 0 <= owner < MAX_OWNER and have >= 0 and want >= 0
    bh, bw = -(-have // page_tokens), -(-want // page_tokens)
    if not ok or bh > max_blocks or bw > max_blocks:
        return False, 0, 0, 0, 0
    return True, have, want, bh, bw


def block_tables(owner, have, want, table, page_tokens, n_pages, free_pages, n_free, owner_map):
    """New (table, free_pages, n_free, owner_map [layers, n_pages], status)."""
    n, width = table.shape
    new_table, new_free, new_map = table.copy(), free_pages.copy(), owner_map.copy()
    status = np.zeros(n, dtype=np.uint32)
    refuse = (table, free_pages, n_free, owner_map, np.full(n, BAD_TABLE, dtype=np.uint32))
    if n_free < 0 or n_free > len(free_pages):
        return refuse
    shapes = [shape(owner[r], have[r], want[r], page_tokens, width) for r in range(n)]
    taken, given, asked = [], [], 0
    for r, (ok, _, _, bh, bw) in enumerate(shapes):
        if not ok:
            status[r] = BAD_DESC
        elif bw > bh:
            asked += bw - bh
            if asked > n_free:
                status[r] = NO_BLOCKS
            else:
                taken += [(r, j) for j in range(bh, bw)]
        else:
            given += [(r, j) for j in range(bw, bh)]
    height = n_free
    moves = []
    for r, j in taken:
        height -= 1
        moves.append((int(free_pages[height]), r, True))
        new_table[r, j] = free_pages[height]
    if height + len(given) > len(free_pages):
        return refuse
    for r, j in given:
        moves.append((int(table[r, j]), r, False))
        new_table[r, j] = -1
        new_free[height] = table[r, j]
        height += 1
    seen = set()
    for page, r, take in moves:
        if not 0 <= page < n_pages or page in seen:
            return refuse
        seen.add(page)
        for layer in range(owner_map.shape[0]):
            label = int(owner_map[layer, page])
            if label not in ((NONE,) if take else (int(owner[r]), NONE, CONFLICT)):
                return refuse
            new_map[layer, page] = owner[r] if take else NONE
    return new_table, new_free, height, new_map, status


def slot_map(owner, have, want, table, page_tokens, n_pages, n_rows, rel=None):
    """dict(slots, req, pos, owner, ptr, total)."""
    n, width = table.shape
    out = dict(slots=np.full(n_rows, -1, np.int64), req=np.full(n_rows, -1, np.int32), pos=np.full(n_rows, -1, np.int32),
               owner=np.full(n_rows, NONE, np.int32), ptr=np.zeros(n + 1, np.int32), total=0)
    rows = []
    ptr = [0]
    for r in range(n):
        ok, h, w, _, _ = shape(owner[r], have[r], want[r], page_tokens, width)
        rows += [(r, i, h, max(0, w - h)) for i in range(max(0, w - h))]
        ptr.append(len(rows))
    out["total"] = len(rows)
    if len(rows) > n_rows:
        return out
    out["ptr"][:] = ptr
    for t, (r, i, h, m) in enumerate(rows):
        out["req"][t], out["owner"][t] = r, owner[r]
        if rel is not None:
            i = int(rel[t])
        if 0 <= i < m:
            p = h + i
            out["pos"][t] = p
            page = int(table[r, p // page_tokens])
            if 0 <= page < n_pages:
                out["slots"][t] = page * page_tokens + p % page_tokens
    return out


def kv_segments(owner, have, want, table, page_tokens, n_pages, serial, layers, token_bytes, cap, seg_dtype,
                whole_pages=False, new_blocks=False):
    """(segs, page_table, total)."""
    n, width = table.shape
    entries = []
    for r in range(n):
        ok, h, w, _, bw = shape(owner[r], have[r], want[r], page_tokens, width)
        first = h // page_tokens if new_blocks else 0
        if new_blocks and w <= h:
            continue
        for b in range(first, bw):
            tokens = page_tokens if whole_pages else min(page_tokens, w - b * page_tokens)
            entries.append((r, b, tokens * token_bytes))
    segs = np.zeros(cap, dtype=seg_dtype)
    segs["owner"], segs["flags"], segs["page0"] = NONE, 1, np.arange(cap)
    page_table = np.full(cap, -1, dtype=np.int32)
    total = len(entries) * layers
    if total <= cap:
        e = 0
        for layer in range(layers):
            for r, b, size in entries:
                segs["owner"][e], segs["flags"][e], segs["len"][e] = owner[r], 0, size
                segs["nonce"][e] = np.frombuffer(np.array([serial[r], layer, b], dtype="<u4").tobytes(), dtype=np.uint8)
                page = int(table[r, b])
                if 0 <= page < n_pages:
                    page_table[e] = layer * n_pages + page
                e += 1
    return segs, page_table, total


def append_status(slots, row_owner, owner_map, n_pages, page_tokens):
    """Per row: (status, written)."""
    st = np.zeros(len(slots), dtype=np.uint32)
    for t, slot in enumerate(slots):
        slot = int(slot)
        if slot == -1:
            continue
        if not 0 <= slot < n_pages * page_tokens:
            st[t] = BAD_DESC
        elif owner_map is not None:
            label = int(owner_map[slot // page_tokens])
            if label in (NONE, CONFLICT):
                st[t] = UNOWNED
            elif label != int(row_owner[t]) or label < 0:
                st[t] = OWNER_MISMATCH
    return st, (st == 0) & (np.asarray(slots) != -1)


def attention(owner, have, want, table, pages, q, scale, tree_mask=None, owner_map=None, n_rows=None):
    """dict(out float64 [rows, heads, dim], lse, row_owner, status); pages float64 [n_pages, page_tokens, 2, heads, dim].

    status is BAD_TABLE for every request (and the rest None) if the step has more rows than q."""
    n, width = table.shape
    n_pages, pt, _, hk, d = pages.shape
    hq = q.shape[1]
    group = hq // hk
    shapes = [shape(owner[r], have[r], want[r], pt, width) for r in range(n)]
    total = sum(max(0, s[2] - s[1]) for s in shapes)
    status = np.zeros(n, dtype=np.uint32)
    if total > q.shape[0]:
        return dict(status=np.full(n, BAD_TABLE, np.uint32), out=None, lse=None, row_owner=None, total=total)
    out = np.zeros((total, hq, d))
    lse = np.full((total, hq), -np.inf)
    row_owner = np.full(total, CONFLICT, dtype=np.int32)
    t0 = 0
    for r, (ok, h, w, bh, bw) in enumerate(shapes):
        m = max(0, w - h)
        if not ok:
            status[r] = BAD_DESC
        if m == 0:
            continue
        for b in range(bw):
            page = int(table[r, b])
            if not 0 <= page < n_pages:
                status[r] |= BAD_DESC
            elif owner_map is not None:
                label = int(owner_map[page])
                if label in (NONE, CONFLICT):
                    status[r] |= UNOWNED
                elif label not in (PARAM, int(owner[r])):
                    status[r] |= OWNER_MISMATCH
        if tree_mask is not None and m > 32 * tree_mask.shape[1]:
            status[r] |= BAD_DESC
        if status[r] & BAD_DESC:
            status[r] = BAD_DESC
        if status[r]:
            t0 += m
            continue
        where = [(int(table[r, p // pt]), p % pt) for p in range(w)]
        kv = np.stack([pages[a, b] for a, b in where])                       # [w, 2, hk, d]
        for i in range(m):
            row_owner[t0 + i] = owner[r]
            sees = list(range(h))
            for j in range(m):
                if (j <= i) if tree_mask is None else (int(tree_mask[t0 + i, j // 32]) >> (j % 32)) & 1:
                    sees.append(h + j)
            if not sees:
                continue
            for x in range(hq):
                s = kv[sees, 0, x // group] @ q[t0 + i, x] * scale
                top = s.max()
                if top == -np.inf:
                    continue
                with np.errstate(invalid="ignore", over="ignore"):
                    p = np.exp(s - top)
                    out[t0 + i, x] = (p[:, None] * kv[sees, 1, x // group]).sum(0) / p.sum()
                    lse[t0 + i, x] = top + math.log(p.sum()) if np.isfinite(top) else np.nan
        t0 += m
    return dict(out=out, lse=lse, row_owner=row_owner, status=status, total=total)
