"""The paged cache in 8 bits, one row, head and pair at a time: rows normed, turned, quantised and written, rows read back,
attention over the values.

Test infrastructure only: plain Python loops and 64-bit numpy, written from the definitions in the C header
(an e4m3 number is sign, 4 exponent bits with bias 7, 3 mantissa bits, no infinities, one NaN a sign).
"""
from __future__ import annotations

import math

import numpy as np

from . import paged as P

LEAST = 2.0 ** -126


def decode(code):
    """The value of an e4m3 code."""
    code = int(code)
    sign, e, m = -1.0 if code & 128 else 1.0, code >> 3 & 15, code & 7
    if code & 127 == 127:
        return math.nan
    return sign * (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))


VALUES = np.array([decode(c) for c in range(256)])


def step(x):
    """Distance of neighbouring e4m3 numbers around x (elementwise; up to 448)."""
    a = np.clip(np.abs(np.asarray(x, dtype=np.float64)), 2.0 ** -6, 448.0)
    return 2.0 ** (np.floor(np.log2(a)) - 3)


def nearest(x):
    """The e4m3 number nearest to x, the even one of two."""
    x = float(x)
    if math.isnan(x):
        return math.nan
    s = float(step(x))
    return math.copysign(min(round(abs(x) / s) * s, 448.0), x)       # round() takes the even one


def token_bytes(heads, dim):
    return -(-2 * heads * (dim + 4) // 16) * 16


def unpack(pages, heads, dim):
    """(codes' values [..., 2, heads, dim], scales [..., heads, 2], padding) of tokens as bytes [..., token_bytes]."""
    m = 2 * heads * dim
    raw = np.ascontiguousarray(pages)
    values = VALUES[raw[..., :m]].reshape(raw.shape[:-1] + (2, heads, dim))
    scales = np.ascontiguousarray(raw[..., m:m + 8 * heads]).view("<f4").reshape(raw.shape[:-1] + (heads, 2))
    return values, scales.astype(np.float64), raw[..., m + 8 * heads:]


def values(pages, heads, dim):
    """What the tokens stand for, in 64 bits [..., 2, heads, dim]."""
    codes, scales, _ = unpack(pages, heads, dim)
    with np.errstate(invalid="ignore"):
        return codes * np.swapaxes(scales, -1, -2)[..., None]


def quantised(x):
    """(codes' values, scale) of one head in 64 bits."""
    x = np.asarray(x, dtype=np.float64)
    if not np.isfinite(x).all():
        return np.zeros_like(x), math.nan
    scale = max(np.abs(x).max() / 448.0, LEAST)
    return np.array([nearest(v / scale) for v in x]), scale


def turned(x, weight, eps, pos, freq, sections, paired):
    """One head x in 64 bits: normed (weight or None), its pairs turned; pos: one position per axis."""
    x = np.asarray(x, dtype=np.float64)
    if weight is not None:
        x = x * np.asarray(weight, dtype=np.float64) / math.sqrt((x * x).mean() + eps)
    y = x.copy()
    pair = 0
    for axis, count in enumerate(sections or []):
        for _ in range(count):
            a, b = (2 * pair, 2 * pair + 1) if paired else (pair, len(freq) + pair)
            angle = float(pos[axis]) * float(freq[pair])
            y[a], y[b] = x[a] * math.cos(angle) - x[b] * math.sin(angle), x[b] * math.cos(angle) + x[a] * math.sin(angle)
            pair += 1
    return y


def read_status(slots, row_owner, owner_map, n_pages, page_tokens):
    """Per row: (status, whether it is read)."""
    st = np.zeros(len(slots), dtype=np.uint32)
    for t, slot in enumerate(slots):
        slot = int(slot)
        if slot == -1:
            continue
        if not 0 <= slot < n_pages * page_tokens:
            st[t] = P.BAD_DESC
        elif owner_map is not None:
            label = int(owner_map[slot // page_tokens])
            if label in (P.NONE, P.CONFLICT):
                st[t] = P.UNOWNED
            elif label not in (P.PARAM, int(row_owner[t])):
                st[t] = P.OWNER_MISMATCH
    return st, (st == 0) & (np.asarray(slots) != -1)


def scores(q, keys, positions, x, scale, softcap=0.0, slope=None):
    """Scores of one query row at position x with keys at positions, in 64 bits."""
    s = keys @ q * scale
    if softcap:
        s = softcap * np.tanh(s / softcap)
    if slope is not None:
        s = s + slope * (positions - x)
    return s


def attention(owner, have, want, table, pages, heads, q, scale, tree_mask=None, owner_map=None, softcap=0.0, window=0, slopes=None):
    """dict(out float64 [rows, heads, dim], lse, row_owner, status, total) over pages as bytes."""
    n, width = table.shape
    n_pages, pt, _ = pages.shape
    hq, d = q.shape[1:]
    kv = values(pages, heads, d)
    group = hq // heads
    shapes = [P.shape(owner[r], have[r], want[r], pt, width) for r in range(n)]
    total = sum(max(0, s[2] - s[1]) for s in shapes)
    if total > q.shape[0]:
        return dict(status=np.full(n, P.BAD_TABLE, np.uint32), out=None, lse=None, row_owner=None, total=total)
    status = np.zeros(n, dtype=np.uint32)
    out, lse, row_owner = np.zeros((total, hq, d)), np.full((total, hq), -np.inf), np.full(total, P.CONFLICT, dtype=np.int32)
    t0 = 0
    for r, (ok, h, w, _, bw) in enumerate(shapes):
        m = max(0, w - h)
        if not ok:
            status[r] = P.BAD_DESC
        if m == 0:
            continue
        low = max(0, h - window + 1) if window else 0
        for b in range(low // pt, bw):
            page = int(table[r, b])
            if not 0 <= page < n_pages:
                status[r] |= P.BAD_DESC
            elif owner_map is not None:
                label = int(owner_map[page])
                if label in (P.NONE, P.CONFLICT):
                    status[r] |= P.UNOWNED
                elif label not in (P.PARAM, int(owner[r])):
                    status[r] |= P.OWNER_MISMATCH
        if tree_mask is not None and m > 32 * tree_mask.shape[1]:
            status[r] |= P.BAD_DESC
        if status[r] & P.BAD_DESC:
            status[r] = P.BAD_DESC
        if status[r]:
            t0 += m
            continue
        for i in range(m):
            row_owner[t0 + i] = owner[r]
            sees = [t for t in range(low, h) if not window or t > h + i - window]
            for j in range(m):
                if (j <= i and (not window or j > i - window)) if tree_mask is None else (int(tree_mask[t0 + i, j // 32]) >> (j % 32)) & 1:
                    sees.append(h + j)
            if not sees:
                continue
            at = np.array(sees)
            mine = kv[table[r, at // pt], at % pt]                              # [tokens, 2, heads, d]
            for x in range(hq):
                with np.errstate(invalid="ignore", over="ignore"):
                    s = scores(q[t0 + i, x], mine[:, 0, x // group], at, h + i, scale, softcap, None if slopes is None else float(slopes[x]))
                    top = s.max()
                    if top == -np.inf:
                        continue
                    p = np.exp(s - top)
                    out[t0 + i, x] = (p[:, None] * mine[:, 1, x // group]).sum(0) / p.sum()
                    lse[t0 + i, x] = top + math.log(p.sum()) if np.isfinite(top) else np.nan
        t0 += m
    return dict(out=out, lse=lse, row_owner=row_owner, status=status, total=total)
