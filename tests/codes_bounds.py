"""Steps over 8-bit pages on the host, and bounds on what a call may return, from the arithmetic alone.

Rows that are written (u = 2^-24, half a 32-bit step; D = head_dim):
 - the norm's mean is a sum of D squares, off by D u at most, its root and reciprocal by 2^-22 more; a weight's and the norm's
   products are two roundings, so a normed element is off by n = D u / 2 + 2^-21 of itself
 - an angle's fraction of a turn is rounded to 2^-24 of half a turn: the angle is off by pi 2^-24, sine and cosine by that and 2^-22 (two
   steps): an element of a pair (a, b) by (|a| + |b|) (n + 2^-20), with the products' roundings
 - q is rounded once: half a step of its type
 - a scale is max / 448 with two roundings, and the elements' error: relative 2^-22 + d, d = max of the errors over max
 - a code is the nearest to x / scale: half an e4m3 step of it, moved by (error of x) / scale + |x / scale| (2^-22 + d)
Rows that are read: code * scale is rounded to 32 bits (u) and to the type (half a step).

Attention, per row and head, with e half a step of the result's type, n visible tokens, S the largest sum |q k| (k a value), scale s,
w_t = p_t * (V's scale):
 - a score: a 32-bit sum of D exact products (a step of 2^-23 of S each), four factors and roundings of s; capped: the tanh's
   error is 2^-21 of the cap and of itself; the bias one rounding of itself and one of the sum:
   z = |s| S (D + 8) 2^-23 + cap 2^-20 + bias 2^-23 (in natural units)
 - exp2 is off by 2^-21; the maximum in use may change with every tile and at joins: x = (n / 16 + 8) 2^-21
 - lse: z + x + n 2^-23 + 2^-22 |lse|
 - a weight w_t is rounded to fp16: 2^-11 of itself, or, far below the largest weight W so far, half of the smallest fp16 step in units in
   which W is at least 2^7: 2^-32 W
 - out: e |o| + (2^-11 + 2 z + 2 x + n 2^-23) A + n 2^-32 448 W / sum p + the result type's smallest step, with A = sum p |v| / sum p"""
import numpy as np
import torch

from oracle import paged as P, paged8 as E

U = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def smallest(dtype):
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


def pages_of(x):
    """Bytes of tokens that hold x (float64 [..., 2, heads, dim], exactly representable or not) quantised by the oracle's rule, vectorised."""
    heads, dim = x.shape[-2:]
    flat = x.reshape(-1, 2, heads, dim)
    scale = np.maximum(np.abs(flat).max(-1) / 448.0, E.LEAST).astype(np.float32)
    codes = torch.from_numpy(flat / scale.astype(np.float64)[..., None]).float().clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    out = np.zeros((flat.shape[0], E.token_bytes(heads, dim)), np.uint8)
    m = 2 * heads * dim
    out[:, :m] = codes.reshape(-1, m)
    out[:, m:m + 8 * heads] = np.ascontiguousarray(scale.transpose(0, 2, 1)).view(np.uint8).reshape(-1, 8 * heads)
    return out.reshape(x.shape[:-3] + (-1,))


def step(seed, dtype, have, new, heads, group, dim, pt, tree=False, spare=4):
    """A step with scattered pages on the host: what is cached and drafted lies in the pages already."""
    rng = np.random.default_rng(seed)
    have, new = np.array(have, np.int32), np.array(new, np.int32)
    want, n = have + new, len(have)
    blocks = -(-want // pt)
    pages = int(blocks.sum()) + spare
    table = np.full((n, max(1, int(blocks.max()))), -1, np.int32)
    table[np.arange(table.shape[1])[None, :] < blocks[:, None]] = rng.permutation(pages).astype(np.int32)[: int(blocks.sum())]
    owner = rng.permutation(60)[:n].astype(np.int32)
    label = np.full(pages, P.NONE, np.int32)
    for r in range(n):
        label[table[r, : blocks[r]]] = owner[r]
    rows = int(new.sum())
    pool = pages_of(rng.standard_normal((pages, pt, 2, heads, dim)))
    q = torch.from_numpy(rng.standard_normal((rows, heads * group, dim))).to(dtype)
    mask = None
    if tree:
        mask, t = np.zeros((rows, max(1, -(-int(new.max()) // 32))), np.uint32), 0
        for r in range(n):
            for i in range(new[r]):
                up = int(rng.integers(-1, i)) if i else -1
                if up >= 0:
                    mask[t + i] = mask[t + up]
                mask[t + i, i // 32] |= np.uint32(1 << (i % 32))
            t += int(new[r])
    return dict(owner=owner, have=have, want=want, table=table, label=label, pool=pool, heads=heads, q=q, mask=mask, pt=pt, rows=rows)


def bounds(x, scale, softcap=0.0, window=0, slopes=None):
    """dict(out, lse, out_tol, lse_tol) of a step whose requests are all served."""
    q = x["q"].double().numpy()
    rows, hq, d = q.shape
    heads, group, pt = x["heads"], hq // x["heads"], x["pt"]
    codes, scales, _ = E.unpack(x["pool"], heads, d)
    e, least = half_step(x["q"].dtype), smallest(x["q"].dtype)
    r = dict(out=np.zeros(q.shape), lse=np.full((rows, hq), -np.inf), out_tol=np.zeros(q.shape), lse_tol=np.zeros((rows, hq)))
    t = 0
    for k, (h, w) in enumerate(zip(x["have"], x["want"])):
        for i in range(max(0, w - h)):
            pos = h + i
            own = [h + j for j in range(w - h) if ((j <= i) if x["mask"] is None else (int(x["mask"][t, j // 32]) >> (j % 32)) & 1)]
            at = np.array([p for p in list(range(h)) + own if not window or p > pos - window], dtype=np.int64)
            if len(at):
                c, s = codes[x["table"][k][at // pt], at % pt], scales[x["table"][k][at // pt], at % pt]
                for y in range(hq):
                    g = y // group
                    key, val = c[:, 0, g] * s[:, g, :1], c[:, 1, g] * s[:, g, 1:]
                    slope = None if slopes is None else float(slopes[y])
                    z = E.scores(q[t, y], key, at, pos, scale, softcap, slope)
                    p = np.exp(z - z.max())
                    o, lse = p @ val / p.sum(), z.max() + np.log(p.sum())
                    err = abs(scale) * (np.abs(key) @ np.abs(q[t, y])).max() * (d + 8) * 2.0 ** -23 + softcap * 2.0 ** -20
                    err += 0.0 if slope is None else abs(slope) * float(np.abs(at - pos).max()) * 2.0 ** -23
                    n, ex = len(at), (len(at) / 16 + 8) * 2.0 ** -21
                    a, big = p @ np.abs(val) / p.sum(), float((p * s[:, g, 1]).max())
                    r["out"][t, y], r["lse"][t, y] = o, lse
                    r["out_tol"][t, y] = e * np.abs(o) + (2.0 ** -11 + 2 * err + 2 * ex + n * 2.0 ** -23) * a + n * 2.0 ** -32 * 448 * big / p.sum() + least
                    r["lse_tol"][t, y] = err + ex + n * 2.0 ** -23 + 2.0 ** -22 * abs(lse)
            t += 1
    return r


def worst(got, want, tol):
    """Largest error as a share of what is allowed."""
    return float((np.abs(got - want) / np.maximum(tol, 1e-300)).max()) if got.size else 0.0
