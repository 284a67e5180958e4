"""Inputs of small attention steps on the host, and bounds on a result's error from the arithmetic alone.

Per row and head, with e = torch.finfo(type).eps / 2 (half a step of the pool's type), n visible tokens in T tiles
of 64, S = max over them of sum |q k|, A = sum p |v| / sum p:
 - a score is a 32-bit sum of D exact products, an addition off by at most 2^-23 of S (the matrix instructions may cut
   off instead of rounding); scale * log2(e) and the product with it take three roundings, the maximum's subtraction one
   of a difference of up to 2 scale S:  s = scale S (D + 4) 2^-23, in natural units;
 - exp2 is off by 2^-21 at most; a rescaling by a new maximum is one more of them, so is a join: x = (T + 4) 2^-21;
 - lse:  s + x + n 2^-24 + 2^-22 |lse|
 - a weight's relative error moves the quotient by at most twice itself times A; rounding to the pool's type (only
   in the numerator) by e A, the 32-bit sum over tokens by n 2^-23 A, the result's rounding by e |o|:
   out:  e |o| + (e + 2 s + 2 x + n 2^-23) A
   and for fp16 n 2^-25 max |v| (weights below 2^-14 lose up to 2^-25 each, and the weights' sum is at least 1) and
   2^-25 (the result's smallest step)."""
import numpy as np
import torch

from oracle import paged as P


def step(seed, dtype, have, new, heads, group, dim, pt, tree=True):
    """A step with scattered pages and a tree of drafted tokens, on the host."""
    rng = np.random.default_rng(seed)
    have, new = np.array(have, np.int32), np.array(new, np.int32)
    want, n = have + new, len(have)
    blocks = -(-want // pt)
    pages = int(blocks.sum()) + 3
    perm = rng.permutation(pages).astype(np.int32)
    table = np.full((n, int(blocks.max())), -1, np.int32)
    table[np.arange(table.shape[1])[None, :] < blocks[:, None]] = perm[: int(blocks.sum())]
    owner = np.arange(n, dtype=np.int32)
    label = np.full(pages, P.NONE, np.int32)
    for r in range(n):
        label[table[r, : blocks[r]]] = owner[r]
    g = torch.Generator().manual_seed(seed)
    rows = int(new.sum())
    pool = torch.randn((pages, pt, 2, heads, dim), generator=g).to(dtype)
    q = torch.randn((rows, heads * group, dim), generator=g).to(dtype)
    mask = None
    if tree:
        mask, t = np.zeros((rows, -(-int(new.max()) // 32)), np.uint32), 0
        for r in range(n):
            for i in range(new[r]):
                up = int(rng.integers(-1, i)) if i else -1
                if up >= 0:
                    mask[t + i] = mask[t + up]
                mask[t + i, i // 32] |= np.uint32(1 << (i % 32))
            t += int(new[r])
    return dict(owner=owner, have=have, want=want, table=table, label=label, pool=pool, q=q, mask=mask, pt=pt, rows=rows)


def visible(x):
    """Per row: (request, positions that it sees)."""
    t = 0
    for r, (h, w) in enumerate(zip(x["have"], x["want"])):
        for i in range(max(0, w - h)):
            own = [h + j for j in range(w - h) if ((j <= i) if x["mask"] is None else (int(x["mask"][t, j // 32]) >> (j % 32)) & 1)]
            yield t, r, np.array(list(range(h)) + own, dtype=np.int64)
            t += 1


def bounds(x, scale):
    """dict(out, lse: 64-bit values; out_tol, lse_tol: how far a result may be off them)."""
    pool, q = x["pool"].double().cpu().numpy(), x["q"].double().cpu().numpy()
    rows, hq, d = q.shape
    group = hq // pool.shape[3]
    e = torch.finfo(x["q"].dtype).eps / 2
    scale = float(np.float32(scale))
    r = dict(out=np.zeros(q.shape), lse=np.full((rows, hq), -np.inf), out_tol=np.zeros(q.shape), lse_tol=np.zeros((rows, hq)))
    for t, req, at in visible(x):
        if len(at) == 0:
            continue
        kv = pool[x["table"][req][at // x["pt"]], at % x["pt"]]                  # [n, 2, heads, d]
        tiles = -(-int(x["want"][req]) // 64)
        for h in range(hq):
            k, v = kv[:, 0, h // group], kv[:, 1, h // group]
            z = k @ q[t, h] * scale
            p = np.exp(z - z.max())
            o = p @ v / p.sum()
            lse = z.max() + np.log(p.sum())
            s = abs(scale) * (np.abs(k) @ np.abs(q[t, h])).max() * (d + 4) * 2.0 ** -23
            a = p @ np.abs(v) / p.sum()
            err = (tiles + 4) * 2.0 ** -21
            tol = e * np.abs(o) + (e + 2 * s + 2 * err + len(at) * 2.0 ** -23) * a
            if x["q"].dtype == torch.float16:
                tol = tol + len(at) * 2.0 ** -25 * np.abs(v).max() + 2.0 ** -25
            r["out"][t, h], r["out_tol"][t, h] = o, tol
            r["lse"][t, h], r["lse_tol"][t, h] = lse, s + err + len(at) * 2.0 ** -24 + 2.0 ** -22 * abs(lse)
    return r


def worst(got, want, tol):
    """Largest error as a share of what is allowed."""
    return float((np.abs(got - want) / np.maximum(tol, 1e-300)).max())
