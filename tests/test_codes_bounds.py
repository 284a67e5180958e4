"""The bounds of codes_bounds on the CPU: what a right computation does stays inside, a rounding too many does not."""
import numpy as np
import pytest
import torch

import codes_bounds as B
from oracle import paged8 as E


def computed(x, scale, drop=None):
    """Attention as the kernels do it, in numpy: 32-bit scores, weights in fp16 (or cut to `drop`'s type), one rounding at the end."""
    q = x["q"].double().numpy()
    rows, hq, d = q.shape
    codes, scales, _ = E.unpack(x["pool"], x["heads"], d)
    out = np.zeros(q.shape)
    t = 0
    for k, (h, w) in enumerate(zip(x["have"], x["want"])):
        for i in range(w - h):
            at = np.arange(h + i + 1)
            c, s = codes[x["table"][k][at // x["pt"]], at % x["pt"]], scales[x["table"][k][at // x["pt"]], at % x["pt"]]
            for y in range(hq):
                g = y // (hq // x["heads"])
                z = (c[:, 0, g] @ q[t, y] * s[:, g, 0] * scale).astype(np.float32).astype(np.float64)
                p = np.exp(z - z.max())
                weight = torch.from_numpy(p * s[:, g, 1] / (p * s[:, g, 1]).max() * 256).to(drop or torch.float16).double().numpy()
                o = weight @ c[:, 1, g] / 256 * (p * s[:, g, 1]).max() / p.sum()
                out[t, y] = torch.from_numpy(o).to(x["q"].dtype).double().numpy()
            t += 1
    return out


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_bounds_hold_and_catch(dtype):
    x = B.step(1, dtype, [60, 3], [2, 4], 2, 2, 64, 16)
    b = B.bounds(x, 0.125)
    assert B.worst(computed(x, 0.125), b["out"], b["out_tol"]) <= 1
    if dtype == torch.float16:
        assert B.worst(computed(x, 0.125, torch.bfloat16), b["out"], b["out_tol"]) > 1
    assert B.worst(computed(x, 0.13), b["out"], b["out_tol"]) > 1
    y = dict(x, q=x["q"].float().to(torch.float8_e4m3fn).to(dtype))
    assert B.worst(computed(y, 0.125), b["out"], b["out_tol"]) > 1


def test_bounds_agree_with_the_oracle():
    x = B.step(2, torch.float16, [20, 0], [3, 5], 1, 3, 64, 8, tree=True)
    b = B.bounds(x, 0.2, softcap=4.0)
    r = E.attention(x["owner"], x["have"], x["want"], x["table"], x["pool"], 1, x["q"].double().numpy(), 0.2, x["mask"], x["label"], softcap=4.0)
    assert not r["status"].any() and np.allclose(r["out"], b["out"], rtol=1e-12) and np.allclose(r["lse"], b["lse"], rtol=1e-12)
    x = B.step(3, torch.float16, [20, 0], [3, 5], 1, 2, 64, 8)
    slopes = np.array([0.5, 0.1], np.float32)
    b = B.bounds(x, 0.2, window=6, slopes=slopes)
    r = E.attention(x["owner"], x["have"], x["want"], x["table"], x["pool"], 1, x["q"].double().numpy(), 0.2, None, x["label"], window=6, slopes=slopes)
    assert not r["status"].any() and np.allclose(r["out"], b["out"], rtol=1e-12) and np.allclose(r["lse"], b["lse"], rtol=1e-12)
