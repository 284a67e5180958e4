"""The bounds that GPU results are held to: a result with the roundings that are meant stays inside them, one with a
rounding too many does not (no GPU needed: the mistakes are made in the 64-bit computation)."""
import numpy as np
import pytest
import torch

import kv_bounds as B


def rounded(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).double().numpy()


def attend(x, scale, p_type, o_type, lse_off=0.0):
    """The step in 64 bits but for its weights' and results' types."""
    pool, q = x["pool"].double().numpy(), x["q"].double().numpy()
    group = q.shape[1] // pool.shape[3]
    out, lse = np.zeros(q.shape), np.full(q.shape[:2], -np.inf)
    for t, req, at in B.visible(x):
        kv = pool[x["table"][req][at // x["pt"]], at % x["pt"]]
        for h in range(q.shape[1]):
            z = kv[:, 0, h // group] @ q[t, h] * scale
            p = np.exp(z - z.max())
            out[t, h] = rounded(rounded(p, p_type) @ kv[:, 1, h // group] / p.sum(), o_type)
            lse[t, h] = z.max() + np.log(p.sum()) + lse_off
    return out, lse


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("dim", [64, 128])
def test_bounds(dtype, dim):
    x = B.step(5, dtype, [40, 0, 130, 7], [5, 9, 3, 20], 2, 4, dim, 16)
    scale = float(np.float32(dim ** -0.5))
    r = B.bounds(x, scale)
    out, lse = attend(x, scale, dtype, dtype)
    assert B.worst(out, r["out"], r["out_tol"]) <= 1 and B.worst(lse, r["lse"], r["lse_tol"]) <= 1
    assert B.worst(attend(x, scale, dtype, dtype, 3e-3)[1], r["lse"], r["lse_tol"]) > 1
    if dtype == torch.float16:
        for p_type, o_type in ((torch.bfloat16, dtype), (dtype, torch.bfloat16)):
            assert B.worst(attend(x, scale, p_type, o_type)[0], r["out"], r["out_tol"]) > 1
    else:
        # a type of 8 bits, and a result that was rounded twice as coarsely
        assert B.worst(attend(x, scale, torch.float8_e4m3fn, dtype)[0], r["out"], r["out_tol"]) > 1
        assert B.worst(attend(x, scale, dtype, torch.float8_e4m3fn)[0], r["out"], r["out_tol"]) > 1
