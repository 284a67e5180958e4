"""Numbers that do not fit the C-ABI's types are refused by the binding (no GPU needed: nothing is reached)."""
import types

import pytest
import torch

from paper_2608_25431_b200 import binding


def fake_tensor(n, shape=None):
    """What the checks ask of a tensor, on a GPU that is not there."""
    return types.SimpleNamespace(numel=lambda: n, get_device=lambda: 0, dim=lambda: len(shape or (n,)), shape=shape or (n,), dtype=torch.int32,
                                 is_contiguous=lambda: True, data_ptr=lambda: 0x10000, element_size=lambda: 4)


def batch(page_tokens=16, n_pages=8):
    t = fake_tensor(4)
    return binding.Batch(t, t, t, fake_tensor(8, (4, 2)), page_tokens, n_pages)


def test_batches():
    assert batch().c.page_tokens == 16
    for kw in (dict(page_tokens=2 ** 32 + 16), dict(n_pages=2 ** 32 + 8)):
        with pytest.raises(ValueError, match="does not fit"):
            batch(**kw)


def ctx():
    c = binding.Ctx.__new__(binding.Ctx)
    c._h, c.device = None, 0
    return c


@pytest.mark.parametrize("layers,token", [(2 ** 32 + 1, 64), (-1, 64), (1, 2 ** 64 + 64), (1, -64)])
def test_layers_and_token_bytes(layers, token):
    with pytest.raises(ValueError, match="does not fit"):
        ctx().kv_segments(batch(), fake_tensor(4), fake_tensor(100), fake_tensor(10), layers, token, stream=0)
    if layers != 1:
        with pytest.raises(ValueError, match="does not fit"):
            ctx().block_tables(batch(n_pages=0), fake_tensor(8), fake_tensor(1), fake_tensor(8), fake_tensor(4), layers=layers, stream=0)


@pytest.mark.parametrize("ns", [-1, 2 ** 64 + 1])
def test_wait_limits(ns):
    with pytest.raises(ValueError, match="does not fit"):
        ctx().wait_limit(ns)
