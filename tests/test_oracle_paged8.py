"""The oracle of the 8-bit cache, pinned by hand-computed cases."""
import math

import numpy as np
import pytest
import torch

from oracle import paged as P, paged8 as E


def test_codes_have_the_values_of_their_format():
    assert [E.decode(c) for c in (0x00, 0x01, 0x07, 0x08, 0x38, 0x39, 0x7E, 0xFE, 0xB8)] == \
        [0.0, 2.0 ** -9, 7 * 2.0 ** -9, 2.0 ** -6, 1.0, 1.125, 448.0, -448.0, -1.0]
    assert math.isnan(E.decode(0x7F)) and math.isnan(E.decode(0xFF))
    theirs = torch.arange(256, dtype=torch.int16).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.nan_to_num(E.VALUES, nan=1e9), np.nan_to_num(theirs, nan=1e9))


def test_nearest_code():
    # 1 and 1.125 are neighbours; 1.0625 lies between them, the even one is 1; 1.1875 goes up to the even 1.25
    assert [E.nearest(x) for x in (1.0, 1.06, 1.0625, 1.063, 1.1875, -1.1875, 500.0, 2.0 ** -10, 3 * 2.0 ** -11)] == \
        [1.0, 1.0, 1.0, 1.125, 1.25, -1.25, 448.0, 0.0, 2.0 ** -9]
    x = np.linspace(-460, 460, 5001)
    theirs = torch.from_numpy(x).float().clamp(-448, 448).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal([E.nearest(np.float32(v)) for v in x], theirs)


def test_a_head_quantised():
    codes, scale = E.quantised([896.0, -2.0, 0.0, 1.0])
    assert scale == 2.0 and codes.tolist() == [448.0, -1.0, 0.0, 0.5]
    codes, scale = E.quantised([0.0, 0.0])
    assert scale == 2.0 ** -126 and codes.tolist() == [0.0, 0.0]
    codes, scale = E.quantised([1.0, math.inf])
    assert math.isnan(scale) and codes.tolist() == [0.0, 0.0]


@pytest.mark.parametrize("heads, dim, size", [(8, 128, 2112), (1, 64, 144), (3, 80, 512), (32, 128, 8448)])
def test_size_of_a_token(heads, dim, size):
    assert E.token_bytes(heads, dim) == size


def test_a_token_unpacked():
    raw = np.zeros((1, E.token_bytes(1, 16)), dtype=np.uint8)                     # K 16, V 16, two scales, 8 of padding
    raw[0, 0], raw[0, 17], raw[0, 32:36], raw[0, 36:40] = 0x38, 0xB8, np.frombuffer(np.float32(3).tobytes(), np.uint8), np.frombuffer(np.float32(5).tobytes(), np.uint8)
    v = E.values(raw, 1, 16)
    assert v.shape == (1, 2, 1, 16) and v[0, 0, 0, 0] == 3.0 and v[0, 1, 0, 1] == -5.0 and np.count_nonzero(v) == 2


def test_turns_and_norms():
    quarter = [math.pi / 2, math.pi / 2]
    # a quarter turn takes (a, b) to (-b, a): halves, neighbours, and the rest of the head as it was
    assert np.allclose(E.turned([1, 2, 3, 4, 9], None, 0, [1], quarter, [2], False), [-3, -4, 1, 2, 9])
    assert np.allclose(E.turned([1, 2, 3, 4, 9], None, 0, [1], quarter, [2], True), [-2, 1, -4, 3, 9])
    # two axes: the second pair stands still at position 0
    assert np.allclose(E.turned([1, 2, 3, 4], None, 0, [1, 0], quarter, [1, 1], True), [-2, 1, 3, 4])
    # mean square of (3, 4) is 12.5; with eps 3.5 the root is 4
    assert np.allclose(E.turned([3, 4], [2, 10], 3.5, None, None, None, False), [1.5, 10.0])


def cache(tokens, heads=1, dim=16):
    """Pages of one token whose K and V are given as codes times 1."""
    raw = np.zeros((len(tokens), 1, E.token_bytes(heads, dim)), dtype=np.uint8)
    for i, (k, v) in enumerate(tokens):
        raw[i, 0, 0] = int(np.flatnonzero(E.VALUES == k)[0])
        raw[i, 0, dim] = int(np.flatnonzero(E.VALUES == v)[0])
        raw[i, 0, 2 * dim:2 * dim + 8] = np.frombuffer(np.array([1, 1], "<f4").tobytes(), np.uint8)
    return raw


def test_attention_capped_biased_windowed():
    pages = cache([(1.0, 1.0), (2.0, 2.0), (0.5, 4.0)])
    q = np.zeros((1, 1, 16))
    q[0, 0, 0] = 1.0
    call = dict(owner=[7], have=[2], want=[3], table=np.array([[0, 1, 2]]), pages=pages, heads=1, q=q, scale=1.0)
    r = E.attention(**call)
    p = np.exp([1.0, 2.0, 0.5])
    assert np.isclose(r["out"][0, 0, 0], (p * [1, 2, 4]).sum() / p.sum()) and np.isclose(r["lse"][0, 0], math.log(p.sum()))
    r = E.attention(**call, softcap=0.5)
    p = np.exp(0.5 * np.tanh(np.array([2.0, 4.0, 1.0])))
    assert np.isclose(r["out"][0, 0, 0], (p * [1, 2, 4]).sum() / p.sum())
    r = E.attention(**call, slopes=[0.25])
    p = np.exp(np.array([1.0 - 0.5, 2.0 - 0.25, 0.5]))
    assert np.isclose(r["out"][0, 0, 0], (p * [1, 2, 4]).sum() / p.sum())
    assert E.attention(**call, window=1)["out"][0, 0, 0] == 4.0
    p = np.exp(np.array([2.0, 0.5]))
    assert np.isclose(E.attention(**call, window=2)["out"][0, 0, 0], (p * [2, 4]).sum() / p.sum())


def test_a_page_behind_the_window_is_not_judged():
    pages, label = cache([(1.0, 1.0), (2.0, 2.0), (0.5, 4.0)]), np.array([3, 7, 7])
    call = dict(owner=[7], have=[2], want=[3], table=np.array([[0, 1, 2]]), pages=pages, heads=1, q=np.ones((1, 1, 16)), scale=1.0, owner_map=label)
    assert E.attention(**call)["status"].tolist() == [P.OWNER_MISMATCH]
    assert E.attention(**call, window=2)["status"].tolist() == [0]
    assert E.attention(**call, window=3)["status"].tolist() == [P.OWNER_MISMATCH]
