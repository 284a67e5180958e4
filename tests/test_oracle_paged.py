"""The paged-cache oracle pinned by values worked out by hand, and the shared length arithmetic of the
kernels (compiled for the host) against it."""
import ctypes as C

import numpy as np
import pytest

from oracle import paged as P
from paper_2608_25431_b200 import build as B, workloads as W


@pytest.fixture(scope="module")
def hc():
    return C.CDLL(B.build_hostcheck())


def _i(*v):
    return np.array(v, dtype=np.int32)


def test_block_tables_grow_shrink_and_run_short_by_hand():
    # page_tokens 4.  r0: 3 -> 5 tokens (1 -> 2 blocks), r1: 9 -> 4 (3 -> 1), r2: 0 -> 8 (0 -> 2), r3: 1 -> 9 (needs 2)
    owner, have, want = _i(7, 5, 9, 2), _i(3, 9, 0, 1), _i(5, 4, 8, 9)
    table = np.full((4, 3), -1, dtype=np.int32)
    table[0, 0], table[1], table[3, 0] = 10, [11, 12, 13], 14
    free = _i(1, 2, 3, 4, 0, 0, 0, 0)
    label = np.full((2, 16), P.NONE, dtype=np.int32)
    label[:, 10], label[:, 11:14], label[:, 14] = 7, 5, 2
    t, f, n, l, st = P.block_tables(owner, have, want, table, 4, 16, free, 4, label)
    assert st.tolist() == [0, 0, 0, P.NO_BLOCKS]                 # needs 1 + 0 + 2 + 2 of 4
    assert t.tolist() == [[10, 4, -1], [11, -1, -1], [3, 2, -1], [14, -1, -1]]
    assert n == 3 and f[:3].tolist() == [1, 12, 13]
    assert l[0].tolist() == l[1].tolist() == [-2, -2, 9, 9, 7, -2, -2, -2, -2, -2, 7, 5, -2, -2, 2, -2]


@pytest.mark.parametrize("spoil", ["range", "twice", "owned", "foreign", "height", "room"])
def test_a_malformed_stack_or_table_refuses_the_call(spoil):
    owner, have, want = _i(1, 2), _i(0, 8), _i(8, 0)
    table = np.array([[-1, -1], [4, 5]], dtype=np.int32)
    free, n_free = _i(0, 1, 2, 0, 0), 3
    label = np.full((1, 8), P.NONE, dtype=np.int32)
    label[0, 4:6] = 2
    if spoil == "range":
        free[2] = 8
    elif spoil == "twice":
        free[1] = free[2]
    elif spoil == "owned":
        label[0, 1] = 3
    elif spoil == "foreign":
        label[0, 5] = 1
    elif spoil == "height":
        n_free = 6
    elif spoil == "room":
        want[0] = 0                       # nothing taken, two given back, room for one in all
        free, n_free = _i(0), 1
    t, f, n, l, st = P.block_tables(owner, have, want, table, 4, 8, free, n_free, label)
    assert st.tolist() == [P.BAD_TABLE] * 2
    assert np.array_equal(t, table) and np.array_equal(f, free) and n == n_free and np.array_equal(l, label)


def test_slot_map_by_hand():
    owner, have, want = _i(3, 8, 4), _i(2, 5, 1), _i(4, 5, 2)
    table = np.array([[6, -1], [1, 2], [9, 0]], dtype=np.int32)
    m = P.slot_map(owner, have, want, table, 3, 9, 5)
    # r0: positions 2 (page 6, offset 2) and 3 (no page); r1: none; r2: position 1 (page 9 is out of range)
    assert m["slots"].tolist() == [20, -1, -1, -1, -1] and m["pos"].tolist() == [2, 3, 1, -1, -1]
    assert m["req"].tolist() == [0, 0, 2, -1, -1] and m["owner"].tolist() == [3, 3, 4, -2, -2]
    assert m["ptr"].tolist() == [0, 2, 2, 3] and m["total"] == 3
    m = P.slot_map(owner, have, want, table, 3, 9, 5, rel=_i(-1, 0, 1, 0, 0))
    assert m["slots"].tolist() == [-1, 20, -1, -1, -1] and m["pos"].tolist() == [-1, 2, -1, -1, -1]
    assert P.slot_map(owner, have, want, table, 3, 9, 2)["ptr"].tolist() == [0, 0, 0, 0]


def test_segments_by_hand_match_the_handoff_workload():
    w = W.config3(layers=2, n_users=3, min_len=20, max_len=60, fill=False)
    x = w.extra
    width = int(x["nblk"].max())
    table = np.full((3, width), -1, dtype=np.int32)
    for u in range(3):
        table[u, : x["nblk"][u]] = x["perm"][x["first"][u]: x["first"][u] + x["nblk"][u]]
    zero = np.zeros(3, dtype=np.int32)
    segs, pt, total = P.kv_segments(w.user_ids, zero, x["prompt"].astype(np.int32), table, 16, x["n_slots"], w.user_ids,
                                    2, W.KV_TOKEN_BYTES, len(w.segs) + 1, W.SEG_DTYPE, whole_pages=True)
    assert total == len(w.segs) and np.array_equal(segs[:-1], w.segs) and np.array_equal(pt[:-1], w.page_table)
    assert segs["flags"][-1] == 1 and pt[-1] == -1


def test_append_status_by_hand():
    label = _i(4, P.PARAM, P.NONE, P.CONFLICT, 5)
    st, wrote = P.append_status([0, 2, 4, 6, 8, 10, -1, -2], [4] * 8, label, 5, 2)
    assert st.tolist() == [0, P.OWNER_MISMATCH, P.UNOWNED, P.UNOWNED, P.OWNER_MISMATCH, P.BAD_DESC, 0, P.BAD_DESC]
    assert wrote.tolist() == [True] + [False] * 7


def test_attention_by_hand_and_against_a_direct_sum():
    # two cached tokens and two drafted ones; the second drafted token does not see the first
    pages = np.zeros((3, 2, 2, 1, 2))
    pages[2, 0] = [[[1.0, 0.0]], [[1.0, 2.0]]]
    pages[2, 1] = [[[0.0, 0.0]], [[3.0, 4.0]]]
    pages[0, 0] = [[[0.0, 0.0]], [[5.0, 6.0]]]
    pages[0, 1] = [[[0.0, 0.0]], [[7.0, 8.0]]]
    q = np.zeros((2, 1, 2))
    table, mask = np.array([[2, 0]], dtype=np.int32), np.array([[1], [2]], dtype=np.int32)
    r = P.attention(_i(1), _i(2), _i(4), table, pages, q, 1.0, mask, owner_map=_i(1, P.NONE, P.PARAM))
    assert r["status"].tolist() == [0] and r["row_owner"].tolist() == [1, 1]
    assert np.allclose(r["out"][:, 0], [[3.0, 4.0], [11 / 3, 14 / 3]]) and np.allclose(r["lse"], np.log(3))
    q[:] = [np.log(2.0), 0.0]
    r = P.attention(_i(1), _i(2), _i(4), table, pages, q, 1.0)            # causal: weights 2, 1, 1 and 2, 1, 1, 1
    assert np.allclose(r["out"][:, 0], [[2.5, 3.5], [17 / 5, 22 / 5]]) and np.allclose(np.exp(r["lse"]), [[4.0], [5.0]])
    r = P.attention(_i(1), _i(0), _i(1), table, pages, q[:1], 1.0, np.zeros((1, 1), np.int32))
    assert not r["out"].any() and np.isneginf(r["lse"]).all() and r["status"][0] == 0
    for label, want in ((_i(9, 0, 1), P.OWNER_MISMATCH), (_i(1, 0, P.CONFLICT), P.UNOWNED), (_i(9, 0, -2), 6)):
        r = P.attention(_i(1), _i(2), _i(4), table, pages, q, 1.0, owner_map=label)
        assert r["status"][0] == want and not r["out"].any() and (r["row_owner"] == P.CONFLICT).all()
    assert P.attention(_i(1), _i(2), _i(4), _i(2, 3)[None], pages, q, 1.0)["status"][0] == P.BAD_DESC
    assert P.attention(_i(1), _i(2), _i(4), table, pages, q[:1], 1.0)["status"][0] == P.BAD_TABLE


def test_request_shapes_of_the_kernels_match_the_oracle(hc):
    rng = np.random.default_rng(5)
    edge = [-1, 0, 1, 15, 16, 17, 255, 2 ** 31 - 1]
    out = (C.c_uint32 * 6)()
    for _ in range(4000):
        owner = int(rng.choice([-3, -1, 0, 5, 2 ** 20 - 1, 2 ** 20]))
        have, want = (int(rng.choice(edge)) if rng.random() < 0.5 else int(rng.integers(0, 300)) for _ in range(2))
        pt, width = int(rng.choice([1, 3, 16, 24, 65536])), int(rng.choice([1, 2, 20, 2 ** 31 - 1]))
        hc.hc_req_shape(owner, have, want, pt, C.c_uint32(width), out)
        ok, h, w, bh, bw = P.shape(owner, have, want, pt, width)
        assert list(out) == [int(ok), h, w, bh, bw, max(0, w - h)]


def test_fixed_division_of_the_kernels(hc):
    rng = np.random.default_rng(7)
    hc.hc_quot.restype = C.c_uint32
    for d in [1, 2, 3, 5, 7, 16, 24, 125, 1023, 1024, 65535, 65536, 2 ** 30 + 1] + rng.integers(1, 65537, size=60).tolist():
        edge = [0, 1, d - 1, d, d + 1, 2 ** 31 - 1, 2 ** 31 - 2, (2 ** 31 - 1) // d * d, (2 ** 31 - 1) // d * d - 1]
        for t in edge + rng.integers(0, 2 ** 31, size=200).tolist():
            if 0 <= t < 2 ** 31:
                assert hc.hc_quot(d, t) == t // d, (d, t)


def test_prefix_search_of_the_kernels(hc):
    rng = np.random.default_rng(6)
    for _ in range(200):
        counts = rng.integers(0, 4, size=int(rng.integers(1, 40)))
        first = np.concatenate([[0], np.cumsum(counts)[:-1]]).astype(np.uint32)
        want = np.repeat(np.arange(counts.size), counts)
        for k, r in enumerate(want):
            assert hc.hc_req_of(first.ctypes.data_as(C.c_void_p), counts.size, k) == r


def test_label_checks_of_the_kernels(hc):
    for label in (-3, -2, -1, 0, 1, 2, 2 ** 20 - 1):
        assert not hc.hc_label_claimed(label) and hc.hc_label_claimed(hc.hc_label_flip(label))
        assert hc.hc_label_flip(hc.hc_label_flip(label)) == label
        for owner in (0, 1, 2 ** 20 - 1):
            st, _ = P.append_status([0], [owner], [label], 1, 1)
            assert hc.hc_label_write_status(label, owner) == st[0]
            pages = np.zeros((1, 1, 2, 1, 1))
            r = P.attention(_i(owner), _i(0), _i(1), _i(0)[None], pages, np.zeros((1, 1, 1)), 1.0, owner_map=_i(label))
            assert hc.hc_label_read_status(label, owner) == r["status"][0]


@pytest.mark.parametrize("total,ctas,least", [(1, 296, 1), (295, 296, 1), (296, 296, 2), (297, 296, 1), (10 ** 12, 148, 4), (7, 3, 2)])
def test_slices_cover_the_work(hc, total, ctas, least):
    hc.hc_slice_units.restype = C.c_uint64
    s = hc.hc_slice_units(C.c_uint64(total), ctas, least)
    assert s >= least and s * ctas >= total and (s == least or (s - 1) * ctas < total)
