"""The arithmetic that cuts a prompt's attention into items (no GPU needed): which token tiles a group of step rows meets, and the sums
over groups that a slice's place is found by, against loops over rows and groups."""
import ctypes as C

import numpy as np
import pytest

from paper_2608_25431_b200 import build as B


@pytest.fixture(scope="module")
def hc():
    lib = C.CDLL(B.build_hostcheck())
    lib.hc_group.argtypes = [C.c_uint32] * 4 + [C.c_int, C.c_uint32, C.c_uint32, C.c_void_p]
    return lib


def by_rows(have, rows, per, window, tree):
    """(first tile, tiles) of every group, from what each of its rows sees."""
    out = []
    for g in range(-(-rows // per)):
        mine = range(g * per, min(rows, (g + 1) * per))
        if tree:
            lo, hi = 0, have + rows
        else:
            lo = min(max(0, have + i - window + 1) if window else 0 for i in mine)
            hi = max(have + i + 1 for i in mine)
        out.append((lo // 64, -(-hi // 64) - lo // 64))
    return out


def check(hc, have, rows, per, window, tree, extra):
    ref, out, before = by_rows(have, rows, per, window, tree), (C.c_uint64 * 3)(), 0
    for g in range(len(ref) + 1):
        hc.hc_group(have, rows, per, window, tree, extra, g, out)
        assert out[2] == before, (have, rows, per, window, tree, g)
        if g < len(ref):
            assert (out[0], out[1]) == ref[g], (have, rows, per, window, tree, g)
            before += ref[g][1] + extra


def test_small_shapes(hc):
    for have in (0, 1, 5, 63, 64, 65, 200):
        for rows in (1, 2, 7, 64, 130):
            for per in (1, 3, 25, 64, 128):
                for window in (0, 1, 4, 64, 70, 300):
                    check(hc, have, rows, per, window, False, 8)
                check(hc, have, rows, per, 0, True, 8)


def test_random_shapes(hc):
    rng = np.random.default_rng(3)
    for _ in range(1500):
        rows = int(np.exp(rng.uniform(0, np.log(5000))))
        per = int(rng.choice([1, 16, 25, 32, 50, 64, 128, 256]))
        tree = bool(rng.random() < 0.2)                    # trees have no window
        check(hc, int(np.exp(rng.uniform(0, np.log(60000)))) - 1, rows, per, 0 if tree else int(rng.choice([0, 0, 1, 100, 4096, 2 ** 31 - 1])), tree, int(rng.integers(0, 9)))


def test_long_shapes(hc):
    """Sums past 32 bits: differences of neighbouring groups are what their rows see."""
    out, nxt = (C.c_uint64 * 3)(), (C.c_uint64 * 3)()
    for have, rows, per, window in ((0, 2 ** 31 - 64, 128, 0), (2 ** 30, 2 ** 30 - 1, 16, 0), (2 ** 30, 2 ** 30 - 1, 50, 10 ** 6), (5, 2 ** 31 - 10, 1, 2 ** 20)):
        groups = -(-rows // per)
        for g in (0, 1, groups // 3, groups - 2, groups - 1):
            hc.hc_group(have, rows, per, window, False, 8, g, out)
            hc.hc_group(have, rows, per, window, False, 8, g + 1, nxt)
            lo = max(0, have + g * per - window + 1) if window else 0
            hi = min(have + rows, have + (g + 1) * per)
            assert out[0] == lo // 64 and out[1] == -(-hi // 64) - lo // 64 and nxt[2] - out[2] == out[1] + 8
