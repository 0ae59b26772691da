"""What rows that are taken back leave in a cache: a scale they raised stays
raised, and earlier codes rounded to it, until the block is begun again or put
back."""
import numpy as np
import pytest

from oracle import kv8


def filled(fmt, parts):
    c = kv8.Cache(fmt, 32, 1, 1, 64, 64)
    for pos, x in parts:
        c.store(x, [pos])
    return c


@pytest.mark.parametrize("fmt", [kv8.E4M3, kv8.INT8], ids=["e4m3", "int8"])
def test_rows_taken_back(fmt):
    rng = np.random.default_rng(4)
    rows = rng.standard_normal((1, 41, 2, 1, 64))
    large = 100.0 * rng.standard_normal((1, 3, 2, 1, 64))
    plain = filled(fmt, [(0, rows[:, :40]), (40, rows[:, 40:])])
    drafted = filled(fmt, [(0, rows[:, :40]), (40, large), (40, rows[:, 40:])])
    first, last = slice(0, 32), slice(32, 41)
    # blocks that were full before are as without the draft; the one it went into is not
    np.testing.assert_array_equal(drafted.read()[..., first, :], plain.read()[..., first, :])
    assert np.all(drafted.scale[..., 1] > plain.scale[..., 1])
    assert np.any(drafted.read()[..., last, :] != plain.read()[..., last, :])
    # the block stored again from its first position, or its codes and scale put back
    again = filled(fmt, [(0, rows[:, :40]), (40, large), (32, rows[:, 32:])])
    np.testing.assert_array_equal(again.read()[..., last, :], filled(fmt, [(0, rows)]).read()[..., last, :])
    back = filled(fmt, [(0, rows[:, :40])])
    code, scale = back.code.copy(), back.scale.copy()
    back.store(large, [40])
    back.code[..., 32:64, :], back.scale[..., 1] = code[..., 32:64, :], scale[..., 1]
    back.store(rows[:, 40:], [40])
    np.testing.assert_array_equal(back.read()[..., :41, :], plain.read()[..., :41, :])
