"""Shapes of the gated feed-forward block at the ends of the range that its sizes are said to have (CPU)."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def sizes():
    import paper_1901_05350_b200 as pkg

    def ask(tokens, width, hidden, out_width, dtype):
        got = (ctypes.c_int64 * 4)()
        at = [ctypes.cast(ctypes.byref(got, 8 * i), ctypes.POINTER(ctypes.c_int64)) for i in range(4)]
        rc = pkg.lib.tfjsb_gated_ffn_sizes(ctypes.byref(pkg.Ffn(tokens, width, hidden, out_width, dtype, 0)), *at)
        return rc, list(got)

    return ask


def true_sizes(t, d, f, o, dtype):
    """h, z and the two workspaces in whole numbers of any length, without the rounding up of rows and buffers."""
    planes = 3 if dtype == 0 else 1
    e = 2 * planes
    return t * f * e, t * f * 8, t * f * e if t > 8 else 0, 2 * t * f * e


MOST = 2 ** 30


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("shape", [(t, d, f, o) for t in (1, 33, 2 ** 29, MOST) for d in (1, MOST) for f in (1, 2 ** 27, MOST) for o in (1, MOST - 1)], ids=str)
def test_byte_counts_are_right_or_the_shape_is_refused(sizes, shape, dtype):
    rc, got = sizes(*shape, dtype)
    want = true_sizes(*shape, dtype)
    if rc == 0:
        assert all(g >= w for g, w in zip(got, want)), (got, want)
        assert all(g <= 2 ** 60 for g in got)
    else:
        assert rc == 2  # TFJSB_ERR_SHAPE
        weights = max(shape[1], shape[3]) * shape[2] * 12 + shape[0] * max(shape[1], shape[3]) * 12
        assert max(want) + 2 * weights > 2 ** 59  # only what no machine holds


def test_a_shape_that_is_refused_is_refused_by_the_calls(sizes):
    import paper_1901_05350_b200 as pkg

    assert sizes(MOST, 1, MOST, 1, 1)[0] == 2 and sizes(MOST, 1, MOST, 1, 0)[0] == 2
    assert sizes(70001, 64, 32768, 64, 1)[0] == 0 and sizes(2 ** 24, 4096, 16384, 4096, 0)[0] == 0
    assert pkg.STATUS_NAMES[2] == "SHAPE"
