"""What the dense layers of transformer blocks decide on the host, without a GPU: sizes, refusals, null contexts."""
import ctypes

import pytest


@pytest.fixture(scope="module")
def pkg():
    import paper_1901_05350_b200 as p

    return p


def sizes(pkg, tokens, width, hidden, out_width, dtype=1, gate=0):
    got = (ctypes.c_int64 * 4)()
    at = [ctypes.cast(ctypes.byref(got, 8 * i), ctypes.POINTER(ctypes.c_int64)) for i in range(4)]
    rc = pkg.lib.tfjsb_gated_ffn_sizes(ctypes.byref(pkg.Ffn(tokens, width, hidden, out_width, dtype, gate)), *at)
    return rc, list(got)


@pytest.mark.parametrize("shape,dtype", [((1, 1, 1, 1), 1), ((7, 64, 128, 64), 1), ((1000, 1024, 2730, 1024), 1), ((515, 512, 1365, 512), 0), ((70001, 64, 32768, 64), 1)], ids=str)
def test_what_is_kept_and_the_workspaces_hold_what_they_have_to(pkg, shape, dtype):
    rc, (h, z, forward, backward) = sizes(pkg, *shape, dtype=dtype)
    t, d, f, o = shape
    planes = 1 if dtype == 1 else 3
    assert rc == 0
    assert h >= 2 * planes * t * f and z >= 8 * t * f  # h in the storage type or three planes, g and u in fp32
    assert forward >= 2 * planes * t * f or t <= 8     # h, where it is not kept (fp32 for a few tokens)
    assert backward >= 4 * planes * t * f              # the gradients of g and u
    assert all(v % 16 == 0 for v in (h, z, forward, backward))


def test_operands_that_are_copied_need_room(pkg):
    whole, odd = sizes(pkg, 100, 64, 128, 64)[1], sizes(pkg, 100, 63, 127, 61)[1]
    assert odd[2] > whole[2] and odd[3] > whole[3]  # smaller, but copied: rows of no multiple of 16 bytes


@pytest.mark.parametrize("shape", [(-1, 8, 8, 8), (8, 0, 8, 8), (8, 8, 0, 8), (8, 8, 8, 0), (2 ** 30 + 1, 8, 8, 8), (8, 2 ** 30 + 1, 8, 8)], ids=str)
def test_shapes_that_are_refused(pkg, shape):
    assert sizes(pkg, *shape)[0] == 2  # TFJSB_ERR_SHAPE


def test_enumerations_that_are_refused(pkg):
    assert sizes(pkg, 8, 8, 8, 8, dtype=2)[0] == 1 and sizes(pkg, 8, 8, 8, 8, gate=5)[0] == 1 and sizes(pkg, 8, 8, 8, 8, gate=-1)[0] == 1
    assert pkg.lib.tfjsb_gated_ffn_sizes(None, None, None, None, None) == 1


def test_the_workspace_of_an_8_bit_layer(pkg):
    size = pkg.lib.tfjsb_dense_int8_workspace
    assert size(3, 100) >= 3 * 112 + 12 and size(1, 131072) >= 131072 + 4
    assert size(-1, 16) == size(3, 0) == size(3, 131073) == 0


def test_a_null_context_is_refused(pkg):
    lib, f = pkg.lib, pkg.Ffn(1, 8, 8, 8, 1, 0)
    assert lib.tfjsb_gated_ffn(None, ctypes.byref(f), *[None] * 8, 0, None) == 1
    assert lib.tfjsb_gated_ffn_backprop(None, ctypes.byref(f), *[None] * 12, 0, None) == 1
    assert lib.tfjsb_dropout(None, 0, None, None, None, 1, None, None, 0.5, 0, 0, None) == 1
    assert lib.tfjsb_dropout_backprop(None, 0, None, None, 1, None, None, 0.5, 0, 0, None) == 1
    assert lib.tfjsb_quantize_int8(None, 0, None, 1, 1, None, None, None) == 1
    assert lib.tfjsb_matmul_int8(None, None, None, None, None, None, 0, None, 0, 1, 1, 16, None) == 1
    assert lib.tfjsb_dense_int8(None, 0, None, None, None, None, 0, None, 0, 1, 1, 16, None, 0, None) == 1
