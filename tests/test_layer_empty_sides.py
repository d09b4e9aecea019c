"""A layer of experts with an empty side, its weights in 8 bits: what is empty has
scales without an address, and such a call is no mixture of kinds.  Only calls that
launch nothing; the others are the GPU tests'."""
import ctypes
import struct

import pytest

import paper_2609_09095_amd as oz


@pytest.fixture(scope="module", autouse=True)
def built_library():
    import os
    if not os.path.exists(oz.library_path()):
        from paper_2609_09095_amd import build
        build.build()
    oz.lib()


def call(tokens, top, experts, width, inner, out, gated=True, no_scales=()):
    """The call as the binding packs it: an empty tensor has address 0."""
    at = iter(range(1, 20))

    def place(*shape):
        return 0 if 0 in shape else next(at) << 32

    def stack(name, rows, cols):
        rb, cb = -(-rows // 128), -(-cols // 128)
        scales = 0 if name in no_scales else place(experts, rb, cb)
        return struct.pack("6q", place(experts, rows, cols), cols or 1, rows * (cols or 1), scales, cb or 1, rb * (cb or 1))

    up, down = stack("up", inner, width), stack("down", out, inner)
    gate = stack("gate", inner, width) if gated else None
    p = ctypes.c_void_p
    return oz.lib().ozaki25_expert_layer(tokens, top, experts, width, inner, out, p(place(tokens, width)), width or 1,
                                         p(place(tokens, top)), p(place(tokens, top)), up, gate, down, p(place(tokens, out)),
                                         out or 1, oz.BF16, None, 0, None)


@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("sizes", [(4, 2, 3, 200, 100, 0), (0, 2, 3, 0, 100, 200), (0, 2, 3, 200, 0, 200), (0, 2, 0, 200, 100, 200),
                                   (0, 0, 3, 200, 100, 200), (4, 2, 3, 0, 100, 0), (4, 2, 3, 200, 0, 0), (0, 2, 3, 200, 100, 200)])
def test_nothing_to_write(sizes, gated):
    assert call(*sizes, gated=gated) == oz.SUCCESS


@pytest.mark.parametrize("sizes,no", [((4, 2, 3, 200, 100, 200), ("up",)), ((4, 2, 3, 200, 100, 200), ("gate",)),
                                      ((4, 2, 3, 200, 100, 200), ("down",)), ((0, 2, 3, 200, 100, 200), ("down",)),
                                      ((4, 2, 3, 200, 100, 0), ("gate",)), ((4, 2, 3, 200, 100, 0), ("up",))])
def test_mixed_stacks_that_are_not_empty(sizes, no):
    assert call(*sizes, no_scales=no) == oz.ERR_INVALID_VALUE
