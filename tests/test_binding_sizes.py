"""The binding's sizes: an argument that does not fit into the 32 bits of its C
parameter is refused, not cut off."""
import ctypes

import pytest

from test_binding_kinds import function, recorder


@pytest.fixture(scope="module")
def px():
    import paper_2607_22595_amd as px
    return px


def test_ints_of_32_bits(px):
    seen = []
    call = function(px, recorder(seen, ctypes.c_int32, ctypes.c_int64), "a:int32 b:int", "a b")
    for a in (0, -1, 2 ** 31 - 1, -2 ** 31):
        assert call(a, 2 ** 40) == 2 and seen[-1] == (a, 2 ** 40)  # a handle has all its bits
    n = len(seen)
    for a in (2 ** 31, -2 ** 31 - 1, 2 ** 32 + 1, 2 ** 63 - 1, 2 ** 70):
        with pytest.raises(OverflowError):
            call(a, 0)
    for a in (1.5, "1", None):
        with pytest.raises(TypeError):
            call(a, 0)
    assert len(seen) == n


def test_dims_of_31_bits(px):
    seen = []
    call = function(px, recorder(seen, ctypes.c_int32), "n:dim", "n")
    assert call(2 ** 31 - 1) == 1 and seen[-1] == (2 ** 31 - 1,)
    for n in (2 ** 31, 2 ** 32, 2 ** 32 + 5):
        with pytest.raises(OverflowError):
            call(n)
    rt = px.Route(8, 2, "cpu")
    call = function(px, recorder(seen, ctypes.c_int32), "r:rt(Route)", "T")
    assert call(rt) == 1 and seen[-1] == (8,)
    for T in (2 ** 31, 2 ** 32 + 8):
        rt.T_max = T
        with pytest.raises(OverflowError):
            call(rt)
    assert len(seen) == 2
