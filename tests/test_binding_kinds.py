"""The binding's floats and optional structs: where each arrives in the C call."""
import ctypes

import numpy as np
import pytest


@pytest.fixture(scope="module")
def px():
    import paper_2607_22595_amd as px
    return px


def recorder(seen, *types):
    """A C function that notes its arguments and returns their number."""
    @ctypes.CFUNCTYPE(ctypes.c_int32, *types)
    def note(*args):
        seen.append(args)
        return len(args)
    return note


def function(px, note, args, c_args):
    return px._call.Function("note", ctypes.cast(note, ctypes.c_void_p).value, args, c_args,
                             {"Route": px.XmixRoute})


def test_floats_arrive_wherever_they_stand(px):
    """Floats have registers of their own: the integers around them keep their order,
    those on the stack (past the sixth) too."""
    i, f, seen = ctypes.c_int64, ctypes.c_float, []
    note = recorder(seen, i, f, i, i, i, i, i, f, i, i)
    call = function(px, note, "a:int x:float b:int c:int d:int e:int g:int y:float h:int k:int",
                    "a x b c d e g y h k")
    assert call(1, 0.1, 2, 3, 4, 5, 6, -2.5, 7, -8) == 10
    assert seen == [(1, np.float32(0.1), 2, 3, 4, 5, 6, -2.5, 7, -8)]
    for value in (3, np.float64(0.25), np.float32(1e-30), float("inf"), True):
        call(0, value, 0, 0, 0, 0, 0, 0.0, 0, 0)
        assert seen[-1][1] == np.float32(value)
    # an argument may be left out of the C call, or a float come first
    last = function(px, recorder(seen, f, i), "a:int b:int x:float", "x b")
    assert last(9, 4, 1.5) == 2 and seen[-1] == (1.5, 4)
    for wrong in ("1", None, [1.0]):
        with pytest.raises(TypeError):
            last(9, 4, wrong)


def test_more_floats_than_registers_are_refused(px):
    with pytest.raises(ValueError):
        function(px, recorder([], ctypes.c_float), "x:float y:float z:float", "x y z")


def test_optional_structs(px):
    seen, p = [], ctypes.c_void_p
    rt = px.Route(8, 2, "cpu")
    note = recorder(seen, p, ctypes.c_int64)
    call = function(px, note, "r?:struct(Route) n:int", "r n")
    assert call(None, 3) == 2 and seen[-1] == (None, 3)
    assert call(rt, 4) == 2 and seen[-1] == (ctypes.addressof(rt.struct), 4)
    need = function(px, note, "r:struct(Route) n:int", "r n")
    with pytest.raises(AttributeError):
        need(None, 3)
