"""Which fields of a shape the calls of gsit_ops.h look at, answered without a GPU."""
import ctypes

import pytest

from test_ops_refusals import P, Rotary, _call, _shape, g   # noqa: F401


def _odd(g, **kw):
    """A shape whose fields outside the block pattern are right."""
    s = _shape(g, **kw)
    s.phase, s.custom_mask = 77, 0xFFFF
    return s


def test_layer_norm_reads_neither_heads_type_nor_pattern(g):
    lib = g.load()
    fn = lib.gsit_layer_norm_bwd_workspace
    fn.restype = ctypes.c_size_t
    want = fn(ctypes.byref(_shape(g)))
    for heads, dtype in ((0, 0), (-1, 1), (7, 9), (4, -3)):
        s = _odd(g)
        s.heads, s.dtype = heads, dtype
        assert fn(ctypes.byref(s)) == want
    s = _odd(g)
    s.batch = 0
    assert fn(ctypes.byref(s)) == ctypes.c_size_t(-1).value
    assert fn(None) == ctypes.c_size_t(-1).value


@pytest.mark.parametrize("name", ["gsit_rotary_fwd", "gsit_rotary_bwd"])
def test_rotary_reads_no_pattern(g, name):
    """More pairs than the kernels take: unsupported, whatever stands in the fields of the pattern (which were answered as invalid)."""
    lib, vp = g.load(), ctypes.c_void_p(P)
    r = Rotary(P, 20, 10, (ctypes.c_int32 * 3)(65, 0, 0), 0, 0, 10000.0)
    call = lambda s: _call(lib, name, s, r, vp, 256, vp, 256, vp, 256, vp, 256, None)
    assert call(_shape(g, d=256, heads=1)) == 2
    assert call(_odd(g, d=256, heads=1)) == 2


def test_rotary_refuses_positions_between_integers(g):
    lib, vp = g.load(), ctypes.c_void_p(P)
    r = Rotary(P + 2, 20, 10, (ctypes.c_int32 * 3)(4, 2, 2), 0, 0, 10000.0)
    assert _call(lib, "gsit_rotary_fwd", _shape(g), r, vp, 64, vp, 64, vp, 64, vp, 64, None) == 1
