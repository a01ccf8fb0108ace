"""Calls of gsit_ops.h that are refused before anything is launched: bad sizes, pointers and rules, answered without a GPU."""
import ctypes

import pytest

P = 0x10000   # an aligned address that is never read


class Rotary(ctypes.Structure):
    _fields_ = [("positions", ctypes.c_void_p), ("axis_stride", ctypes.c_int64), ("batch_stride", ctypes.c_int64), ("sections", ctypes.c_int32 * 3),
                ("interleaved", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("base", ctypes.c_double)]


class Rule(ctypes.Structure):
    _fields_ = [("softcap", ctypes.c_float), ("causal", ctypes.c_int32), ("kv_heads", ctypes.c_int32), ("slopes", ctypes.c_void_p), ("times", ctypes.c_void_p),
                ("documents", ctypes.c_void_p), ("prefix", ctypes.c_void_p), ("tail", ctypes.c_int32), ("q_len", ctypes.c_int32 * 3)]


@pytest.fixture(scope="module")
def g():
    from paper_2505_01068_b200 import build as lib_build
    import paper_2505_01068_b200 as lib
    lib_build.build()
    return lib


def _shape(g, dtype="bf16", d=64, heads=4, seg=(3, 5, 2), batch=2, phase=None, mask=0):
    return g.make_shape(batch, seg, d, heads, None, g.DTYPE_BF16 if dtype == "bf16" else g.DTYPE_F32, g.PHASE_INTRA if phase is None else phase, mask)


def _call(lib, name, *args):
    fn = getattr(lib, name)
    fn.restype = ctypes.c_int
    wrap = {int: ctypes.c_int64, float: ctypes.c_float, type(None): ctypes.c_void_p}
    return fn(*[a if isinstance(a, (ctypes._SimpleCData, ctypes.c_void_p)) else ctypes.byref(a) if isinstance(a, ctypes.Structure) else wrap[type(a)](a) for a in args])


def test_rotary_refuses(g):
    lib, vp = g.load(), ctypes.c_void_p(P)

    def call(shape=None, q=vp, k=vp, q_out=vp, k_out=vp, ldq=64, ldk=64, **kw):
        r = Rotary(P, 20, 10, (ctypes.c_int32 * 3)(4, 2, 2), 0, 0, 10000.0)
        for n, v in kw.items():
            setattr(r, n, (ctypes.c_int32 * 3)(*v) if n == "sections" else v)
        shape = _shape(g) if shape is None else shape
        return _call(lib, "gsit_rotary_fwd", shape, r, q, ldq, k, ldk, q_out, 64, k_out, 64, None)

    for kw in (dict(q=ctypes.c_void_p()), dict(q_out=ctypes.c_void_p()), dict(k=ctypes.c_void_p()), dict(k_out=ctypes.c_void_p()), dict(ldq=63), dict(ldk=32),
               dict(positions=None), dict(sections=(0, 0, 0)), dict(sections=(4, 4, 1)), dict(sections=(9, -1, 0)), dict(base=0.0), dict(base=float("nan")),
               dict(kv_heads=-1), dict(axis_stride=-1), dict(q=ctypes.c_void_p(P + 1)), dict(shape=_shape(g, d=65)), dict(shape=_shape(g, batch=0))):
        assert call(**kw) == 1, kw
    packed = _shape(g)
    packed.row_start, packed.packed_capacity, packed.valid_len = P, 64, P
    assert call(shape=packed) == 2


def test_layer_norm_refuses(g):
    lib, vp, none = g.load(), ctypes.c_void_p(P), ctypes.c_void_p()
    i32 = ctypes.c_int32

    def fwd(shape=None, xt=0, x=vp, ldx=64, gamma=vp, yt=1, y=vp, ldy=64, mean=vp, rstd=vp):
        return _call(lib, "gsit_layer_norm_fwd", _shape(g) if shape is None else shape, i32(xt), x, ldx, gamma, vp, 1e-5, i32(yt), y, ldy, mean, rstd, None)

    for kw in (dict(x=none), dict(y=none), dict(ldx=63), dict(ldy=1), dict(xt=2), dict(yt=-1), dict(mean=none), dict(gamma=ctypes.c_void_p(P + 2)), dict(x=ctypes.c_void_p(P + 2))):
        assert fwd(**kw) == 1, kw
    assert fwd(shape=_shape(g, "f32", d=8193, heads=1), ldx=8193, ldy=8193) == 2

    def bwd(dy=vp, x=vp, mean=vp, residual=none, ldres=0, dgamma=vp, dbeta=vp, ws=vp, size=1 << 20, dx=vp):
        return _call(lib, "gsit_layer_norm_bwd", _shape(g), i32(1), dy, 64, i32(0), x, 64, mean, vp, vp, residual, ldres, dx, 64, dgamma, dbeta, ws,
                     ctypes.c_size_t(size), None)

    for kw in (dict(dy=none), dict(x=none), dict(mean=none), dict(dx=none), dict(residual=vp, ldres=60), dict(dgamma=none), dict(ws=ctypes.c_void_p(P + 4))):
        assert bwd(**kw) == 1, kw
    assert bwd(ws=none) == 3 and bwd(size=8) == 3
    lib.gsit_layer_norm_bwd_workspace.restype = ctypes.c_size_t
    assert 0 < lib.gsit_layer_norm_bwd_workspace(ctypes.byref(_shape(g))) < 1 << 20


def test_scored_attention_refuses(g):
    lib, vp, none = g.load(), ctypes.c_void_p(P), ctypes.c_void_p()

    def rule(**kw):
        r = Rule(30.0, 0, 2, None, None, None, None, 0, (ctypes.c_int32 * 3)())
        for n, v in kw.items():
            setattr(r, n, (ctypes.c_int32 * 3)(*v) if n == "q_len" else v)
        return r

    def fwd(shape=None, r=None, q=vp, ldq=64, k=vp, ldk=32, v=vp, ldv=32, out=vp, lse=none):
        return _call(lib, "gsit_im_scored_attention_fwd", _shape(g) if shape is None else shape, rule() if r is None else r, q, ldq, k, ldk, v, ldv, out, lse,
                     none, ctypes.c_size_t(0), None)

    for kw in (dict(q=none), dict(k=none), dict(v=none), dict(out=none), dict(ldq=63), dict(ldk=31), dict(ldv=33), dict(ldq=68), dict(k=ctypes.c_void_p(P + 8)),
               dict(r=rule(kv_heads=3)), dict(r=rule(kv_heads=-2)), dict(r=rule(softcap=float("nan"))), dict(r=rule(slopes=P + 1)), dict(r=rule(tail=1, q_len=(4, 0, 0))),
               dict(r=rule(tail=1, q_len=(0, 0, 0))), dict(r=rule(tail=1, q_len=(-1, 1, 1))), dict(shape=_shape(g, phase=7)),
               dict(shape=_shape(g, phase=g.PHASE_CUSTOM, mask=0x200)), dict(lse=ctypes.c_void_p(P + 2))):
        assert fwd(**kw) == 1, kw
    for cap in (float("inf"), 1e-45):   # a cap without an end, and one that no score can be divided by
        assert fwd(r=rule(softcap=cap)) == 1, cap
    assert fwd(shape=_shape(g, d=96)) == 2 and fwd(shape=_shape(g, "f32", d=516, heads=4), ldq=516) == 2

    def bwd(r=None, lse=vp, dout=vp, dq=vp, lddq=64, dk=vp, ws=vp, size=1 << 20, lddo=64):
        return _call(lib, "gsit_im_scored_attention_bwd", _shape(g), rule() if r is None else r, vp, 64, vp, 32, vp, 32, vp, 64, lse, dout, lddo, dq, lddq, dk, 32,
                     vp, 32, ws, ctypes.c_size_t(size), None)

    for kw in (dict(lse=none), dict(dout=none), dict(dq=none), dict(dk=none), dict(lddq=60), dict(lddo=12), dict(ws=ctypes.c_void_p(P + 4))):
        assert bwd(**kw) == 1, kw
    assert bwd(ws=none) == 3 and bwd(size=8) == 3 and bwd(r=rule(tail=1, q_len=(1, 1, 1))) == 2
    for n in ("fwd", "bwd"):
        fn = getattr(lib, f"gsit_scored_attention_{n}_workspace")
        fn.restype = ctypes.c_size_t
        assert fn(ctypes.byref(_shape(g)), ctypes.byref(rule())) < 1 << 20
        assert fn(ctypes.byref(_shape(g, d=96)), ctypes.byref(rule())) == ctypes.c_size_t(-1).value
