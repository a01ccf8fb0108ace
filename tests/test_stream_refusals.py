"""Calls of gsit_stream.h and of gsit_head_norm_rotary_* that are refused before anything is launched, answered without a GPU."""
import ctypes

import pytest

from test_ops_refusals import P, Rotary, Rule, _call, _shape, g   # noqa: F401


class Cache(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_int32) for n in ("kind", "dtype", "batch", "kv_heads", "head_dim", "pages", "blocks")] +
                [(n, ctypes.c_void_p) for n in ("keys", "values", "key_scale", "value_scale", "times", "open_keys", "open_values", "tables", "lengths", "free_list", "n_free")])


def _cache(**kw):
    c = Cache(0, 1, 2, 2, 16, 100, 8, P, P, P, P, None, P, P, P, P, P, P)
    for n, v in kw.items():
        setattr(c, n, v)
    return c


VP, NONE, ODD = ctypes.c_void_p(P), ctypes.c_void_p(), ctypes.c_void_p(P + 2)


def test_plan_refuses(g):
    lib = g.load()

    def call(shape=None, cache=None, held=NONE, ended=NONE, slots=VP):
        return _call(lib, "gsit_cache_plan", _shape(g) if shape is None else shape, _cache() if cache is None else cache, held, ended, slots, None)

    for kw in (dict(cache=_cache(batch=3)), dict(cache=_cache(pages=0)), dict(cache=_cache(blocks=0)), dict(cache=_cache(tables=None)), dict(cache=_cache(lengths=None)),
               dict(cache=_cache(free_list=None)), dict(cache=_cache(n_free=None)), dict(cache=_cache(tables=P + 2)), dict(slots=NONE), dict(slots=ODD), dict(held=ODD),
               dict(ended=ODD), dict(shape=_shape(g, seg=(0, 0, 0))), dict(shape=_shape(g, seg=(1, -1, 4))), dict(shape=_shape(g, batch=0))):
        assert call(**kw) == 1, kw
    assert call(cache=_cache(pages=1 << 26)) == 2 and call(cache=_cache(blocks=1 << 22)) == 2
    assert call(shape=_shape(g, batch=65536), cache=_cache(batch=65536)) == 2
    packed = _shape(g)
    packed.row_start, packed.packed_capacity, packed.valid_len = P, 64, P
    assert call(shape=packed) == 2
    assert _call(lib, "gsit_cache_plan", _shape(g), NONE, NONE, NONE, VP, None) == 1


def test_append_and_read_refuse(g):
    lib = g.load()

    def append(cache=None, k=VP, ldk=32, v=VP, ldv=32, slots=VP, times=NONE, shape=None):
        return _call(lib, "gsit_cache_append", _shape(g) if shape is None else shape, _cache() if cache is None else cache, k, ldk, v, ldv, slots, times, 10, 1, None)

    def read(cache=None, k=VP, ldk=32, v=VP, ldv=32):
        return _call(lib, "gsit_cache_read", _shape(g), _cache() if cache is None else cache, k, ldk, v, ldv, None)

    for kw in (dict(k=NONE), dict(v=NONE), dict(ldk=31), dict(ldv=24), dict(ldk=36), dict(k=ctypes.c_void_p(P + 8)), dict(cache=_cache(kind=2)), dict(cache=_cache(kind=-1)),
               dict(cache=_cache(dtype=2)), dict(cache=_cache(kv_heads=0)), dict(cache=_cache(keys=None)), dict(cache=_cache(values=P + 8)), dict(cache=_cache(key_scale=None)),
               dict(cache=_cache(value_scale=P + 2)), dict(cache=_cache(open_keys=None)), dict(cache=_cache(open_values=P + 4)), dict(cache=_cache(batch=1)),
               dict(cache=_cache(times=P + 4))):
        assert append(**kw) == 1, kw
        assert read(**kw) == 1, kw
    for kw in (dict(slots=NONE), dict(slots=ODD), dict(times=ODD), dict(cache=_cache(times=P))):
        assert append(**kw) == 1, kw
    for hd in (4, 24, 128):
        assert append(cache=_cache(head_dim=hd), ldk=512, ldv=512) == 2 and read(cache=_cache(head_dim=hd), ldk=512, ldv=512) == 2


def test_attention_refuses(g):
    lib = g.load()

    def rule(**kw):
        r = Rule(30.0, 0, 2, None, None, None, None, 0, (ctypes.c_int32 * 3)())
        for n, v in kw.items():
            setattr(r, n, v)
        return r

    def call(shape=None, r=None, cache=None, q=VP, ldq=64, times=NONE, out=VP, lse=NONE):
        return _call(lib, "gsit_im_cached_attention_fwd", _shape(g) if shape is None else shape, rule() if r is None else r, _cache() if cache is None else cache, q, ldq, times,
                     10, 1, out, lse, NONE, ctypes.c_size_t(0), None)

    for kw in (dict(q=NONE), dict(out=NONE), dict(ldq=63), dict(ldq=68), dict(q=ctypes.c_void_p(P + 8)), dict(lse=ODD), dict(times=ODD), dict(shape=_shape(g, "f32")),
               dict(shape=_shape(g, d=32)), dict(r=rule(kv_heads=4)), dict(r=rule(softcap=float("nan"))), dict(r=rule(softcap=float("inf"))), dict(r=rule(softcap=1e-45)),
               dict(r=rule(slopes=P + 1)), dict(cache=_cache(kv_heads=3), r=rule(kv_heads=0)), dict(shape=_shape(g, phase=7)),
               dict(shape=_shape(g, phase=g.PHASE_CUSTOM, mask=0x200)), dict(r=rule(causal=1), times=VP), dict(r=rule(causal=1), cache=_cache(times=P)),
               dict(r=rule(slopes=P), cache=_cache(times=P))):
        assert call(**kw) == 1, kw
    for r in (rule(times=P), rule(documents=P), rule(causal=1, prefix=P), rule(tail=1)):
        assert call(r=r) == 2
    assert call(cache=_cache(head_dim=24), shape=_shape(g, d=96), ldq=96) == 2
    fn = lib.gsit_cached_attention_workspace
    fn.restype = ctypes.c_size_t
    bad = ctypes.c_size_t(-1).value
    assert fn(None, ctypes.byref(rule()), ctypes.byref(_cache())) == bad and fn(ctypes.byref(_shape(g)), None, ctypes.byref(_cache())) == bad
    assert fn(ctypes.byref(_shape(g)), ctypes.byref(rule()), None) == bad


def test_head_norm_refuses(g):
    lib = g.load()

    def rotary(**kw):
        r = Rotary(P, 20, 10, (ctypes.c_int32 * 3)(4, 2, 2), 0, 0, 10000.0)
        for n, v in kw.items():
            setattr(r, n, (ctypes.c_int32 * 3)(*v) if n == "sections" else v)
        return r

    def fwd(shape=None, r=None, eps=1e-6, q=VP, ldq=64, qg=VP, k=VP, ldk=64, kg=VP, qo=VP, ldqo=64, ko=VP, ldko=64):
        return _call(lib, "gsit_head_norm_rotary_fwd", _shape(g) if shape is None else shape, rotary() if r is None else r, eps, q, ldq, qg, k, ldk, kg, qo, ldqo, ko, ldko, None)

    def bwd(dq=VP, dk=VP, gq=VP, gk=VP, ws=VP, size=1 << 22, k=VP, ko=VP):
        return _call(lib, "gsit_head_norm_rotary_bwd", _shape(g), rotary(), 1e-6, VP, 64, VP, k, 64, VP, dq, 64, dk, 64, VP, 64, ko, 64, gq, gk, ws, ctypes.c_size_t(size), None)

    for kw in (dict(q=NONE), dict(qo=NONE), dict(ko=NONE), dict(k=NONE), dict(ldq=63), dict(ldk=32), dict(ldqo=8), dict(ldko=8), dict(q=ctypes.c_void_p(P + 1)), dict(qg=ODD),
               dict(kg=ODD), dict(r=rotary(positions=None)), dict(r=rotary(positions=P + 2)), dict(r=rotary(sections=(4, 4, 1))), dict(r=rotary(sections=(9, -1, 0))),
               dict(r=rotary(base=0.0)), dict(r=rotary(base=float("nan"))), dict(r=rotary(kv_heads=-1)), dict(r=rotary(axis_stride=-1)), dict(eps=float("nan")),
               dict(eps=float("inf")), dict(shape=_shape(g, batch=0))):
        assert fwd(**kw) == 1, kw
    assert fwd(shape=_shape(g, "f32", d=514, heads=2), ldq=514, ldk=514, ldqo=514, ldko=514) == 2
    assert fwd(shape=_shape(g, "f32", d=512, heads=2), r=rotary(sections=(65, 0, 0)), ldq=512, ldk=512, ldqo=512, ldko=512) == 2
    for kw in (dict(dq=NONE), dict(dk=NONE), dict(gq=NONE), dict(gk=NONE), dict(ws=ctypes.c_void_p(P + 4)), dict(k=NONE), dict(ko=NONE)):
        assert bwd(**kw) == 1, kw
    assert bwd(ws=NONE) == 3 and bwd(size=8) == 3
