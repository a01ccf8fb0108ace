"""What the streaming calls refuse at the ends of their ranges, answered without a GPU."""
import ctypes

from test_ops_refusals import P, Rule, _call, _shape, g   # noqa: F401
from test_stream_refusals import NONE, VP, _cache


def _rule(**kw):
    r = Rule(0.0, 0, 2, None, None, None, None, 0, (ctypes.c_int32 * 3)())
    for n, v in kw.items():
        setattr(r, n, v)
    return r


def _attention(g, rule, cache, times):
    return _call(g.load(), "gsit_im_cached_attention_fwd", _shape(g), rule, cache, VP, 64, times, 10, 1, VP, NONE, NONE, ctypes.c_size_t(0), None)


def test_indices_that_float_does_not_hold(g):
    """Causality and slopes by the index inside the segment: tables of 2^24 positions and no more."""
    fn = g.load().gsit_cached_attention_workspace
    fn.restype = ctypes.c_size_t
    bad = ctypes.c_size_t(-1).value
    for kw in (dict(causal=1), dict(slopes=P), dict(causal=1, slopes=P)):
        assert _attention(g, _rule(**kw), _cache(blocks=(1 << 19) + 1), NONE) == 2
        assert fn(ctypes.byref(_shape(g)), ctypes.byref(_rule(**kw)), ctypes.byref(_cache(blocks=(1 << 19) + 1))) == bad
