"""What the streaming calls refuse at the ends of their ranges, answered without a GPU."""
import ctypes

import pytest
import torch

from test_ops_refusals import P, Rule, _call, _shape, g   # noqa: F401
from test_stream_refusals import NONE, ODD, VP, _cache


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


@pytest.mark.parametrize("kw, code", [(dict(slots=NONE), 1), (dict(ended=ODD), 1), (dict(held=ODD), 1), (dict(q=NONE), 1), (dict(k=NONE), 1), (dict(v=ODD), 1), (dict(ldq=40), 1), (dict(ldk=16), 1),
                                      (dict(out=NONE), 1), (dict(lse=ODD), 1), (dict(rule=dict(softcap=float("nan"))), 1), (dict(rule=dict(documents=P)), 2),
                                      (dict(rule=dict(causal=1, prefix=P)), 2), (dict(rule=dict(causal=1), times=VP), 1), (dict(cache=dict(times=P)), 1),
                                      (dict(cache=dict(free_list=None)), 1), (dict(cache=dict(head_dim=24)), 2), (dict(cache=dict(kind=2)), 1), (dict(cache=dict(batch=3)), 1)])
def test_a_step_refuses_what_its_calls_refuse(g, kw, code):
    kw = dict(kw)
    c, r = _cache(**kw.pop("cache", {})), _rule(**kw.pop("rule", {}))
    a = dict(held=NONE, ended=NONE, slots=VP, q=VP, ldq=64, k=VP, ldk=32, v=VP, ldv=32, times=NONE, out=VP, lse=NONE)
    a.update(kw)
    assert _call(g.load(), "gsit_cache_step", _shape(g), r, c, a["held"], a["ended"], a["slots"], a["q"], a["ldq"], a["k"], a["ldk"], a["v"], a["ldv"], a["times"], 10, 1, a["out"],
                 a["lse"], NONE, ctypes.c_size_t(0), None) == code


def test_a_cache_that_no_call_takes(g):
    """Refused when it is opened, before a plan has given pages to rows that nothing can hold."""
    for kw in (dict(head_dim=24), dict(head_dim=128), dict(head_dim=4), dict(dtype=torch.float16), dict(dtype=torch.float64), dict(held_as="fp8")):
        with pytest.raises(ValueError):
            g.stream_cache(**{**dict(batch=1, max_len=(3, 3, 3), kv_heads=1, head_dim=16, device="cpu"), **kw})
    cache = g.stream_cache(2, (40, 0, 64), 3, 8, torch.float32, "e4m3", device="cpu")
    assert cache.tables.shape == (2, 3, 2) and cache.keys.shape == (8, 3, 256) and cache.open_keys.dtype is torch.float32
