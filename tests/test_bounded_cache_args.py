"""Refusals of the rotary and bounded-cache calls: bad arguments are reported before anything is
launched, so they can be tested without a GPU (the pointers are never followed)."""
import ctypes

import pytest

fdp = pytest.importorskip("paper_2607_14898_gb300.flashdec")

P = 1 << 20  # an aligned address that is never used
INVALID, CONFIG = 1, 2


def rotary_config(**kw):
    d = dict(head_dim=64, rot_dim=64, layout=0, axes=3, axis_dims=(24, 20, 20), scaling=0,
             base=10000.0, factor=1.0, trained_len=1, fast_turns=32.0, slow_turns=1.0,
             amplitude=1.0)
    d.update(kw)
    d["axis_dims"] = (ctypes.c_int32 * 3)(*d["axis_dims"])
    return fdp.fd_rotary_config(*[d[n] for n, _ in fdp.fd_rotary_config._fields_])


def create(c):
    out = ctypes.c_void_p()
    return fdp.lib().fd_rotary_create(ctypes.byref(c), ctypes.byref(out)), out


@pytest.mark.parametrize("bad", [
    dict(head_dim=0), dict(head_dim=257, rot_dim=64), dict(rot_dim=63), dict(rot_dim=66),
    dict(head_dim=32), dict(layout=2), dict(layout=-1), dict(axes=0), dict(axes=4),
    dict(axis_dims=(24, 20, 18)), dict(axis_dims=(23, 21, 20)), dict(axis_dims=(44, 20, 0)),
    dict(axis_dims=(64, -20, 20)), dict(scaling=4), dict(base=0.0), dict(base=float("inf")),
    dict(scaling=1, factor=0.0), dict(scaling=2, factor=float("nan")),
    dict(scaling=3, trained_len=0), dict(scaling=3, fast_turns=1.0), dict(amplitude=float("nan")),
], ids=str)
def test_rotary_configurations_that_are_refused(bad):
    code, out = create(rotary_config(**bad))
    assert code == CONFIG and not out.value


def test_rotary_arguments():
    L = fdp.lib()
    assert L.fd_rotary_create(None, None) == INVALID
    assert L.fd_rotary_destroy(None) == INVALID
    code, plan = create(rotary_config())
    assert code == 0

    def call(**kw):
        d = dict(plan=plan, backward=0, dtype=1, tokens=4, pos=P, qh=2, q=P, qt=128, qs=64, qo=P,
                 qot=128, qos=64, kh=1, k=P, kt=64, ks=64, ko=P, kot=64, kos=64)
        d.update(kw)
        return L.fd_op_rotary(*d.values(), None)

    for bad in (dict(plan=None), dict(backward=2), dict(dtype=2), dict(dtype=-1), dict(tokens=-1),
                dict(pos=None), dict(pos=P + 2), dict(qh=-1), dict(kh=-1), dict(q=None),
                dict(qo=None), dict(q=P + 1), dict(k=None), dict(ko=P + 1), dict(qh=65537)):
        assert call(**bad) == INVALID, bad
    assert call(tokens=0) == 0 and call(qh=0, kh=0) == 0
    assert L.fd_rotary_destroy(plan) == 0


def cache(**kw):
    d = dict(streams=2, groups=4, capacity=100, head_dim=64, dtype=1, reserved=0, k=P, v=P,
             stream_stride=25600, group_stride=6400, slot_stride=64, pos=P, weight=P)
    d.update(kw)
    return fdp.fd_cache(*d.values())


BAD_CACHES = [
    dict(streams=-1), dict(groups=0), dict(capacity=-1), dict(capacity=(1 << 20) + 1),
    dict(head_dim=96), dict(dtype=0), dict(dtype=2), dict(reserved=1), dict(k=None), dict(v=None),
    dict(k=P + 8), dict(v=P + 2), dict(slot_stride=63), dict(slot_stride=56),
    dict(stream_stride=4), dict(group_stride=-8), dict(pos=None), dict(weight=None),
    dict(pos=P + 2)]


def attend(c, L, **kw):
    d = dict(used=100, heads=16, n_q=1, q=P, qs=1024, qt=1024, qh=64, q_pos=P, scale=0.125,
             decay=1.0, out=P, os=1024, ot=1024, oh=64, weight_out=P, work=P, err=P)
    d.update(kw)
    return L.fd_op_cache_attention(ctypes.byref(c), *d.values(), None)


def insert(c, L, **kw):
    d = dict(n=1, k=P, v=P, s=256, t=256, g=64, pos=P, sinks=0, recent=0, pos_out=P, weight_out=P,
             slots=P)
    d.update(kw)
    return L.fd_op_cache_insert(ctypes.byref(c), *d.values(), None)


def compact(c, dst, L, **kw):
    d = dict(now=P, sinks=0, recent=0, slots=P)
    d.update(kw)
    used = d.pop("used", 100)
    return L.fd_op_cache_compact(ctypes.byref(c), used, ctypes.byref(dst), *d.values(), None)


@pytest.mark.parametrize("bad", BAD_CACHES, ids=str)
def test_caches_that_are_refused(bad):
    L = fdp.lib()
    c, ok = cache(**bad), cache(capacity=10, k=2 * P, v=2 * P, pos=2 * P, weight=2 * P)
    assert attend(c, L, used=0) == INVALID
    assert insert(c, L) == INVALID
    assert compact(c, ok, L) == INVALID
    assert compact(cache(k=2 * P, v=2 * P, pos=2 * P, weight=2 * P), c, L) == INVALID
    assert L.fd_cache_attention_workspace_bytes(ctypes.byref(c), 0, 16, 1) == 0


def test_attention_arguments():
    L, c = fdp.lib(), cache()
    for bad in (dict(used=-1), dict(used=101), dict(heads=3), dict(heads=6), dict(heads=0),
                dict(n_q=-1), dict(q=None), dict(q=P + 2), dict(qt=1023), dict(qh=4), dict(qs=2),
                dict(q_pos=None), dict(out=None), dict(out=P + 4), dict(oh=60), dict(ot=2),
                dict(os=2), dict(weight_out=P + 1), dict(work=None), dict(work=P + 4),
                dict(err=None), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=0.0),
                dict(scale=-1.0),
                dict(decay=float("nan"))):
        assert attend(c, L, **bad) == INVALID, bad
    assert attend(cache(streams=0), L) == 0
    assert attend(c, L, n_q=0, weight_out=None) == 0
    assert L.fd_cache_attention_workspace_bytes(ctypes.byref(c), 100, 16, 0) == 0
    assert L.fd_cache_attention_workspace_bytes(ctypes.byref(c), 100, 6, 1) == 0
    assert L.fd_cache_attention_workspace_bytes(None, 100, 16, 1) == 0
    assert L.fd_cache_attention_workspace_bytes(ctypes.byref(c), 100, 16, 1) > 0


def test_rows_that_share_elements_are_refused():
    L, c = fdp.lib(), cache()
    for bad in (dict(qs=0), dict(qs=-1024), dict(qt=0, n_q=2), dict(qh=0), dict(qh=56),
                dict(os=0), dict(ot=0, n_q=2), dict(ot=-1024, n_q=2), dict(oh=32)):
        assert attend(c, L, **bad) == INVALID, bad
    for bad in (dict(stream_stride=0), dict(group_stride=0), dict(group_stride=56)):
        assert attend(cache(**bad), L) == INVALID, bad
        assert insert(cache(**bad), L) == INVALID, bad


def test_insert_arguments():
    L, c = fdp.lib(), cache()
    for bad in (dict(n=-1), dict(n=101), dict(k=None), dict(v=None), dict(k=P + 8), dict(v=P + 2),
                dict(s=4), dict(t=2), dict(g=60), dict(pos=None), dict(sinks=-1), dict(recent=-1),
                dict(pos_out=None), dict(weight_out=None), dict(pos_out=P + 1), dict(slots=None),
                dict(slots=P + 2)):
        assert insert(c, L, **bad) == INVALID, bad
    assert insert(cache(streams=0), L) == 0
    assert insert(cache(capacity=0), L, n=0) == 0
    assert insert(c, L, n=0) == 0  # the cache's own arrays: nothing to write


def test_compact_arguments():
    L, c = fdp.lib(), cache()
    other = dict(capacity=10, k=2 * P, v=2 * P, pos=2 * P, weight=2 * P)
    for bad in (dict(streams=1), dict(groups=2), dict(head_dim=128, slot_stride=128), dict(dtype=3),
                dict(k=P), dict(v=P), dict(pos=P), dict(weight=P)):
        assert compact(c, cache(**{**other, **bad}), L) == INVALID, bad
    ok = cache(**other)
    for bad in (dict(now=None), dict(now=P + 1), dict(slots=None), dict(sinks=-1), dict(recent=-1),
                dict(used=-1), dict(used=101), dict(used=9)):
        assert compact(c, ok, L, **bad) == INVALID, bad
    assert compact(cache(streams=0), cache(**{**other, "streams": 0}), L) == 0
    assert compact(c, cache(**{**other, "capacity": 0}), L, used=0) == 0
