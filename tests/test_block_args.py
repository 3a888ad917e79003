"""Refusals of the checkpoint and block-join calls: bad arguments are reported before anything is
launched, so they can be tested without a GPU (the pointers are never followed)."""
import ctypes

import pytest

fdp = pytest.importorskip("paper_2607_14898_gb300.flashdec")

P = 1 << 20  # an aligned address that is never used
INVALID = 1


def test_checkpoint_save():
    L = fdp.lib()

    def call(**kw):
        d = dict(dtype=1, rows=4, width=64, x=P, stride=64, codes=P, exps=P)
        d.update(kw)
        return L.fd_op_checkpoint_save(*d.values(), None)

    for bad in (dict(dtype=2), dict(dtype=-1), dict(dtype=4), dict(rows=-1), dict(width=0), dict(width=60),
                dict(width=-8), dict(width=(1 << 20) + 8), dict(x=None), dict(x=P + 8),
                dict(stride=63), dict(codes=None), dict(codes=P + 4), dict(exps=None)):
        assert call(**bad) == INVALID, bad
    assert call(rows=0, x=None, codes=None, exps=None) == 0


def test_checkpoint_load():
    L = fdp.lib()

    def call(**kw):
        d = dict(dtype=1, transposed=0, rows=4, width=64, codes=P, exps=P, x=P, stride=64)
        d.update(kw)
        return L.fd_op_checkpoint_load(*d.values(), None)

    for bad in (dict(dtype=2), dict(transposed=2), dict(transposed=-1), dict(rows=-1), dict(width=4),
                dict(codes=None), dict(codes=P + 1), dict(exps=None), dict(x=None), dict(x=P + 2),
                dict(stride=60), dict(stride=56), dict(transposed=1, stride=3),
                dict(transposed=1, x=P + 1, stride=4), dict(transposed=1, dtype=0, x=P + 2, stride=4)):
        assert call(**bad) == INVALID, bad
    assert call(rows=0, x=None) == 0


def view(**kw):
    d = dict(rows=4, width=64, dtype=1, stream_dtype=0, post=P, pre=P, gate=P, gate_rows=2, scale=1.0)
    d.update(kw)
    return ctypes.byref(fdp.fd_block_join(*d.values()))


BAD_VIEWS = [dict(rows=-1), dict(width=0), dict(width=68), dict(width=8200), dict(dtype=0),
             dict(dtype=2), dict(stream_dtype=3), dict(dtype=3, stream_dtype=1), dict(stream_dtype=2),
             dict(post=P + 4), dict(pre=P + 8), dict(gate=P + 4), dict(gate_rows=0),
             dict(scale=float("nan")), dict(scale=float("inf"))]


def join(L, j, **kw):
    d = dict(h=P, hs=64, b=P, bs=64, eps=1e-6, y=P, ys=64, u=P, us=64, r_post=P, r_pre=P, hc=P, he=P,
             bc=P, be=P)
    d.update(kw)
    return L.fd_op_block_join(j, *d.values(), None)


def test_block_join():
    L = fdp.lib()
    assert join(L, None) == INVALID
    for bad in BAD_VIEWS:
        assert join(L, view(**bad)) == INVALID, bad
    for bad in (dict(h=None), dict(h=P + 8), dict(hs=63), dict(hs=56), dict(b=None), dict(b=P + 2),
                dict(bs=8), dict(y=None), dict(ys=60), dict(u=None), dict(u=P + 2), dict(us=0),
                dict(eps=-1.0), dict(eps=float("nan")), dict(r_post=P + 2), dict(r_pre=P + 1),
                dict(hc=None), dict(he=None), dict(hc=P + 4), dict(bc=None), dict(be=None),
                dict(bc=P + 1)):
        assert join(L, view(), **bad) == INVALID, bad
    assert join(L, view(pre=None)) == INVALID  # u without a gain
    assert join(L, view(rows=0), h=None, b=None, y=None, u=None) == 0


def test_block_join_bwd():
    L = fdp.lib()

    def call(j, **kw):
        d = dict(dy=P, dys=64, du=P, dus=64, h=P, hs=64, he=None, b=P, bs=64, be=None, r_post=P,
                 r_pre=P, dh=P, dhs=64, db=P, dbs=64, d_post=P, d_pre=P, d_gate=P, work=P)
        d.update(kw)
        return L.fd_op_block_join_bwd(j, *d.values(), None)

    assert call(None) == INVALID
    for bad in BAD_VIEWS:
        assert call(view(**bad)) == INVALID, bad
    for bad in (dict(dy=P + 8), dict(dys=60), dict(du=None), dict(du=P + 4), dict(h=None), dict(hs=8),
                dict(he=P, hs=72), dict(he=P, h=P + 4), dict(b=None), dict(be=P, bs=72),
                dict(be=P, b=P + 1), dict(r_post=None), dict(r_pre=None), dict(dh=P + 2), dict(dhs=8),
                dict(db=P + 2), dict(dbs=8), dict(d_post=P + 4), dict(d_pre=P + 4),
                dict(d_gate=P + 4), dict(work=None), dict(work=P + 8)):
        assert call(view(), **bad) == INVALID, bad
    # sums of what is not there; no gradient at all
    assert call(view(post=None)) == INVALID
    assert call(view(gate=None)) == INVALID
    assert call(view(pre=None), d_pre=None) == INVALID  # du without a gain
    assert call(view(pre=None), d_pre=None, du=None, dy=None) == INVALID
    assert call(view(rows=0), d_post=None, d_pre=None) == 0


def test_workspace():
    L = fdp.lib()
    for rows, width in ((0, 64), (-1, 64), (4, 60), (4, 0), (4, 8200)):
        assert L.fd_block_join_bwd_workspace_bytes(rows, width) == 0
    assert L.fd_block_join_bwd_workspace_bytes(1, 64) == 4 * 64 * 4


def test_rows_past_the_limit():
    L = fdp.lib()
    assert join(L, view(rows=(1 << 30) + 1)) == INVALID
    assert L.fd_block_join_bwd_workspace_bytes((1 << 30) + 1, 64) == 0
    assert L.fd_block_join_bwd_workspace_bytes(1 << 30, 64) > 0
    assert L.fd_op_checkpoint_save(1, (1 << 30) + 1, 64, P, 64, P, P, None) == INVALID
    assert L.fd_op_checkpoint_load(1, 0, (1 << 30) + 1, 64, P, P, P, 64, None) == INVALID


JOIN = ("h", "b", "y", "u", "r_post", "r_pre", "hc", "he", "bc", "be")
JOIN_BWD = ("dy", "du", "h", "b", "r_post", "r_pre", "dh", "db", "d_post", "d_pre", "d_gate", "work")


@pytest.mark.parametrize("a,b,more", [
    ("y", "u", {}), ("y", "b", {}), ("u", "h", {}), ("r_post", "r_pre", {}), ("hc", "bc", {}), ("he", "be", {}),
    ("y", "h", dict(ys=72)), ("u", "b", dict(bs=72))])
def test_join_results_in_each_others_place(a, b, more):
    at = {name: P * (2 + i) for i, name in enumerate(JOIN)}
    assert join(fdp.lib(), view(), **{**at, a: at[b], **more}) == INVALID


@pytest.mark.parametrize("a,b,more", [
    ("dh", "db", {}), ("dh", "du", {}), ("dh", "h", {}), ("dh", "b", {}), ("db", "dy", {}), ("db", "h", {}),
    ("d_post", "d_pre", {}), ("d_post", "d_gate", {}), ("d_pre", "d_gate", {}), ("dh", "dy", dict(dhs=72)),
    ("db", "du", dict(dbs=72)), ("db", "b", dict(bs=72)), ("db", "b", dict(be=P))])
def test_gradients_in_each_others_place(a, b, more):
    d = dict(dy=P, dys=64, du=P, dus=64, h=P, hs=64, he=None, b=P, bs=64, be=None, r_post=P, r_pre=P, dh=P,
             dhs=64, db=P, dbs=64, d_post=P, d_pre=P, d_gate=P, work=P)
    d.update({name: P * (2 + i) for i, name in enumerate(JOIN_BWD)})
    d.update({a: d[b], **more})
    assert fdp.lib().fd_op_block_join_bwd(view(), *d.values(), None) == INVALID
