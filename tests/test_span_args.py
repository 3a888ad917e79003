"""Refusals of the span-attention calls: bad arguments are reported before anything is launched, so they
can be tested without a GPU (the pointers are never followed)."""
import ctypes

import pytest

fdp = pytest.importorskip("paper_2607_14898_gb300.flashdec")

P = 1 << 20  # an aligned address that is never used
INVALID = 1


def view(**kw):
    d = dict(n_q=100, n_k=300, heads=8, groups=2, head_dim=64, dtype=1, scale=0.125)
    d.update(kw)
    return ctypes.byref(fdp.fd_span_attention(*d.values()))


BAD_VIEWS = [dict(n_q=-1), dict(n_k=-1), dict(n_q=(1 << 24) + 1), dict(n_k=(1 << 24) + 1), dict(heads=0),
             dict(heads=7), dict(groups=0), dict(heads=-8), dict(heads=129, groups=1), dict(heads=65536, groups=65536),
             dict(n_q=1 << 24, heads=8192, groups=64), dict(n_k=1 << 24, heads=8192, groups=8192),
             dict(head_dim=32), dict(head_dim=96), dict(dtype=0), dict(dtype=2), dict(scale=0.0),
             dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf"))]

ROWS = [dict(p=None), dict(p=P + 8), dict(t=63), dict(t=56), dict(t=-512), dict(h=60), dict(h=8), dict(h=0)]


def forward(L, a, **kw):
    d = dict(q_p=P, q_t=512, q_h=64, k_p=P, k_t=128, k_h=64, v_p=P, v_t=128, v_h=64, spans=P, out_p=P, out_t=512,
             out_h=64, lse=P, work=P, err=P)
    d.update(kw)
    return L.fd_op_span_attention(a, *d.values(), None)


def backward(L, a, **kw):
    d = dict(q_p=P, q_t=512, q_h=64, k_p=P, k_t=128, k_h=64, v_p=P, v_t=128, v_h=64, spans=P, out_p=P, out_t=512,
             out_h=64, lse=P, dout_p=P, dout_t=512, dout_h=64, dq_p=P, dq_t=512, dq_h=64, dk_p=P, dk_t=128,
             dk_h=64, dv_p=P, dv_t=128, dv_h=64, work=P, err=P)
    d.update(kw)
    return L.fd_op_span_attention_bwd(a, *d.values(), None)


@pytest.mark.parametrize("call,names", [(forward, ("q", "k", "v", "out")),
                                        (backward, ("q", "k", "v", "out", "dout", "dq", "dk", "dv"))])
def test_arguments(call, names):
    L = fdp.lib()
    assert call(L, None) == INVALID
    for bad in BAD_VIEWS:
        assert call(L, view(**bad)) == INVALID, bad
    for name in names:
        for bad in ROWS:
            if bad.get("t") == 56 or bad.get("h") == 8:  # rows that share elements
                bad = {**bad}
            assert call(L, view(), **{f"{name}_{x}": v for x, v in bad.items()}) == INVALID, (name, bad)
    for bad in (dict(spans=None), dict(spans=P + 4), dict(lse=None), dict(lse=P + 2), dict(err=None),
                dict(err=P + 1)):
        assert call(L, view(), **bad) == INVALID, bad


def test_workspace_is_required_where_there_are_parts():
    L = fdp.lib()
    assert backward(L, view(), work=None) == INVALID and backward(L, view(), work=P + 8) == INVALID
    # few queries over many keys are split between blocks
    many = dict(n_q=1, n_k=100000, heads=1, groups=1)
    if L.fd_span_attention_workspace_bytes(view(**many), 0):
        assert forward(L, view(**many), work=None) == INVALID


def test_nothing_to_do():
    L = fdp.lib()
    assert forward(L, view(n_q=0), q_p=None, out_p=None, spans=None, lse=None) == 0
    assert backward(L, view(n_q=0, n_k=0)) == 0


def test_workspace_bytes():
    L = fdp.lib()
    assert L.fd_span_attention_workspace_bytes(None, 0) == 0
    for bad in BAD_VIEWS:
        for backward_ in (0, 1):
            assert L.fd_span_attention_workspace_bytes(view(**bad), backward_) == 0
    assert L.fd_span_attention_workspace_bytes(view(n_q=0), 1) == 0
    assert L.fd_span_attention_workspace_bytes(view(n_k=0), 1) == 0
    assert L.fd_span_attention_workspace_bytes(view(), 1) > 0


def distinct(names):
    """An address of its own for each name, far apart."""
    return {name: P * (2 + i) for i, name in enumerate(names)}


@pytest.mark.parametrize("shared,with_", [("out_p", n) for n in ("q_p", "k_p", "v_p", "spans", "lse")])
def test_result_in_the_place_of_an_input(shared, with_):
    at = distinct(("q_p", "k_p", "v_p", "spans", "out_p", "lse", "work", "err"))
    assert forward(fdp.lib(), view(), **{**at, shared: at[with_]}) == INVALID


@pytest.mark.parametrize("shared,with_", [(a, b) for i, a in enumerate(("dq_p", "dk_p", "dv_p")) for b in (
    "q_p", "k_p", "v_p", "spans", "out_p", "lse", "dout_p", "work", *("dq_p", "dk_p", "dv_p")[i + 1:])])
def test_gradient_in_the_place_of_another(shared, with_):
    at = distinct(("q_p", "k_p", "v_p", "spans", "out_p", "lse", "dout_p", "dq_p", "dk_p", "dv_p", "work", "err"))
    assert backward(fdp.lib(), view(), **{**at, shared: at[with_]}) == INVALID


@pytest.mark.parametrize("call,name,token,head", [
    (forward, "out", 448, 64), (forward, "out", 64, 64), (forward, "out", 64, 6392), (backward, "dq", 448, 64),
    (backward, "dk", 64, 64), (backward, "dv", 64, 19192)])
def test_results_whose_rows_share_elements(call, name, token, head):
    # (8 heads or 2 groups of 64 within a token's stride, or 100 or 300 tokens within a head's)
    at = distinct(("q_p", "k_p", "v_p", "out_p", "lse", "work", "err")) if call is forward else distinct(
        ("q_p", "k_p", "v_p", "out_p", "lse", "dout_p", "dq_p", "dk_p", "dv_p", "work", "err"))
    assert call(fdp.lib(), view(), **at, **{f"{name}_t": token, f"{name}_h": head}) == INVALID
