"""Refusals of the layer operators at the C boundary: every check runs before
anything is enqueued, so these need no GPU."""
import ctypes

import pytest

from paper_2506_08520_amd import binding as B

OK, ENULL, ESHAPE, EDTYPE, EALIGN, EOVERLAP, EUNSUP, EHIP, EARG, EWS = range(10)
M = 1 << 24
A = [M * (i + 1) for i in range(16)]     # fake, aligned, 16 MB apart


@pytest.fixture(scope="module")
def L():
    return B.lib()


def norm(L, x=A[0], xs=180, w=A[1], b=A[2], y=A[3], ys=180, mean=A[4], rstd=A[5], rows=64, C=180,
         eps=1e-5, dtype=1):
    return L.nystra_layer_norm_forward(x, xs, w, b, y, ys, mean, rstd, rows, C, eps, dtype, None)


def test_layer_norm_refusals(L):
    assert norm(L, dtype=2) == EDTYPE
    for kw in [dict(rows=-1), dict(rows=1 << 31), dict(C=0), dict(C=4097, xs=5000, ys=5000),
               dict(xs=179), dict(ys=0), dict(xs=-180), dict(xs=1 << 41)]:
        assert norm(L, **kw) == ESHAPE, kw
    for eps in (-1e-5, float("nan"), float("inf")):
        assert norm(L, eps=eps) == EARG
    for kw in [dict(x=None), dict(y=None), dict(mean=None), dict(rstd=None)]:
        assert norm(L, **kw) == ENULL, kw
    for kw in [dict(x=A[0] + 1), dict(y=A[3] + 1), dict(w=A[1] + 1), dict(mean=A[4] + 2),
               dict(dtype=0, b=A[2] + 2)]:
        assert norm(L, **kw) == EALIGN, kw
    n = 64 * 180 * 2
    for kw in [dict(y=A[0]), dict(y=A[0] + n - 2), dict(y=A[1] - n + 2), dict(mean=A[3]),
               dict(rstd=A[4] + 4), dict(mean=A[0] + 4)]:
        assert norm(L, **kw) == EOVERLAP, kw
    assert norm(L, rows=0, x=None, y=None) == OK


def norm_back(L, dy=A[0], dys=180, x=A[1], xs=180, w=A[2], mean=A[3], rstd=A[4], dx=A[5],
              dxs=180, dw=A[6], db=A[7], rows=64, C=180, dtype=1, ws=A[8], wsb=1 << 22):
    return L.nystra_layer_norm_backward(dy, dys, x, xs, w, mean, rstd, dx, dxs, dw, db, rows, C,
                                        dtype, ws, wsb, None)


def test_layer_norm_backward_refusals(L):
    assert norm_back(L, dtype=-1) == EDTYPE
    assert norm_back(L, C=5000) == ESHAPE and norm_back(L, dys=100) == ESHAPE
    for k in ("dy", "x", "mean", "rstd", "dx"):
        assert norm_back(L, **{k: None}) == ENULL, k
    for k in ("dy", "x", "w", "dx", "dw", "db"):
        assert norm_back(L, **{k: A[9] + 1}) == EALIGN, k
    for kw in [dict(dx=A[0]), dict(dx=A[1]), dict(dw=A[2]), dict(db=A[6] + 2), dict(dw=A[5]),
               dict(db=A[4])]:
        assert norm_back(L, **kw) == EOVERLAP, kw
    need = B.nystra_layer_norm_workspace_size(64, 180)
    assert need > 0
    for kw in [dict(ws=None), dict(wsb=need - 1), dict(ws=A[8] + 128), dict(ws=A[0]),
               dict(ws=A[7])]:
        assert norm_back(L, **kw) == EWS, kw
    n = ctypes.c_size_t(0)
    assert L.nystra_layer_norm_workspace_size(4, 180, None) == ENULL
    assert L.nystra_layer_norm_workspace_size(4, 0, ctypes.byref(n)) == ESHAPE
    assert norm_back(L, rows=0, dw=None, db=None, dy=None, x=None, mean=None, rstd=None, dx=None,
                     ws=None, wsb=0) == OK


def drop(L, x=A[0], r=A[1], y=A[2], n=1000, p=0.1, state=None, dtype=0):
    return L.nystra_dropout(x, r, y, n, p, 1, 2, state, dtype, None)


def test_dropout_refusals(L):
    assert drop(L, dtype=7) == EDTYPE
    assert drop(L, n=-1) == ESHAPE and drop(L, n=(1 << 34) + 1) == ESHAPE
    for p in (-0.01, 1.01, float("nan")):
        assert drop(L, p=p) == EARG
    assert drop(L, x=None) == ENULL and drop(L, y=None) == ENULL
    for kw in [dict(x=A[0] + 2), dict(r=A[1] + 1), dict(y=A[2] + 2), dict(state=A[3] + 4)]:
        assert drop(L, **kw) == EALIGN, kw
    for kw in [dict(y=A[0] + 4), dict(y=A[1] - 4), dict(state=A[2] + 8)]:
        assert drop(L, **kw) == EOVERLAP, kw
    assert drop(L, n=0, x=None, y=None) == OK


def shape(W=2, H=4, G=2, nq=64, nk=300, d=30, dv=60, causal=0, scale=0.0):
    return B.DiffShape(W, H, G, nq, nk, d, dv, causal, scale)


def views(s):
    """Contiguous views of every tensor at its own fake address."""
    def c(at, heads, tokens, width):
        return B.View(at, heads * tokens * width, tokens * width, width)
    W, H, G, nq, nk, d, dv = (s.n_windows, s.heads, s.kv_heads, s.n_q, s.n_k, s.d_qk, s.d_v)
    return dict(q=c(A[0], 2 * H, nq, d), k=c(A[1], 2 * G, nk, d), v=c(A[2], G, nk, dv),
                o=c(A[3], H, nq, dv), do=c(A[4], H, nq, dv), dq=c(A[5], 2 * H, nq, d),
                dk=c(A[6], 2 * G, nk, d), dv=c(A[7], G, nk, dv))


def forward(L, s=None, lam=A[8], kv=None, maps=A[9], sums=A[10], dtype=1, ws=None, wsb=0, **kw):
    s = shape() if s is None else s
    t = {**views(s), **kw}
    return L.nystra_diff_attn_forward(t["q"], t["k"], t["v"], lam, kv, t["o"], maps, sums, s, dtype,
                                      ws, wsb, None)


def backward(L, s=None, lam=A[8], kv=None, maps=A[9], sums=A[10], dlam=A[11], dtype=1, ws=A[12],
             wsb=1 << 23, **kw):
    s = shape() if s is None else s
    t = {**views(s), **kw}
    return L.nystra_diff_attn_backward(t["do"], t["q"], t["k"], t["v"], lam, kv, t["o"], maps, sums,
                                       t["dq"], t["dk"], t["dv"], dlam, s, dtype, ws, wsb, None)


@pytest.mark.parametrize("call", [forward, backward])
def test_diff_attention_shapes(L, call):
    assert call(L, dtype=2) == EDTYPE
    for kw in [dict(W=-1), dict(G=0), dict(H=1, G=2), dict(H=5, G=2), dict(nq=0), dict(nk=0),
               dict(nq=(1 << 20) + 1), dict(nk=(1 << 20) + 1), dict(d=0), dict(d=65), dict(dv=0),
               dict(dv=129), dict(W=1 << 22, H=4), dict(W=1 << 20, nq=64)]:
        assert call(L, s=shape(**kw)) == ESHAPE, kw
    for kw in [dict(causal=3), dict(causal=-1), dict(scale=float("nan")),
               dict(scale=float("inf"))]:
        assert call(L, s=shape(**kw)) == EARG, kw
    n = ctypes.c_size_t(0)
    assert L.nystra_diff_attn_workspace_size(None, 0, 1, ctypes.byref(n)) == ENULL
    assert L.nystra_diff_attn_workspace_size(shape(), 0, 1, None) == ENULL
    assert L.nystra_diff_attn_workspace_size(shape(d=65), 0, 1, ctypes.byref(n)) == ESHAPE


@pytest.mark.parametrize("call,outputs", [(forward, ("o",)), (backward, ("dq", "dk", "dv"))])
def test_diff_attention_tensors(L, call, outputs):
    t = views(shape())
    inputs = ("q", "k", "v") + (("do", "o") if call is backward else ())
    for name in inputs + outputs:
        v = t[name]
        assert call(L, **{name: B.View(None, v.window, v.head, v.token)}) == ENULL, name
        assert call(L, **{name: B.View(v.data + 1, v.window, v.head, v.token)}) == EALIGN, name
        assert call(L, **{name: B.View(v.data, -8, v.head, v.token)}) == ESHAPE, name
        assert call(L, **{name: B.View(v.data, v.window, 1 << 41, v.token)}) == ESHAPE, name
    for name in outputs:
        v = t[name]
        # rows that lie inside each other, heads and windows in one place
        for bad in ((v.window, v.head, v.token - 1), (v.window, 0, v.token), (0, v.head, v.token),
                    (v.token, v.head, v.token)):
            assert call(L, **{name: B.View(v.data, *bad)}) == EOVERLAP, (name, bad)
        assert call(L, **{name: B.View(t["q"].data, v.window, v.head, v.token)}) == EOVERLAP, name
        assert call(L, **{name: B.View(A[8], v.window, v.head, v.token)}) == EOVERLAP, name
    assert call(L, lam=None) == ENULL
    assert call(L, lam=A[8] + 2) == EALIGN and call(L, kv=A[13] + 2) == EALIGN
    assert call(L, sums=A[10] + 2) == EALIGN


def test_diff_attention_saved_values(L):
    # bf16, many keys: both; few: the sums alone; fp32: both; inference: neither
    assert forward(L, sums=None) == ENULL
    assert forward(L, maps=None) == ENULL
    assert forward(L, s=shape(nk=256)) == ENULL
    assert backward(L, maps=None) == ENULL and backward(L, sums=None) == ENULL
    assert backward(L, s=shape(nk=256)) == ENULL
    assert forward(L, s=shape(nk=256), dtype=0, maps=None) == ENULL
    assert backward(L, s=shape(nk=256), dtype=0, maps=None) == ENULL
    assert backward(L, dlam=None) == ENULL and backward(L, dlam=A[11] + 1) == EALIGN
    assert forward(L, sums=A[3]) == EOVERLAP and forward(L, maps=A[0]) == EOVERLAP
    assert backward(L, dlam=A[5]) == EOVERLAP and backward(L, dlam=A[8]) == EOVERLAP


def test_diff_attention_workspaces(L):
    need = B.nystra_diff_attn_workspace_size(shape(), True)
    for kw in [dict(ws=None), dict(wsb=need - 1), dict(ws=A[12] + 64), dict(ws=A[0]),
               dict(ws=A[7])]:
        assert backward(L, **kw) == EWS, kw
    s = shape(W=1, nq=1, nk=4096)
    need = B.nystra_diff_attn_workspace_size(s)
    assert need > 0
    for kw in [dict(ws=None, wsb=need), dict(ws=A[12], wsb=need - 1), dict(ws=A[12] + 4, wsb=need),
               dict(ws=A[3], wsb=need)]:
        assert forward(L, s=s, maps=None, sums=None, **kw) == EWS, kw
    assert B.nystra_diff_attn_workspace_size(shape(W=0), True) == 0


def test_no_windows_is_a_no_op(L):
    null = B.View(None, 0, 0, 0)
    s = shape(W=0)
    assert forward(L, s=s, q=null, k=null, v=null, o=null, lam=None, maps=None, sums=None) == OK


def test_binding_refuses_host_tensors():
    import torch
    x = torch.zeros(4, 8)
    q = torch.zeros(1, 2, 4, 8)
    for f in (lambda: B.nystra_layer_norm_forward(x), lambda: B.nystra_dropout(x, 0.1),
              lambda: B.nystra_diff_attn_forward(q, q, q[:, :1], torch.zeros(1)),
              lambda: B.nystra_dropout(x=x, p=0.5)):
        with pytest.raises(ValueError):
            f()
