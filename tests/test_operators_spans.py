"""Strides whose product with a size no memory holds are refused before addresses are formed
from them (no GPU needed)."""
import ctypes

import pytest

from paper_2506_08520_amd import binding as B
from test_operators_host import A, ESHAPE, L, norm, norm_back  # noqa: F401


@pytest.mark.parametrize("stride,rows", [(1 << 40, (1 << 31) - 1), (1 << 40, 1 << 24),
                                         (1 << 33, (1 << 31) - 1)])
def test_norm_rows_beyond_any_memory(L, stride, rows):  # noqa: F811
    far = dict(rows=rows, C=4)
    assert norm(L, xs=stride, ys=4, **far) == ESHAPE
    assert norm(L, xs=4, ys=stride, **far) == ESHAPE
    ws = dict(ws=A[8], wsb=1 << 30)
    for k in ("dys", "xs", "dxs"):
        assert norm_back(L, **{"dys": 4, "xs": 4, "dxs": 4, k: stride}, **far, **ws) == ESHAPE


@pytest.mark.parametrize("which", range(4))
@pytest.mark.parametrize("W,window,head", [((1 << 23), 1 << 40, 64), (1 << 22, 1 << 26, 1 << 40),
                                           (1 << 21, 1 << 39, 1 << 39)])
def test_views_beyond_any_memory(L, which, W, window, head):  # noqa: F811
    shape = B.DiffShape(W, 1, 1, 1, 1, 8, 16, 0, 0.0)
    views = [B.View(A[i], 64, 16, 16) for i in range(4)]
    views[which] = B.View(A[which], window, head, 16)
    q, k, v, o = (ctypes.byref(x) for x in views)
    assert L.nystra_diff_attn_forward(q, k, v, A[5], None, o, None, None, ctypes.byref(shape), 1,
                                      None, 0, None) == ESHAPE
