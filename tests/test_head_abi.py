"""Refusals of the head's entry points, without a GPU: every check comes before the first launch."""
import ctypes

import pytest

from paper_1910_00932_amd import binding as B

A = 1 << 20      # fake, aligned, never dereferenced
BIG = 1 << 40


def _p(i):
    return A + i * BIG


def _recur(**kw):
    v = dict(N=2, T=300, C=64, H=1, W=1, dtype=B.TSM_BF16)
    v.update(kw)
    return B.RecurDesc(**v)


def _fwd(d, x=_p(0), g=_p(1), h0=None, y=_p(2), hl=None, saved=None, ws=_p(3), n=1 << 40):
    return B.lib().tsm_recur_fwd(ctypes.addressof(d) if d else None, x, g, h0, y, hl, saved, ws, n, None)


def _bwd(d, x=_p(0), g=_p(1), h0=None, saved=_p(4), dy=_p(5), dl=None, dx=_p(6), dg=_p(7), dh0=None, ws=_p(3), n=1 << 40):
    return B.lib().tsm_recur_bwd(ctypes.addressof(d) if d else None, x, g, h0, saved, dy, dl, dx, dg, dh0, ws, n, None)


def test_recur_refusals():
    d = _recur()
    assert _fwd(None) == -1 and _fwd(d, x=None) == -1 and _fwd(d, g=None) == -1 and _fwd(d, y=None) == -1
    for bad in (dict(N=0), dict(T=0), dict(T=-3), dict(C=0), dict(H=0), dict(W=-1), dict(N=2 ** 31 - 1, T=2 ** 31 - 1, C=2 ** 31 - 1)):
        assert _fwd(_recur(**bad)) == -2 and _bwd(_recur(**bad)) == -2, bad
        assert B.tsm_recur_saved_bytes(_recur(**bad)) == 0 and B.tsm_recur_workspace_bytes(_recur(**bad)) == 0
    assert _fwd(_recur(dtype=2)) == -4 and _bwd(_recur(dtype=-1)) == -4
    assert _fwd(d, x=_p(0) + 2) == -7 and _bwd(d, dg=_p(7) + 8) == -7
    n = 2 * 300 * 64 * 2
    assert _fwd(d, y=_p(0)) == -2 and _fwd(d, y=_p(1) + n - 16) == -2 and "overlap" in B.tsm_last_error()
    assert _fwd(d, h0=_p(8), hl=_p(8) + 16) == -2                       # in place, or apart
    assert _bwd(d, dx=_p(0)) == -2 and _bwd(d, dx=_p(7)) == -2 and _bwd(d, dl=_p(9), dh0=_p(9)) == -2
    assert _bwd(d, saved=None) == -1 and _bwd(d, dy=None) == -1 and _bwd(d, dx=None) == -1
    assert B.tsm_recur_saved_bytes(_recur(T=128)) == 0 and B.tsm_recur_saved_bytes(_recur(T=129)) == 2 * 64 * 4
    need = B.tsm_recur_workspace_bytes(d)
    assert need > 0
    assert _fwd(d, n=need - 1) == -6 and _bwd(d, n=need - 1) == -6 and _fwd(d, ws=None, n=need) == -1
    assert "workspace" in B.tsm_last_error() and B.tsm_recur_workspace_bytes(_recur(T=1)) == 0


def _ln(**kw):
    v = dict(rows=100, C=64, dtype=B.TSM_BF16, eps=1e-5)
    v.update(kw)
    return B.LayerNormDesc(**v)


def test_layernorm_refusals():
    L = B.lib()

    def fwd(d, x=_p(0), g=_p(1), b=_p(2), y=_p(3), m=None, r=None):
        return L.tsm_layernorm_fwd(ctypes.addressof(d) if d else None, x, g, b, y, m, r, None)

    def bwd(d, x=_p(0), dy=_p(1), g=_p(2), m=_p(3), r=_p(4), dx=_p(5), dg=_p(6), db=_p(7), ws=_p(8), n=1 << 40):
        return L.tsm_layernorm_bwd(ctypes.addressof(d) if d else None, x, dy, g, m, r, dx, dg, db, ws, n, None)
    d = _ln()
    assert fwd(None) == -1 and fwd(d, x=None) == -1 and fwd(d, b=None) == -1 and bwd(d, m=None) == -1 and bwd(d, dg=None) == -1
    for bad in (dict(rows=0), dict(C=0), dict(C=-4), dict(rows=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(rows=2 ** 62, C=1000)):
        assert fwd(_ln(**bad)) == -2 and bwd(_ln(**bad)) == -2, bad
        assert B.tsm_layernorm_workspace_bytes(_ln(**bad)) == 0
    assert fwd(_ln(dtype=7)) == -4 and bwd(_ln(dtype=7)) == -4
    assert fwd(d, y=_p(0)) == -2 and fwd(d, y=_p(0) + 100 * 64 * 2 - 16) == -2 and fwd(d, m=_p(9), r=_p(9)) == -2
    assert bwd(d, dx=_p(1)) == -2 and bwd(d, dg=_p(7)) == -2 and bwd(d, ws=_p(0)) == -2
    assert fwd(d, x=_p(0) + 4) == -7 and bwd(d, r=_p(4) + 4) == -7
    need = B.tsm_layernorm_workspace_bytes(d)
    assert need >= 2 * 64 * 4 and bwd(d, n=need - 1) == -6 and bwd(d, ws=None, n=need) == -1


def _xe(**kw):
    v = dict(rows=100, features=64, classes=400, dtype=B.TSM_BF16)
    v.update(kw)
    return B.XentDesc(**v)


def test_xent_refusals():
    L = B.lib()

    def fwd(d, x=_p(0), w=_p(1), b=None, lab=_p(2), loss=_p(3), lse=_p(4), ws=_p(5), n=1 << 40):
        return L.tsm_xent_fwd(ctypes.addressof(d) if d else None, x, w, b, lab, loss, lse, ws, n, None)

    def bwd(d, x=_p(0), w=_p(1), b=None, lab=_p(2), lse=_p(4), up=_p(6), dx=_p(7), dw=_p(8), db=None, ws=_p(5), n=1 << 40):
        return L.tsm_xent_bwd(ctypes.addressof(d) if d else None, x, w, b, lab, lse, up, dx, dw, db, ws, n, None)
    d = _xe()
    assert fwd(None) == -1 and fwd(d, lab=None) == -1 and fwd(d, lse=None) == -1 and bwd(d, up=None) == -1
    assert bwd(d, dx=None, dw=None) == -1 and "gradient" in B.tsm_last_error()
    for bad in (dict(rows=0), dict(features=0), dict(classes=0), dict(classes=-5), dict(rows=2 ** 31 - 1, features=2 ** 31 - 1)):
        assert fwd(_xe(**bad)) == -2 and bwd(_xe(**bad)) == -2, bad
        assert B.tsm_xent_workspace_bytes(_xe(**bad)) == 0
    assert fwd(_xe(dtype=3)) == -4 and bwd(_xe(dtype=3)) == -4
    assert fwd(d, loss=_p(4)) == -2 and bwd(d, dx=_p(0)) == -2 and bwd(d, dw=_p(1)) == -2 and bwd(d, db=_p(6)) == -2
    assert fwd(d, w=_p(1) + 2) == -7 and bwd(d, dw=_p(8) + 4) == -7
    need = B.tsm_xent_workspace_bytes(d)
    assert need > 0 and fwd(d, n=need - 1) == -6 and bwd(d, n=need - 1) == -6 and fwd(d, ws=None, n=need) == -1


def test_tensors_that_are_not_contiguous_are_refused():
    import torch
    t = torch.zeros(4, 6).t()
    with pytest.raises(ValueError):
        B.tsm_layernorm_fwd(_ln(), t, t, t, t, None, None)


@pytest.mark.parametrize("dtype", [B.TSM_BF16, B.TSM_F32])
@pytest.mark.parametrize("rows", [1, 5, 64, 65, 255, 300, 5000])
def test_xent_workspace_does_not_grow_with_the_classes(rows, dtype):
    """A piece of G has 512 MB at most, rounded-up rows included, so that from some number of classes on the workspace grows by the
    forward pass's 8 bytes per row and tile of classes alone."""
    few, many = (B.tsm_xent_workspace_bytes(_xe(rows=rows, features=8, classes=n, dtype=dtype)) for n in (3000000, 300000000))
    tiles = rows * 8 * (300000000 // 32 + 1000)
    assert few < (1 << 30) + (1 << 29) and many < (1 << 30) + (1 << 29) + tiles, (few, many)
