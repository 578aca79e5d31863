"""Layer norm and its backward pass against the definition in 64 bits.

Bounds.  A sum of C values over lanes has chains of at most n = 48 + C/256 additions: off by n units of 2^-24 of the sum of
magnitudes.  With m = n units of mean |x| for the mean, xhat is off by rstd*m plus (2n + 8) units of |xhat| (the variance's
relative error, halved by the root, and a few roundings)."""
import numpy as np
import pytest
import torch

from oracle import head_oracle as H
from paper_1910_00932_amd import binding as B
from head_util import CDT, HALF, TDT, U, Guarded, scratch, values, within

pytestmark = pytest.mark.gpu

SHAPES = [  # rows, C
    (1, 1), (5, 1), (3, 2), (9, 7), (700, 64), (1300, 65), (33, 127), (40, 128), (31, 129), (50, 250), (64, 256), (37, 257), (20, 511),
    (21, 513), (300, 1000), (41, 1024), (19, 1025), (2100, 2048), (17, 2049), (13, 4095), (12, 4097), (9, 8192), (70, 8193), (3, 20001),
]
EPS = 1e-5


def _run(rows, C, dtype, shift, eps=EPS, x=None):
    d = B.LayerNormDesc(rows=rows, C=C, dtype=CDT[dtype], eps=eps)
    xd, xn = values((rows, C), 0, dtype, scale=1.5, shift=shift) if x is None else x
    dyd, dyn = values((rows, C), 1, dtype)
    gd, gn = values((C,), 2, "f32", scale=0.3, shift=1.0)
    bd, bn = values((C,), 3, "f32")
    y, mean, rstd = Guarded((rows, C), TDT[dtype]), Guarded((rows,), torch.float32), Guarded((rows,), torch.float32)
    B.tsm_layernorm_fwd(d, xd, gd, bd, y.t, mean.t, rstd.t)
    dx, dg, db = Guarded((rows, C), TDT[dtype]), Guarded((C,), torch.float32), Guarded((C,), torch.float32)
    B.tsm_layernorm_bwd(d, xd, dyd, gd, mean.t, rstd.t, dx.t, dg.t, db.t, scratch(B.tsm_layernorm_workspace_bytes(d)))
    torch.cuda.synchronize()
    return (xn, dyn, gn, bn), [v.np() for v in (y, mean, rstd, dx, dg, db)]


@pytest.mark.parametrize("shift", [0.3, 50.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward_and_backward(shape, dtype, shift):
    rows, C = shape
    (x, dy, gamma, beta), (y, mean, rstd, dx, dg, db) = _run(rows, C, dtype, shift)
    ry, rmean, rrstd = H.layernorm_fwd(x, gamma, beta, EPS)
    n = 48 + C / 256
    m = n * U * np.abs(x).mean(1)
    within(mean, rmean, m + U * np.abs(rmean), "mean")
    # (the centred values are off by the mean's error and their own rounding, c; their mean square by 2 c sqrt(var) + c^2)
    c = m + U * np.abs(x).max(1)
    var = ((x - rmean[:, None]) ** 2).mean(1)
    rel = ((n + 4) * U * var + 2 * c * np.sqrt(var) + c ** 2) / (var + EPS) + 4 * U
    within(rstd, rrstd, rel * rrstd, "rstd")
    xhat = (x - rmean[:, None]) * rrstd[:, None]
    exh = (c * rrstd)[:, None] + (rel + 4 * U)[:, None] * (np.abs(xhat) + (c * rrstd)[:, None])
    within(y, ry, np.abs(gamma) * exh + 4 * U * (np.abs(gamma * xhat) + np.abs(beta)) + HALF[dtype] * np.abs(ry), "y")
    rdx, rdg, rdb = H.layernorm_bwd(x, dy, gamma, EPS)
    v = np.abs(dy * gamma)
    e1 = (n + 2) * U * v.mean(1)
    e2 = (n + 4) * U * (v * np.abs(xhat)).mean(1) + (v * exh).mean(1)
    m2 = np.abs((dy * gamma * xhat).mean(1))
    size = v + v.mean(1, keepdims=True) + np.abs(xhat) * (m2 + e2)[:, None]
    bound = rrstd[:, None] * (e1[:, None] + np.abs(xhat) * e2[:, None] + exh * (m2 + e2)[:, None] + 8 * U * size) + rel[:, None] * rrstd[:, None] * size
    within(dx, rdx, bound + HALF[dtype] * np.abs(rdx), "dx")
    k = rows / 256 + 64                           # chain of the weights' gradients: a block's rows, its groups, the blocks
    within(dg, rdg, (np.abs(dy) * exh).sum(0) + k * U * (np.abs(dy * xhat)).sum(0), "dgamma")
    within(db, rdb, k * U * np.abs(dy).sum(0), "dbeta")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_are_constant(dtype):
    x = np.tile(np.array([[0.0], [3.0], [-512.0]], np.float32), (1, 100))
    t = torch.from_numpy(x).to(TDT[dtype])
    (_, dy, gamma, beta), (y, mean, rstd, dx, dg, db) = _run(3, 100, dtype, 0, x=(t.cuda(), t.double().numpy()))
    assert np.array_equal(mean, x[:, 0].astype(np.float64))
    within(y, np.tile(beta, (3, 1)), HALF[dtype] * np.abs(beta) + 1e-30, "y")
    within(rstd, np.full(3, EPS ** -0.5), 4 * U * EPS ** -0.5, "rstd")


def test_bad_rows_stay_alone():
    xd, xn = values((40, 300), 0, "f32")
    xd[7, 299] = float("inf")
    xd[20, 0] = float("nan")
    _, (y, mean, rstd, dx, dg, db) = _run(40, 300, "f32", 0, x=(xd, xn))
    bad = np.zeros(40, bool)
    bad[[7, 20]] = True
    assert np.isnan(y[bad]).all() and np.isfinite(y[~bad]).all() and np.isfinite(dx[~bad]).all()


def test_statistics_are_optional_and_bits_repeat():
    for C in (2048, 9000):
        d = B.LayerNormDesc(rows=77, C=C, dtype=B.TSM_BF16, eps=EPS)
        a, b = _run(77, C, "bf16", 0.3)[1], _run(77, C, "bf16", 0.3)[1]
        assert all(np.array_equal(p, q) for p, q in zip(a, b))
        xd, _ = values((77, C), 0, "bf16", scale=1.5, shift=0.3)
        gd, _ = values((C,), 2, "f32", scale=0.3, shift=1.0)
        bd, _ = values((C,), 3, "f32")
        y = Guarded((77, C), torch.bfloat16)
        B.tsm_layernorm_fwd(d, xd, gd, bd, y.t, None, None)
        assert np.array_equal(y.np(), a[0])


@pytest.mark.parametrize("dtype,C,x0,spread", [("f32", 1 << 23, 0.3, 0.0), ("f32", 3 << 21, 1.0, 0.1), ("bf16", (1 << 24) + 1, 0.3, 0.02)])
def test_sums_over_very_long_rows(dtype, C, x0, spread):
    """Values of one sign, or one value, in which every rounding of a long sum leans the same way.  A value is among at most n = 400
    additions in turn -- 8 of a vector, 64, 64 and up to 256 of them, the wavefront's and the block's -- and the sums are off by n units of
    2^-24 of their magnitudes, whatever C.  As above, xhat is off by c = n units of mean |x|, and a unit of |x|, times rstd."""
    rng = np.random.default_rng(5)
    t = torch.from_numpy((x0 + spread * rng.standard_normal((1, C))).astype(np.float32)).to(TDT[dtype])
    x, g, b = t.double().numpy(), np.full(C, 0.75), np.full(C, 0.5)
    dyt = torch.from_numpy((0.3 + spread * rng.standard_normal((1, C))).astype(np.float32)).to(TDT[dtype])
    dy = dyt.double().numpy()
    d = B.LayerNormDesc(rows=1, C=C, dtype=CDT[dtype], eps=EPS)
    xd, dyd, gd, bd = t.cuda(), dyt.cuda(), torch.full((C,), 0.75, device="cuda"), torch.full((C,), 0.5, device="cuda")
    y, mean, rstd = Guarded((1, C), TDT[dtype]), Guarded((1,), torch.float32), Guarded((1,), torch.float32)
    B.tsm_layernorm_fwd(d, xd, gd, bd, y.t, mean.t, rstd.t)
    n = 400
    rmean = x.mean()
    var = ((x - rmean) ** 2).mean()
    rrstd = (var + EPS) ** -0.5
    m = n * U * np.abs(x).mean() + U * abs(rmean)
    c = m + U * np.abs(x).max()
    rel = ((n + 4) * U * var + 2 * c * np.sqrt(var) + c ** 2) / (var + EPS) + 4 * U
    within(mean.np(), np.array([rmean]), m, "mean")
    within(rstd.np(), np.array([rrstd]), rel * rrstd, "rstd")
    xhat = (x - rmean) * rrstd
    exh = c * rrstd + (rel + 4 * U) * (np.abs(xhat) + c * rrstd)
    ry = xhat * g + b
    within(y.np(), ry, g * exh + 4 * U * (np.abs(g * xhat) + np.abs(b)) + HALF[dtype] * np.abs(ry), "y")
    dx, dg, db = Guarded((1, C), TDT[dtype]), Guarded((C,), torch.float32), Guarded((C,), torch.float32)
    B.tsm_layernorm_bwd(d, xd, dyd, gd, mean.t, rstd.t, dx.t, dg.t, db.t, scratch(B.tsm_layernorm_workspace_bytes(d)))
    v = dy * g
    m1, m2 = v.mean(), (v * xhat).mean()
    rdx = rrstd * (v - m1 - xhat * m2)
    e1 = (n + 2) * U * np.abs(v).mean()
    e2 = (n + 4) * U * np.abs(v * xhat).mean() + (np.abs(v) * exh).mean()
    size = np.abs(v) + np.abs(v).mean() + np.abs(xhat) * (abs(m2) + e2)
    bound = rrstd * (e1 + np.abs(xhat) * e2 + exh * (abs(m2) + e2) + 8 * U * size) + rel * rrstd * size
    within(dx.np(), rdx, bound + HALF[dtype] * np.abs(rdx), "dx")


@pytest.mark.parametrize("rows,C", [(1 << 26, 8), (90001, 4100)])
def test_weight_gradients_of_very_many_rows(rows, C):
    """One value in all rows, so that every rounding of a long sum leans the same way.  A term of dbeta is among at most 512 additions of its
    thread, 16 of its block, and n / 16 and 16 of the n blocks' sums, of which a block has 512 times 16 or, of rows past the registers, 512
    times 4 rows: as many units of 2^-24.  dgamma's terms are off by a few units more."""
    d = B.LayerNormDesc(rows=rows, C=C, dtype=B.TSM_F32, eps=EPS)
    x = torch.full((rows, C), 0.75, device="cuda")
    dy = torch.full((rows, C), 0.2385874, device="cuda")
    gamma = torch.ones(C, device="cuda")
    mean, rstd = torch.full((rows,), 0.25, device="cuda"), torch.full((rows,), 1.7, device="cuda")
    dx, dg, db = torch.empty_like(x), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    B.tsm_layernorm_bwd(d, x, dy, gamma, mean, rstd, dx, dg, db, scratch(B.tsm_layernorm_workspace_bytes(d)))
    blocks = rows / 512 / (4 if C > 4096 else 16)
    k = 512 + 16 + max(blocks, 512) / 16 + 16
    up = float(dy[0, 0])
    want = rows * up
    within(db.double().cpu().numpy(), np.full(C, want), k * U * want, "dbeta")
    want = rows * up * 0.5 * float(rstd[0])
    within(dg.double().cpu().numpy(), np.full(C, want), (k + 8) * U * want, "dgamma")
