"""The temporal head's operators together -- layer norm, recurrence over the frames, classifier with its loss -- and what each has
to hold beyond its own arithmetic: capture into a graph, streams, sizes past 32 bits, refusals of the binding."""
import numpy as np
import pytest
import torch

from oracle import head_oracle as H
from paper_1910_00932_amd import binding as B
from head_util import CDT, HALF, TDT, U, Guarded, scratch, values, within

pytestmark = pytest.mark.gpu
EPS = 1e-5


class Head:
    """Frame features [N,T,C] -> layer norm -> gated recurrence (gates given) -> logits of every frame -> loss, and back."""

    def __init__(self, N, T, C, V, dtype, seed=0):
        self.N, self.T, self.C, self.V, self.dtype = N, T, C, V, dtype
        rows, dt = N * T, TDT[dtype]
        self.ln = B.LayerNormDesc(rows=rows, C=C, dtype=CDT[dtype], eps=EPS)
        self.rc = B.RecurDesc(N=N, T=T, C=C, H=1, W=1, dtype=CDT[dtype])
        self.xe = B.XentDesc(rows=rows, features=C, classes=V, dtype=CDT[dtype])
        self.f, self.fn = values((rows, C), seed, dtype, scale=1.5, shift=0.2)
        self.g, self.gn = values((N, T, C), seed + 1, dtype, shift=1.0)
        self.w, self.wn = values((V, C), seed + 2, dtype, scale=2 / np.sqrt(C))
        self.b, self.bn = values((V,), seed + 3, "f32", scale=0.3)
        self.gamma, self.gamman = values((C,), seed + 4, "f32", scale=0.1, shift=1.0)
        self.beta, self.betan = values((C,), seed + 5, "f32", scale=0.1)
        self.h0, self.h0n = values((N, C), seed + 6, "f32")
        lab = np.random.default_rng(seed + 7).integers(0, V, rows).astype(np.int32)
        lab[::7] = -1
        self.lab, self.labn = torch.from_numpy(lab).cuda(), lab
        self.up = torch.where(self.lab >= 0, 1.0 / float((lab >= 0).sum()), 0.0).float()
        e = lambda *s, t=dt: torch.empty(s, dtype=t, device="cuda")  # noqa: E731
        f32 = torch.float32
        self.o = {"z": e(rows, C), "mean": e(rows, t=f32), "rstd": e(rows, t=f32), "y": e(N, T, C), "h_last": e(N, C, t=f32),
                  "loss": e(rows, t=f32), "lse": e(rows, t=f32), "dy": e(N, T, C), "dw": e(V, C), "db": e(V, t=f32), "dz": e(N, T, C),
                  "dg": e(N, T, C), "dh0": e(N, C, t=f32), "df": e(rows, C), "dgamma": e(C, t=f32), "dbeta": e(C, t=f32)}
        self.saved = scratch(B.tsm_recur_saved_bytes(self.rc))
        self.ws = scratch(max(B.tsm_layernorm_workspace_bytes(self.ln), B.tsm_recur_workspace_bytes(self.rc), B.tsm_xent_workspace_bytes(self.xe)))

    def run(self):
        o = self.o
        B.tsm_layernorm_fwd(self.ln, self.f, self.gamma, self.beta, o["z"], o["mean"], o["rstd"])
        B.tsm_recur_fwd(self.rc, o["z"], self.g, self.h0, o["y"], o["h_last"], self.saved, self.ws)
        B.tsm_xent_fwd(self.xe, o["y"], self.w, self.b, self.lab, o["loss"], o["lse"], self.ws)
        B.tsm_xent_bwd(self.xe, o["y"], self.w, self.b, self.lab, o["lse"], self.up, o["dy"], o["dw"], o["db"], self.ws)
        B.tsm_recur_bwd(self.rc, o["z"], self.g, self.h0, self.saved, o["dy"], None, o["dz"], o["dg"], o["dh0"], self.ws)
        B.tsm_layernorm_bwd(self.ln, self.f, o["dz"], self.gamma, o["mean"], o["rstd"], o["df"], o["dgamma"], o["dbeta"], self.ws)

    def bits(self):
        return {k: v.float().cpu().numpy().copy() for k, v in self.o.items()}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_head_forward_and_backward(dtype):
    """The chain in 64 bits, every tensor by its relative 2-norm.  Each of at most six operators rounds its results and what it reads
    once more: six half steps; fp32 sums of up to 1000 terms add 1000 units of 2^-24 at most to each."""
    h = Head(3, 37, 200, 431, dtype)
    h.run()
    torch.cuda.synchronize()
    N, T, C = h.N, h.T, h.C
    z, _, _ = H.layernorm_fwd(h.fn, h.gamman, h.betan, EPS)
    y = H.recur_fwd(z.reshape(N, T, C), h.gn, h.h0n)
    loss, lse = H.xent_fwd(y.reshape(-1, C), h.wn, h.bn, h.labn)
    dy, dw, db = H.xent_bwd(y.reshape(-1, C), h.wn, h.bn, h.labn, h.up.double().cpu().numpy())
    dz, dg, dh0 = H.recur_bwd(z.reshape(N, T, C), h.gn, h.h0n, dy.reshape(N, T, C))
    df, dgamma, dbeta = H.layernorm_bwd(h.fn, dz.reshape(-1, C), h.gamman, EPS)
    want = dict(z=z, y=y, loss=loss, lse=lse, dy=dy, dw=dw, db=db, dz=dz, dg=dg, dh0=dh0, df=df, dgamma=dgamma, dbeta=dbeta, h_last=y[:, -1])
    tol = 6 * HALF[dtype] if dtype == "bf16" else 6 * 1000 * U
    for k, v in want.items():
        got = h.o[k].double().cpu().numpy().ravel()
        rel = np.linalg.norm(got - v.ravel()) / np.linalg.norm(v)
        assert rel < tol, (k, rel, tol)


@pytest.mark.parametrize("shape", [(2, 8, 96, 130), (1, 700, 64, 500)])
def test_head_in_a_graph(shape):
    """Captured once, replayed with new inputs, eager work of the same operators between the replays."""
    h, other = Head(*shape, "bf16"), Head(*shape, "bf16", seed=50)
    h.run()                                        # the first call on a device is outside of capture
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            h.run()
    torch.cuda.current_stream().wait_stream(s)
    for k in range(4):
        new, _ = values((h.N * h.T, h.C), 100 + k, "bf16", scale=1.5)
        h.f.copy_(new)
        for v in h.o.values():
            v.fill_(float("nan"))
        graph.replay()
        other.run()
        torch.cuda.synchronize()
        got = h.bits()
        for v in h.o.values():
            v.fill_(float("nan"))
        h.run()
        torch.cuda.synchronize()
        for key, v in h.bits().items():
            assert np.array_equal(got[key], v), (k, key)


def test_two_streams_at_once():
    a, b = Head(2, 300, 64, 500, "bf16"), Head(2, 300, 64, 500, "bf16", seed=20)
    a.run()
    b.run()
    torch.cuda.synchronize()
    want = a.bits(), b.bits()
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(s):
            a.run()
        with torch.cuda.stream(t):
            b.run()
    torch.cuda.synchronize()
    for head, w in zip((a, b), want):
        for k, v in head.bits().items():
            assert np.array_equal(v, w[k]), k


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,T,M", [(1, 1, 2), (3, 5, 3), (2, 30, 1), (2, 61, 2), (1, 900, 1), (3, 400, 3), (2, 140, 4), (2, 140, 5), (1, 64, 7), (1, 65, 6)])
def test_recurrence_of_few_columns(N, T, M, dtype):
    d = B.RecurDesc(N=N, T=T, C=M, H=1, W=1, dtype=CDT[dtype])
    x, xn = values((N, T, M), 0, dtype)
    g, gn = values((N, T, M), 1, dtype, shift=1.0)
    dy, dyn = values((N, T, M), 2, dtype)
    y, dx, dg = (Guarded((N, T, M), TDT[dtype]) for _ in range(3))
    saved, ws = scratch(B.tsm_recur_saved_bytes(d)), scratch(B.tsm_recur_workspace_bytes(d))
    B.tsm_recur_fwd(d, x, g, None, y.t, None, saved, ws)
    B.tsm_recur_bwd(d, x, g, None, saved, dy, None, dx.t, dg.t, None, ws)
    X = np.abs(xn).max()
    h = H.recur_fwd(xn, gn)
    F = 8 * T * U * X
    within(y.np(), h, F + HALF[dtype] * np.abs(h), "y")
    rdx, rdg, _ = H.recur_bwd(xn, gn, None, dyn)
    D = np.abs(dyn).sum(1).max()
    within(dx.np(), rdx, 8 * T * U * D + HALF[dtype] * np.abs(rdx), "dx")
    within(dg.np(), rdg, (8 * T * U * D * X + D * F + 8 * U * D * X) + HALF[dtype] * np.abs(rdg), "dg")


@pytest.mark.parametrize("dtype,D", [("f32", 24), ("bf16", 9), ("f32", 9)])
def test_classes_in_pieces_as_operands_of_the_workspace(dtype, D):
    """Several pieces where x and w are made into operands piece by piece, in both passes; labels in every piece."""
    R, V = 70000, 3500
    d = B.XentDesc(rows=R, features=D, classes=V, dtype=CDT[dtype])
    x, _ = values((R, D), 0, dtype)
    w, _ = values((V, D), 1, dtype, scale=0.5)
    b, _ = values((V,), 2, "f32")
    lab = torch.arange(R, device="cuda", dtype=torch.int32) % (V + 1)          # V: no class
    up, _ = values((R,), 3, "f32")
    ws = scratch(B.tsm_xent_workspace_bytes(d))
    loss, lse, dx, dw, db = (Guarded(s, t) for s, t in (((R,), torch.float32), ((R,), torch.float32), ((R, D), TDT[dtype]), ((V, D), TDT[dtype]), ((V,), torch.float32)))
    B.tsm_xent_fwd(d, x, w, b, lab, loss.t, lse.t, ws)
    B.tsm_xent_bwd(d, x, w, b, lab, lse.t, up, dx.t, dw.t, db.t, ws)
    s = x.double() @ w.double().t() + b.double()
    rlse = torch.logsumexp(s, 1)
    ok = lab < V
    at = torch.where(ok, lab, torch.zeros_like(lab)).long()
    rows = torch.arange(R, device="cuda")
    rloss = torch.where(ok, rlse - s[rows, at], torch.zeros_like(rlse))
    # logits of magnitude below 30 in fp32: 1e-5 covers 40 roundings of them
    within(lse.np(), rlse.cpu().numpy(), 1e-5, "lse")
    within(loss.np(), rloss.cpu().numpy(), 2e-5, "loss")
    G = s.sub_(rlse[:, None]).exp_()
    G[rows, at] -= 1
    G.mul_(torch.where(ok, up, torch.zeros_like(up)).double()[:, None])
    half, mag = HALF[dtype], G.abs()
    entry = (half if dtype == "bf16" else 0) + 3e-5                            # of an entry of G, relative
    for got, want, size in ((dx, G @ w.double(), mag @ w.double().abs()), (dw, G.t() @ x.double(), mag.t() @ x.double().abs())):
        want, size = want.cpu().numpy(), size.cpu().numpy()
        within(got.np(), want, entry * size + half * np.abs(want) + 1e-30, "gradient")
    within(db.np(), G.sum(0).cpu().numpy(), 5e-5 * mag.sum(0).cpu().numpy() + 1e-30, "dbias")


def test_recurrence_past_32_bits():
    """2.3e9 values: the last clip alone gives the same bits."""
    N, T, M = 3, 1500, 512 * 1024 + 6
    x = torch.randn(N, T, M, device="cuda", dtype=torch.bfloat16)
    g = torch.randn(N, T, M, device="cuda", dtype=torch.bfloat16)
    y = torch.empty_like(x)
    d = B.RecurDesc(N=N, T=T, C=M, H=1, W=1, dtype=B.TSM_BF16)
    saved = torch.empty(B.tsm_recur_saved_bytes(d), dtype=torch.uint8, device="cuda")
    B.tsm_recur_fwd(d, x, g, None, y, None, saved, scratch(B.tsm_recur_workspace_bytes(d)))
    dx, dg = torch.empty_like(x), torch.empty_like(x)
    B.tsm_recur_bwd(d, x, g, None, saved, y, None, dx, dg, None, scratch(B.tsm_recur_workspace_bytes(d)))
    one = B.RecurDesc(N=1, T=T, C=M, H=1, W=1, dtype=B.TSM_BF16)
    y1, dx1, dg1 = (torch.empty(1, T, M, device="cuda", dtype=torch.bfloat16) for _ in range(3))
    s1 = torch.empty(B.tsm_recur_saved_bytes(one), dtype=torch.uint8, device="cuda")
    B.tsm_recur_fwd(one, x[2:].contiguous(), g[2:].contiguous(), None, y1, None, s1, scratch(B.tsm_recur_workspace_bytes(one)))
    B.tsm_recur_bwd(one, x[2:].contiguous(), g[2:].contiguous(), None, s1, y1, None, dx1, dg1, None, scratch(B.tsm_recur_workspace_bytes(one)))
    assert torch.equal(y[2:], y1) and torch.equal(dx[2:], dx1) and torch.equal(dg[2:], dg1)
    k = M - 3                                      # and the definition, at the last columns
    want = H.recur_fwd(x[2:, :, k:].double().cpu().numpy(), g[2:, :, k:].double().cpu().numpy())
    within(y1[:, :, k:].double().cpu().numpy(), want, 8 * T * U * 6 + HALF["bf16"] * np.abs(want), "y")


def test_layernorm_past_32_bits():
    rows, C = 1100003, 2048
    x = torch.randn(rows, C, device="cuda", dtype=torch.bfloat16)
    gamma, beta = torch.randn(C, device="cuda"), torch.randn(C, device="cuda")
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    d = B.LayerNormDesc(rows=rows, C=C, dtype=B.TSM_BF16, eps=EPS)
    B.tsm_layernorm_fwd(d, x, gamma, beta, y, mean, rstd)
    dx, dg, db = torch.empty_like(x), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    B.tsm_layernorm_bwd(d, x, y, gamma, mean, rstd, dx, dg, db, scratch(B.tsm_layernorm_workspace_bytes(d)))
    e = B.LayerNormDesc(rows=100, C=C, dtype=B.TSM_BF16, eps=EPS)
    tail = x[-100:].contiguous()
    y1, m1, r1, dx1, dg1, db1 = torch.empty_like(tail), torch.empty(100, device="cuda"), torch.empty(100, device="cuda"), torch.empty_like(tail), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    B.tsm_layernorm_fwd(e, tail, gamma, beta, y1, m1, r1)
    B.tsm_layernorm_bwd(e, tail, y1, gamma, m1, r1, dx1, dg1, db1, scratch(B.tsm_layernorm_workspace_bytes(e)))
    assert torch.equal(y[-100:], y1) and torch.equal(mean[-100:], m1) and torch.equal(dx[-100:], dx1)
    # sums over a million rows: chains of at most rows / 512 / 4 + 64 additions of a block, then 512 blocks'
    want = torch.zeros(C, dtype=torch.float64, device="cuda")
    size = torch.zeros(C, dtype=torch.float64, device="cuda")
    for part in y.split(100000):
        want += part.double().sum(0)
        size += part.double().abs().sum(0)
    within(db.double().cpu().numpy(), want.cpu().numpy(), (rows / 2048 + 128) * U * size.cpu().numpy(), "dbeta")


def test_cross_entropy_past_32_bits():
    """Weights of 2.25e9 values, labels among the last classes."""
    R, D, V = 8, 2048, 1100003
    x = torch.randn(R, D, device="cuda", dtype=torch.bfloat16)
    w = torch.empty(V, D, device="cuda", dtype=torch.bfloat16)
    for part in w.split(100000):
        part.copy_(torch.randn(part.shape, device="cuda") * (2 / D ** 0.5))
    lab = torch.tensor([V - 1, V - 2, 0, 5, V - 300, V, 1048576, -1], dtype=torch.int32, device="cuda")
    up = torch.full((R,), 0.125, device="cuda")
    d = B.XentDesc(rows=R, features=D, classes=V, dtype=B.TSM_BF16)
    ws = torch.empty(B.tsm_xent_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    loss, lse = torch.empty(R, device="cuda"), torch.empty(R, device="cuda")
    B.tsm_xent_fwd(d, x, w, None, lab, loss, lse, ws)
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    B.tsm_xent_bwd(d, x, w, None, lab, lse, up, dx, dw, None, ws)
    s = torch.cat([x.double() @ p.double().t() for p in w.split(100000)], 1)
    rlse = torch.logsumexp(s, 1)
    within(lse.double().cpu().numpy(), rlse.cpu().numpy(), 2e-5, "lse")
    ok = (lab >= 0) & (lab < V)
    at = torch.where(ok, lab, torch.zeros_like(lab)).long()
    rows = torch.arange(R, device="cuda")
    within(loss.double().cpu().numpy(), torch.where(ok, rlse - s[rows, at], torch.zeros_like(rlse)).cpu().numpy(), 4e-5, "loss")
    G = (s - rlse[:, None]).exp_()
    G[rows, at] -= 1
    G *= torch.where(ok, up, torch.zeros_like(up)).double()[:, None]
    want = sum(g @ p.double() for g, p in zip(G.split(100000, 1), w.split(100000)))
    size = sum(g.abs() @ p.double().abs() for g, p in zip(G.split(100000, 1), w.split(100000)))
    half = HALF["bf16"]
    within(dx.double().cpu().numpy(), want.cpu().numpy(), ((half + 1e-4) * size + half * want.abs()).cpu().numpy(), "dx")
    for a, b in ((0, 300), (1048500, 1048700), (V - 500, V)):
        want, size = G[:, a:b].t() @ x.double(), G[:, a:b].abs().t() @ x.double().abs()
        within(dw[a:b].double().cpu().numpy(), want.cpu().numpy(), ((half + 1e-4) * size + half * want.abs()).cpu().numpy(), "dw %d" % a)


def test_layernorm_gradient_is_that_of_its_own_forward():
    """Central differences of the library's forward pass in fp32 along one direction: the rounding of a sum of 19200 products of
    order 1 is some 1e-5 of it, over 2e-2, and the third-order term 1e-4 of the slope's scale."""
    rows, C = 60, 320
    d = B.LayerNormDesc(rows=rows, C=C, dtype=B.TSM_F32, eps=EPS)
    x, _ = values((rows, C), 0, "f32", scale=1.5, shift=0.5)
    gamma, _ = values((C,), 1, "f32", shift=1.0)
    beta, _ = values((C,), 2, "f32")
    dy, _ = values((rows, C), 3, "f32")
    dirs = [values(t.shape, 10 + i, "f32")[0] for i, t in enumerate((x, gamma, beta))]
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")

    def loss(x, gamma, beta):
        y = torch.empty_like(x)
        B.tsm_layernorm_fwd(d, x, gamma, beta, y, mean, rstd)
        return float((y.double() * dy.double()).sum())
    h = 1e-2
    slope = (loss(*[t + h * u for t, u in zip((x, gamma, beta), dirs)]) - loss(*[t - h * u for t, u in zip((x, gamma, beta), dirs)])) / (2 * h)
    loss(x, gamma, beta)
    grads = [torch.empty_like(t) for t in (x, gamma, beta)]
    B.tsm_layernorm_bwd(d, x, dy, gamma, mean, rstd, *grads, scratch(B.tsm_layernorm_workspace_bytes(d)))
    want = sum(float((g.double() * u.double()).sum()) for g, u in zip(grads, dirs))
    scale = float(np.sqrt(sum((g.double() ** 2).sum().item() for g in grads)))
    assert abs(slope - want) < 1e-2 * scale, (slope, want, scale)


def test_binding_refuses_other_sizes_types_and_devices(monkeypatch):
    h = Head(2, 200, 64, 100, "bf16")
    o = h.o
    with pytest.raises(ValueError, match="x: expected"):
        B.tsm_recur_fwd(h.rc, o["z"][:-1], h.g, None, o["y"], None, None, h.ws)
    with pytest.raises(ValueError, match="y: expected"):
        B.tsm_recur_fwd(h.rc, o["z"], h.g, None, o["y"].float(), None, None, h.ws)
    with pytest.raises(ValueError, match="saved"):
        B.tsm_recur_fwd(h.rc, o["z"], h.g, None, o["y"], None, h.saved[:-4], h.ws)
    with pytest.raises(ValueError, match="mean"):
        B.tsm_layernorm_fwd(h.ln, h.f, h.gamma, h.beta, o["z"], o["mean"][:100], None)
    with pytest.raises(ValueError, match="labels: expected"):
        B.tsm_xent_fwd(h.xe, o["y"], h.w, h.b, h.lab.long(), o["loss"], o["lse"], h.ws)
    with pytest.raises(ValueError, match="contiguous"):
        B.tsm_xent_fwd(h.xe, o["y"], h.w.t(), h.b, h.lab, o["loss"], o["lse"], h.ws)
    with pytest.raises(B.TsmError):
        B.tsm_xent_fwd(h.xe, o["y"], h.w, h.b, h.lab, o["loss"], o["lse"], None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError, match="current device"):
        B.tsm_layernorm_fwd(h.ln, h.f, h.gamma, h.beta, o["z"], None, None, stream=0)


def test_layernorm_weight_gradients_of_very_long_rows():
    """2 x 2^27 sums of partial rows, as many threads as no launch has.  Bounds: dgamma and dbeta are sums of 33 terms, of which dgamma's are
    off by 4 units; dx as in the layer norm's own tests, with chains of 400 additions."""
    rows, C = 33, 1 << 27
    x, dy = (torch.randn(rows, C, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    gamma = torch.randn(C, device="cuda")
    mean, rstd = torch.linspace(-0.5, 0.5, rows, device="cuda"), torch.linspace(0.5, 2.0, rows, device="cuda")
    dx, dg, db = torch.empty_like(x), torch.full((C,), float("nan"), device="cuda"), torch.full((C,), float("nan"), device="cuda")
    d = B.LayerNormDesc(rows=rows, C=C, dtype=B.TSM_BF16, eps=EPS)
    B.tsm_layernorm_bwd(d, x, dy, gamma, mean, rstd, dx, dg, db, scratch(B.tsm_layernorm_workspace_bytes(d)))
    s1, s2, a1, a2 = (torch.zeros(rows, dtype=torch.float64, device="cuda") for _ in range(4))
    m, r = mean.double()[:, None], rstd.double()[:, None]
    step = 1 << 23
    for c in range(0, C, step):
        up = dy[:, c:c + step].double()
        xhat = (x[:, c:c + step].double() - m) * r
        prod, v = up * xhat, up * gamma[c:c + step].double()
        assert bool(((dg[c:c + step].double() - prod.sum(0)).abs() <= 68 * U * prod.abs().sum(0)).all()), c
        assert bool(((db[c:c + step].double() - up.sum(0)).abs() <= 64 * U * up.abs().sum(0)).all()), c
        s1 += v.sum(1)
        s2 += (v * xhat).sum(1)
        a1 += v.abs().sum(1)
        a2 += (v * xhat).abs().sum(1)
    s1, s2, a1, a2 = s1[:, None] / C, s2[:, None] / C, a1[:, None] / C, a2[:, None] / C
    for c in (0, C // 2, C - 5000):
        v = dy[:, c:c + 5000].double() * gamma[c:c + 5000].double()
        xhat = (x[:, c:c + 5000].double() - m) * r
        want = r * (v - s1 - xhat * s2)
        bound = r * (402 * U * a1 + xhat.abs() * 408 * U * a2 + 8 * U * (v.abs() + a1 + xhat.abs() * a2))
        within(dx[:, c:c + 5000].double().cpu().numpy(), want.cpu().numpy(), (bound + HALF["bf16"] * want.abs()).cpu().numpy(), "dx %d" % c)
