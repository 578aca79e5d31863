"""fp64 numpy definitions of the operators of a temporal head: gated recurrence, layer norm, linear classifier with softmax
cross entropy, each with its gradients written from the formula.  Test infrastructure only."""
import numpy as np


def sigmoid(g):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-np.asarray(g, np.float64)))


def recur_fwd(x, g, h0=None):
    """x, g [N,T,M], h0 [N,M] -> h [N,T,M]."""
    x, a, k = np.asarray(x, np.float64), sigmoid(g), sigmoid(-np.asarray(g, np.float64))
    h = np.zeros_like(x[:, 0]) if h0 is None else np.asarray(h0, np.float64)
    out = np.empty_like(x)
    for t in range(x.shape[1]):
        h = a[:, t] * h + k[:, t] * x[:, t]
        out[:, t] = h
    return out


def recur_bwd(x, g, h0, dy, dh_last=None):
    """-> dx, dg [N,T,M], dh0 [N,M]."""
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    a, k = sigmoid(g), sigmoid(-np.asarray(g, np.float64))
    h = recur_fwd(x, g, h0)
    first = np.zeros_like(x[:, 0]) if h0 is None else np.asarray(h0, np.float64)
    before = np.concatenate([first[:, None], h[:, :-1]], 1)
    e = np.zeros_like(x[:, 0]) if dh_last is None else np.asarray(dh_last, np.float64)
    dx, dg = np.empty_like(x), np.empty_like(x)
    for t in reversed(range(x.shape[1])):
        d = dy[:, t] + e
        e = a[:, t] * d
        dx[:, t] = k[:, t] * d
        dg[:, t] = e * k[:, t] * (before[:, t] - x[:, t])
    return dx, dg, e


def layernorm_fwd(x, gamma, beta, eps):
    """x [rows,C] -> y, mean, rstd."""
    x = np.asarray(x, np.float64)
    mean = x.mean(1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    return (x - mean[:, None]) * rstd[:, None] * gamma + beta, mean, rstd


def layernorm_bwd(x, dy, gamma, eps):
    """-> dx, dgamma, dbeta."""
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    _, mean, rstd = layernorm_fwd(x, gamma, np.zeros_like(np.asarray(gamma, np.float64)), eps)
    xhat = (x - mean[:, None]) * rstd[:, None]
    v = dy * gamma
    dx = rstd[:, None] * (v - v.mean(1, keepdims=True) - xhat * (v * xhat).mean(1, keepdims=True))
    return dx, (dy * xhat).sum(0), dy.sum(0)


def xent_fwd(x, w, bias, labels):
    """x [R,D], w [V,D] -> loss, lse [R]; rows whose label is no class lose nothing."""
    x, w, labels = np.asarray(x, np.float64), np.asarray(w, np.float64), np.asarray(labels)
    s = x @ w.T + (0.0 if bias is None else np.asarray(bias, np.float64))
    top = s.max(1, keepdims=True)
    with np.errstate(divide="ignore", invalid="ignore"):
        lse = np.where(np.isneginf(top[:, 0]), -np.inf, top[:, 0] + np.log(np.exp(s - top).sum(1)))
    valid = (labels >= 0) & (labels < w.shape[0])
    with np.errstate(invalid="ignore"):
        loss = np.where(valid, lse - s[np.arange(len(labels)), np.where(valid, labels, 0)], 0.0)
    return loss, lse


def xent_grad(x, w, bias, labels, dloss):
    """The gradient of the logits, G [R,V]."""
    x, w, labels = np.asarray(x, np.float64), np.asarray(w, np.float64), np.asarray(labels)
    s = x @ w.T + (0.0 if bias is None else np.asarray(bias, np.float64))
    _, lse = xent_fwd(x, w, bias, labels)
    valid = (labels >= 0) & (labels < w.shape[0])
    with np.errstate(invalid="ignore"):
        p = np.exp(s - lse[:, None])
    r = np.nonzero(valid)[0]
    p[r, labels[r]] -= 1.0
    return np.where(valid[:, None], p * np.asarray(dloss, np.float64)[:, None], 0.0)


def xent_bwd(x, w, bias, labels, dloss):
    """-> dx, dw, dbias."""
    g = xent_grad(x, w, bias, labels, dloss)
    used = (g != 0).any(1)[:, None]
    return g @ np.asarray(w, np.float64), g.T @ np.where(used, np.asarray(x, np.float64), 0.0), g.sum(0)
