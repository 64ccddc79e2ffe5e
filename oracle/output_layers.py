"""fp64 CPU oracle of the output layers and the beam search (test infrastructure only).

Written from the formulas of include/stacklstm.h with plain numpy, row by row where that is
the definition; it imports nothing from the product package. Scores of the search are
rounded to fp32 after each operation, as the definition says, so its choices are exact.
"""
from __future__ import annotations

import math

import numpy as np

_erf = np.vectorize(math.erf)
_f64 = lambda a: np.asarray(a, np.float64)


# ------------------------------------------------------------------ layer norm
def norm_forward(x, gamma, beta, eps):
    """y, mean, rstd of the rows of x [R, N]."""
    x = _f64(x)
    mean = x.mean(1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    xh = (x - mean[:, None]) * rstd[:, None]
    return xh * (1.0 if gamma is None else _f64(gamma)) + (0.0 if beta is None else _f64(beta)), mean, rstd


def norm_backward(dy, x, gamma, mean, rstd):
    """dx, dgamma, dbeta."""
    dy, x, mean, rstd = map(_f64, (dy, x, mean, rstd))
    xh = (x - mean[:, None]) * rstd[:, None]
    a = dy * (1.0 if gamma is None else _f64(gamma))
    dx = rstd[:, None] * (a - a.mean(1, keepdims=True) - xh * (a * xh).mean(1, keepdims=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


# ------------------------------------------------------------------ linear layer
ACTS = ("none", "relu", "tanh", "gelu", "silu")


def act(z, name):
    if name == "relu":
        return np.maximum(z, 0.0)
    if name == "tanh":
        return np.tanh(z)
    if name == "gelu":
        return z * 0.5 * (1.0 + _erf(z / math.sqrt(2.0)))
    if name == "silu":
        return z / (1.0 + np.exp(-z))
    return z


def act_grad(z, name):
    if name == "relu":
        return (z > 0).astype(np.float64)
    if name == "tanh":
        return 1.0 - np.tanh(z) ** 2
    if name == "gelu":
        return 0.5 * (1.0 + _erf(z / math.sqrt(2.0))) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        s = 1.0 / (1.0 + np.exp(-z))
        return s + z * s * (1.0 - s)
    return np.ones_like(z)


def linear_forward(x, W, bias, residual, name):
    """y, pre."""
    pre = _f64(x) @ _f64(W).T + (0.0 if bias is None else _f64(bias))
    return act(pre, name) + (0.0 if residual is None else _f64(residual)), pre


def linear_backward(dy, x, W, pre, add, name):
    """dx, dW, dbias, and dz (for error bounds)."""
    dz = _f64(dy) if name == "none" else _f64(dy) * act_grad(_f64(pre), name)
    return dz @ _f64(W) + (0.0 if add is None else _f64(add)), dz.T @ _f64(x), dz.sum(0), dz


# ------------------------------------------------------------------ distillation
def _log_softmax(z):
    m = z.max()
    return z - (m + math.log(np.exp(z - m).sum()))


def distill(logits, t_idx, t_logit, gold, tau, alpha, scale):
    """loss rows [R] and dlogits [R, V]."""
    z = _f64(logits)
    R, V = z.shape
    loss, d = np.zeros(R), np.zeros((R, V))
    for r in range(R):
        if z[r].max() == -math.inf:
            continue
        on = [j for j in range(t_idx.shape[1]) if 0 <= t_idx[r, j] < V and t_logit[r, j] > -math.inf]
        if on and alpha > 0:
            lq = _log_softmax(_f64(t_logit[r, on]) / tau)
            lp = _log_softmax(z[r] / tau)
            for q, j in zip(lq, on):
                if math.exp(q) > 0:
                    loss[r] += alpha * tau * tau * math.exp(q) * (q - lp[t_idx[r, j]])
                d[r, t_idx[r, j]] -= alpha * tau * math.exp(q)
            d[r] += alpha * tau * np.exp(lp)
        if gold is not None and 0 <= gold[r] < V and alpha < 1:
            lp = _log_softmax(z[r])
            loss[r] -= (1 - alpha) * lp[gold[r]]
            d[r] += (1 - alpha) * np.exp(lp)
            d[r, gold[r]] -= 1 - alpha
    return scale * loss, scale * d


# ------------------------------------------------------------------ beam search
def lse(logits):
    z = _f64(logits)
    out = np.full(z.shape[:2], -math.inf)
    for i in np.ndindex(*out.shape):
        m = z[i].max()
        out[i] = m + math.log(np.exp(z[i] - m).sum()) if m > -math.inf else m
    return out


def select(logits, lse, score, done):
    """new_score, parent, token [B, K]."""
    z = np.asarray(logits, np.float32)
    B, K, V = z.shape
    new, parent, token = np.full((B, K), -np.inf, np.float32), np.full((B, K), -1, np.int32), np.full((B, K), -1, np.int32)
    for b in range(B):
        found = []
        for k in range(K):
            if done is not None and done[b, k]:
                found.append((float(score[b, k]), k * V, k, -1))
                continue
            with np.errstate(invalid="ignore"):
                step = z[b, k] - (np.float32(0) if lse is None else np.float32(lse[b, k]))
                c = np.float32(score[b, k]) + step
            found += [(float(c[v]), k * V + v, k, v) for v in range(V)]
        found = [f for f in found if f[0] > -math.inf]  # neither -inf nor NaN
        found.sort(key=lambda f: (-f[0], f[1]))
        for i, (s, _, k, v) in enumerate(found[:K]):
            new[b, i], parent[b, i], token[b, i] = s, k, v
    return new, parent, token


def reorder(parent, p, h, c, h_out, c_out):
    """p_out, h_out, c_out (what is above the top as given), top_h, top_c."""
    B, K = parent.shape
    h_out, c_out, p_out = h_out.copy(), c_out.copy(), np.zeros_like(p)
    top_h, top_c = np.zeros_like(h[0]), np.zeros_like(c[0])
    for n in range(B * K):
        b, k = divmod(n, K)
        src = b * K + (k if parent[b, k] < 0 else parent[b, k])
        p_out[n] = p[src]
        h_out[:p[src] + 1, n], c_out[:p[src] + 1, n] = h[:p[src] + 1, src], c[:p[src] + 1, src]
        top_h[n], top_c[n] = h[p[src], src], c[p[src], src]
    return p_out, h_out, c_out, top_h, top_c


def push(ops, h_new, c_new, p, h, c):
    """p, h, c, top_h, top_c after one step; what cannot be done is a hold."""
    p, h, c = p.copy(), h.copy(), c.copy()
    S, N = h.shape[:2]
    top_h, top_c = np.zeros_like(h[0]), np.zeros_like(c[0])
    for n in range(N):
        op = int(ops[n])
        if op not in (-1, 0, 1) or not 0 <= p[n] + op < S:
            op = 0
        p[n] += op
        if op == 1:
            h[p[n], n], c[p[n], n] = h_new[n], c_new[n]
        top_h[n], top_c[n] = h[p[n], n], c[p[n], n]
    return p, h, c, top_h, top_c
