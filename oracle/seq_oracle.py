"""Selective scan, causal convolution and layer norm in float64, from their
definitions (test infrastructure only).  Beside a result comes the same sum with all
its terms made positive ("size"), the scale that rounding errors of the terms are
measured on.
"""
import numpy as np


def _f(x):
    return None if x is None else np.asarray(x, np.float64)


def _p(x):
    return None if x is None else np.abs(np.asarray(x, np.float64))


def sigmoid(x):
    e = np.exp(-np.abs(x))
    return np.where(x >= 0, 1.0, e) / (1.0 + e)


def step_sizes(delta, bias, softplus):
    raw = _f(delta) + (0.0 if bias is None else _f(bias))
    return (np.logaddexp(raw, 0.0) if softplus else raw), raw


def _gate(z):
    """silu and its slope."""
    if z is None:
        return 1.0, None
    s = sigmoid(_f(z))
    return _f(z) * s, s + _f(z) * s * (1.0 - s)


def _spread(x, D):
    return np.repeat(x, D // x.shape[-2], axis=-2)


def scan_forward(u, delta, A, B, C, D=None, z=None, bias=None, softplus=True, lens=None, state=None,
                 positive=False):
    """u, delta, z [B,T,D], B, C [B,T,G,N] -> y [B,T,D], h [B,D,N].  positive: the
    results' sizes."""
    s, _ = step_sizes(delta, bias, softplus)
    gate, _ = _gate(z)
    k = _p if positive else _f
    u, B, C, A = k(u), k(B), k(C), _f(A)
    if positive:
        gate = np.abs(gate)
    nB, T, nD = u.shape
    lens = [T] * nB if lens is None else lens
    h = np.zeros((nB, nD, A.shape[1])) if state is None else k(state).copy()
    y = np.zeros_like(u)
    skip = 0.0 if D is None else k(D)
    x = (np.abs(s) if positive else s) * u
    for b in range(nB):
        for t in range(min(max(lens[b], 0), T)):
            h[b] = np.exp(s[b, t][:, None] * A) * h[b] + x[b, t][:, None] * _spread(B[b, t], nD)
            y[b, t] = (h[b] * _spread(C[b, t], nD)).sum(-1) + skip * u[b, t]
    return y * gate, h


def scan_backward(u, delta, A, B, C, gy, D=None, z=None, bias=None, softplus=True, lens=None, state=None,
                  gstate=None, positive=False):
    """Gradients of <y, gy> + <h, gstate> as a dict ("s": that of the step, before softplus)."""
    s, raw = step_sizes(delta, bias, softplus)
    gate, slope = _gate(z)
    k = _p if positive else _f
    u, B, C, gy, A = k(u), k(B), k(C), k(gy), _f(A)
    A_size = np.abs(A) if positive else A
    s_size = np.abs(s) if positive else s
    if positive:
        gate = np.abs(gate)
        slope = None if slope is None else 1.1 * np.ones_like(slope)   # |silu'| < 1.1; its terms too
    nB, T, nD = u.shape
    G = B.shape[2]
    lens = [T] * nB if lens is None else lens
    skip = np.zeros(nD) if D is None else k(D)
    o = {"u": np.zeros_like(u), "delta": np.zeros_like(u), "A": np.zeros_like(A), "B": np.zeros_like(B),
         "C": np.zeros_like(C), "D": np.zeros(nD), "z": np.zeros_like(u),
         "state": np.zeros((nB, nD, A.shape[1]))}
    sums = lambda v: v.reshape(G, nD // G, -1).sum(1)
    for b in range(nB):
        n = min(max(lens[b], 0), T)
        h = [np.zeros(A.shape) if state is None else k(state)[b]]
        for t in range(n):
            h.append(np.exp(s[b, t][:, None] * A) * h[-1] + (s_size[b, t] * u[b, t])[:, None] * _spread(B[b, t], nD))
        g = np.zeros(A.shape) if gstate is None else k(gstate)[b].copy()
        for t in range(n - 1, -1, -1):
            Bt, Ct, ut, st = _spread(B[b, t], nD), _spread(C[b, t], nD), u[b, t], s_size[b, t]
            ga = gate if np.isscalar(gate) else gate[b, t]
            dy = gy[b, t] * ga
            if z is not None:
                o["z"][b, t] = gy[b, t] * ((h[t + 1] * Ct).sum(-1) + skip * ut) * slope[b, t]
            o["D"] += dy * ut
            o["C"][b, t] = sums(dy[:, None] * h[t + 1])
            g = g + dy[:, None] * Ct
            o["B"][b, t] = sums(g * (st * ut)[:, None])
            w = (g * Bt).sum(-1)
            g = np.exp(s[b, t][:, None] * A) * g
            q = g * h[t]
            o["A"] += q * st[:, None]
            o["u"][b, t] = st * w + skip * dy
            o["delta"][b, t] = ut * w + (q * A_size).sum(-1)
        o["state"][b] = g
    o["s"] = o["delta"].copy()
    if softplus:
        o["delta"] *= sigmoid(raw)
    o["bias"] = o["delta"].sum((0, 1))
    return o


def conv_forward(x, w, bias=None, act="none", lens=None, state=None, positive=False):
    """x [B,T,C], w [C,W] -> y, the last W - 1 inputs; positive: the size of the
    pre-activation (times 1.1, the activation's steepest)."""
    x, w = _f(x), _f(w)
    nB, T, C = x.shape
    W = w.shape[1]
    lens = [T] * nB if lens is None else lens
    y, end = np.zeros_like(x), np.zeros((nB, W - 1, C))
    k = np.abs if positive else (lambda v: v)
    for b in range(nB):
        n = min(max(lens[b], 0), T)
        before = np.zeros((W - 1, C)) if state is None else _f(state)[b]
        rows = np.concatenate([before, x[b, :n]])
        end[b] = rows[n:]
        p = sum(k(w[:, j]) * k(rows[j:j + n]) for j in range(W)) + (0.0 if bias is None else k(_f(bias)))
        y[b, :n] = 1.1 * p if positive else p * sigmoid(p) if act == "silu" else p
    return y, end


def conv_backward(x, w, gy, bias=None, act="none", lens=None, state=None, gstate=None, positive=False):
    """Gradients of <y, gy> + <end, gstate>: x, w, bias, state."""
    x, w, gy = _f(x), _f(w), _f(gy)
    nB, T, C = x.shape
    W = w.shape[1]
    lens = [T] * nB if lens is None else lens
    o = {"x": np.zeros_like(x), "w": np.zeros_like(w), "bias": np.zeros(C), "state": np.zeros((nB, W - 1, C))}
    k = np.abs if positive else (lambda v: v)
    for b in range(nB):
        n = min(max(lens[b], 0), T)
        rows = np.concatenate([np.zeros((W - 1, C)) if state is None else _f(state)[b], x[b, :n]])
        p = sum(w[:, j] * rows[j:j + n] for j in range(W)) + (0.0 if bias is None else _f(bias))
        if act == "silu":
            s = sigmoid(p)
            slope = s + p * s * (1.0 - s)
            if positive:   # its terms, and what the pre-activation's rounding does to it (|silu''| <= 1/2)
                size = sum(np.abs(w[:, j] * rows[j:j + n]) for j in range(W)) + np.abs(0.0 if bias is None else _f(bias))
                slope = 1.1 + 0.5 * size
            d = k(gy[b, :n]) * slope
        else:
            d = k(gy[b, :n])
        g = np.zeros_like(rows)
        if gstate is not None:
            g[n:] += k(_f(gstate)[b])
        for j in range(W):
            g[j:j + n] += k(w[:, j]) * d
            o["w"][:, j] += (d * k(rows[j:j + n])).sum(0)
        o["bias"] += d.sum(0)
        o["state"][b], o["x"][b, :n] = g[:W - 1], g[W - 1:]
    return o


def layer_norm_forward(x, w=None, b=None, eps=1e-5):
    x = _f(x)
    e = x - x.mean(-1, keepdims=True)
    r = 1.0 / np.sqrt((e * e).mean(-1, keepdims=True) + eps)
    return e * r * (1.0 if w is None else _f(w)) + (0.0 if b is None else _f(b))


def layer_norm_backward(x, w, gy, eps=1e-5, positive=False):
    x, gy = _f(x), _f(gy)
    e = x - x.mean(-1, keepdims=True)
    r = 1.0 / np.sqrt((e * e).mean(-1, keepdims=True) + eps)
    e = e * r
    k = np.abs if positive else (lambda v: v)
    minus = 1.0 if positive else -1.0
    g = k(gy) * (1.0 if w is None else k(_f(w)))
    e, mean = k(e), lambda v: v.mean(-1, keepdims=True)
    return {"x": r * (g + minus * mean(g) + minus * e * mean(g * e)), "w": (k(gy) * e).sum(0), "b": k(gy).sum(0)}
