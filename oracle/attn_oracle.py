"""Leaky attention and block norms in float64, from their definitions (test
infrastructure only).

Attention, token by token for each sequence b and query head h, with
hk = h // (H / Hk):
    S_t = beta_h S_{t-1} + k_t v_t^T,    o_t = scale S_t^T q_t
Alongside every result comes the same sum with all its terms made positive
("size"), the scale that rounding errors of the terms are measured on.
"""
import numpy as np


def _positive(x):
    return np.abs(np.asarray(x, np.float64))


def _expand(x, G):
    return np.repeat(np.asarray(x, np.float64), G, axis=2)


def attn_forward(q, k, v, beta, scale=1.0, lens=None, state=None):
    """q [B,T,H,Dk], k [B,T,Hk,Dk], v [B,T,Hk,Dv] -> o [B,T,H,Dv], S [B,H,Dk,Dv]."""
    q = np.asarray(q, np.float64)
    B, T, H, Dk = q.shape
    G = H // k.shape[2]
    k, v = _expand(k, G), _expand(v, G)
    lens = [T] * B if lens is None else lens
    S = np.zeros((B, H, Dk, v.shape[-1])) if state is None else np.array(state, np.float64)
    o = np.zeros((B, T, H, v.shape[-1]))
    bt = np.asarray(beta, np.float64)[:, None, None]
    for b in range(B):
        for t in range(lens[b]):
            S[b] = bt * S[b] + k[b, t][:, :, None] * v[b, t][:, None, :]
            o[b, t] = scale * np.einsum("hd,hde->he", q[b, t], S[b])
    return o, S


def attn_forward_size(q, k, v, beta, scale=1.0, lens=None, state=None):
    return attn_forward(_positive(q), _positive(k), _positive(v), beta, abs(scale), lens,
                        None if state is None else _positive(state))


def attn_backward(q, k, v, beta, do, scale=1.0, lens=None, state=None, dstate=None):
    """Gradients (dq, dk, dv, dS_in) of <o, do> + <S_out, dstate>."""
    q, do = np.asarray(q, np.float64), np.asarray(do, np.float64)
    B, T, H, Dk = q.shape
    Hk = k.shape[2]
    G = H // Hk
    k, v = _expand(k, G), _expand(v, G)
    Dv = v.shape[-1]
    lens = [T] * B if lens is None else lens
    bt = np.asarray(beta, np.float64)[:, None, None]
    S = np.zeros((B, H, Dk, Dv)) if state is None else np.array(state, np.float64)
    R = np.zeros((B, H, Dk, Dv)) if dstate is None else np.array(dstate, np.float64)
    dq, dk, dv = np.zeros_like(q), np.zeros(k.shape), np.zeros(v.shape)
    for b in range(B):
        for t in range(lens[b]):
            S[b] = bt * S[b] + k[b, t][:, :, None] * v[b, t][:, None, :]
            dq[b, t] = scale * np.einsum("hde,he->hd", S[b], do[b, t])
        for t in range(lens[b] - 1, -1, -1):
            # R: gradient of S_t, through o_t and through S_{t+1}
            R[b] = R[b] + scale * q[b, t][:, :, None] * do[b, t][:, None, :]
            dk[b, t] = np.einsum("hde,he->hd", R[b], v[b, t])
            dv[b, t] = np.einsum("hde,hd->he", R[b], k[b, t])
            R[b] = bt * R[b]
    shared = lambda x: x.reshape(B, T, Hk, G, -1).sum(3)
    return dq, shared(dk), shared(dv), R


def attn_backward_size(q, k, v, beta, do, scale=1.0, lens=None, state=None, dstate=None):
    p = _positive
    return attn_backward(p(q), p(k), p(v), beta, p(do), abs(scale), lens,
                         None if state is None else p(state),
                         None if dstate is None else p(dstate))


def _act(z, gate):
    """act(z) and its slope."""
    if gate == "none":
        return 1.0, 0.0
    sg = 1.0 / (1.0 + np.exp(-z))
    if gate == "sigmoid":
        return sg, sg * (1 - sg)
    return z * sg, sg + z * sg * (1 - sg)


def _factor(x, group, eps):
    """1/rms of each group, spread over its channels."""
    M, N = x.shape
    g = x.reshape(M, N // group, group)
    f = 1.0 / np.sqrt((g * g).mean(-1, keepdims=True) + eps)
    return np.broadcast_to(f, g.shape).reshape(M, N)


def _mean(x, group):
    M, N = x.shape
    g = x.reshape(M, N // group, group)
    return np.broadcast_to(g.mean(-1, keepdims=True), g.shape).reshape(M, N)


def block_norm_forward(r, a, z, w_post, res_scale, w_pre, eps, group=0, gate="none"):
    """(r', y); a None: (r, y)."""
    r2 = np.asarray(r, np.float64)
    N = r2.shape[1]
    if a is not None:
        n = a * _factor(a, group or N, eps) * (1.0 if w_post is None else w_post)
        r2 = r2 + (1.0 if res_scale is None else res_scale) * n * _act(z, gate)[0]
    y = None if w_pre is None else r2 * _factor(r2, N, eps) * w_pre
    return r2, y


def block_norm_backward(r2, a, z, w_post, res_scale, w_pre, gro, gy, eps, group=0, gate="none"):
    """dict of gradients from the stored r'."""
    N = r2.shape[1]
    d = np.zeros(r2.shape) if gro is None else np.array(gro, np.float64)
    out = {}
    if gy is not None:
        f = _factor(r2, N, eps)
        e = r2 * f
        g = gy * w_pre
        d = d + f * (g - e * _mean(g * e, N))
        out["grad_w_pre"] = (gy * e).sum(0)
    out["grad_r"] = d
    if a is not None:
        group = group or N
        wp = np.ones(N) if w_post is None else w_post
        sc = np.ones(N) if res_scale is None else res_scale
        f = _factor(a, group, eps)
        h = a * f
        act, slope = _act(z, gate)
        out["grad_scale"] = (d * h * wp * act).sum(0)
        out["grad_w_post"] = (d * sc * act * h).sum(0)
        if z is not None:
            out["grad_z"] = d * sc * h * wp * slope
        m = d * sc * act * wp
        out["grad_a"] = f * (m - h * _mean(m * h, group))
    return out
