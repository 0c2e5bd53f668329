"""PyTorch autograd over the C ABI: a scan layer usable inside an ordinary
torch training graph (as snnTorch's neurons are), with the forward and BPTT
running in libsnn's kernels.

``LeakyScan.apply(I, beta, thr, workload)`` returns the spike tensor
[T, B, N]; its backward returns dL/dI and the beta / threshold gradients
(reduced to their layouts).  The Synaptic and recurrent neurons take alpha
or v as a fourth tensor and return its gradient as well.  Only the spike
output is differentiable; the membrane trace is not returned.

``leaky_attention`` and ``block_norm`` wrap the two operators of a residual
block of a sequence network in the same way, ``selective_scan``,
``causal_conv`` and ``layer_norm`` those of a block whose leak follows its
input; their gradients have none of their own (asked for, they raise).
"""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import snn
from . import workloads as W


class _ScanFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, I, beta, thr, third, w: W.ScanWorkload):
        layer = snn.ScanLayer(w, device=I.device, want_syn=w.neuron == "synaptic")
        I = I.contiguous()
        kw = {}
        if w.neuron == "synaptic":
            kw["alpha"] = third
        elif w.neuron == "rleaky":
            kw["v"] = third
        layer.forward(I, beta, thr, **kw)
        ctx.layer, ctx.kw = layer, kw
        ctx.save_for_backward(I, beta, thr)
        return layer.spk.clone()

    @staticmethod
    def backward(ctx, grad_spk):
        I, beta, thr = ctx.saved_tensors
        layer = ctx.layer
        g = grad_spk.to(layer.spk.dtype).contiguous()
        layer.backward(I, beta, thr, g, want_state_grads=False, **ctx.kw)
        third = None
        if layer.synaptic:
            third = layer.grad_alpha.clone()
        elif layer.recurrent:
            third = layer.grad_v.clone()
        return layer.grad_I.clone(), layer.grad_beta.clone(), layer.grad_thr.clone(), third, None


def scan(I, beta, thr, w: W.ScanWorkload, third=None):
    """Spikes of a scan layer described by ``w`` (its shape, dtypes, reset,
    surrogate, parameter layouts and save variant); differentiable in I,
    beta, thr and the third parameter (alpha or v)."""
    if (w.T, w.B, w.N) != tuple(I.shape):
        raise ValueError("scan: I does not have the workload's [T, B, N] shape")
    return _ScanFunction.apply(I, beta, thr, third, w)


def _starts(t):
    """Whether t starts on the 16-byte boundary that the library wants."""
    return t.data_ptr() % 16 == 0


def _copied(t):
    """A contiguous copy, on a boundary of its own."""
    return torch.empty(t.shape, dtype=t.dtype, device=t.device).copy_(t)


def _whole(t):
    """t contiguous and on a boundary (or None)."""
    return t if t is None or (t.is_contiguous() and _starts(t)) else _copied(t)


def _tokens(t):
    """A [B, T, heads, D] tensor as the library reads it in place, or a copy: D
    contiguous, the other steps positive multiples of 8."""
    n, st = t.shape, t.stride()
    ok = _starts(t) and (n[3] == 1 or st[3] == 1) and all(
        n[i] <= 1 or (st[i] > 0 and st[i] % 8 == 0) for i in range(3))
    return t if ok else _copied(t)


def _matrix(t, N, group, dtype=None):
    """t as rows of N, as the library reads them in place, or a copy (or None);
    with groups the rows have to be whole vectors apart."""
    if t is None:
        return None
    t = (t if dtype is None else t.to(dtype)).reshape(-1, N)
    step = t.stride(0)
    ok = _starts(t) and (N == 1 or t.stride(1) == 1) and (
        t.shape[0] <= 1 or (step >= N and (step % 8 == 0 or group in (0, N))))
    return t if ok else _copied(t)


def _attention_workspace(q, *shape, backward=False):
    """A call's workspace: zero where its status word is, the rest is written
    before it is read."""
    ws = torch.empty(snn.snn_leaky_attn_workspace_bytes(*shape, backward=backward), dtype=torch.uint8,
                     device=q.device)
    ws[:256].zero_()
    return ws


def _keep_status(status, ws):
    """What a call left in its workspace's status word, into the caller's."""
    if status is not None:
        torch.maximum(status, ws[:4].view(torch.int32), out=status)


class _AttentionFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, beta, state, scale, seq_lens, status):
        q, k, v = _tokens(q), _tokens(k), _tokens(v)
        beta, state, seq_lens = _whole(beta), _whole(state), _whole(seq_lens)
        B, T, H, Dk = q.shape
        Hk, Dv = k.shape[2], v.shape[-1]
        o = torch.empty((B, T, H, Dv), dtype=q.dtype, device=q.device)
        end = torch.empty((B, H, Dk, Dv), dtype=torch.float32, device=q.device)
        ws = _attention_workspace(q, B, T, H, Hk, Dk, Dv)
        snn.snn_leaky_attn_fwd(q, k, v, beta, o, ws, scale=scale, seq_lens=seq_lens,
                               state_in=state, state_out=end)
        ctx.save_for_backward(q, k, v, beta, state, seq_lens)
        _keep_status(status, ws)
        ctx.scale, ctx.status = scale, status
        ctx.set_materialize_grads(False)
        return o, end

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_o, grad_end):
        q, k, v, beta, state, seq_lens = ctx.saved_tensors
        B, T, H, Dk = q.shape
        Hk, Dv = k.shape[2], v.shape[-1]
        gq, gk, gv = (torch.empty(x.shape, dtype=q.dtype, device=q.device) for x in (q, k, v))
        gs = torch.empty((B, H, Dk, Dv), dtype=torch.float32, device=q.device) \
            if state is not None and ctx.needs_input_grad[4] else None
        ws = _attention_workspace(q, B, T, H, Hk, Dk, Dv, backward=True)
        grad_o = torch.zeros((B, T, H, Dv), dtype=q.dtype, device=q.device) if grad_o is None \
            else _tokens(grad_o.to(q.dtype))
        snn.snn_leaky_attn_bwd(q, k, v, beta, grad_o, gq, gk, gv, ws, scale=ctx.scale,
                               seq_lens=seq_lens, state_in=state,
                               grad_state_out=_whole(grad_end),
                               grad_state_in=gs)
        _keep_status(ctx.status, ws)
        return gq, gk, gv, None, gs, None, None, None


def leaky_attention(q, k, v, beta, state=None, scale=1.0, seq_lens=None, status=None):
    """(o, state after the last token) of leaky attention, S_t = beta_h S_{t-1}
    + k_t v_t^T and o_t = scale S_t^T q_t: q [B, T, H, Dk], k [B, T, Hk, Dk], v
    [B, T, Hk, Dv] (bf16 or fp16), state fp32 [B, H, Dk, Dv] or None.
    Differentiable in q, k, v and state; beta (fp32 [H]) is a fixed schedule
    over the heads, and one that wants a gradient is refused.
    status: an int32 tensor [1] on the same device, 0 before.  A kernel of the
    call or of its backward that gave up on a wait (its results are undefined
    then) leaves SNN_ERR_TIMEOUT there until the caller clears it."""
    if beta.requires_grad and torch.is_grad_enabled():
        raise ValueError("leaky_attention: beta is a fixed schedule and has no gradient")
    if any(t.dim() != 4 for t in (q, k, v)):
        raise ValueError("leaky_attention: q, k and v must be of shape [B, T, heads, D]")
    if status is not None and (status.shape != (1,) or status.dtype != torch.int32):
        raise ValueError("leaky_attention: status must be an int32 tensor of shape [1]")
    return _AttentionFunction.apply(q, k, v, beta, state, float(scale), seq_lens, status)


class _BlockNormFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, r, a, z, w_post, res_scale, w_pre, eps, group, gate):
        shape = r.shape
        r2, a2, z2 = (_matrix(t, shape[-1], group) for t in (r, a, z))
        w_post, res_scale, w_pre = _whole(w_post), _whole(res_scale), _whole(w_pre)
        r_out = torch.empty(r2.shape, dtype=r.dtype, device=r.device)
        y = torch.empty(r2.shape, dtype=a.dtype, device=a.device) if w_pre is not None else None
        snn.snn_block_norm_fwd(r2, a2, z2, w_post, res_scale, w_pre, r_out, y, eps=eps, group=group,
                               gate=gate)
        ctx.save_for_backward(r_out, a2, z2, w_post, res_scale, w_pre)
        ctx.opts, ctx.shape = dict(eps=eps, group=group, gate=gate), shape
        ctx.set_materialize_grads(False)
        return r_out.view(shape), None if y is None else y.view(shape)

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_r, grad_y):
        r_out, a, z, w_post, res_scale, w_pre = ctx.saved_tensors
        M, N = r_out.shape
        group = ctx.opts["group"]
        grad_r, grad_y = _matrix(grad_r, N, group, r_out.dtype), _matrix(grad_y, N, group, a.dtype)
        if grad_r is None and grad_y is None:
            return (None,) * 9
        like = lambda t: None if t is None else torch.empty(t.shape, dtype=t.dtype, device=t.device)
        gr, ga, gz = like(r_out), like(a), like(z)
        gp, gs = like(w_post), like(res_scale)
        gw = like(w_pre)
        ws = torch.empty(snn.snn_block_norm_workspace_bytes(M, N), dtype=torch.uint8, device=a.device)
        snn.snn_block_norm_bwd(r_out, a, z, w_post, res_scale, w_pre, grad_r, grad_y, gr, ga, gz, gp,
                               gs, gw, ws, **ctx.opts)
        shaped = lambda t: None if t is None else t.view(ctx.shape)
        return shaped(gr), shaped(ga), shaped(gz), gp, gs, gw, None, None, None


def block_norm(r, a, z=None, w_post=None, res_scale=None, w_pre=None, eps=1e-6, group=0,
               gate="none"):
    """(r', y): r' = r + res_scale * norm(a) w_post * act(z) and y = norm(r')
    w_pre (None without w_pre) over the last dimension, the norm of a per
    `group` channels.  r, a and z have one shape.  Differentiable in all the
    tensors.  (The norm of r alone, without a block before it:
    snn.snn_block_norm_fwd and snn_block_norm_bwd.)"""
    if a is None:
        raise ValueError("block_norm: needs a; snn.snn_block_norm_fwd takes the norm of r alone")
    if a.shape != r.shape or (z is not None and z.shape != r.shape):
        raise ValueError("block_norm: r, a and z must have one shape")
    return _BlockNormFunction.apply(r, a, z, w_post, res_scale, w_pre, eps, group, gate)


def _channels(t, dtype):
    """A [B, T, C] tensor as the library reads it in place, or a copy (or None):
    C contiguous, the other steps positive."""
    if t is None:
        return None
    t = t.to(dtype)
    n, st = t.shape, t.stride()
    ok = _starts(t) and (n[2] <= 1 or st[2] == 1) and all(n[i] <= 1 or st[i] > 0 for i in range(2))
    return t if ok else _copied(t)


def _grouped(t):
    """A [B, T, G, N] tensor as the library reads it in place, or a copy."""
    n, st = t.shape, t.stride()
    ok = _starts(t) and (n[3] <= 1 or st[3] == 1) and all(n[i] <= 1 or st[i] > 0 for i in range(3))
    return t if ok else _copied(t)


def _like(t):
    return None if t is None else torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _scratch(n, like):
    return torch.empty(n, dtype=torch.uint8, device=like.device)


def _recorded(*tensors):
    """Whether a backward pass may follow (inside a Function's forward torch no longer says)."""
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)


class _SelectiveScanFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, u, delta, A, B, C, D, z, delta_bias, state, softplus, seq_lens, recorded):
        u, delta, z = (_channels(t, u.dtype) for t in (u, delta, z))
        B, C = _grouped(B), _grouped(C)
        A, D, delta_bias, state, seq_lens = map(_whole, (A, D, delta_bias, state, seq_lens))
        shape = (*u.shape, A.shape[1], B.shape[2])
        y = torch.empty(u.shape, dtype=u.dtype, device=u.device)
        end = torch.empty((u.shape[0], *A.shape), dtype=torch.float32, device=u.device)
        ckpt = None
        if recorded:
            ckpt = torch.empty(snn.snn_selective_scan_ckpt_elems(*shape), dtype=torch.float32, device=u.device)
        snn.snn_selective_scan_fwd(u, delta, A, B, C, y,
                                   _scratch(snn.snn_selective_scan_workspace_bytes(*shape), u), D=D, z=z,
                                   delta_bias=delta_bias, softplus=softplus, seq_lens=seq_lens,
                                   state_in=state, state_out=end, ckpt=ckpt)
        ctx.save_for_backward(u, delta, A, B, C, D, z, delta_bias, state, seq_lens, ckpt)
        ctx.softplus = softplus
        ctx.set_materialize_grads(False)
        return y, end

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_y, grad_end):
        u, delta, A, B, C, D, z, delta_bias, state, seq_lens, ckpt = ctx.saved_tensors
        if grad_y is None and grad_end is None:
            return (None,) * 12
        shape = (*u.shape, A.shape[1], B.shape[2])
        grad_y = torch.zeros(u.shape, dtype=u.dtype, device=u.device) if grad_y is None \
            else _channels(grad_y, u.dtype)
        gu, gd, gA, gB, gC, gD, gz, gb = map(_like, (u, delta, A, B, C, D, z, delta_bias))
        gs = _like(state) if state is not None and ctx.needs_input_grad[8] else None
        snn.snn_selective_scan_bwd(u, delta, A, B, C, grad_y, ckpt, gu, gd, gA, gB, gC,
                                   _scratch(snn.snn_selective_scan_workspace_bytes(*shape, backward=True), u),
                                   D=D, z=z, delta_bias=delta_bias, softplus=ctx.softplus, seq_lens=seq_lens,
                                   grad_state_out=_whole(grad_end), grad_D=gD, grad_z=gz,
                                   grad_delta_bias=gb, grad_state_in=gs)
        return gu, gd, gA, gB, gC, gD, gz, gb, gs, None, None, None


def selective_scan(u, delta, A, B, C, D=None, z=None, delta_bias=None, softplus=True, state=None,
                   seq_lens=None):
    """(y, state after the last token) of the selective scan, s = softplus(delta +
    delta_bias), h_t = exp(s A) h_{t-1} + s u B and y = (C h + D u) silu(z): u, delta, z
    [B, T, D] and B, C [B, T, G, N] of one type (fp32, bf16 or fp16), G dividing D; A [D, N],
    D and delta_bias [D] fp32; state fp32 [B, D, N] or None.  Differentiable in all the tensors."""
    if u.dim() != 3 or B.dim() != 4 or C.dim() != 4 or A.dim() != 2:
        raise ValueError("selective_scan: u must be [B, T, D], B and C [B, T, G, N], A [D, N]")
    if any(t is not None and t.dtype != u.dtype for t in (delta, z, B, C)):
        raise ValueError("selective_scan: u, delta, z, B and C must have one type")
    return _SelectiveScanFunction.apply(u, delta, A, B, C, D, z, delta_bias, state, bool(softplus), seq_lens,
                                        _recorded(u, delta, A, B, C, D, z, delta_bias, state))


class _CausalConvFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, bias, state, act, seq_lens):
        x = _channels(x, x.dtype)
        w, bias, state, seq_lens = map(_whole, (w, bias, state, seq_lens))
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        end = torch.empty((x.shape[0], w.shape[1] - 1, x.shape[2]), dtype=x.dtype, device=x.device)
        snn.snn_causal_conv_fwd(x, w, bias, y, act=act, seq_lens=seq_lens, state_in=state, state_out=end)
        ctx.save_for_backward(x, w, bias, state, seq_lens)
        ctx.act = act
        ctx.set_materialize_grads(False)
        return y, end

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_y, grad_end):
        x, w, bias, state, seq_lens = ctx.saved_tensors
        if grad_y is None and grad_end is None:
            return (None,) * 6
        grad_y = torch.zeros(x.shape, dtype=x.dtype, device=x.device) if grad_y is None \
            else _channels(grad_y, x.dtype)
        gx, gw, gb = map(_like, (x, w, bias))
        gs = _like(state) if state is not None and ctx.needs_input_grad[3] else None
        snn.snn_causal_conv_bwd(x, w, bias, grad_y, gx, gw, gb,
                                _scratch(snn.snn_causal_conv_workspace_bytes(*x.shape, w.shape[1]), x),
                                act=ctx.act, seq_lens=seq_lens, state_in=state,
                                grad_state_out=_whole(grad_end), grad_state_in=gs)
        return gx, gw, gb, gs, None, None


def causal_conv(x, w, bias=None, act="silu", state=None, seq_lens=None):
    """(y, the last W - 1 inputs) of the causal convolution of each channel, y_t =
    act(bias + sum_j w[j] x_{t-W+1+j}): x [B, T, C] (fp32, bf16 or fp16), w [C, W] and bias
    [C] fp32, state [B, W-1, C] of x's type or None.  Differentiable in all the tensors."""
    if x.dim() != 3 or w.dim() != 2:
        raise ValueError("causal_conv: x must be [B, T, C] and w [C, W]")
    if state is not None and state.dtype != x.dtype:
        raise ValueError("causal_conv: the state must have x's type")
    return _CausalConvFunction.apply(x, w, bias, state, act, seq_lens)


class _LayerNormFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, b, eps, dtype, recorded):
        shape, N = x.shape, x.shape[-1]
        x2 = _matrix(x, N, 0)
        w, b = _whole(w), _whole(b)
        y = torch.empty(x2.shape, dtype=dtype, device=x.device)
        stats = torch.empty((2, x2.shape[0]), dtype=torch.float32, device=x.device) \
            if recorded else None
        snn.snn_layer_norm_fwd(x2, w, b, y, stats=stats, eps=eps)
        ctx.save_for_backward(x2, w, b, stats)
        ctx.shape, ctx.dtype = shape, dtype
        return y.view(shape)

    @staticmethod
    @once_differentiable
    def backward(ctx, grad_y):
        x, w, b, stats = ctx.saved_tensors
        M, N = x.shape
        gx, gw, gb = map(_like, (x, w, b))
        snn.snn_layer_norm_bwd(x, w, stats, _matrix(grad_y, N, 0, ctx.dtype), gx, gw, gb,
                               _scratch(snn.snn_layer_norm_workspace_bytes(M, N), x))
        return gx.view(ctx.shape), gw, gb, None, None, None


def layer_norm(x, w=None, b=None, eps=1e-5, dtype=None):
    """(x - mean) rsqrt(var + eps) w + b over the last dimension, as `dtype` (x's own, or a
    16-bit type of an fp32 x).  w and b: fp32 or None.  Differentiable in x, w and b."""
    return _LayerNormFunction.apply(x, w, b, float(eps), dtype or x.dtype, _recorded(x, w, b))
