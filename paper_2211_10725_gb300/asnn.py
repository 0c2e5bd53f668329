"""A sequence network of leaky-attention blocks on spikes, as one training
step through the C ABI and as a stream of single steps.

The residual stream r [T*B, width] is fp32 and starts as the input current of
all T*B rows (one GEMM).  Per block:

  y    = norm(r) w_pre                                  (block norm)
  I    = W y, one tensor-core GEMM for queries, keys, values and the gate
  Leaky scan of I (Eqs. 3-4): the spikes of the first neurons are the
         queries, keys and values, the membrane potential of the others the gate
  o    = leaky attention of the spikes, read in place ([T, B, ...] strides)
  r'   = r + scale * norm_per_head(o) w_post * silu(gate)   (block norm, which
         also gives the next block's y)

The last y feeds a dense Leaky readout and the rate-coded cross-entropy.  The
reverse pass runs the same chain backwards: the scans' BPTT takes the
attention's gradients as spike gradients and the gate's as gradients of the
membrane trace.  AdamW updates the weights and the norms' parameters; the heads'
decays are a fixed schedule.

Everything but one cast (the fp32 gradient of the input current to bf16 for its
weight gradient) is a library call.  Shapes: T*B a multiple of 8.
"""
from __future__ import annotations

import torch

from . import snn
from . import workloads as W

EPS = 1e-6


def _pad8(n: int) -> int:
    return (n + 7) // 8 * 8


def head_decays(heads: int) -> torch.Tensor:
    """One decay for each head, memories from 8 to 8 * 2^(heads-1) steps."""
    return 1.0 - torch.exp2(-(3.0 + torch.arange(heads, dtype=torch.float32)))


class _Flat:
    """fp32 parameters of several shapes in one buffer, with their gradients
    and AdamW moments (every part starts on a 64-element boundary)."""

    def __init__(self, parts, dev, bf16: bool):
        offs = [0]
        for p in parts:
            offs.append(offs[-1] + (p.numel() + 63) // 64 * 64)
        host = torch.zeros(offs[-1])
        for o, p in zip(offs, parts):
            host[o:o + p.numel()] = p.flatten().float()
        self.w32 = host.to(dev)
        self.w16 = self.w32.to(torch.bfloat16) if bf16 else None
        self.grad = torch.zeros_like(self.w32)
        self.m, self.v = torch.zeros_like(self.w32), torch.zeros_like(self.w32)
        self.counter = torch.zeros(2, dtype=torch.int64, device=dev)
        view = lambda x: [x[o:o + p.numel()].view(p.shape) for o, p in zip(offs, parts)]
        self.parts = view(self.w16 if bf16 else self.w32)
        self.grads = view(self.grad)


class AttnSNN:
    """Buffers and calls of the network for sequences of w.T steps."""

    def __init__(self, w: W.AttnWorkload, weights, device="cuda", lr: float = 1e-3,
                 betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 1e-2):
        self.w, self.device = w, torch.device(device)
        self.lr, self.betas, self.eps, self.weight_decay = lr, betas, eps, weight_decay
        dev, T, B, N, S = self.device, w.T, w.B, w.width, w.spikes
        self.M, self.n_out = T * B, _pad8(w.n_classes)
        pad = torch.zeros((self.n_out, N), dtype=torch.bfloat16)
        pad[:w.n_classes] = weights[-1]
        self.weights = _Flat([*weights[:-1], pad], dev, bf16=True)
        one = torch.ones(N)
        # per block: w_pre, w_post, residual scale; then the last norm's w_pre
        norms = [x for _ in range(w.blocks) for x in (one, one, 0.5 * one)] + [one]
        self.norms = _Flat(norms, dev, bf16=False)
        self.decay = head_decays(w.heads).to(dev)
        self.beta = torch.full((1,), w.beta, dtype=torch.float32, device=dev)
        self.thr = torch.full((1,), w.thr, dtype=torch.float32, device=dev)
        f32 = lambda *s: torch.empty(s, dtype=torch.float32, device=dev)
        b16 = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=dev)
        self.scans = [self._scan(T, B, S + N, f"asnn_block{l}") for l in range(w.blocks)]
        self.readout = self._scan(T, B, self.n_out, "asnn_readout")
        self.r = [f32(self.M, N) for _ in range(w.blocks + 1)]
        self.y = [b16(self.M, N) for _ in range(w.blocks + 1)]
        self.I = f32(self.M, S + N)
        self.I_out = f32(self.M, self.n_out)
        self.o = [b16(T, B, N) for _ in range(w.blocks)]
        self.state = [f32(B, w.heads, w.head_dim, w.head_dim) for _ in range(w.blocks)]
        # zeros where a block's neurons get no gradient of that kind
        self.g_spk, self.g_mem = b16(T, B, S + N), b16(T, B, S + N)
        self.g_y, self.g_o = b16(self.M, N), b16(self.M, N)
        self.g_r = [f32(self.M, N) for _ in range(2)]
        self.g_in = b16(self.M, N)
        self.g_out = torch.empty((T, B, self.n_out), dtype=torch.bfloat16, device=dev)
        self.loss = torch.zeros(1, dtype=torch.float32, device=dev)
        u8 = lambda n: torch.zeros(n, dtype=torch.uint8, device=dev)
        self.ws = u8(256)
        self.ws_attn = u8(snn.snn_leaky_attn_workspace_bytes(
            B, T, w.heads, w.kv_heads, w.head_dim, w.head_dim, backward=True))
        self.ws_norm = u8(snn.snn_block_norm_workspace_bytes(self.M, N))
        self.ws_dense = [u8(snn.snn_dense_workspace_bytes(self.M, p.shape[1], p.shape[0]))
                         for p in self.weights.parts]
        self.ws_loss = u8(snn.snn_rate_ce_workspace_bytes(B))
        # single steps after a prompt: layers of one step, and the membrane
        # potentials that they go on from (here, so that prompt and token
        # allocate and initialise nothing and run on any stream)
        self._token = {"scans": [self._scan(1, B, S + N, "asnn_token") for _ in range(w.blocks)],
                       "readout": self._scan(1, B, self.n_out, "asnn_token_out")}
        self.mem = [torch.zeros_like(sc.mem_final) for sc in [*self.scans, self.readout]]

    def _scan(self, T, B, n, name):
        w = self.w
        return snn.ScanLayer(W.ScanWorkload(
            name=name, neuron="leaky", T=T, B=B, N=n, in_dtype=W.F32, io_dtype=W.BF16,
            beta=("const", w.beta), thr=("const", w.thr), surrogate="fast_sigmoid",
            sg_param=w.sg_param, save="mem", want_mem=True), device=self.device)

    def _qkv(self, x):
        """Queries, keys and values [B, T, heads, D] in the first columns of a
        [T, B, spikes + width] tensor, in place."""
        w, D = self.w, self.w.head_dim
        at = [0, w.heads * D, (w.heads + w.kv_heads) * D, w.spikes]
        return [x[..., i:j].unflatten(-1, (-1, D)).transpose(0, 1) for i, j in zip(at, at[1:])]

    def _heads(self, x):
        return x.view(self.w.T, self.w.B, self.w.heads, -1).transpose(0, 1)

    def _norm_args(self, l):
        """(w_post, residual scale, the next norm's w_pre) of block l."""
        p = self.norms.parts
        return p[3 * l + 1], p[3 * l + 2], p[3 * l + 3]

    def _norm_kw(self):
        return dict(eps=EPS, group=self.w.head_dim, gate="silu")

    def _forward_ops(self, X, stream, want_state):
        w, S = self.w, self.w.spikes
        T, B = w.T, w.B
        Wp = self.weights.parts
        out = [("dense_in", lambda: snn.snn_dense_layer_fwd(X, Wp[0], self.r[0], self.ws, stream)),
               ("norm_in", lambda: snn.snn_block_norm_fwd(
                   self.r[0], None, None, None, None, self.norms.parts[0], None, self.y[0],
                   eps=EPS, stream=stream))]
        for l, sc in enumerate(self.scans):
            q, k, v = self._qkv(sc.spk)
            out.append((f"dense{l}", lambda l=l: snn.snn_dense_layer_fwd(
                self.y[l], Wp[l + 1], self.I, self.ws, stream)))
            out.append((f"scan{l}", lambda sc=sc: sc.forward(
                self.I.view(T, B, -1), self.beta, self.thr, stream=stream)))
            out.append((f"attn{l}", lambda l=l, q=q, k=k, v=v: snn.snn_leaky_attn_fwd(
                q, k, v, self.decay, self._heads(self.o[l]), self.ws_attn, scale=self._scale(),
                state_out=self.state[l] if want_state else None, stream=stream)))
            out.append((f"norm{l}", lambda l=l, sc=sc: snn.snn_block_norm_fwd(
                self.r[l], self.o[l].view(self.M, -1), sc.mem.view(self.M, -1)[:, S:],
                *self._norm_args(l), self.r[l + 1], self.y[l + 1], stream=stream,
                **self._norm_kw())))
        out.append(("dense_out", lambda: snn.snn_dense_layer_fwd(
            self.y[-1], Wp[-1], self.I_out, self.ws, stream)))
        out.append(("scan_out", lambda: self.readout.forward(
            self.I_out.view(T, B, -1), self.beta, self.thr, stream=stream)))
        return out

    def _scale(self):
        return self.w.head_dim ** -0.5

    def _backward_ops(self, X, labels, stream):
        w, S, M = self.w, self.w.spikes, self.M
        Wp, dW, gn = self.weights.parts, self.weights.grads, self.norms.grads
        ro = self.readout
        out = [("ce_loss", lambda: snn.snn_rate_ce_leaky_bwd(
                   ro.desc, ro.spk, labels, w.n_classes, self.beta, self.thr, ro.mem, None,
                   self.loss, self.g_out, ro.grad_I, self.ws_loss, stream)),
               ("dense_out_bwd", lambda: snn.snn_dense_layer_bwd(
                   self.y[-1], Wp[-1], ro.grad_I.view(M, -1), self.g_y, dW[-1], self.ws_dense[-1],
                   stream))]
        for l in range(w.blocks - 1, -1, -1):
            sc, last = self.scans[l], l == w.blocks - 1
            q, k, v = self._qkv(sc.spk)
            gq, gk, gv = self._qkv(self.g_spk)
            g_in, g_to = self.g_r[(l + 1) % 2], self.g_r[l % 2]
            out.append((f"norm_bwd{l}", lambda l=l, sc=sc, g_in=g_in, g_to=g_to, last=last:
                        snn.snn_block_norm_bwd(
                            self.r[l + 1], self.o[l].view(M, -1), sc.mem.view(M, -1)[:, S:],
                            *self._norm_args(l), None if last else g_in, self.g_y, g_to, self.g_o,
                            self.g_mem.view(M, -1)[:, S:], gn[3 * l + 1], gn[3 * l + 2],
                            gn[3 * l + 3], self.ws_norm, stream=stream, **self._norm_kw())))
            out.append((f"attn_bwd{l}", lambda q=q, k=k, v=v, gq=gq, gk=gk, gv=gv:
                        snn.snn_leaky_attn_bwd(
                            q, k, v, self.decay, self._heads(self.g_o), gq, gk, gv, self.ws_attn,
                            scale=self._scale(), stream=stream)))
            out.append((f"scan_bwd{l}", lambda sc=sc: sc.backward(
                None, self.beta, self.thr, self.g_spk, grad_mem=self.g_mem, want_param_grads=False,
                want_state_grads=False, stream=stream)))
            out.append((f"dense_bwd{l}", lambda l=l, sc=sc: snn.snn_dense_layer_bwd(
                self.y[l], Wp[l + 1], sc.grad_I.view(M, -1), self.g_y, dW[l + 1],
                self.ws_dense[l + 1], stream)))
        g0 = self.g_r[1]
        out.append(("norm_in_bwd", lambda: snn.snn_block_norm_bwd(
            self.r[0], None, None, None, None, self.norms.parts[0],
            self.g_r[0] if w.blocks else None, self.g_y, g0, None, None, None, None, gn[0],
            self.ws_norm, eps=EPS, stream=stream)))
        out.append(("cast_in", lambda: self._on(stream, lambda: self.g_in.copy_(g0))))
        out.append(("dense_in_bwd", lambda: snn.snn_dense_layer_bwd(
            X, Wp[0], self.g_in, None, dW[0], self.ws_dense[0], stream)))
        return out

    @staticmethod
    def _on(stream, call):
        if stream is None:
            return call()
        with torch.cuda.stream(stream):
            return call()

    def ops(self, X, labels, stream=None):
        """The training step as a list of (name, call) in launch order.  X: bf16
        [T*B, n_in] spikes on the device, labels int32 [B]."""
        out = self._forward_ops(X, stream, False) + self._backward_ops(X, labels, stream)
        out.append(("adamw", lambda: self.update(stream)))
        return out

    def update(self, stream=None):
        for f, decay in ((self.weights, self.weight_decay), (self.norms, 0.0)):
            snn.snn_adamw_step(f.w32, f.w16, f.grad, f.m, f.v, self.lr, self.betas[0],
                               self.betas[1], self.eps, decay, step_counter=f.counter,
                               stream=stream)

    def train_step(self, X, labels, stream=None):
        """Forward, loss, reverse pass and AdamW update; returns the loss [1]."""
        for _, call in self.ops(X, labels, stream):
            call()
        return self.loss

    def gradients(self, X, labels, stream=None):
        """The step without its update; returns the weights' gradients."""
        for _, call in self.ops(X, labels, stream)[:-1]:
            call()
        return self.weights.grads

    def prompt(self, X, stream=None):
        """The forward over w.T steps, leaving every state for `token`;
        returns the readout's spikes [T, B, n_classes]."""
        for _, call in self._forward_ops(X, stream, True):
            call()
        self._on(stream, self._keep_mem)
        return self.readout.spk[..., :self.w.n_classes]

    def _keep_mem(self):
        for mem, sc in zip(self.mem, [*self.scans, self.readout]):
            mem.copy_(sc.mem_final)

    def token(self, x, stream=None):
        """One more step x [B, n_in] of every sequence after `prompt`: the
        scans go on from their membrane potentials, the attention from its
        states, which are updated in place.  Returns the readout's spikes [B,
        n_classes]; the block outputs are in `token_o`."""
        w, B, N, S, D = self.w, self.w.B, self.w.width, self.w.spikes, self.w.head_dim
        Wp = self.weights.parts
        r, y = self.r[0][:B], self.y[0][:B]
        snn.snn_dense_layer_fwd(x, Wp[0], r, self.ws, stream)
        snn.snn_block_norm_fwd(r, None, None, None, None, self.norms.parts[0], None, y, eps=EPS,
                               stream=stream)
        self.token_o = []
        for l, sc in enumerate(self._token["scans"]):
            snn.snn_dense_layer_fwd(y, Wp[l + 1], self.I[:B], self.ws, stream)
            sc.forward(self.I[:B].view(1, B, -1), self.beta, self.thr, mem0=self.mem[l],
                       stream=stream)
            self.mem[l], sc.mem_final = sc.mem_final, self.mem[l]
            spk = sc.spk[0]
            at = [0, w.heads * D, (w.heads + w.kv_heads) * D, S]
            q, k, v = (spk[:, i:j].unflatten(-1, (-1, D)) for i, j in zip(at, at[1:]))
            o = self.o[l][0]
            snn.snn_leaky_attn_step(q, k, v, self.decay, self.state[l],
                                    o.view(B, w.heads, D), scale=self._scale(), stream=stream)
            self.token_o.append(o)
            r_out, y = self.r[l + 1][:B], self.y[l + 1][:B]
            snn.snn_block_norm_fwd(r, o, sc.mem[0][:, S:], *self._norm_args(l), r_out, y,
                                   stream=stream, **self._norm_kw())
            r = r_out
        snn.snn_dense_layer_fwd(y, Wp[-1], self.I_out[:B], self.ws, stream)
        ro = self._token["readout"]
        ro.forward(self.I_out[:B].view(1, B, -1), self.beta, self.thr, mem0=self.mem[-1],
                   stream=stream)
        self.mem[-1], ro.mem_final = ro.mem_final, self.mem[-1]
        return ro.spk[0, :, :w.n_classes]
