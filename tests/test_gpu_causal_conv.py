"""Causal convolution on the GPU against its float64 definition.

fp32 arithmetic: W products and additions and an activation, so c = 32 units of
2^-24 of the terms' size beside the result's own rounding (half unit u_t); 16-bit results
take the approximate power of two and reciprocal, |p| 2^-24 of the result and two
units each: c = 64.  A parameter's gradient adds up to B T terms: c + B T.
"""
import numpy as np
import pytest
import torch

from oracle import seq_oracle as O
from paper_2211_10725_gb300 import snn
from tests.test_gpu_sel_scan import BF, F32, HF, NAN, _np, close

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, dev, B, T, C, W, dtype=BF, act="silu", bias=True, state=True, lens=None, pad=0, seed=0):
        g = torch.Generator().manual_seed(99 * seed + B + 3 * T + C + W)
        self.dev, self.B, self.T, self.C, self.W, self.act, self.lens_list = dev, B, T, C, W, act, lens

        def rows(*s):
            x = torch.full((*s[:-1], s[-1] + pad), NAN, dtype=dtype)
            x[..., :s[-1]] = torch.randn(s, generator=g).to(dtype)
            return x.to(dev)[..., :s[-1]]
        self.x, self.gy = rows(B, T, C), rows(B, T, C)
        self.w = (torch.randn(C, W, generator=g) * W ** -0.5).to(dev)
        self.bias = (0.3 * torch.randn(C, generator=g)).to(dev) if bias else None
        st = lambda: torch.randn(B, W - 1, C, generator=g).to(dtype).to(dev)
        self.state, self.gs = (st() if state else None), st()
        if lens is not None:
            for b, n in enumerate(lens):
                self.x[b, n:] = NAN
                self.gy[b, n:] = NAN
        self.lens = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=dev)

    def new(self, t):
        return torch.full(t.shape, NAN, dtype=t.dtype, device=self.dev)

    def oracle(self):
        return dict(bias=_np(self.bias), act=self.act, lens=self.lens_list, state=_np(self.state))

    def check(self, gs=True):
        y, end = self.new(self.x), self.new(self.gs)
        snn.snn_causal_conv_fwd(self.x, self.w, self.bias, y, act=self.act, seq_lens=self.lens, state_in=self.state,
                                state_out=end)
        x, w = np.nan_to_num(_np(self.x)), _np(self.w)
        want, last = O.conv_forward(x, w, **self.oracle())
        size, _ = O.conv_forward(x, w, positive=True, **self.oracle())
        close("y", y, want, size, 64)
        assert np.array_equal(_np(end), last)
        o = {"x": self.new(self.x), "w": self.new(self.w), "bias": None if self.bias is None else self.new(self.bias),
             "state": self.new(self.gs)}
        ws = torch.full((snn.snn_causal_conv_workspace_bytes(self.B, self.T, self.C, self.W),), 255,
                        dtype=torch.uint8, device=self.dev)
        snn.snn_causal_conv_bwd(self.x, self.w, self.bias, self.gy, o["x"], o["w"], o["bias"], ws, act=self.act,
                                seq_lens=self.lens, state_in=self.state, grad_state_out=self.gs if gs else None,
                                grad_state_in=o["state"])
        gy, gstate = np.nan_to_num(_np(self.gy)), _np(self.gs) if gs else None
        want = O.conv_backward(x, w, gy, gstate=gstate, **self.oracle())
        size = O.conv_backward(x, w, gy, gstate=gstate, positive=True, **self.oracle())
        for name, t in o.items():
            if t is not None:
                close(name, t, want[name], size[name], 64 + (self.B * self.T if name in ("w", "bias") else 0))
        if self.lens_list:
            for b, n in enumerate(self.lens_list):
                assert torch.count_nonzero(y[b, n:]) == 0 and torch.count_nonzero(o["x"][b, n:]) == 0
        return o


@pytest.mark.parametrize("dtype", [F32, BF, HF])
@pytest.mark.parametrize("W", [2, 3, 4])
@pytest.mark.parametrize("B,T,C", [(1, 1, 1), (2, 2, 8), (1, 37, 64), (3, 100, 24), (2, 9, 13), (1, 300, 264)])
def test_sizes(B, T, C, W, dtype, cuda_device):
    Case(cuda_device, B, T, C, W, dtype).check()


@pytest.mark.parametrize("pad", [1, 2, 8])
@pytest.mark.parametrize("C", [16, 20, 7])
def test_strides(C, pad, cuda_device):
    Case(cuda_device, 2, 40, C, 4, BF, pad=pad).check()
    Case(cuda_device, 2, 40, C, 3, F32, pad=pad).check()


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("bias,state,gs", [(False, False, False), (True, False, True), (False, True, True)])
def test_absent_parts(act, bias, state, gs, cuda_device):
    Case(cuda_device, 2, 23, 40, 4, F32, act, bias, state).check(gs)


@pytest.mark.parametrize("T,lens", [(30, [30, 0, 17, 1, 2]), (64, [64, 63, 33, 32, 3]), (2, [0, 1, 2, 2, 0])])
@pytest.mark.parametrize("W", [2, 4])
def test_padded_batches(T, lens, W, cuda_device):
    Case(cuda_device, 5, T, 24, W, F32, lens=lens).check()
    Case(cuda_device, 5, T, 9, W, HF, lens=lens).check()


def test_long_runs(cuda_device):
    """Enough threads for the longest runs of tokens."""
    Case(cuda_device, 4, 1100, 2048, 4, BF).check()


def test_tokens_of_no_length(cuda_device):
    c = Case(cuda_device, 2, 0, 8, 4, F32)
    end, gs = c.new(c.gs), c.new(c.gs)
    snn.snn_causal_conv_fwd(c.x, c.w, c.bias, c.new(c.x), state_in=c.state, state_out=end)
    assert torch.equal(end, c.state)
    gw = c.new(c.w)
    ws = torch.empty(snn.snn_causal_conv_workspace_bytes(2, 0, 8, 4), dtype=torch.uint8, device=cuda_device)
    snn.snn_causal_conv_bwd(c.x, c.w, c.bias, c.gy, None, gw, None, ws, state_in=c.state, grad_state_out=c.gs,
                            grad_state_in=gs)
    assert torch.equal(gs, c.gs) and torch.count_nonzero(gw) == 0


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("B,C,W", [(1, 8, 4), (4, 40, 3), (5, 33, 2), (3, 1, 4)])
def test_steps(B, C, W, dtype, cuda_device):
    c = Case(cuda_device, B, 1, C, W, dtype, pad=3)
    pool = torch.randn(B + 2, W - 1, C, device=cuda_device).to(dtype)
    before = pool.clone()
    at = [B + 1 - b for b in range(B)]
    at[-1] = -1 if B > 1 else at[-1]
    slots = torch.tensor(at, dtype=torch.int32, device=cuda_device)
    y = c.new(c.x)[:, 0]
    snn.snn_causal_conv_step(c.x[:, 0], c.w, c.bias, pool, y, act="silu", slots=slots)
    state = np.zeros((B, W - 1, C))
    used = [b for b in range(B) if at[b] >= 0]
    state[used] = _np(before)[[at[b] for b in used]]
    kw = dict(bias=_np(c.bias), act="silu", lens=[int(b in used) for b in range(B)], state=state)
    want, end = O.conv_forward(_np(c.x), _np(c.w), **kw)
    size, _ = O.conv_forward(_np(c.x), _np(c.w), positive=True, **kw)
    close("y", y, want[:, 0], size[:, 0], 64)
    for p in range(B + 2):
        assert np.array_equal(_np(pool[p]), end[at.index(p)] if p in at else _np(before[p]))


def test_state_over_the_one_read(cuda_device):
    c = Case(cuda_device, 2, 50, 24, 4, F32)
    y, end = c.new(c.x), c.new(c.gs)
    snn.snn_causal_conv_fwd(c.x, c.w, c.bias, y, state_in=c.state, state_out=end)
    y2, state = c.new(c.x), c.state.clone()
    snn.snn_causal_conv_fwd(c.x, c.w, c.bias, y2, state_in=state, state_out=state)
    assert torch.equal(y, y2) and torch.equal(end, state)
    short = c.state.clone()     # shorter than the state: rows move up
    lens = torch.tensor([1, 0], dtype=torch.int32, device=cuda_device)
    snn.snn_causal_conv_fwd(c.x, c.w, c.bias, y2, state_in=short, state_out=short, seq_lens=lens)
    assert torch.equal(short[0], torch.cat([c.state[0, 1:], c.x[0, :1]])) and torch.equal(short[1], c.state[1])


def test_results_repeat_in_a_graph(cuda_device):
    c = Case(cuda_device, 2, 200, 64, 4, BF)
    first = c.check()
    ws = torch.empty(snn.snn_causal_conv_workspace_bytes(2, 200, 64, 4), dtype=torch.uint8, device=cuda_device)
    o = [c.new(c.x), c.new(c.w), c.new(c.bias)]
    run = lambda: snn.snn_causal_conv_bwd(c.x, c.w, c.bias, c.gy, *o, ws, act="silu", state_in=c.state,
                                          grad_state_out=c.gs)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for t in o:
        t.fill_(NAN)
    graph.replay()
    for t, name in zip(o, ("x", "w", "bias")):
        assert torch.equal(t, first[name])


def test_refusals_of_the_binding(cuda_device):
    c = Case(cuda_device, 2, 8, 16, 4, BF)
    y = c.new(c.x)
    for bad in (dict(w=c.w.t()), dict(y=y.float()), dict(bias=c.w[0]), dict(x=c.x[:, :, ::2]), dict(act="tanh"),
                dict(state_in=c.state.float())):
        kw = {**dict(x=c.x, w=c.w, bias=c.bias, y=y), **bad}
        with pytest.raises(ValueError):
            snn.snn_causal_conv_fwd(**kw)
    with pytest.raises(snn.SnnError):
        snn.snn_causal_conv_fwd(c.x, c.w, c.bias, y, act="sigmoid")


@pytest.mark.parametrize("dtype", [F32, BF, HF])
@pytest.mark.parametrize("W", [2, 3, 4])
@pytest.mark.parametrize("B,C", [(5, 40), (3, 33)])
def test_steps_over_their_input(B, C, W, dtype, cuda_device):
    """y may be x itself: the state takes the inputs, as with a y of its own."""
    c = Case(cuda_device, B, 1, C, W, dtype)
    slots = torch.tensor([B - b for b in range(B - 1)] + [-1], dtype=torch.int32, device=cuda_device)
    pools = [torch.randn(B + 2, W - 1, C, device=cuda_device).to(dtype)]
    pools.append(pools[0].clone())
    y, x = c.new(c.x), c.x.clone()
    for t in range(W + 1):
        snn.snn_causal_conv_step(c.x[:, 0], c.w, c.bias, pools[0], y[:, 0], act="silu", slots=slots)
        snn.snn_causal_conv_step(x[:, 0], c.w, c.bias, pools[1], x[:, 0], act="silu", slots=slots)
        assert torch.equal(x, y) and torch.equal(*pools)
        c.x.copy_(y)
