"""Layer norm on the GPU against its float64 definition.

All arithmetic is fp32.  The mean's error is (16 + 25) units of 2^-24 of the row's
mean magnitude (16 values in a thread and a tree), the deviation's a few more, so a
normalised value errs by c = 96 units of rstd (|x| + mean |x|) and of its own
size; a gradient's sums over a row the same.  A parameter's gradient adds
up to M terms, at most M / 152 + 160 in a chain.
"""
import numpy as np
import pytest
import torch

from oracle import seq_oracle as O
from paper_2211_10725_gb300 import snn
from tests.test_gpu_sel_scan import BF, F32, HF, NAN, _np, close

pytestmark = pytest.mark.gpu
EPS = 1e-5
TYPES = [(F32, F32), (BF, BF), (BF, F32), (HF, HF), (HF, F32)]


class Case:
    def __init__(self, dev, M, N, dtype, res, pad=0, offset=0.3, w=True, b=True):
        g = torch.Generator().manual_seed(M + 5 * N)
        self.dev, self.M, self.N, self.dtype, self.res, self.pad = dev, M, N, dtype, res, pad

        def rows(dt, scale, shift):
            x = torch.full((M, N + pad), NAN, dtype=dt)
            x[:, :N] = (scale * torch.randn(M, N, generator=g) + shift).to(dt)
            return x.to(dev)[:, :N]
        self.rows = rows
        self.x, self.gy = rows(res, 2.0, offset), rows(dtype, 0.3, 0.0)
        self.w = (1 + 0.2 * torch.randn(N, generator=g)).to(dev) if w else None
        self.b = (0.2 * torch.randn(N, generator=g)).to(dev) if b else None

    def check(self):
        y = self.rows(self.dtype, 1.0, 0.0)
        y.fill_(NAN)
        stats = torch.full((2, self.M), NAN, device=self.dev)
        snn.snn_layer_norm_fwd(self.x, self.w, self.b, y, stats=stats, eps=EPS)
        x, w, b = _np(self.x), _np(self.w), _np(self.b)
        r = 1.0 / np.sqrt(x.var(-1, keepdims=True) + EPS)
        aw = 1.0 if w is None else np.abs(w)
        near = r * (np.abs(x) + np.abs(x).mean(-1, keepdims=True))
        close("y", y, O.layer_norm_forward(x, w, b, EPS), near * aw + (0.0 if b is None else np.abs(b)), 96)
        gx = self.rows(self.res, 1.0, 0.0)
        gx.fill_(NAN)
        gw, gb = (torch.full((self.N,), NAN, device=self.dev) for _ in range(2))
        ws = torch.full((snn.snn_layer_norm_workspace_bytes(self.M, self.N),), 255, dtype=torch.uint8, device=self.dev)
        snn.snn_layer_norm_bwd(self.x, self.w, stats, self.gy, gx, gw, gb, ws)
        gy = _np(self.gy)
        want = O.layer_norm_backward(x, w, gy, EPS)
        g = np.abs(gy) * aw
        mean = lambda v: v.mean(-1, keepdims=True)
        close("grad_x", gx, want["x"], r * (g + mean(g) + near * mean(g * near)), 96)
        chain = 96 + 160 + self.M / 152
        close("grad_w", gw, want["w"], (np.abs(gy) * near).sum(0), chain)
        close("grad_b", gb, want["b"], np.abs(gy).sum(0), chain)
        return gx, gw, gb


@pytest.mark.parametrize("dtype,res", TYPES)
@pytest.mark.parametrize("M,N", [(1, 8), (7, 264), (33, 1024), (5, 2048), (3, 4096), (2, 8192), (400, 48)])
def test_sizes(M, N, dtype, res, cuda_device):
    Case(cuda_device, M, N, dtype, res).check()


@pytest.mark.parametrize("dtype,res", TYPES)
@pytest.mark.parametrize("M,N", [(1, 1), (4, 3), (9, 255), (5, 1001), (2, 4099), (3, 8191), (1, 1000)])
def test_odd_sizes(M, N, dtype, res, cuda_device):
    Case(cuda_device, M, N, dtype, res).check()


@pytest.mark.parametrize("pad", [1, 8])
@pytest.mark.parametrize("N", [96, 250, 2048])
def test_strides(N, pad, cuda_device):
    Case(cuda_device, 11, N, BF, F32, pad=pad).check()
    Case(cuda_device, 11, N, F32, F32, pad=pad).check()


def test_rows_far_from_zero(cuda_device):
    """The variance about the mean: with E[x^2] - mean^2 nothing would be left."""
    Case(cuda_device, 8, 512, F32, F32, offset=300.0).check()


def test_equal_values(cuda_device):
    c = Case(cuda_device, 3, 40, F32, F32)
    c.x.fill_(0.0)
    y = torch.empty_like(c.x)
    snn.snn_layer_norm_fwd(c.x, c.w, c.b, y, eps=EPS)
    assert torch.equal(y, c.b.expand(3, 40))


def test_absent_parameters_and_outputs(cuda_device):
    Case(cuda_device, 6, 200, BF, BF, w=False, b=False).check()
    c = Case(cuda_device, 6, 200, F32, F32, b=False)
    gx, gw, gb = c.check()
    stats = torch.empty(2, 6, device=cuda_device)
    snn.snn_layer_norm_fwd(c.x, c.w, None, torch.empty_like(c.x), stats=stats, eps=EPS)
    only = torch.full_like(gx, NAN)
    snn.snn_layer_norm_bwd(c.x, c.w, stats, c.gy, only, None, None, None)
    assert torch.equal(only, gx)
    ws = torch.empty(snn.snn_layer_norm_workspace_bytes(6, 200), dtype=torch.uint8, device=cuda_device)
    w2 = torch.full_like(gw, NAN)
    snn.snn_layer_norm_bwd(c.x, c.w, stats, c.gy, None, w2, None, ws)
    assert torch.equal(w2, gw)


def test_many_rows_repeat_and_no_rows(cuda_device):
    c = Case(cuda_device, 3001, 72, BF, F32)
    for a, b in zip(c.check(), c.check()):
        assert torch.equal(a, b)
    gw, gb = (torch.full((72,), NAN, device=cuda_device) for _ in range(2))
    ws = torch.empty(snn.snn_layer_norm_workspace_bytes(0, 72), dtype=torch.uint8, device=cuda_device)
    none = torch.empty(0, 72, device=cuda_device)
    snn.snn_layer_norm_bwd(none, c.w, torch.empty(2, 0, device=cuda_device), none.to(BF), None, gw, gb, ws)
    assert torch.count_nonzero(gw) == 0 and torch.count_nonzero(gb) == 0


# rows of several warps are worked on two at a time: teams with an odd count, the last rows alone
@pytest.mark.parametrize("dtype,res", [(BF, F32), (HF, HF), (F32, F32)])
@pytest.mark.parametrize("M,N", [(2000, 1024), (1001, 2048), (461, 4096), (305, 4090), (306, 8192), (4100, 512)])
def test_several_rows_of_a_team(M, N, dtype, res, cuda_device):
    Case(cuda_device, M, N, dtype, res).check()


@pytest.mark.parametrize("N", [1024, 1001, 200])
def test_a_row_without_values_stays_alone(N, cuda_device):
    """Whatever lies in some rows, the others' results are the same bits."""
    c = Case(cuda_device, 2500, N, F32, F32)
    got = []
    for bad in (None, NAN, float("inf")):
        if bad is not None:
            c.x[5::100] = bad
        y, stats, gx = torch.empty_like(c.x), torch.empty(2, 2500, device=cuda_device), torch.empty_like(c.x)
        snn.snn_layer_norm_fwd(c.x, c.w, c.b, y, stats=stats, eps=EPS)
        snn.snn_layer_norm_bwd(c.x, c.w, stats, c.gy, gx, None, None, None)
        got.append((y, gx))
    good = torch.ones(2500, dtype=torch.bool, device=cuda_device)
    good[5::100] = False
    for y, gx in got[1:]:
        assert torch.equal(y[good], got[0][0][good]) and torch.equal(gx[good], got[0][1][good])
        assert torch.isnan(y[~good]).all() and torch.isnan(gx[~good]).all()


def test_in_place(cuda_device):
    for N in (64, 61):
        c = Case(cuda_device, 700, N, F32, F32)
        y = torch.empty_like(c.x)
        stats = torch.empty(2, 700, device=cuda_device)
        snn.snn_layer_norm_fwd(c.x, c.w, c.b, y, stats=stats, eps=EPS)
        gx = torch.empty_like(c.x)
        snn.snn_layer_norm_bwd(c.x, c.w, stats, c.gy, gx, None, None, None)
        g2, x2 = c.gy.clone(), c.x.clone()
        snn.snn_layer_norm_bwd(c.x, c.w, stats, g2, g2, None, None, None)
        snn.snn_layer_norm_fwd(x2, c.w, c.b, x2, eps=EPS)
        assert torch.equal(g2, gx) and torch.equal(x2, y)


@pytest.mark.parametrize("M,N", [(1500, 1024), (700, 2048), (400, 8192), (700, 4095)])
def test_in_place_with_rows_on_their_way(M, N, cuda_device):
    c = Case(cuda_device, M, N, BF, BF)
    y, stats, gx = torch.empty_like(c.x), torch.empty(2, M, device=cuda_device), torch.empty_like(c.x)
    snn.snn_layer_norm_fwd(c.x, c.w, c.b, y, stats=stats, eps=EPS)
    snn.snn_layer_norm_bwd(c.x, c.w, stats, c.gy, gx, None, None, None)
    g2, x2 = c.gy.clone(), c.x.clone()
    snn.snn_layer_norm_bwd(c.x, c.w, stats, g2, g2, None, None, None)
    snn.snn_layer_norm_fwd(x2, c.w, c.b, x2, eps=EPS)
    assert torch.equal(g2, gx) and torch.equal(x2, y)


def test_refusals_of_the_binding(cuda_device):
    c = Case(cuda_device, 4, 32, BF, F32)
    y = torch.empty(4, 32, dtype=BF, device=cuda_device)
    for bad in (dict(w=c.w[:8]), dict(x=c.x.t()), dict(stats=torch.empty(4, 2, device=cuda_device)),
                dict(y=y.to(torch.float64))):
        with pytest.raises(ValueError):
            snn.snn_layer_norm_fwd(**{**dict(x=c.x, w=c.w, b=c.b, y=y), **bad})
    with pytest.raises(snn.SnnError):
        snn.snn_layer_norm_fwd(c.x.to(HF), c.w, c.b, y)
