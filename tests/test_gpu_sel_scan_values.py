"""Selective scan on the GPU: steps of the largest, lowest and infinite values.
Tolerances as in test_gpu_sel_scan.py.
"""
import numpy as np
import pytest
import torch

from oracle import seq_oracle as O
from paper_2211_10725_gb300 import snn
from tests import test_gpu_sel_scan as scan_tests
from tests.test_gpu_sel_scan import BF, Case, F32, HALF_UNIT, HF, NAN, _np, close

pytestmark = pytest.mark.gpu
INF = float("inf")


def _far(c):
    """Of every channel: tokens that do nothing (delta -inf, the type's lowest value, -1e38) and
    some that forget all (two next to each other, whose sum is past fp32).  There
    u and B are small enough for s u B and, but for fp16, every gradient to have a value."""
    info = torch.finfo(c.dtype)
    lowest = [-INF, info.min, max(-1e38, info.min)]
    most = min(3e38, info.max)
    g = torch.Generator().manual_seed(5)
    for t in range(c.T):
        kind = int(torch.randint(0, 4, (), generator=g))
        if kind < 3 and t % 3 == 0:
            c.delta[:, t, kind::3] = lowest[kind]
        elif t % 16 in (7, 8):
            c.delta[:, t] = most
            c.u[:, t] = c.u[:, t].clamp(-2, 2) * (1.0 / most if c.dtype != HF else 1e-4)
            if c.dtype != HF:
                c.Bm[:, t] *= 1e-19
    return c


def _far_close(name, got, want, size, units, lost=0.0):
    """As close; a value past the type's largest (within its tolerance) may be infinite: in
    fp16 the product of a step of 65504 and the sum over states that it is given."""
    most = torch.finfo(got.dtype).max
    tol = HALF_UNIT[got.dtype] * np.abs(want) + units * 2.0 ** -24 * size
    past = torch.isinf(got) & torch.from_numpy(np.abs(want) + tol > most).to(got.device)
    past &= torch.sign(got) == torch.from_numpy(np.sign(want)).to(got.device)
    zero = past.cpu().numpy()
    close(name, got.masked_fill(past, 0.0), np.where(zero, 0.0, want), np.where(zero, 0.0, size), units, lost)


@pytest.mark.parametrize("dtype", [F32, BF, HF])
@pytest.mark.parametrize("T,N,pad", [(24, 16, 0), (300, 16, 1), (300, 5, 0), (700, 20, 0)])
def test_far_steps(T, N, pad, dtype, cuda_device, monkeypatch):
    monkeypatch.setattr(scan_tests, "close", _far_close)
    c = _far(Case(cuda_device, 2, T, 22, N, dtype, pad=pad))
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("dtype", [F32, BF, HF])
@pytest.mark.parametrize("N", [5, 16])
def test_far_steps_of_single_tokens(N, dtype, cuda_device):
    """A token with a step of zero leaves the pool's states as they are."""
    c = Case(cuda_device, 3, 1, 24, N, dtype, bias=False)
    info = torch.finfo(dtype)
    for i, v in enumerate((-INF, info.min, max(-1e38, info.min))):
        c.delta[:, :, i::3] = v
    pool = c.state.clone()
    one = lambda x: x[:, 0]
    y = c.new(c.u)[:, 0]
    snn.snn_selective_scan_step(one(c.u), one(c.delta), c.A, one(c.Bm), one(c.Cm), pool, y, D=c.D_skip, z=one(c.z))
    assert torch.equal(pool, c.state)
    args, kw = c.oracle_args()
    want, _ = O.scan_forward(*args, **kw)
    size, _ = O.scan_forward(*args, positive=True, **kw)
    close("y", y, want[:, 0], size[:, 0], 160 + N)


@pytest.mark.parametrize("T", [20, 300])
@pytest.mark.parametrize("dtype", [F32, BF])
def test_a_nan_step_stays_one(T, dtype, cuda_device):
    c = Case(cuda_device, 2, T, 12, 8, dtype)
    c.delta[1, 9, 3] = NAN
    y, end = c.forward()
    hit = torch.zeros_like(y, dtype=torch.bool)
    hit[1, 9:, 3] = True
    assert torch.equal(torch.isnan(y), hit)
    assert torch.isnan(end[1, 3]).all() and torch.isfinite(end[0]).all()


@pytest.mark.parametrize("T,N", [(100, 8), (600, 8), (603, 5)])
def test_growing_states(T, N, cuda_device):
    """Negative steps, over whose spans the decays alone are past fp32 while the states are not:
    states of zero, and small ones that grow by up to e^115 in 12 tokens near
    the first or the last."""
    c = Case(cuda_device, 2, T, 12, N, F32, softplus=False, bias=False)
    for x in (c.u, c.gy):
        x[:, :, :8] = 0
    c.delta[:, :, :8] = 0
    c.state[:, :4] = c.gs[:, :4] = 0
    c.delta[:, :, :4] = -0.6
    c.state[:, 4:8] = c.gs[:, 4:8] = 1e-30
    c.delta[:, 2:14, 4:6] = -1.2
    c.delta[:, T - 14:T - 2, 6:8] = -1.2
    c.A[:, :] = -torch.arange(1, N + 1, device=cuda_device)
    c.check_forward()
    for name, x in c.check_backward().items():
        assert x is None or torch.isfinite(x).all(), name
