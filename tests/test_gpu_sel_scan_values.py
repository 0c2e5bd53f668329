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


# Long memories.  A state that remembers m tokens (|s A| = 1 / m) is a product of m rounded
# decays.  A decay errs by 0.6 units of 2^-24 (root mean square; a rounding to fp32 between 1/2 and
# 1 alone by 0.29 to 0.58), the addition to the state by 0.42, independently from token to
# token where the steps differ: 0.73 sqrt(m / 2) of the state, 8.7 units for the longest memory
# here, m = 286.  What is left of the approximate power's bias after its correction adds
# at most 15 units where steps differ most, and 2 where they are alike: their root of squares is
# below 20 units, which is a state's tolerance in the 2-norm over channels (no
# correction: 51 units for steps alike; one from the sum of eight unequal steps: 45).  A gradient that is a sum of
# products of two such states: sqrt(2) of that, 28, and for its own additions in order, 0.2 sqrt(terms) units for
# random signs, up to 10: 30.  That of A is a sum over sequences whose own sums have random signs too, so that
# what it is off by is measured on the square root of the sum of their squares.  Of only two channels it
# is the 2-norm of two normal numbers, above sqrt(x) of what is expected with a chance of e^-x: sqrt(7.4) = 2.7 for
# one in a hundred among 16 states.
UNIT = 2.0 ** -24


def _memories(dev, B, T, D, kind):
    """A case with |s A| of 0.0035 to 0.056 on average: steps alike (spread by 30%), or one in eight
    of eight times that among steps near zero, or one of each eight among steps of zero."""
    c = Case(dev, B, T, D, 16, F32, gate=False, softplus=False, bias=False)
    g = torch.Generator().manual_seed(17)
    n = torch.randn(B, T, D, generator=g)
    s = 0.056 * torch.exp(0.3 * n - 0.045)
    if kind == "sparse":
        s = s * torch.where(torch.rand(B, T, D, generator=g) < 1 / 8, 8.0, 1e-3)
    if kind == "single":
        s = 8 * s * (torch.arange(T) % 8 == torch.randint(0, 8, (B, T // 8, 1), generator=g).repeat_interleave(8, 1)[..., 0])[..., None]
    c.delta.copy_(s)
    c.A.copy_(-(torch.arange(1, 17) / 16.0).expand(D, 16) * torch.exp(0.02 * torch.randn(D, 16, generator=g)))
    c.kw["delta_bias"] = None
    return c


def _definition(c):
    """y, the last state and the gradients in 64 bits (G = 1, no gate, steps as they are)."""
    d = lambda x: x.double()
    u, s, A, Bm, Cm, gy, skip = map(d, (c.u, c.delta, c.A, c.Bm[:, :, 0], c.Cm[:, :, 0], c.gy, c.D_skip))
    h, hs, y = d(c.state), [d(c.state)], torch.empty_like(u)
    for t in range(c.T):
        h = torch.exp(s[:, t, :, None] * A) * h + (s[:, t] * u[:, t])[..., None] * Bm[:, t, None]
        y[:, t] = (h * Cm[:, t, None]).sum(-1) + skip * u[:, t]
        hs.append(h)
    g, o = d(c.gs), {k: torch.zeros_like(v) for k, v in (("u", u), ("delta", s), ("B", Bm), ("C", Cm), ("A", h))}
    for t in range(c.T - 1, -1, -1):
        a = torch.exp(s[:, t, :, None] * A)
        o["C"][:, t] = (gy[:, t, :, None] * hs[t + 1]).sum(1)
        g = g + gy[:, t, :, None] * Cm[:, t, None]
        o["B"][:, t] = (g * (s[:, t] * u[:, t])[..., None]).sum(1)
        w, q = (g * Bm[:, t, None]).sum(-1), a * g * hs[t]
        o["A"] += q * s[:, t, :, None]
        o["u"][:, t] = s[:, t] * w + skip * gy[:, t]
        o["delta"][:, t] = u[:, t] * w + (q * A).sum(-1)
        g = a * g
    o["state"] = g
    return y, h, o


def _off(got, want, dims=None):
    """Units of 2^-24 of the 2-norm that a result is off by (dims: of each of its other places)."""
    e = (got.double() - want).square()
    if dims is None:
        return float((e.sum() / want.square().sum()).sqrt()) / UNIT
    return float((e.sum(dims) / want.square().sum(dims)).sqrt().max()) / UNIT


def _sum_off(got, parts):
    """The same of a sum over sequences, on their 2-norm."""
    e = (got.double() - parts.sum(0)).square().sum(0)
    return float((e / parts.square().sum((0, 1))).sqrt().max()) / UNIT


# a cut axis, and sequences enough for whole ones
@pytest.mark.parametrize("B,T,D", [(2, 4096, 64), (1300, 1024, 2)])
@pytest.mark.parametrize("kind", ["alike", "sparse", "single"])
def test_long_memories(B, T, D, kind, cuda_device):
    c = _memories(cuda_device, B, T, D, kind)
    y, end = c.forward(ckpt=True)
    got = c.backward()
    want_y, want_end, want = _definition(c)
    off = {"y": _off(y, want_y), "end": _off(end, want_end, (0, 1)), "state": _off(got["state"], want["state"], (0, 1)),
           "A": _sum_off(got["A"], want["A"]) / (1.5 * (2.7 if D == 2 else 1.0)), "B": _off(got["B"][:, :, 0], want["B"]),
           "C": _off(got["C"][:, :, 0], want["C"])}
    for name in ("u", "delta"):
        off[name] = _off(got[name], want[name]) / 1.5
    assert max(off.values()) < 20, off


@pytest.mark.parametrize("N", [16, 7])
@pytest.mark.parametrize("kind", ["alike", "single"])
def test_long_memories_of_single_tokens(kind, N, cuda_device):
    """700 tokens one by one, as far from the definition as a sequence may be."""
    c = _memories(cuda_device, 4, 704, 64, kind)
    c.A, c.state = c.A[:, :N].contiguous(), c.state[..., :N].contiguous()
    c.Bm, c.Cm = c.Bm[..., :N], c.Cm[..., :N]   # (of rows of 16: every token's start on 16 bytes)
    pool, y = c.state.clone(), c.new(c.u)
    h, want = c.state.double(), torch.empty_like(c.u, dtype=torch.float64)
    d = lambda x, t: x[:, t].double()
    for t in range(c.T):
        one = lambda x: x[:, t]
        snn.snn_selective_scan_step(one(c.u), one(c.delta), c.A, one(c.Bm), one(c.Cm), pool, y[:, t], D=c.D_skip,
                                    softplus=False)
        h = torch.exp(d(c.delta, t)[..., None] * c.A.double()) * h \
            + (d(c.delta, t) * d(c.u, t))[..., None] * d(c.Bm, t)
        want[:, t] = (h * d(c.Cm, t)).sum(-1) + c.D_skip.double() * d(c.u, t)
    off = {"y": _off(y, want), "pool": _off(pool, h, (0, 1))}
    assert max(off.values()) < 20, off


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("N", [16, 20, 6, 50])
def test_the_largest_steps_of_single_tokens(N, dtype, cuda_device):
    """A step near the largest number forgets all: with log2(e) it is past fp32, and no state,
    absent ones among them, may become infinity times zero."""
    c = Case(cuda_device, 2, 1, 24, N, dtype, bias=False)
    c.delta[:] = 3e38
    c.u[:] *= 1e-38
    pool = c.state.clone()
    one = lambda x: x[:, 0]
    y = c.new(c.u)[:, 0]
    snn.snn_selective_scan_step(one(c.u), one(c.delta), c.A, one(c.Bm), one(c.Cm), pool, y, D=c.D_skip, z=one(c.z))
    args, kw = c.oracle_args()
    want, h = O.scan_forward(*args, **kw)
    size, hs = O.scan_forward(*args, positive=True, **kw)
    close("y", y, want[:, 0], size[:, 0], 160 + N)
    close("pool", pool, h, hs, 80)


def test_two_backward_passes_at_once(cuda_device):
    """On streams of their own, each with its tensor memory (of two sizes) on the same SMs."""
    cases = [Case(cuda_device, 2, 2000, 256, N, BF, seed=N) for N in (16, 64)]
    want = []
    for c in cases:
        c.forward(ckpt=True)
        want.append(c.backward())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[], []]
    for i in range(3):
        for c, s, g in zip(cases, streams, got):
            if i == 0:
                s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                g.append(c.backward())
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        for x in g:
            for name in w:
                assert torch.equal(w[name], x[name]), name
