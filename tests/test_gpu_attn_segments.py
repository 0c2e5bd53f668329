"""Leaky attention cut into segments of several chunks, against its definition
token by token in float64 on the GPU.

The shapes are such that the library cuts the tokens, into a few segments
(whose states the blocks sum themselves) and into more (a scan does); each test
checks that from the workspace it asks for, which holds one fp32 state a
segment.  Outputs and gradients are rounded once (tolerances as in
test_gpu_attn_rounding).  A state that is an output is a sum of fp32 terms
whose weighted values keep 22 bits or more: per element 2^-16 of the sum with
all terms positive, as elsewhere, and in the 2-norm of a head 2^-18, the error
of 64 additions that all lose up to 2^-24.
"""
import numpy as np
import pytest
import torch

from oracle import attn_oracle as A
from paper_2211_10725_gb300 import snn
from tests.test_gpu_attn import BF, HF, STATE_U, Case, _close, _forward, _np
from tests.test_gpu_attn_rounding import FLOOR, rounded_once

pytestmark = pytest.mark.gpu


def definition(q, k, v, beta, do, scale, lens, S, R):
    """(o, S at the end, dq, dk, dv, dS at the start), everything float64 on one device; k and v hold
    the query heads' own copies."""
    B, T, H, _ = q.shape
    live = torch.tensor([[t < n for t in range(T)] for n in lens], device=q.device)[..., None, None, None]
    bt = beta[:, None, None]
    o, dq, dk, dv = (torch.zeros_like(x) for x in (v, q, q, v))
    for t in range(T):
        S = torch.where(live[:, t], bt * S + k[:, t, :, :, None] * v[:, t, :, None], S)
        o[:, t] = scale * (q[:, t, :, None] @ S)[:, :, 0]
        dq[:, t] = scale * (S @ do[:, t, :, :, None])[..., 0]
    for t in reversed(range(T)):
        with_t = R + scale * q[:, t, :, :, None] * do[:, t, :, None]
        dk[:, t] = (with_t @ v[:, t, :, :, None])[..., 0]
        dv[:, t] = (k[:, t, :, None] @ with_t)[:, :, 0]
        R = torch.where(live[:, t], bt * with_t, R)
    past = ~live[..., 0]
    return (o.masked_fill(past, 0), S, *(x.masked_fill(past, 0) for x in (dq, dk, dv)), R)


def of_case(c, sizes=False):
    """The definition on a case: (o, S, dq, dk, dv, dS) as numpy arrays; with sizes, every term
    positive."""
    B, T, H, Hk, Dk, Dv = c.shape
    take = lambda x: (np.abs(x) + FLOOR[c.dtype]) if sizes else x
    t = lambda x: torch.from_numpy(take(np.ascontiguousarray(x))).to(c.dev)
    q, k, v = (t(c.clean(x)) for x in (c.q, c.k, c.v))
    spread = lambda x: x.repeat_interleave(H // Hk, 2)
    pos = (lambda x: x.abs()) if sizes else (lambda x: x)
    out = definition(q, spread(k), spread(v), c.beta.double(), t(c.clean(c.do)), c.scale, c.lens or [T] * B,
                     pos(c.state.double()), pos(c.dstate.double()))
    o, S, dq, dk, dv, dS = (x.cpu().numpy() for x in out)
    shared = lambda x: x.reshape(B, T, Hk, H // Hk, -1).sum(3)
    return o, S, dq, shared(dk), shared(dv), dS


def check_state(name, got, want, size):
    _close(name, got, want, size, STATE_U)
    for h in range(want.shape[1]):
        norm = lambda x: np.linalg.norm(x[:, h])
        assert norm(_np(got) - want) <= 2.0 ** -18 * norm(want), (name, h)


def segments(c, backward):
    """Segments that the library cuts the case's tokens into, and the chunks of one.  (The plan does
    not look at Hk; with one key/value head the backward's workspace is never the smaller one.)"""
    B, T, H, _, Dk, Dv = c.shape
    tile = lambda D: 64 if D <= 64 else 128
    da, dc, roles, shares = tile(Dk), tile(Dv), 1, 0
    if backward:      # three roles in one launch, on square tiles
        da = dc = max(da, dc)
        roles = 3
        shares = sum(-(-B * T * H * D * 4 // 256) * 256 for D in (Dk, Dv))
    states = snn.snn_leaky_attn_workspace_bytes(B, T, H, 1, Dk, Dv, backward=backward) - 256 - shares
    n, rest = divmod(states, roles * B * H * da * dc * 4)
    assert rest == 0
    return n, -(-(-(-T // 64)) // max(n, 1))


def test_the_definition_is_the_oracle_s(cuda_device):
    c = Case(cuda_device, 3, 9, 4, 2, 16, 24, BF, lens=[9, 0, 5])
    args = (*c.args(), c.clean(c.do), c.scale, c.lens, _np(c.state), _np(c.dstate))
    want = (*A.attn_forward(*args[:4], *args[5:8]), *A.attn_backward(*args))
    for got, w in zip(of_case(c), want):
        assert np.abs(got - w).max() <= 1e-12 * np.abs(w).max()


WIDTHS = [(64, 64), (48, 120), (120, 48), (128, 128)]
FEW = dict(B=4, T=1300, lens=[1300, 0, 65, 1001])
MORE = dict(B=2, T=2500, lens=[2500, 1410])


@pytest.mark.parametrize("Dk,Dv", WIDTHS)
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("cut", ["few", "more"])
def test_forward(Dk, Dv, dtype, cut, cuda_device):
    s = FEW if cut == "few" else MORE
    c = Case(cuda_device, s["B"], s["T"], 24, 8, Dk, Dv, dtype, lens=s["lens"])
    n, chunks = segments(c, False)
    assert chunks >= 4 and (2 <= n <= 4 if cut == "few" else n > 4)
    want, size = of_case(c), of_case(c, sizes=True)
    o, state = _forward(c, True)
    rounded_once("o", o, want[0], size[0], dtype)
    check_state("state", state, want[1], size[1])
    for b, n in enumerate(s["lens"]):
        assert torch.count_nonzero(o[b, n:]) == 0


@pytest.mark.parametrize("Dk,Dv", WIDTHS)
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("cut,H,Hk", [("few", 8, 8), ("few", 8, 2), ("more", 6, 6), ("more", 6, 2)])
def test_backward(Dk, Dv, dtype, cut, H, Hk, cuda_device):
    s = FEW if cut == "few" else MORE
    c = Case(cuda_device, s["B"], s["T"], H, Hk, Dk, Dv, dtype, lens=s["lens"])
    n, chunks = segments(c, True)
    assert chunks >= 4 and (2 <= n <= 4 if cut == "few" else n > 4)
    want, size = of_case(c), of_case(c, sizes=True)
    grads = [c.make(H, Dk), c.make(Hk, Dk), c.make(Hk, Dv)]
    for x in grads:
        x.fill_(float("nan"))
    gin = torch.full_like(c.state, float("nan"))
    snn.snn_leaky_attn_bwd(c.q, c.k, c.v, c.beta, c.do, *grads, c.ws, scale=c.scale, seq_lens=c.seq,
                           state_in=c.state, grad_state_out=c.dstate, grad_state_in=gin)
    c.ok()
    for name, got, w, sz in zip(("grad_q", "grad_k", "grad_v"), grads, want[2:], size[2:]):
        rounded_once(name, got, w, sz, dtype)
    check_state("grad_state_in", gin, want[5], size[5])
