"""Leaky attention's outputs and gradients are rounded to 16 bits once.

Against the float64 definition, per element, with A the sum with all terms
positive: u |o| for the output's own rounding (u = 2^-8 bf16, 2^-11 fp16) and
c A for everything before it.  Operands of the products are two 16-bit parts,
each residual rounded: 2^-16 of a term in bf16 for the weighted score, the
state's copy, the weighted value and its weight, and the fp32 sums of up to a
few hundred terms, 400 * 2^-24 < 2^-15: together 4 * 2^-16 + 2^-15 < c = 2^-13.
In fp16 the parts carry 2^-22 and c = 2^-14 is the sums' with as much again;
weighted values there are kept to 2^-25, as if every |v| were 2^-9 larger
(2^-25 = 2^-16 * 2^-9 < c 2^-9), and outputs to fp16's smallest step 2^-24.

In the 2-norm of a head such errors are independent, below 2^-13 of the
result, so the error is at most a tenth more than that of the exact result
rounded once, and 2^-13 of the result.
"""
import numpy as np
import pytest
import torch

from oracle import attn_oracle as A
from paper_2211_10725_gb300 import snn
from tests.test_gpu_attn import BF, HF, Case, _forward, _np

pytestmark = pytest.mark.gpu

UNIT = {BF: 2.0 ** -8, HF: 2.0 ** -11}
ARITHMETIC = {BF: 2.0 ** -13, HF: 2.0 ** -14}
STEP = {BF: 0.0, HF: 2.0 ** -24}
FLOOR = {BF: 0.0, HF: 2.0 ** -9}


def rounded_once(name, got, want, size, dtype):
    got = _np(got)
    tol = UNIT[dtype] * np.abs(want) + ARITHMETIC[dtype] * size + STEP[dtype] + 1e-30
    # a result past fp16's range is infinite (from 65520 on by rounding to nearest)
    past = np.isinf(got) & (dtype == HF) & (np.abs(want) + tol >= 65520.0) & (np.sign(got) == np.sign(want))
    err = np.where(past, 0.0, np.abs(np.where(past, want, got) - want))
    assert (err <= tol).all(), (name, float(np.nanmax(err / tol)))
    once = np.where(past, 0.0, torch.from_numpy(want).to(dtype).double().numpy() - want)
    once[np.isinf(once)] = 0.0
    for h in range(want.shape[2]):
        norm = lambda x: np.linalg.norm(x[:, :, h])
        most = 1.1 * norm(once) + 2.0 ** -13 * norm(want) + STEP[dtype] * want[:, :, h].size ** 0.5
        assert norm(err) <= most, (name, h, norm(err) / most)


def check(c, with_state):
    """Outputs and gradients of the case, each rounded once."""
    B, T, H, Hk, Dk, Dv = c.shape
    o, _ = _forward(c, with_state)
    st, ds = (_np(c.state), _np(c.dstate)) if with_state else (None, None)
    q, k, v, beta = c.args()
    do = c.clean(c.do)
    up = lambda x: np.abs(x) + FLOOR[c.dtype]
    rounded_once("o", o, A.attn_forward(q, k, v, beta, c.scale, c.lens, st)[0],
                 A.attn_forward_size(up(q), up(k), up(v), beta, c.scale, c.lens, st)[0], c.dtype)
    grads = [c.make(H, Dk), c.make(Hk, Dk), c.make(Hk, Dv)]
    snn.snn_leaky_attn_bwd(c.q, c.k, c.v, c.beta, c.do, *grads, c.ws, scale=c.scale, seq_lens=c.seq,
                           state_in=c.state if with_state else None,
                           grad_state_out=c.dstate if with_state else None)
    c.ok()
    want = A.attn_backward(q, k, v, beta, do, c.scale, c.lens, st, ds)
    size = A.attn_backward_size(up(q), up(k), up(v), beta, up(do), c.scale, c.lens, st, ds)
    for name, g, w, s in zip(("grad_q", "grad_k", "grad_v"), grads, want, size):
        rounded_once(name, g, w, s, c.dtype)


# one chunk from no state: the weighted scores are all there is
@pytest.mark.parametrize("T", [1, 2, 12, 40, 64])
@pytest.mark.parametrize("H,Hk,Dk,Dv", [(8, 8, 104, 120), (4, 2, 64, 64), (3, 3, 40, 72), (3, 1, 128, 48)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_one_chunk(T, H, Hk, Dk, Dv, dtype, cuda_device):
    check(Case(cuda_device, 5, T, H, Hk, Dk, Dv, dtype), False)


# from a state and over several chunks: what the state adds is rounded once as well
@pytest.mark.parametrize("T", [1, 65, 200, 700])
@pytest.mark.parametrize("H,Hk,Dk,Dv", [(6, 6, 128, 128), (4, 2, 64, 64), (6, 3, 40, 72), (3, 1, 128, 48)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_states(T, H, Hk, Dk, Dv, dtype, cuda_device):
    check(Case(cuda_device, 2, T, H, Hk, Dk, Dv, dtype), True)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_ragged(dtype, cuda_device):
    check(Case(cuda_device, 4, 300, 6, 2, 96, 120, dtype, lens=[300, 0, 1, 131]), True)


# Scores of about 6e3, 2e4 and 4e5 (times 4 and more in the tail) where fp16 ends at 65504, in the
# forward's roles (q, k large) and in those of grad_q and grad_k (grad_o, v large); the other two
# factors keep the results in its range, but for a few of the head without decay.
@pytest.mark.parametrize("gain", [2.0 ** 5, 2.0 ** 6, 2.0 ** 8])
@pytest.mark.parametrize("large", ["qk", "ov"])
@pytest.mark.parametrize("H,Hk,Dk,Dv", [(2, 2, 128, 128), (2, 1, 64, 64), (2, 2, 48, 120), (2, 2, 104, 64)])
def test_fp16_scores_past_its_range(gain, large, H, Hk, Dk, Dv, cuda_device):
    c = Case(cuda_device, 2, 150, H, Hk, Dk, Dv, HF)
    for x, big in ((c.q, "qk"), (c.k, "qk"), (c.v, "ov"), (c.do, "ov")):
        x.mul_(gain if big == large else 4.0 / gain)
    check(c, False)


# A state far above the scores, which are tiny or nothing: the scaling that keeps them is bounded.
@pytest.mark.parametrize("small", [0.0, 2.0 ** -10])
def test_fp16_scores_far_below_the_state(small, cuda_device):
    c = Case(cuda_device, 2, 150, 2, 2, 128, 64, HF)
    c.k.mul_(small)
    c.state.mul_(2.0 ** 8)
    check(c, True)


# Values and gradients near fp16's smallest, as those of a mean over many tokens are: what a decayed
# value keeps in the state goes by the chunk's largest, not by fp16's last bit.
@pytest.mark.parametrize("T", [150, 1300])
@pytest.mark.parametrize("H,Hk,Dk,Dv", [(2, 2, 128, 128), (2, 1, 64, 64), (2, 2, 48, 120), (2, 2, 104, 64)])
def test_fp16_small_values(T, H, Hk, Dk, Dv, cuda_device):
    c = Case(cuda_device, 2, T, H, Hk, Dk, Dv, HF)
    for x in (c.q, c.k):
        x.mul_(16.0)
    for x in (c.v, c.do):
        x.mul_(2.0 ** -16)
    check(c, False)
