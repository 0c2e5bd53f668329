"""The gates of fp32 block norms keep fp32's relative accuracy far out.

With r = 0 the stream after the block is s n act(z) alone, so every element is
a product: in units of 2^-24, expf takes 4, 1 + p and its reciprocal one each,
z act one, the factor 1/rms 12 (a sum of 256 squares, eps, rsqrt), the other
products one each: below 32, and fp32's smallest step 2^-149 for a result
below 2^-126.  (A product z log2(e) rounded to fp32 before the
power of two would alone take up to 44 at |z| of 64 to 87.)"""
import numpy as np
import pytest
import torch

from oracle import attn_oracle as A
from paper_2211_10725_gb300 import snn
from tests.test_gpu_block_norm import EPS, F32, Case, _np

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("gate", ["sigmoid", "silu"])
@pytest.mark.parametrize("N", [256, 255])
@pytest.mark.parametrize("z", [(-87.0, -64.0), (-64.0, -20.0), (-20.0, 20.0), (20.0, 200.0)])
def test_gates_far_out(gate, N, z, cuda_device):
    c = Case(cuda_device, 40, N, F32, F32, gate=gate)
    c.r.zero_()
    c.z.copy_(z[0] + (z[1] - z[0]) * torch.rand(40, N, generator=torch.Generator().manual_seed(1)))
    close = lambda got, want: (np.abs(_np(got) - want) <= 32 * 2.0 ** -24 * np.abs(want) + 2.0 ** -149).all()
    r2 = torch.empty_like(c.r)
    snn.snn_block_norm_fwd(c.r, c.a, c.z, c.w_post, c.scale, None, r2, None, **c.kw())
    args = [_np(t) for t in (c.a, c.z, c.w_post, c.scale)]
    assert close(r2, A.block_norm_forward(_np(c.r), *args, None, **c.kw())[0])
    gz = torch.empty_like(c.z)
    snn.snn_block_norm_bwd(c.r, c.a, c.z, c.w_post, c.scale, None, c.gro, None, None, None, gz, None, None,
                           None, None, **c.kw())
    want = A.block_norm_backward(_np(c.r), *args, None, _np(c.gro), None, **c.kw())["grad_z"]
    if z[1] <= -20.0 or z[0] < 0.0:       # (past 20 the slope of the sigmoid is 1 - s, a difference)
        keep = _np(c.z) < -2.0            # (and near the silu's minimum the slope is one)
        assert close(torch.from_numpy(np.where(keep, _np(gz), 0.0)), np.where(keep, want, 0.0))
