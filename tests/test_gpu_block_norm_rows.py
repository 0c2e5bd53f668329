"""Block norms over many rows, where blocks take several each and the rows of
any length and alignment are staged ahead (tolerances as in
test_gpu_block_norm)."""
import pytest
import torch

from tests.test_gpu_block_norm import BF, F32, HF, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,res", [(F32, F32), (BF, F32), (HF, HF)])
@pytest.mark.parametrize("M,N", [(5001, 33), (5000, 255), (1300, 257), (1300, 511), (1300, 1001),
                                 (1000, 2047), (700, 4095), (500, 5003)])
def test_odd_rows_in_turn(M, N, dtype, res, cuda_device):
    c = Case(cuda_device, M, N, dtype, res)
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("dtype,res", [(F32, F32), (BF, F32), (HF, HF)])
@pytest.mark.parametrize("M,N", [(5001, 64), (1300, 512), (1300, 1000), (1000, 2048), (700, 4096), (500, 8192)])
def test_whole_vectors_in_turn(M, N, dtype, res, cuda_device):
    c = Case(cuda_device, M, N, dtype, res, group=64 if N % 64 == 0 else 0)
    c.check_forward()
    c.check_backward()
    c.check_backward(with_gy=False)
    c.check_backward(with_gro=False)


def _shift(t, by):
    """The same values at an address `by` bytes past a 256-byte boundary."""
    M, N = t.shape
    buf = torch.zeros(M * N + 64, dtype=t.dtype, device=t.device)
    n = by // t.element_size()
    at = buf[n:n + M * N].view(M, N)
    at.copy_(t)
    assert at.data_ptr() % 256 == by
    return at


@pytest.mark.parametrize("N,group", [(768, 128), (8192, 0), (1001, 0)])
def test_matrices_between_32_byte_boundaries(N, group, cuda_device):
    c = Case(cuda_device, 400, N, F32, F32, group=group)
    for name in ("r", "a", "z", "gro", "gy"):
        setattr(c, name, _shift(getattr(c, name), 16))
    c.check_forward()
    c.check_backward()


def test_in_place_gradients_and_stream(cuda_device):
    from paper_2211_10725_gb300 import snn
    c = Case(cuda_device, 900, 333, F32, F32)
    ws = torch.empty(snn.snn_block_norm_workspace_bytes(900, 333), dtype=torch.uint8, device=cuda_device)
    outs = []
    for same in (False, True):
        gro, gy, r, a = c.gro.clone(), c.gy.clone(), c.r.clone(), c.a.clone()
        gr = gro if same else torch.empty_like(gro)
        ga = gy if same else torch.empty_like(gy)
        gz, p = torch.empty_like(c.z), [torch.empty(333, device=cuda_device) for _ in range(3)]
        snn.snn_block_norm_bwd(r, a, c.z, c.w_post, c.scale, c.w_pre, gro, gy, gr, ga, gz, *p, ws, **c.kw())
        r_out = r if same else torch.empty_like(r)
        y = torch.empty_like(a)
        snn.snn_block_norm_fwd(r, a, c.z, c.w_post, c.scale, c.w_pre, r_out, y, **c.kw())
        outs.append((gr, ga, gz, *p, r_out, y))
    assert all(torch.equal(x, y) for x, y in zip(*outs))
