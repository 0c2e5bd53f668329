"""Block norms on the GPU against their float64 definition.

All arithmetic is fp32.  Per element of a result rounded to type t with half
unit u_t (2^-8 bf16, 2^-11 fp16, 2^-24 fp32), on the size s of its sum of
terms: u_t |x| for the rounding and C 2^-24 s for the arithmetic.  A row's
factors come from sums of up to 8192 squares, 16 per thread and then a tree
of at most 25 additions, and from rsqrt and exp with a few units each; with
the products around them C = 64 covers a row's results.  A parameter's
gradient adds up to M rows' terms, at most M / 152 + 160 in a chain:
C = 64 + M / 152 + 160.
"""
import numpy as np
import pytest
import torch

from oracle import attn_oracle as A
from paper_2211_10725_gb300 import snn

pytestmark = pytest.mark.gpu

F32, BF, HF = torch.float32, torch.bfloat16, torch.float16
HALF_UNIT = {F32: 2.0 ** -24, BF: 2.0 ** -8, HF: 2.0 ** -11}
TINY = {F32: 0.0, BF: 0.0, HF: 2.0 ** -24}   # fp16's smallest step
EPS = 1e-5


def _np(t):
    return None if t is None else t.double().cpu().numpy()


class Case:
    def __init__(self, dev, M, N, dtype, res, group=0, gate="silu", pad=0, seed=0):
        g = torch.Generator().manual_seed(100 * seed + M + N)
        self.M, self.N, self.group, self.gate, self.dtype, self.res = M, N, group, gate, dtype, res
        self.dev = dev

        def rows(dt, scale=1.0):
            x = torch.full((M, N + pad), float("nan"), dtype=dt)
            x[:, :N] = (scale * torch.randn(M, N, generator=g)).to(dt)
            return x.to(dev)[:, :N]
        vec = lambda a, b: (a + b * torch.randn(N, generator=g)).to(dev)
        self.rows = rows
        self.r, self.a = rows(res, 2.0), rows(dtype, 0.7)
        self.z = None if gate == "none" else rows(dtype)
        self.gro, self.gy = rows(res, 0.1), rows(dtype, 0.1)
        self.w_post, self.scale, self.w_pre = vec(1.0, 0.2), vec(0.3, 0.2), vec(1.0, 0.2)

    def kw(self):
        return dict(eps=EPS, group=self.group, gate=self.gate)

    def close(self, name, got, want, size, dt, c=64.0):
        err = np.abs(_np(got) - want)
        tol = HALF_UNIT[dt] * np.abs(want) + c * 2.0 ** -24 * size + TINY[dt]
        assert (err <= tol).all(), (name, float(np.nanmax(err / tol)))

    def check_forward(self, w_post=True, scale=True):
        r2, y = self.rows(self.res), self.rows(self.dtype)
        r2.fill_(float("nan"))
        y.fill_(float("nan"))
        wp, sc = self.w_post if w_post else None, self.scale if scale else None
        snn.snn_block_norm_fwd(self.r, self.a, self.z, wp, sc, self.w_pre, r2, y, **self.kw())
        r, a, z = _np(self.r), _np(self.a), _np(self.z)
        want, wy = A.block_norm_forward(r, a, z, _np(wp), _np(sc), _np(self.w_pre), **self.kw())
        size = np.abs(r) + np.abs(want - r)
        f = A._factor(want, self.N, EPS) * np.abs(_np(self.w_pre))
        self.close("r'", r2, want, size, self.res)
        self.close("y", y, wy, size * f, self.dtype)
        return r2

    def check_backward(self, with_gy=True, with_gro=True):
        gro, gy = self.gro if with_gro else None, self.gy if with_gy else None
        new = lambda dt: torch.full((self.M, self.N), float("nan"), dtype=dt, device=self.dev)
        vec = lambda: torch.full((self.N,), float("nan"), device=self.dev)
        got = {"grad_r": new(self.res), "grad_a": new(self.dtype),
               "grad_z": None if self.z is None else new(self.dtype), "grad_w_post": vec(),
               "grad_scale": vec(), "grad_w_pre": vec()}
        ws = torch.empty(snn.snn_block_norm_workspace_bytes(self.M, self.N), dtype=torch.uint8,
                         device=self.dev)
        snn.snn_block_norm_bwd(self.r, self.a, self.z, self.w_post, self.scale, self.w_pre, gro, gy,
                               *got.values(), ws, **self.kw())
        r, a, z, o = _np(self.r), _np(self.a), _np(self.z), np.zeros((self.M, self.N))
        want = A.block_norm_backward(r, a, z, _np(self.w_post), _np(self.scale), _np(self.w_pre),
                                     _np(gro), _np(gy), **self.kw())
        # sizes: the same formulas with every term positive
        N, group, p = self.N, self.group or self.N, np.abs
        d = p(_np(gro)) if with_gro else o
        if with_gy:
            f = A._factor(r, N, EPS)
            e, gw = p(r) * f, p(_np(gy)) * p(_np(self.w_pre))
            d = d + f * (gw + e * A._mean(gw * e, N))
        f = A._factor(a, group, EPS)
        h = p(a) * f
        act, slope = A._act(z, self.gate)
        wp, sc = p(_np(self.w_post)), p(_np(self.scale))
        m = d * sc * p(act) * wp
        size = {"grad_r": d, "grad_z": d * sc * h * wp * 2.0, "grad_a": f * (m + h * A._mean(m * h, group)),
                "grad_scale": (d * h * wp * p(act)).sum(0), "grad_w_post": (d * sc * p(act) * h).sum(0)}
        for name in ("grad_r", "grad_a", "grad_z"):
            if got[name] is not None:
                self.close(name, got[name], want[name], size[name],
                           self.res if name == "grad_r" else self.dtype)
        chain = 64.0 + 160.0 + self.M / 152
        self.close("grad_scale", got["grad_scale"], want["grad_scale"], size["grad_scale"], F32, chain)
        self.close("grad_w_post", got["grad_w_post"], want["grad_w_post"], size["grad_w_post"], F32, chain)
        if with_gy:
            self.close("grad_w_pre", got["grad_w_pre"], want["grad_w_pre"],
                       (p(_np(gy)) * e).sum(0), F32, chain)
        else:
            assert torch.count_nonzero(got["grad_w_pre"]) == 0


TYPES = [(F32, F32), (BF, BF), (BF, F32), (HF, HF), (HF, F32)]


@pytest.mark.parametrize("dtype,res", TYPES)
@pytest.mark.parametrize("M,N", [(1, 8), (7, 264), (33, 1024), (5, 2048), (3, 4096), (2, 8192)])
def test_sizes(M, N, dtype, res, cuda_device):
    c = Case(cuda_device, M, N, dtype, res)
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("dtype,res", TYPES)
@pytest.mark.parametrize("M,N", [(1, 1), (4, 3), (9, 255), (5, 1001), (2, 4099), (3, 8191)])
def test_odd_sizes(M, N, dtype, res, cuda_device):
    c = Case(cuda_device, M, N, dtype, res)
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("group", [8, 16, 32, 64, 128, 256])
@pytest.mark.parametrize("N", [256, 768, 5120])
def test_groups(group, N, cuda_device):
    c = Case(cuda_device, 6, N, BF, F32, group=group)
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("gate", ["none", "sigmoid", "silu"])
def test_gates_and_absent_parameters(gate, cuda_device):
    c = Case(cuda_device, 10, 320, HF, HF, gate=gate)
    c.check_forward()
    c.check_forward(w_post=False, scale=False)
    c.check_backward()
    c.check_backward(with_gy=False)
    c.check_backward(with_gro=False)


# rows that are parts of wider ones: whole vectors apart, and not
@pytest.mark.parametrize("pad", [8, 64, 3])
@pytest.mark.parametrize("dtype,res", [(F32, F32), (BF, F32), (HF, HF)])
def test_row_strides(pad, dtype, res, cuda_device):
    c = Case(cuda_device, 12, 512, dtype, res, pad=pad)
    c.check_forward()
    c.check_backward()


def test_many_rows_and_repeatability(cuda_device):
    c = Case(cuda_device, 4001, 96, BF, BF)
    c.check_backward()
    c = Case(cuda_device, 3000, 520, F32, F32)
    c.check_forward()
    c.check_backward()
    outs = []
    for _ in range(2):
        p = [torch.empty(520, device=cuda_device) for _ in range(3)]
        ws = torch.empty(snn.snn_block_norm_workspace_bytes(3000, 520), dtype=torch.uint8, device=cuda_device)
        snn.snn_block_norm_bwd(c.r, c.a, c.z, c.w_post, c.scale, c.w_pre, c.gro, c.gy, None, None, None,
                               *p, ws, **c.kw())
        outs.append(p)
    assert all(torch.equal(x, y) for x, y in zip(*outs))


def test_norm_alone_and_last_block(cuda_device):
    c = Case(cuda_device, 9, 648, BF, F32)
    y = c.rows(BF)
    snn.snn_block_norm_fwd(c.r, None, None, None, None, c.w_pre, None, y, eps=EPS)
    want = A.block_norm_forward(_np(c.r), None, None, None, None, _np(c.w_pre), EPS)[1]
    c.close("y", y, want, np.abs(want), BF)
    gr, gw = torch.empty_like(c.r), torch.empty_like(c.w_pre)
    ws = torch.empty(snn.snn_block_norm_workspace_bytes(9, 648), dtype=torch.uint8, device=cuda_device)
    snn.snn_block_norm_bwd(c.r, None, None, None, None, c.w_pre, None, c.gy, gr, None, None, None, None,
                           gw, ws, eps=EPS)
    ref = A.block_norm_backward(_np(c.r), None, None, None, None, _np(c.w_pre), None, _np(c.gy), EPS)
    f = A._factor(_np(c.r), 648, EPS)
    g, e = np.abs(_np(c.gy) * _np(c.w_pre)), np.abs(_np(c.r)) * f
    c.close("grad_r", gr, ref["grad_r"], f * (g + e * A._mean(g * e, 648)), F32)
    c.close("grad_w_pre", gw, ref["grad_w_pre"], (np.abs(_np(c.gy)) * e).sum(0), F32, 225.0)
    # the last block: r' in place of r, no y
    want = A.block_norm_forward(_np(c.r), _np(c.a), _np(c.z), _np(c.w_post), _np(c.scale), None, **c.kw())[0]
    size = np.abs(_np(c.r)) + np.abs(want - _np(c.r))
    snn.snn_block_norm_fwd(c.r, c.a, c.z, c.w_post, c.scale, None, c.r, None, **c.kw())
    c.close("r'", c.r, want, size, F32)


def test_zero_and_extreme_rows(cuda_device):
    """A row of zeros (only eps under the root) and gates far out."""
    c = Case(cuda_device, 4, 256, F32, F32)
    c.a[0] = 0
    c.r[1] = 0
    c.z[2, ::2] = 200.0
    c.z[2, 1::2] = -200.0
    c.check_forward()
    c.check_backward()


def test_rows_past_32_bits(cuda_device):
    far = (1 << 31) + 64
    buf = torch.zeros(2 * far + 512, dtype=BF, device=cuda_device)
    c = Case(cuda_device, 3, 512, BF, F32)
    wide = buf.as_strided((3, 512), (far, 1))
    wide.copy_(c.a)
    c.a = wide
    c.check_forward()
    c.check_backward()


def test_no_rows(cuda_device):
    c = Case(cuda_device, 0, 64, BF, F32)
    c.check_forward()
    p = [torch.full((64,), float("nan"), device=cuda_device) for _ in range(3)]
    ws = torch.empty(snn.snn_block_norm_workspace_bytes(0, 64), dtype=torch.uint8, device=cuda_device)
    snn.snn_block_norm_bwd(c.r, c.a, c.z, c.w_post, c.scale, c.w_pre, c.gro, c.gy, None, None, None, *p,
                           ws, **c.kw())
    assert all(torch.count_nonzero(x) == 0 for x in p)


def test_wrapper_refusals(cuda_device):
    c = Case(cuda_device, 4, 64, BF, F32)
    r2, y = torch.empty_like(c.r), torch.empty_like(c.a)
    fwd = lambda **k: snn.snn_block_norm_fwd(**{**dict(r=c.r, a=c.a, z=c.z, w_post=c.w_post,
                                                       res_scale=c.scale, w_pre=c.w_pre, r_out=r2, y=y,
                                                       gate="silu"), **k})
    fwd()
    for bad in (dict(a=c.a[:3]), dict(z=c.z.half()), dict(w_post=c.w_post.bfloat16()),
                dict(y=y.t().contiguous().t()), dict(gate="tanh"), dict(r=c.r.double())):
        with pytest.raises(ValueError):
            fwd(**bad)
    with pytest.raises(snn.SnnError):
        fwd(gate="none")
