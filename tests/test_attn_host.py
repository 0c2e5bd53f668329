"""Leaky attention and block norms without a GPU: the float64 definitions'
gradients against differences, and the library's refusals (each before
anything is launched)."""
import ctypes

import numpy as np
import pytest

from oracle import attn_oracle as A
from paper_2211_10725_gb300 import build_lib, snn

INVALID, ALIGNMENT, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4


@pytest.fixture(scope="module")
def lib():
    build_lib.build()
    return snn.load_library()


def _slope(f, x, i, step):
    """Central difference of f in element i of x."""
    old = x.flat[i]
    x.flat[i] = old + step
    hi = f()
    x.flat[i] = old - step
    lo = f()
    x.flat[i] = old
    return (hi - lo) / (2 * step)


# <o, do> + <S_out, dS> is linear in q and v and in k for the others fixed, so
# central differences are exact up to rounding: |f| eps / step with |f| < 1e3
# and step 0.5 is below 1e-12 of the sums' size.
@pytest.mark.parametrize("B,T,H,Hk,Dk,Dv,lens", [(1, 1, 1, 1, 8, 8, None), (2, 7, 4, 2, 8, 16, [7, 3]),
                                                 (3, 5, 2, 1, 16, 8, [0, 5, 1])])
def test_attention_gradients_against_differences(B, T, H, Hk, Dk, Dv, lens):
    g = np.random.default_rng(5)
    x = {"q": g.standard_normal((B, T, H, Dk)), "k": g.standard_normal((B, T, Hk, Dk)),
         "v": g.standard_normal((B, T, Hk, Dv)), "S": g.standard_normal((B, H, Dk, Dv))}
    do, dS = g.standard_normal((B, T, H, Dv)), g.standard_normal((B, H, Dk, Dv))
    beta = np.linspace(0.0, 1.0, H + 1)[1:]
    scale = 0.7

    def f():
        o, S = A.attn_forward(x["q"], x["k"], x["v"], beta, scale, lens, x["S"])
        return (o * do).sum() + (S * dS).sum()

    got = dict(zip("qkvS", A.attn_backward(x["q"], x["k"], x["v"], beta, do, scale, lens, x["S"], dS)))
    for name, grad in got.items():
        for i in g.choice(grad.size, min(grad.size, 24), replace=False):
            assert abs(_slope(f, x[name], i, 0.5) - grad.flat[i]) < 1e-9, (name, i)


# the norms are smooth: central differences err by f''' step^2 / 6 (below
# 1e-7 for step 1e-4 and derivatives below 50) and by eps |f| / step ~ 1e-10
@pytest.mark.parametrize("gate", ["none", "sigmoid", "silu"])
@pytest.mark.parametrize("group", [0, 4])
def test_norm_gradients_against_differences(gate, group):
    g = np.random.default_rng(6)
    M, N, eps = 3, 8, 1e-5
    x = {"r": g.standard_normal((M, N)), "a": g.standard_normal((M, N)),
         "z": g.standard_normal((M, N)), "w_post": g.standard_normal(N),
         "scale": g.standard_normal(N), "w_pre": g.standard_normal(N)}
    gro, gy = g.standard_normal((M, N)), g.standard_normal((M, N))
    z = lambda: None if gate == "none" else x["z"]

    def f():
        r2, y = A.block_norm_forward(x["r"], x["a"], z(), x["w_post"], x["scale"], x["w_pre"], eps,
                                     group, gate)
        return (r2 * gro).sum() + (y * gy).sum()

    r2, _ = A.block_norm_forward(x["r"], x["a"], z(), x["w_post"], x["scale"], x["w_pre"], eps,
                                 group, gate)
    got = A.block_norm_backward(r2, x["a"], z(), x["w_post"], x["scale"], x["w_pre"], gro, gy, eps,
                                group, gate)
    for name, grad in got.items():
        for i in range(grad.size):
            assert abs(_slope(f, x[name[5:]], i, 1e-4) - grad.flat[i]) < 1e-6, (name, i)


def test_descriptor_layouts(lib):
    assert lib.snn_attn_desc_size() == ctypes.sizeof(snn.AttnDesc)
    assert lib.snn_norm_desc_size() == ctypes.sizeof(snn.NormDesc)


def _attn(**over):
    d = snn.AttnDesc(2, 16, 4, 2, 64, 32, 1, 1.0)
    for k, v in over.items():
        setattr(d, k, v)
    return d


def _t(data=16, sb=1 << 20, st=1 << 12, sh=128):
    return ctypes.byref(snn.Bthd(data, sb, st, sh))


BIG = 1 << 40


def _fwd(lib, d, q=None, k=None, v=None, o=None, beta=16, lens=None, s_in=None, s_out=None,
         slots=None, n=0, ws=256, nws=BIG):
    return lib.snn_leaky_attn_fwd(ctypes.byref(d), q or _t(), k or _t(), v or _t(), beta, lens,
                                  s_in, s_out, slots, n, o or _t(), ws, nws, None)


BAD_ATTN = [(dict(B=-1), INVALID), (dict(T=-1), INVALID), (dict(H=0), INVALID),
            (dict(Hk=3), INVALID), (dict(Hk=0), INVALID), (dict(Dk=0), INVALID),
            (dict(dtype=3), INVALID), (dict(scale=float("nan")), INVALID),
            (dict(scale=float("inf")), INVALID), (dict(dtype=0), UNSUPPORTED),
            (dict(Dk=12), UNSUPPORTED), (dict(Dv=136), UNSUPPORTED), (dict(T=1 << 31), UNSUPPORTED),
            (dict(B=1 << 29), UNSUPPORTED)]


@pytest.mark.parametrize("over,want", BAD_ATTN)
def test_attention_refuses_bad_descriptors(lib, over, want):
    d = _attn(**over)
    assert lib.snn_leaky_attn_workspace_bytes(ctypes.byref(d), 1) == 0
    assert _fwd(lib, d) == want
    d.T = 1 if d.T == 16 else d.T
    assert lib.snn_leaky_attn_step(ctypes.byref(d), _t(), _t(), _t(), 16, 16, None, 2, _t(),
                                   None) == want


def test_attention_refuses_reserved_bits(lib):
    d = _attn()
    d.reserved[1] = 1
    assert _fwd(lib, d) == INVALID


def test_attention_forward_refusals(lib):
    d = _attn()
    assert _fwd(lib, d, q=_t(data=None)) == INVALID
    assert _fwd(lib, d, k=_t(data=24)) == ALIGNMENT
    assert _fwd(lib, d, v=_t(st=12)) == ALIGNMENT
    assert _fwd(lib, d, o=_t(sh=4)) == ALIGNMENT
    assert _fwd(lib, d, q=_t(sb=0)) == INVALID         # a broadcast batch
    assert _fwd(lib, d, q=_t(st=-8)) == INVALID
    assert _fwd(lib, d, beta=None) == INVALID
    for name in ("beta", "lens", "s_in", "s_out", "slots"):
        assert _fwd(lib, d, **{name: 20}) == ALIGNMENT, name
    assert _fwd(lib, d, slots=16, n=-1) == INVALID
    assert _fwd(lib, d, ws=None) == WORKSPACE
    assert _fwd(lib, d, nws=0) == WORKSPACE
    assert lib.snn_leaky_attn_fwd(ctypes.byref(d), None, _t(), _t(), 16, None, None, None, None, 0,
                                  _t(), 256, BIG, None) == INVALID


def test_attention_accepts_an_empty_batch(lib):
    assert _fwd(lib, _attn(B=0)) == 0


def test_attention_backward_refusals(lib):
    def bwd(d, grad_k=None, s_in=None, gs_out=None, gs_in=None, beta=16, nws=BIG):
        return lib.snn_leaky_attn_bwd(ctypes.byref(d), _t(), _t(), _t(), beta, None, s_in, _t(),
                                      gs_out, _t(), grad_k or _t(), _t(), gs_in, 256, nws, None)
    d = _attn()
    assert bwd(_attn(scale=0.0)) == INVALID
    assert bwd(d, grad_k=_t(data=None)) == INVALID
    assert bwd(d, grad_k=_t(st=20)) == ALIGNMENT
    assert bwd(d, beta=None) == INVALID
    assert bwd(d, s_in=8) == ALIGNMENT
    assert bwd(d, gs_out=64, gs_in=64) == INVALID
    need = lib.snn_leaky_attn_workspace_bytes(ctypes.byref(d), 1)
    assert need > 0 and bwd(d, nws=need - 1) == WORKSPACE


def test_attention_step_refusals(lib):
    def step(d, q=None, beta=16, state=16, slots=16, n=2):
        return lib.snn_leaky_attn_step(ctypes.byref(d), q or _t(), _t(), _t(), beta, state, slots,
                                       n, _t(), None)
    assert step(_attn()) == INVALID                       # T is not 1
    d = _attn(T=1)
    assert step(d, q=_t(data=None)) == INVALID
    assert step(d, q=_t(sh=4)) == ALIGNMENT
    assert step(d, beta=None) == INVALID
    assert step(d, state=None) == INVALID
    assert step(d, state=24) == ALIGNMENT
    assert step(d, n=-1) == INVALID
    assert step(d, slots=None, n=1) == INVALID            # fewer places than sequences
    assert step(_attn(T=1, B=0)) == 0


def _norm(**over):
    d = snn.NormDesc(4, 256, 0, 1, 0, 2, 1e-6)
    for k, v in over.items():
        setattr(d, k, v)
    return d


def _r(data=16, ld=256):
    return ctypes.byref(snn.Rows(data, ld))


NO = object()


def _nfwd(lib, d, **over):
    names = ["r", "a", "z", "w_post", "res_scale", "w_pre", "r_out", "y"]
    base = dict(r=_r(), a=_r(), z=_r(), w_post=16, res_scale=16, w_pre=16, r_out=_r(), y=_r())
    base.update({k: None if v is NO else v for k, v in over.items()})
    return lib.snn_block_norm_fwd(ctypes.byref(d), *[base[n] for n in names], None)


BAD_NORM = [(dict(M=-1), INVALID), (dict(N=0), INVALID), (dict(group=-8), INVALID),
            (dict(group=48), INVALID), (dict(dtype=3), INVALID), (dict(res_dtype=-1), INVALID),
            (dict(gate=3), INVALID), (dict(eps=0.0), INVALID), (dict(eps=float("nan")), INVALID),
            (dict(N=8200), UNSUPPORTED), (dict(dtype=0, res_dtype=1), UNSUPPORTED),
            (dict(dtype=2, res_dtype=1), UNSUPPORTED), (dict(group=4), UNSUPPORTED),
            (dict(N=1536, group=512), UNSUPPORTED), (dict(N=192, group=96), UNSUPPORTED)]


@pytest.mark.parametrize("over,want", BAD_NORM)
def test_norm_refuses_bad_descriptors(lib, over, want):
    assert _nfwd(lib, _norm(**over)) == want


def test_norm_forward_refusals(lib):
    d = _norm()
    assert _nfwd(lib, d, r=NO) == INVALID
    assert _nfwd(lib, d, r_out=NO) == INVALID          # a without r'
    assert _nfwd(lib, d, a=NO) == INVALID              # r' without a
    assert _nfwd(lib, d, y=NO) == INVALID
    assert _nfwd(lib, d, w_pre=NO) == INVALID
    assert _nfwd(lib, d, z=NO) == INVALID
    assert _nfwd(lib, _norm(gate=0)) == INVALID        # a gate that is not used
    assert _nfwd(lib, d, a=_r(data=24)) == ALIGNMENT
    assert _nfwd(lib, d, w_post=20) == ALIGNMENT
    assert _nfwd(lib, d, y=_r(ld=255)) == INVALID
    # rows that are not whole vectors: only the whole row as a group
    assert _nfwd(lib, _norm(group=64), z=_r(ld=257)) == UNSUPPORTED
    assert _nfwd(lib, _norm(M=0)) == 0


def test_norm_backward_refusals(lib):
    names = ["r_out", "a", "z", "w_post", "res_scale", "w_pre", "grad_r_out", "grad_y", "grad_r",
             "grad_a", "grad_z", "grad_w_post", "grad_scale", "grad_w_pre", "ws"]

    def bwd(d, nws=BIG, **over):
        base = dict(r_out=_r(), a=_r(), z=_r(), w_post=16, res_scale=16, w_pre=16, grad_r_out=_r(),
                    grad_y=_r(), grad_r=_r(), grad_a=_r(), grad_z=_r(), grad_w_post=16,
                    grad_scale=16, grad_w_pre=16, ws=256)
        base.update({k: None if v is NO else v for k, v in over.items()})
        return lib.snn_block_norm_bwd(ctypes.byref(d), *[base[n] for n in names], nws, None)
    d = _norm()
    assert bwd(d, grad_y=NO, grad_r_out=NO) == INVALID
    assert bwd(d, w_pre=NO) == INVALID                 # grad_y without w_pre
    assert bwd(d, r_out=NO) == INVALID
    assert bwd(d, z=NO) == INVALID
    assert bwd(d, a=NO, z=NO) == INVALID               # gradients of an absent block
    assert bwd(_norm(gate=0), z=NO) == INVALID         # grad_z without z
    assert bwd(d, grad_a=_r(data=8)) == ALIGNMENT
    assert bwd(d, grad_scale=4) == ALIGNMENT
    assert bwd(d, ws=NO) == WORKSPACE
    assert bwd(d, nws=64) == WORKSPACE
    assert bwd(_norm(res_dtype=2)) == UNSUPPORTED
    assert lib.snn_block_norm_workspace_bytes(4, 8200) == 0


def test_attention_backward_refuses_a_state_written_while_it_is_read(lib):
    d = _attn()
    call = lambda s_in, gs_out, gs_in: lib.snn_leaky_attn_bwd(
        ctypes.byref(d), _t(), _t(), _t(), 16, None, s_in, _t(), gs_out, _t(), _t(), _t(), gs_in, 256,
        BIG, None)
    assert call(64, None, 64) == INVALID
    assert call(None, 64, 64) == INVALID


class _Library:
    """Keeps what the binding hands to a call."""

    def __init__(self):
        self.seen = []

    def __getattr__(self, name):
        def call(desc, *args):
            d = desc._obj
            self.seen.append(d.scale if isinstance(d, snn.AttnDesc) else d.eps)
            return 0
        return call


def test_a_scale_or_eps_that_is_a_tensor_is_read_at_each_call(monkeypatch):
    """A learned or scheduled scalar, changed in place between calls."""
    import torch
    lib = _Library()
    monkeypatch.setattr(snn, "load_library", lambda: lib)
    monkeypatch.setattr(snn, "_bthd", lambda *a: (16, 8, 8, 8))
    monkeypatch.setattr(snn, "_rows", lambda *a: (16, 8))
    monkeypatch.setattr(snn, "_flat", lambda *a: 16)
    monkeypatch.setattr(snn, "_stream", lambda s: None)
    x, ws = torch.zeros(1, 1, 1, 8, dtype=torch.bfloat16), torch.zeros(256, dtype=torch.uint8)
    row, value = torch.zeros(1, 8), torch.tensor(0.5)
    calls = [lambda: snn.snn_leaky_attn_fwd(x, x, x, None, x, ws, scale=value),
             lambda: snn.snn_leaky_attn_bwd(x, x, x, None, x, x, x, x, ws, scale=value),
             lambda: snn.snn_leaky_attn_step(x[0], x[0], x[0], None, x, x[0], scale=value),
             lambda: snn.snn_block_norm_fwd(row, None, None, None, None, None, None, row, eps=value),
             lambda: snn.snn_block_norm_bwd(row, None, None, None, None, None, row, None, row, None, None, None,
                                            None, None, ws, eps=value)]
    for call in calls:
        for want in (0.5, 0.25):
            value.fill_(want)
            call()
            assert lib.seen[-1] == want


@pytest.mark.parametrize("scale", [1e-40, -1e-40, 2.0 ** -127, 2.0 ** 127, -2.0 ** 127])
def test_attention_backward_refuses_a_scale_without_a_reciprocal(lib, scale):
    """The gradient of the end state is divided by it: infinite below 2^-126, short of bits above
    2^126."""
    d = _attn(scale=scale)
    assert lib.snn_leaky_attn_bwd(ctypes.byref(d), _t(), _t(), _t(), 16, None, None, _t(), 64, _t(), _t(), _t(),
                                  None, 256, BIG, None) == INVALID
    assert _fwd(lib, d, ws=None) == WORKSPACE      # the forward takes it
