"""Selective scan, causal convolution and layer norm without a GPU: the float64
definitions' gradients against differences, and the library's refusals (each before
anything is launched)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import seq_oracle as O
from paper_2211_10725_gb300 import build_lib, snn

INVALID, ALIGNMENT, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4


@pytest.fixture(scope="module")
def lib():
    build_lib.build()
    return snn.load_library()


def _slope(f, x, i, step):
    old = x.flat[i]
    x.flat[i] = old + step
    hi = f()
    x.flat[i] = old - step
    lo = f()
    x.flat[i] = old
    return (hi - lo) / (2 * step)


def _differences(f, x, got, names):
    """Smooth functions: central differences err by f''' step^2 / 6 (below 1e-7
    for step 1e-4 and third derivatives below 60) and by eps |f| / step ~ 1e-10."""
    g = np.random.default_rng(3)
    for name in names:
        grad = got[name]
        for i in g.choice(grad.size, min(grad.size, 16), replace=False):
            assert abs(_slope(f, x[name], i, 1e-4) - grad.flat[i]) < 1e-6, (name, i)


@pytest.mark.parametrize("gate,softplus", [(True, True), (False, False)])
@pytest.mark.parametrize("B,T,D,G,N,lens", [(1, 1, 2, 1, 1, None), (2, 6, 4, 2, 3, [6, 2]), (3, 4, 3, 1, 2, [0, 4, 1])])
def test_scan_gradients_against_differences(B, T, D, G, N, lens, gate, softplus):
    g = np.random.default_rng(5)
    n = g.standard_normal
    x = {"u": n((B, T, D)), "delta": 0.3 + 0.5 * n((B, T, D)) ** 2, "A": -np.exp(0.3 * n((D, N))),
         "B": n((B, T, G, N)), "C": n((B, T, G, N)), "D": n(D), "z": n((B, T, D)), "bias": 0.2 * n(D),
         "state": n((B, D, N))}
    gy, gh = n((B, T, D)), n((B, D, N))
    z = lambda: x["z"] if gate else None
    kw = lambda: dict(D=x["D"], z=z(), bias=x["bias"], softplus=softplus, lens=lens, state=x["state"])

    def f():
        y, h = O.scan_forward(x["u"], x["delta"], x["A"], x["B"], x["C"], **kw())
        return (y * gy).sum() + (h * gh).sum()

    got = O.scan_backward(x["u"], x["delta"], x["A"], x["B"], x["C"], gy, gstate=gh, **kw())
    _differences(f, x, got, [k for k in x if gate or k != "z"])


@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("B,T,C,W,lens", [(1, 1, 2, 4, None), (2, 7, 3, 3, [7, 1]), (3, 5, 2, 2, [0, 5, 2])])
def test_conv_gradients_against_differences(B, T, C, W, lens, act):
    n = np.random.default_rng(6).standard_normal
    x = {"x": n((B, T, C)), "w": n((C, W)), "bias": n(C), "state": n((B, W - 1, C))}
    gy, ge = n((B, T, C)), n((B, W - 1, C))

    def f():
        y, end = O.conv_forward(x["x"], x["w"], x["bias"], act, lens, x["state"])
        return (y * gy).sum() + (end * ge).sum()

    got = O.conv_backward(x["x"], x["w"], gy, x["bias"], act, lens, x["state"], ge)
    _differences(f, x, got, x)


def test_layer_norm_gradients_against_differences():
    n = np.random.default_rng(7).standard_normal
    x = {"x": n((4, 9)), "w": n(9), "b": n(9)}
    gy = n((4, 9))
    got = O.layer_norm_backward(x["x"], x["w"], gy)
    _differences(lambda: (O.layer_norm_forward(x["x"], x["w"], x["b"]) * gy).sum(), x, got, x)


def test_descriptor_layouts(lib):
    assert lib.snn_sscan_desc_size() == ctypes.sizeof(snn.SscanDesc)
    assert lib.snn_conv_desc_size() == ctypes.sizeof(snn.ConvDesc)
    assert lib.snn_layer_norm_desc_size() == ctypes.sizeof(snn.LayerNormDesc)


# No pointer below is ever followed: every call is refused, or has nothing to do.
BIG = 1 << 50
NO = object()


def _put(d, over):
    for k, v in over.items():
        if k == "reserved0":
            d.reserved[0] = v
        else:
            setattr(d, k, v)
    return d


def _scan(**over):
    return _put(snn.SscanDesc(2, 16, 64, 16, 2, 1, 1), over)


def _s(data=16, sb=1 << 20, st=1 << 10):
    return ctypes.byref(snn.Btc(data, sb, st))


def _g(data=16, sb=1 << 20, st=1 << 10, sg=16):
    return ctypes.byref(snn.Bthd(data, sb, st, sg))


def _call(fn, names, base, d, over, tail):
    args = {**base, **over}
    return fn(ctypes.byref(d), *[None if args[n] is NO else args[n] for n in names], *tail)


SCAN_FWD = ["u", "delta", "A", "B", "C", "D", "z", "bias", "lens", "s_in", "s_out", "slots", "n", "ckpt", "y",
            "ws", "nws"]


def _scan_fwd(lib, d, **over):
    base = dict(u=_s(), delta=_s(), A=16, B=_g(), C=_g(), D=16, z=_s(), bias=16, lens=None, s_in=None,
                s_out=None, slots=None, n=2, ckpt=None, y=_s(), ws=256, nws=BIG)
    return _call(lib.snn_selective_scan_fwd, SCAN_FWD, base, d, over, [None])


BAD_SCAN = [(dict(B=-1), INVALID), (dict(T=-1), INVALID), (dict(D=0), INVALID), (dict(N=0), INVALID),
            (dict(G=0), INVALID), (dict(G=3), INVALID), (dict(dtype=3), INVALID), (dict(dtype=-1), INVALID),
            (dict(softplus=2), INVALID), (dict(reserved0=1), INVALID), (dict(N=65), UNSUPPORTED),
            (dict(T=1 << 30), UNSUPPORTED), (dict(B=1 << 30), UNSUPPORTED), (dict(D=1 << 30), UNSUPPORTED),
            (dict(B=1 << 20, T=1 << 20), UNSUPPORTED)]


@pytest.mark.parametrize("over,want", BAD_SCAN)
def test_scan_refuses_bad_descriptors(lib, over, want):
    d = _scan(**over)
    assert _scan_fwd(lib, d) == want
    if "dtype" not in over and "softplus" not in over:
        assert lib.snn_selective_scan_workspace_bytes(ctypes.byref(d), 1) == 0
        assert lib.snn_selective_scan_ckpt_elems(ctypes.byref(d)) == 0


def test_scan_forward_refusals(lib):
    d = _scan()
    for name in ("u", "delta", "B", "C", "y", "A"):
        assert _scan_fwd(lib, d, **{name: NO}) == INVALID, name
    for name in ("u", "delta", "z", "y"):
        assert _scan_fwd(lib, d, **{name: _s(data=24)}) == ALIGNMENT, name
        assert _scan_fwd(lib, d, **{name: _s(st=0)}) == INVALID, name      # a broadcast axis
        assert _scan_fwd(lib, d, **{name: _s(sb=-8)}) == INVALID, name
    for name in ("B", "C"):
        assert _scan_fwd(lib, d, **{name: _g(data=None)}) == INVALID, name
        assert _scan_fwd(lib, d, **{name: _g(data=20)}) == ALIGNMENT, name
        assert _scan_fwd(lib, d, **{name: _g(sg=0)}) == INVALID, name
    for name in ("A", "D", "bias", "lens", "s_in", "s_out", "slots", "ckpt", "ws"):
        assert _scan_fwd(lib, d, **{name: 24}) == ALIGNMENT, name
    assert _scan_fwd(lib, d, n=-1) == INVALID
    assert _scan_fwd(lib, d, s_in=16, n=1) == INVALID          # fewer places than sequences
    assert _scan_fwd(lib, _scan(B=0)) == 0
    assert _scan_fwd(lib, _scan(T=0)) == 0                     # no state to pass on


def test_scan_workspaces(lib):
    long = _scan(B=1, T=8192)
    need = lib.snn_selective_scan_workspace_bytes(ctypes.byref(long), 0)
    assert need > 256
    assert _scan_fwd(lib, long, ws=None) == WORKSPACE
    assert _scan_fwd(lib, long, nws=need - 256 if need % 256 == 0 else need - 1) == WORKSPACE
    assert lib.snn_selective_scan_workspace_bytes(ctypes.byref(long), 1) >= need
    d = _scan()
    # states before every eighth token, in twos of two channels of a group
    assert lib.snn_selective_scan_ckpt_elems(ctypes.byref(d)) == 2 * 2 * 64 * 16
    assert lib.snn_selective_scan_ckpt_elems(ctypes.byref(_scan(D=6, N=5, T=17))) == 2 * 3 * 2 * 3 * 2 * 4


SCAN_BWD = ["u", "delta", "A", "B", "C", "D", "z", "bias", "lens", "ckpt", "gy", "gs_out", "gu", "gdelta", "gA",
            "gB", "gC", "gD", "gz", "gbias", "gs_in", "ws", "nws"]


def test_scan_backward_refusals(lib):
    def bwd(d, **over):
        base = dict(u=_s(), delta=_s(), A=16, B=_g(), C=_g(), D=16, z=_s(), bias=16, lens=None, ckpt=16, gy=_s(),
                    gs_out=None, gu=_s(), gdelta=_s(), gA=16, gB=_g(), gC=_g(), gD=16, gz=_s(), gbias=16,
                    gs_in=None, ws=256, nws=BIG)
        return _call(lib.snn_selective_scan_bwd, SCAN_BWD, base, d, over, [None])
    d = _scan()
    for name in ("u", "delta", "A", "B", "C", "ckpt", "gy", "gu", "gdelta", "gA", "gB", "gC"):
        assert bwd(d, **{name: NO}) == INVALID, name
    assert bwd(d, z=NO) == INVALID                             # grad_z without z
    assert bwd(d, gz=NO) == INVALID
    assert bwd(d, gu=_s(data=8)) == ALIGNMENT
    assert bwd(d, gB=_g(st=0)) == INVALID
    for name in ("gA", "gD", "gbias", "gs_in", "gs_out", "ckpt"):
        assert bwd(d, **{name: 20}) == ALIGNMENT, name
    assert bwd(d, gs_out=64, gs_in=64) == INVALID
    need = lib.snn_selective_scan_workspace_bytes(ctypes.byref(d), 1)
    assert bwd(d, ws=None) == WORKSPACE and bwd(d, nws=need - 1) == WORKSPACE
    assert bwd(_scan(N=65)) == UNSUPPORTED


def test_scan_step_refusals(lib):
    def step(d, **over):
        names = ["u", "delta", "A", "B", "C", "D", "z", "bias", "state", "slots", "n", "y"]
        base = dict(u=_s(), delta=_s(), A=16, B=_g(), C=_g(), D=16, z=_s(), bias=16, state=16, slots=16, n=2, y=_s())
        return _call(lib.snn_selective_scan_step, names, base, d, over, [None])
    d = _scan(T=1)
    assert step(_scan()) == INVALID                            # T is not 1
    for name in ("u", "delta", "A", "B", "C", "state", "y"):
        assert step(d, **{name: NO}) == INVALID, name
    assert step(d, state=24) == ALIGNMENT
    assert step(d, n=-1) == INVALID
    assert step(d, slots=None, n=1) == INVALID
    assert step(_scan(T=1, B=70000)) == UNSUPPORTED
    assert step(_scan(T=1, B=0)) == 0


def _conv(**over):
    return _put(snn.ConvDesc(2, 16, 64, 4, 1, 2), over)


def _conv_fwd(lib, d, **over):
    names = ["x", "w", "bias", "lens", "s_in", "s_out", "slots", "n", "y"]
    base = dict(x=_s(), w=16, bias=16, lens=None, s_in=None, s_out=None, slots=None, n=2, y=_s())
    return _call(lib.snn_causal_conv_fwd, names, base, d, over, [None])


BAD_CONV = [(dict(B=-1), INVALID), (dict(T=-1), INVALID), (dict(C=0), INVALID), (dict(W=0), INVALID),
            (dict(dtype=3), INVALID), (dict(act=3), INVALID), (dict(reserved0=1), INVALID),
            (dict(act=1), UNSUPPORTED), (dict(W=1), UNSUPPORTED), (dict(W=5), UNSUPPORTED),
            (dict(T=1 << 30), UNSUPPORTED), (dict(B=1 << 20, T=1 << 20), UNSUPPORTED)]


@pytest.mark.parametrize("over,want", BAD_CONV)
def test_conv_refuses_bad_descriptors(lib, over, want):
    d = _conv(**over)
    assert _conv_fwd(lib, d) == want
    assert lib.snn_causal_conv_workspace_bytes(ctypes.byref(d)) == 0


def test_conv_refusals(lib):
    d = _conv()
    for name in ("x", "w", "y"):
        assert _conv_fwd(lib, d, **{name: NO}) == INVALID, name
    assert _conv_fwd(lib, d, x=_s(data=8)) == ALIGNMENT
    assert _conv_fwd(lib, d, y=_s(st=0)) == INVALID
    for name in ("w", "bias", "lens", "s_in", "s_out", "slots"):
        assert _conv_fwd(lib, d, **{name: 24}) == ALIGNMENT, name
    assert _conv_fwd(lib, d, n=-1) == INVALID
    assert _conv_fwd(lib, d, s_out=16, n=1) == INVALID
    assert _conv_fwd(lib, _conv(B=0)) == 0 and _conv_fwd(lib, _conv(T=0)) == 0

    def bwd(d, **over):
        names = ["x", "w", "bias", "lens", "s_in", "gy", "gs_out", "gx", "gw", "gb", "gs_in", "ws", "nws"]
        base = dict(x=_s(), w=16, bias=16, lens=None, s_in=None, gy=_s(), gs_out=None, gx=_s(), gw=16, gb=16,
                    gs_in=None, ws=256, nws=BIG)
        return _call(lib.snn_causal_conv_bwd, names, base, d, over, [None])
    for name in ("x", "w", "gy"):
        assert bwd(d, **{name: NO}) == INVALID, name
    assert bwd(d, gx=_s(data=8)) == ALIGNMENT and bwd(d, gw=20) == ALIGNMENT
    assert bwd(d, gs_in=64, s_in=64) == INVALID and bwd(d, gs_in=64, gs_out=64) == INVALID
    need = lib.snn_causal_conv_workspace_bytes(ctypes.byref(d))
    assert bwd(d, ws=None) == WORKSPACE and bwd(d, nws=need - 1) == WORKSPACE

    def step(d, **over):
        names = ["x", "w", "bias", "state", "slots", "n", "y"]
        base = dict(x=_s(), w=16, bias=16, state=16, slots=16, n=2, y=_s())
        return _call(lib.snn_causal_conv_step, names, base, d, over, [None])
    assert step(d) == INVALID
    assert step(_conv(T=1), state=NO) == INVALID
    assert step(_conv(T=1), slots=None, n=1) == INVALID
    assert step(_conv(T=1, B=0)) == 0


def _ln(**over):
    return _put(snn.LayerNormDesc(4, 256, 1, 0, 1e-5), over)


def _r(data=16, ld=256):
    return ctypes.byref(snn.Rows(data, ld))


def _ln_fwd(lib, d, **over):
    base = dict(x=_r(), w=16, b=16, y=_r(), stats=16)
    return _call(lib.snn_layer_norm_fwd, ["x", "w", "b", "y", "stats"], base, d, over, [None])


@pytest.mark.parametrize("over,want", [
    (dict(M=-1), INVALID), (dict(N=0), INVALID), (dict(dtype=3), INVALID), (dict(res_dtype=-1), INVALID),
    (dict(eps=0.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(reserved=1), INVALID),
    (dict(N=8200), UNSUPPORTED), (dict(dtype=0, res_dtype=1), UNSUPPORTED), (dict(dtype=2, res_dtype=1), UNSUPPORTED)])
def test_layer_norm_refuses_bad_descriptors(lib, over, want):
    assert _ln_fwd(lib, _ln(**over)) == want


def test_layer_norm_refusals(lib):
    d = _ln()
    assert _ln_fwd(lib, d, x=NO) == INVALID and _ln_fwd(lib, d, y=NO) == INVALID
    assert _ln_fwd(lib, d, x=_r(data=8)) == ALIGNMENT and _ln_fwd(lib, d, stats=20) == ALIGNMENT
    assert _ln_fwd(lib, d, y=_r(ld=255)) == INVALID
    assert _ln_fwd(lib, _ln(M=0)) == 0

    def bwd(d, **over):
        base = dict(x=_r(), w=16, stats=16, gy=_r(), gx=_r(), gw=16, gb=16, ws=256, nws=BIG)
        return _call(lib.snn_layer_norm_bwd, list(base), base, d, over, [None])
    for name in ("x", "stats", "gy"):
        assert bwd(d, **{name: NO}) == INVALID, name
    assert bwd(d, gx=_r(ld=4)) == INVALID and bwd(d, gb=8) == ALIGNMENT
    assert bwd(d, ws=None) == WORKSPACE and bwd(d, nws=8) == WORKSPACE
    assert lib.snn_layer_norm_workspace_bytes(4, 8200) == 0


@pytest.mark.parametrize("call", [
    lambda x, f: snn.snn_selective_scan_fwd(x, x, f, x[:, :, None], x[:, :, None], x, f),
    lambda x, f: snn.snn_causal_conv_fwd(x, f, None, x),
    lambda x, f: snn.snn_layer_norm_fwd(x[0], None, None, x[0])])
def test_the_binding_refuses_tensors_of_the_host(call):
    with pytest.raises(ValueError, match="current CUDA device"):
        call(torch.zeros(2, 3, 4), torch.zeros(4, 4))
