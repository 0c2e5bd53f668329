"""Leaky attention on the GPU against its float64 definition.

Tolerances, per element, on the size A of its sum (the sum with all terms
positive), with u = 2^-8 for bf16 and for the state operand of fp16 products
(which is rounded to bf16 for its range), 2^-11 for other fp16 values:
- an output takes at most four roundings to 16 bits per term (weighted score,
  or query, key-value product and state) and its own: 4u A + u |o|, here 5u A;
- a gradient of a shared head is the sum of such;
- a state is a sum of fp32 products whose weighted values keep 16 bits or
  more (two 16-bit parts): 2^-16 A covers them and the fp32 additions.
"""
import numpy as np
import pytest
import torch

from oracle import attn_oracle as A
from paper_2211_10725_gb300 import snn

pytestmark = pytest.mark.gpu

BF, HF = torch.bfloat16, torch.float16
U = 2.0 ** -8
STATE_U = 2.0 ** -16


def _np(t):
    return None if t is None else t.double().cpu().numpy()


def _close(name, got, want, size, u):
    err = np.abs(_np(got) - want)
    bad = ~(err <= u * size + 1e-30)
    assert not bad.any(), (name, int(bad.sum()), float(np.nanmax(err / (size + 1e-30)) / u))


def _beta(H, dev):
    """Decays of no memory, short, long and endless ones over the heads."""
    b = [0.9, 1.0 - 2.0 ** -10, 0.0, 1.0, 0.5, 0.99]
    return torch.tensor([b[h % 6] for h in range(H)], device=dev)


class Case:
    def __init__(self, dev, B, T, H, Hk, Dk, Dv, dtype=BF, lens=None, layout="btd", seed=0,
                 scale=0.5, beta=None):
        g = torch.Generator().manual_seed(1000 * seed + 7 * T + Dk + Dv)
        self.shape = (B, T, H, Hk, Dk, Dv)
        self.dtype, self.lens, self.scale, self.dev = dtype, lens, scale, dev
        rnd = lambda *s: torch.randn(s, generator=g)

        def make(heads, D):
            x = rnd(B, T, heads, D).to(dtype)
            if lens is not None:   # places that must not be looked at
                for b, n in enumerate(lens):
                    x[b, n:] = float("nan") if b % 2 == 0 else float("inf")
            x = x.to(dev)
            if layout == "tbd":
                return x.transpose(0, 1).contiguous().transpose(0, 1)
            if layout == "bhtd":
                return x.transpose(1, 2).contiguous().transpose(1, 2)
            if layout == "packed":
                rows = torch.zeros(B, T, heads * D + 24, dtype=dtype, device=dev)
                rows[..., 8:8 + heads * D] = x.flatten(2)
                return rows[..., 8:8 + heads * D].unflatten(-1, (heads, D))
            return x
        self.make = make
        self.q, self.k, self.v, self.do = make(H, Dk), make(Hk, Dk), make(Hk, Dv), make(H, Dv)
        self.state = rnd(B, H, Dk, Dv).to(dev)
        self.dstate = rnd(B, H, Dk, Dv).to(dev)
        self.beta = _beta(H, dev) if beta is None else beta.to(dev)
        self.seq = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=dev)
        self.ws = torch.zeros(snn.snn_leaky_attn_workspace_bytes(*self.shape, backward=True),
                              dtype=torch.uint8, device=dev)

    def clean(self, x):
        x = _np(x)
        if self.lens is not None:
            x = x.copy()
            for b, n in enumerate(self.lens):
                x[b, n:] = 0
        return x

    def args(self):
        return [self.clean(x) for x in (self.q, self.k, self.v)] + [_np(self.beta)]

    def ok(self):
        assert snn.snn_workspace_status(self.ws) == 0


def _forward(c, with_state):
    B, T, H, Hk, Dk, Dv = c.shape
    o = c.make(H, Dv)
    o.fill_(float("nan"))
    out = torch.full_like(c.state, float("nan")) if with_state else None
    snn.snn_leaky_attn_fwd(c.q, c.k, c.v, c.beta, o, c.ws, scale=c.scale, seq_lens=c.seq,
                           state_in=c.state if with_state else None, state_out=out)
    c.ok()
    return o, out


def check_forward(c, with_state=True):
    o, out = _forward(c, with_state)
    st = _np(c.state) if with_state else None
    want, end = A.attn_forward(*c.args(), c.scale, c.lens, st)
    size, end_size = A.attn_forward_size(*c.args(), c.scale, c.lens, st)
    _close("o", o, want, size, 5 * U)
    if with_state:
        _close("state", out, end, end_size, STATE_U)
    return o


def check_backward(c, with_state=True):
    B, T, H, Hk, Dk, Dv = c.shape
    grads = [c.make(H, Dk), c.make(Hk, Dk), c.make(Hk, Dv)]
    for x in grads:
        x.fill_(float("nan"))
    gin = torch.full_like(c.state, float("nan")) if with_state else None
    snn.snn_leaky_attn_bwd(c.q, c.k, c.v, c.beta, c.do, *grads, c.ws, scale=c.scale,
                           seq_lens=c.seq, state_in=c.state if with_state else None,
                           grad_state_out=c.dstate if with_state else None, grad_state_in=gin)
    c.ok()
    st, ds = (_np(c.state), _np(c.dstate)) if with_state else (None, None)
    want = A.attn_backward(*c.args(), c.clean(c.do), c.scale, c.lens, st, ds)
    size = A.attn_backward_size(*c.args(), c.clean(c.do), c.scale, c.lens, st, ds)
    for name, got, w, s in zip(("grad_q", "grad_k", "grad_v"), grads, want, size):
        _close(name, got, w, s, 5 * U)
    if with_state:
        _close("grad_state_in", gin, want[3], size[3], STATE_U)


LENGTHS = [1, 2, 15, 63, 64, 65, 100, 127, 128, 129, 200]


@pytest.mark.parametrize("T", LENGTHS)
@pytest.mark.parametrize("D", [64, 128])
def test_lengths(T, D, cuda_device):
    c = Case(cuda_device, 2, T, 2, 2, D, D)
    check_forward(c)
    check_backward(c)


@pytest.mark.parametrize("Dk,Dv", [(8, 8), (16, 128), (128, 16), (40, 72), (72, 40), (64, 128),
                                   (128, 64), (96, 96), (120, 104)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_widths(Dk, Dv, dtype, cuda_device):
    c = Case(cuda_device, 2, 150, 6, 6, Dk, Dv, dtype)
    check_forward(c)
    check_backward(c)


# one width up to 64, the other above, and heads enough that the backward takes two launches; in the
# longer case the second launch cuts its tokens into segments and the first does not
@pytest.mark.parametrize("B,T,H,Hk,Dk,Dv,lens", [(4, 200, 38, 38, 64, 128, None),
                                                 (4, 200, 38, 19, 104, 24, [200, 0, 77, 128]),
                                                 (5, 1500, 22, 22, 16, 72, [1500, 767, 1, 1499, 769])])
def test_mixed_widths_of_many_heads(B, T, H, Hk, Dk, Dv, lens, cuda_device):
    c = Case(cuda_device, B, T, H, Hk, Dk, Dv, lens=lens)
    check_forward(c)
    check_backward(c)


@pytest.mark.parametrize("H,Hk", [(6, 1), (6, 2), (6, 3)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_shared_heads(H, Hk, dtype, cuda_device):
    c = Case(cuda_device, 2, 90, H, Hk, 64, 32, dtype)
    check_forward(c)
    check_backward(c)


# empty, one-token, chunk-sized, odd and full sequences; NaN and infinities past them
@pytest.mark.parametrize("lens", [[0, 1, 64, 130], [130, 0, 0, 0], [65, 63, 129, 128], [0, 0, 0, 0]])
@pytest.mark.parametrize("with_state", [True, False])
def test_ragged(lens, with_state, cuda_device):
    c = Case(cuda_device, 4, 130, 4, 2, 72, 64, HF, lens=lens)
    o = check_forward(c, with_state)
    for b, n in enumerate(lens):
        assert torch.count_nonzero(o[b, n:]) == 0
    check_backward(c, with_state)


@pytest.mark.parametrize("layout", ["tbd", "bhtd", "packed"])
def test_layouts(layout, cuda_device):
    c = Case(cuda_device, 3, 140, 4, 2, 64, 128, BF, lens=[140, 77, 3], layout=layout)
    check_forward(c)
    check_backward(c)


# few heads and a long axis, where the tokens are split over blocks
@pytest.mark.parametrize("B,T,H,Dk,Dv", [(1, 2500, 2, 64, 64), (1, 1999, 1, 128, 128), (2, 1300, 3, 40, 128)])
@pytest.mark.parametrize("ragged", [False, True])
def test_long(B, T, H, Dk, Dv, ragged, cuda_device):
    c = Case(cuda_device, B, T, H, H, Dk, Dv, BF, lens=[T - 700, T][:B] if ragged else None)
    check_forward(c)
    check_backward(c)


def test_without_state_and_without_tokens(cuda_device):
    c = Case(cuda_device, 2, 70, 2, 2, 64, 64)
    check_forward(c, False)
    check_backward(c, False)
    c = Case(cuda_device, 2, 0, 2, 2, 64, 64)
    _, out = _forward(c, True)
    assert torch.equal(out, c.state)
    gin = torch.empty_like(c.state)
    snn.snn_leaky_attn_bwd(c.q, c.k, c.v, c.beta, c.do, torch.empty_like(c.q), torch.empty_like(c.k),
                           torch.empty_like(c.v), c.ws, scale=0.5, state_in=c.state,
                           grad_state_out=c.dstate, grad_state_in=gin)
    c.ok()
    _close("grad_state_in", gin, _np(c.dstate), np.abs(_np(c.dstate)), 2.0 ** -22)


def test_state_places_and_in_place_states(cuda_device):
    c = Case(cuda_device, 4, 1100, 1, 1, 64, 64, BF, lens=[1100, 0, 30, 64])
    pool = torch.randn(6, 1, 64, 64, generator=torch.Generator().manual_seed(3)).to(cuda_device)
    first = pool.clone()
    slots = torch.tensor([4, 0, -1, 9], dtype=torch.int32, device=cuda_device)
    o = torch.empty_like(c.do)
    snn.snn_leaky_attn_fwd(c.q, c.k, c.v, c.beta, o, c.ws, scale=0.5, seq_lens=c.seq, state_in=pool,
                           state_out=pool, slots=slots)
    c.ok()
    st = np.zeros((4, 1, 64, 64))
    st[0], st[1] = _np(first[4]), _np(first[0])
    want, end = A.attn_forward(*c.args(), 0.5, c.lens, st)
    size, end_size = A.attn_forward_size(*c.args(), 0.5, c.lens, st)
    _close("o", o, want, size, 5 * U)
    _close("state", pool[4], end[0], end_size[0], STATE_U)
    for p in (0, 1, 2, 3, 5):
        assert torch.equal(pool[p], first[p])


def test_large_fp16_states_stay_finite(cuda_device):
    """A state past fp16's range (a sum of many equal products)."""
    c = Case(cuda_device, 1, 600, 1, 1, 64, 64, HF, beta=torch.ones(1))
    c.k.fill_(24.0)
    c.v.fill_(24.0)
    c.q.fill_(2.0 ** -10)
    check_forward(c)


def test_prompt_then_tokens_equals_the_whole(cuda_device):
    c = Case(cuda_device, 2, 133, 4, 2, 72, 40, BF)
    whole, end_size = A.attn_forward(*c.args(), 0.5, None, _np(c.state)), None
    size = A.attn_forward_size(*c.args(), 0.5, None, _np(c.state))
    st = c.state.clone()
    o = torch.empty_like(c.do)
    n = 130
    snn.snn_leaky_attn_fwd(c.q[:, :n], c.k[:, :n], c.v[:, :n], c.beta, o[:, :n], c.ws, scale=0.5,
                           state_in=st, state_out=st)
    for t in range(n, 133):
        snn.snn_leaky_attn_step(c.q[:, t], c.k[:, t], c.v[:, t], c.beta, st, o[:, t], scale=0.5)
    c.ok()
    _close("o", o, whole[0], size[0], 5 * U)
    _close("state", st, whole[1], size[1], STATE_U)


# fp32 throughout: the roundings of o to 16 bits and of about 130 fp32 additions
@pytest.mark.parametrize("B,H,Hk,Dk,Dv", [(1, 1, 1, 8, 8), (3, 4, 2, 64, 64), (5, 6, 2, 96, 128),
                                          (2, 2, 2, 128, 72), (7, 3, 1, 40, 24)])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_step(B, H, Hk, Dk, Dv, dtype, cuda_device):
    c = Case(cuda_device, B, 1, H, Hk, Dk, Dv, dtype)
    st, o = c.state.clone(), torch.empty_like(c.do)
    snn.snn_leaky_attn_step(c.q[:, 0], c.k[:, 0], c.v[:, 0], c.beta, st, o[:, 0], scale=c.scale)
    want, end = A.attn_forward(*c.args(), c.scale, None, _np(c.state))
    size, end_size = A.attn_forward_size(*c.args(), c.scale, None, _np(c.state))
    _close("o", o, want, size, 2.0 ** -16 + (U if dtype == BF else 2.0 ** -11))
    _close("state", st, end, end_size, 2.0 ** -22)


def test_step_places(cuda_device):
    c = Case(cuda_device, 5, 1, 2, 1, 64, 72, HF)
    pool = torch.randn(7, 2, 64, 72, generator=torch.Generator().manual_seed(4)).to(cuda_device)
    first = pool.clone()
    where = [6, -1, 0, 7, 3]
    o = torch.full_like(c.do, float("nan"))
    snn.snn_leaky_attn_step(c.q[:, 0], c.k[:, 0], c.v[:, 0], c.beta, pool, o[:, 0], scale=0.5,
                            slots=torch.tensor(where, dtype=torch.int32, device=cuda_device))
    st = np.stack([_np(first[p]) if 0 <= p < 7 else np.zeros((2, 64, 72)) for p in where])
    want, end = A.attn_forward(*c.args(), 0.5, None, st)
    size, end_size = A.attn_forward_size(*c.args(), 0.5, None, st)
    for b, p in enumerate(where):
        if 0 <= p < 7:
            _close("o", o[b], want[b], size[b], 2.0 ** -16 + 2.0 ** -11)
            _close("state", pool[p], end[b], end_size[b], 2.0 ** -22)
        else:
            assert torch.count_nonzero(o[b]) == 0
    for p in (1, 2, 4, 5):
        assert torch.equal(pool[p], first[p])


def test_step_state_past_4_gib(cuda_device):
    n = (1 << 32) // (128 * 128 * 4) + 3
    pool = torch.zeros(n, 1, 128, 128, device=cuda_device)
    c = Case(cuda_device, 1, 1, 1, 1, 128, 128)
    o = torch.empty_like(c.do)
    snn.snn_leaky_attn_step(c.q[:, 0], c.k[:, 0], c.v[:, 0], c.beta, pool, o[:, 0],
                            slots=torch.tensor([n - 1], dtype=torch.int32, device=cuda_device))
    want = _np(c.k[0, 0, 0])[:, None] * _np(c.v[0, 0, 0])[None]
    _close("state", pool[n - 1, 0], want, np.abs(want), 2.0 ** -22)
    assert torch.count_nonzero(pool[:n - 1]) == 0


def test_strides_past_32_bits(cuda_device):
    """Sequences more than 2^32 bytes apart."""
    far = (1 << 31) + 64
    buf = torch.zeros(far + 70 * 64, dtype=BF, device=cuda_device)
    c = Case(cuda_device, 2, 70, 1, 1, 64, 64)
    wide = buf.as_strided((2, 70, 1, 64), (far, 64, 64, 1))
    wide.copy_(c.v)
    c.v = wide
    check_forward(c)
    check_backward(c)


def test_side_stream_and_repeatability(cuda_device):
    c = Case(cuda_device, 2, 700, 4, 2, 128, 128, BF)
    o, out = _forward(c, True)
    o, out = o.clone(), out.clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    o2, out2 = torch.empty_like(o), torch.empty_like(out)
    with torch.cuda.stream(side):
        snn.snn_leaky_attn_fwd(c.q, c.k, c.v, c.beta, o2, c.ws, scale=c.scale, state_in=c.state,
                               state_out=out2)
    side.synchronize()
    assert torch.equal(o, o2) and torch.equal(out, out2)


def test_wrapper_refusals(cuda_device):
    c = Case(cuda_device, 2, 16, 2, 1, 64, 32)
    o = torch.empty_like(c.do)
    fwd = lambda **k: snn.snn_leaky_attn_fwd(**{**dict(q=c.q, k=c.k, v=c.v, beta=c.beta, o=o, ws=c.ws), **k})
    for bad in (dict(k=c.k[:, :15]), dict(v=c.v.half()), dict(beta=c.beta.double()),
                dict(o=o.transpose(-1, -2).contiguous().transpose(-1, -2)), dict(q=c.q.cpu()),
                dict(seq_lens=torch.ones(2, dtype=torch.int64, device=cuda_device)),
                dict(state_in=c.state[:1].contiguous())):
        with pytest.raises(ValueError):
            fwd(**bad)
    with pytest.raises(snn.SnnError):
        fwd(q=c.q.float(), k=c.k.float(), v=c.v.float(), o=o.float())
    with pytest.raises(snn.SnnError):
        fwd(ws=torch.empty(16, dtype=torch.uint8, device=cuda_device))
