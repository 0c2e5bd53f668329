"""What the autograd wrappers of the selective scan, the causal convolution and the
layer norm hand to the library, without a GPU: the calls are replaced by functions
that look at their arguments."""
import pytest
import torch

from paper_2211_10725_gb300 import autograd, snn

NAMES = ["snn_selective_scan_fwd", "snn_selective_scan_bwd", "snn_causal_conv_fwd", "snn_causal_conv_bwd",
         "snn_layer_norm_fwd", "snn_layer_norm_bwd"]


class Calls:
    """Stands in for the library's calls; fills outputs so that they are values."""

    def __init__(self, monkeypatch):
        self.seen = []
        for name in NAMES:
            monkeypatch.setattr(snn, name, self._call(name))

    def _call(self, name):
        def call(*args, **kw):
            self.seen.append((name, args, kw))
            for t in (*args, *kw.values()):
                if isinstance(t, torch.Tensor) and t.is_floating_point() and not t.requires_grad:
                    torch.nan_to_num_(t)
        return call

    def names(self):
        return [n for n, _, _ in self.seen]

    def tensors(self):
        for name, args, kw in self.seen:
            for t in (*args, *kw.values()):
                if isinstance(t, torch.Tensor) and t.dtype != torch.uint8:
                    yield name, t


@pytest.fixture
def calls(monkeypatch):
    return Calls(monkeypatch)


def _scan(B=2, T=5, D=8, N=3, G=2, dtype=torch.bfloat16):
    r = lambda *s: torch.randn(s).to(dtype).requires_grad_()
    return dict(u=r(B, T, D), delta=r(B, T, D), A=(-torch.rand(D, N)).requires_grad_(), B=r(B, T, G, N), C=r(B, T, G, N),
                D=torch.ones(D, requires_grad=True), z=r(B, T, D), delta_bias=torch.zeros(D, requires_grad=True),
                state=torch.zeros(B, D, N, requires_grad=True))


def test_every_input_of_the_scan_gets_a_gradient(calls):
    x = _scan()
    y, end = autograd.selective_scan(**x)
    (y.float().sum() + end.sum()).backward()
    for name, t in x.items():
        assert t.grad is not None and t.grad.shape == t.shape and t.grad.dtype == t.dtype, name
    assert calls.names() == ["snn_selective_scan_fwd", "snn_selective_scan_bwd"]


def test_absent_parts_stay_absent(calls):
    x = _scan()
    for name in ("D", "z", "delta_bias", "state"):
        x[name] = None
    y, _ = autograd.selective_scan(**x, softplus=False)
    y.float().sum().backward()
    kw = calls.seen[1][2]
    assert kw["softplus"] is False
    assert all(kw[k] is None for k in ("D", "z", "delta_bias", "grad_D", "grad_z", "grad_delta_bias", "grad_state_in",
                                       "grad_state_out"))


def test_checkpoints_only_where_a_gradient_may_be_asked_for(calls):
    x = _scan()
    with torch.no_grad():
        autograd.selective_scan(**x)
    autograd.selective_scan(**x)
    assert calls.seen[0][2]["ckpt"] is None
    assert calls.seen[1][2]["ckpt"].numel() == snn.snn_selective_scan_ckpt_elems(2, 5, 8, 3, 2)


def test_an_output_that_nothing_uses_has_no_gradient_of_zeros(calls):
    x = _scan()
    _, end = autograd.selective_scan(**x)
    end.sum().backward()
    name, args, kw = calls.seen[1]
    assert torch.count_nonzero(args[5]) == 0 and kw["grad_state_out"] is not None
    calls.seen.clear()
    xc = torch.randn(2, 6, 8, requires_grad=True)
    y, _ = autograd.causal_conv(xc, torch.randn(8, 3), None)
    y.sum().backward()
    assert calls.seen[1][2]["grad_state_out"] is None


def _library_takes(t):
    """The C ABI's rules on one tensor: 16-byte start, contiguous last dimension, positive steps."""
    if t.numel() == 0:
        return True
    steps = [s for n, s in zip(t.shape, t.stride()) if n > 1]
    return t.data_ptr() % 16 == 0 and all(s > 0 for s in steps) and (t.shape[-1] <= 1 or t.stride(-1) == 1)


def _expanded(shape, dtype=torch.bfloat16):
    return torch.randn(shape[0], 1, *shape[2:]).to(dtype).expand(shape).requires_grad_(False)


@pytest.mark.parametrize("view", [
    lambda s: _expanded(s),                                             # broadcast over the tokens
    lambda s: torch.randn(*s[::-1]).to(torch.bfloat16).permute(*range(len(s))[::-1]),
    lambda s: torch.randn(*s[:-1], s[-1] + 1).to(torch.bfloat16)[..., 1:],   # off the boundary
    lambda s: torch.randn(*s[:-1], 2 * s[-1]).to(torch.bfloat16)[..., ::2]])
def test_tensors_of_any_layout(calls, view):
    x = _scan()
    for name in ("u", "delta", "z", "B", "C"):
        x[name] = view(tuple(x[name].shape))
    y, _ = autograd.selective_scan(**x)
    y.backward(view(tuple(y.shape)).to(y.dtype))
    w = torch.randn(8, 4, requires_grad=True)
    y, _ = autograd.causal_conv(view((2, 5, 8)), w, torch.randn(8))
    y.backward(view((2, 5, 8)).to(y.dtype))
    ln = torch.ones(8, requires_grad=True)
    y = autograd.layer_norm(view((2, 5, 8)), ln)
    y.backward(view((2, 5, 8)).to(y.dtype))
    assert len(calls.seen) == 6
    for name, t in calls.tensors():
        assert _library_takes(t), name


def test_parameters_and_states_of_any_layout(calls):
    x = _scan()
    x["A"] = torch.randn(3, 8).t()
    x["D"] = torch.ones(1).expand(8)
    x["state"] = torch.zeros(3, 8, 2).permute(2, 1, 0)
    x["seq_lens"] = torch.tensor([[5, 0], [3, 0]], dtype=torch.int32)[:, 0]
    y, end = autograd.selective_scan(**x)
    (y.float().sum() + end.sum()).backward()
    for name, t in calls.tensors():
        assert _library_takes(t), name


def test_the_norm_of_a_32_bit_stream_in_16_bits(calls):
    x = torch.randn(2, 3, 16, requires_grad=True)
    w = torch.ones(16, requires_grad=True)
    y = autograd.layer_norm(x, w, dtype=torch.bfloat16)
    assert y.dtype == torch.bfloat16 and y.shape == x.shape
    y.float().sum().backward()
    assert x.grad.dtype == torch.float32 and w.grad.shape == (16,)
    assert calls.seen[1][1][3].dtype == torch.bfloat16


def test_second_derivatives_are_refused(calls):
    """Not given as zero: a gradient penalty would go unnoticed."""
    x = _scan(dtype=torch.float32)
    c = torch.randn(2, 6, 8, requires_grad=True)
    for out, t in ((autograd.selective_scan(**x)[0], x["u"]), (autograd.causal_conv(c, torch.randn(8, 4))[0], c),
                   (autograd.layer_norm(c), c)):
        g, = torch.autograd.grad(out.square().sum(), t, create_graph=True)
        with pytest.raises(RuntimeError, match="twice"):
            g.square().sum().backward()


@pytest.mark.parametrize("bad", [dict(u=torch.zeros(2, 8)), dict(B=torch.zeros(2, 5, 3)), dict(A=torch.zeros(8)),
                                 dict(delta=torch.zeros(2, 5, 8)), dict(z=torch.zeros(2, 5, 8))])
def test_scan_refusals(calls, bad):
    with pytest.raises(ValueError):
        autograd.selective_scan(**{**_scan(), **bad})
    assert not calls.seen


def test_conv_refusals(calls):
    x, w = torch.zeros(2, 5, 8), torch.zeros(8, 4)
    for bad in (dict(x=x[0]), dict(w=w[0]), dict(state=torch.zeros(2, 3, 8, dtype=torch.bfloat16))):
        with pytest.raises(ValueError):
            autograd.causal_conv(**{**dict(x=x, w=w), **bad})
    assert not calls.seen
