"""What the autograd wrappers of leaky attention and the block norms hand to
the library, without a GPU: the calls are replaced by functions that look at
their arguments."""
import pytest
import torch

from paper_2211_10725_gb300 import autograd, snn


class Calls:
    """Stands in for the library's calls; fills outputs so that they are values."""

    def __init__(self, monkeypatch):
        self.seen = []
        for name in ("snn_leaky_attn_fwd", "snn_leaky_attn_bwd", "snn_block_norm_fwd", "snn_block_norm_bwd"):
            monkeypatch.setattr(snn, name, self._call(name))

    def _call(self, name):
        def call(*args, **kw):
            self.seen.append((name, args, kw))
            for t in args:
                if isinstance(t, torch.Tensor) and t.is_floating_point() and not t.requires_grad:
                    torch.nan_to_num_(t)
        return call

    def tensors(self):
        for name, args, kw in self.seen:
            for t in (*args, *kw.values()):
                if isinstance(t, torch.Tensor) and t.dtype != torch.uint8:
                    yield name, t


@pytest.fixture
def calls(monkeypatch):
    return Calls(monkeypatch)


def _qkv(B=2, T=5, H=4, Hk=2, D=16, grad=True):
    make = lambda h: torch.randn(B, T, h, D).to(torch.bfloat16).requires_grad_(grad)
    return make(H), make(Hk), make(Hk)


def test_a_decay_that_wants_a_gradient_is_refused(calls):
    beta = torch.full((4,), 0.9, requires_grad=True)
    with pytest.raises(ValueError, match="beta"):
        autograd.leaky_attention(*_qkv(), beta)
    assert not calls.seen
    with torch.no_grad():        # nothing asks for it
        autograd.leaky_attention(*_qkv(), beta)
    autograd.leaky_attention(*_qkv(), beta.detach())
    assert len(calls.seen) == 2


def _rows(M=3, N=24, dtype=torch.float32):
    return torch.randn(M, N).to(dtype).requires_grad_()


def test_second_derivatives_are_refused(calls):
    """Not given as zero: a gradient penalty would go unnoticed."""
    q, k, v = _qkv()
    r = _rows()
    for out, x in ((autograd.leaky_attention(q, k, v, torch.full((4,), 0.9))[0], q),
                   (autograd.block_norm(r, _rows(), w_pre=torch.ones(24))[1], r)):
        g, = torch.autograd.grad(out.float().square().sum(), x, create_graph=True)
        with pytest.raises(RuntimeError, match="twice"):
            g.float().square().sum().backward()
