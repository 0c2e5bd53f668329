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


def _library_takes(name, t):
    """The C ABI's rules on one tensor: 16-byte start; strides of [B, T, heads, D] positive multiples
    of 8, of rows at least their length; the rest contiguous."""
    if t.numel() == 0:
        return True
    if t.data_ptr() % 16:
        return False
    steps = [s for n, s in zip(t.shape, t.stride()) if n > 1]
    if t.dim() == 4 and t.dtype != torch.float32:
        return t.stride(-1) == 1 and all(s > 0 and s % 8 == 0 for s in steps[:-1])
    if t.dim() == 2:
        return (t.shape[1] == 1 or t.stride(1) == 1) and (t.shape[0] == 1 or t.stride(0) >= t.shape[1])
    return t.is_contiguous()


def test_attention_inputs_of_any_layout(calls):
    """Broadcast sequences, another order of dimensions, parts that start or step off 16 bytes."""
    B, T, H, D = 2, 6, 4, 16
    bf = lambda *s: torch.randn(*s).to(torch.bfloat16)
    layouts = [bf(B, T, H, D), bf(1, T, H, D).expand(B, T, H, D), bf(B, T, 1, D).expand(B, T, H, D),
               bf(B, T, D, H).transpose(2, 3), bf(B * T * H * D + 3)[3:].view(B, T, H, D),
               bf(B, T, H * D + 4)[..., 4:].unflatten(-1, (H, D)), bf(B, T, H, 2 * D)[..., ::2]]
    beta, lens = torch.rand(H + 1)[1:], torch.tensor([9, 6, 3], dtype=torch.int32)[1:]
    state = torch.randn(B, H, D, D).transpose(2, 3)
    for x in layouts:
        q, k, v, s = (t.detach().requires_grad_() for t in (x, x, x, state))
        o, end = autograd.leaky_attention(q, k, v, beta, s, seq_lens=lens)
        torch.autograd.backward([o, end], [bf(B * T * H * D + 1)[1:].view(B, T, H, D),
                                           torch.randn(B, H, D, D).transpose(2, 3)])
    assert len(calls.seen) == 2 * len(layouts)
    for name, t in calls.tensors():
        assert _library_takes(name, t), (name, t.shape, t.stride(), t.data_ptr() % 16)


@pytest.mark.parametrize("group", [0, 8])
def test_norm_inputs_and_gradients_of_any_layout(group, calls):
    """Odd rows whose gradient is a part of another tensor (as torch.cat hands back), broadcast and
    transposed rows, parameters inside a longer vector."""
    M, N = 3, 24 if group else 9
    f = torch.randn
    layouts = [f(M, N), f(1, N).expand(M, N), f(N, M).t(), f(M * N + 1)[1:].view(M, N), f(M, 2 * N)[:, ::2],
               f(M, N + 3)[:, :N]]
    for x in layouts:
        par = [f(N + 1)[1:].requires_grad_() for _ in range(3)]
        r, a, z = (x.detach().requires_grad_() for _ in range(3))
        out = autograd.block_norm(r, a, z, *par, group=group, gate="silu")
        other = torch.randn(1, N, requires_grad=True)
        joined = [torch.cat([other, t]) for t in out]
        torch.autograd.backward(joined, [f(M + 1, N) for _ in joined])
    assert len(calls.seen) == 2 * len(layouts)
    for name, t in calls.tensors():
        assert _library_takes(name, t), (name, t.shape, t.stride(), t.data_ptr() % 16)
        if group and t.dim() == 2:     # groups are for rows of whole vectors
            assert t.stride(0) % 8 == 0


def test_shapes_that_do_not_match_are_refused(calls):
    """As many elements in another order are not the same rows."""
    r = torch.randn(2, 5, 16)
    for a, z in ((torch.randn(5, 2, 16), None), (torch.randn(2, 10, 8), None), (torch.randn(10, 16), None),
                 (torch.randn(2, 5, 16), torch.randn(5, 2, 16))):
        with pytest.raises(ValueError, match="shape"):
            autograd.block_norm(r, a, z, w_pre=torch.ones(16), gate="none" if z is None else "silu")
    q, k, v = _qkv()
    with pytest.raises(ValueError, match="shape"):
        autograd.leaky_attention(q[0], k[0], v[0], torch.full((4,), 0.9))
    with pytest.raises(ValueError, match="needs a"):
        autograd.block_norm(r, None, w_pre=torch.ones(16))
    assert not calls.seen


def test_attention_zeroes_the_status_word_alone(calls, monkeypatch):
    """Workspaces hold segment states and shared heads' sums, which kernels write before they read."""
    empty = torch.empty

    def dirty(*a, **k):
        t = empty(*a, **k)
        return t.fill_(0xA5) if t.dtype == torch.uint8 else t
    monkeypatch.setattr(torch, "empty", dirty)
    q, k, v = _qkv(T=200)
    o, _ = autograd.leaky_attention(q, k, v, torch.full((4,), 0.9))
    o.sum().backward()
    for name, args, kw in calls.seen:
        ws = next(t for t in args if isinstance(t, torch.Tensor) and t.dtype == torch.uint8)
        assert torch.count_nonzero(ws[:256]) == 0
        assert ws.numel() == 256 or (ws[256:] == 0xA5).all()
    assert any(next(t for t in args if t.dtype == torch.uint8).numel() > 256 for _, args, _ in calls.seen)


def test_outputs_that_nothing_uses_bring_no_gradients(calls):
    q, k, v = _qkv()
    o, end = autograd.leaky_attention(q, k, v, torch.full((4,), 0.9))
    o.sum().backward()
    assert calls.seen[-1][2]["grad_state_out"] is None
    r = _rows()
    autograd.block_norm(r, _rows(), w_pre=torch.ones(24))[1].sum().backward()
    assert calls.seen[-1][1][6] is None and calls.seen[-1][1][7] is not None   # grad_r_out, grad_y


def test_a_call_that_gave_up_shows_in_the_status(calls, monkeypatch):
    """A kernel's bounded wait that runs out leaves its code in the workspace."""
    give_up = {"snn_leaky_attn_fwd": 0, "snn_leaky_attn_bwd": 0}
    for name in give_up:
        real = getattr(snn, name)

        def call(*a, real=real, name=name, **kw):
            real(*a, **kw)
            next(t for t in a if t.dtype == torch.uint8)[:4].view(torch.int32).fill_(give_up[name])
        monkeypatch.setattr(snn, name, call)
    beta = torch.full((4,), 0.9)
    for fwd, bwd in ((0, 0), (6, 0), (0, 6)):
        give_up.update(snn_leaky_attn_fwd=fwd, snn_leaky_attn_bwd=bwd)
        status = torch.zeros(1, dtype=torch.int32)
        o, _ = autograd.leaky_attention(*_qkv(), beta, status=status)
        assert status.item() == fwd
        o.sum().backward()
        assert status.item() == max(fwd, bwd)
    give_up.update(snn_leaky_attn_fwd=0, snn_leaky_attn_bwd=0)
    status.fill_(6)                     # it stays until the caller clears it
    autograd.leaky_attention(*_qkv(), beta, status=status)
    assert status.item() == 6
    for bad in (torch.zeros(2, dtype=torch.int32), torch.zeros(1)):
        with pytest.raises(ValueError, match="status"):
            autograd.leaky_attention(*_qkv(), beta, status=bad)
