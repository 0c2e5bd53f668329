"""The autograd wrappers of leaky attention and the block norms."""
import pytest
import torch

from paper_2211_10725_gb300 import snn
from paper_2211_10725_gb300.autograd import block_norm, leaky_attention

pytestmark = pytest.mark.gpu


# The wrappers run the C ABI's own calls, so their gradients are its bits.
@pytest.mark.parametrize("with_state", [True, False])
def test_leaky_attention_gradients_are_the_abi_s(with_state, cuda_device):
    g = torch.Generator().manual_seed(2)
    rnd = lambda *s: torch.randn(s, generator=g)
    B, T, Hq, Hk, Dk, Dv = 2, 90, 4, 2, 40, 64
    leaf = lambda t: t.to(cuda_device).requires_grad_()
    q, k, v = (leaf(rnd(B, T, h, d).to(torch.bfloat16)) for h, d in ((Hq, Dk), (Hk, Dk), (Hk, Dv)))
    state = leaf(rnd(B, Hq, Dk, Dv)) if with_state else None
    beta = torch.tensor([0.5, 0.9, 0.99, 1.0], device=cuda_device)
    lens = torch.tensor([90, 33], dtype=torch.int32, device=cuda_device)
    o, end = leaky_attention(q, k, v, beta, state, 0.3, lens)
    do = rnd(B, T, Hq, Dv).to(torch.bfloat16).to(cuda_device)
    de = rnd(B, Hq, Dk, Dv).to(cuda_device)
    torch.autograd.backward([o, end], [do, de])
    grads = [torch.empty_like(x) for x in (q, k, v)]
    gs = torch.empty(B, Hq, Dk, Dv, device=cuda_device) if with_state else None
    ws = torch.zeros(snn.snn_leaky_attn_workspace_bytes(B, T, Hq, Hk, Dk, Dv, True), dtype=torch.uint8,
                     device=cuda_device)
    st = state.detach() if with_state else None
    snn.snn_leaky_attn_bwd(q.detach(), k.detach(), v.detach(), beta, do, *grads, ws, scale=0.3,
                           seq_lens=lens, state_in=st, grad_state_out=de, grad_state_in=gs)
    for x, want in zip((q, k, v), grads):
        assert torch.equal(x.grad, want)
    if with_state:
        assert torch.equal(state.grad, gs)


def test_block_norm_gradients_are_the_abi_s(cuda_device):
    g = torch.Generator().manual_seed(3)
    rnd = lambda *s: torch.randn(s, generator=g).to(cuda_device)
    leaf = lambda t: t.requires_grad_()
    r, a, z = leaf(rnd(3, 5, 128)), leaf(rnd(3, 5, 128).to(torch.bfloat16)), leaf(rnd(3, 5, 128).to(torch.bfloat16))
    wp, sc, pre = leaf(rnd(128)), leaf(rnd(128)), leaf(rnd(128))
    r2, y = block_norm(r, a, z, wp, sc, pre, group=32, gate="silu")
    gr, gy = rnd(3, 5, 128), rnd(3, 5, 128).to(torch.bfloat16)
    torch.autograd.backward([r2, y], [gr, gy])
    flat = lambda t: t.detach().reshape(15, 128)
    out = [torch.empty_like(flat(t)) for t in (r, a, z)] + [torch.empty(128, device=cuda_device) for _ in range(3)]
    ws = torch.empty(snn.snn_block_norm_workspace_bytes(15, 128), dtype=torch.uint8, device=cuda_device)
    snn.snn_block_norm_bwd(flat(r2), flat(a), flat(z), wp.detach(), sc.detach(), pre.detach(), flat(gr),
                           flat(gy), *out, ws, eps=1e-6, group=32, gate="silu")
    for t, want in zip((r, a, z, wp, sc, pre), out):
        assert torch.equal(t.grad.reshape(want.shape), want)


def test_other_layouts_give_the_same_bits(cuda_device):
    """Odd fp32 rows whose gradient is a part of torch.cat's, and attention on broadcast keys and
    shifted values: as with contiguous tensors."""
    g = torch.Generator().manual_seed(4)
    rnd = lambda *s: torch.randn(s, generator=g).to(cuda_device)
    r, a, w, up = rnd(3, 1001), rnd(3, 1001), rnd(1001), rnd(4, 1001)
    grads = []
    for first in (0, 1):
        x = [t.clone().requires_grad_() for t in (r, a, w)]
        out, y = block_norm(x[0], x[1], w_pre=x[2])
        y = torch.cat([torch.zeros(first, 1001, device=cuda_device, requires_grad=True), y])
        torch.autograd.backward([out, y], [up[1:], up[1 - first:]])
        grads.append([t.grad for t in x])
    assert all(torch.equal(s, t) for s, t in zip(*grads))
    B, T, H, D = 2, 70, 2, 64
    q, k1, v1 = (rnd(*s).to(torch.bfloat16) for s in ((B, T, H, D), (1, T, H, D), (B * T * H * D + 3,)))
    beta, do = torch.tensor([0.9, 1.0], device=cuda_device), rnd(B, T, H, D).to(torch.bfloat16)
    results = []
    for copied in (False, True):
        k, v = k1.expand(B, T, H, D), v1[3:].view(B, T, H, D)
        if copied:
            k, v = k.contiguous(), v.clone()
        x = [t.detach().requires_grad_() for t in (q, k, v)]
        o, end = leaky_attention(*x, beta)
        o.backward(do)
        results.append([o.detach(), end.detach(), *(t.grad for t in x)])
    assert all(torch.equal(s, t) for s, t in zip(*results))


def test_status_of_calls_that_finish(cuda_device):
    status = torch.zeros(1, dtype=torch.int32, device=cuda_device)
    x = [torch.randn(2, 700, 2, 64, device=cuda_device).to(torch.bfloat16).requires_grad_() for _ in range(3)]
    o, _ = leaky_attention(*x, torch.tensor([0.9, 1.0], device=cuda_device), status=status)
    o.sum().backward()
    assert status.item() == 0
    status.fill_(6)            # SNN_ERR_TIMEOUT
    leaky_attention(*x, torch.tensor([0.9, 1.0], device=cuda_device), status=status)
    assert status.item() == 6
