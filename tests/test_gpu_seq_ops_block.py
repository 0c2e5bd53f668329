"""The operators as a residual block uses them: layer norm, projection, causal
convolution, projections, gated selective scan, projection, residual; trained through
autograd, and run on from a prompt token by token.

Each of the block's six stages errs by less than 1200 units of 2^-24 of its terms' size (as
the operators' own tests count them, 64 + 24 T with T = 41; fp32 products of up to 48 terms err
by 48), and a sum's terms are in 2-norm less than 2.5 times the sum here: 6 * 1200 * 2.5 * 2^-24 =
1.1e-3 of a result's 2-norm.
"""
import numpy as np
import pytest
import torch

from paper_2211_10725_gb300 import autograd, snn

pytestmark = pytest.mark.gpu
TOL = 1.1e-3
W, D, N, G, WIDTH = 4, 48, 16, 2, 24


def _params(dev, seed=0):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g)
    p = dict(ln_w=1 + 0.1 * r(WIDTH), ln_b=0.1 * r(WIDTH), w_in=r(2 * D, WIDTH) * WIDTH ** -0.5,
             conv_w=r(D, W) * W ** -0.5, conv_b=0.1 * r(D), w_bc=r(2 * G * N, D) * D ** -0.5,
             w_delta=r(D, D) * D ** -0.5, bias=0.5 * r(D) - 2.0,
             A=-torch.exp(torch.log(torch.arange(1, N + 1).float()) + 0.1 * r(D, N)), skip=1 + 0.1 * r(D),
             w_out=r(WIDTH, D) * D ** -0.5)
    return {k: v.to(dev).requires_grad_() for k, v in p.items()}


def block(p, r, lens):
    y = autograd.layer_norm(r, p["ln_w"], p["ln_b"])
    xz = y @ p["w_in"].t()
    x, conv = autograd.causal_conv(xz[..., :D], p["conv_w"], p["conv_b"], seq_lens=lens)
    bc = (x @ p["w_bc"].t()).unflatten(-1, (2 * G, N))
    o, state = autograd.selective_scan(x, x @ p["w_delta"].t(), p["A"], bc[:, :, :G], bc[:, :, G:], D=p["skip"],
                                       z=xz[..., D:], delta_bias=p["bias"], seq_lens=lens)
    return r + o @ p["w_out"].t(), (conv, state)


def plain(p, r, lens):
    """The same in torch, token by token (fp64 where its inputs are)."""
    F = torch.nn.functional
    y = F.layer_norm(r, (WIDTH,), p["ln_w"], p["ln_b"])
    xz = y @ p["w_in"].t()
    x, z = xz[..., :D], xz[..., D:]
    B, T = r.shape[:2]
    live = torch.arange(T, device=r.device)[None] < torch.tensor(lens, device=r.device)[:, None]
    x = x * live[..., None]
    x = F.silu(F.conv1d(F.pad(x.transpose(1, 2), (W - 1, 0)), p["conv_w"][:, None], p["conv_b"], groups=D)).transpose(1, 2)
    x = x * live[..., None]
    bc = (x @ p["w_bc"].t()).unflatten(-1, (2 * G, N)).repeat_interleave(D // G, dim=2)
    s = F.softplus(x @ p["w_delta"].t() + p["bias"]) * live[..., None]
    h, out = torch.zeros(B, D, N, dtype=r.dtype, device=r.device), []
    for t in range(T):
        h = torch.exp(s[:, t, :, None] * p["A"]) * h + (s[:, t] * x[:, t])[..., None] * bc[:, t, :D]
        out.append((h * bc[:, t, D:]).sum(-1))
    o = (torch.stack(out, 1) + p["skip"] * x) * F.silu(z) * live[..., None]
    return r + o @ p["w_out"].t(), h


def _close(name, got, want):
    err = (got.double() - want).norm() / want.norm()
    assert err <= TOL, (name, float(err))


@pytest.mark.parametrize("lens", [[41, 41], [41, 17], [0, 41]])
def test_block_and_its_gradients(lens, cuda_device):
    p = _params(cuda_device)
    p64 = {k: v.detach().double().requires_grad_() for k, v in p.items()}
    g = torch.Generator().manual_seed(3)
    r = torch.randn(2, 41, WIDTH, generator=g).to(cuda_device).requires_grad_()
    r64 = r.detach().double().requires_grad_()
    go = torch.randn(2, 41, WIDTH, generator=g).to(cuda_device)
    n = torch.tensor(lens, dtype=torch.int32, device=cuda_device)
    y, (_, state) = block(p, r, n)
    want, h = plain(p64, r64, lens)
    _close("y", y, want)
    _close("state", state, h)
    (y * go).sum().backward()
    (want * go.double()).sum().backward()
    _close("r", r.grad, r64.grad)
    for k in p:
        _close(k, p[k].grad, p64[k].grad)


def test_a_stream_after_a_prompt(cuda_device):
    """Tokens one by one from the prompt's states give what the whole sequence gives."""
    p = {k: v.detach() for k, v in _params(cuda_device, 1).items()}
    r = torch.randn(3, 30, WIDTH, generator=torch.Generator().manual_seed(4)).to(cuda_device)
    whole, _ = block(p, r, None)
    cut = 25
    _, (conv, state) = block(p, r[:, :cut], None)
    for t in range(cut, 30):
        rt = r[:, t]
        y = torch.empty_like(rt)
        snn.snn_layer_norm_fwd(rt, p["ln_w"], p["ln_b"], y)
        xz = y @ p["w_in"].t()
        x, o = torch.empty(3, D, device=cuda_device), torch.empty(3, D, device=cuda_device)
        snn.snn_causal_conv_step(xz[:, :D], p["conv_w"], p["conv_b"], conv, x, act="silu")
        bc = (x @ p["w_bc"].t()).unflatten(-1, (2 * G, N))
        snn.snn_selective_scan_step(x, x @ p["w_delta"].t(), p["A"], bc[:, :G], bc[:, G:], state, o, D=p["skip"],
                                    z=xz[:, D:], delta_bias=p["bias"])
        _close(t, rt + o @ p["w_out"].t(), whole[:, t].double())


def test_a_training_step_in_a_graph(cuda_device):
    """Captured with its backward pass and replayed on other values: as issued."""
    p = _params(cuda_device, 2)
    r = torch.randn(2, 96, WIDTH, device=cuda_device)
    n = torch.tensor([96, 50], dtype=torch.int32, device=cuda_device)

    def step():
        y, _ = block(p, r, n)
        return [y.detach()] + list(torch.autograd.grad(y.square().sum(), list(p.values())))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    r.copy_(torch.randn_like(r))
    graph.replay()
    torch.cuda.synchronize()
    got = [x.clone() for x in out]
    for i, (a, b) in enumerate(zip(got, step())):
        # the projections' library products may take other algorithms in a graph
        _close(i, a, b.double())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_16_bit_gradients_against_32(dtype, cuda_device):
    """The same inputs (rounded first) in both types: apart by roundings of the results."""
    g = torch.Generator().manual_seed(6)
    r = lambda *s: torch.randn(s, generator=g).to(dtype).to(cuda_device)
    B, T = 2, 50
    x = dict(u=r(B, T, D), delta=r(B, T, D), B=r(B, T, G, N), C=r(B, T, G, N), z=r(B, T, D))
    A = -torch.rand(D, N, generator=g).to(cuda_device) - 0.1
    gy = r(B, T, D)
    grads = []
    for dt in (dtype, torch.float32):
        v = {k: t.detach().to(dt, copy=True).requires_grad_() for k, t in x.items()}
        a = A.clone().requires_grad_()
        y, _ = autograd.selective_scan(**v, A=a, delta_bias=torch.full((D,), -2.0, device=cuda_device))
        y.backward(gy.to(dt))
        grads.append([y.detach()] + [t.grad for t in v.values()] + [a.grad])
    half = torch.finfo(dtype).eps / 2
    for a, b in zip(*grads):
        limit = half + TOL if a.dtype == dtype else TOL
        assert (a.double() - b.double()).norm() <= limit * b.double().norm()
