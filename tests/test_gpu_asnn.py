"""The sequence network: its forward stage by stage, its reverse pass against
torch's engine over the autograd wrappers, streaming against the whole
sequence, and training."""
import numpy as np
import pytest
import torch

from oracle import attn_oracle as A
from paper_2211_10725_gb300 import autograd as G
from paper_2211_10725_gb300 import snn
from paper_2211_10725_gb300 import workloads as W
from paper_2211_10725_gb300.asnn import EPS, AttnSNN, head_decays

pytestmark = pytest.mark.gpu

SMALL = W.ASNN.scaled(name="asnn_small", T=70, B=8, n_in=72, heads=4, kv_heads=2, head_dim=32,
                      blocks=2)


def _net(w, dev, seed=None):
    inp = W.make_attn_inputs(w, seed)
    X = inp["X"].view(w.T * w.B, -1).to(dev)
    return AttnSNN(w, inp["W"], device=dev), X, inp["labels"].to(dev)


def _f64(t):
    return t.detach().double().cpu().numpy()


def test_forward_stages(cuda_device):
    """Each stage from the network's own inputs to it, so that one stage's
    rounding does not flip another's spikes."""
    w = SMALL
    net, X, labels = _net(w, cuda_device)
    net.prompt(X)
    S, N, D = w.spikes, w.width, w.head_dim
    for l in range(w.blocks):
        sc = net.scans[l]
        assert 0.01 < sc.spk[..., :S].float().mean() < 0.9
        q, k, v = (_f64(t) for t in net._qkv(sc.spk))
        o, end = A.attn_forward(q, k, v, _f64(net.decay), D ** -0.5)
        size, end_size = A.attn_forward_size(q, k, v, _f64(net.decay), D ** -0.5)
        got = _f64(net._heads(net.o[l]))
        assert (np.abs(got - o) <= 5 * 2.0 ** -8 * size + 1e-30).all()
        assert (np.abs(_f64(net.state[l]) - end) <= 2.0 ** -16 * end_size).all()
        wp, rs, pre = (_f64(t) for t in net._norm_args(l))
        z = _f64(sc.mem.view(net.M, -1)[:, S:])
        r2, y = A.block_norm_forward(_f64(net.r[l]), _f64(net.o[l].view(net.M, -1)), z, wp, rs, pre, EPS,
                                     D, "silu")
        big = np.abs(_f64(net.r[l])) + np.abs(r2 - _f64(net.r[l]))
        assert (np.abs(_f64(net.r[l + 1]) - r2) <= 2.0 ** -18 * big + 1e-30).all()
        f = A._factor(r2, N, EPS)
        assert (np.abs(_f64(net.y[l + 1]) - y) <= 2.0 ** -8 * np.abs(y) + 2.0 ** -18 * big * f).all()


def test_reverse_pass_matches_torch_engine(cuda_device):
    """The same network written with the autograd wrappers and torch's
    matmul.  Its products are in fp32 from the same bf16 values, so currents
    agree to fp32 rounding and the spikes do unless a potential lies that
    close to the threshold; the gradients then differ by the roundings to
    bf16 that both sides take between the stages, each 2^-8 of a term: eight
    stages deep, 8 * 2^-8 in the norm over a weight's elements."""
    w = SMALL
    net, X, labels = _net(w, cuda_device)
    got = [g.clone() for g in net.gradients(X, labels)]
    norms = [g.clone() for g in net.norms.grads]
    T, B, S, D = w.T, w.B, w.spikes, w.head_dim
    leaf = lambda t: t.detach().clone().requires_grad_()
    Wp = [leaf(p) for p in net.weights.parts]
    Np = [leaf(p) for p in net.norms.parts]

    def scan(I, n):
        sw = W.ScanWorkload(name="ref", neuron="leaky", T=T, B=B, N=n, in_dtype=W.F32, io_dtype=W.BF16,
                            surrogate="fast_sigmoid", sg_param=w.sg_param, save="mem", want_mem=True)
        return sw, G.scan(I.view(T, B, n), net.beta, net.thr, sw)

    class Mem(torch.autograd.Function):   # the membrane trace, with its gradient
        @staticmethod
        def forward(ctx, I, sw):
            layer = snn.ScanLayer(sw, device=I.device)
            layer.forward(I.contiguous(), net.beta, net.thr)
            ctx.layer = layer
            return layer.mem.clone()

        @staticmethod
        def backward(ctx, g):
            layer = ctx.layer
            zero = torch.zeros_like(layer.spk)
            layer.backward(None, net.beta, net.thr, zero, grad_mem=g.to(torch.bfloat16).contiguous(),
                           want_param_grads=False, want_state_grads=False)
            return layer.grad_I.float(), None

    r = X.float() @ Wp[0].float().t()
    y = (r * torch.rsqrt(r.square().mean(-1, keepdim=True) + EPS) * Np[0]).to(torch.bfloat16)
    for l in range(w.blocks):
        I = y.float() @ Wp[l + 1].float().t()
        sw, spk = scan(I, S + w.width)
        assert (spk != net.scans[l].spk).float().mean() < 1e-3
        z = Mem.apply(I.view(T, B, -1), sw)[..., S:].reshape(T * B, -1)
        q, k, v = net._qkv(spk)
        o, _ = G.leaky_attention(q, k, v, net.decay, scale=D ** -0.5)
        a = o.transpose(0, 1).reshape(T * B, -1)
        r, y = G.block_norm(r, a, z, Np[3 * l + 1], Np[3 * l + 2], Np[3 * l + 3], eps=EPS, group=D,
                            gate="silu")
    _, spk = scan(y.float() @ Wp[-1].float().t(), net.n_out)
    counts = spk.float().sum(0)[:, :w.n_classes]
    loss = torch.nn.functional.cross_entropy(counts, labels.long())
    loss.backward()
    assert abs(loss.item() - net.loss.item()) < 0.05 * abs(loss.item())
    for name, g, p in [(f"W{i}", g, p) for i, (g, p) in enumerate(zip(got, Wp))] + \
                      [(f"norm{i}", g, p) for i, (g, p) in enumerate(zip(norms, Np))]:
        ref = p.grad.double()
        assert (g.double() - ref).norm() <= 8 * 2.0 ** -8 * ref.norm() + 1e-12, name


def test_streaming_goes_on_from_the_prompt(cuda_device):
    """The last steps one at a time: the first block's spikes are exactly the
    whole sequence's (they depend on the input alone), its attention agrees to
    the two forms' roundings."""
    w = SMALL
    whole, X, labels = _net(w, cuda_device)
    whole.prompt(X)
    first = w.scaled(T=w.T - 3)
    inp = W.make_attn_inputs(w)
    net = AttnSNN(first, inp["W"], device=cuda_device)
    x = X.view(w.T, w.B, -1)
    net.prompt(x[:first.T].reshape(-1, w.n_in).contiguous())
    for t in range(first.T, w.T):
        out = net.token(x[t].contiguous())
        assert out.shape == (w.B, w.n_classes)
        q, k, v = (_f64(a) for a in whole._qkv(whole.scans[0].spk))
        size, _ = A.attn_forward_size(q[:, :t + 1], k[:, :t + 1], v[:, :t + 1], _f64(net.decay),
                                      w.head_dim ** -0.5)
        want = _f64(whole.o[0][t])
        got = _f64(net.token_o[0])
        assert torch.equal(net._token["scans"][0].spk[0], whole.scans[0].spk[t])
        assert (np.abs(got - want) <= 6 * 2.0 ** -8 * size[:, t].reshape(w.B, -1) + 1e-30).all()
    err = np.abs(_f64(net.state[0]) - _f64(whole.state[0]))
    scale = np.abs(_f64(whole.state[0])).max()
    assert err.max() <= 2.0 ** -14 * scale


def test_training_lowers_the_loss_and_graph_replays(cuda_device):
    w = SMALL
    net, X, labels = _net(w, cuda_device)
    first = net.train_step(X, labels).item()
    assert snn.snn_workspace_status(net.ws_attn) == 0
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        net.train_step(X, labels)
    for _ in range(60):
        graph.replay()
    torch.cuda.synchronize()
    assert snn.snn_workspace_status(net.ws_attn) == 0
    assert net.loss.item() < 0.7 * first


def test_head_decays_are_a_schedule():
    d = head_decays(4)
    assert torch.equal(d, torch.tensor([1 - 1 / 8, 1 - 1 / 16, 1 - 1 / 32, 1 - 1 / 64]))


def test_prompt_and_tokens_on_a_side_stream(cuda_device):
    """On a stream that is kept busy first, with nothing else waiting for it."""
    w = SMALL
    n = w.T - 2
    inp = W.make_attn_inputs(w)
    x = inp["X"].to(cuda_device)
    outs = []
    for side in (None, torch.cuda.Stream()):
        net = AttnSNN(w.scaled(T=n), inp["W"], device=cuda_device)
        big = torch.randn(8192, 8192, device=cuda_device)
        torch.cuda.synchronize()
        if side is not None:
            with torch.cuda.stream(side):
                for _ in range(8):
                    big = big @ big
        net.prompt(x[:n].reshape(-1, w.n_in).contiguous(), stream=side)
        for t in range(n, w.T):
            net.token(x[t], stream=side)
        torch.cuda.synchronize()
        outs.append([*(t.clone() for t in net.mem), *(t.clone() for t in net.state),
                     *(t.clone() for t in net.token_o)])
    assert all(torch.equal(a, b) for a, b in zip(*outs))
