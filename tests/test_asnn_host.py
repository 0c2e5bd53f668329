"""Host-side sequencing of the sequence network (no GPU needed): the launches of
a training step, and the views its operators read and write in place."""
import pytest
import torch

from paper_2211_10725_gb300 import build_lib, snn
from paper_2211_10725_gb300 import workloads as W
from paper_2211_10725_gb300.asnn import AttnSNN


@pytest.fixture(autouse=True)
def host_only(monkeypatch):
    build_lib.build()
    monkeypatch.setattr(snn, "snn_workspace_init", lambda *a, **k: None)


def _net(**over):
    w = W.ASNN.scaled(**{**dict(T=8, B=4, n_in=24, head_dim=16), **over})
    return w, AttnSNN(w, W.make_attn_inputs(w)["W"], device="cpu")


def test_launch_order():
    _, net = _net()
    assert [n for n, _ in net.ops(None, None)] == [
        "dense_in", "norm_in", "dense0", "scan0", "attn0", "norm0", "dense1", "scan1", "attn1",
        "norm1", "dense_out", "scan_out", "ce_loss", "dense_out_bwd", "norm_bwd1", "attn_bwd1",
        "scan_bwd1", "dense_bwd1", "norm_bwd0", "attn_bwd0", "scan_bwd0", "dense_bwd0",
        "norm_in_bwd", "cast_in", "dense_in_bwd", "adamw"]


def test_queries_keys_and_values_are_views_of_the_spikes():
    w, net = _net()
    spk = net.scans[0].spk
    spk.copy_(torch.arange(spk.numel()).view_as(spk) % 251)
    q, k, v = net._qkv(spk)
    assert q.shape == (w.B, w.T, w.heads, w.head_dim)
    assert k.shape == v.shape == (w.B, w.T, w.kv_heads, w.head_dim)
    D, at = w.head_dim, w.heads * w.head_dim
    for t, b, h in ((0, 0, 0), (3, 2, 1), (7, 3, 1)):
        assert torch.equal(q[b, t, h], spk[t, b, h * D:(h + 1) * D])
        assert torch.equal(k[b, t, h], spk[t, b, at + h * D:at + (h + 1) * D])
        at_v = at + w.kv_heads * D
        assert torch.equal(v[b, t, h], spk[t, b, at_v + h * D:at_v + (h + 1) * D])
    assert q.data_ptr() == spk.data_ptr()


def test_parameters_share_one_buffer_each():
    w, net = _net()
    assert len(net.weights.parts) == w.blocks + 2 and len(net.norms.parts) == 3 * w.blocks + 1
    for f in (net.weights, net.norms):
        # 64-element boundaries of the buffer (whose own address is the allocator's)
        assert all((p.data_ptr() - f.grad.data_ptr()) % 256 == 0 for p in f.grads)
    assert torch.equal(net.weights.parts[0], W.make_attn_inputs(w)["W"][0])
    assert net.weights.parts[-1].shape == (16, w.width)
    assert torch.count_nonzero(net.weights.parts[-1][w.n_classes:]) == 0


class _Queue:
    """A stream whose work waits until something torch does is ordered behind it."""

    def __init__(self):
        self.work = []

    def __enter__(self):      # torch.cuda.stream(queue): torch's calls come after what is queued
        for call in self.work:
            call()
        self.work = []

    def __exit__(self, *exc):
        pass


def test_a_prompt_on_a_stream_keeps_what_that_stream_computes(monkeypatch):
    w, net = _net()
    for name in ("snn_dense_layer_fwd", "snn_block_norm_fwd", "snn_leaky_attn_fwd"):
        monkeypatch.setattr(snn, name, lambda *a, **k: None)
    monkeypatch.setattr(snn.ScanLayer, "forward", lambda self, *a, stream=None, **k: stream.work.append(
        lambda: self.mem_final.fill_(7.0)))
    monkeypatch.setattr(torch.cuda, "stream", lambda s: s)
    allocated = []
    monkeypatch.setattr(snn, "snn_workspace_init", lambda *a, **k: allocated.append(a))
    net.prompt(torch.zeros(w.T * w.B, w.n_in, dtype=torch.bfloat16), stream=_Queue())
    assert len(net.mem) == w.blocks + 1
    for mem in net.mem:
        assert torch.all(mem == 7.0)
    assert not allocated       # nothing is set up on a stream that is not the caller's
