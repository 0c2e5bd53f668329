"""Selective scan on the GPU against its float64 definition.

All arithmetic is fp32.  A result rounded to type t with half unit u_t (2^-8
bf16, 2^-11 fp16, 2^-24 fp32) errs by u_t |x| for the rounding and by c 2^-24
of the size of its sum of terms for the arithmetic.  A token's decay exp(s A) errs by
at most 8 + 12 |s A| units (the power of two 4, s from exp, reciprocal and series
8, products and log2(e) 4), its term by 12; over the tokens that a state remembers |s A|
adds up to a factor x e^-x < 1/2 of the term it is on.  So a state, or a gradient
of one, carries 64 + 10 T units; a product of the two, and a sum over states, channels
and tokens, 128 + 24 T.  Gates add 16 (their exp and reciprocal; 16-bit results: 40, the
rounding of z log2(e) for |z| < 8).
"""
import numpy as np
import pytest
import torch

from oracle import seq_oracle as O
from paper_2211_10725_gb300 import snn

pytestmark = pytest.mark.gpu

F32, BF, HF = torch.float32, torch.bfloat16, torch.float16
HALF_UNIT = {F32: 2.0 ** -24, BF: 2.0 ** -8, HF: 2.0 ** -11}
TINY = {F32: 1e-37, BF: 1e-37, HF: 2.0 ** -24}
NAN = float("nan")


def _np(t):
    return None if t is None else t.double().cpu().numpy()


def close(name, got, want, size, units, lost=0.0):
    """lost: what may be missing besides (a factor below the smallest normal number)."""
    dt = got.dtype
    err = np.abs(_np(got) - want)
    tol = HALF_UNIT[dt] * np.abs(want) + units * 2.0 ** -24 * size + TINY[dt] + lost
    assert (err <= tol).all(), (name, float(np.nanmax(err / tol)), int((~(err <= tol)).sum()))


class Case:
    """Inputs of a scan; pad > 0: parts of wider rows, with NaN around them."""

    def __init__(self, dev, B, T, D, N, dtype=BF, G=1, gate=True, softplus=True, bias=True, skip=True, lens=None,
                 state=True, pad=0, seed=0):
        g = torch.Generator().manual_seed(1000 * seed + 7 * B + T + D + N)
        self.B, self.T, self.D, self.N, self.G, self.dtype, self.dev = B, T, D, N, G, dtype, dev
        self.lens_list = lens

        def rows(*shape):
            x = torch.full((*shape[:2], *shape[2:-1], shape[-1] + pad), NAN, dtype=dtype)
            x[..., :shape[-1]] = torch.randn(shape, generator=g).to(dtype)
            return x.to(dev)[..., :shape[-1]]
        self.rows = rows
        self.u, self.delta = rows(B, T, D), rows(B, T, D)
        if not softplus:
            self.delta = (0.02 + 0.1 * self.delta.abs()).to(dtype)
        self.z = rows(B, T, D) if gate else None
        self.Bm, self.Cm = rows(B, T, G, N), rows(B, T, G, N)
        f = lambda *s: torch.randn(s, generator=g)
        self.A = -torch.exp(torch.log(torch.arange(1, N + 1).float()) + 0.1 * f(D, N)).to(dev)
        self.D_skip = (1 + 0.1 * f(D)).to(dev) if skip else None
        # without softplus s itself: positive, as exp(5 * 2.5 * T) has no fp32 value
        self.bias = (f(D) - 2.5 if softplus else 0.02 * f(D).abs()).to(dev) if bias else None
        self.state = f(B, D, N).to(dev) if state else None
        self.gy, self.gs = rows(B, T, D), f(B, D, N).to(dev)
        self.lens = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=dev)
        self.softplus = softplus
        self.shape = (B, T, D, N, G)
        if lens is not None:   # places past the end hold anything
            for x in (self.u, self.delta, self.Bm, self.Cm, self.gy) + ((self.z,) if gate else ()):
                for b, n in enumerate(lens):
                    x[b, max(n, 0):] = NAN
        self.kw = dict(D=self.D_skip, z=self.z, delta_bias=self.bias, softplus=softplus, seq_lens=self.lens)

    def oracle_args(self):
        ins = [_np(x) for x in (self.u, self.delta, self.A, self.Bm, self.Cm)]
        clean = [np.nan_to_num(x) for x in ins]
        z = None if self.z is None else np.nan_to_num(_np(self.z))
        return clean, dict(D=_np(self.D_skip), z=z, bias=_np(self.bias), softplus=self.softplus,
                           lens=self.lens_list, state=_np(self.state))

    def new(self, like):
        return torch.full(like.shape, NAN, dtype=like.dtype, device=self.dev)

    def forward(self, ckpt=False, stream=None):
        y = self.new(self.u)
        end = torch.full((self.B, self.D, self.N), NAN, device=self.dev)
        ws = torch.full((snn.snn_selective_scan_workspace_bytes(*self.shape),), 255, dtype=torch.uint8, device=self.dev)
        self.ckpt = torch.full((max(1, snn.snn_selective_scan_ckpt_elems(*self.shape)),), NAN, device=self.dev) \
            if ckpt else None
        snn.snn_selective_scan_fwd(self.u, self.delta, self.A, self.Bm, self.Cm, y, ws, state_in=self.state,
                                   state_out=end, ckpt=self.ckpt, stream=stream, **self.kw)
        return y, end

    def check_forward(self):
        y, end = self.forward(ckpt=True)
        args, kw = self.oracle_args()
        want = O.scan_forward(*args, **kw)
        size = O.scan_forward(*args, positive=True, **kw)
        units = 64 + 10 * self.T
        close("y", y, want[0], size[0], units + 64 + self.N)
        close("state", end, want[1], size[1], units)
        if self.lens_list:
            for b, n in enumerate(self.lens_list):
                assert torch.count_nonzero(y[b, max(n, 0):]) == 0

    def backward(self, gs=True, gs_in=True):
        o = {"u": self.new(self.u), "delta": self.new(self.u), "A": self.new(self.A), "B": self.new(self.Bm),
             "C": self.new(self.Cm), "D": None if self.D_skip is None else self.new(self.D_skip),
             "z": None if self.z is None else self.new(self.z),
             "bias": None if self.bias is None else self.new(self.bias),
             "state": self.new(self.gs) if gs_in else None}
        ws = torch.full((snn.snn_selective_scan_workspace_bytes(*self.shape, backward=True),), 255, dtype=torch.uint8,
                        device=self.dev)
        snn.snn_selective_scan_bwd(self.u, self.delta, self.A, self.Bm, self.Cm, self.gy, self.ckpt, o["u"],
                                   o["delta"], o["A"], o["B"], o["C"], ws, grad_state_out=self.gs if gs else None,
                                   grad_D=o["D"], grad_z=o["z"], grad_delta_bias=o["bias"],
                                   grad_state_in=o["state"], **self.kw)
        return o

    def check_backward(self, gs=True):
        self.forward(ckpt=True)
        got = self.backward(gs)
        args, kw = self.oracle_args()
        gy = np.nan_to_num(_np(self.gy))
        gstate = _np(self.gs) if gs else None
        want = O.scan_backward(*args, gy, gstate=gstate, **kw)
        size = O.scan_backward(*args, gy, gstate=gstate, positive=True, **kw)
        # sums over channels, sequences and tokens: their additions too
        units = 192 + 24 * self.T + self.N
        more = {"A": self.B * self.T, "D": self.B * self.T, "bias": self.B * self.T, "B": self.D, "C": self.D}
        for name, x in got.items():
            if x is not None:
                # softplus' slope e^x below x = -87.3 is under 2^-126 and may be zero
                lost = {"delta": size["s"], "bias": size["s"].sum((0, 1))}.get(name, 0.0) * 2.0 ** -126
                close(name, x, want[name], size[name], units + more.get(name, 0), lost)
        return got


@pytest.mark.parametrize("dtype", [F32, BF, HF])
@pytest.mark.parametrize("B,T,D,N,G", [(1, 1, 1, 1, 1), (2, 5, 8, 16, 1), (1, 33, 64, 16, 2), (2, 17, 66, 3, 1),
                                       (1, 130, 40, 8, 4), (2, 40, 36, 64, 2), (1, 24, 130, 20, 1)])
def test_sizes(B, T, D, N, G, dtype, cuda_device):
    c = Case(cuda_device, B, T, D, N, dtype, G)
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("N", list(range(1, 65, 3)) + [2, 12, 24, 32, 48])
def test_every_number_of_thread_states(N, cuda_device):
    c = Case(cuda_device, 1, 19, 10, N, F32, seed=1)
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("dtype", [F32, HF])
@pytest.mark.parametrize("D,G,pad", [(7, 1, 0), (9, 3, 0), (10, 1, 1), (12, 2, 5), (1, 1, 3), (15, 5, 1), (14, 2, 0)])
def test_odd_channels_and_strides(D, G, pad, dtype, cuda_device):
    c = Case(cuda_device, 2, 21, D, 6, dtype, G, pad=pad)
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("softplus,bias,skip,state", [(True, True, True, False), (True, False, False, True),
                                                      (False, True, True, True), (False, False, False, False)])
def test_absent_parts(gate, softplus, bias, skip, state, cuda_device):
    c = Case(cuda_device, 2, 30, 24, 5, BF, gate=gate, softplus=softplus, bias=bias, skip=skip, state=state)
    c.check_forward()
    c.check_backward()
    c.check_backward(gs=False)


@pytest.mark.parametrize("T,lens", [(40, [40, 0, 17, 1]), (16, [16, 8, 7, 9]), (300, [300, 64, 65, 0]), (9, [0, 0, 0, 0]),
                                    (5, [-3, 9, 5, 2])])
def test_padded_batches(T, lens, cuda_device):
    c = Case(cuda_device, 4, T, 18, 16, F32, lens=[min(max(n, 0), T) for n in lens], pad=2)
    c.lens = torch.tensor(lens, dtype=torch.int32, device=cuda_device)    # clamped by the call
    c.kw["seq_lens"] = c.lens
    c.check_forward()
    got = c.check_backward()
    for b, n in enumerate(lens):
        for name in ("u", "delta", "z", "B", "C"):
            assert torch.count_nonzero(got[name][b, max(n, 0):]) == 0


# long enough to be cut into spans, which end inside tiles, checkpoints and sequences
@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("B,T,D,N,G,lens", [(1, 1000, 8, 16, 1, None), (2, 777, 6, 10, 2, [777, 130]),
                                            (1, 515, 70, 4, 1, None), (3, 400, 20, 33, 1, [0, 400, 399])])
def test_spans(B, T, D, N, G, lens, dtype, cuda_device):
    c = Case(cuda_device, B, T, D, N, dtype, G, lens=lens)
    c.check_forward()
    c.check_backward()


@pytest.mark.parametrize("T", [127, 128, 129, 255, 1030])
@pytest.mark.parametrize("N", [5, 20, 64])
def test_short_spans(T, N, cuda_device):
    """Where cutting begins, spans that are no multiple of a tile, sequences that end in
    the first, in the middle of one, at a cut and in the last."""
    c = Case(cuda_device, 4, T, 10, N, F32, lens=[T, 16, 1, T - 3])
    c.check_forward()
    c.check_backward()


def test_tokens_of_no_length(cuda_device):
    c = Case(cuda_device, 2, 0, 8, 16, F32)
    _, end = c.forward(ckpt=True)
    assert torch.equal(end, c.state)
    got = c.backward()
    assert torch.equal(got["state"], c.gs)
    for name in ("A", "D", "bias"):
        assert torch.count_nonzero(got[name]) == 0


@pytest.mark.parametrize("T", [12, 900])
def test_state_in_place_and_slots(T, cuda_device):
    """Places in an order of their own, an empty one, and the state written over
    the one read (spans start from it side by side)."""
    c = Case(cuda_device, 3, T, 8, 16, F32)
    args, kw = c.oracle_args()
    pool = torch.randn(5, 8, 16, device=cuda_device)
    before = pool.clone()
    slots = torch.tensor([4, -1, 1], dtype=torch.int32, device=cuda_device)
    y = c.new(c.u)
    ws = torch.empty(snn.snn_selective_scan_workspace_bytes(*c.shape), dtype=torch.uint8, device=cuda_device)
    snn.snn_selective_scan_fwd(c.u, c.delta, c.A, c.Bm, c.Cm, y, ws, state_in=pool, state_out=pool, slots=slots, **c.kw)
    state = _np(before)[[4, 0, 1]]
    state[1] = 0
    kw["state"] = state
    want, h = O.scan_forward(*args, **kw)
    size, hs = O.scan_forward(*args, positive=True, **kw)
    close("y", y, want, size, 64 + 10 * T + 80)
    close("pool", pool[[4, 1]], h[[0, 2]], hs[[0, 2]], 64 + 10 * T)
    assert torch.equal(pool[[0, 2, 3]], before[[0, 2, 3]])


@pytest.mark.parametrize("dtype", [F32, BF, HF])
@pytest.mark.parametrize("B,D,N,G,pad", [(1, 1, 1, 1, 0), (3, 40, 16, 1, 0), (5, 33, 7, 3, 1), (2, 64, 64, 2, 0),
                                         (4, 300, 20, 1, 4), (2, 6, 50, 2, 3), (2, 512, 4, 1, 0)])
def test_steps(B, D, N, G, pad, dtype, cuda_device):
    c = Case(cuda_device, B, 1, D, N, dtype, G, pad=pad)
    pool = torch.randn(B + 2, D, N, device=cuda_device)
    before = pool.clone()
    at = [(3 * b + 1) % (B + 2) for b in range(B)] if (B + 2) % 3 else [B + 1 - b for b in range(B)]
    at[-1] = B + 2 if B > 1 else at[-1]          # outside: an empty place
    slots = torch.tensor(at, dtype=torch.int32, device=cuda_device)
    one = lambda x: None if x is None else x[:, 0]
    y = torch.full((B, D + pad), NAN, dtype=dtype, device=cuda_device)[:, :D]
    snn.snn_selective_scan_step(one(c.u), one(c.delta), c.A, one(c.Bm), one(c.Cm), pool, y, D=c.D_skip, z=one(c.z),
                                delta_bias=c.bias, slots=slots)
    used = [b for b in range(B) if at[b] < B + 2]
    args, kw = c.oracle_args()
    state = np.zeros((B, D, N))
    state[used] = _np(before)[[at[b] for b in used]]
    kw["state"], kw["lens"] = state, [int(b in used) for b in range(B)]
    want, h = O.scan_forward(*args, **kw)
    size, hs = O.scan_forward(*args, positive=True, **kw)
    close("y", y, want[:, 0], size[:, 0], 160 + N)
    for b in range(B + 2):
        if b in at:
            close("pool", pool[b], h[at.index(b)], hs[at.index(b)], 80)
        else:
            assert torch.equal(pool[b], before[b])


def test_steps_follow_a_prompt(cuda_device):
    """The last tokens one by one from the prompt's state: as the whole sequence."""
    B, T, D, N = 2, 70, 48, 16
    c = Case(cuda_device, B, T, D, N, F32)
    y, end = c.forward()
    p = Case(cuda_device, B, T, D, N, F32)
    cut = T - 3
    part = lambda x: None if x is None else x[:, :cut]
    kw = dict(D=c.D_skip, delta_bias=c.bias)
    y2, state = c.new(c.u), c.new(c.state)
    ws = torch.empty(snn.snn_selective_scan_workspace_bytes(B, cut, D, N), dtype=torch.uint8, device=cuda_device)
    snn.snn_selective_scan_fwd(part(c.u), part(c.delta), c.A, part(c.Bm), part(c.Cm), y2[:, :cut], ws, z=part(c.z),
                               state_in=c.state, state_out=state, **kw)
    for t in range(cut, T):
        one = lambda x: x[:, t]
        snn.snn_selective_scan_step(one(c.u), one(c.delta), c.A, one(c.Bm), one(c.Cm), state, y2[:, t], z=one(c.z), **kw)
    args, okw = c.oracle_args()
    size, hs = O.scan_forward(*args, positive=True, **okw)
    tol = (64 + 10 * T) * 2.0 ** -23
    assert (np.abs(_np(y2) - _np(y)) <= tol * size + 1e-37).all()
    assert (np.abs(_np(state) - _np(end)) <= tol * hs).all()


def test_far_values(cuda_device):
    """Large and small deltas: a step that forgets all, one that forgets nothing."""
    c = Case(cuda_device, 1, 24, 16, 16, F32, bias=False)
    c.delta[:, ::3] = 90.0
    c.delta[:, 1::3] = -95.0
    c.z[:, ::2] = -60.0
    c.z[:, 1::4] = 40.0
    c.check_forward()
    got = c.check_backward()
    assert all(torch.isfinite(x).all() for x in got.values() if x is not None)


def test_a_nan_stays_with_its_sequence_and_later_tokens(cuda_device):
    c = Case(cuda_device, 2, 20, 12, 8, F32)
    y0, end0 = c.forward()
    c.u[1, 9, 3] = NAN
    y, end = c.forward()
    hit = torch.zeros_like(y, dtype=torch.bool)
    hit[1, 9:, 3] = True
    assert torch.equal(torch.isnan(y), hit)
    assert torch.equal(y[~hit], y0[~hit])
    assert torch.equal(end[0], end0[0]) and torch.isnan(end[1, 3]).all()


def test_results_repeat_and_graphs_replay(cuda_device):
    c = Case(cuda_device, 2, 500, 40, 16, BF)
    c.forward(ckpt=True)
    first = c.backward()
    for name, x in c.backward().items():
        assert torch.equal(x, first[name]), name
    # captured on a stream of its own; other inputs at the replay
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c.forward(ckpt=True)
        c.backward()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, end = c.forward(ckpt=True)
        got = c.backward()
    graph.replay()
    torch.cuda.synchronize()
    for name, x in got.items():
        assert torch.equal(x, first[name]), name
    c.u.copy_(torch.randn_like(c.u))
    graph.replay()
    y2, end2 = c.forward(ckpt=True)
    second = c.backward()
    assert torch.equal(y, y2) and torch.equal(end, end2)
    for name, x in got.items():
        assert torch.equal(x, second[name]), name


def test_two_calls_at_once(cuda_device):
    """Workspaces of their own on streams of their own."""
    cases = [Case(cuda_device, 1, 2000, 64, 16, BF, seed=i) for i in range(2)]
    want = [c.forward() for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = []
    for c, s in zip(cases, streams):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            got.append(c.forward())
    torch.cuda.synchronize()
    for w, x in zip(want, got):
        assert torch.equal(w[0], x[0]) and torch.equal(w[1], x[1])


def test_refusals_of_the_binding(cuda_device):
    c = Case(cuda_device, 2, 8, 16, 4, BF)
    ws = torch.empty(1 << 16, dtype=torch.uint8, device=cuda_device)
    y = c.new(c.u)
    call = lambda u=c.u, delta=c.delta, A=c.A, B=c.Bm, C=c.Cm, y=y, ws=ws, **kw: snn.snn_selective_scan_fwd(
        u, delta, A, B, C, y, ws, **kw)
    call()
    for bad in (dict(delta=c.delta.float()), dict(A=c.A.t()), dict(B=c.Bm[:, :, :, :3]), dict(y=y.cpu()),
                dict(u=c.u.transpose(1, 2).contiguous().transpose(1, 2)), dict(D=c.A[:, 0]),
                dict(slots=torch.zeros(2, dtype=torch.int64, device=cuda_device)),
                dict(state_in=torch.zeros(3, 16, 4, device=cuda_device)),
                dict(ckpt=torch.zeros(8, device=cuda_device))):
        with pytest.raises(ValueError):
            call(**bad)
    with pytest.raises(snn.SnnError):
        call(u=c.u[:1].expand(2, 8, 16))
