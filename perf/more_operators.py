"""Cases of the selective scan (a leaky scan whose leak follows its input, with
a diagonal state for every channel), of the short causal convolution before it and
of the layer norm around the block, in plain torch and through the library.

Selective scan, for channel d of group g and its N states n:
    s_t    = softplus(delta_t + delta_bias)
    h_t[n] = exp(s_t A[d, n]) h_{t-1}[n] + s_t u_t B_t[g, n]
    y_t    = (sum_n C_t[g, n] h_t[n] + D_d u_t) silu(z_t)
over u, delta, z [B, T, D] and B, C [B, T, G, N].  Causal convolution of each
channel: y_t = silu(bias + sum_j w[j] x_{t-W+1+j}), the W - 1 inputs before the
sequence from a state.  Tokens at t >= seq_lens[b] do not exist: their outputs
and gradients are zero and the states pass over them.  Layer norm, per row:
    y = (x - mean) / sqrt(var + eps) * w + b.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
CHUNK = 64
EPS = 1e-5


# --------------------------------------------------------------------------
# cases
# --------------------------------------------------------------------------

def scan(name, kind, B, T, D, N, dtype, G=1, gate=True, ragged=False):
    return {"name": name, "kind": "scan_" + kind, "B": B, "T": T, "D": D, "N": N, "G": G,
            "dtype": dtype, "gate": gate, "ragged": ragged}


def conv(name, kind, B, T, C, W, dtype, ragged=False):
    return {"name": name, "kind": "conv_" + kind, "B": B, "T": T, "C": C, "W": W, "dtype": dtype,
            "ragged": ragged}


def norm(name, kind, M, N, dtype, res):
    return {"name": name, "kind": "ln_" + kind, "M": M, "N": N, "dtype": dtype, "res": res}


def listed():
    return [
        # one user's next token, a small model's layer: latency
        scan("scan_token_one", "step", 1, 1, 1024, 16, "bf16"),
        # a full serving batch in a pool of states: the states' bandwidth
        scan("scan_token_batch", "step", 192, 1, 5120, 16, "bf16", ragged=True),
        # a short prompt for one user
        scan("scan_prompt_short", "prefill", 1, 100, 1024, 16, "bf16"),
        # one long document: few channels for the GPU, a long axis
        scan("scan_prompt_long", "prefill", 1, 16384, 2048, 16, "bf16"),
        # a training step on padded samples, two groups, an odd number of states
        scan("scan_train_ragged", "train", 3, 777, 1000, 20, "f16", G=2, ragged=True),
        # a training step of ordinary size, forward and backward
        scan("scan_train_full", "train", 2, 4096, 4096, 16, "bf16"),
        # a serving batch's next tokens
        conv("conv_token", "step", 64, 1, 4096, 4, "bf16", ragged=True),
        # prompts of several users, padded to the longest
        conv("conv_prompt_ragged", "prefill", 6, 1500, 2056, 3, "f16", ragged=True),
        # a training step, forward and backward
        conv("conv_train", "train", 2, 4096, 4096, 4, "bf16"),
        # the norm before one token's block
        norm("ln_one", "fwd", 1, 1000, "bf16", "bf16"),
        # the norm of a long prompt, 16-bit activations from a 32-bit residual stream
        norm("ln_prompt", "fwd", 16384, 4096, "bf16", "f32"),
        # a training step's norm, forward and backward
        norm("ln_train", "train", 16384, 2048, "bf16", "bf16"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["scan", "scan", "conv", "ln"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "ln":
        kind = rng.choice(["fwd", "train"])
        N = _log(rng, 48, 8192)
        if rng.random() < 0.7:
            N = 8 * max(1, N // 8)
        most = 16384 * (2048 if kind == "train" else 4096) // (2 if dtype == "f32" else 1)
        res = rng.choice([dtype, "f32"])
        if kind == "train" and res == "f32":
            most //= 2
        return {"kind": "ln_" + kind, "M": _log(rng, 1, max(1, min(32768, most // N))), "N": N,
                "dtype": dtype, "res": res}
    kind = rng.choice(["step", "prefill", "train"])
    width = _log(rng, 32, 8192)
    if rng.random() < 0.8:
        width = 8 * max(1, width // 8)
    T, B = 1, 1
    if op == "conv":
        most = (2 * 4096 * 4096) // (width * (2 if dtype == "f32" else 1))
        if kind == "step":
            B = _log(rng, 1, min(256, most))
        else:
            B = rng.randint(1, 8)
            T = _log(rng, 1, max(1, min(16384, most // B)))
        return {"kind": "conv_" + kind, "B": B, "T": T, "C": width, "W": rng.choice([2, 3, 4, 4]),
                "dtype": dtype, "ragged": B > 1 and rng.random() < 0.5}
    N = rng.choice([16, 16, 16, 8, 32, 64, rng.randint(1, 64)])
    G = rng.choice([1, 1, 1, 2, 4])
    width = G * max(1, width // G)
    if kind == "step":
        B = _log(rng, 1, max(1, min(256, 192 * 5120 * 16 // (width * N))))
    else:
        # a step of few tokens costs more for each of them: half of the largest case's work
        most = (2 * 4096 * 4096 * 16) // (2 * width * 16 * -(-N // 16)) // (2 if dtype == "f32" else 1)
        B = rng.randint(1, 8)
        T = _log(rng, 1, max(1, min(16384 if kind == "prefill" else 4096, most // B)))
    return {"kind": "scan_" + kind, "B": B, "T": T, "D": width, "N": N, "G": G, "dtype": dtype,
            "gate": rng.random() < 0.75, "ragged": B > 1 and rng.random() < 0.5}


def work(case):
    e = SIZE[case["dtype"]]
    kind = case["kind"]
    if kind.startswith("ln"):
        M, N, r = case["M"], case["N"], SIZE[case["res"]]
        if kind == "ln_fwd":
            return {"bytes": M * N * (r + e) + 8 * N, "flops": 8 * M * N}
        # x in, y out; dy in, dx and the parameters' gradients out
        return {"bytes": M * N * (2 * r + 2 * e) + 16 * N, "flops": 22 * M * N}
    B, T = case["B"], case["T"]
    n = B * T
    if kind.endswith("step"):
        n = sum(1 for s in _slots(case) if s >= 0) if case["ragged"] else B
    elif case["ragged"]:
        n = sum(_lens(case))
    if kind.startswith("conv"):
        C, W = case["C"], case["W"]
        par = 4 * C * (W + 1)
        if kind == "conv_step":
            return {"bytes": e * C * (n + B + 2 * n * (W - 1)) + par, "flops": n * C * (2 * W + 5)}
        if kind == "conv_prefill":
            return {"bytes": e * C * (n + B * T + 2 * B * (W - 1)) + par, "flops": n * C * (2 * W + 5)}
        # x in, y out, dy in, dx out
        return {"bytes": e * C * 2 * (n + B * T) + 2 * par, "flops": n * C * (8 * W + 16)}
    D, N, G, z = case["D"], case["N"], case["G"], 1 if case["gate"] else 0
    par = 4 * D * (N + 2)
    io = e * (D * (2 + z) + 2 * G * N)
    if kind == "scan_step":
        return {"bytes": n * io + e * B * D + 8 * n * D * N + par, "flops": 7 * n * D * N}
    if kind == "scan_prefill":
        return {"bytes": n * io + e * B * T * D + 8 * B * D * N + par, "flops": 7 * n * D * N}
    grads = e * B * T * (D * (2 + z) + 2 * G * N)
    return {"bytes": n * io + e * B * T * D + e * n * D + grads + 2 * par, "flops": 34 * n * D * N}


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

def _lens(case):
    """Lengths of a padded batch: the longest, an empty place, the rest spread."""
    B, T = case["B"], case["T"]
    return [T, 0][:B] + [max(1, (T * (2 * b + 3)) // (2 * B + 3)) for b in range(2, B)]


def _slots(case):
    """Places of a batch in the pool of states, in an order of its own; every
    fifth place of a ragged batch is empty (-1)."""
    B = case["B"]
    step = next(s for s in (7, 5, 3, 1) if math.gcd(s, B + 3) == 1)
    at = [(1 + step * b) % (B + 3) for b in range(B)]
    return [-1 if case["ragged"] and b % 5 == 3 else at[b] for b in range(B)]


def _pad8(n):
    return (n + 7) // 8 * 8


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g, device=dev)  # noqa: E731
    dt = DTYPES[case["dtype"]]
    kind = case["kind"]
    st = {"case": case}
    if kind.startswith("ln"):
        M, N = case["M"], case["N"]
        st |= {"x": (2.0 * rand(M, N) + 0.3).to(DTYPES[case["res"]]), "w": 1.0 + 0.1 * rand(N),
               "b": 0.1 * rand(N)}
        if kind == "ln_train":
            st["grad_y"] = (0.05 * rand(M, N)).to(dt)
        return st
    B, T = case["B"], case["T"]
    st["lens"] = st["slots"] = None
    if kind.endswith("step"):
        st["slots"] = torch.tensor(_slots(case), dtype=torch.int32, device=dev)
    elif case["ragged"]:
        st["lens"] = torch.tensor(_lens(case), dtype=torch.int32, device=dev)
    if kind.startswith("conv"):
        C, W = case["C"], case["W"]
        # the convolution's input is a part of a projection's rows
        st["x"] = rand(B, T, 2 * _pad8(C)).to(dt)[..., :C]
        st["w"], st["b"] = rand(C, W) * W ** -0.5, 0.1 * rand(C)
        if kind == "conv_step":
            st["x"], st["pool"] = st["x"][:, 0], rand(B + 3, W - 1, C).to(dt)
        elif kind == "conv_prefill":
            st["state"] = rand(B, W - 1, C).to(dt)
        else:
            st["grad_y"] = (0.1 * rand(B, T, C)).to(dt)
        return st
    D, N, G = case["D"], case["N"], case["G"]
    st["u"] = torch.nn.functional.silu(rand(B, T, D)).to(dt)
    # the gate is a part of a projection's rows, B and C are parts of another's; parts
    # start on whole vectors
    half, part = _pad8(D), _pad8(G * N)
    st["z"] = rand(B, T, 2 * half).to(dt)[..., half:half + D] if case["gate"] else None
    st["delta"] = (0.5 * rand(B, T, D)).to(dt)
    bc = rand(B, T, 2 * part).to(dt)
    st["Bm"], st["Cm"] = (bc[..., i:i + G * N].unflatten(-1, (G, N)) for i in (0, part))
    # memories from about one step to a thousand
    st["A"] = -torch.exp(torch.log(torch.arange(1, N + 1, device=dev).float()) + 0.05 * rand(D, N))
    step = torch.exp(torch.rand(D, generator=g, device=dev) * math.log(100.0) + math.log(1e-3))
    st["delta_bias"] = torch.log(torch.expm1(step))
    st["D"] = 1.0 + 0.1 * rand(D)
    if kind == "scan_step":
        for x in ("u", "z", "delta", "Bm", "Cm"):
            st[x] = None if st[x] is None else st[x][:, 0]
        st["pool"] = rand(B + 3, D, N)
    elif kind == "scan_prefill":
        st["state"] = rand(B, D, N)
    else:
        st["grad_y"] = (0.1 * rand(B, T, D)).to(dt)
    return st


# --------------------------------------------------------------------------
# plain forms
# --------------------------------------------------------------------------

def _softplus(x):
    return x.clamp(min=0) + torch.log1p(torch.exp(-x.abs()))


def _silu(x):
    return x * torch.sigmoid(x)


def _silu_slope(x):
    s = torch.sigmoid(x)
    return s * (1 + x * (1 - s))


class _Spans:
    """A batch of sequences in 32 bits, cut into spans of CHUNK tokens that go
    through their tokens side by side: [B, spans, G, channels of a group, ...]."""

    def __init__(self, st):
        c = st["case"]
        self.B, self.T, self.G, self.Dg, self.N = c["B"], c["T"], c["G"], c["D"] // c["G"], c["N"]
        self.n = -(-self.T // CHUNK)
        t = torch.arange(self.T, device=st["u"].device)
        self.valid = None if st["lens"] is None else t[None] < st["lens"][:, None]   # [B, T]
        self.A = st["A"].view(self.G, self.Dg, self.N)
        s = _softplus(st["delta"].float() + st["delta_bias"])
        self.s = self.cut(s).unflatten(-1, (self.G, self.Dg))
        self.u = self.cut(st["u"].float()).unflatten(-1, (self.G, self.Dg))
        self.su = self.s * self.u
        self.Bm, self.Cm = self.cut(st["Bm"].float()), self.cut(st["Cm"].float())
        self.decay = torch.exp(self.s.sum(2)[..., None] * self.A)   # over a whole span

    def cut(self, x):
        """[B, T, ...] -> [B, spans, CHUNK, ...], zero where there is no token."""
        if self.valid is not None:
            x = torch.where(self.valid.view(self.B, self.T, *([1] * (x.dim() - 2))), x,
                            torch.zeros((), device=x.device))
        pad = torch.zeros(self.B, self.n * CHUNK - self.T, *x.shape[2:], device=x.device)
        return torch.cat([x, pad], 1).unflatten(1, (self.n, CHUNK))

    def join(self, x):
        """[B, spans, CHUNK, ...] -> [B, T, ...], zero where there is no token."""
        x = x.flatten(1, 2)[:, :self.T]
        if self.valid is None:
            return x
        return torch.where(self.valid.view(self.B, self.T, *([1] * (x.dim() - 2))), x,
                           torch.zeros((), device=x.device))

    def a(self, i):
        return torch.exp(self.s[:, :, i, ..., None] * self.A)

    def add(self, i):
        return self.su[:, :, i, ..., None] * self.Bm[:, :, i, :, None, :]

    def over_tokens(self, h, keep=False):
        """States after each span from those before it, y, and the states after
        each token if they are to be kept."""
        ys, hs = [], []
        for i in range(CHUNK):
            h = self.a(i) * h + self.add(i)
            ys.append((h * self.Cm[:, :, i, :, None, :]).sum(-1))
            if keep:
                hs.append(h)
        return h, torch.stack(ys, 2), hs

    def starts(self, state):
        """States before each span, and the last one."""
        h = torch.zeros(self.B, self.n, self.G, self.Dg, self.N, device=self.s.device)
        for i in range(CHUNK):
            h = self.a(i) * h + self.add(i)
        at = torch.zeros_like(h[:, 0]) if state is None else state.view(h[:, 0].shape).float()
        out = []
        for j in range(self.n):
            out.append(at)
            at = self.decay[:, j] * at + h[:, j]
        return torch.stack(out, 1), at

    def ends(self, dy):
        """Gradients that reach each span's last state from the tokens after it."""
        g = torch.zeros(self.B, self.n, self.G, self.Dg, self.N, device=dy.device)
        for i in reversed(range(CHUNK)):
            g = self.a(i) * (g + dy[:, :, i, ..., None] * self.Cm[:, :, i, :, None, :])
        at, out = torch.zeros_like(g[:, 0]), []
        for j in reversed(range(self.n)):
            out.append(at)
            at = self.decay[:, j] * at + g[:, j]
        return torch.stack(out[::-1], 1)


def _gated(st, y):
    y = y + st["D"] * st["u"].float()
    return y if st["z"] is None else y * _silu(st["z"].float())


def _existing(sp, x):
    return x if sp.valid is None else torch.where(sp.valid[..., None], x,
                                                  torch.zeros((), device=x.device))


def plain_scan_step(st):
    G, pool, slots = st["case"]["G"], st["pool"], st["slots"].long()
    used = slots >= 0
    s = _softplus(st["delta"].float() + st["delta_bias"])
    u = st["u"].float()
    per = u.shape[-1] // G
    Bm, Cm = (st[x].float().repeat_interleave(per, 1) for x in ("Bm", "Cm"))
    h = torch.exp(s[..., None] * st["A"]) * pool[slots.clamp(min=0)] + (s * u)[..., None] * Bm
    y = _gated(st, (h * Cm).sum(-1))
    y = torch.where(used[:, None], y, torch.zeros((), device=y.device))
    pool.index_copy_(0, slots[used], h[used])
    return {"y": y.to(st["u"].dtype), "pool": pool}


def plain_scan_prefill(st):
    sp = _Spans(st)
    h, end = sp.starts(st["state"])
    y = sp.join(sp.over_tokens(h)[1]).flatten(2)
    return {"y": _existing(sp, _gated(st, y)).to(st["u"].dtype), "state": end.flatten(1, 2)}


def plain_scan_train(st):
    sp = _Spans(st)
    dt = st["u"].dtype
    h0, _ = sp.starts(None)
    _, y, hs = sp.over_tokens(h0, keep=True)
    plain = sp.join(y).flatten(2)
    out = {"y": _existing(sp, _gated(st, plain)).to(dt)}
    do, u = _existing(sp, st["grad_y"].float()), _existing(sp, st["u"].float())
    dy = do
    if st["z"] is not None:
        z = st["z"].float()
        out["dz"] = _existing(sp, do * (plain + st["D"] * u) * _silu_slope(z)).to(dt)
        dy = _existing(sp, do * _silu(z))
    out["dD"] = (dy * u).sum((0, 1))
    dyc = sp.cut(dy).unflatten(-1, (sp.G, sp.Dg))
    g = sp.ends(dyc)
    dA = torch.zeros_like(sp.A)
    dB, dC, ds, du = [], [], [], []
    for i in reversed(range(CHUNK)):
        a, Bm = sp.a(i), sp.Bm[:, :, i, :, None, :]
        g = g + dyc[:, :, i, ..., None] * sp.Cm[:, :, i, :, None, :]
        dC.append((dyc[:, :, i, ..., None] * hs[i]).sum(-2))
        dB.append((sp.su[:, :, i, ..., None] * g).sum(-2))
        w = (g * Bm).sum(-1)
        q = g * a * (hs[i - 1] if i else h0)
        ds.append(sp.u[:, :, i] * w + (q * sp.A).sum(-1))
        du.append(sp.s[:, :, i] * w)
        dA += (q * sp.s[:, :, i, ..., None]).sum((0, 1))
        g = a * g
    whole = lambda x: sp.join(torch.stack(x[::-1], 2))  # noqa: E731
    slope = torch.sigmoid(st["delta"].float() + st["delta_bias"])
    ddelta = _existing(sp, whole(ds).flatten(2) * slope)
    out |= {"du": _existing(sp, whole(du).flatten(2) + st["D"] * dy).to(dt),
            "ddelta": ddelta.to(dt), "ddelta_bias": ddelta.sum((0, 1)), "dA": dA.flatten(0, 1),
            "dB": whole(dB).to(dt), "dC": whole(dC).to(dt)}
    return out


def _conv_rows(st):
    """Inputs with the W - 1 before them, zero where there is no token."""
    c, x = st["case"], st["x"].float()
    if st["lens"] is not None:
        live = torch.arange(c["T"], device=x.device)[None] < st["lens"][:, None]
        x = torch.where(live[..., None], x, torch.zeros((), device=x.device))
    before = st["state"].float() if "state" in st else x.new_zeros(c["B"], c["W"] - 1, c["C"])
    return torch.cat([before, x], 1)


def _conv_pre(st, rows):
    T = rows.shape[1] - st["w"].shape[1] + 1
    return st["b"] + sum(st["w"][:, j] * rows[:, j:j + T] for j in range(st["w"].shape[1]))


def _conv_live(st, y):
    if st["lens"] is None:
        return y
    live = torch.arange(y.shape[1], device=y.device)[None] < st["lens"][:, None]
    return torch.where(live[..., None], y, torch.zeros((), device=y.device))


def plain_conv_step(st):
    pool, slots, x = st["pool"], st["slots"].long(), st["x"]
    used = slots >= 0
    rows = torch.cat([pool[slots.clamp(min=0)], x[:, None]], 1)
    y = _silu(_conv_pre(st, rows.float()))[:, 0]
    y = torch.where(used[:, None], y, torch.zeros((), device=y.device))
    pool.index_copy_(0, slots[used], rows[used][:, 1:])
    return {"y": y.to(x.dtype), "pool": pool}


def plain_conv_prefill(st):
    c, rows = st["case"], _conv_rows(st)
    y = _conv_live(st, _silu(_conv_pre(st, rows)))
    n = torch.full((c["B"],), c["T"], device=rows.device) if st["lens"] is None else st["lens"]
    at = n.long()[:, None] + torch.arange(c["W"] - 1, device=rows.device)
    end = rows.gather(1, at[..., None].expand(-1, -1, c["C"]))
    return {"y": y.to(st["x"].dtype), "state": end.to(st["x"].dtype)}


def plain_conv_train(st):
    rows = _conv_rows(st)
    T, W = st["x"].shape[1], st["w"].shape[1]
    pre = _conv_pre(st, rows)
    y = _conv_live(st, _silu(pre))
    d = _conv_live(st, st["grad_y"].float() * _silu_slope(pre))
    dx = torch.zeros_like(rows)
    for j in range(W):
        dx[:, j:j + T] += st["w"][:, j] * d
    dw = torch.stack([(d * rows[:, j:j + T]).sum((0, 1)) for j in range(W)], 1)
    dt = st["x"].dtype
    return {"y": y.to(dt), "dx": _conv_live(st, dx[:, W - 1:]).to(dt), "dw": dw, "db": d.sum((0, 1))}


def _ln(st):
    x = st["x"].float()
    x = x - x.mean(-1, keepdim=True)
    rstd = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    return x * rstd, rstd


def plain_ln(st):
    hat, rstd = _ln(st)
    dt = DTYPES[st["case"]["dtype"]]
    out = {"y": (hat * st["w"] + st["b"]).to(dt)}
    if st["case"]["kind"] == "ln_train":
        dy = st["grad_y"].float()
        g = dy * st["w"]
        dx = rstd * (g - g.mean(-1, keepdim=True) - hat * (g * hat).mean(-1, keepdim=True))
        out |= {"dx": dx.to(st["x"].dtype), "dw": (dy * hat).sum(0), "db": dy.sum(0)}
    return out


# --------------------------------------------------------------------------
# the library's calls
# --------------------------------------------------------------------------

def _scan_args(st):
    return (st["u"], st["delta"], st["A"], st["Bm"], st["Cm"])


def _scan_kw(st):
    return dict(D=st["D"], z=st["z"], delta_bias=st["delta_bias"], softplus=True)


def _bytes(n, like):
    return torch.empty(n, dtype=torch.uint8, device=like.device)


def _new(t, dtype=None):
    return torch.empty(t.shape, dtype=dtype or t.dtype, device=t.device)


def own_scan_step(st, snn):
    y = _new(st["u"])
    snn.snn_selective_scan_step(*_scan_args(st), st["pool"], y, slots=st["slots"], **_scan_kw(st))
    return {"y": y, "pool": st["pool"]}


def own_scan_prefill(st, snn):
    c, y, end = st["case"], _new(st["u"]), _new(st["state"])
    shape = [c[x] for x in ("B", "T", "D", "N", "G")]
    ws = _bytes(snn.snn_selective_scan_workspace_bytes(*shape), y)
    snn.snn_selective_scan_fwd(*_scan_args(st), y, ws, seq_lens=st["lens"], state_in=st["state"],
                               state_out=end, **_scan_kw(st))
    return {"y": y, "state": end}


def own_scan_train(st, snn):
    c, y = st["case"], _new(st["u"])
    shape = [c[x] for x in ("B", "T", "D", "N", "G")]
    ws = _bytes(snn.snn_selective_scan_workspace_bytes(*shape, backward=True), y)
    ckpt = torch.empty(snn.snn_selective_scan_ckpt_elems(*shape), dtype=torch.float32,
                       device=y.device)
    snn.snn_selective_scan_fwd(*_scan_args(st), y, ws, seq_lens=st["lens"], ckpt=ckpt,
                               **_scan_kw(st))
    out = {"y": y, "du": _new(st["u"]), "ddelta": _new(st["delta"]), "dA": _new(st["A"]),
           "dB": _new(st["Bm"]), "dC": _new(st["Cm"]), "dD": _new(st["D"]),
           "ddelta_bias": _new(st["delta_bias"])}
    if st["z"] is not None:
        out["dz"] = _new(st["u"])
    snn.snn_selective_scan_bwd(*_scan_args(st), st["grad_y"], ckpt, out["du"], out["ddelta"],
                               out["dA"], out["dB"], out["dC"], ws, seq_lens=st["lens"],
                               grad_D=out["dD"], grad_z=out.get("dz"),
                               grad_delta_bias=out["ddelta_bias"], **_scan_kw(st))
    return out


def own_conv_step(st, snn):
    y = _new(st["x"])
    snn.snn_causal_conv_step(st["x"], st["w"], st["b"], st["pool"], y, act="silu",
                             slots=st["slots"])
    return {"y": y, "pool": st["pool"]}


def own_conv_prefill(st, snn):
    y, end = _new(st["x"]), _new(st["state"])
    snn.snn_causal_conv_fwd(st["x"], st["w"], st["b"], y, act="silu", seq_lens=st["lens"],
                            state_in=st["state"], state_out=end)
    return {"y": y, "state": end}


def own_conv_train(st, snn):
    x, y = st["x"], _new(st["x"])
    snn.snn_causal_conv_fwd(x, st["w"], st["b"], y, act="silu", seq_lens=st["lens"])
    out = {"y": y, "dx": _new(x), "dw": _new(st["w"]), "db": _new(st["b"])}
    ws = _bytes(snn.snn_causal_conv_workspace_bytes(*x.shape, st["w"].shape[1]), x)
    snn.snn_causal_conv_bwd(x, st["w"], st["b"], st["grad_y"], out["dx"], out["dw"], out["db"], ws,
                            act="silu", seq_lens=st["lens"])
    return out


def own_ln(st, snn):
    x = st["x"]
    y = _new(x, DTYPES[st["case"]["dtype"]])
    if st["case"]["kind"] == "ln_fwd":
        snn.snn_layer_norm_fwd(x, st["w"], st["b"], y, eps=EPS)
        return {"y": y}
    stats = torch.empty(2, len(x), dtype=torch.float32, device=x.device)
    snn.snn_layer_norm_fwd(x, st["w"], st["b"], y, stats=stats, eps=EPS)
    out = {"y": y, "dx": _new(x), "dw": _new(st["w"]), "db": _new(st["b"])}
    ws = _bytes(snn.snn_layer_norm_workspace_bytes(*x.shape), x)
    snn.snn_layer_norm_bwd(x, st["w"], stats, st["grad_y"], out["dx"], out["dw"], out["db"], ws)
    return out


PLAIN = {"scan_step": plain_scan_step, "scan_prefill": plain_scan_prefill,
         "scan_train": plain_scan_train, "conv_step": plain_conv_step,
         "conv_prefill": plain_conv_prefill, "conv_train": plain_conv_train, "ln_fwd": plain_ln,
         "ln_train": plain_ln}
OWN = {"scan_step": own_scan_step, "scan_prefill": own_scan_prefill, "scan_train": own_scan_train,
       "conv_step": own_conv_step, "conv_prefill": own_conv_prefill, "conv_train": own_conv_train,
       "ln_fwd": own_ln, "ln_train": own_ln}


def run(state):
    kind = state["case"]["kind"]
    if own:
        from paper_2211_10725_gb300 import snn
        return OWN[kind](state, snn)
    return PLAIN[kind](state)


# --------------------------------------------------------------------------
# the definitions in 64 bits, the scan token by token
# --------------------------------------------------------------------------

def _exact_scan(case, st):
    B, D, N, G = (case[x] for x in ("B", "D", "N", "G"))
    step = case["kind"] == "scan_step"
    f = lambda x: st[x].double()[:, None] if step else st[x].double()  # noqa: E731
    raw, u, Bm, Cm = f("delta") + st["delta_bias"].double(), f("u"), f("Bm"), f("Cm")
    T = u.shape[1]
    s = torch.logaddexp(raw, torch.zeros_like(raw))
    slots = st["slots"].tolist() if step else None
    lens = [int(p >= 0) for p in slots] if step else _lens(case) if case["ragged"] else [T] * B
    live = torch.tensor([[t < n for n in lens] for t in range(T)], device=u.device).view(T, B, 1, 1)
    if step:
        h = st["pool"].double()[[max(p, 0) for p in slots]].clone()
    else:
        h = st["state"].double().clone() if "state" in st else u.new_zeros(B, D, N)
    A, skip = st["A"].double(), st["D"].double()
    group = torch.arange(D, device=u.device) // (D // G)
    train = case["kind"] == "scan_train"
    y, before = torch.zeros_like(u), u.new_zeros(T, B, D, N) if train else None
    for t in range(T):
        if train:
            before[t] = h
        nxt = torch.exp(s[:, t, :, None] * A) * h + (s[:, t] * u[:, t])[..., None] * Bm[:, t, group]
        h = torch.where(live[t], nxt, h)
        y[:, t] = torch.einsum("bdn,bdn->bd", h, Cm[:, t, group])
    y = y + skip * u
    at = live[..., 0].transpose(0, 1)
    z = f("z") if st["z"] is not None else None
    gate = 1.0 if z is None else z / (1.0 + torch.exp(-z))
    out = {"y": torch.where(at, y * gate, 0.0)}
    if step:
        out["y"], out["pool"] = out["y"][:, 0], st["pool"].double().clone()
        for b, p in enumerate(slots):
            if p >= 0:
                out["pool"][p] = h[b]
        return out
    if not train:
        return out | {"state": h}
    do = st["grad_y"].double()
    if z is not None:
        sig = 1.0 / (1.0 + torch.exp(-z))
        out["dz"] = torch.where(at, do * y * (sig + z * sig * (1.0 - sig)), 0.0)
    dy = torch.where(at, do * gate, 0.0)
    du, ds = dy * skip, torch.zeros_like(u)
    dB, dC, dA = torch.zeros_like(Bm), torch.zeros_like(Cm), torch.zeros_like(A)
    g = torch.zeros_like(h)
    for t in reversed(range(T)):
        a = torch.exp(s[:, t, :, None] * A)
        bt, ct, ut, st_ = Bm[:, t, group], Cm[:, t, group], u[:, t], s[:, t]
        now = a * before[t] + (st_ * ut)[..., None] * bt
        gt = g + dy[:, t, :, None] * ct
        dec = gt * a * before[t]
        sums = lambda x: x.view(B, G, D // G, N).sum(2)  # noqa: E731
        dC[:, t] = torch.where(live[t], sums(dy[:, t, :, None] * now), 0.0)
        dB[:, t] = torch.where(live[t], sums(gt * (st_ * ut)[..., None]), 0.0)
        w = (gt * bt).sum(-1)
        du[:, t] += torch.where(live[t][..., 0], st_ * w, 0.0)
        ds[:, t] = torch.where(live[t][..., 0], ut * w + (dec * A).sum(-1), 0.0)
        dA += torch.where(live[t], dec * st_[..., None], 0.0).sum(0)
        g = torch.where(live[t], a * gt, g)
    ds = ds / (1.0 + torch.exp(-raw))
    return out | {"du": du, "ddelta": ds, "dA": dA, "dB": dB, "dC": dC, "ddelta_bias": ds.sum((0, 1)),
                  "dD": (dy * u).sum((0, 1))}


def _exact_conv(case, st):
    B, C, W = case["B"], case["C"], case["W"]
    step = case["kind"] == "conv_step"
    x = st["x"].double()[:, None] if step else st["x"].double()
    T = x.shape[1]
    slots = st["slots"].tolist() if step else None
    lens = [int(p >= 0) for p in slots] if step else _lens(case) if case["ragged"] else [T] * B
    if step:
        before = st["pool"].double()[[max(p, 0) for p in slots]]
    else:
        before = st["state"].double() if "state" in st else x.new_zeros(B, W - 1, C)
    w, bias = st["w"].double(), st["b"].double()
    out = {k: [] for k in ("y", "state", "dx")}
    dw, db = torch.zeros_like(w), torch.zeros_like(bias)
    for b in range(B):
        n = lens[b]
        rows = torch.cat([before[b], x[b, :n]])
        end = rows[n:]
        windows = torch.stack([rows[j:j + n] for j in range(W)], -1)      # [n, C, W]
        pre = torch.einsum("tcw,cw->tc", windows, w) + bias
        sig = 1.0 / (1.0 + torch.exp(-pre))
        rest = x.new_zeros(T - n, C)
        out["y"].append(torch.cat([pre * sig, rest]))
        out["state"].append(end)
        if case["kind"] == "conv_train":
            d = st["grad_y"][b, :n].double() * (sig + pre * sig * (1.0 - sig))
            late = torch.cat([d, x.new_zeros(W - 1, C)])
            out["dx"].append(torch.cat([sum(w[:, W - 1 - j] * late[j:j + n] for j in range(W)), rest]))
            dw += torch.einsum("tc,tcw->cw", d, windows)
            db += d.sum(0)
    y = torch.stack(out["y"])
    if step:
        pool = st["pool"].double().clone()
        for b, p in enumerate(slots):
            if p >= 0:
                pool[p] = out["state"][b]
        return {"y": y[:, 0], "pool": pool}
    if case["kind"] == "conv_prefill":
        return {"y": y, "state": torch.stack(out["state"])}
    return {"y": y, "dx": torch.stack(out["dx"]), "dw": dw, "db": db}


def _exact_ln(case, st):
    train = case["kind"] == "ln_train"
    p = {k: st[k].double().requires_grad_(train) for k in ("x", "w", "b")}
    with torch.enable_grad():
        var, mean = torch.var_mean(p["x"], dim=-1, keepdim=True, unbiased=False)
        y = (p["x"] - mean) / (var + EPS).sqrt() * p["w"] + p["b"]
        if not train:
            return {"y": y}
        y.backward(st["grad_y"].double())
    return {"y": y.detach(), "dx": p["x"].grad, "dw": p["w"].grad, "db": p["b"].grad}


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"].split("_")[0]
    return {"scan": _exact_scan, "conv": _exact_conv, "ln": _exact_ln}[kind](case, st)
