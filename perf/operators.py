"""Cases of the leaky-state attention (linear attention with a decay for each
head) and of the block norms (the norm after a block, its gate and residual
scale, and the norm before the next block), in plain torch and through the
library.

Attention.  Each head h keeps a matrix state that leaks like a membrane,
    S_t = beta_h S_{t-1} + k_t v_t^T,      o_t = scale * S_t^T q_t,
over q [B, T, H, Dk], k [B, T, Hk, Dk], v [B, T, Hk, Dv] (query head h reads
key/value head h // (H / Hk)).  Tokens at t >= seq_lens[b] do not exist: their
outputs and gradients are zero and the state passes over them.

Block norm, per row of N channels:
    n  = a * rsqrt(mean(a^2 over each group) + eps) * w_post
    r' = r + res_scale * n * silu(z)
    y  = r' * rsqrt(mean(r'^2) + eps) * w_pre
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
CHUNK = 64
EPS = 1e-6


# --------------------------------------------------------------------------
# cases
# --------------------------------------------------------------------------

def attn(name, kind, B, T, H, Hk, Dk, Dv, dtype, ragged=False):
    return {"name": name, "kind": kind, "B": B, "T": T, "H": H, "Hk": Hk, "Dk": Dk, "Dv": Dv,
            "dtype": dtype, "ragged": ragged}


def norm(name, kind, M, N, dtype, res, group=0, gate=True):
    return {"name": name, "kind": kind, "M": M, "N": N, "dtype": dtype, "res": res,
            "group": group, "gate": gate}


def listed():
    return [
        # one user's next token, a small model's layer: latency
        attn("step_one", "step", 1, 1, 8, 8, 64, 64, "bf16"),
        # a batch of requests in a pool of states, some places of the batch empty
        attn("step_pool", "step", 24, 1, 12, 4, 96, 128, "f16", ragged=True),
        # a full serving batch: the states' bandwidth
        attn("step_full", "step", 128, 1, 16, 16, 128, 128, "bf16"),
        # a short prompt for one user
        attn("prefill_short", "prefill", 1, 100, 8, 8, 64, 64, "bf16"),
        # prompts of several users, padded to the longest; shared key/value heads
        attn("prefill_ragged", "prefill", 6, 1500, 16, 4, 64, 128, "f16", ragged=True),
        # one long document: few heads, a long axis
        attn("prefill_long", "prefill", 1, 16384, 16, 16, 128, 128, "bf16"),
        # a training step on padded samples with shared key/value heads, an odd width
        attn("train_ragged", "train", 3, 777, 12, 4, 72, 72, "f16", ragged=True),
        # a training step of ordinary size, forward and backward
        attn("train_full", "train", 2, 4096, 32, 32, 128, 128, "bf16"),
        # the norms around one token's block
        norm("norm_one", "norm", 1, 1000, "bf16", "bf16"),
        # the norms of a long prompt, 16-bit activations on a 32-bit residual stream
        norm("norm_prompt", "norm", 16384, 4096, "bf16", "f32"),
        # a training step's way back with an odd width, in 32 bits
        norm("norm_bwd_odd", "norm_bwd", 3001, 1001, "f32", "f32"),
        # a training step's way back, the norm after the block taken per head
        norm("norm_bwd_heads", "norm_bwd", 16384, 2048, "bf16", "bf16", group=128),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["step", "prefill", "train", "norm", "norm_bwd"])
    if kind in ("norm", "norm_bwd"):
        group = rng.choice([0, 0, 64, 128])
        N = _log(rng, 64, 8192)
        if group:
            N = max(1, N // group) * group
        most = (16384 * 2048) if kind == "norm_bwd" else (16384 * 4096)
        M = _log(rng, 1, max(1, min(32768, most // N)))
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        res = rng.choice([dtype, "f32"])
        if kind == "norm_bwd" and res == "f32":
            M = max(1, M // 2)
        return {"kind": kind, "M": M, "N": N, "dtype": dtype, "res": res, "group": group,
                "gate": rng.random() < 0.75}
    Hk = rng.choice([1, 2, 4, 8, 16])
    H = Hk * rng.choice([1, 1, 2, 3])
    Dk = 8 * rng.randint(4, 16)
    Dv = rng.choice([Dk, 8 * rng.randint(4, 16)])
    if kind == "step":
        T, B = 1, _log(rng, 1, max(1, 128 * 16 // H))
    else:
        tokens = (2 * 4096 * 32 if kind == "train" else 16384 * 16) // (2 * H)
        B = rng.randint(1, min(8, max(1, tokens // 256)))
        T = _log(rng, 1, max(1, min(16384, tokens // B)))
    return {"kind": kind, "B": B, "T": T, "H": H, "Hk": Hk, "Dk": Dk, "Dv": Dv,
            "dtype": rng.choice(["bf16", "f16"]), "ragged": B > 1 and rng.random() < 0.5}


def work(case):
    size = lambda d: 4 if d == "f32" else 2  # noqa: E731
    if case["kind"] in ("norm", "norm_bwd"):
        M, N, e, r = case["M"], case["N"], size(case["dtype"]), size(case["res"])
        # r, a, z in; r', y out
        b = M * N * (2 * r + e * (3 if case["gate"] else 2)) + 12 * N
        f = 12 * M * N
        if case["kind"] == "norm_bwd":
            # r', a, z, dr', dy in; dr, da, dz and the three parameters' gradients out
            b = M * N * (3 * r + e * (5 if case["gate"] else 3)) + 24 * N
            f = 30 * M * N
        return {"bytes": b, "flops": f}
    B, T, H, Hk, Dk, Dv = (case[x] for x in ("B", "T", "H", "Hk", "Dk", "Dv"))
    if case["ragged"]:
        lens = _lens(case)
        n = B if case["kind"] == "step" else sum(lens)
        if case["kind"] == "step":
            n = sum(1 for s in _slots(case) if s >= 0)
    else:
        n = B * T
    io = 2 * (H * Dk + Hk * Dk + Hk * Dv)
    states = 4 * H * Dk * Dv
    if case["kind"] == "step":
        return {"bytes": n * (io + 2 * states) + 2 * B * H * Dv, "flops": 4 * n * H * Dk * Dv}
    out = 2 * B * T * H * Dv  # padded places are written too (zeros)
    if case["kind"] == "prefill":
        return {"bytes": n * io + out + 2 * B * states, "flops": 4 * n * H * Dk * Dv}
    grads = 2 * B * T * (H * Dk + Hk * Dk + Hk * Dv)
    return {"bytes": n * io + out + 2 * n * H * Dv + grads, "flops": 14 * n * H * Dk * Dv}


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


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g, device=dev)  # noqa: E731
    dt = DTYPES[case["dtype"]]
    if case["kind"] in ("norm", "norm_bwd"):
        M, N = case["M"], case["N"]
        st = {"case": case, "r": (2.0 * rand(M, N)).to(DTYPES[case["res"]]),
              "a": (0.7 * rand(M, N)).to(dt), "z": rand(M, N).to(dt) if case["gate"] else None,
              "w_post": 1.0 + 0.1 * rand(N), "res_scale": 0.3 + 0.1 * rand(N),
              "w_pre": 1.0 + 0.1 * rand(N)}
        if case["kind"] == "norm_bwd":
            # here r is the stream after the block, as the forward stored it
            st["grad_r"] = (0.05 * rand(M, N)).to(DTYPES[case["res"]])
            st["grad_y"] = (0.05 * rand(M, N)).to(dt)
        return st
    B, T, H, Hk, Dk, Dv = (case[x] for x in ("B", "T", "H", "Hk", "Dk", "Dv"))
    # q, k and v are parts of one projection's rows
    rows = rand(B, T, H * Dk + Hk * Dk + Hk * Dv)
    rows[..., H * Dk:H * Dk + Hk * Dk] *= Dk ** -0.5
    rows = rows.to(dt)
    q, k, v = rows.split([H * Dk, Hk * Dk, Hk * Dv], dim=-1)
    # memories from tens to thousands of tokens over the heads
    beta = 1.0 - torch.exp2(-torch.linspace(4.0, 11.0, H, device=dev))
    st = {"case": case, "q": q.unflatten(-1, (H, Dk)), "k": k.unflatten(-1, (Hk, Dk)),
          "v": v.unflatten(-1, (Hk, Dv)), "beta": beta, "scale": 1.0, "lens": None, "slots": None}
    if case["kind"] == "step":
        for x in ("q", "k", "v"):
            st[x] = st[x][:, 0]
        st["pool"] = rand(B + 3, H, Dk, Dv)
        st["slots"] = torch.tensor(_slots(case), dtype=torch.int32, device=dev)
        return st
    if case["ragged"]:
        st["lens"] = torch.tensor(_lens(case), dtype=torch.int32, device=dev)
    if case["kind"] == "prefill":
        st["state"] = rand(B, H, Dk, Dv)
    else:
        st["grad_o"] = (0.1 * rand(B, T, H, Dv)).to(dt)
    return st


# --------------------------------------------------------------------------
# plain forms
# --------------------------------------------------------------------------

def _powers(beta, n):
    """beta^n in 32 bits for a tensor n of exponents, [H, *n.shape]; 0 where n < 0."""
    b = beta.float().view(-1, *([1] * n.dim()))
    return torch.where(n >= 0, b ** n.clamp(min=0).float(), torch.zeros((), device=n.device))


class _Chunks:
    """A batch of sequences cut into chunks, in 32 bits, [B, H, chunks, CHUNK, D]."""

    def __init__(self, st):
        q, k = st["q"], st["k"]
        self.B, self.T, self.H, self.Hk = q.shape[0], q.shape[1], q.shape[2], k.shape[2]
        self.nc = -(-self.T // CHUNK)
        t = torch.arange(self.T, device=q.device)
        lens = st["lens"]
        self.lens = (torch.full((self.B,), self.T, device=q.device) if lens is None else lens).long()
        self.valid = t[None] < self.lens[:, None]                       # [B, T]
        i = torch.arange(CHUNK, device=q.device)
        n = torch.arange(self.nc, device=q.device)
        self.within = _powers(st["beta"], i[:, None] - i[None])         # [H, i, j]
        self.first = _powers(st["beta"], i + 1)                         # to token i from before it
        self.last = _powers(st["beta"], CHUNK - 1 - i)                  # from token j to the end
        self.across = _powers(st["beta"], (n[:, None] - 1 - n[None]) * CHUNK)  # [H, n, m < n]
        self.start = _powers(st["beta"], n * CHUNK)
        # [B, H, T]: from token t to the sequence's last one
        self.to_end = _powers(st["beta"], self.lens[:, None] - 1 - t[None]).transpose(0, 1)

    def heads(self, x):
        """[B, T, heads, D] -> [B, H, T, D], padded places zero, shared heads repeated."""
        x = torch.where(self.valid[..., None, None], x.float(), torch.zeros((), device=x.device))
        x = x.transpose(1, 2)
        return x.repeat_interleave(self.H // x.shape[1], dim=1)

    def cut(self, x):
        x = torch.nn.functional.pad(x, (0, 0, 0, self.nc * CHUNK - self.T))
        return x.unflatten(2, (self.nc, CHUNK))

    def join(self, x):
        """[B, H, chunks, CHUNK, D] -> [B, T, H, D], padded places zero."""
        x = x.flatten(2, 3)[:, :, :self.T].transpose(1, 2)
        return torch.where(self.valid[..., None, None], x, torch.zeros((), device=x.device))

    def shared(self, x):
        """[B, T, H, D] -> [B, T, Hk, D]: the sum over each group of query heads."""
        return x.unflatten(2, (self.Hk, self.H // self.Hk)).sum(3)

    def before(self, k, v, state):
        """States before each chunk, [B, H, chunks, Dk, Dv]."""
        parts = (k * self.last[:, None, :, None]).transpose(-1, -2) @ v
        s = (self.across @ parts.flatten(3)).unflatten(3, parts.shape[3:])
        return s if state is None else s + self.start[..., None, None] * state.float()[:, :, None]

    def after(self, q, do):
        """Gradients of the states after each chunk, [B, H, chunks, Dk, Dv]."""
        parts = (q * self.first[:, None, :, None]).transpose(-1, -2) @ do
        back = self.across.transpose(-1, -2)
        return (back @ parts.flatten(3)).unflatten(3, parts.shape[3:])


def plain_forward(st, c, state=None):
    q, k, v = (c.cut(c.heads(st[x])) for x in ("q", "k", "v"))
    o = ((q @ k.transpose(-1, -2)) * c.within[:, None]) @ v
    o = o + (q * c.first[:, None, :, None]) @ c.before(k, v, state)
    return c.join(st["scale"] * o)


def plain_step(st):
    beta, pool, slots = st["beta"], st["pool"], st["slots"].long()
    q, k, v = st["q"].float(), st["k"].float(), st["v"].float()
    G = q.shape[1] // k.shape[1]
    k, v = k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)
    used = slots >= 0
    old = pool[slots.clamp(min=0)]
    new = beta[:, None, None] * old + k[..., :, None] * v[..., None, :]
    o = st["scale"] * (q[..., None, :] @ new).squeeze(-2)
    o = torch.where(used[:, None, None], o, torch.zeros((), device=o.device))
    pool.index_copy_(0, slots[used], new[used])
    return {"o": o.to(st["q"].dtype), "pool": pool}


def plain_prefill(st):
    c = _Chunks(st)
    o = plain_forward(st, c, st["state"])
    k, v = c.heads(st["k"]), c.heads(st["v"])
    end = (k * c.to_end[..., None]).transpose(-1, -2) @ v
    end = end + _powers(st["beta"], c.lens).transpose(0, 1)[..., None, None] * st["state"].float()
    return {"o": o.to(st["q"].dtype), "state": end}


def plain_train(st):
    c = _Chunks(st)
    dt = st["q"].dtype
    o = plain_forward(st, c)
    q, k, v, do = (c.cut(c.heads(st[x])) for x in ("q", "k", "v", "grad_o"))
    s, r = c.before(k, v, None), c.after(q, do)
    w = c.within[:, None]
    scores = (q @ k.transpose(-1, -2)) * w
    grads = (do @ v.transpose(-1, -2)) * w
    first, last = c.first[:, None, :, None], c.last[:, None, :, None]
    dq = grads @ k + (do * first) @ s.transpose(-1, -2)
    dk = grads.transpose(-1, -2) @ q + (v * last) @ r.transpose(-1, -2)
    dv = scores.transpose(-1, -2) @ do + (k * last) @ r
    dq, dk, dv = (st["scale"] * c.join(x) for x in (dq, dk, dv))
    return {"o": o.to(dt), "dq": dq.to(dt), "dk": c.shared(dk).to(dt), "dv": c.shared(dv).to(dt)}


def _normed(x, group):
    """x over the root of its mean square in each group, and that factor."""
    g = x.unflatten(-1, (-1, group))
    rstd = torch.rsqrt(g.square().mean(-1, keepdim=True) + EPS)
    return (g * rstd).flatten(-2), rstd.expand_as(g).flatten(-2)


def _norm_back(d, hat, rstd, group):
    """Gradient of x given that of x * rstd."""
    m = (d * hat).unflatten(-1, (-1, group)).mean(-1, keepdim=True)
    return rstd * (d - hat * m.expand(*m.shape[:-1], group).flatten(-2))


def plain_norm(st):
    N = st["a"].shape[-1]
    hat = _normed(st["a"].float(), st["case"]["group"] or N)[0]
    gate = 1.0 if st["z"] is None else st["z"].float() * torch.sigmoid(st["z"].float())
    r2 = st["r"].float() + st["res_scale"] * (hat * st["w_post"]) * gate
    y = _normed(r2, N)[0] * st["w_pre"]
    return {"r": r2.to(st["r"].dtype), "y": y.to(st["a"].dtype)}


def plain_norm_bwd(st):
    N, dt = st["a"].shape[-1], st["a"].dtype
    group = st["case"]["group"] or N
    hat, rstd = _normed(st["a"].float(), group)
    hat2, rstd2 = _normed(st["r"].float(), N)
    dy = st["grad_y"].float()
    d = st["grad_r"].float() + _norm_back(dy * st["w_pre"], hat2, rstd2, N)
    z = None if st["z"] is None else st["z"].float()
    sg = 1.0 if z is None else torch.sigmoid(z)
    gate = 1.0 if z is None else z * sg
    n = hat * st["w_post"]
    dn = d * st["res_scale"] * gate
    out = {"grad_r": d.to(st["r"].dtype), "grad_a": _norm_back(dn * st["w_post"], hat, rstd, group).to(dt),
           "grad_w_post": (dn * hat).sum(0), "grad_scale": (d * n * gate).sum(0),
           "grad_w_pre": (dy * hat2).sum(0)}
    if z is not None:
        out["grad_z"] = (d * st["res_scale"] * n * sg * (1.0 + z * (1.0 - sg))).to(dt)
    return out


# --------------------------------------------------------------------------
# the library's calls
# --------------------------------------------------------------------------

def own_step(st, snn):
    q, v = st["q"], st["v"]
    o = torch.empty((*q.shape[:2], v.shape[-1]), dtype=q.dtype, device=q.device)
    snn.snn_leaky_attn_step(q, st["k"], v, st["beta"], st["pool"], o, scale=st["scale"],
                            slots=st["slots"])
    return {"o": o, "pool": st["pool"]}


def _workspace(st, snn, backward):
    q, k, v = st["q"], st["k"], st["v"]
    n = snn.snn_leaky_attn_workspace_bytes(*q.shape[:3], k.shape[2], q.shape[3], v.shape[3],
                                           backward=backward)
    return torch.empty(n, dtype=torch.uint8, device=q.device)


def own_prefill(st, snn):
    q, v = st["q"], st["v"]
    o = torch.empty((*q.shape[:3], v.shape[-1]), dtype=q.dtype, device=q.device)
    end = torch.empty_like(st["state"])
    snn.snn_leaky_attn_fwd(q, st["k"], v, st["beta"], o, _workspace(st, snn, False),
                           scale=st["scale"], state_in=st["state"], state_out=end,
                           seq_lens=st["lens"])
    return {"o": o, "state": end}


def own_train(st, snn):
    q, k, v = st["q"], st["k"], st["v"]
    new = lambda x, d: torch.empty((*x.shape[:3], d), dtype=q.dtype, device=q.device)  # noqa: E731
    o, dq = new(q, v.shape[-1]), new(q, q.shape[-1])
    dk, dv = new(k, q.shape[-1]), new(k, v.shape[-1])
    ws = _workspace(st, snn, True)
    snn.snn_leaky_attn_fwd(q, k, v, st["beta"], o, ws, scale=st["scale"], seq_lens=st["lens"])
    snn.snn_leaky_attn_bwd(q, k, v, st["beta"], st["grad_o"], dq, dk, dv, ws, scale=st["scale"],
                           seq_lens=st["lens"])
    return {"o": o, "dq": dq, "dk": dk, "dv": dv}


def own_norm(st, snn):
    r, y = torch.empty_like(st["r"]), torch.empty_like(st["a"])
    snn.snn_block_norm_fwd(st["r"], st["a"], st["z"], st["w_post"], st["res_scale"], st["w_pre"],
                           r, y, eps=EPS, group=st["case"]["group"], gate=_gate(st))
    return {"r": r, "y": y}


def _gate(st):
    return "none" if st["z"] is None else "silu"


def own_norm_bwd(st, snn):
    like = torch.empty_like
    a, z = st["a"], st["z"]
    out = {"grad_r": like(st["r"]), "grad_a": like(a), "grad_w_post": like(st["w_post"]),
           "grad_scale": like(st["w_post"]), "grad_w_pre": like(st["w_post"])}
    if z is not None:
        out["grad_z"] = like(z)
    ws = torch.empty(snn.snn_block_norm_workspace_bytes(*a.shape), dtype=torch.uint8,
                     device=a.device)
    snn.snn_block_norm_bwd(st["r"], a, z, st["w_post"], st["res_scale"], st["w_pre"],
                           st["grad_r"], st["grad_y"], out["grad_r"], out["grad_a"],
                           out.get("grad_z"), out["grad_w_post"], out["grad_scale"],
                           out["grad_w_pre"], ws, eps=EPS, group=st["case"]["group"],
                           gate=_gate(st))
    return out


PLAIN = {"step": plain_step, "prefill": plain_prefill, "train": plain_train, "norm": plain_norm,
         "norm_bwd": plain_norm_bwd}
OWN = {"step": own_step, "prefill": own_prefill, "train": own_train, "norm": own_norm,
       "norm_bwd": own_norm_bwd}


def run(state):
    kind = state["case"]["kind"]
    if own:
        from paper_2211_10725_gb300 import snn
        return OWN[kind](state, snn)
    return PLAIN[kind](state)


# --------------------------------------------------------------------------
# the definition, token by token in 64 bits
# --------------------------------------------------------------------------

def _exact_attn(case, st):
    B, T, H, Hk, Dk, Dv = (case[x] for x in ("B", "T", "H", "Hk", "Dk", "Dv"))
    G = H // Hk
    if case["kind"] == "step":
        T = 1
        q, k, v = (st[x].double()[:, None] for x in ("q", "k", "v"))
        slots = st["slots"].tolist()
        lens = [1 if s >= 0 else 0 for s in slots]
        S = st["pool"].double()[[max(s, 0) for s in slots]].clone()
    else:
        q, k, v = (st[x].double() for x in ("q", "k", "v"))
        lens = _lens(case) if case["ragged"] else [T] * B
        S = st["state"].double().clone() if "state" in st else q.new_zeros(B, H, Dk, Dv)
    live = torch.tensor([[t < n for n in lens] for t in range(T)], device=q.device)
    beta = st["beta"].double()[:, None, None]
    group = [h // G for h in range(H)]
    o, dq = q.new_zeros(B, T, H, Dv), q.new_zeros(B, T, H, Dk)
    do = st["grad_o"].double() if "grad_o" in st else None
    for t in range(T):
        on = live[t][:, None, None, None]
        kt, vt = k[:, t, group], v[:, t, group]
        S = torch.where(on, beta * S + kt[..., :, None] * vt[..., None, :], S)
        o[:, t] = torch.where(on[..., 0], (q[:, t][..., None, :] @ S)[..., 0, :], 0.0)
        if do is not None:
            dq[:, t] = torch.where(on[..., 0], (S @ do[:, t][..., :, None])[..., 0], 0.0)
    sc = st["scale"]
    if case["kind"] == "step":
        pool = st["pool"].double().clone()
        for b, s in enumerate(slots):
            if s >= 0:
                pool[s] = S[b]
        return {"o": sc * o[:, 0], "pool": pool}
    if do is None:
        return {"o": sc * o, "state": S}
    dk, dv = torch.zeros_like(k), torch.zeros_like(v)
    R = torch.zeros_like(S)
    for t in reversed(range(T)):
        on = live[t][:, None, None, None]
        kt, vt = k[:, t, group], v[:, t, group]
        R = torch.where(on, beta * R + q[:, t][..., :, None] * do[:, t][..., None, :], R)
        gk = torch.where(on[..., 0], (R @ vt[..., :, None])[..., 0], 0.0)
        gv = torch.where(on[..., 0], (kt[..., None, :] @ R)[..., 0, :], 0.0)
        dk[:, t] = gk.view(B, Hk, G, Dk).sum(2)
        dv[:, t] = gv.view(B, Hk, G, Dv).sum(2)
    return {"o": sc * o, "dq": sc * dq, "dk": sc * dk, "dv": sc * dv}


def _exact_norm(case, st):
    f = {x: (None if t is None else t.double()) for x, t in st.items() if x != "case"}
    leaves = ("r", "a", "z", "w_post", "res_scale", "w_pre")
    with torch.enable_grad():
        p = {x: None if f[x] is None else f[x].clone().requires_grad_() for x in leaves}
        M, N = p["a"].shape
        g = case["group"] or N
        blocks = p["a"].reshape(M, N // g, g)
        n = (blocks / (blocks.pow(2).sum(-1, keepdim=True) / g + EPS).sqrt()).reshape(M, N)
        u = p["res_scale"] * p["w_post"] * n
        if p["z"] is not None:
            u = u * p["z"] / (1 + torch.exp(-p["z"]))
        r2 = p["r"] if case["kind"] == "norm_bwd" else p["r"] + u
        y = p["w_pre"] * r2 / (r2.pow(2).sum(-1, keepdim=True) / N + EPS).sqrt()
        if case["kind"] == "norm":
            return {"r": r2, "y": y}
        torch.autograd.backward([r2, y], [f["grad_r"], f["grad_y"]])
        u.backward(p["r"].grad)
    out = {"grad_r": p["r"].grad, "grad_a": p["a"].grad, "grad_w_post": p["w_post"].grad,
           "grad_scale": p["res_scale"].grad, "grad_w_pre": p["w_pre"].grad}
    if p["z"] is not None:
        out["grad_z"] = p["z"].grad
    return out


def exact(case, seed):
    st = prepare(case, seed)
    out = (_exact_norm if case["kind"] in ("norm", "norm_bwd") else _exact_attn)(case, st)
    return {x: t.detach() for x, t in out.items()}
