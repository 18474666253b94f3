"""The operators of a training step of the layer's base model, and what is timed of them.

The base model of the layer is its single-state form (arXiv 2606.10650, Sec. 2.1):
S_t = exp(g_t) S_{t-1} + k_t v_t^T, o_t = scale S_t^T q_t.  Three operators train it
and carry its state from token to token:

  recurrence   that recurrence over long sequences ("fwd"), with its backward pass
               ("train": forward, then backward) and token by token ("step")
  norm         root-mean-square norm of the residual stream plus a branch's output:
               forward and backward ("train"), or with an 8-bit output ("fp8")
  adamw        one AdamW step over all tensors of a model at once, its states in
               float32 or in 8 bits with a scale per 256 elements

Layouts are those of a program around them: q, k and v are slices of one projection's
output, [batch][token][head][d] in memory, gates are another projection's output.
"""
import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
F8 = torch.float8_e4m3fn
F8_MAX = 448.0
BLOCK = 256          # elements per scale of the 8-bit states


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def _rec(name, kind, **kw):
    c = {"name": name, "op": "recurrence", "kind": kind, "B": 1, "H": 16, "Hk": 0, "T": 1,
         "dk": 128, "dv": 128, "dtype": "bf16", "state": False, "ragged": False, "docs": 0,
         "g_lo": -0.05}
    c.update(kw)
    c["Hk"] = c["Hk"] or c["H"]
    return c


def _norm(name, kind, **kw):
    c = {"name": name, "op": "norm", "kind": kind, "rows": 1, "D": 2048, "dtype": "bf16"}
    c.update(kw)
    return c


def _adamw(name, **kw):
    c = {"name": name, "op": "adamw", "D": 2048, "H": 16, "layers": 1, "params": "bf16",
         "states": "f32"}
    c.update(kw)
    return c


def listed():
    return [
        # a training step's longest sequences: 4 x 16k tokens of 16 heads
        _rec("train_4x16k", "train", B=4, H=16, T=16384),
        # ordinary training batches, documents of about 1000 tokens packed into sequences
        _rec("train_8x4k_docs", "train", B=8, H=16, T=4096, docs=1000),
        # the head shape of Mamba-2-780M: 48 heads that share one key head
        _rec("train_shared_keys", "train", B=2, H=48, Hk=1, T=2048, dv=64),
        # a float32 layer, small heads, ragged sequences of a batch (one of them empty)
        # that go on from the state of the tokens before (truncated backpropagation)
        _rec("train_f32_ragged", "train", B=3, H=5, T=1531, dk=64, dv=64, dtype="f32",
             state=True, ragged=True),
        # the prompt of one very long document
        _rec("prompt_64k", "fwd", B=1, H=8, T=65536, state=True, g_lo=-0.01),
        # serving: a token for each of 64 sequences of 32 heads, and for one sequence
        _rec("step_64x32", "step", B=64, H=32, state=True),
        _rec("step_1x32", "step", B=1, H=32, state=True),
        # training: the norm before a layer, 4 x 16k tokens
        _norm("norm_train_64k", "train", rows=65536),
        # serving: 64 tokens, the norm's output in 8 bits for the projection that follows
        _norm("norm_fp8_64", "fp8", rows=64, D=4096),
        # a small float32 model's parameters, where launches count
        _adamw("adamw_small", D=128, H=2, layers=2, params="f32"),
        # 134M parameters in bfloat16 with float32 masters, states in float32 and in 8 bits
        _adamw("adamw_134m", layers=8),
        _adamw("adamw_134m_fp8", layers=8, states="fp8"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["recurrence", "recurrence", "recurrence", "norm", "adamw"])
    if op == "norm":
        D = rng.choice([_log(rng, 32, 8192), 128 * _log(rng, 1, 20)])
        c = _norm("", rng.choice(["train", "fp8"]), D=D, dtype=rng.choice(["bf16", "bf16", "f32"]),
                  rows=_log(rng, 1, min(131072, 134000000 // D)))
    elif op == "adamw":
        c = _adamw("", D=rng.choice([_log(rng, 32, 2048), 64 * _log(rng, 1, 32)]),
                   H=rng.choice([1, 2, 5, 16, 32]), params=rng.choice(["bf16", "f32"]),
                   states=rng.choice(["f32", "fp8"]))
        c["layers"] = _log(rng, 1, max(1, min(40, 134000000 // (4 * c["D"] ** 2 + c["D"] * c["H"]))))
    else:
        kind = rng.choice(["train", "train", "fwd", "step"])
        c = _rec("", kind, g_lo=rng.choice([-0.01, -0.05, -0.5]))
        c["dk"], c["dv"] = rng.choice([(128, 128), (128, 128), (128, 64), (64, 64), (64, 128)])
        c["dtype"] = rng.choice(["bf16", "bf16", "bf16", "f32"])
        c["H"] = rng.choice([1, 3, 5, 8, 16, 24, 32, 48])
        c["Hk"] = rng.choice([h for h in (1, c["H"], c["H"], c["H"] // 2, c["H"] // 3)
                              if h and c["H"] % h == 0])
        if kind == "step":
            c["B"], c["T"], c["state"] = _log(rng, 1, 64), rng.choice([1, 1, 1, 2, 5]), True
        else:
            c["T"] = _log(rng, 2, 16384 if c["dtype"] == "bf16" else 4096)
            c["B"] = max(1, min(_log(rng, 1, 32), 1048576 // (c["T"] * c["H"])))
            c["state"], c["ragged"] = rng.random() < 0.4, rng.random() < 0.4
            c["docs"] = rng.choice([0, 0, _log(rng, 10, 2000)])
    del c["name"]
    return c if 3072 not in c.values() else draw(rng)    # no configuration here has that size


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + 17)


def _heads(x, off, n, d):
    """n heads of size d of a projection's output [B, T, width], as [B, n, T, d]."""
    return x[..., off:off + n * d].unflatten(-1, (n, d)).transpose(1, 2)


def _prepare_recurrence(c, seed):
    gen = _gen(seed)
    B, H, Hk, T, dk, dv, dt = (c[x] for x in ("B", "H", "Hk", "T", "dk", "dv", "dtype"))
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    # one projection's output: queries and keys of length one, values N(0, 1)
    qk = torch.nn.functional.normalize(rnd(B, T, 2 * Hk, dk), dim=-1).flatten(2)
    x = torch.cat([qk, rnd(B, T, H * dv)], -1).to(DT[dt])
    g = c["g_lo"] * torch.rand((B, T, H), generator=gen, device="cuda")
    if c["docs"]:      # a document's first token forgets what was before it
        g[torch.rand((B, T), generator=gen, device="cuda") < 1.0 / c["docs"]] = -math.inf
    s = {"case": c, "x": x, "g": g.transpose(1, 2), "scale": 1.0,
         "q": _heads(x, 0, Hk, dk), "k": _heads(x, Hk * dk, Hk, dk),
         "v": _heads(x, 2 * Hk * dk, H, dv), "S": None, "len": None}
    if c["state"]:
        s["S"] = rnd(B, H, dk, dv) / dk ** 0.5
    if c["ragged"]:
        n = torch.randint(0, T + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
        n[0], n[-1] = T, 0 if B > 1 else T - T // 3
        s["len"] = n
        pad = torch.arange(T, device="cuda")[None] >= n[:, None]
        x[pad] = math.nan        # what lies behind a sequence's end is not read as a token
        s["g"].transpose(1, 2)[pad] = math.nan
    if c["kind"] == "train":
        s["do"] = rnd(B, T, H, dv).to(DT[dt]).transpose(1, 2)
        s["dS"] = rnd(B, H, dk, dv) / dk ** 0.5 if c["state"] else None
    if own:
        from paper_2606_10650_amd import train
        s["workspace"] = torch.empty(
            max(256, train.recurrence_workspace_bytes(B, H, Hk, T, dk, dv, DT[dt],
                                                      backward=c["kind"] == "train")),
            dtype=torch.uint8, device="cuda")
    return s


def _prepare_norm(c, seed):
    gen = _gen(seed)
    N, D, dt = c["rows"], c["D"], DT[c["dtype"]]
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    s = {"case": c, "x": rnd(N, D).to(dt), "res": (2 * rnd(N, D)).to(dt),
         "w": (1 + 0.1 * rnd(D)).to(dt), "eps": 1e-6}
    if c["kind"] == "train":
        s["dy"], s["dres"] = rnd(N, D).to(dt), rnd(N, D).to(dt)
        if own:
            from paper_2606_10650_amd import train
            s["workspace"] = torch.empty(max(256, train.rms_norm_workspace_bytes(N, D)),
                                         dtype=torch.uint8, device="cuda")
    return s


def _tensors(c):
    """(elements, whether weight decay applies) of a model's parameters: per layer the
    projections of q, k, v and the output, the gates' with its bias, and a norm."""
    D, H = c["D"], c["H"]
    return [(D * D, True)] * 4 + [(D * H, True), (H, False), (D, False)]


def _prepare_adamw(c, seed):
    gen = _gen(seed)
    sizes = _tensors(c) * c["layers"]
    at, ends = [0], []
    for n, _ in sizes:           # each tensor starts at a multiple of a block
        ends.append(at[-1] + n)
        at.append(at[-1] + -(-n // BLOCK) * BLOCK)
    total, dt = at[-1], DT[c["params"]]
    inside = torch.ones(total, device="cuda", dtype=torch.bool)
    for a, e, z in zip(at, ends, at[1:]):
        inside[e:z] = False

    def rnd(f):
        return f * torch.randn(total, generator=gen, device="cuda") * inside

    master = rnd(0.02)
    m = rnd(1e-3)
    # second moments whose sizes differ between neighbours, as those of weights do
    r = 1e-3 * torch.exp(0.7 * torch.randn(total, generator=gen, device="cuda")) * inside
    s = {"case": c, "sizes": sizes, "at": at, "step": 1000, "grad": rnd(1e-3).to(dt),
         "p": master.to(dt), "master": master if c["params"] == "bf16" else None,
         "hyper": {"lr": 3e-4, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "weight_decay": 0.1}}
    if c["states"] == "f32":
        s["m"], s["v"] = m, r * r
    else:
        (s["m"], s["ms"]), (s["v"], s["vs"]) = _codes(m, None), _codes(r, None)
    # per block: its tensor's number, its first element's index there, its weight decay
    nb = torch.tensor([(z - a) // BLOCK for a, z in zip(at, at[1:])], device="cuda")
    first = torch.tensor(at[:-1], device="cuda") // BLOCK
    s["tensor"] = torch.arange(len(sizes), device="cuda").repeat_interleave(nb)
    s["first"] = (torch.arange(total // BLOCK, device="cuda") - first.repeat_interleave(nb)) * BLOCK
    s["wd"] = torch.tensor([0.1 if d else 0.0 for _, d in sizes], device="cuda").repeat_interleave(nb)
    if own:
        from paper_2606_10650_amd import train
        part = lambda x, i: x[at[i]:ends[i]]  # noqa: E731
        blocks = lambda x, i: x[at[i] // BLOCK:at[i + 1] // BLOCK]  # noqa: E731
        plan = train.AdamW()
        for i, (_, decay) in enumerate(sizes):
            q = c["states"] == "fp8"
            plan.add(part(s["p"], i), part(s["grad"], i), part(s["m"], i), part(s["v"], i),
                     master=part(master, i) if c["params"] == "bf16" else None,
                     m_scale=blocks(s["ms"], i) if q else None,
                     v_scale=blocks(s["vs"], i) if q else None,
                     weight_decay=0.1 if decay else 0.0)
        s["plan"] = plan
    return s


def prepare(case, seed):
    f = {"recurrence": _prepare_recurrence, "norm": _prepare_norm, "adamw": _prepare_adamw}
    return f[case["op"]](case, seed)


# ---------------------------------------------------------------------------
# the recurrence in its plain form: chunks of tokens, products of whole matrices
# ---------------------------------------------------------------------------
CHUNK = 64


class _Chunks:
    """Tokens by chunks, in float32, and the decays between them.  Sums of log decays
    are taken in float64: their differences are what counts, after any number of
    tokens.  A gate of -inf is counted apart, so that nothing subtracts infinities."""

    def __init__(self, c, g, n):
        self.c, self.T, self.nc = c, c["T"], -(-c["T"] // CHUNK)
        B, H = c["B"], c["H"]
        t = torch.arange(self.T, device="cuda")
        self.live = None if n is None else (t[None] < n[:, None])[:, None]       # [B, 1, T]
        g = g.double() if self.live is None else torch.where(self.live, g.double(), 0.0)
        g = torch.nn.functional.pad(g, (0, self.nc * CHUNK - self.T)).view(B, H, self.nc, CHUNK)
        cut = torch.isinf(g)
        a, r = torch.where(cut, 0.0, g).cumsum(-1), cut.cumsum(-1)
        self.whole = lambda a, r: torch.where(r == 0, torch.exp(a), 0.0).float()  # noqa: E731
        tri = torch.ones((CHUNK, CHUNK), device="cuda", dtype=torch.bool).tril()
        same = (r[..., :, None] == r[..., None, :]) & tri
        self.D = torch.where(same, torch.exp(torch.where(tri, a[..., :, None] - a[..., None, :], 0.0)),
                             0.0).float()
        self.into = self.whole(a, r)[..., None]                       # from before the chunk
        self.end = self.whole(a[..., -1:] - a, r[..., -1:] - r)[..., None]   # to the chunk's end
        # from the end of chunk j - 1 (0: before all) to the end of chunk i - 1
        A = torch.nn.functional.pad(a[..., -1].cumsum(-1), (1, 0))
        R = torch.nn.functional.pad(r[..., -1].cumsum(-1), (1, 0))
        tri = torch.ones((self.nc + 1,) * 2, device="cuda", dtype=torch.bool).tril()
        same = (R[..., :, None] == R[..., None, :]) & tri
        self.W = torch.where(same, torch.exp(torch.where(tri, A[..., :, None] - A[..., None, :], 0.0)),
                             0.0).float()
        self.tot = self.whole(a[..., -1], r[..., -1])                 # a whole chunk's decay

    def __call__(self, x):
        """[B, heads, T, d] -> [B, H, nc, CHUNK, d], zero behind the sequences' ends."""
        x = x.float()
        if self.live is not None:
            x = torch.where(self.live[..., None], x, 0.0)
        x = x.repeat_interleave(self.c["H"] // x.shape[1], 1)
        x = torch.nn.functional.pad(x, (0, 0, 0, self.nc * CHUNK - self.T))
        return x.view(*x.shape[:2], self.nc, CHUNK, x.shape[-1])

    def tokens(self, x, heads, dtype):
        """Back to [B, heads, T, d]; heads that share a tensor's head add up."""
        x = x.flatten(2, 3)[:, :, :self.T]
        B, H, T, d = x.shape
        if heads != H:
            x = x.view(B, heads, H // heads, T, d).sum(2)
        return x.to(dtype)


def _states(ch, k, v, S0):
    """State before each chunk, and behind the last."""
    kv = (k * ch.end).transpose(-1, -2) @ v                          # [B, H, nc, dk, dv]
    first = torch.zeros_like(kv[:, :, :1]) if S0 is None else S0[:, :, None]
    z = torch.cat([first, kv], 2)
    S = (ch.W @ z.flatten(3)).view_as(z)
    return S[:, :, :-1], S[:, :, -1]


def _plain_forward(s):
    c = s["case"]
    ch = _Chunks(c, s["g"], s["len"])
    q, k, v = ch(s["q"]) * s["scale"], ch(s["k"]), ch(s["v"])
    S, last = _states(ch, k, v, s["S"])
    o = (q @ k.transpose(-1, -2) * ch.D) @ v + ch.into * (q @ S)
    return ch.tokens(o, c["H"], DT[c["dtype"]]), last


def _plain_backward(s):
    c = s["case"]
    dt, Hk = DT[c["dtype"]], c["Hk"]
    ch = _Chunks(c, s["g"], s["len"])
    q, k, v, do = ch(s["q"]) * s["scale"], ch(s["k"]), ch(s["v"]), ch(s["do"])
    S, last = _states(ch, k, v, s["S"])
    # what later chunks, and the last state, ask of the state behind each chunk
    qd = (q * ch.into).transpose(-1, -2) @ do
    end = torch.zeros_like(qd[:, :, :1]) if s["dS"] is None else s["dS"][:, :, None]
    z = torch.cat([qd, end], 2)
    R = (ch.W.transpose(-1, -2).contiguous() @ z.flatten(3)).view_as(z)
    dS0, R = R[:, :, 0], R[:, :, 1:]
    qk, dov = q @ k.transpose(-1, -2), do @ v.transpose(-1, -2)
    into = ch.into * (do @ S.transpose(-1, -2))
    outof = ch.end * (v @ R.transpose(-1, -2))
    dq = ((dov * ch.D) @ k + into) * s["scale"]
    dk = (dov * ch.D).transpose(-1, -2) @ q + outof
    dv = (qk * ch.D).transpose(-1, -2) @ do + ch.end * (k @ R)
    # g_t decays what tokens s < t leave for tokens u >= t: pairs inside the chunk, those
    # with one end before or behind it, and those that span it
    strict = torch.ones((CHUNK, CHUNK), device="cuda").tril(-1)
    A = qk * dov * ch.D * strict
    before = A.cumsum(-1) - A                                         # [u, t]: sum over s < t
    dg = (before * torch.ones((CHUNK, CHUNK), device="cuda").tril()).sum(-2)
    dg += (q * into).sum(-1).flip(-1).cumsum(-1).flip(-1)
    right = (k * outof).sum(-1)
    dg += right.cumsum(-1) - right
    dg += (ch.tot * (R * S).sum((-1, -2)))[..., None]
    # a gate of -inf lets nothing through
    dg = dg.flatten(2)[:, :, :c["T"]]
    dg = torch.where(torch.isinf(s["g"]), 0.0, dg)
    if ch.live is not None:
        dg = torch.where(ch.live, dg, 0.0)
    return (ch.tokens(dq, Hk, dt), ch.tokens(dk, Hk, dt), ch.tokens(dv, c["H"], dt), dg.to(dt),
            dS0 if s["S"] is not None else None)


def _run_recurrence(s):
    c = s["case"]
    if own:
        from paper_2606_10650_amd import train
        kw = dict(scale=s["scale"], state=s["S"], lengths=s["len"], workspace=s["workspace"])
        step = c["kind"] == "step"      # serving keeps one state and updates it
        out, last = train.recurrence(s["q"], s["k"], s["v"], s["g"], **kw,
                                     state_out=s["S"] if step else None, want_state=c["state"])
    else:
        out, last = _plain_forward(s)
        if c["kind"] == "step":
            s["S"].copy_(last)
    r = {"out": out, "state": last if c["state"] else None}
    if c["kind"] == "train":
        if own:
            g = train.recurrence_backward(s["q"], s["k"], s["v"], s["g"], s["do"],
                                          dstate=s["dS"], **kw)
        else:
            g = _plain_backward(s)
        r.update(zip(("dq", "dk", "dv", "dg", "dstate"), g))
    return r


# ---------------------------------------------------------------------------
# norm and AdamW in their plain forms
# ---------------------------------------------------------------------------
def _run_norm(s):
    c = s["case"]
    fp8, dt = c["kind"] == "fp8", DT[c["dtype"]]
    if own:
        from paper_2606_10650_amd import train
        if fp8:
            y, h, scale = train.rms_norm_fp8(s["x"], s["w"], s["res"], eps=s["eps"])
            return {"y": y, "h": h, "scale": scale}
        y, h, rstd = train.rms_norm(s["x"], s["w"], s["res"], eps=s["eps"])
        dx, dw = train.rms_norm_backward(s["dy"], h, s["w"], rstd, dres=s["dres"],
                                         workspace=s["workspace"])
        return {"y": y, "h": h, "dx": dx, "dw": dw}
    h = s["x"].float() + s["res"].float()
    w = s["w"].float()
    rstd = torch.rsqrt(h.square().mean(-1, keepdim=True) + s["eps"])
    n = h * rstd
    y = n * w
    if fp8:
        amax = y.abs().amax(-1, keepdim=True)
        q = torch.where(amax > 0, y * (F8_MAX / amax), 0.0).clamp(-F8_MAX, F8_MAX)
        return {"y": q.to(F8), "h": h.to(dt), "scale": amax[:, 0] / F8_MAX}
    # the backward pass starts from what the forward pass stored
    h16 = h.to(dt)
    n = h16.float() * rstd
    dn = s["dy"].float() * w
    dx = (dn - n * (dn * n).mean(-1, keepdim=True)) * rstd + s["dres"].float()
    return {"y": y.to(dt), "h": h16, "dx": dx.to(dt), "dw": (s["dy"].float() * n).sum(0)}


def _codes(x, u, least=False):
    """8-bit floating-point codes of x and their scales, a block of 256 at a time.  u: a
    number in [0, 1) per element that decides which neighbour a value is rounded to, or
    None for the nearest.  least: a value above zero gets a code above zero."""
    x = x.view(-1, BLOCK)
    amax = x.abs().amax(-1, keepdim=True)
    y = torch.where(amax > 1e-30, x * (F8_MAX / amax), 0.0).clamp(-F8_MAX, F8_MAX)
    if u is not None:
        step = torch.exp2(torch.frexp(y).exponent.clamp(min=-5).float() - 4)
        n = torch.floor(y.abs() / step + u.view_as(y)) * step
        y = torch.copysign(n.clamp(max=F8_MAX), y)
    if least:
        y = torch.where((x > 0) & (amax > 1e-30), y.clamp(min=2.0 ** -9), y)
    return y.to(F8).view(-1), torch.where(amax > 1e-30, amax / F8_MAX, 0.0).view(-1)


def _values(code, scale):
    return (code.view(-1, BLOCK).float() * scale[:, None]).view(-1)


def _uniform(s, seed):
    """Two numbers in [0, 1) of 16 bits per element, from the seed, the tensor's number
    and the element's index in it."""
    low = 0xFFFFFFFF
    i = s["first"][:, None] + torch.arange(BLOCK, device="cuda")[None]
    h = (i + 0x9E3779B9 * (s["tensor"][:, None] + 1) & low) ^ seed
    h = h * 0x2545F491 & low
    h = h ^ h >> 16
    h = h * 0x9E3779B1 & low
    h = (h ^ h >> 15).view(-1)
    return (h >> 16).float() / 65536, (h & 0xFFFF).float() / 65536


def _run_adamw(s):
    c, hy = s["case"], s["hyper"]
    s["step"] += 1
    seed = s["step"] * 40503 % 65521 + 1      # the program's random numbers: one per step
    fp8 = c["states"] == "fp8"
    if own:
        s["plan"].step(s["step"], lr=hy["lr"], betas=(hy["beta1"], hy["beta2"]), eps=hy["eps"],
                       seed=seed if fp8 else 0)
    else:
        g = s["grad"].float()
        m = _values(s["m"], s["ms"]) if fp8 else s["m"]
        v = _values(s["v"], s["vs"]).square() if fp8 else s["v"]
        m = hy["beta1"] * m + (1 - hy["beta1"]) * g
        v = hy["beta2"] * v + (1 - hy["beta2"]) * g * g
        p = s["p"].float() if s["master"] is None else s["master"]
        denom = (v / (1 - hy["beta2"] ** s["step"])).sqrt() + hy["eps"]
        decay = (1 - hy["lr"] * s["wd"])[:, None].expand(-1, BLOCK).reshape(-1)
        p = p * decay - hy["lr"] / (1 - hy["beta1"] ** s["step"]) * m / denom
        if s["master"] is not None:
            s["master"].copy_(p)
        s["p"].copy_(p)
        if fp8:
            um, uv = _uniform(s, seed)
            for name, x in (("m", _codes(m, um)), ("v", _codes(v.sqrt(), uv, least=True))):
                s[name].copy_(x[0])
                s[name + "s"].copy_(x[1])
        else:
            s["m"].copy_(m)
            s["v"].copy_(v)
    names = ("p", "master", "m", "v") + (("ms", "vs") if fp8 else ())
    return {n: s[n] for n in names if s[n] is not None}


def run(state):
    f = {"recurrence": _run_recurrence, "norm": _run_norm, "adamw": _run_adamw}
    return f[state["case"]["op"]](state)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    c = case
    if c["op"] == "norm":
        e, n = 2 if c["dtype"] == "bf16" else 4, c["rows"] * c["D"]
        # x, residual, h; then y, or in training also dy, dres, h again and dx
        b = n * (3 * e + 1) + 4 * c["rows"] if c["kind"] == "fp8" else n * 8 * e + 4 * c["rows"]
        return {"bytes": b + 4 * c["D"], "flops": n * (8 if c["kind"] == "fp8" else 20)}
    if c["op"] == "adamw":
        n = sum(x for x, _ in _tensors(c)) * c["layers"]
        e = 2 if c["params"] == "bf16" else 4
        b = 2 * e + (8 if c["params"] == "bf16" else 0) + (e if c["params"] == "f32" else 0)
        return {"bytes": n * (b + (16 if c["states"] == "f32" else 4)), "flops": 16 * n}
    e = 2 if c["dtype"] == "bf16" else 4
    B, H, Hk, T, dk, dv = (c[x] for x in ("B", "H", "Hk", "T", "dk", "dv"))
    if c["ragged"]:
        T = T / 2                               # sequences' lengths are spread over 0..T
    keys, vals, D = B * Hk * T * dk * e, B * H * T * dv * e, B * H * dk * dv
    b = 2 * keys + 2 * vals + 4 * B * H * T + (8 * D if c["state"] else 0)
    f = 4 * D * T                               # k v^T into the state, the state times q
    if c["kind"] == "train":
        b += 4 * keys + 3 * vals + (4 + e) * B * H * T + (12 * D if c["state"] else 0)
        f += 10 * D * T                         # the states again, their adjoints, dq, dk, dv
    return {"bytes": b, "flops": f}


# ---------------------------------------------------------------------------
# the same in 64 bits, token by token and from the definitions
# ---------------------------------------------------------------------------
def _exact_recurrence(c, s):
    B, H, T, dk, dv = (c[x] for x in ("B", "H", "T", "dk", "dv"))
    nh, f64 = B * H, torch.float64
    n = s["len"].tolist() if s["len"] is not None else [T] * B
    behind = torch.tensor(n, device="cuda")[:, None] <= torch.arange(T, device="cuda")[None]

    def rows(x):       # [T, B * H, d], contiguous per token
        x = x.double().masked_fill(behind[:, None, :, None], 0.0)
        x = x.repeat_interleave(H // x.shape[1], 1)
        return x.permute(2, 0, 1, 3).reshape(T, nh, x.shape[-1]).contiguous()

    q, k, v = rows(s["q"]) * s["scale"], rows(s["k"]), rows(s["v"])
    gate = s["g"].double().masked_fill(behind[:, None], 0.0).exp().permute(2, 0, 1).reshape(T, nh, 1, 1)
    zero = torch.zeros((nh, dk, dv), dtype=f64, device="cuda")
    S = zero if s["S"] is None else s["S"].double().view(nh, dk, dv)
    o = torch.empty((T, nh, dv), dtype=f64, device="cuda")
    train = c["kind"] == "train"
    if train:
        do = rows(s["do"])
        dq = torch.empty_like(q)
    for t in range(T):
        S = torch.baddbmm(S * gate[t], k[t, :, :, None], v[t, :, None])
        o[t] = (S * q[t, :, :, None]).sum(1)
        if train:
            dq[t] = (S * do[t, :, None]).sum(2)
    heads = lambda x: x.view(T, B, H, -1).permute(1, 2, 0, 3)  # noqa: E731
    r = {"out": heads(o), "state": S.view(B, H, dk, dv) if c["state"] else None}
    if not train:
        return r
    # the adjoint of S_t, from the last token back; dg_t = <adjoint, exp(g_t) S_{t-1}>,
    # where <adjoint of S_t, S_t> is carried along
    R = zero if s["dS"] is None else s["dS"].double().view(nh, dk, dv)
    dk_, dv_ = torch.empty_like(k), torch.empty_like(v)
    dg = torch.empty((T, nh), dtype=f64, device="cuda")
    along = (R * S).sum((1, 2))
    qdq = (q * dq).sum(-1)
    for t in reversed(range(T)):
        R = torch.baddbmm(R, q[t, :, :, None], do[t, :, None])
        dk_[t] = (R * v[t, :, None]).sum(2)
        dv_[t] = (R * k[t, :, :, None]).sum(1)
        along = along + qdq[t] - (k[t] * dk_[t]).sum(-1)
        dg[t] = along = along * (gate[t, :, 0, 0] != 0)
        R = R * gate[t]
    group = lambda x: heads(x).unflatten(1, (c["Hk"], -1)).sum(2)  # noqa: E731
    dg = heads(dg)[..., 0].masked_fill(behind[:, None], 0.0)
    r.update(dq=group(dq) * s["scale"], dk=group(dk_), dv=heads(dv_), dg=dg,
             dstate=R.view(B, H, dk, dv) if c["state"] else None)
    return r


def _exact_norm(c, s):
    x, r, w = s["x"].double(), s["res"].double(), s["w"].double()
    h = x + r
    rms = (h.pow(2).sum(-1, keepdim=True) / c["D"] + s["eps"]).sqrt()
    y = h / rms * w
    if c["kind"] == "fp8":
        top = y.abs().max(-1, keepdim=True).values
        return {"y": y / top * F8_MAX, "h": h, "scale": top[:, 0] / F8_MAX}
    # y_i = w_i h_i / rms, rms = sqrt(|h|^2 / D + eps)
    wdy = w * s["dy"].double()
    dx = wdy / rms - h * (wdy * h).sum(-1, keepdim=True) / (c["D"] * rms ** 3)
    return {"y": y, "h": h, "dx": dx + s["dres"].double(), "dw": (s["dy"].double() * h / rms).sum(0)}


def _exact_adamw(c, s):
    hy, t, fp8 = s["hyper"], s["step"] + 1, c["states"] == "fp8"
    spread = lambda x: x.double().repeat_interleave(BLOCK)  # noqa: E731
    m, v = s["m"].double(), s["v"].double()
    if fp8:
        m, v = m * spread(s["ms"]), (v * spread(s["vs"])) ** 2
    g = s["grad"].double()
    m += (1 - hy["beta1"]) * (g - m)
    v += (1 - hy["beta2"]) * (g ** 2 - v)
    p = (s["p"] if s["master"] is None else s["master"]).double()
    p = p - hy["lr"] * spread(s["wd"]) * p
    p -= hy["lr"] * (m / (1 - hy["beta1"] ** t)) / ((v / (1 - hy["beta2"] ** t)).sqrt() + hy["eps"])
    r = {"p": p, "master": p}
    if not fp8:
        r.update(m=m, v=v)
    else:
        # what the codes stand for before they are rounded, in units of the scale
        for name, x in (("m", m), ("v", v.sqrt())):
            top = x.view(-1, BLOCK).abs().max(1).values
            r[name] = torch.nan_to_num(x / top.repeat_interleave(BLOCK)) * F8_MAX
            r[name + "s"] = top / F8_MAX
    if s["master"] is None:
        del r["master"]
    return r


def exact(case, seed):
    global own
    if case["op"] == "recurrence" and case["T"] > 20000:
        return None                              # too many tokens to go one by one
    was, own = own, False                        # inputs only
    try:
        s = prepare(case, seed)
    finally:
        own = was
    f = {"recurrence": _exact_recurrence, "norm": _exact_norm, "adamw": _exact_adamw}
    return f[case["op"]](case, s)
