"""The operators around the recurrence of the layer's base model, and what is timed of them.

A block of the base model (arXiv 2606.10650, Sec. 2.1) projects its input to queries, keys
and values, runs the recurrence and projects back.  Four operators complete such a model,
for training ("train": forward, then backward) and for serving ("fwd", "step"):

  conv       a short causal convolution per channel in front of the recurrence, with its
             SiLU; documents that start inside a sequence, ragged ends, a state of the last
             inputs that is carried from call to call
  norm       the norm behind a block, per head or over the row, with its gate, the scaled
             residual sum, and the norm before the next block
  logprobs   log probabilities of given tokens, the entropy, the top alternatives, and the
             gradient with respect to the logits
  ff         the gated feed-forward block: both projections, the activation, the product

Layouts are those of a program around them: a convolution's inputs and a norm's gates are
slices of a wider projection's output.
"""
import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def _conv(name, kind, **kw):
    c = {"name": name, "op": "conv", "kind": kind, "B": 1, "T": 1, "C": 6144, "W": 4, "extra": 64,
         "dtype": "bf16", "silu": True, "bias": False, "state": False, "ragged": False, "docs": 0}
    c.update(kw)
    return c


def _norm(name, kind, **kw):
    c = {"name": name, "op": "norm", "kind": kind, "rows": 1, "G": 1, "D": 2048, "dtype": "bf16",
         "gate": False, "residual": False, "next": False, "scale": 1.0, "per_group": False}
    c.update(kw)
    return c


def _logprobs(name, kind, **kw):
    c = {"name": name, "op": "logprobs", "kind": kind, "rows": 1, "V": 50304, "dtype": "bf16",
         "entropy": False, "top": 0, "ignored": 0.0, "masked": 0.0}
    c.update(kw)
    return c


def _ff(name, kind, **kw):
    c = {"name": name, "op": "ff", "kind": kind, "rows": 1, "D": 2048, "F": 5504, "dtype": "bf16"}
    c.update(kw)
    return c


def listed():
    return [
        # q, k and v of 16 heads of 128, a training step's 4 x 16k tokens, packed documents
        _conv("conv_train_4x16k", "train", B=4, T=16384, docs=1000),
        # a float32 layer of odd width, ragged sequences that go on from earlier tokens
        _conv("conv_f32_ragged", "train", B=3, T=1531, C=321, W=3, extra=0, dtype="f32", bias=True,
              state=True, ragged=True),
        # serving: one token for each of 64 sequences
        _conv("conv_step_64", "step", B=64, state=True),
        # behind the recurrence: 4 x 16k tokens of 16 heads of 128, gated by a projection
        _norm("heads_norm_train", "train", rows=65536, G=16, D=128, gate=True),
        # between two blocks: norm, scaled residual sum, norm; 4 x 4k tokens
        _norm("block_norm_train", "train", rows=16384, residual=True, next=True, scale=0.5),
        # the same for the tokens of 64 sequences, with a gate
        _norm("block_norm_64", "fwd", rows=64, gate=True, residual=True, next=True, scale=0.5),
        # the loss of 8k tokens, with the entropy of every prediction
        _logprobs("loss_8k", "train", rows=8192, entropy=True),
        # a float32 model's loss, an odd vocabulary, prompt tokens that do not count, some of
        # the vocabulary shut out
        _logprobs("loss_f32_odd", "train", rows=1000, V=32003, dtype="f32", ignored=0.3, masked=0.01),
        # serving: the answer tokens of 64 sequences, each with 20 alternatives
        _logprobs("answers_64", "fwd", rows=64, entropy=True, top=20),
        # a training step's 16k tokens
        _ff("ff_train_16k", "train", rows=16384),
        # a small float32 model, odd sizes
        _ff("ff_train_f32", "train", rows=1531, D=321, F=1000, dtype="f32"),
        # serving: the tokens of 16 sequences
        _ff("ff_step_16", "fwd", rows=16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["conv", "norm", "logprobs", "ff"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op == "conv":
        kind = rng.choice(["train", "train", "fwd", "step"])
        c = _conv("", kind, C=rng.choice([_log(rng, 24, 6144), 64 * _log(rng, 1, 96)]), W=rng.choice([2, 3, 4, 4]),
                  extra=rng.choice([0, 1, 64, 2048]), silu=rng.random() < 0.8, bias=rng.random() < 0.4)
        if kind == "step":
            c["B"], c["T"], c["state"] = _log(rng, 1, 256), rng.choice([1, 1, 1, 2, 5]), True
        else:
            c["T"] = _log(rng, 2, 16384)
            c["B"] = max(1, min(_log(rng, 1, 64), 100000000 // (c["T"] * (c["C"] + c["extra"]))))
            c["state"], c["ragged"] = rng.random() < 0.4, rng.random() < 0.4
            c["docs"] = rng.choice([0, 0, _log(rng, 3, 2000)])
    elif op == "norm":
        c = _norm("", rng.choice(["train", "train", "fwd"]), scale=rng.choice([1.0, 0.5, 0.17]))
        if rng.random() < 0.5:      # heads
            c["G"], c["D"] = rng.choice([1, 3, 8, 16, 32, 48]), rng.choice([64, 64, 128, 128, _log(rng, 16, 256)])
            c["gate"], c["per_group"] = rng.random() < 0.8, rng.random() < 0.4
        else:                       # rows
            c["D"] = rng.choice([_log(rng, 32, 8192), 128 * _log(rng, 1, 40)])
            c["gate"], c["residual"], c["next"] = rng.random() < 0.4, rng.random() < 0.8, rng.random() < 0.7
        c["rows"] = _log(rng, 1, max(1, min(65536, 67000000 // (c["G"] * c["D"]))))
    elif op == "logprobs":
        c = _logprobs("", rng.choice(["train", "fwd"]), V=rng.choice([_log(rng, 64, 262144), 128 * _log(rng, 8, 1200)]),
                      entropy=rng.random() < 0.5, ignored=rng.choice([0.0, 0.3]), masked=rng.choice([0.0, 0.0, 0.01, 0.9]))
        if c["kind"] == "fwd":
            c["top"] = rng.choice([0, 1, 5, 20])
        c["rows"] = _log(rng, 1, max(1, min(16384, (200 if c["kind"] == "train" else 20) * 1000000 // c["V"])))
    else:
        c = _ff("", rng.choice(["train", "train", "fwd"]), D=rng.choice([_log(rng, 32, 4096), 128 * _log(rng, 1, 32)]),
                F=rng.choice([_log(rng, 32, 8192), 128 * _log(rng, 1, 64)]))
        most = (180 if dtype == "bf16" else 20) * 1000000000 // (c["D"] * c["F"])
        c["rows"] = _log(rng, 1, max(1, min(16384, most)))
    c["dtype"] = dtype
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + 29)


def _prepare_conv(c, seed):
    gen = _gen(seed)
    B, T, C, W, dt = c["B"], c["T"], c["C"], c["W"], DT[c["dtype"]]
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    wide = torch.empty((B, T, C + c["extra"]), device="cuda", dtype=dt)   # one projection's output
    for b in range(B):
        wide[b] = rnd(T, C + c["extra"])
    s = {"case": c, "x": wide[..., :C], "w": (rnd(C, W) / W ** 0.5).to(dt),
         "bias": (0.1 * rnd(C)).to(dt) if c["bias"] else None, "act": "silu" if c["silu"] else None,
         "S": rnd(B, W - 1, C).to(dt) if c["state"] else None, "len": None, "starts": None}
    if c["docs"]:
        s["starts"] = torch.rand((B, T), generator=gen, device="cuda") < 1.0 / c["docs"]
    if c["ragged"]:
        n = torch.randint(0, T + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
        n[0], n[-1] = T, 0 if B > 1 else T - T // 3
        s["len"] = n
        # what lies behind a sequence's end is not read as a token
        wide[torch.arange(T, device="cuda")[None] >= n[:, None]] = math.nan
    if c["kind"] == "train":
        s["dy"] = torch.empty((B, T, C), device="cuda", dtype=dt)
        for b in range(B):
            s["dy"][b] = rnd(T, C)
        s["dS"] = rnd(B, W - 1, C).to(dt) if c["state"] else None
        if own:
            from paper_2606_10650_amd import block
            s["workspace"] = torch.empty(max(256, block.short_conv_workspace_bytes(B, T, C, W, dt)),
                                         dtype=torch.uint8, device="cuda")
    return s


def _prepare_norm(c, seed):
    gen = _gen(seed)
    N, G, D, dt = c["rows"], c["G"], c["D"], DT[c["dtype"]]
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    weight = lambda *s: (1 + 0.1 * rnd(*s)).to(dt)  # noqa: E731
    s = {"case": c, "x": (0.3 * rnd(N, G, D)).to(dt), "w": weight(G, D) if c["per_group"] else weight(D),
         "eps": 1e-6, "gate": None, "res": None, "w2": None, "workspace": None}
    if c["gate"]:        # a slice of a wider projection's output
        s["gate"] = rnd(N, G * D + 64).to(dt)[:, 64:].unflatten(1, (G, D))
    if c["residual"]:
        s["res"] = (2 * rnd(N, G, D)).to(dt)
    if c["next"]:
        s["w2"] = weight(D)
    if c["kind"] == "train":
        s["dh"] = rnd(N, G, D).to(dt)
        s["dy"] = rnd(N, G, D).to(dt) if c["next"] else None
        if own:
            from paper_2606_10650_amd import block
            s["workspace"] = torch.empty(max(256, block.gated_norm_workspace_bytes(N, G, D, dt)),
                                         dtype=torch.uint8, device="cuda")
    return s


def _prepare_logprobs(c, seed):
    gen = _gen(seed)
    N, V = c["rows"], c["V"]
    logits = torch.empty((N, V), device="cuda", dtype=DT[c["dtype"]])
    step = max(1, 67000000 // V)
    for i in range(0, N, step):
        logits[i:i + step] = 2.5 * torch.randn((min(step, N - i), V), generator=gen, device="cuda")
    # what is asked for is likely, and never shut out
    tokens = torch.randint(0, V, (N,), generator=gen, device="cuda")
    likely = torch.rand((N,), generator=gen, device="cuda") * 14
    if c["masked"]:
        shut = torch.rand((V,), generator=gen, device="cuda") < c["masked"]
        logits[:, shut] = -math.inf
    logits[torch.arange(N, device="cuda"), tokens] = likely.to(logits.dtype)
    if c["ignored"]:
        tokens[torch.rand((N,), generator=gen, device="cuda") < c["ignored"]] = -100
    s = {"case": c, "logits": logits, "tokens": tokens}
    if c["kind"] == "train":
        s["dlp"] = torch.full((N,), -1.0 / N, device="cuda")
        # the entropies' weight in the loss, token by token
        s["dent"] = 0.01 / N * torch.rand((N,), generator=gen, device="cuda") if c["entropy"] else None
    return s


def _prepare_ff(c, seed):
    gen = _gen(seed)
    N, D, F, dt = c["rows"], c["D"], c["F"], DT[c["dtype"]]
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    s = {"case": c, "x": rnd(N, D).to(dt), "wg": (rnd(F, D) / D ** 0.5).to(dt), "wu": (rnd(F, D) / D ** 0.5).to(dt),
         "workspace": None}
    if c["kind"] == "train":
        s["dy"] = rnd(N, F).to(dt)
    if own:
        from paper_2606_10650_amd import block
        s["workspace"] = torch.empty(max(256, block.gated_ff_workspace_bytes(N, D, F, dt, backward=c["kind"] == "train")),
                                     dtype=torch.uint8, device="cuda")
    return s


def prepare(case, seed):
    f = {"conv": _prepare_conv, "norm": _prepare_norm, "logprobs": _prepare_logprobs, "ff": _prepare_ff}
    return f[case["op"]](case, seed)


# ---------------------------------------------------------------------------
# plain forms and calls
# ---------------------------------------------------------------------------
def _conv_inputs(s):
    """Inputs in float32 with the state in front, zero behind the sequences' ends; which taps
    of a token see the same document; which tokens there are."""
    c = s["case"]
    B, T, C, W = c["B"], c["T"], c["C"], c["W"]
    t = torch.arange(T, device="cuda")
    live = None if s["len"] is None else t[None] < s["len"][:, None]
    x = s["x"].float()
    if live is not None:
        x = torch.where(live[..., None], x, 0.0)
    first = torch.zeros((B, W - 1, C), device="cuda") if s["S"] is None else s["S"].float()
    x = torch.cat([first, x], 1)
    doc = None
    if s["starts"] is not None:
        doc = torch.nn.functional.pad(s["starts"].int().cumsum(1), (W - 1, 0))
    return x, doc, live


def _conv_plain(s):
    c = s["case"]
    B, T, C, W, dt = c["B"], c["T"], c["C"], c["W"], DT[c["dtype"]]
    x, doc, live = _conv_inputs(s)
    w = s["w"].float()

    def tap(j):
        """The inputs that tap j of each token sees."""
        y = x[:, j:j + T]
        return y if doc is None else y * (doc[:, j:j + T] == doc[:, W - 1:])[..., None]

    z = tap(0) * w[:, 0]
    for j in range(1, W):
        z = z + tap(j) * w[:, j]
    if s["bias"] is not None:
        z = z + s["bias"].float()
    sig = torch.sigmoid(z) if c["silu"] else None
    y = z * sig if c["silu"] else z
    if live is not None:
        y = torch.where(live[..., None], y, 0.0)
    r = {"out": y.to(dt)}
    n = torch.full((B,), T, device="cuda") if s["len"] is None else s["len"].long()
    at = n[:, None] + torch.arange(W - 1, device="cuda")[None]          # where the last inputs are
    seen = torch.ones((B, W - 1, 1), device="cuda")
    if doc is not None:
        seen = (doc.gather(1, at) == doc.gather(1, at[:, -1:]))[..., None].float()
    if c["state"]:
        r["state"] = (x.gather(1, at[..., None].expand(-1, -1, C)) * seen).to(dt)
    if c["kind"] != "train":
        if c["kind"] == "step":
            s["S"].copy_(r["state"])
            r["state"] = s["S"]
        return r
    dz = s["dy"].float()
    if c["silu"]:
        dz = dz * (sig * (1 + z * (1 - sig)))
    if live is not None:
        dz = torch.where(live[..., None], dz, 0.0)
    dx = torch.zeros_like(x)
    dw = []
    for j in range(W):
        d = dz if doc is None else dz * (doc[:, j:j + T] == doc[:, W - 1:])[..., None]
        dx[:, j:j + T] += d * w[:, j]
        dw.append((dz * tap(j)).sum((0, 1), dtype=torch.float64).float())
    if c["state"]:
        dx.scatter_add_(1, at[..., None].expand(-1, -1, C), s["dS"].float() * seen)
        r["dstate"] = dx[:, :W - 1].to(dt)
    r["dx"], r["dw"] = dx[:, W - 1:].to(dt), torch.stack(dw, 1)
    if s["bias"] is not None:
        r["dbias"] = dz.sum((0, 1), dtype=torch.float64).float()
    return r


def _run_conv(s):
    c = s["case"]
    if not own:
        return _conv_plain(s)
    from paper_2606_10650_amd import block
    kw = dict(activation=s["act"], state=s["S"], lengths=s["len"], starts=s["starts"])
    step = c["kind"] == "step"       # serving keeps one state and updates it
    out, last = block.short_conv(s["x"], s["w"], s["bias"], state_out=s["S"] if step else None,
                                 want_state=c["state"], **kw)
    r = {"out": out}
    if c["state"]:
        r["state"] = last
    if c["kind"] == "train":
        r["dx"], r["dw"], db, ds = block.short_conv_backward(s["x"], s["w"], s["dy"], s["bias"], dstate=s["dS"],
                                                             workspace=s["workspace"], **kw)
        if s["bias"] is not None:
            r["dbias"] = db
        if c["state"]:
            r["dstate"] = ds
    return r


def _run_norm(s):
    c = s["case"]
    if own:
        from paper_2606_10650_amd import block
        h, y, rstd, y_rstd = block.gated_norm(s["x"], s["w"], s["gate"], s["res"], scale=c["scale"],
                                              next_weight=s["w2"], eps=s["eps"])
        r = {"h": h, "y": y}
        if c["kind"] == "train":
            g = block.gated_norm_backward(s["dh"], s["x"], s["w"], rstd, s["gate"], s["res"], scale=c["scale"],
                                          next_weight=s["w2"], dy=s["dy"], y_rstd=y_rstd, workspace=s["workspace"])
            r.update(zip(("dx", "dgate", "dres", "dw", "dw2"), g))
            if not c["residual"]:
                r["dres"] = None
        return r
    dt, k, eps = DT[c["dtype"]], c["scale"], s["eps"]
    x, w = s["x"].float(), s["w"].float()
    rstd = torch.rsqrt(x.square().mean(-1, keepdim=True) + eps)
    n = x * rstd
    b = n * w
    if c["gate"]:
        z = s["gate"].float()
        sig = torch.sigmoid(z)
        b = b * (z * sig)
    h = k * b
    if c["residual"]:
        h = s["res"].float() + h
    r = {"h": h.to(dt), "y": None}
    if c["next"]:
        w2 = s["w2"].float()
        rstd2 = torch.rsqrt(h.square().mean(-1, keepdim=True) + eps)
        r["y"] = (h * rstd2 * w2).to(dt)
    if c["kind"] != "train":
        return r
    r.update(dgate=None, dres=None, dw2=None)
    dh = s["dh"].float()
    if c["next"]:
        n2 = h * rstd2
        dy = s["dy"].float()
        d = dy * w2
        r["dw2"] = (dy * n2).sum((0, 1), dtype=torch.float64).float()
        dh = dh + rstd2 * (d - n2 * (d * n2).mean(-1, keepdim=True))
    if c["residual"]:
        r["dres"] = dh.to(dt)
    db = k * dh
    if c["gate"]:
        r["dgate"] = (db * (n * w) * (sig * (1 + z * (1 - sig)))).to(dt)
        db = db * (z * sig)
    r["dw"] = (db * n).sum(0 if c["per_group"] else (0, 1), dtype=torch.float64).float()
    d = db * w
    r["dx"] = (rstd * (d - n * (d * n).mean(-1, keepdim=True))).to(dt)
    return r


def _run_logprobs(s):
    c = s["case"]
    if own:
        from paper_2606_10650_amd import block
        lp, lse, ent, ids, tops = block.token_logprobs(s["logits"], s["tokens"], top=c["top"], entropy=c["entropy"])
        r = {"logprob": lp, "entropy": ent, "ids": ids, "tops": tops}
        if c["kind"] == "train":
            r["dlogits"] = block.token_logprobs_backward(s["logits"], s["tokens"], lp, lse, s["dlp"], entropy=ent,
                                                         dentropy=s["dent"])
        return r
    l, asked = s["logits"].float(), s["tokens"] >= 0
    at = s["tokens"].clamp(min=0)[:, None]
    top = l.amax(-1, keepdim=True)
    e = torch.exp(l - top)
    lse = top + torch.log(e.sum(-1, keepdim=True))
    r = {"logprob": torch.where(asked, (l.gather(1, at) - lse)[:, 0], 0.0), "entropy": None, "ids": None, "tops": None}
    logp = l - lse
    p = torch.exp(logp)
    if c["entropy"]:
        r["entropy"] = torch.where(p > 0, -p * logp, 0.0).sum(-1)
    if c["top"]:
        v, i = torch.sort(l, dim=-1, descending=True, stable=True)     # ties: the lowest index first
        r["ids"], r["tops"] = i[:, :c["top"]].contiguous(), v[:, :c["top"]] - lse
    if c["kind"] == "train":
        dlp = torch.where(asked, s["dlp"], 0.0)[:, None]
        d = -dlp * p
        d.scatter_add_(1, at, dlp)
        if c["entropy"]:
            d -= torch.where(p > 0, s["dent"][:, None] * p * (logp + r["entropy"][:, None]), 0.0)
        r["dlogits"] = d.to(l.dtype if c["dtype"] == "f32" else torch.bfloat16)
    return r


def _run_ff(s):
    c = s["case"]
    train = c["kind"] == "train"
    if own:
        from paper_2606_10650_amd import block
        y, parts = block.gated_ff(s["x"], s["wg"], s["wu"], want_parts=train, workspace=s["workspace"])
        r = {"y": y}
        if train:
            r["dx"], r["dwg"], r["dwu"] = block.gated_ff_backward(s["x"], s["wg"], s["wu"], parts, s["dy"],
                                                                  workspace=s["workspace"])
        return r
    dt = DT[c["dtype"]]
    x, wg, wu = s["x"].float(), s["wg"].float(), s["wu"].float()
    g, u = x @ wg.t(), x @ wu.t()
    sig = torch.sigmoid(g)
    r = {"y": (g * sig * u).to(dt)}
    if train:
        dy = s["dy"].float()
        dg, du = dy * u * (sig * (1 + g * (1 - sig))), dy * (g * sig)
        r.update(dx=(dg @ wg + du @ wu).to(dt), dwg=(dg.t() @ x).to(dt), dwu=(du.t() @ x).to(dt))
    return r


def run(state):
    f = {"conv": _run_conv, "norm": _run_norm, "logprobs": _run_logprobs, "ff": _run_ff}
    return f[state["case"]["op"]](state)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    c, train = case, case["kind"] == "train"
    e = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "conv":
        n = c["B"] * c["T"] * c["C"]
        if c["ragged"]:
            n /= 2                              # sequences' lengths are spread over 0..T
        state = c["B"] * (c["W"] - 1) * c["C"] * e if c["state"] else 0
        b = n * e * (4 if train else 2) + state * (4 if train else 2) + c["C"] * c["W"] * (e + (4 if train else 0))
        return {"bytes": b + (c["B"] * c["T"] if c["docs"] else 0),
                "flops": n * (2 * c["W"] * (4 if train else 1) + (20 if train else 8))}
    if c["op"] == "norm":
        n = c["rows"] * c["G"] * c["D"]
        arrays = 2 + c["gate"] + c["residual"] + c["next"]         # x, h; gate, residual, y
        if train:
            arrays += 2 + c["gate"] + c["residual"] + c["next"]    # dh, dx; dgate, dres, dy
        return {"bytes": n * e * arrays + 8 * c["G"] * c["D"], "flops": n * (40 if train else 16)}
    if c["op"] == "logprobs":
        n = c["rows"] * c["V"]
        return {"bytes": n * e * (2 if train else 1) + c["rows"] * (16 + 12 * c["top"]), "flops": n * (12 if train else 6)}
    N, D, F = c["rows"], c["D"], c["F"]
    if train:
        return {"bytes": e * (2 * N * D + 2 * N * F + 4 * F * D), "flops": 12 * N * D * F}
    return {"bytes": e * (N * D + N * F + 2 * F * D), "flops": 4 * N * D * F}


# ---------------------------------------------------------------------------
# the same in 64 bits, from the definitions
# ---------------------------------------------------------------------------
def _exact_conv(c, s):
    B, T, C, W = c["B"], c["T"], c["C"], c["W"]
    n = [T] * B if s["len"] is None else s["len"].tolist()
    f64 = torch.float64
    w = s["w"].double()
    zeros = lambda *sh: torch.zeros(sh, dtype=f64, device="cuda")  # noqa: E731
    train = c["kind"] == "train"
    dw, db = zeros(C, W), zeros(C)
    outs, states, dxs, dstates = [], [], [], []
    for b in range(B):
        x = s["x"][b, :n[b]].double()
        S = zeros(W - 1, C) if s["S"] is None else s["S"][b].double()
        all_ = torch.cat([S, x])                     # row i is token i - (W - 1)
        # how many tokens back a token's document reaches: those of the state, and all since
        # the last start
        t = torch.arange(n[b], device="cuda")
        begin = torch.full((n[b],), -(W - 1), device="cuda")
        if s["starts"] is not None and n[b]:
            begin = torch.where(s["starts"][b, :n[b]], t, begin).cummax(0).values
        z = zeros(n[b], C)
        if s["bias"] is not None:
            z += s["bias"].double()
        for back in range(W):
            ok = (t - back >= begin)[:, None]
            z += ok * all_[W - 1 - back:W - 1 - back + n[b]] * w[:, W - 1 - back]
        y = z / (1 + torch.exp(-z)) if c["silu"] else z
        outs.append(torch.cat([y, zeros(T - n[b], C)]))
        last = all_[n[b]:].clone()
        if n[b]:
            gone = torch.arange(n[b] - W + 1, n[b], device="cuda") < begin[-1]
            last[gone] = 0
        states.append(last)
        if not train:
            continue
        dz = s["dy"][b, :n[b]].double()
        if c["silu"]:
            q = 1 / (1 + torch.exp(-z))
            dz = dz * (q + z * q * (1 - q))
        d = zeros(n[b] + W - 1, C)
        for back in range(W):
            part = (t - back >= begin)[:, None] * dz
            rows = slice(W - 1 - back, W - 1 - back + n[b])
            d[rows] += part * w[:, W - 1 - back]
            dw[:, W - 1 - back] += (part * all_[rows]).sum(0)
        db += dz.sum(0)
        if s["dS"] is not None:
            dS = s["dS"][b].double()
            if n[b]:
                dS = dS.masked_fill(gone[:, None], 0.0)
            d[n[b]:] += dS
        dxs.append(torch.cat([d[W - 1:], zeros(T - n[b], C)]))
        dstates.append(d[:W - 1])
    r = {"out": torch.stack(outs)}
    if c["state"]:
        r["state"] = torch.stack(states)
    if train:
        r["dx"], r["dw"] = torch.stack(dxs), dw
        if s["bias"] is not None:
            r["dbias"] = db
        if c["state"]:
            r["dstate"] = torch.stack(dstates)
    return r


def _exact_norm(c, s):
    x, w, k, D = s["x"].double(), s["w"].double(), c["scale"], c["D"]
    rms = ((x * x).sum(-1, keepdim=True) / D + s["eps"]).sqrt()
    act = slope = 1.0
    if c["gate"]:
        z = s["gate"].double()
        q = 1 / (1 + torch.exp(-z))
        act, slope = z * q, q + z * q * (1 - q)
    h = k * w * x / rms * act + (s["res"].double() if c["residual"] else 0.0)
    r = {"h": h, "y": None}
    if c["next"]:
        w2, rms2 = s["w2"].double(), ((h * h).sum(-1, keepdim=True) / D + s["eps"]).sqrt()
        r["y"] = w2 * h / rms2
    if c["kind"] != "train":
        return r
    r.update(dgate=None, dres=None, dw2=None)
    dh = s["dh"].double()
    if c["next"]:
        dy = s["dy"].double()
        r["dw2"] = (dy * h / rms2).sum((0, 1))
        dh = dh + w2 * dy / rms2 - h * (w2 * dy * h).sum(-1, keepdim=True) / (D * rms2 ** 3)
    if c["residual"]:
        r["dres"] = dh
    if c["gate"]:
        r["dgate"] = dh * k * w * x / rms * slope
    dn = k * dh * act
    dw = dn * x / rms
    r["dw"] = dw.sum(0) if c["per_group"] else dw.sum((0, 1))
    dn = dn * w
    r["dx"] = dn / rms - x * (dn * x).sum(-1, keepdim=True) / (D * rms ** 3)
    return r


def _exact_logprobs(c, s):
    N, V = c["rows"], c["V"]
    train = c["kind"] == "train"
    r = {"logprob": [], "entropy": [], "tops": [], "dlogits": []}
    step = max(1, 50000000 // V)
    for i in range(0, N, step):                     # rows by parts, for their 64-bit copies
        logp = torch.log_softmax(s["logits"][i:i + step].double(), -1)
        tok = s["tokens"][i:i + step]
        asked, at = tok >= 0, tok.clamp(min=0)[:, None]
        r["logprob"].append((logp.gather(1, at)[:, 0]).masked_fill(~asked, 0.0))
        p = logp.exp()
        plogp = (p * logp).masked_fill(p == 0, 0.0)
        ent = -plogp.sum(-1, keepdim=True)
        r["entropy"].append(ent[:, 0])
        if c["top"]:
            r["tops"].append(logp.topk(c["top"], -1).values)
        if train:
            one = torch.zeros_like(p).scatter_(1, at, 1.0)
            d = (asked * s["dlp"][i:i + step].double())[:, None] * (one - p)
            if c["entropy"]:
                d -= s["dent"][i:i + step].double()[:, None] * (plogp + p * ent)
            r["dlogits"].append(d)
    out = {"logprob": torch.cat(r["logprob"]), "entropy": torch.cat(r["entropy"]) if c["entropy"] else None,
           "ids": None, "tops": torch.cat(r["tops"]) if c["top"] else None}
    if train:
        out["dlogits"] = torch.cat(r["dlogits"])
    return out


def _exact_ff(c, s):
    x, wg, wu = s["x"].double(), s["wg"].double(), s["wu"].double()
    g, u = torch.mm(x, wg.t().contiguous()), torch.mm(x, wu.t().contiguous())
    q = 1 / (1 + torch.exp(-g))
    r = {"y": g * q * u}
    if c["kind"] == "train":
        dy = s["dy"].double()
        dg, du = dy * u * (q + g * q * (1 - q)), dy * g * q
        r["dx"] = torch.mm(dg, wg) + torch.mm(du, wu)
        r["dwg"], r["dwu"] = torch.mm(dg.t().contiguous(), x), torch.mm(du.t().contiguous(), x)
    return r


def exact(case, seed):
    global own
    was, own = own, False                        # inputs only
    try:
        s = prepare(case, seed)
    finally:
        own = was
    f = {"conv": _exact_conv, "norm": _exact_norm, "logprobs": _exact_logprobs, "ff": _exact_ff}
    return f[case["op"]](case, s)
