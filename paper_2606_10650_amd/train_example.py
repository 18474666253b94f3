"""A small model of the layer's base form, trained and then run token by token.

    python -m paper_2606_10650_amd.train_example [--steps N] [--states f32|fp8] [--full]

Each layer is a root-mean-square norm of the residual stream, the gated single-state
recurrence over its projections, and an output projection; the model is trained with AdamW
on associative recall: a sequence of (key, value) tokens, then keys whose values are to be
named.  The norm, the recurrence and the optimizer are the library's; projections and the
loss are torch's.  Afterwards the model answers one sequence token by token, carrying each
layer's state, the norms' outputs in 8 bits, and its answers are compared with those over
the whole sequence.

With --full a layer is a whole block: a short convolution in front of the recurrence, a gated norm
of its heads, a norm behind each branch with the residual sum and the norm of the next, a gated
feed-forward branch, and the loss of the answers' log probabilities; all of them the library's.
"""
from __future__ import annotations

import argparse

import torch

from . import block, train


class Model:
    """Parameters in bfloat16, with float32 masters in the optimizer."""

    def __init__(self, vocab: int, layers: int = 2, heads: int = 2, d: int = 64, width: int = 128,
                 states: str = "f32", seed: int = 0, full: bool = False):
        self.layers, self.heads, self.d, self.width, self.full = layers, heads, d, width, full
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.opt, self.params, self.masters = train.AdamW(states), {}, {}

        def add(name, *shape, std=0.0, fill=0.0, decay=0.0):
            master = fill + std * torch.randn(shape, generator=gen, device="cuda")
            p = master.to(torch.bfloat16).requires_grad_()
            p.grad = torch.zeros_like(p)
            self.params[name], self.masters[name] = p, master
            self.opt.add(p, p.grad, master=master, weight_decay=decay)

        add("embed", vocab, width, std=0.5)
        for i in range(layers):
            add(f"{i}.norm", width, fill=1.0)
            add(f"{i}.qkv", 3 * heads * d, width, std=width ** -0.5, decay=0.01)
            if not full:
                add(f"{i}.mix", 2, width, std=0.3)      # of a token with the one before it
            add(f"{i}.gate", heads, width, std=0.02)
            add(f"{i}.out", width, heads * d, std=0.5 * (heads * d) ** -0.5, decay=0.01)
        add("norm", width, fill=1.0)
        if full:
            inner = heads * d
            for i in range(layers):
                add(f"{i}.conv", 3 * inner, 4, std=0.4)
                add(f"{i}.z", inner, width, std=width ** -0.5, decay=0.01)
                add(f"{i}.heads", d, fill=1.0)
                add(f"{i}.post", width, fill=1.0)
                add(f"{i}.ff_norm", width, fill=1.0)
                for name in ("ff_gate", "ff_up"):
                    add(f"{i}.{name}", 2 * width, width, std=width ** -0.5, decay=0.01)
                add(f"{i}.ff_down", width, 2 * width, std=0.5 * (2 * width) ** -0.5, decay=0.01)
                add(f"{i}.ff_post", width, fill=1.0)

    def _unit(self, x, y, i):
        """q, k [B, H, T, d] of unit length and v of a convolution's outputs, and log gates [B, H, T] <= 0 of the
        inputs y."""
        q, k, v = (t.transpose(1, 2) for t in x.unflatten(-1, (3, self.heads, self.d)).unbind(2))
        unit = lambda t: torch.nn.functional.normalize(t.float(), dim=-1).to(t.dtype)  # noqa: E731
        g = torch.nn.functional.logsigmoid((y @ self.params[f"{i}.gate"].t()).float() + 5.0)
        return unit(q), unit(k), v, g.transpose(1, 2)

    def _next(self, i):
        return self.params[f"{i + 1}.norm" if i + 1 < self.layers else "norm"]

    def _whole_blocks(self, tokens):
        """Logits of whole sequences by whole blocks."""
        p, s = self.params, 0.5 ** 0.5
        h = p["embed"][tokens]
        y, _ = train.RMSNorm.apply(h, None, p["0.norm"])
        for i in range(self.layers):
            x, _ = block.ShortConv.apply(y @ p[f"{i}.qkv"].t(), p[f"{i}.conv"])
            o, _ = train.Recurrence.apply(*self._unit(x, y, i), None, self.d ** 0.5)
            z = (y @ p[f"{i}.z"].t()).unflatten(-1, (self.heads, self.d))
            o, _ = block.GatedNorm.apply(o.transpose(1, 2), p[f"{i}.heads"], z)
            h, y = block.GatedNorm.apply(o.flatten(2) @ p[f"{i}.out"].t(), p[f"{i}.post"], None, h, s, p[f"{i}.ff_norm"])
            u = block.GatedFF.apply(y, p[f"{i}.ff_gate"], p[f"{i}.ff_up"])
            h, y = block.GatedNorm.apply(u @ p[f"{i}.ff_down"].t(), p[f"{i}.ff_post"], None, h, s, self._next(i))
        return (y @ p["embed"].t()).float()

    def _step_blocks(self, token, carried):
        """`step` by whole blocks; carried: per layer the recurrence's state and the convolution's."""
        p, s, B = self.params, 0.5 ** 0.5, token.shape[0]
        h = p["embed"][token]
        y = train.rms_norm(h, p["0.norm"])[0]
        for i in range(self.layers):
            if i not in carried:
                carried[i] = (torch.zeros((B, self.heads, self.d, self.d), device="cuda"),
                              torch.zeros((B, 3, 3 * self.heads * self.d), dtype=h.dtype, device="cuda"))
            state, inputs = carried[i]
            x, _ = block.short_conv((y @ p[f"{i}.qkv"].t())[:, None], p[f"{i}.conv"], state=inputs, state_out=inputs)
            o, _ = train.recurrence(*self._unit(x, y[:, None], i), scale=self.d ** 0.5, state=state, state_out=state)
            z = (y @ p[f"{i}.z"].t()).unflatten(-1, (self.heads, self.d))
            o = block.gated_norm(o[:, :, 0], p[f"{i}.heads"], z)[0]
            h, y, _, _ = block.gated_norm(o.flatten(1) @ p[f"{i}.out"].t(), p[f"{i}.post"], None, h, scale=s,
                                          next_weight=p[f"{i}.ff_norm"])
            u, _ = block.gated_ff(y, p[f"{i}.ff_gate"], p[f"{i}.ff_up"])
            h, y, _, _ = block.gated_norm(u @ p[f"{i}.ff_down"].t(), p[f"{i}.ff_post"], None, h, scale=s,
                                          next_weight=self._next(i))
        return (y @ p["embed"].t()).float()

    def loss(self, logits, answers):
        """Mean cross entropy of logits [B, T, vocab] with answers [B, T]."""
        if self.full:
            return -block.TokenLogprobs.apply(logits, answers)[0].mean()
        return torch.nn.functional.cross_entropy(logits.flatten(0, 1), answers.flatten())

    def _project(self, i, y, before):
        """q, k [B, H, T, d] of unit length, v, and log gates [B, H, T] <= 0 of a layer's
        normed inputs [B, T, width] and those one token before."""
        p = self.params
        mixed = y * (1 + p[f"{i}.mix"][0]) + before * p[f"{i}.mix"][1]
        x = (mixed @ p[f"{i}.qkv"].t()).unflatten(-1, (3, self.heads, self.d))
        q, k, v = (t.transpose(1, 2) for t in x.unbind(2))
        unit = lambda t: torch.nn.functional.normalize(t.float(), dim=-1).to(t.dtype)  # noqa: E731
        g = torch.nn.functional.logsigmoid((y @ p[f"{i}.gate"].t()).float() + 5.0)
        return unit(q), unit(k), v, g.transpose(1, 2)

    def __call__(self, tokens):
        """Logits [B, T, vocab] of whole sequences."""
        if self.full:
            return self._whole_blocks(tokens)
        p = self.params
        h = p["embed"][tokens]
        branch = torch.zeros_like(h)
        for i in range(self.layers):
            y, h = train.RMSNorm.apply(branch, h, p[f"{i}.norm"])
            before = torch.nn.functional.pad(y, (0, 0, 1, 0))[:, :-1]
            o, _ = train.Recurrence.apply(*self._project(i, y, before), None, self.d ** 0.5)
            branch = o.transpose(1, 2).flatten(2) @ p[f"{i}.out"].t()
        y, _ = train.RMSNorm.apply(branch, h, p["norm"])
        return (y @ p["embed"].t()).float()

    @torch.no_grad()
    def step(self, token, carried):
        """Logits [B, vocab] of one more token per sequence; carried: what the tokens so far
        left, per layer the state and the last normed input ({} at the start), updated."""
        if self.full:
            return self._step_blocks(token, carried)
        p, B = self.params, token.shape[0]
        h = p["embed"][token]
        branch = torch.zeros_like(h)

        def norm(name, branch, h):
            y, h, scale = train.rms_norm_fp8(branch, p[name], h)
            return (y.float() * scale[:, None]).to(h.dtype), h

        for i in range(self.layers):
            y, h = norm(f"{i}.norm", branch, h)
            if i not in carried:
                carried[i] = [torch.zeros((B, self.heads, self.d, self.d), device="cuda"), torch.zeros_like(y)]
            state, before = carried[i]
            o, _ = train.recurrence(*self._project(i, y[:, None], before[:, None]), scale=self.d ** 0.5,
                                    state=state, state_out=state)
            carried[i][1] = y
            branch = o.transpose(1, 2).flatten(1) @ p[f"{i}.out"].t()
        y, _ = norm("norm", branch, h)
        return (y @ p["embed"].t()).float()

    def update(self, t, lr):
        """AdamW's t-th step, with the gradients clipped to a norm of one on the device."""
        norm = torch.stack([p.grad.float().norm() for p in self.params.values()]).norm()
        self.opt.step(t, lr=lr, betas=(0.9, 0.98), seed=t if self.opt.states == "fp8" else 0,
                      grad_scale=(1.0 / norm.clamp(min=1.0)).reshape(1))
        for p in self.params.values():
            p.grad = None


def recall(B, pairs, queries, keys, values, gen):
    """Tokens [B, T], the answers [B, queries] and where they are to be given: pairs of a
    key and a value, then keys again."""
    k = torch.rand((B, keys), generator=gen, device="cuda").argsort(1)[:, :pairs]
    v = torch.randint(0, values, (B, pairs), generator=gen, device="cuda")
    which = torch.randint(0, pairs, (B, queries), generator=gen, device="cuda")
    told = torch.stack([k, keys + v], 2).flatten(1)
    return torch.cat([told, k.gather(1, which)], 1), keys + v.gather(1, which), slice(2 * pairs, None)


def main(steps: int = 300, states: str = "f32", say=print, full: bool = False):
    gen = torch.Generator(device="cuda").manual_seed(1)
    keys, values = 32, 32
    model = Model(keys + values, states=states, full=full)
    losses = []
    for t in range(1, steps + 1):
        tokens, answers, at = recall(64, 16, 24, keys, values, gen)
        logits = model(tokens)[:, at]
        loss = model.loss(logits, answers)
        loss.backward()
        model.update(t, lr=3e-3 * min(1.0, t / 30))
        losses.append(loss.detach())
        if t % 50 == 0 or t == 1:
            right = (logits.argmax(-1) == answers).float().mean()
            say(f"step {t}: loss {loss.item():.3f}, {100 * right.item():.0f}% of the answers right")
    # the same model, one token at a time
    tokens, answers, at = recall(8, 16, 24, keys, values, gen)
    with torch.no_grad():
        whole = model(tokens)
    carried = {}
    single = torch.stack([model.step(tokens[:, i], carried) for i in range(tokens.shape[1])], 1)
    off = ((single - whole).norm() / whole.norm()).item()
    same = (single[:, at].argmax(-1) == whole[:, at].argmax(-1)).float().mean().item()
    say(f"token by token: logits {off:.3f} of their norm off{'' if full else ' (norms in 8 bits)'}, "
        f"{100 * same:.0f}% of the answers the same")
    if full:
        # what the model finds likely in place of the last answers
        _, _, entropy, ids, tops = block.token_logprobs(single[:, -1].contiguous(), answers[:, -1].contiguous(), top=3,
                                                        entropy=True)
        for b in range(2):
            say(f"answer {answers[b, -1].item()}: entropy {entropy[b].item():.2f}, " +
                ", ".join(f"{i} ({p:.2f})" for i, p in zip(ids[b].tolist(), tops[b].exp().tolist())))
    return torch.stack(losses).tolist(), off, same


if __name__ == "__main__":
    a = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    a.add_argument("--steps", type=int, default=300)
    a.add_argument("--states", choices=("f32", "fp8"), default="f32")
    a.add_argument("--full", action="store_true")
    main(**vars(a.parse_args()))
