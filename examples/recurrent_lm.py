"""A small recurrent language model out of the library's operators: token embedding, layer norm over a
32-bit residual stream, gated linear recurrence.

    python examples/recurrent_lm.py [--steps N] [--dtype bf16]

Trains on synthetic documents packed into rows (each document repeats a few tokens with a period of its own, so
that the next token is known once the period has been seen), then continues a prompt token by token with
the recurrence's single-token form and checks that it says what the whole prompt says.
"""
import argparse
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2506_15976_amd as lb  # noqa: E402
from paper_2506_15976_amd.autograd import gated_linear_recurrence, layer_norm, token_embedding  # noqa: E402


class RecurrentLM:
    """Embedding, `layers` blocks of norm, projections, recurrence and output projection, a norm, and the logits
    through the embedding table.  Parameters are fp32; the rows between the operators have the type `dtype`."""

    def __init__(self, vocab, dim, layers, *, dtype=torch.float32, device="cuda", seed=0):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.dim, self.layers = dtype, dim, layers
        p = {"table": 0.02 * torch.randn(vocab, dim, generator=g)}
        for k in range(layers + 1):
            p[f"norm{k}.weight"], p[f"norm{k}.bias"] = torch.ones(dim), torch.zeros(dim)
        for k in range(layers):
            for name in ("x", "a", "i", "out"):
                p[f"{name}{k}"] = torch.randn(dim, dim, generator=g) / dim ** 0.5
            # open gates keep 0.9 .. 0.999 of the state: -8 softplus(decay) is the log of that
            keep = torch.empty(dim).uniform_(0.9, 0.999, generator=g)
            p[f"decay{k}"] = torch.log(torch.expm1(-torch.log(keep) / 8))
        self.parameters = {k: v.to(device).requires_grad_(True) for k, v in p.items()}

    def _embed(self, ids):
        return token_embedding(ids, self.parameters["table"].to(self.dtype), scale=self.dim ** 0.5)

    def _norm(self, k, x, stream):
        """The norm in front of block k: of the stream plus what the block before added, and that sum."""
        p = self.parameters
        return layer_norm(x, p[f"norm{k}.weight"], p[f"norm{k}.bias"], residual=stream)

    def _logits(self, h):
        return F.linear(h, self.parameters["table"].to(self.dtype)).float()

    def forward(self, ids, starts=None, states=None):
        """Logits of ids (B, L).  starts (B, L): where the packed documents begin.  states: a list that receives
        each block's leaving state (B, dim)."""
        p = self.parameters
        x = self._embed(ids)
        stream = torch.zeros(x.shape, device=x.device)
        for k in range(self.layers):
            h, stream = self._norm(k, x, stream)
            # the recurrence runs along the last axis
            u, a, i = (F.linear(h, p[f"{n}{k}"].to(self.dtype)).transpose(1, 2).contiguous() for n in ("x", "a", "i"))
            y = gated_linear_recurrence(u, a, i, p[f"decay{k}"], starts=starts, return_state=states is not None)
            if states is not None:
                y, hT = y
                states.append(hT)
            x = F.linear(y.transpose(1, 2).contiguous(), p[f"out{k}"].to(self.dtype))
        h, _ = self._norm(self.layers, x, stream)
        return self._logits(h)

    @torch.no_grad()
    def step(self, ids, states):
        """Logits of one token of each sequence, ids (B); the states (B, dim) are updated in place."""
        p = self.parameters
        x = lb.lbscan_embed_fwd(ids.contiguous(), p["table"].to(self.dtype), scale=self.dim ** 0.5)
        stream = torch.zeros(x.shape, device=x.device)
        for k in range(self.layers):
            h, stream = lb.lbscan_norm_fwd(x, p[f"norm{k}.weight"], p[f"norm{k}.bias"], residual=stream)
            u, a, i = (F.linear(h, p[f"{n}{k}"].to(self.dtype)) for n in ("x", "a", "i"))
            y = lb.lbscan_gated_step(u, a, i, p[f"decay{k}"], states[k])
            x = F.linear(y, p[f"out{k}"].to(self.dtype))
        h, _ = lb.lbscan_norm_fwd(x, p[f"norm{self.layers}.weight"], p[f"norm{self.layers}.bias"], residual=stream)
        return self._logits(h)


def documents(rows, length, vocab, generator):
    """Packed rows of documents, (ids, starts): a document repeats 2 to 6 random tokens for 20 to 60 tokens."""
    ids, starts = torch.empty(rows, length, dtype=torch.int64), torch.zeros(rows, length, dtype=torch.bool)
    for r in range(rows):
        t = 0
        while t < length:
            period = int(torch.randint(2, 7, (1,), generator=generator))
            n = min(int(torch.randint(20, 61, (1,), generator=generator)), length - t)
            word = torch.randint(0, vocab, (period,), generator=generator)
            ids[r, t:t + n] = word.repeat(n // period + 1)[:n]
            starts[r, t] = True
            t += n
    return ids, starts


def loss_of(model, ids, starts):
    """Mean cross entropy of the next token, where it belongs to the same document."""
    logits = model.forward(ids, starts)
    same = ~starts[:, 1:]
    return F.cross_entropy(logits[:, :-1][same], ids[:, 1:][same])


def train(model, steps, *, vocab, rows=16, length=197, lr=3e-3, seed=1, report=None):
    """Adam on fresh documents every step; the losses."""
    g = torch.Generator().manual_seed(seed)
    adam = torch.optim.Adam(model.parameters.values(), lr=lr)
    losses = []
    for k in range(steps):
        ids, starts = (t.cuda() for t in documents(rows, length, vocab, g))
        loss = loss_of(model, ids, starts)
        adam.zero_grad()
        loss.backward()
        adam.step()
        losses.append(float(loss.detach()))
        if report and k % report == 0:
            print(f"step {k}: loss {losses[-1]:.3f}", flush=True)
    return losses


@torch.no_grad()
def generate(model, ids, tokens):
    """Continues ids (B, L) greedily: the whole prompt at once, then a token at a time.  (B, tokens)."""
    states = []
    last = model.forward(ids, states=states)[:, -1].argmax(-1)
    out = [last]
    for _ in range(tokens - 1):
        last = model.step(last, states).argmax(-1)
        out.append(last)
    return torch.stack(out, 1)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--dtype", choices=("fp32", "bf16"), default="fp32")
    a = ap.parse_args()
    vocab = 64
    model = RecurrentLM(vocab, 128, 2, dtype=torch.bfloat16 if a.dtype == "bf16" else torch.float32)
    losses = train(model, a.steps, vocab=vocab, report=20)
    g = torch.Generator().manual_seed(5)
    prompt = torch.stack([torch.randint(0, vocab, (4,), generator=g).repeat(8) for _ in range(8)]).cuda()
    said = generate(model, prompt, 12)
    # the same tokens with the whole sequence given each time
    again = model.forward(torch.cat([prompt, said], 1)).argmax(-1)[:, prompt.shape[1] - 1:-1]
    right = (said == prompt[:, :12]).float().mean()
    print(f"loss {losses[0]:.3f} -> {losses[-1]:.3f}; continued tokens that repeat the prompt: {float(right):.0%}; "
          f"token by token and at once agree: {float((said == again).float().mean()):.0%}")


if __name__ == "__main__":
    main()
