"""A small state-space language model out of the library's operators: token embedding, the norms around a block,
convolution and selective scan, the cross entropy that keeps no logits; prompts and single tokens in a pool of states.

    python examples/state_space_lm.py [--steps N] [--dtype bf16]

Trains on synthetic documents of different lengths (each repeats a few tokens with a period of its own, so that
the next token is known once the period has been seen), then serves prompts of different lengths: each takes a slot of the
pool, a captured step continues all of them, and the same tokens are asked for with the whole sequence given.
"""
import argparse
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2506_15976_amd as lb  # noqa: E402
from paper_2506_15976_amd.autograd import (block_norm, causal_conv1d_silu, lb_selective_scan,  # noqa: E402
                                           linear_cross_entropy, token_embedding)

CONV = 4


class StateSpaceLM:
    """Embedding, `layers` blocks (norm of the residual stream, input projection to x and its gate, convolution, scan, gated norm,
    output projection), a norm, and the loss through the embedding table.  Parameters are fp32; the rows between
    the operators have the type `dtype`, the residual stream is fp32."""

    def __init__(self, vocab, dim, layers, *, states=16, dtype=torch.float32, device="cuda", seed=0):
        g = torch.Generator().manual_seed(seed)
        inner, rank = 2 * dim, max(dim // 16, 1)
        self.dtype, self.dim, self.inner, self.layers, self.states, self.rank = dtype, dim, inner, layers, states, rank

        def random(*shape):
            return torch.randn(*shape, generator=g) / shape[-1] ** 0.5
        p = {"table": random(vocab, dim), "norm": torch.ones(dim)}
        for k in range(layers):
            p[f"norm{k}"], p[f"gated{k}"] = torch.ones(dim), torch.ones(inner)
            p[f"in{k}"], p[f"out{k}"] = random(2 * inner, dim), random(dim, inner)
            p[f"conv{k}"], p[f"conv_bias{k}"] = random(inner, CONV), torch.zeros(inner)
            p[f"x{k}"], p[f"dt{k}"] = random(rank + 2 * states, inner), random(inner, rank)
            # time steps of 0.001 to 0.1
            dt = torch.exp(torch.empty(inner).uniform_(-6.9, -2.3, generator=g))
            p[f"dt_bias{k}"] = torch.log(torch.expm1(dt))
            p[f"A{k}"] = torch.log(torch.arange(1, states + 1.0)).repeat(inner, 1)
            p[f"skip{k}"] = torch.ones(inner)
        self.parameters = {k: v.to(device).requires_grad_(True) for k, v in p.items()}

    def _linear(self, x, name):
        return F.linear(x, self.parameters[name].to(self.dtype))

    def _scan_inputs(self, u, k):
        """delta, B and C from the rows u (.., inner) behind the convolution."""
        low, Bm, Cm = self._linear(u, f"x{k}").split([self.rank, self.states, self.states], -1)
        return self._linear(low, f"dt{k}"), Bm, Cm

    def hidden(self, ids):
        """Rows (B, L, dim) that the table turns into logits."""
        p = self.parameters
        x = token_embedding(ids, p["table"].to(self.dtype))
        stream = torch.zeros(x.shape, device=x.device)
        for k in range(self.layers):
            h, stream = block_norm(x, p[f"norm{k}"], residual=stream)
            x, z = self._linear(h, f"in{k}").split(self.inner, -1)
            u = causal_conv1d_silu(x.transpose(1, 2).contiguous(), p[f"conv{k}"], p[f"conv_bias{k}"])
            delta, Bm, Cm = (t.transpose(1, 2).contiguous() for t in self._scan_inputs(u.transpose(1, 2), k))
            y = lb_selective_scan(u, delta, -torch.exp(p[f"A{k}"]), Bm, Cm, p[f"skip{k}"], None, p[f"dt_bias{k}"], window=1)
            y = block_norm(y.transpose(1, 2).contiguous(), p[f"gated{k}"], gate=z.contiguous())
            x = self._linear(y, f"out{k}")
        return block_norm(x, p["norm"], residual=stream)[0]

    def loss(self, ids, targets, *, square=1e-4):
        """Mean cross entropy of the targets that are tokens (the others, -1 by custom, are left out), and
        `square` times the mean of the squared log of the softmax's sum, which keeps the logits near zero."""
        loss, lse = linear_cross_entropy(self.hidden(ids), self.parameters["table"].to(self.dtype), targets)
        return (loss.sum() + square * (lse * lse).sum()) / (targets >= 0).sum()

    def logits(self, h):
        return self._linear(h, "table").float()

    def pool(self, slots):
        """States of `slots` sequences: for each block what the scan and the convolution keep."""
        device = self.parameters["table"].device
        return [(torch.zeros(slots, self.inner, self.states, device=device),
                 torch.zeros(slots, self.inner, CONV - 1, device=device, dtype=self.dtype)) for _ in range(self.layers)]

    @torch.no_grad()
    def prompt(self, ids, lengths, pool, slots):
        """Logits behind the last token of the prompts ids (B, L), which are as long as lengths (B) int32 says; their states go to
        the rows slots (B) int32 of the pool."""
        p, at = self.parameters, slots.long()
        x = lb.lbscan_embed_fwd(ids.contiguous(), p["table"].to(self.dtype))
        stream = torch.zeros(x.shape, device=x.device)
        behind = torch.arange(ids.shape[1], device=x.device) >= lengths[:, None]
        for k in range(self.layers):
            h, stream = lb.lbscan_block_norm_fwd(x, p[f"norm{k}"], residual=stream)
            x, z = self._linear(h, f"in{k}").split(self.inner, -1)
            scan_state, conv_state = pool[k]
            conv_state[at] = 0
            u = lb.lbscan_conv1d_prompt(x.transpose(1, 2).contiguous(), conv_state, p[f"conv{k}"], p[f"conv_bias{k}"],
                                        lengths=lengths, slots=slots)
            delta, Bm, Cm = (t.transpose(1, 2).contiguous() for t in self._scan_inputs(u.transpose(1, 2), k))
            # behind a prompt time stands still: softplus of this is 0, and the state stays
            delta.masked_fill_(behind[:, None], -1e4)
            y, scan_state[at] = lb.lbscan_fwd(u, delta, -torch.exp(p[f"A{k}"]), Bm, Cm, p[f"skip{k}"], None, p[f"dt_bias{k}"],
                                              window=1, return_state=True)
            y = lb.lbscan_block_norm_fwd(y.transpose(1, 2).contiguous(), p[f"gated{k}"], gate=z.contiguous())
            x = self._linear(y, f"out{k}")
        h, _ = lb.lbscan_block_norm_fwd(x, p["norm"], residual=stream)
        last = (lengths.long() - 1)[:, None, None].expand(-1, 1, self.dim)
        return self.logits(h.gather(1, last)[:, 0])

    @torch.no_grad()
    def step(self, ids, pool, slots):
        """Logits behind one more token of each sequence, ids (B); the rows slots (B) int32 of the pool are updated in
        place, rows of ids whose slot is none (-1) are padding."""
        p = self.parameters
        x = lb.lbscan_embed_fwd(ids.contiguous(), p["table"].to(self.dtype))
        stream = torch.zeros(x.shape, device=x.device)
        for k in range(self.layers):
            h, stream = lb.lbscan_block_norm_fwd(x, p[f"norm{k}"], residual=stream)
            x, z = self._linear(h, f"in{k}").split(self.inner, -1)
            scan_state, conv_state = pool[k]
            # the scan's inputs are products of what the convolution returns, so it goes in front by itself
            u = lb.lbscan_conv1d_step(x, conv_state, p[f"conv{k}"], p[f"conv_bias{k}"], slots=slots)
            delta, Bm, Cm = self._scan_inputs(u, k)
            y = lb.lbscan_step(u, delta, -torch.exp(p[f"A{k}"]), Bm, Cm, scan_state, p[f"skip{k}"], None, p[f"dt_bias{k}"],
                               slots=slots)
            y = lb.lbscan_block_norm_fwd(y, p[f"gated{k}"], gate=z.contiguous())
            x = self._linear(y, f"out{k}")
        h, _ = lb.lbscan_block_norm_fwd(x, p["norm"], residual=stream)
        return self.logits(h)


def documents(rows, length, vocab, generator):
    """(ids, targets) of rows of 1/2 to 1 times `length` tokens, padded: each repeats 2 to 6 random tokens."""
    ids = torch.zeros(rows, length, dtype=torch.int64)
    targets = torch.full((rows, length), -1)
    for r in range(rows):
        period, n = (int(torch.randint(lo, hi, (1,), generator=generator)) for lo, hi in ((2, 7), (length // 2, length + 1)))
        word = torch.randint(0, vocab, (period,), generator=generator).repeat(n // period + 2)
        ids[r, :n], targets[r, :n] = word[:n], word[1:n + 1]
    return ids, targets


def train(model, steps, *, vocab, rows=16, length=160, lr=3e-3, seed=1, report=None):
    """Adam on fresh documents every step; the losses."""
    g = torch.Generator().manual_seed(seed)
    adam = torch.optim.Adam(model.parameters.values(), lr=lr)
    losses = []
    for k in range(steps):
        ids, targets = (t.cuda() for t in documents(rows, length, vocab, g))
        loss = model.loss(ids, targets)
        adam.zero_grad()
        loss.backward()
        adam.step()
        losses.append(float(loss.detach()))
        if report and k % report == 0:
            print(f"step {k}: loss {losses[-1]:.3f}", flush=True)
    return losses


class Server:
    """A pool of `slots` sequences, and a captured step of `batch` rows that continues any of them."""

    def __init__(self, model, slots, batch):
        self.model, self.pool = model, model.pool(slots)
        device = self.pool[0][0].device
        self.ids = torch.zeros(batch, dtype=torch.int64, device=device)
        self.slots = torch.full((batch,), -1, dtype=torch.int32, device=device)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            model.step(self.ids, self.pool, self.slots)           # (padding alone: no state is touched)
        torch.cuda.current_stream().wait_stream(side)
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self.logits = model.step(self.ids, self.pool, self.slots)

    def prompt(self, ids, lengths, slots):
        return self.model.prompt(ids, lengths, self.pool, slots)

    def step(self, ids, slots):
        """One more token, ids (n), of the sequences in slots (n) int32, n up to the captured batch."""
        n = ids.shape[0]
        self.ids[:n], self.slots[:n] = ids, slots
        self.slots[n:] = -1
        self.graph.replay()
        return self.logits[:n].clone()

    def generate(self, ids, lengths, slots, tokens):
        """Continues prompts greedily, (B, tokens)."""
        out = [self.prompt(ids, lengths, slots).argmax(-1)]
        for _ in range(tokens - 1):
            out.append(self.step(out[-1], slots).argmax(-1))
        return torch.stack(out, 1)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--dtype", choices=("fp32", "bf16"), default="fp32")
    a = ap.parse_args()
    vocab, tokens = 64, 12
    model = StateSpaceLM(vocab, 128, 2, dtype=torch.bfloat16 if a.dtype == "bf16" else torch.float32)
    losses = train(model, a.steps, vocab=vocab, report=20)
    server = Server(model, slots=16, batch=10)
    g = torch.Generator().manual_seed(5)
    lengths = torch.randint(20, 41, (8,), generator=g, dtype=torch.int32)
    prompts = torch.stack([torch.randint(0, vocab, (4,), generator=g).repeat(10) for _ in range(8)]).cuda()
    slots = torch.randperm(16, generator=g)[:8].int().cuda()
    said = server.generate(prompts, lengths.cuda(), slots, tokens)
    right = agree = 0.0
    for r, n in enumerate(lengths.tolist()):
        whole = torch.cat([prompts[r, :n], said[r]])[None]
        with torch.no_grad():
            again = model.logits(model.hidden(whole)).argmax(-1)[0, n - 1:-1]
        right += float((said[r] == prompts[r, n % 4:n % 4 + tokens]).float().mean()) / 8
        agree += float((said[r] == again).float().mean()) / 8
    print(f"loss {losses[0]:.3f} -> {losses[-1]:.3f}; continued tokens that repeat the prompt: {right:.0%}; "
          f"token by token and at once agree: {agree:.0%}")


if __name__ == "__main__":
    main()
