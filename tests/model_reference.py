"""The operators of state space language models in 64 bits, plainly: rows and tokens one after the other, gradients by
autograd of the definition.  Tensors in and out, on the CPU; inputs of any float type."""
import torch


def wide(t):
    return None if t is None else t.detach().double().cpu() if t.is_floating_point() else t.detach().cpu()


def silu(v):
    return v / (1 + torch.exp(-v))


def places(slots, batch, pool):
    """The row of the pools for each row of the batch, -1 for padding."""
    if slots is None:
        return list(range(batch))
    slots, seen = [int(s) for s in slots], set()
    out = []
    for s in slots:
        out.append(s if 0 <= s < pool and s not in seen else -1)
        seen.add(s)
    return out


def conv_prompt(x, state, weight, bias=None, *, activation=True, lengths=None, slots=None):
    """(y, new state); x (B,D,L)."""
    x, state, weight, bias = wide(x), wide(state).clone(), wide(weight), wide(bias)
    B, D, L = x.shape
    K = weight.shape[1]
    y = torch.zeros_like(x)
    for b, s in enumerate(places(slots, B, state.shape[0])):
        if s < 0:
            continue
        n = L if lengths is None else min(max(int(lengths[b]), 0), L)
        tokens = torch.cat([state[s], x[b, :, :n]], 1)
        for t in range(n):
            pre = (tokens[:, t:t + K] * weight).sum(1) + (0 if bias is None else bias)
            y[b, :, t] = silu(pre) if activation else pre
        state[s] = tokens[:, n:]
    return y, state


def step(x, delta, A, Bm, Cm, state, Dskip=None, z=None, delta_bias=None, *, delta_softplus=True, conv_state=None,
         conv_weight=None, conv_bias=None, activation=True, slots=None):
    """(y, new state, new conv_state)."""
    x, delta, A, Bm, Cm, state = (wide(t).clone() for t in (x, delta, A, Bm, Cm, state))
    Dskip, z, delta_bias = wide(Dskip), wide(z), wide(delta_bias)
    if conv_weight is not None:
        rows, conv_state = conv_prompt(x[..., None], conv_state, conv_weight, conv_bias, activation=activation, slots=slots)
        x = rows[..., 0]
    if delta_bias is not None:
        delta = delta + delta_bias
    if delta_softplus:
        delta = torch.logaddexp(delta, torch.zeros_like(delta))
    y = torch.zeros_like(x)
    for b, s in enumerate(places(slots, x.shape[0], state.shape[0])):
        if s < 0:
            continue
        state[s] = torch.exp(delta[b][:, None] * A) * state[s] + (delta[b] * x[b])[:, None] * Bm[b]
        y[b] = state[s] @ Cm[b] + (0 if Dskip is None else Dskip * x[b])
        if z is not None:
            y[b] = y[b] * silu(z[b])
    return y, state, conv_state


def block_norm(x, weight=None, *, gate=None, branch_weight=None, residual=None, residual_scale=1.0, norm_branch=False,
               norm_stream=True, eps=1e-5, frozen=False):
    """y, or (y, sum); differentiable, of tensors in 64 bits.  frozen: as if the deviations were constants (the gradients are
    then the first of the two terms whose difference they are)."""
    deviation = lambda v: torch.sqrt(((v.detach() if frozen else v) ** 2).mean(-1, keepdim=True) + eps)  # noqa: E731
    v = x if gate is None else x * silu(gate)
    if norm_branch:
        v = v / deviation(v)
    s = v if branch_weight is None else v * branch_weight
    if residual is not None:
        s = s + residual_scale * residual
    y = s
    if norm_stream:
        y = s / deviation(s)
        if weight is not None:
            y = y * weight
    return y if residual is None else (y, s)


def gradients(function, inputs, downs):
    """Values of function(**inputs) and the gradients of sum(value * down) by the inputs that are floats, a dict."""
    leaves = {k: wide(v).requires_grad_(True) if torch.is_tensor(v) and v.is_floating_point() else v for k, v in inputs.items()}
    out = function(**leaves)
    out = out if isinstance(out, tuple) else (out,)
    named = {k: v for k, v in leaves.items() if torch.is_tensor(v) and v.requires_grad}
    pairs = [(o, wide(d)) for o, d in zip(out, downs) if d is not None]
    grads = torch.autograd.grad([o for o, _ in pairs], list(named.values()), [d for _, d in pairs], allow_unused=True)
    return tuple(o.detach() for o in out), {k: torch.zeros_like(named[k]) if g is None else g for k, g in zip(named, grads)}


def loss(x, weight, targets, *, scale=1.0):
    """(loss, lse) of the tokens; differentiable, of tensors in 64 bits."""
    live = (targets >= 0) & (targets < weight.shape[0])
    rows = torch.nonzero(live)[:, 0]
    logits = scale * x[rows] @ weight.T
    lse = torch.logsumexp(logits, 1)
    own = logits.gather(1, targets[rows].long()[:, None])[:, 0] if len(rows) else lse
    zero = torch.zeros(len(targets), dtype=x.dtype)
    return zero.index_put((rows,), lse - own), zero.index_put((rows,), lse)
