"""Operators of state space language models: the loss over a large vocabulary, the scan's and the convolution's forms for
serving, the norms around a block; as training and serving call them.

A case names what is called ("op"), the sizes, the storage type and the options:

    op "loss_fwd"     losses of tokens from their rows and the table of the vocabulary (scoring, evaluation)
    op "loss_train"   the same and the gradients of the rows and of the table, through autograd
    op "step"         one token of every sequence through the selective scan (with "conv": through the convolution
                      in front of it, too); states in a pool, updated in place
    op "conv_prompt"  prompts of a padded batch through the convolution: outputs, and states for the steps that follow
    op "norm_fwd"     the norms around a block with its gate and its residual stream
    op "norm_train"   the same and its gradients, through autograd

Formulas (sums, states and statistics in 32 bits or more; silu(v) = v / (1 + exp(-v))):

    loss   l_tv = scale x_t . W_v, lse_t = log sum_v exp l_tv, loss_t = lse_t - l_t,target(t); tokens whose target is no
           row of the table count nowhere (loss, lse and gradients zero)
    step   dt = softplus(delta + delta_bias), h = exp(dt A) h + dt B x, y = (sum_n C h + Dskip x) silu(z); with the
           convolution x is silu(bias + sum_k weight_k x_{t-K+1+k}) of the K tokens that end with this one.  A
           sequence's states are at its slot of the pool; rows whose slot is none (padding) give zeros
    norm   v = x silu(gate), u = v / sqrt(mean v^2 + eps) branch_weight, s = residual_scale residual + u,
           y = s / sqrt(mean s^2 + eps) weight; each norm, the gate and the residual may be absent

Sizes are those of the package's named workloads, where it has them, and generic ones.  Values: rows,
gates, gradients ~ N(0,1); logits of deviation 2; targets by Zipf's law, as text has them; time steps in 0.001 .. 0.1.
"""
import math

import torch

own = False

_EPS = 1e-5

# the package's named workloads vim_tiny, vim_small and hires_4096
_TINY = dict(batch=64, dim=384, seqlen=197)
_SMALL = dict(batch=128, dim=768, seqlen=197)
_DENSE = dict(batch=8, dim=768, seqlen=4096)


def _loss(name, op, dtype, tokens, vocab, dim, *, ids="int64", ignored=0.0, dlse=False):
    return dict(name=name, op=op, dtype=dtype, tokens=tokens, vocab=vocab, dim=dim, ids=ids, ignored=ignored, dlse=dlse)


def _step(name, dtype, batch, dim, *, dstate=16, gate=True, conv=0, pool=0, padded=0):
    return dict(name=name, op="step", dtype=dtype, batch=batch, dim=dim, dstate=dstate, gate=gate, conv=conv, pool=pool,
                padded=padded)


def _prompt(name, dtype, batch, dim, seqlen, *, conv=4, pool=0, ragged=False):
    return dict(name=name, op="conv_prompt", dtype=dtype, batch=batch, dim=dim, seqlen=seqlen, conv=conv, pool=pool,
                padded=0, ragged=ragged)


def _norm(name, op, dtype, rows, dim, *, gate, branch, stream, residual, residual_scale=1.0):
    return dict(name=name, op=op, dtype=dtype, rows=rows, dim=dim, gate=gate, branch=branch, stream=stream,
                residual=residual, residual_scale=residual_scale)


def listed():
    return [
        # scoring: the losses of one token of each of 64 sequences, where reading the table counts
        _loss("loss_score", "loss_fwd", "bf16", 64, 50000, 768),
        # fine-tuning on short texts, 32 bits, odd sizes, some of the tokens padding
        _loss("loss_train_odd", "loss_train", "fp32", _TINY["seqlen"] * 8, 32003, 385, ids="int32", ignored=0.2),
        # fine-tuning a wider model of many words on answers alone, with a penalty on lse
        _loss("loss_train_answers", "loss_train", "bf16", 4096, 131072, 2048, ignored=0.6, dlse=True),
        # pre-training: a batch of long sequences
        _loss("loss_train", "loss_train", "bf16", 16384, 50000, 768),
        # decoding for one user, where latency counts
        _step("step_one", "fp32", 1, _TINY["dim"]),
        # decoding: 64 rows, a few of them padding, states in a pool
        _step("step_decode", "bf16", 64, _DENSE["dim"], conv=4, pool=80, padded=4),
        # decoding: many sequences of a wide model, where the states count
        _step("step_wide", "bf16", 256, 4096, conv=4, pool=256),
        # prompts of several users, padded to the longest
        _prompt("conv_prompts", "bf16", **_DENSE, pool=16, ragged=True),
        # decoding: both norms, gate and stream, a row for each of 64 sequences
        _norm("norm_decode", "norm_fwd", "bf16", 64, 768, gate=True, branch=True, stream=True, residual=True),
        # training, 32 bits, narrow rows: the gated norm inside a block
        _norm("norm_train_gated", "norm_train", "fp32", _SMALL["batch"] * _SMALL["seqlen"], _TINY["dim"], gate=True,
              branch=True, stream=False, residual=False),
        # training: both norms, gate and a scaled stream, the rows of a batch of long sequences
        _norm("norm_train", "norm_train", "bf16", _DENSE["batch"] * _DENSE["seqlen"], _DENSE["dim"], gate=True, branch=True,
              stream=True, residual=True, residual_scale=0.8),
        # training: few wide rows, the norm in front of a block alone
        _norm("norm_train_wide", "norm_train", "bf16", 2048, 8192, gate=False, branch=False, stream=True, residual=True),
    ]


# What a drawn case may need at most: bytes, operations in bf16 and in fp32.
_MOST_BYTES, _MOST_FLOPS = 800e6, {"bf16": 3.7e12, "fp32": 0.45e12}


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["loss_fwd", "loss_train", "loss_train", "step", "step", "conv_prompt", "norm_fwd", "norm_train",
                     "norm_train"])
    dtype = rng.choice(["fp32", "bf16"])
    if op.startswith("loss"):
        c = _loss(None, op, dtype, _log_uniform(rng, 1, 32768), _log_uniform(rng, 256, 131072), _log_uniform(rng, 32, 4096),
                  ids=rng.choice(["int64", "int32"]), ignored=rng.choice([0.0, 0.0, 0.1, 0.5, 0.9]), dlse=rng.random() < 0.3)
        shrink = ("tokens", "vocab", "dim")
    elif op == "step":
        batch = _log_uniform(rng, 1, 1024)
        pooled = rng.random() < 0.5
        c = _step(None, dtype, batch, _log_uniform(rng, 32, 8192), dstate=rng.choice([1, 4, 7, 8, 16, 16, 16]),
                  gate=rng.random() < 0.7, conv=rng.choice([0, 2, 3, 4, 4]), pool=batch + batch // 4 if pooled else 0,
                  padded=batch // 10 if pooled else 0)
        shrink = ("dim",)
    elif op == "conv_prompt":
        batch = _log_uniform(rng, 1, 64)
        c = _prompt(None, dtype, batch, _log_uniform(rng, 32, 4096), _log_uniform(rng, 1, 32768),
                    conv=rng.choice([2, 3, 4]), pool=batch + 3 if rng.random() < 0.5 else 0, ragged=rng.random() < 0.6)
        shrink = ("dim", "seqlen")
    else:
        stream, residual = rng.random() < 0.7, rng.random() < 0.6
        c = _norm(None, op, dtype, _log_uniform(rng, 1, 65536), _log_uniform(rng, 32, 12288), gate=rng.random() < 0.5,
                  branch=not stream or rng.random() < 0.5, stream=stream, residual=residual,
                  residual_scale=rng.choice([1.0, 1.0, 0.7]) if residual else 1.0)
        shrink = ("rows", "dim")
    del c["name"]
    while work(c)["bytes"] > _MOST_BYTES or work(c)["flops"] > _MOST_FLOPS[dtype]:
        k = max(shrink, key=lambda k: c[k] if k != "dim" else c[k] * 4)
        c[k] = c[k] * 2 // 3
    return c


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _tensors(case, seed):
    """The inputs of one call on the GPU, from the seed alone."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = _type(case)

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    def uniform(n, lo, hi):
        return torch.empty(n, device="cuda").uniform_(lo, hi, generator=g)

    op, D = case["op"], case["dim"]
    if op.startswith("loss"):
        T, V = case["tokens"], case["vocab"]
        u = torch.rand(T, device="cuda", generator=g, dtype=torch.float64)
        targets = (torch.exp(u * math.log(V + 1)) - 1).long().clamp(0, V - 1)
        if case["ignored"]:
            targets = torch.where(torch.rand(T, device="cuda", generator=g) < case["ignored"], -1, targets)
        t = dict(x=normal(T, D).to(dt), weight=(normal(V, D) * (2 / math.sqrt(D))).to(dt),
                 targets=targets.to(torch.int32 if case["ids"] == "int32" else torch.int64))
        if op == "loss_train":
            # weights of a mean over tokens of different worth
            t["dloss"] = uniform(T, 0.5, 1.5) / T
            if case["dlse"]:
                t["dlse"] = uniform(T, 0, 1e-3) / T
        return t
    if op.startswith("norm"):
        n = case["rows"]
        t = dict(x=normal(n, D).to(dt))
        if case["stream"]:
            t["weight"] = 1 + 0.1 * normal(D)
        if case["gate"]:
            t["gate"] = normal(n, D).to(dt)
        if case["branch"]:
            t["branch_weight"] = 0.5 + 0.1 * normal(D)
        if case["residual"]:
            t["residual"] = 3 * normal(n, D) + 0.5
        if op == "norm_train":
            t["dout"] = normal(n, D).to(dt)
            if case["residual"]:
                t["dsum"] = normal(n, D)
        return t
    B, K = case["batch"], case["conv"]
    S = case["pool"] or B
    t = {}
    if K:
        t["conv_weight"], t["conv_bias"] = normal(D, K) / math.sqrt(K), 0.1 * normal(D)
        t["conv_state"] = normal(S, D, K - 1).to(dt)
    if case["pool"]:
        slots = torch.randperm(S, device="cuda", generator=g)[:B].to(torch.int32)
        if case["padded"]:
            slots[B - case["padded"]:] = -1
        t["slots"] = slots
    if op == "conv_prompt":
        t["x"] = normal(B, D, case["seqlen"]).to(dt)
        if case["ragged"]:
            t["lengths"] = torch.randint(case["seqlen"] // 2, case["seqlen"] + 1, (B,), device="cuda", generator=g,
                                         dtype=torch.int32)
        return t
    N = case["dstate"]
    t["x"], t["delta"] = normal(B, D).to(dt), (0.5 * normal(B, D)).to(dt)
    t["Bm"], t["Cm"] = normal(B, N).to(dt), normal(B, N).to(dt)
    t["A"] = -torch.arange(1, N + 1, device="cuda", dtype=torch.float32).expand(D, N).contiguous()
    t["Dskip"] = 1 + 0.1 * normal(D)
    t["delta_bias"] = torch.log(torch.expm1(uniform(D, 1e-3, 0.1)))
    if case["gate"]:
        t["z"] = normal(B, D).to(dt)
    t["state"] = normal(S, D, N)
    return t


_WITH_GRADIENT = ("x", "weight", "gate", "branch_weight", "residual")


def _wanted(t):
    return [t[k] for k in _WITH_GRADIENT if k in t]


def prepare(case, seed):
    t = _tensors(case, seed)
    if case["op"].endswith("train"):
        for v in _wanted(t):
            v.requires_grad_(True)
    return dict(case=case, tensors=t)


def run(state):
    return _own(state) if own else _plain(state)


# ---- the framework's operators -----------------------------------------------------------------

def _norm_options(case, t):
    return dict(gate=t.get("gate"), branch_weight=t.get("branch_weight"), residual=t.get("residual"),
                residual_scale=case["residual_scale"], norm_branch=case["branch"], norm_stream=case["stream"], eps=_EPS)


def _own(state):
    import paper_2506_15976_amd as lb
    from paper_2506_15976_amd.autograd import block_norm, linear_cross_entropy
    case, t = state["case"], state["tensors"]
    op = case["op"]
    if op == "loss_fwd":
        return lb.lbscan_loss_fwd(t["x"], t["weight"], t["targets"])
    if op == "loss_train":
        loss, lse = linear_cross_entropy(t["x"], t["weight"], t["targets"])
        if case["dlse"]:
            return loss, lse, torch.autograd.grad((loss, lse), _wanted(t), (t["dloss"], t["dlse"]))
        return loss, lse, torch.autograd.grad(loss, _wanted(t), t["dloss"])
    if op == "step":
        out = lb.lbscan_step(t["x"], t["delta"], t["A"], t["Bm"], t["Cm"], t["state"], t["Dskip"], t.get("z"),
                             t["delta_bias"], conv_state=t.get("conv_state"), conv_weight=t.get("conv_weight"),
                             conv_bias=t.get("conv_bias"), slots=t.get("slots"))
        return (out, t["state"], t["conv_state"]) if case["conv"] else (out, t["state"])
    if op == "conv_prompt":
        out = lb.lbscan_conv1d_prompt(t["x"], t["conv_state"], t["conv_weight"], t["conv_bias"], lengths=t.get("lengths"),
                                      slots=t.get("slots"))
        return out, t["conv_state"]
    if op == "norm_fwd":
        return lb.lbscan_block_norm_fwd(t["x"], t.get("weight"), **_norm_options(case, t))
    out = block_norm(t["x"], t.get("weight"), **_norm_options(case, t))
    if case["residual"]:
        return out + (torch.autograd.grad(out, _wanted(t), (t["dout"], t["dsum"])),)
    return out, torch.autograd.grad(out, _wanted(t), t["dout"])


# ---- their plain form: elementary operations in 32 bits ----------------------------------------

def _silu32(v):
    return v / (1 + torch.exp(-v))


def _softplus32(v):
    return torch.log1p(torch.exp(-v.abs())) + v.clamp(min=0)


def _loss_plain(case, t):
    dt, V = t["x"].dtype, case["vocab"]
    x, w, targets = t["x"].float(), t["weight"].float(), t["targets"].long()
    live = (targets >= 0) & (targets < V)
    at = targets.clamp(0, V - 1)[:, None]
    logits = x @ w.T
    top = logits.amax(-1, keepdim=True)
    own_logit = logits.gather(1, at)
    p = logits.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (top + torch.log(total)) * live[:, None]
    loss = (lse - own_logit)[:, 0] * live
    lse = lse[:, 0]
    if case["op"] == "loss_fwd":
        return loss, lse
    down = t["dloss"] * live
    both = down + t["dlse"] * live if case["dlse"] else down
    p.mul_(both[:, None] / total)
    p.scatter_add_(1, at, -down[:, None])
    return loss, lse, ((p @ w).to(dt), (p.T @ x).to(dt))


def _rows_of_pool(case, t, pool):
    """The rows' states, and a function that puts new ones in their place."""
    if "slots" not in t:
        return pool.clone(), pool.copy_
    if not case["padded"]:
        at = t["slots"].long()
        return pool[at], lambda new: pool.index_copy_(0, at, new.to(pool.dtype))
    # rows of padding have a place behind the pool
    S = pool.shape[0]
    at = torch.where(t["slots"] < 0, S, t["slots"]).long()
    more = torch.cat([pool, torch.zeros_like(pool[:1])])

    def put(new):
        more.index_put_((at,), new.to(pool.dtype))
        pool.copy_(more[:S])
    return more[at], put


def _step_plain(case, t):
    dt = t["x"].dtype
    x = t["x"].float()
    if case["conv"]:
        before, put = _rows_of_pool(case, t, t["conv_state"])
        window = torch.cat([before.float(), x[..., None]], -1)
        x = _silu32((window * t["conv_weight"]).sum(-1) + t["conv_bias"])
        put(window[..., 1:])
    step = _softplus32(t["delta"].float() + t["delta_bias"])
    h, put = _rows_of_pool(case, t, t["state"])
    h = torch.exp(step[..., None] * t["A"]) * h + (step * x)[..., None] * t["Bm"].float()[:, None]
    put(h)
    y = (h * t["Cm"].float()[:, None]).sum(-1) + t["Dskip"] * x
    if case["gate"]:
        y = y * _silu32(t["z"].float())
    if case["padded"]:
        y = y * (t["slots"] >= 0)[:, None]
    return (y.to(dt), t["state"], t["conv_state"]) if case["conv"] else (y.to(dt), t["state"])


def _prompt_plain(case, t):
    K, L = case["conv"], case["seqlen"]
    before, put = _rows_of_pool(case, t, t["conv_state"])
    x = torch.cat([before, t["x"]], -1)
    y = t["conv_bias"][:, None] + sum(x[..., k:k + L].float() * t["conv_weight"][:, k, None] for k in range(K))
    y = _silu32(y)
    if not case["ragged"]:
        put(x[..., L:])
        return y.to(x.dtype), t["conv_state"]
    n = t["lengths"].long()[:, None, None]
    y = y * (torch.arange(L, device=x.device) < n)
    last = (n + torch.arange(K - 1, device=x.device)).expand(-1, x.shape[1], -1)
    put(x.gather(2, last))
    return y.to(x.dtype), t["conv_state"]


def _norm_plain(case, t):
    dt, x = t["x"].dtype, t["x"].float()
    v = x
    if case["gate"]:
        z = t["gate"].float()
        open_ = 1 / (1 + torch.exp(-z))
        v = x * z * open_
    u = v
    if case["branch"]:
        rv = 1 / torch.sqrt((v * v).mean(-1, keepdim=True) + _EPS)
        hat_v = v * rv
        u = hat_v * t["branch_weight"]
    s = case["residual_scale"] * t["residual"] + u if case["residual"] else u
    y = s
    if case["stream"]:
        rs = 1 / torch.sqrt((s * s).mean(-1, keepdim=True) + _EPS)
        hat_s = s * rs
        y = hat_s * t["weight"]
    out = (y.to(dt), s) if case["residual"] else y.to(dt)
    if case["op"] == "norm_fwd":
        return out
    grads = {}
    ds = t["dout"].float()
    if case["stream"]:
        grads["weight"] = (ds * hat_s).sum(0)
        ds = ds * t["weight"]
        ds = rs * (ds - hat_s * (ds * hat_s).mean(-1, keepdim=True))
    if case["residual"]:
        ds = ds + t["dsum"]
        grads["residual"] = case["residual_scale"] * ds
    if case["branch"]:
        grads["branch_weight"] = (ds * hat_v).sum(0)
        ds = ds * t["branch_weight"]
        ds = rv * (ds - hat_v * (ds * hat_v).mean(-1, keepdim=True))
    if case["gate"]:
        grads["gate"] = (ds * x * open_ * (1 + z * (1 - open_))).to(dt)
        ds = ds * z * open_
    grads["x"] = ds.to(dt)
    grads = tuple(grads[k] for k in _WITH_GRADIENT if k in t)
    return out + (grads,) if case["residual"] else (out, grads)


def _plain(state):
    case, t = state["case"], {k: v.detach() for k, v in state["tensors"].items()}
    op = case["op"]
    if op.startswith("loss"):
        return _loss_plain(case, t)
    if op.startswith("norm"):
        return _norm_plain(case, t)
    return _step_plain(case, t) if op == "step" else _prompt_plain(case, t)


# ---- what a pass cannot do without ---------------------------------------------------------------

def work(case):
    op, e, D = case["op"], 2 if case["dtype"] == "bf16" else 4, case["dim"]
    train = op.endswith("train")
    if op.startswith("loss"):
        T, V = case["tokens"], case["vocab"]
        live = T * (1 - case["ignored"])
        size = live * D * e + V * D * e + T * (8 if case["ids"] == "int64" else 4) + 8 * T
        if train:
            size += T * D * e + V * D * e + 4 * T * (1 + case["dlse"])
        return dict(bytes=int(size), flops=int(live * V * (D * (6 if train else 2) + (8 if train else 4))))
    if op.startswith("norm"):
        n = case["rows"] * D
        size = n * e * (2 + case["gate"]) + 8 * n * case["residual"] + 4 * D * (case["branch"] + case["stream"])
        if train:
            size += n * e * (2 + case["gate"]) + 8 * n * case["residual"] + 4 * D * (case["branch"] + case["stream"])
        per = 4 + 4 * case["branch"] + 4 * case["stream"] + 6 * case["gate"]
        return dict(bytes=size, flops=n * per * (3 if train else 1))
    B, K = case["batch"], case["conv"]
    rows = B - case["padded"]
    conv = D * 4 * (K + 1) + 2 * rows * D * (K - 1) * e if K else 0
    if op == "conv_prompt":
        n = B * D * case["seqlen"]
        return dict(bytes=2 * n * e + conv + 4 * B * (bool(case["pool"]) + case["ragged"]), flops=n * (2 * K + 5))
    N = case["dstate"]
    size = rows * D * (8 * N + e * (2 + case["gate"])) + B * D * e + 2 * rows * N * e + 4 * D * (N + 2) + conv
    return dict(bytes=size + 4 * B * bool(case["pool"]), flops=rows * D * (7 * N + 12 + 2 * K))


# ---- the definition in 64 bits -------------------------------------------------------------------

def _loss_exact(case, t):
    """Token pieces, each with its whole row of logits; the gradients by the softmax's derivative."""
    T, V, D = case["tokens"], case["vocab"], case["dim"]
    x, w, targets = t["x"], t["weight"], t["targets"].long()
    loss, lse = torch.zeros(T, dtype=x.dtype, device=x.device), torch.zeros(T, dtype=x.dtype, device=x.device)
    dx, dw = torch.zeros_like(x), torch.zeros_like(w)
    rows = torch.nonzero((targets >= 0) & (targets < V))[:, 0]
    for part in rows.split(max(1, min(2048, 2 ** 28 // V))):
        xs, ys = x[part], targets[part]
        logits = torch.mm(xs, w.t())
        lse[part] = torch.logsumexp(logits, 1)
        k = torch.arange(len(part), device=x.device)
        loss[part] = lse[part] - logits[k, ys]
        if case["op"] == "loss_train":
            g = t["dloss"][part]
            weight = g + t["dlse"][part] if case["dlse"] else g
            slope = torch.softmax(logits, 1) * weight[:, None]
            slope[k, ys] -= g
            dx[part] = torch.mm(slope, w)
            dw.addmm_(slope.t(), xs)
    return (loss, lse) if case["op"] == "loss_fwd" else (loss, lse, (dx, dw))


def _conv_exact(weight, bias, tokens):
    """Tokens (rows, channels, K - 1 + n): silu of the convolution at the last n."""
    D, K = weight.shape
    return torch.nn.functional.silu(sum(tokens[:, :, k:tokens.shape[2] - K + 1 + k] * weight[:, k].view(1, D, 1)
                                        for k in range(K)) + bias.view(1, D, 1))


def _step_exact(case, t):
    rows = torch.arange(case["batch"], device=t["x"].device)
    slots = t["slots"].long() if "slots" in t else rows
    rows = rows[slots >= 0]
    slots = slots[rows]
    x = t["x"][rows]
    if case["conv"]:
        tokens = torch.cat([t["conv_state"][slots], x.unsqueeze(2)], 2)
        t["conv_state"][slots] = tokens[:, :, 1:]
        x = _conv_exact(t["conv_weight"], t["conv_bias"], tokens)[:, :, 0]
    dt = torch.logaddexp(t["delta"][rows] + t["delta_bias"], torch.zeros_like(x))
    h = t["state"][slots]
    y = t["Dskip"] * x
    for n in range(case["dstate"]):
        h[:, :, n] = h[:, :, n] * torch.exp(dt * t["A"][:, n]) + dt * x * t["Bm"][rows, n].unsqueeze(1)
        y = y + h[:, :, n] * t["Cm"][rows, n].unsqueeze(1)
    t["state"][slots] = h
    if case["gate"]:
        y = y * torch.nn.functional.silu(t["z"][rows])
    out = torch.zeros_like(t["x"])
    out[rows] = y
    return (out, t["state"], t["conv_state"]) if case["conv"] else (out, t["state"])


def _prompt_exact(case, t):
    out = torch.zeros_like(t["x"])
    for b in range(case["batch"]):
        n = int(t["lengths"][b]) if case["ragged"] else case["seqlen"]
        s = int(t["slots"][b]) if case["pool"] else b
        tokens = torch.cat([t["conv_state"][s], t["x"][b, :, :n]], 1)[None]
        out[b, :, :n] = _conv_exact(t["conv_weight"], t["conv_bias"], tokens)[0]
        t["conv_state"][s] = tokens[0, :, n:]
    return out, t["conv_state"]


def _norm_exact(case, t):
    leaves = [t[k].requires_grad_(True) for k in _WITH_GRADIENT if k in t]
    unit = lambda v: v * torch.rsqrt(v.square().mean(-1, keepdim=True) + _EPS)  # noqa: E731
    s = t["x"] * torch.nn.functional.silu(t["gate"]) if case["gate"] else t["x"]
    if case["branch"]:
        s = unit(s) * t["branch_weight"]
    if case["residual"]:
        s = s + case["residual_scale"] * t["residual"]
    y = unit(s) * t["weight"] if case["stream"] else s
    out = (y, s) if case["residual"] else (y,)
    values = tuple(v.detach() for v in out)
    if case["op"] == "norm_fwd":
        return values if case["residual"] else values[0]
    down = (t["dout"], t["dsum"]) if case["residual"] else (t["dout"],)
    return values + (torch.autograd.grad(out, leaves, down),)


def exact(case, seed):
    t = {k: v.double() if v.is_floating_point() else v for k, v in _tensors(case, seed).items()}
    op = case["op"]
    if op.startswith("loss"):
        return _loss_exact(case, t)
    if op.startswith("norm"):
        return _norm_exact(case, t)
    return _step_exact(case, t) if op == "step" else _prompt_exact(case, t)
