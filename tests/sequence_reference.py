"""Plain numpy implementations in 64 bits of the operators around the scan, with their gradients from
the formulas, token by token and row by row.  Test infrastructure."""
import numpy as np


def sigmoid(v):
    return 0.5 * (1 + np.tanh(0.5 * v))


def softplus(v):
    return np.logaddexp(0, v)


def gated_parts(x, ga, gx, decay, rate):
    r, i = sigmoid(ga), sigmoid(gx)
    la = -rate * softplus(decay)[:, None] * r
    return r, i, la, np.exp(la), np.sqrt(-np.expm1(2 * la))


def gated_fwd(x, ga, gx, decay, rate=8.0, starts=None, reverse=False, h0=None):
    """y and the leaving state; with the states before each token, in stored order."""
    B, D, L = x.shape
    r, i, la, a, b = gated_parts(x, ga, gx, decay, rate)
    h = np.zeros((B, D)) if h0 is None else h0.astype(np.float64)
    y, before = np.zeros(x.shape), np.zeros(x.shape)
    for t in (range(L - 1, -1, -1) if reverse else range(L)):
        if starts is not None:
            h = np.where(starts[:, None, t] != 0, 0.0, h)
        before[..., t] = h
        h = a[..., t] * h + b[..., t] * i[..., t] * x[..., t]
        y[..., t] = h
    return y, h, before


def gated_bwd(x, ga, gx, decay, dout, rate=8.0, starts=None, reverse=False, h0=None, dhT=None):
    B, D, L = x.shape
    r, i, la, a, b = gated_parts(x, ga, gx, decay, rate)
    _, _, before = gated_fwd(x, ga, gx, decay, rate, starts, reverse, h0)
    psi = np.zeros((B, D)) if dhT is None else dhT.astype(np.float64)
    s = np.zeros(x.shape)
    for t in (range(L) if reverse else range(L - 1, -1, -1)):
        s[..., t] = dout[..., t] + psi
        psi = a[..., t] * s[..., t]
        if starts is not None:
            psi = np.where(starts[:, None, t] != 0, 0.0, psi)
    # la / b goes to 0 with la
    slope = np.divide(la, b, out=np.zeros_like(la), where=b > 0)
    q = s * (a * before * la - a * a * slope * i * x)
    ratio = np.where(decay < -30, 1.0, sigmoid(decay) / np.maximum(softplus(decay), 1e-300))
    return dict(dx=s * b * i, dgate_a=q * (1 - r), dgate_x=s * b * i * (1 - i) * x, ddecay=q.sum((0, 2)) * ratio, dh0=psi)


def norm_fwd(x, weight=None, bias=None, residual=None, eps=1e-5):
    s = x if residual is None else x + residual
    mean = s.mean(-1, keepdims=True)
    rstd = 1 / np.sqrt(((s - mean) ** 2).mean(-1, keepdims=True) + eps)
    y = (s - mean) * rstd * (1 if weight is None else weight) + (0 if bias is None else bias)
    return y, s, mean[..., 0], rstd[..., 0]


def norm_bwd(s, weight, dout, dsum=None, eps=1e-5):
    _, _, mean, rstd = norm_fwd(s, eps=eps)
    hat = (s - mean[..., None]) * rstd[..., None]
    g = dout * (1 if weight is None else weight)
    ds = rstd[..., None] * (g - g.mean(-1, keepdims=True) - hat * (g * hat).mean(-1, keepdims=True))
    rows = tuple(range(s.ndim - 1))
    return dict(ds=ds + (0 if dsum is None else dsum), dweight=(dout * hat).sum(rows), dbias=dout.sum(rows))


def embed_fwd(ids, weight, scale=1.0):
    ok = (ids >= 0) & (ids < weight.shape[0])
    return np.where(ok[..., None], scale * weight[np.where(ok, ids, 0)], 0.0)


def embed_bwd(ids, dout, vocab, scale=1.0):
    g = np.zeros((vocab, dout.shape[-1]))
    for i, v in enumerate(ids.reshape(-1)):
        if 0 <= v < vocab:
            g[v] += dout.reshape(-1, dout.shape[-1])[i]
    return scale * g
