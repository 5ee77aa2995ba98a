"""float64 definitions of the operators at the ends of a language model (numpy only): token
embedding, layer norm, cross-entropy, and sampling (whole numbers, so it must agree exactly)."""
from __future__ import annotations

import math

import numpy as np

# 2^f on [-1/2, 1/2] for the sampling weights: coefficients of f^1 .. f^5 (f^0 is 1).
EXP2 = tuple(np.float32(c) for c in (0.6931470036506653, 0.24022242426872253, 0.05550733581185341,
                                     0.009671512991189957, 0.001326472731307149))


def _valid(mask, n):
    return np.ones(n, bool) if mask is None else np.asarray(mask).reshape(-1) != 0


def embed(table, tokens, scale=1.0, mask=None):
    """[n, d]; zeros in masked rows, NaN where a token lies outside the table."""
    tokens = np.asarray(tokens).reshape(-1)
    V = table.shape[0]
    ok = (tokens >= 0) & (tokens < V)
    out = np.asarray(table, np.float64)[np.where(ok, tokens, 0)] * scale
    out[~ok] = np.nan
    out[~_valid(mask, tokens.size)] = 0.0
    return out


def embed_backward(d_out, tokens, V, scale=1.0, mask=None):
    tokens = np.asarray(tokens).reshape(-1)
    use = _valid(mask, tokens.size) & (tokens >= 0) & (tokens < V)
    out = np.zeros((V, d_out.shape[1]))
    np.add.at(out, tokens[use], np.asarray(d_out, np.float64)[use])
    return out * scale


def layer_norm(x, gamma=None, beta=None, eps=1e-5, mask=None, ones_column=False):
    """(y, mean, rstd) of rows [n, d]; zeros in masked rows."""
    x = np.asarray(x, np.float64).copy()
    live = _valid(mask, x.shape[0])
    x[~live] = 0.0
    mean = x.mean(1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    y = y * (1.0 if gamma is None else np.asarray(gamma, np.float64))
    y = y + (0.0 if beta is None else np.asarray(beta, np.float64))
    if ones_column:
        y = np.concatenate([y, np.ones((x.shape[0], 1))], 1)
    y[~live] = 0.0
    return y, np.where(live, mean, 0.0), np.where(live, rstd, 0.0)


def layer_norm_backward(dy, x, gamma, mean, rstd, mask=None, residual=None, groups=1):
    """(dx [n, d], d_gamma [groups, d], d_beta [groups, d])."""
    live = _valid(mask, x.shape[0])
    z = lambda v: np.where(live[:, None], np.asarray(v, np.float64), 0.0)   # noqa: E731
    mean = np.where(live, np.asarray(mean, np.float64).reshape(-1), 0.0)[:, None]
    rstd = np.where(live, np.asarray(rstd, np.float64).reshape(-1), 0.0)[:, None]
    dy, xh = z(dy), (z(x) - mean) * rstd
    t = dy * (1.0 if gamma is None else np.asarray(gamma, np.float64))
    dx = rstd * (t - t.mean(1, keepdims=True) - xh * (t * xh).mean(1, keepdims=True))
    if residual is not None:
        dx = dx + z(residual)
    fold = lambda v: v.reshape(groups, -1, v.shape[1]).sum(1)   # noqa: E731
    return dx, fold(dy * xh), fold(dy)


def softmax_xent(logits, labels, mask=None, grad_scale=1.0):
    """(loss [n], d_logits [n, V])."""
    l = np.asarray(logits, np.float64).copy()
    labels = np.asarray(labels).reshape(-1)
    n, V = l.shape
    live = _valid(mask, n) & (labels >= 0) & (labels < V)
    l[~live] = 0.0
    at = np.where(live, labels, 0)
    with np.errstate(invalid="ignore", over="ignore"):
        top = l.max(1, keepdims=True)
        lse = top + np.log(np.exp(l - top).sum(1, keepdims=True))
        p = np.exp(l - lse)
        loss = lse[:, 0] - l[np.arange(n), at]
    p[np.arange(n), at] -= 1.0
    loss[~live] = 0.0
    p[~live] = 0.0
    return loss, p * grad_scale


def _row_weights(l, temperature):
    """floor(2^30 2^t) of one row of float32 logits (NaN already -inf), as int64."""
    most = l.max()
    c = np.float32(math.log2(math.e) / temperature)
    with np.errstate(invalid="ignore", over="ignore"):
        t = np.where(l == most, np.float32(0), (l - most) * c)
    t = np.maximum(t, np.float32(-64))
    k = np.rint(t)
    f = t - k
    p = f * EXP2[4] + EXP2[3]
    for a in (EXP2[2], EXP2[1], EXP2[0], np.float32(1)):
        p = p * f + a
    assert p.dtype == np.float32
    return (p.astype(np.float64) * 2.0 ** 30).astype(np.int64) >> np.minimum(-k, 62).astype(np.int64)


def sample(logits, uniforms, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, mask=None):
    """Tokens [n] by the integer definition of eogp_sample_tokens, in Python's whole numbers."""
    logits = np.asarray(logits, np.float32)
    n, V = logits.shape
    live = _valid(mask, n)
    out = np.full(n, -1, np.int64)
    for i in range(n):
        if not live[i]:
            continue
        l = np.where(np.isnan(logits[i]), np.float32(-np.inf), logits[i])
        if l.max() == -np.inf:
            continue
        if temperature == 0:
            out[i] = int(np.argmax(l))
            continue
        w = _row_weights(l, temperature)
        order = np.lexsort((np.arange(V), -(l.astype(np.float64) + 0.0)))
        kept = order[:top_k] if top_k else order
        p24 = math.floor(top_p * 2.0 ** 24 + 0.5)
        if p24 < 1 << 24:
            mass = np.cumsum(w[kept])
            want = max(1, (int(mass[-1]) * p24) >> 24)
            kept = kept[:int(np.searchsorted(mass, want)) + 1]
        w_kept = np.zeros_like(w)
        w_kept[kept] = w[kept]
        w_kept[w_kept < math.ceil(min_p * 2.0 ** 30)] = 0
        cdf = np.cumsum(w_kept)
        u = float(uniforms[i])
        r = min(max(math.floor(u * 2.0 ** 24) if u == u else 0, 0), 2 ** 24 - 1)
        target = (int(cdf[-1]) * r) >> 24
        out[i] = int(np.searchsorted(cdf, target, side="right"))
    return out
