"""fp64 definitions of the operators in the middle of a block: rotary tables, norms and rotation of heads, attention.

Plain numpy, one head at a time where that is the clearer; no code of the library."""
import numpy as np


def rotary_table(positions, width, base=10000.0, factor=1.0, original=0, low=1.0, high=32.0, magnitude=1.0):
    """[positions, width / 2, 2]: magnitude (cos, sin) of position times frequency."""
    f = base ** (-2.0 * np.arange(width // 2) / width)
    g = np.zeros_like(f)
    if original:
        g = np.clip((original * f / (2 * np.pi) - low) / (high - low), 0.0, 1.0)
    f = f * (g + (1 - g) / factor)
    angle = np.arange(positions)[:, None] * f
    return magnitude * np.stack([np.cos(angle), np.sin(angle)], -1)


def turn(x, table, positions, interleaved, back=False):
    """Pairs of the first elements of heads x [n, H, D] turned by the table's row of each position [n] (transposed if
    back); NaN in turned elements where the table has no such row."""
    y = np.array(x, dtype=np.float64)
    if table is None:
        return y
    half = table.shape[1]
    known = (positions >= 0) & (positions < table.shape[0])
    t = np.where(known[:, None, None], table[np.where(known, positions, 0)].astype(np.float64), np.nan)
    c, s = t[:, None, :, 0], t[:, None, :, 1] * (-1 if back else 1)
    ia, ib = (np.arange(0, 2 * half, 2), np.arange(1, 2 * half, 2)) if interleaved else (np.arange(half), half + np.arange(half))
    a, b = x[:, :, ia], x[:, :, ib]
    y[:, :, ia], y[:, :, ib] = a * c - b * s, a * s + b * c
    return y


def _stats(x, norm, weight, eps):
    """(rstd [n, 1 or H, 1], gain [H, D], elements of a norm) of heads [n, H, D]."""
    n, H, D = x.shape
    if norm == "none":
        return np.ones((n, 1, 1)), np.ones((H, D)), 1
    axes, m = ((2,), D) if norm == "head" else ((1, 2), H * D)
    r = (np.square(x).sum(axes, keepdims=True) / m + eps) ** -0.5
    gain = np.ones((H, D)) if weight is None else np.broadcast_to(weight, (H, D)) if norm == "head" else weight.reshape(H, D)
    return r, gain.astype(np.float64), m


def rotate(x, table, positions, norm="none", weight=None, eps=1e-6, interleaved=False, mask=None):
    """y of heads [n, H, D] of n tokens; zeros for masked tokens."""
    y = np.zeros(x.shape)
    live = np.ones(len(x), bool) if mask is None else mask != 0
    xl = x[live].astype(np.float64)
    r, gain, _ = _stats(xl, norm, weight, eps)
    y[live] = turn(xl * r * gain, table, positions[live], interleaved)
    return y


def rotate_backward(dy, x, table, positions, norm="none", weight=None, eps=1e-6, interleaved=False, mask=None, groups=1):
    """(dx, d_weight [groups, weight] or None) of heads [n, H, D]."""
    n, H, D = dy.shape
    dx = np.zeros(dy.shape)
    live = np.ones(n, bool) if mask is None else mask != 0
    t = turn(dy[live].astype(np.float64), table, positions[live], interleaved, back=True)
    if norm == "none":
        dx[live] = t
        return dx, None
    xl = x[live].astype(np.float64)
    r, gain, m = _stats(xl, norm, weight, eps)
    xh, tw = xl * r, t * gain
    dx[live] = r * (tw - xh * ((tw * xh).sum((2,) if norm == "head" else (1, 2), keepdims=True) / m))
    each = np.zeros((n, H, D))
    each[live] = t * xh
    each = each.reshape(groups, n // groups, H, D).sum(1)
    return dx, each.sum(1) if norm == "head" else each.reshape(groups, H * D)


def sight(n, Tq, Tk, causal=True, window=0, sinks=0, q_start=None, q_mask=None, k_mask=None):
    """[Tq, Tk] bool of example n: which keys each query sees."""
    p = np.arange(Tq)[:, None] + (Tk - Tq if q_start is None else int(q_start[n]))
    j = np.arange(Tk)[None, :]
    see = np.ones((Tq, Tk), bool)
    if causal:
        see &= j <= p
    if window:
        see &= (np.abs(p - j) < window) | (j < sinks)
    if k_mask is not None:
        see &= (k_mask[n] != 0)[None, :]
    if q_mask is not None:
        see &= (q_mask[n] != 0)[:, None]
    return see


def head_weights(q, k, see, scale):
    """(weights [Tq, Tk], log-sum-exp [Tq]) of one head; masked rows may hold anything."""
    rows, cols = see.any(1), see.any(0)
    q, k = np.where(rows[:, None], q, 0.0).astype(np.float64), np.where(cols[:, None], k, 0.0).astype(np.float64)
    l = np.where(see, q @ k.T * scale, -np.inf)
    top = np.where(rows, l.max(1, initial=-np.inf), 0.0)
    e = np.exp(l - top[:, None])
    total = e.sum(1)
    with np.errstate(divide="ignore"):
        return e / np.where(rows, total, 1.0)[:, None], np.where(rows, top + np.log(np.where(rows, total, 1.0)), -np.inf)


def attention(q, k, v, scale, **how):
    """(out, lse) of q [N, Tq, Hq, D] and k, v [N, Tk, Hkv, D]."""
    N, Tq, Hq, D = q.shape
    out, lse = np.zeros(q.shape), np.full((N, Tq, Hq), -np.inf)
    for n in range(N):
        see = sight(n, Tq, k.shape[1], **how)
        cols = see.any(0)[:, None]
        for h in range(Hq):
            hk = h * k.shape[2] // Hq
            p, lse[n, :, h] = head_weights(q[n, :, h], k[n, :, hk], see, scale)
            out[n, :, h] = p @ np.where(cols, v[n, :, hk], 0.0).astype(np.float64)
    return out, lse


def attention_backward(dout, q, k, v, scale, **how):
    """(dq, dk, dv)."""
    N, Tq, Hq, D = q.shape
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for n in range(N):
        see = sight(n, Tq, k.shape[1], **how)
        rows, cols = see.any(1)[:, None], see.any(0)[:, None]
        for h in range(Hq):
            hk = h * k.shape[2] // Hq
            p, _ = head_weights(q[n, :, h], k[n, :, hk], see, scale)
            do, vh = np.where(rows, dout[n, :, h], 0.0).astype(np.float64), np.where(cols, v[n, :, hk], 0.0).astype(np.float64)
            dp = do @ vh.T
            ds = p * (dp - (p * dp).sum(1, keepdims=True)) * scale
            dq[n, :, h] = ds @ np.where(cols, k[n, :, hk], 0.0)
            dk[n, :, hk] += ds.T @ np.where(rows, q[n, :, h], 0.0)
            dv[n, :, hk] += p.T @ do
    return dq, dk, dv
