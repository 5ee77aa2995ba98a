"""The operators in the middle of a block at the ends of their types: scores of any finite size, infinities in places that
count for nothing, the most examples and heads of a call."""
import numpy as np
import pytest
import torch

import test_gpu_block_middle as B
from oracle import block_middle as M
from paper_2609_37842_amd import eogp as E

pytestmark = pytest.mark.gpu
DEV, DT, U, ULP = B.DEV, B.DT, B.U, B.ULP
say, gen, host, dev, near = B.say, B.gen, B.host, B.dev, B.near

# (q, k) with one element each, whose product is exact in fp32 and no power of two: a few bits of mantissa
SCORES = {
    "f32": [(76800.0, 65280.0), (76800.0, -65280.0), (150 * 2.0 ** 14, 255 * 2.0 ** 14), (150 * 2.0 ** 53, -255 * 2.0 ** 55), (19.0, 2.625e5), (150.0, -2.5625)],
    "bf16": [(76800.0, 65280.0), (76800.0, -65280.0), (150 * 2.0 ** 14, 255 * 2.0 ** 14), (150 * 2.0 ** 53, -255 * 2.0 ** 55), (19.0, 2.621e5)],
    "f16": [(19200.0, 16320.0), (19200.0, -16320.0), (38400.0, 65280.0), (1104.0, 9056.0), (1104.0, -9056.0)],
}


def large_scores(a, b, dt, N, Tq, Tk, H, D, g):
    """q, k and v: every third key has the score a b with all queries, the others are further down by at least 2^-9 of it.
    Queries of every second head have scores of 1 and less instead."""
    q, k = np.zeros((N, Tq, H, D)), np.zeros((N, Tk, H, D))
    q[..., 1] = a
    low = b - np.abs(b) * np.exp2(-g.integers(0, 8, (N, Tk, H)))
    k[..., 1] = np.where(np.arange(Tk)[None, :, None] % 3 == 0, b, low)
    q[:, :, 1::2, 1] = 0.0
    q[:, :, 1::2, 0] = 0.5
    k[..., 0] = g.integers(-8, 9, (N, Tk, H)) / 8.0
    return B.rounded(q, dt), B.rounded(k, dt), B.rounded(g.standard_normal((N, Tk, H, D)), dt)


def exact_bounds(q, k, v, scale, dt, how):
    """As attend_bounds, for scores that no rounding of a product or a sum touches: a weight is off by that of the score in
    powers of two, which all weights of its row share, and by its exponential's 2^-21; sums of at most Tk keys."""
    spread, rel = np.zeros(q.shape), np.full(q.shape[:3], 2.0 ** -21 + k.shape[1] * U)
    for n in range(q.shape[0]):
        see = M.sight(n, q.shape[1], k.shape[1], **how)
        cols = see.any(0)[:, None]
        for h in range(q.shape[2]):
            hk = h * k.shape[2] // q.shape[2]
            p, _ = M.head_weights(q[n, :, h], k[n, :, hk], see, scale)
            spread[n, :, h] = p @ np.where(cols, np.abs(v[n, :, hk]), 0.0)
    return spread * ((0.0 if dt == torch.float32 else ULP[dt]) + 2 * rel[..., None]), rel


@pytest.mark.parametrize("dtype,score", [(d, s) for d in DT for s in SCORES[d]])
@pytest.mark.parametrize("Tq", [1, 40])
@pytest.mark.parametrize("Tk", [1, 100, 4200])
def test_large_scores(dtype, score, Tq, Tk):
    """Weights of scores between 2^8 and 2^123 of either sign, few and many queries, keys in one piece and split. The
    log-sum-exp is that of the score, rounded in powers of two and back: 4 roundings."""
    dt = DT[dtype]
    say(f"[attention] scores {score} {dtype}, {Tq} queries, {Tk} keys")
    q, k, v = large_scores(*score, dt, 1, Tq, Tk, 3, 8, gen(31, Tq, Tk))
    how = dict(causal=False)
    ref, rlse = M.attention(q, k, v, 0.5, **how)
    tol, rel = exact_bounds(q, k, v, 0.5, dt, how)
    out, lse = E.eogp_attention(dev(q, dt), dev(k, dt), dev(v, dt), 0.5, **how)
    near(out, ref, tol, "out")
    near(lse, rlse, rel + 4 * U * (np.abs(rlse) + 12), "lse")


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("Tq", [1, 40])
def test_scores_of_minus_infinity(dtype, Tq):
    """Keys whose score is -inf have no weight; the lowest finite ones of a row that has no others have equal weights."""
    dt = DT[dtype]
    say(f"[attention] scores of -inf, {dtype}, {Tq} queries")
    g = gen(33, Tq)
    T, D, low = 200, 64, {"f32": -3e37, "bf16": -3e37, "f16": -6e4}[dtype]
    q, k, v = (B.rounded(x, dt) for x in (np.abs(g.standard_normal((1, Tq, 2, D))), g.standard_normal((1, T, 2, D)),
                                          g.standard_normal((1, T, 2, D))))
    k[0, ::3, 0, 0] = -np.inf
    q[0, :, 1], k[0, :, 1] = 0.0, 0.0
    q[0, :, 1, 3], k[0, :, 1, 3] = 1.0, B.rounded(np.array(low), dt)
    out, lse = E.eogp_attention(dev(q, dt), dev(k, dt), dev(v, dt), 0.75, causal=False)
    keep = np.arange(T) % 3 != 0
    for h, some in ((0, keep), (1, np.ones(T, bool))):
        one = [x[:, :, h:h + 1] if x is q else x[:, some, h:h + 1] for x in (q, k, v)]
        ref, rlse = M.attention(*one, 0.75, causal=False)
        tol, rel = (B.attend_bounds if h == 0 else exact_bounds)(*one, 0.75, dt, dict(causal=False))
        near(out[:, :, h:h + 1], ref, tol, "out")
        near(lse[:, :, h:h + 1], rlse, rel + 4 * U * (np.abs(rlse) + 12), "lse")


def gradient_bounds(q, k, v, scale, dt, how):
    """exact_bounds, and what the backward pass reads: the log-sum-exp is (reference + log2 of the sum) ln 2 in fp32, taken back
    to powers of two: roundings of the sum, both products and both constants, 5 half steps of its size in a weight's exponent.
    From 2^10 in powers of two on (710 in natural units) weights no longer depend on it."""
    tol, rel = exact_bounds(q, k, v, scale, dt, how)
    lse = np.nan_to_num(np.abs(M.attention(q, k, v, scale, **how)[1]), posinf=0.0)
    return tol, rel + 5 * U * np.minimum(lse, 710.0)


@pytest.mark.parametrize("dtype,score", [(d, s) for d in DT for s in SCORES[d] if abs(s[0] * s[1]) < 2.0 ** 60])
@pytest.mark.parametrize("Tq,Tk", [(1, 1), (1, 100), (40, 40), (70, 600)])
@pytest.mark.parametrize("one", [False, True])
def test_gradients_at_large_scores(dtype, score, Tq, Tk, one, monkeypatch):
    """The same scores in the backward pass, where queries see all keys or one: a log-sum-exp in fp32 does not hold what these
    weights are, sums of which are 1 all the same."""
    dt = DT[dtype]
    say(f"[attention_backward] scores {score} {dtype}, {Tq} queries, {Tk} keys, one={one}")
    g = gen(32, Tq, Tk)
    q, k, v = large_scores(*score, dt, 2, Tq, Tk, 3, 8, g)
    dout = B.rounded(0.01 * g.standard_normal(q.shape), dt)
    how = dict(causal=one, window=1 if one else 0)
    qd, kd, vd, dd = (dev(x, dt) for x in (q, k, v, dout))
    out, lse = E.eogp_attention(qd, kd, vd, 0.5, **how)
    got = E.eogp_attention_backward(dd, qd, kd, vd, out, lse, 0.5, **how)
    monkeypatch.setattr(B, "attend_bounds", gradient_bounds)
    ref = M.attention_backward(dout, q, k, v, 0.5, **how)
    for x, y, t, name in zip(got, ref, B.back_bounds(dout, q, k, v, 0.5, dt, how), ("dq", "dk", "dv")):
        near(x, y, t, name)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("D,width,interleaved", [(64, 32, False), (64, 32, True), (33, 14, False), (64, 0, False), (7, 2, True)])
def test_elements_that_pass(dtype, D, width, interleaved):
    """Elements behind the turned part come out as they are, whatever any of them holds, in both directions."""
    say(f"[rotate_heads] infinities behind {width} of {D} elements, {dtype}")
    dt = DT[dtype]
    torch.manual_seed(6)
    q, k = (torch.randn(2, 5, h, D, device=DEV).to(dt) for h in (3, 1))
    for x in (q, k):
        rest = x[..., width:].reshape(-1)
        rest[::5], rest[1::7], rest[2::11], rest[3::13] = float("inf"), float("-inf"), float("nan"), -0.0
        x[..., width:] = rest.view(x[..., width:].shape)
    table = E.eogp_rotary_table(5, width) if width else None
    for got in (E.eogp_rotate_heads(q, k, table, interleaved=interleaved),
                E.eogp_rotate_heads_backward(q, k, table=table, interleaved=interleaved)[:2]):
        for x, y in zip((q, k), got):
            assert torch.equal(torch.nan_to_num(x[..., width:], nan=7.0), torch.nan_to_num(y[..., width:], nan=7.0))
            assert torch.equal(x[..., width:].isnan(), y[..., width:].isnan())
            assert bool(y[..., :width].isfinite().all())


# ---- more blocks than a launch holds
@pytest.mark.parametrize("norm", ["head", "row"])
def test_gradients_of_a_million_examples(norm):
    """2^20 + 5 examples of a token, weights' gradients of each: 2^21 + 10 blocks. Bounds as in test_gpu_block_middle."""
    B.test_rotate_heads_backward(((1 << 20) + 5, 1, 1, 1, 8, 8, norm, False, "all", "split", 0), True, "f32")


def test_millions_of_heads():
    """2^28 + 300 heads of one element: 2^21 + 3 blocks. Without table and norm the heads are copied."""
    say("[rotate_heads] 2^28 + 300 heads")
    q = torch.randint(-(1 << 15), 1 << 15, ((1 << 28) + 300,), dtype=torch.int16, device=DEV).view(1, 1, -1, 1)
    for call in (lambda x, y: E.eogp_rotate_heads(x, q_out=y), lambda x, y: E.eogp_rotate_heads_backward(x, dq_in=y)):
        out = torch.zeros_like(q)
        call(q.view(torch.bfloat16), out.view(torch.bfloat16))
        # (every NaN is as good as another)
        assert bool(((out == q) | (((out & 0x7FFF) > 0x7F80) & ((q & 0x7FFF) > 0x7F80))).all())


@pytest.mark.parametrize("hold", [float("inf"), 60000.0, float("nan")])
@pytest.mark.parametrize("how", [dict(), dict(window=9, sinks=2), dict(q_mask=True), dict(causal=False, window=9)])
def test_fp16_gradients_beside_unseen_values(hold, how):
    """What keys hold that no query sees changes no bit of small gradients: fp16 score gradients are lifted by what the
    seen values allow."""
    say(f"[attention_backward] unseen values {hold} {how}")
    torch.manual_seed(7)
    N, Tq, Tk, H, D = 2, 40, 200, 2, 64
    q, do = (torch.randn(N, Tq, H, D, device=DEV).half() for _ in range(2))
    do *= 1e-4
    k, v = (torch.randn(N, Tk, H, D, device=DEV).half() for _ in range(2))
    start = torch.tensor([30, 60], device=DEV)
    how = dict(how, q_start=start)
    mask = None
    if how.pop("q_mask", False):
        mask = torch.ones(N, Tq, dtype=torch.uint8, device=DEV)
        mask[:, 25:] = 0
        mask[1, :4] = 0
    seen = [M.sight(n, Tq, Tk, **dict(how, q_start=[30, 60], q_mask=None if mask is None else host(mask))).any(0) for n in range(N)]
    unseen = ~torch.from_numpy(np.stack(seen)).to(DEV)
    assert bool(unseen.any(1).all())
    out, lse = E.eogp_attention(q, k, v, q_mask=mask, **how)
    clean = E.eogp_attention_backward(do, q, k, v, out, lse, q_mask=mask, **how)
    for x in (k, v):
        x[unseen] = hold
    for a, b in zip(clean, E.eogp_attention_backward(do, q, k, v, out, lse, q_mask=mask, **how)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Tq", [1, 40])
@pytest.mark.parametrize("size", [2.0 ** 90, 2.0 ** -90])
def test_large_and_small_values(dtype, Tq, size):
    """Values of 2^90 and of 2^-90 over 4,500 keys, scores of either sign: outputs are those of values near 1, times that. (A
    weight's product with 2^-90 is exact down to weights of 2^-36 of the largest; all smaller ones together are below 2^-23.)"""
    dt = DT[dtype]
    say(f"[attention] values of {size}, {dtype}, {Tq} queries")
    g = gen(34, Tq)
    q, k, v = (B.rounded(g.standard_normal((1, n, 2, 64)), dt) for n in (Tq, 4500, 4500))
    ref, _ = M.attention(q, k, v, 0.3, causal=False)
    tol, _ = B.attend_bounds(q, k, v, 0.3, dt, dict(causal=False))
    out, _ = E.eogp_attention(dev(q, dt), dev(k, dt), dev(v * size, dt), 0.3, causal=False)
    near(out, ref * size, (tol + 2.0 ** -23 * np.abs(v).max()) * size, "out")


@pytest.mark.parametrize("dtype,score", [(d, SCORES[d][i]) for d in DT for i in (0, 1, -1)])
@pytest.mark.parametrize("Tq,Tk", [(1, 900), (40, 100), (300, 300)])
def test_large_scores_beside_small_ones(dtype, score, Tq, Tk, monkeypatch):
    """Query heads of one key head, every second of them with scores of 1 and less: rows of both kinds share a wave, forward and
    backward. (A small score rounded in powers of two is off by 2^-25.)"""
    dt = DT[dtype]
    say(f"[attention] scores {score} beside small ones, {dtype}, {Tq} queries, {Tk} keys")
    g = gen(35, Tq, Tk)
    q, k, v = large_scores(*score, dt, 2, Tq, Tk, 4, 64, g)
    k, v = k[:, :, :1].copy(), v[:, :, :1].copy()
    dout = B.rounded(0.01 * g.standard_normal(q.shape), dt)
    how = dict(causal=Tq == Tk)
    qd, kd, vd, dd = (dev(x, dt) for x in (q, k, v, dout))
    out, lse = E.eogp_attention(qd, kd, vd, 0.5, **how)
    ref, rlse = M.attention(q, k, v, 0.5, **how)
    tol, rel = exact_bounds(q, k, v, 0.5, dt, how)
    near(out, ref, tol, "out")
    near(lse, rlse, rel + 4 * U * (np.abs(rlse) + 12), "lse")
    monkeypatch.setattr(B, "attend_bounds", gradient_bounds)
    got = E.eogp_attention_backward(dd, qd, kd, vd, out, lse, 0.5, **how)
    ref = M.attention_backward(dout, q, k, v, 0.5, **how)
    for x, y, t, name in zip(got, ref, B.back_bounds(dout, q, k, v, 0.5, dt, how), ("dq", "dk", "dv")):
        near(x, y, t, name)
