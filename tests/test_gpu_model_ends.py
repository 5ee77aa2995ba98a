"""The operators at the ends of a model against float64, through the binding: every type, widths and
vocabularies on both sides of each kernel's tile, rows at any element, masks that leave nothing."""
import numpy as np
import pytest
import torch

from oracle import model_ends as M
from paper_2609_37842_amd import eogp as E

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
# unit roundoff of significands of 24, 8 and 11 bits; fp16 has a subnormal step of 2^-24
ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}


def say(msg):
    print(msg, flush=True)


def gen(*key):
    return np.random.default_rng(list(key))


def dev(a, dtype=torch.float32, ld=None, shift=0):
    """A device copy of the host rows, rounded to dtype, `ld` apart and starting `shift` elements in."""
    a = torch.from_numpy(np.ascontiguousarray(a)).to(dtype)
    if ld is None:
        return a.to(DEV)
    n, d = a.shape
    buf = torch.full((n * ld + shift + d,), float("nan"), dtype=dtype, device=DEV)
    view = torch.as_strided(buf, (n, d), (ld, 1), shift)
    view.copy_(a)
    return view


def host(t):
    return t.detach().to(torch.float64).cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def near(got, ref, tol, what):
    """|got - ref| <= tol (fp32 arithmetic) + the rounding to got's type; NaN where ref has NaN."""
    g = host(got).reshape(ref.shape)
    bound = tol + ULP[got.dtype] * 1.01 * np.abs(ref) + TINY[got.dtype]
    assert np.array_equal(np.isnan(g), np.isnan(ref)), what
    bad = ~(np.abs(g - ref) <= bound) & ~np.isnan(ref)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} beyond the bound, the first at {np.argwhere(bad)[0]}: " \
        f"{g[bad][0]} for {ref[bad][0]} (+- {np.broadcast_to(bound, ref.shape)[bad][0]})"


def masks(kind, n, g):
    return None if kind == "all" else np.zeros(n, np.uint8) if kind == "none" else (g.random(n) < 0.6).astype(np.uint8)


# ---- layer norm -------------------------------------------------------------------------------
# widths on both sides of one wave's, four waves' and sixteen waves' registers, for 4 and 8 elements a piece
WIDTHS = [1, 2, 7, 63, 64, 65, 255, 257, 511, 768, 1023, 1025, 2047, 2049, 4095, 4097, 5120, 8193, 16383, 16384]


def norm_inputs(d, n, dtype, g, mask):
    x = (g.standard_normal((n, d)) * np.exp(0.5 * g.standard_normal(d)) + 3.0)
    x = torch.from_numpy(x).to(dtype).double().numpy()
    if mask is not None:
        x[mask == 0] = np.nan
    gam = torch.from_numpy(1 + 0.3 * g.standard_normal(d)).to(dtype).double().numpy()
    bet = torch.from_numpy(g.standard_normal(d)).to(dtype).double().numpy()
    return x, gam, bet


def norm_tolerance(x, gam, bet, mean, rstd):
    """Sums of d terms run in fp32 as chains of at most 64 and trees: 80 roundings of 2^-24 of sum |x|;
    the mean's error enters y times rstd, the variance's (two such sums) relative to y; and a dozen
    roundings of the formula itself."""
    u = 2.0 ** -24
    ax = np.nan_to_num(np.abs(x)).mean(1, keepdims=True)
    xh = np.nan_to_num(np.abs(x - mean[:, None])) * rstd[:, None]
    return u * (80 * ax * rstd[:, None] * np.abs(gam) + (100 + 80 * ax * rstd[:, None]) * xh * np.abs(gam) + 2 * np.abs(bet))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d", WIDTHS)
def test_layer_norm(d, dtype):
    dt = DT[dtype]
    g = gen(1, d)
    for n, mk, ones, out32, w32, shift in [(1, "all", False, False, False, 0), (5, "some", True, False, True, 1),
                                           (9, "some", False, True, False, 3), (3, "none", True, False, False, 0)]:
        say(f"[layer_norm] d={d} {dtype} n={n} mask={mk} ones={ones} fp32 out={out32} shift={shift}")
        mask = masks(mk, n, g)
        x, gam, bet = norm_inputs(d, n, dt, g, mask)
        wt = torch.float32 if w32 else dt
        ot = torch.float32 if out32 else dt
        xd = dev(x, dt, d + 5, shift) if shift else dev(x, dt)
        ybuf = torch.full((n, d + 4), 7.0, dtype=ot, device=DEV)
        y = ybuf[:, 1:d + 1 + int(ones)]
        _, mean, rstd = E.eogp_layer_norm(xd, dev(gam, wt), dev(bet, wt), 1e-5, None if mask is None else dev(mask, torch.uint8),
                                          ones, out=y)
        torch.cuda.synchronize()
        ry, rm, rr = M.layer_norm(x, gam, bet, 1e-5, mask, ones)
        tol = norm_tolerance(x, gam, bet, rm, rr)
        tol = np.concatenate([tol, np.zeros((n, 1))], 1) if ones else tol
        near(y, ry, tol, "y")
        near(mean, rm, 80 * 2.0 ** -24 * np.nan_to_num(np.abs(x)).mean(1), "mean")
        near(rstd, rr, rr * (100 + 80 * np.abs(rm) * rr) * 2.0 ** -24, "rstd")
        assert torch.all(ybuf[:, 0] == 7.0) and torch.all(ybuf[:, d + 1 + int(ones):] == 7.0)


def test_layer_norm_constant_rows_infinities_and_defaults():
    say("[layer_norm] constant rows, inf, nan, no weights")
    x = np.full((4, 300), 2.5)
    x[1, 7] = np.inf
    x[2, 299] = np.nan
    x[3] = np.arange(300)
    y, mean, rstd = E.eogp_layer_norm(dev(x))
    torch.cuda.synchronize()
    assert torch.all(y[0] == 0) and abs(float(rstd[0]) - 1e-5 ** -0.5) < 1e-3 and float(mean[0]) == 2.5
    assert torch.isnan(y[1, 7]) and torch.isnan(y[2]).all()
    near(y[3:], M.layer_norm(x[3:])[0], 2e-5, "y")
    empty = E.eogp_layer_norm(torch.empty((0, 8), device=DEV))
    assert empty[0].shape == (0, 8) and empty[1].shape == (0,)


def back_tolerance(x, dy, gam, mean, rstd, live):
    u = 2.0 ** -24
    ax = np.where(live[:, None], np.nan_to_num(np.abs(x - mean[:, None])), 0) * rstd[:, None]
    t = np.where(live[:, None], np.nan_to_num(np.abs(dy)), 0) * np.abs(gam)
    # xh carries 2 u |x| rstd of its difference besides its own roundings
    xe = np.where(live[:, None], np.nan_to_num(np.abs(x)) + np.abs(mean[:, None]), 0) * rstd[:, None]
    sums = 90 * (t.mean(1, keepdims=True) + ax * (t * (ax + xe)).mean(1, keepdims=True)) + xe * (t * ax).mean(1, keepdims=True)
    return u * rstd[:, None] * (8 * t + 4 * sums + 4 * ax * (t * ax).mean(1, keepdims=True))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d", WIDTHS)
def test_layer_norm_backward(d, dtype):
    dt = DT[dtype]
    g = gen(2, d)
    cases = [(1, 1, "all", False, False, 0), (3, 7, "some", True, True, 1), (2, 41, "some", False, True, 0),
             (4, 3, "none", True, False, 0), (1, 130, "some", True, False, 3)]
    for N, T, mk, res, per, shift in cases:
        n = N * T
        say(f"[layer_norm_backward] d={d} {dtype} N={N} T={T} mask={mk} residual={res} per_example={per} shift={shift}")
        mask = masks(mk, n, g)
        live = np.ones(n, bool) if mask is None else mask != 0
        x, gam, bet = norm_inputs(d, n, dt, g, mask)
        _, mean, rstd = M.layer_norm(x, gam, bet, 1e-5, mask)
        mean, rstd = mean.astype(np.float32), rstd.astype(np.float32)
        rows = lambda: torch.from_numpy(np.where(live[:, None], g.standard_normal((n, d)), np.nan)).to(dt).double().numpy()   # noqa: E731
        dy, rs = rows(), rows() if res else None
        put = lambda a: (dev(a, dt, d + 5, shift) if shift else dev(a, dt))   # noqa: E731
        three = lambda t: torch.as_strided(t, (N, T, d), (T * t.stride(0), t.stride(0), 1), t.storage_offset()) if n > 1 else t.view(N, T, d)   # noqa: E731
        dx, dg, db = E.eogp_layer_norm_backward(
            three(put(dy)), three(put(x)), dev(gam, dt), dev(mean).view(N, T), dev(rstd).view(N, T),
            None if mask is None else dev(mask, torch.uint8).view(N, T), three(put(rs)) if res else None, per)
        torch.cuda.synchronize()
        rdx, rdg, rdb = M.layer_norm_backward(dy, x, gam, mean, rstd, mask, rs, N if per else 1)
        tol = back_tolerance(x, dy, gam, mean.astype(np.float64), rstd.astype(np.float64), live)
        if res:
            tol = tol + 2.0 ** -23 * np.where(live[:, None], np.nan_to_num(np.abs(rs)), 0)
        near(dx, rdx, tol, "dx")
        # chains of at most 130 rows; a term carries 4 u of itself and 2 u (|x| + |mean|) rstd |dy|
        a = np.where(live[:, None], np.nan_to_num(np.abs(dy)), 0)
        xh = np.where(live[:, None], np.nan_to_num(np.abs(x)) + np.abs(mean[:, None]), 0) * rstd[:, None]
        fold = lambda v: v.reshape(N if per else 1, -1, d).sum(1)   # noqa: E731
        near(dg, rdg, 150 * 2.0 ** -24 * fold(a * xh), "dgamma")
        near(db, rdb, 140 * 2.0 ** -24 * fold(a), "dbeta")


def test_layer_norm_backward_over_the_residual_and_repeatable():
    say("[layer_norm_backward] dx is residual; repeated calls; no rows")
    g = gen(3)
    N, T, d = 9, 33, 770
    x, dy, res = (dev(g.standard_normal((N * T, d))).view(N, T, d) for _ in range(3))
    gam = dev(1 + 0.1 * g.standard_normal(d))
    _, mean, rstd = E.eogp_layer_norm(x, gam)
    first = E.eogp_layer_norm_backward(dy, x, gam, mean, rstd, residual=res)
    again = E.eogp_layer_norm_backward(dy, x, gam, mean, rstd, residual=res)
    over = res.clone()
    E.eogp_layer_norm_backward(dy, x, gam, mean, rstd, residual=over, dx=over)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, again)) and torch.equal(over, first[0])
    e = torch.empty((2, 0, 5), device=DEV)
    m = torch.empty((2, 0), device=DEV)
    _, dg, db = E.eogp_layer_norm_backward(e, e, None, m, m, per_example=True)
    torch.cuda.synchronize()
    assert torch.all(dg == 0) and torch.all(db == 0) and dg.shape == (2, 5)


# ---- embedding --------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("d", [1, 5, 64, 255, 257, 513, 768, 1027, 2048, 5121])
def test_embed_tokens(d, dtype):
    dt = DT[dtype]
    g = gen(4, d)
    for n, V, mk, out32, acc, shift in [(1, 1, "all", False, False, 0), (37, 50, "some", False, False, 1),
                                        (130, 7, "some", True, True, 0), (6, 9, "none", False, True, 0)]:
        say(f"[embed] d={d} {dtype} n={n} V={V} mask={mk} fp32 out={out32} accumulate={acc} shift={shift}")
        mask = masks(mk, n, g)
        table = torch.from_numpy(g.standard_normal((V, d))).to(dt).double().numpy()
        tok = g.integers(0, V, n)
        if n > 30:
            tok[3], tok[4] = -1, V                          # outside: NaN
            if mask is not None:
                mask[3], tok[7], mask[7] = 1, V + 10 ** 12, 0     # masked: not looked at
        ot = torch.float32 if out32 else dt
        start = torch.from_numpy(g.standard_normal((n, d))).to(ot)
        buf = torch.full((n, d + 3), 7.0, dtype=ot, device=DEV)
        out = buf[:, 1:d + 1]
        out.copy_(start)
        E.eogp_embed_tokens(dev(table, dt, d + 2, shift), torch.from_numpy(tok).to(DEV), 1.7,
                            None if mask is None else dev(mask, torch.uint8), out, acc)
        torch.cuda.synchronize()
        ref = M.embed(table, tok, 1.7, mask)
        ref = ref + start.double().numpy() if acc else ref
        near(out, ref, 2.0 ** -22 * np.nan_to_num(np.abs(ref) + np.abs(start.double().numpy())), "out")
        assert torch.all(buf[:, 0] == 7.0) and torch.all(buf[:, d + 1:] == 7.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,V,d", [(1, 1, 1), (63, 5, 64), (64, 1, 33), (65, 300, 257), (129, 2, 515), (1000, 70000, 20),
                                   (2047, 511, 100), (2049, 512, 7), (4097, 3, 70), (5000, 300000, 9),
                                   (20011, 1000, 65), (70003, 17, 40)])
def test_embed_backward(n, V, d, dtype):
    dt = DT[dtype]
    g = gen(5, n, V, d)
    for mk, acc, shift, spread in [("all", False, 0, "even"), ("some", True, 1, "zipf"), ("none", False, 0, "even"),
                                   ("some", False, 0, "one")]:
        say(f"[embed_backward] n={n} V={V} d={d} {dtype} mask={mk} accumulate={acc} tokens={spread}")
        mask = masks(mk, n, g)
        tok = (g.integers(0, V, n) if spread == "even" else np.full(n, V // 2) if spread == "one" else
               np.minimum((np.exp(g.random(n) * np.log(V + 1)) - 1).astype(np.int64), V - 1))
        if n > 10:
            tok[0], tok[n // 2], tok[n - 1] = -5, V, 1 << 40     # count for no token
        do = torch.from_numpy(g.standard_normal((n, d))).to(dt).double().numpy()
        if mask is not None:
            do[mask == 0] = np.nan
        if n > 10:
            do[[0, n // 2, n - 1]] = np.nan
        start = g.standard_normal((V, d)).astype(np.float32)
        buf = torch.full((V, d + 3), 7.0, device=DEV)
        dtab = buf[:, 2:d + 2]
        dtab.copy_(torch.from_numpy(start))
        E.eogp_embed_backward(dev(do, dt, d + 1, shift), torch.from_numpy(tok).to(DEV), V, 0.75,
                              None if mask is None else dev(mask, torch.uint8), dtab, acc)
        torch.cuda.synchronize()
        ref = M.embed_backward(do, tok, V, 0.75, mask)
        # chains of 64 rows, then of n / 256 chunk sums, then a few
        size = M.embed_backward(np.nan_to_num(np.abs(do)), tok, V, 0.75, mask)
        tol = (72 + n / 256) * 2.0 ** -24 * size + (2.0 ** -23 * np.abs(start) if acc else 0)
        near(dtab, ref + (start if acc else 0.0), tol, "dtable")
        assert torch.all(buf[:, :2] == 7.0) and torch.all(buf[:, d + 2:] == 7.0)


def test_embed_backward_no_rows_and_repeatable():
    say("[embed_backward] no rows; repeated calls")
    t = E.eogp_embed_backward(torch.empty((0, 6), device=DEV), torch.empty(0, dtype=torch.int64, device=DEV), 5)
    torch.cuda.synchronize()
    assert torch.all(t == 0)
    g = gen(6)
    do = dev(g.standard_normal((9000, 130)), torch.bfloat16)
    tok = torch.from_numpy(g.integers(0, 40, 9000)).to(DEV)
    a, b = (E.eogp_embed_backward(do, tok, 40) for _ in range(2))
    torch.cuda.synchronize()
    assert torch.equal(a, b)


# ---- cross-entropy ----------------------------------------------------------------------------
# vocabularies on both sides of each block shape, and beyond the registers of one block
VOCABS = [1, 2, 3, 63, 1000, 1025, 2047, 4097, 8190, 16385, 32771, 50257, 65537, 100352, 131073]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", VOCABS)
def test_softmax_xent(V, dtype):
    dt = DT[dtype]
    g = gen(7, V)
    for n, mk, pad, shift, over in [(1, "all", 0, 0, False), (6, "some", 1, 1, False), (3, "none", 0, 0, True),
                                    (4, "some", 0, 3, True)]:
        say(f"[xent] V={V} {dtype} n={n} mask={mk} pad={pad} shift={shift} in place={over}")
        mask = masks(mk, n, g)
        live = np.ones(n, bool) if mask is None else mask != 0
        l = torch.from_numpy(g.standard_normal((n, V)) * 4 + 10).to(dt).double().numpy()
        if pad and V > 1:
            l[:, V - pad:] = -np.inf
        lab = g.integers(0, max(1, V - pad), n)
        if n > 3:
            lab[1] = -100                                   # ignored, whatever its mask
            live[1] = False
        l[~live] = np.nan
        buf = dev(l, dt, V + 3, shift)
        dl = buf if over else None
        loss, dl = E.eogp_softmax_xent(buf, torch.from_numpy(lab).to(DEV), None if mask is None else dev(mask, torch.uint8),
                                       0.5, dlogits=dl)
        torch.cuda.synchronize()
        rl, rd = M.softmax_xent(l, lab, mask, 0.5)
        # exponents of up to 40 carry a few roundings of themselves (2^-24 each), a sum's chain of at
        # most V / 256 terms and its log as many
        rel = (6 * 60 + min(V / 256, 600) + 20) * 2.0 ** -24
        near(loss, rl, rel + 6 * 2.0 ** -24 * (np.abs(rl) + 20), "loss")
        near(dl, rd, rel * (np.abs(rd) + 2.0 ** -24) + 2.0 ** -23, "dlogits")


def test_xent_infinite_logits_gradientless_and_repeatable():
    say("[xent] infinities, NaN, large values, loss only")
    l = np.zeros((6, 700))
    l[0] = 1e4 * gen(8).standard_normal(700)             # differences of 1e4: one token has it all
    l[1, 5:] = -np.inf                                   # five tokens left
    l[2] = -np.inf                                       # none left: no distribution
    l[3, 9] = np.nan
    l[4, 3] = np.inf
    l[5] = -65504.0
    lab = np.array([int(np.argmax(l[0])), 6, 0, 0, 3, 699])
    ld, labd = dev(l), torch.from_numpy(lab).to(DEV)
    loss, dl = E.eogp_softmax_xent(ld, labd)
    only, none = E.eogp_softmax_xent(ld, labd, grad=False)
    torch.cuda.synchronize()
    assert none is None and torch.equal(loss[:2], only[:2]) and torch.equal(loss[5:], only[5:])
    assert abs(float(loss[0])) < 1e-6 and float(loss[1]) == np.inf and abs(float(loss[5]) - np.log(700)) < 1e-5
    assert torch.isnan(loss[2]) and torch.isnan(loss[3]) and torch.isnan(dl[3]).all()
    assert np.allclose(host(dl[1, :5]), 0.2, rtol=1e-6) and float(dl[1, 6]) == -1.0 and torch.all(dl[1, 7:] == 0)
    assert np.allclose(host(dl[5, :699]), 1 / 700, rtol=1e-6)


# ---- sampling ---------------------------------------------------------------------------------
OPTIONS = [dict(), dict(temperature=0.0), dict(temperature=0.7, min_p=0.05), dict(top_k=1), dict(top_k=5, temperature=2.5),
           dict(top_p=0.9), dict(top_p=0.0), dict(top_k=40, top_p=0.8, min_p=0.01, temperature=0.8),
           dict(top_p=0.999999), dict(top_k=300, top_p=0.5), dict(min_p=1.0)]


def sample_both(l, u, mask=None, dtype=torch.float32, ld=None, shift=0, **opt):
    l32 = torch.from_numpy(l).to(dtype).float().numpy()
    got = E.eogp_sample_tokens(dev(l, dtype, ld, shift), dev(u.astype(np.float32)),
                               token_mask=None if mask is None else dev(mask, torch.uint8), **opt)
    torch.cuda.synchronize()
    ref = M.sample(l32, u.astype(np.float32), mask=mask, **opt)
    assert np.array_equal(got.cpu().numpy(), ref), (opt, got.cpu().numpy(), ref)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", VOCABS)
def test_sample_tokens(V, dtype):
    g = gen(9, V)
    for opt in OPTIONS:
        say(f"[sample] V={V} {dtype} {opt}")
        l = g.standard_normal((5, V)) * 3
        mask = np.array([1, 0, 1, 1, 1], np.uint8)
        l[1] = np.nan
        sample_both(l, g.random(5), mask, DT[dtype], V + 3, 1, **opt)


@pytest.mark.parametrize("opt", OPTIONS, ids=str)
def test_sample_ties_infinities_and_ends_of_the_unit_interval(opt):
    """Ties go to the lowest index in every filter; rows without a finite logit give no token."""
    say(f"[sample] ties and infinities {opt}")
    g = gen(10)
    V = 3001
    l = np.round(g.standard_normal((14, V)) * 1.5)         # a dozen values: long runs of ties
    l[1] = 0.0                                             # all equal
    l[2] = -np.inf
    l[3] = np.nan
    l[4, 5:] = -np.inf
    l[5, ::3] = np.nan
    l[6, 100] = l[6, 2000] = np.inf                        # two tokens share everything
    l[7] = -0.0
    l[7, ::2] = 0.0
    l[8] = -1e30 * np.arange(V)
    l[9, 17] = 500.0
    l[10] = np.linspace(0, -40, V)
    u = g.random(14)
    u[11:] = [0.0, 1.0 - 2.0 ** -24, 1.5]
    sample_both(l, u, **opt)
    sample_both(l, 1 - u, **opt)


@pytest.mark.parametrize("k", [1, 2, 255, 256, 257, 2999, 3000, 3001, 5000])
@pytest.mark.parametrize("p", [1.0, 0.6])
def test_sample_top_k_counts_among_ties(k, p):
    say(f"[sample] top_k={k} top_p={p} among ties")
    g = gen(11, k)
    l = np.round(g.standard_normal((24, 3001)) * 0.7)
    sample_both(l, np.linspace(0, 0.9999, 24), top_k=k, top_p=p)
    sample_both(np.zeros((8, 3001)), np.linspace(0, 0.9999, 8), top_k=k, top_p=p)


def test_sample_largest_vocabulary():
    say("[sample] V = 2^20")
    g = gen(12)
    l = g.standard_normal((2, 1 << 20))
    for opt in (dict(), dict(top_k=1000, top_p=0.9)):
        sample_both(l, g.random(2), **opt)
    with pytest.raises(E.EogpError, match="2\\^20"):
        E.eogp_sample_tokens(torch.zeros((1, (1 << 20) + 1), device=DEV), torch.zeros(1, device=DEV))


def test_sampled_tokens_follow_the_probabilities():
    """Evenly spread uniform numbers give each token its share of the draws: within two draws, and the
    roundings of the weights (under 1e-5 of 200,000 draws)."""
    say("[sample] 200,000 draws")
    n, V = 200_000, 61
    l = gen(13).standard_normal(V) * 2
    got = E.eogp_sample_tokens(dev(l).expand(n, V).contiguous(), (torch.arange(n, device=DEV) + 0.5) / n, temperature=1.5)
    torch.cuda.synchronize()
    p = np.exp(l.astype(np.float32).astype(np.float64) / 1.5)
    got = np.bincount(got.cpu().numpy(), minlength=V)
    assert np.all(np.abs(got - n * p / p.sum()) <= 4)


# ---- streams, graphs, refusals ----------------------------------------------------------------
def chain(tok, table, gam, bet, wts, u, mask, stream=None):
    """Every operator once, each fed by the one before."""
    x = E.eogp_embed_tokens(table, tok, 4.0, mask, stream=stream)
    y, mean, rstd = E.eogp_layer_norm(x, gam, bet, token_mask=mask, stream=stream)
    lab = E.eogp_sample_tokens(y, u, top_k=30, top_p=0.9, token_mask=mask, stream=stream)
    loss, dy = E.eogp_softmax_xent(y, lab, mask, stream=stream)
    dx, dg, db = E.eogp_layer_norm_backward(dy, x, gam, mean, rstd, mask, per_example=True, stream=stream)
    dt = E.eogp_embed_backward(dx, tok, table.shape[0], 4.0, mask, stream=stream)
    return x, y, lab, loss, dy, dx, dg, db, dt


def chain_inputs(seed):
    g = gen(14, seed)
    V, d, N, T = 500, 300, 5, 40
    return (torch.from_numpy(g.integers(0, V, (N, T))).to(DEV), dev(g.standard_normal((V, d))),
            dev(1 + 0.1 * g.standard_normal(d)), dev(g.standard_normal(d)), None,
            dev(g.random((N, T))), dev((g.random((N, T)) < 0.8).astype(np.uint8), torch.uint8))


def test_another_stream_and_graph_replays_agree_with_the_eager_calls():
    say("[chain] another stream, then a captured graph replayed on new inputs")
    ins = [chain_inputs(k) for k in range(4)]
    eager = [chain(*a) for a in ins]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = chain(*ins[0], stream=side)
    for _ in range(3):
        torch.empty(1 << 20, device=DEV).fill_(1.0)         # what the call left free is used again at once
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, eager[0]))
    fixed = [t.clone() if t is not None else None for t in ins[0]]
    graph = torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain(*fixed)
    torch.cuda.current_stream().wait_stream(side)
    with torch.cuda.graph(graph):
        out = chain(*fixed)
    for k in (1, 2, 3, 0):
        for t, new in zip(fixed, ins[k]):
            if t is not None:
                t.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager[k])), k
        chain(*ins[(k + 1) % 4])                            # eager work between the replays
        torch.cuda.synchronize()


def test_refusals_leave_the_outputs_alone():
    say("[refusals]")
    x = torch.zeros((4, 8), device=DEV)
    out = torch.full((4, 8), 7.0, device=DEV)
    with pytest.raises(ValueError, match="out must"):
        E.eogp_layer_norm(x, out=out[:, :7])
    with pytest.raises(ValueError, match="gamma"):
        E.eogp_layer_norm(x, torch.zeros(8, dtype=torch.float16, device=DEV), out=out)
    with pytest.raises(E.EogpError):
        E.eogp_layer_norm(x, eps=-1.0, out=out)
    with pytest.raises(ValueError, match="token_mask"):
        E.eogp_layer_norm(x, token_mask=torch.ones(4, dtype=torch.bool, device=DEV), out=out)
    with pytest.raises(ValueError, match="tokens"):
        E.eogp_embed_tokens(x, torch.zeros(4, dtype=torch.int32, device=DEV), out=out)
    with pytest.raises(ValueError, match="accumulate"):
        E.eogp_embed_tokens(x, torch.zeros(4, dtype=torch.int64, device=DEV), accumulate=True)
    with pytest.raises(ValueError, match="workspace"):
        E.eogp_embed_backward(x, torch.zeros(4, dtype=torch.int64, device=DEV), 4,
                              ws=torch.empty(16, dtype=torch.uint8, device=DEV))
    with pytest.raises(ValueError, match="labels"):
        E.eogp_softmax_xent(x, torch.zeros(3, dtype=torch.int64, device=DEV), dlogits=out)
    with pytest.raises(E.EogpError):
        E.eogp_sample_tokens(x, torch.zeros(4, device=DEV), top_p=1.5)
    with pytest.raises(E.EogpError):
        E.eogp_sample_tokens(x)                              # no uniform numbers
    torch.cuda.synchronize()
    assert torch.all(out == 7.0)
