"""The operators at the ends of a model, without a GPU: the oracle's gradients against differences,
its sampling against the probabilities, and the refusals of the C ABI and of the binding."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import model_ends as M
from paper_2609_37842_amd import eogp as E

FAKE = ctypes.c_void_p(0x1000)


def directional(f, x, d, h):
    return (f(x + h * d) - f(x - h * d)) / (2 * h)


def test_layer_norm_gradients_against_differences():
    """Central differences in float64 at h = 1e-5: truncation h^2 and rounding 1e-16 / h, both about
    1e-10 of values of order 10, so 1e-7 bounds them."""
    g = np.random.default_rng(1)
    n, d = 6, 37
    x, dy, gam, bet = g.standard_normal((n, d)), g.standard_normal((n, d)), g.standard_normal(d), g.standard_normal(d)
    res = g.standard_normal((n, d))
    _, mean, rstd = M.layer_norm(x, gam, bet)
    dx, dg, db = M.layer_norm_backward(dy, x, gam, mean, rstd, residual=res)
    at = lambda xx, gg, bb: (M.layer_norm(xx, gg, bb)[0] * dy).sum() + (xx * res).sum()   # noqa: E731
    v, w = g.standard_normal((n, d)), g.standard_normal(d)
    assert abs(directional(lambda q: at(q, gam, bet), x, v, 1e-5) - (dx * v).sum()) < 1e-7
    assert abs(directional(lambda q: at(x, q, bet), gam, w, 1e-5) - (dg[0] * w).sum()) < 1e-7
    assert abs(directional(lambda q: at(x, gam, q), bet, w, 1e-5) - (db[0] * w).sum()) < 1e-7
    _, per, _ = M.layer_norm_backward(dy, x, gam, mean, rstd, groups=3)
    assert np.allclose(per.sum(0), dg[0])


def test_xent_and_embedding_gradients_against_differences():
    g = np.random.default_rng(2)
    n, V, d = 5, 23, 7
    l, lab = g.standard_normal((n, V)) * 3, g.integers(0, V, n)
    _, dl = M.softmax_xent(l, lab, grad_scale=0.5)
    v = g.standard_normal((n, V))
    assert abs(directional(lambda q: 0.5 * M.softmax_xent(q, lab)[0].sum(), l, v, 1e-5) - (dl * v).sum()) < 1e-7
    table, tok, dout = g.standard_normal((V, d)), g.integers(0, 4, 11), g.standard_normal((11, d))
    dt = M.embed_backward(dout, tok, V, 1.5)
    w = g.standard_normal((V, d))
    assert abs(directional(lambda q: (M.embed(q, tok, 1.5) * dout).sum(), table, w, 1e-5) - (dt * w).sum()) < 1e-7


@pytest.mark.parametrize("top_k,top_p,min_p,temperature", [(0, 1.0, 0.0, 1.0), (7, 1.0, 0.0, 0.6), (0, 0.8, 0.0, 1.3),
                                                           (20, 0.9, 0.05, 1.0)])
def test_oracle_sampling_follows_the_probabilities(top_k, top_p, min_p, temperature):
    """Evenly spread uniform numbers give each token its probability's share of the draws, within two
    draws (one at each end of its interval) and the weights' relative error of 2e-7."""
    g = np.random.default_rng(3)
    V, n = 50, 4000
    l = (g.standard_normal(V) * 2).astype(np.float32)
    u = ((np.arange(n) + 0.5) / n).astype(np.float32)
    got = np.bincount(M.sample(np.tile(l, (n, 1)), u, temperature, top_k, top_p, min_p), minlength=V)
    p = np.exp((l.astype(np.float64) - l.max()) / temperature)
    order = np.argsort(-l, kind="stable")
    keep = np.zeros(V, bool)
    keep[order[:top_k] if top_k else order] = True
    if top_p < 1:
        run = np.cumsum((p * keep)[order])
        cut = np.searchsorted(run, top_p * (p * keep).sum()) + 1
        keep[order[cut:]] = False
    keep &= p >= min_p
    p = p * keep / (p * keep).sum()
    assert np.all(np.abs(got - n * p) <= 2.01)
    assert np.all(got[~keep] == 0)


def test_weights_are_two_to_the_t():
    l = np.linspace(-18, 0, 4001).astype(np.float32)
    w = M._row_weights(l, 1.0)
    ref = np.exp(l.astype(np.float64)) * 2.0 ** 30
    # t = l log2 e carries one rounding of l log2 e (|t| 2^-24, times ln 2), the polynomial 2e-7, the floor 1
    assert np.all(np.abs(w - ref) <= ref * (np.abs(l) * 2.0 ** -23 + 3e-7) + 1)


def test_abi_refusals_without_device():
    L = E.load()
    inf, nan = float("inf"), float("nan")
    emb = lambda **k: L.eogp_embed_tokens(*(k.get(a, b) for a, b in dict(   # noqa: E731
        table=FAKE, tt=0, ldt=8, V=4, d=8, tok=FAKE, mask=None, n=3, scale=1.0, acc=0, out=FAKE, ot=0, ldo=8,
        s=None).items()))
    assert emb(n=-1) == -1 and emb(d=0) == -1 and emb(V=0) == -1 and emb(V=1 << 31) == -1 and emb(n=1 << 31) == -1
    assert emb(ldt=7) == -1 and emb(ldo=7) == -1 and emb(ldo=1 << 31) == -1 and emb(tt=5) == -1
    assert emb(tt=0, ot=1) == -2 and emb(tt=1, ot=2) == -2
    assert emb(table=None) == -1 and emb(tok=None) == -1 and emb(out=None) == -1
    assert emb(table=ctypes.c_void_p(0x1002)) == -1
    assert emb(n=0) == 0
    back = lambda **k: L.eogp_embed_backward(*(k.get(a, b) for a, b in dict(   # noqa: E731
        dout=FAKE, t=0, ldd=8, tok=FAKE, mask=None, n=3, V=4, d=8, scale=1.0, acc=0, dt=FAKE, ldt=8, ws=FAKE,
        wsb=1 << 30, s=None).items()))
    need = L.eogp_embed_backward_workspace_size(3, 4, 8)
    assert need > 0 and L.eogp_embed_backward_workspace_size(0, 4, 8) == 0
    assert L.eogp_embed_backward_workspace_size(3, 0, 8) == 0
    assert back(n=-1) == -1 and back(V=0) == -1 and back(ldd=7) == -1 and back(ldt=7) == -1 and back(t=3) == -1
    assert back(dout=None) == -1 and back(dt=None) == -1
    assert back(wsb=need - 1) == -4 and back(ws=None) == -4
    norm = lambda **k: L.eogp_layer_norm(*(k.get(a, b) for a, b in dict(   # noqa: E731
        x=FAKE, xt=0, ldx=8, g=FAKE, b=FAKE, wt=0, eps=1e-5, mask=None, n=3, d=8, y=FAKE, yt=0, ldy=8, ones=0,
        mean=None, rstd=None, s=None).items()))
    assert norm(n=-1) == -1 and norm(d=0) == -1 and norm(ldx=7) == -1 and norm(ldy=7) == -1
    assert norm(ones=1) == -1                                   # no room for the column
    assert norm(eps=-1.0) == -1 and norm(eps=nan) == -1 and norm(eps=inf) == -1
    assert norm(d=16385, ldx=16385, ldy=16385) == -2
    assert norm(xt=1, wt=2) == -2 and norm(xt=1, yt=2) == -2 and norm(xt=9) == -1 and norm(yt=9) == -1
    assert norm(x=None) == -1 and norm(y=None) == -1 and norm(n=0, x=None) == 0
    nb = lambda **k: L.eogp_layer_norm_backward(*(k.get(a, b) for a, b in dict(   # noqa: E731
        dy=FAKE, lddy=8, x=FAKE, ldx=8, t=0, g=FAKE, wt=0, mean=FAKE, rstd=FAKE, mask=None, res=None, ldr=0,
        groups=2, rows=3, d=8, dx=FAKE, lddx=8, dg=FAKE, db=FAKE, ws=FAKE, wsb=1 << 30, s=None).items()))
    need = L.eogp_layer_norm_backward_workspace_size(2, 3, 8, 0)
    assert need > 0 and L.eogp_layer_norm_backward_workspace_size(2, 3, 16385, 0) == 0
    assert nb(groups=-1) == -1 and nb(rows=-1) == -1 and nb(groups=1 << 20, rows=1 << 12) == -1
    assert nb(lddy=7) == -1 and nb(lddx=7) == -1 and nb(res=FAKE, ldr=7) == -1
    assert nb(mean=None) == -1 and nb(dx=None) == -1 and nb(wsb=need - 1) == -4 and nb(ws=None) == -4
    assert nb(t=2, wt=1) == -2 and nb(groups=0) == 0
    xe = lambda **k: L.eogp_softmax_xent(*(k.get(a, b) for a, b in dict(   # noqa: E731
        l=FAKE, t=0, ldl=8, lab=FAKE, mask=None, n=3, V=8, gs=1.0, loss=FAKE, dl=ctypes.c_void_p(0x9000), ldd=8,
        s=None).items()))
    assert xe(n=-1) == -1 and xe(V=0) == -1 and xe(ldl=7) == -1 and xe(ldd=7) == -1 and xe(t=4) == -1
    assert xe(l=None) == -1 and xe(lab=None) == -1 and xe(loss=None, dl=None) == -1
    assert xe(dl=FAKE, ldd=9) == -1 and xe(n=0) == 0
    sa = lambda **k: L.eogp_sample_tokens(*(k.get(a, b) for a, b in dict(   # noqa: E731
        l=FAKE, t=0, ldl=8, n=3, V=8, u=FAKE, mask=None, temp=1.0, top_k=0, top_p=1.0, min_p=0.0, out=FAKE,
        s=None).items()))
    assert sa(n=-1) == -1 and sa(V=0) == -1 and sa(ldl=7) == -1 and sa(V=(1 << 20) + 1, ldl=1 << 21) == -2
    for bad in (-0.5, nan, inf):
        assert sa(temp=bad) == -1
    for bad in (-0.01, 1.01, nan):
        assert sa(top_p=bad) == -1 and sa(min_p=bad) == -1
    assert sa(top_k=-1) == -1 and sa(u=None) == -1 and sa(out=None) == -1 and sa(l=None) == -1 and sa(n=0) == 0
    assert b"sample" in L.eogp_last_error()


def test_binding_refuses_bad_layouts():
    """Device tensors are asked for first; the layout helpers are checked on host tensors."""
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="device"):
        E.eogp_layer_norm(x)
    with pytest.raises(ValueError, match="device"):
        E.eogp_sample_tokens(x, torch.zeros(4))
    with pytest.raises(ValueError, match="unit column stride"):
        E._rows_of(torch.zeros(8, 4).t(), "x")
    with pytest.raises(ValueError, match="constant row stride"):
        E._rows_of(torch.zeros(3, 5, 8)[:, :4], "x")
    with pytest.raises(ValueError, match="overlapping"):
        E._rows_of(torch.zeros(8).expand(4, 8), "x")
    with pytest.raises(ValueError, match=r"\[n, d\]"):
        E._rows_of(torch.zeros(8), "x")
    with pytest.raises(ValueError, match="float32, bfloat16 or float16"):
        E._model_dtype(x.double(), "x")
    with pytest.raises(ValueError, match="labels"):
        E._per_row(torch.zeros(4, dtype=torch.int32), (4,), torch.int64, "labels")
    with pytest.raises(ValueError, match="gamma"):
        E._weight(torch.zeros(8, dtype=torch.bfloat16), 8, x, "gamma")
    assert E._rows_of(torch.zeros(3, 5, 9)[:, :, :8], "x") == (15, 8, 9)
    assert E._rows_of(torch.zeros(1, 5, 8)[:, ::2], "x") == (3, 8, 16)
    assert E._rows_of(torch.zeros(0, 8), "x") == (0, 8, 8)
    assert E._rows_of(torch.zeros(4, 1), "x") == (4, 1, 1)
