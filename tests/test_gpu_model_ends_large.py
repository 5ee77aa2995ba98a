"""The operators at the ends of a model where a launch holds fewer blocks or waves than rows, lists have many
tiles, and tables are large: what small cases do not reach. Against float64 on the rows that are looked at, or
against smaller calls that the small cases cover."""
import numpy as np
import pytest
import torch

from oracle import model_ends as M
from paper_2609_37842_amd import eogp as E
from test_gpu_model_ends import DEV, DT, ULP, gen, host, near, norm_tolerance, say

pytestmark = pytest.mark.gpu


def randn(seed, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=torch.Generator(DEV).manual_seed(seed), device=DEV).to(dtype)


def some(seed, n, share):
    """A uint8 mask with about `share` ones, and a run of zeros longer than any tile of rows."""
    m = (torch.rand(n, generator=torch.Generator(DEV).manual_seed(seed), device=DEV) < share).to(torch.uint8)
    m[n // 3:n // 3 + n // 10] = 0
    return m


# ---- rows in turn in one block -----------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,V", [(9000, 700), (5000, 1500), (2500, 3001), (1300, 9001), (1300, 20011), (900, 40009)])
def test_xent_rows_in_turn(n, V, dtype):
    say(f"[xent] n={n} V={V} {dtype}")
    dt, g = DT[dtype], gen(20, n, V)
    l = randn(V, n, V, dtype=dt) * 3
    mask = some(n, n, 0.8)
    lab = torch.from_numpy(g.integers(-2, V + 2, n)).to(DEV)
    live = (mask != 0) & (lab >= 0) & (lab < V)
    l[~live] = float("nan")
    loss, dl = E.eogp_softmax_xent(l, lab, mask, 0.5)
    only, _ = E.eogp_softmax_xent(l, lab, mask, grad=False)
    torch.cuda.synchronize()
    assert torch.equal(loss, only)
    assert torch.all(loss[~live] == 0) and not torch.any(dl[~live])
    lse = torch.logsumexp(l[live].double(), 1)
    at = lab[live][:, None]
    ref = lse - l[live].double().gather(1, at)[:, 0]
    # exponents of up to 40 carry a few roundings of 2^-24 each, a sum's chain V / 256 terms
    rel = (6 * 40 + V / 256 + 20) * 2.0 ** -24
    near(loss[live], ref.cpu().numpy(), rel + 8 * 2.0 ** -24 * (np.abs(ref.cpu().numpy()) + 20), "loss")
    p = torch.exp(l[live].double() - lse[:, None])
    p.scatter_add_(1, at, -torch.ones_like(at, dtype=torch.float64))
    p *= 0.5
    bound = rel * (p.abs() + 2.0 ** -24) + 2.0 ** -23 + ULP[dt] * 1.01 * p.abs() + 2.0 ** -25
    assert bool(((dl[live].double() - p).abs() <= bound).all())


@pytest.mark.parametrize("opt", [dict(), dict(temperature=0.0), dict(min_p=0.02, temperature=0.8), dict(top_k=30, top_p=0.9),
                                 dict(top_p=0.95, temperature=1.5)], ids=str)
@pytest.mark.parametrize("n,V,dtype", [(9000, 700, "bf16"), (2500, 3001, "f32"), (1300, 9001, "bf16"), (1300, 20011, "f32"),
                                       (900, 40009, "f16")])
def test_sample_rows_in_turn(n, V, dtype, opt):
    """Rows alone give the tokens that they give among many, and the first, middle and last are the oracle's."""
    say(f"[sample] n={n} V={V} {dtype} {opt}")
    l = randn(V + 1, n, V, dtype=DT[dtype]) * 3
    u = torch.rand(n, generator=torch.Generator(DEV).manual_seed(n), device=DEV)
    mask = some(V, n, 0.8)
    l[mask == 0] = float("nan")
    got = E.eogp_sample_tokens(l, u, token_mask=mask, **opt)
    torch.cuda.synchronize()
    assert torch.all(got[mask == 0] == -1)
    for a in range(0, n, 150):                             # fewer rows than blocks: each block has one
        assert torch.equal(got[a:a + 150], E.eogp_sample_tokens(l[a:a + 150], u[a:a + 150], token_mask=mask[a:a + 150], **opt)), a
    look = [0, 1, n // 2, n - 2, n - 1]
    ref = M.sample(l[look].float().cpu().numpy(), u[look].cpu().numpy(), mask=mask[look].cpu().numpy(), **opt)
    assert np.array_equal(got[look].cpu().numpy(), ref)


@pytest.mark.parametrize("opt", [dict(top_k=300), dict(top_k=1000, top_p=0.99), dict(top_p=0.99, temperature=1.5),
                                 dict(top_p=0.999, temperature=4.0), dict(top_k=17000, temperature=3.0)], ids=str)
@pytest.mark.parametrize("V", [7001, 50257])
def test_sample_wide_filters(V, opt):
    say(f"[sample] V={V} {opt}")
    for dt, scale in ((torch.float32, 1.0), (torch.bfloat16, 3.0)):
        l = randn(V, 6, V, dtype=dt) * scale
        u = torch.tensor([0.0, 0.2, 0.5, 0.9, 0.999, 1.0 - 2.0 ** -24], device=DEV)
        got = E.eogp_sample_tokens(l, u, **opt)
        torch.cuda.synchronize()
        assert np.array_equal(got.cpu().numpy(), M.sample(l.float().cpu().numpy(), u.cpu().numpy(), **opt))


def test_sample_more_rows_than_a_launch_holds():
    n = (1 << 21) + 1037
    say(f"[sample] n={n} V=5")
    l, u = randn(5, n, 5), torch.rand(n, generator=torch.Generator(DEV).manual_seed(6), device=DEV)
    for opt in (dict(), dict(temperature=0.0), dict(top_k=2), dict(top_p=0.7)):
        got = E.eogp_sample_tokens(l, u, **opt)
        half = n // 2
        torch.cuda.synchronize()
        assert torch.equal(got[:half], E.eogp_sample_tokens(l[:half], u[:half], **opt)), opt
        assert torch.equal(got[half:], E.eogp_sample_tokens(l[half:], u[half:], **opt)), opt


# ---- layer norm: many rows per wave -------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d", [(20_000, 64), (600_000, 5), (300_000, 40), (9000, 1100), (3000, 5000), (2000, 9000), (1500, 16384)])
def test_layer_norm_rows_in_turn(n, d, dtype):
    say(f"[layer_norm] n={n} d={d} {dtype}")
    dt = DT[dtype]
    mask = some(d, n, 0.7)
    x, dy, res = (randn(k, n, d, dtype=dt) for k in (1, 2, 3))
    x += 2.0
    gam, bet = (1 + 0.3 * randn(4, d)).to(dt), randn(5, d, dtype=dt)
    x[mask == 0] = dy[mask == 0] = float("nan")
    y, mean, rstd = E.eogp_layer_norm(x, gam, bet, token_mask=mask)
    dx, dg, db = E.eogp_layer_norm_backward(dy, x, gam, mean, rstd, mask, residual=res)
    torch.cuda.synchronize()
    look = np.unique(np.concatenate([[0, n - 1], gen(21, d).integers(0, n, 300)]))
    at = torch.from_numpy(look).to(DEV)
    sub = [host(t[at]) for t in (x, dy, res)]
    mk = mask[at].cpu().numpy()
    ry, rm, rr = M.layer_norm(sub[0], host(gam), host(bet), 1e-5, mk)
    tol = norm_tolerance(sub[0], host(gam), host(bet), rm, rr)
    near(y[at], ry, tol, "y")
    near(mean[at], rm, 80 * 2.0 ** -24 * np.nan_to_num(np.abs(sub[0])).mean(1), "mean")
    rdx = M.layer_norm_backward(sub[1], sub[0], host(gam), host(mean[at]), host(rstd[at]), mk, sub[2])[0]
    # a mean of d fp32 terms and a dozen roundings, of values of at most a few tens
    big = np.abs(np.nan_to_num(sub[1])).max(1, keepdims=True) * (1 + np.abs(host(gam))) * rr[:, None] * 12
    near(dx[at], rdx, 100 * 2.0 ** -24 * (big + np.abs(sub[2])), "dx")
    # weight gradients, in float64 on the device
    lv = mask != 0
    xh = ((x.double() - mean.double()[:, None]) * rstd.double()[:, None])[lv]
    dyl = dy.double()[lv]
    # chains of the rows of one wave (under n / 256 + 64) and trees
    u = (n / 256 + 120) * 2.0 ** -24
    near(dg, (dyl * xh).sum(0).cpu().numpy(), u * (dyl * (xh.abs() + 4)).abs().sum(0).cpu().numpy(), "dgamma")
    near(db, dyl.sum(0).cpu().numpy(), u * dyl.abs().sum(0).cpu().numpy(), "dbeta")


def test_layer_norm_backward_many_examples():
    say("[layer_norm_backward] 40,000 examples of 3 rows")
    N, T, d = 40_000, 3, 33
    x, dy = randn(7, N, T, d), randn(8, N, T, d)
    mask = some(9, N * T, 0.6).view(N, T)
    y, mean, rstd = E.eogp_layer_norm(x, token_mask=mask)
    dx, dg, db = E.eogp_layer_norm_backward(dy, x, None, mean, rstd, mask, per_example=True)
    torch.cuda.synchronize()
    rdx, rg, rb = M.layer_norm_backward(*(host(t).reshape(N * T, d) for t in (dy, x)), None, host(mean).reshape(-1),
                                        host(rstd).reshape(-1), mask.reshape(-1).cpu().numpy(), groups=N)
    near(dx, rdx.reshape(N, T, d), 2e-5 * (1 + np.abs(rdx).max()), "dx")
    near(dg, rg, 16 * 2.0 ** -24 * 3 * 30, "dgamma")
    near(db, rb, 4 * 2.0 ** -24 * 3 * 6, "dbeta")


# ---- embedding -----------------------------------------------------------------------------------
@pytest.mark.parametrize("n,V,d,dtype", [(140_000, 3000, 40, "bf16"), (131_072, 600, 33, "f32"), (131_073, 200_000, 8, "f16"),
                                         (5000, 70_000, 1000, "f32"), (160_000, 70_000, 1000, "bf16"), (40_000, 50, 1300, "f32"),
                                         (2048, 70_000, 1000, "f32"), (300_000, 1, 16, "f32")])
def test_embed_backward_large(n, V, d, dtype):
    say(f"[embed_backward] n={n} V={V} d={d} {dtype}")
    dt, g = DT[dtype], gen(22, n, V)
    tok = np.minimum((np.exp(g.random(n) * np.log(V + 1)) - 1).astype(np.int64), V - 1)
    tok[::97] = -1
    tok[::101] = V
    t = torch.from_numpy(tok).to(DEV)
    mask = some(V, n, 0.9)
    do = randn(n, n, d, dtype=dt)
    dead = (mask == 0) | (t < 0) | (t >= V)
    do[dead] = float("nan")
    for acc in (False, True):
        dtab = torch.full((V, d), 0.5, device=DEV)
        E.eogp_embed_backward(do, t, V, 0.5, mask, dtab, acc)
        torch.cuda.synchronize()
        ref = torch.zeros((V, d), dtype=torch.float64, device=DEV)
        size = torch.zeros((V, d), dtype=torch.float64, device=DEV)
        keep = (~dead).nonzero()[:, 0]
        for part in keep.split(20_000):
            rows = do[part].double()
            ref.index_add_(0, t[part], rows)
            size.index_add_(0, t[part], rows.abs())
        # chains of 64 rows, then of a quarter of a token's chunks, then a few
        bound = (72 + n / 128) * 2.0 ** -24 * 0.5 * size + 2.0 ** -23
        assert bool(((dtab.double() - ref * 0.5 - (0.5 if acc else 0.0)).abs() <= bound).all()), acc


def test_embed_tokens_more_rows_than_waves():
    say("[embed_tokens] 200,000 rows of 70; 70,000 of 1,300")
    for n, V, d, dt in ((200_000, 900, 70, torch.float32), (70_000, 5000, 1300, torch.bfloat16)):
        table = randn(d, V, d, dtype=dt)
        t = torch.from_numpy(gen(23, n).integers(0, V, n)).to(DEV)
        mask = some(d, n, 0.8)
        got = E.eogp_embed_tokens(table, t, token_mask=mask)
        add = torch.ones((n, d), dtype=torch.float32, device=DEV)
        E.eogp_embed_tokens(table, t, 2.0, mask, out=add, accumulate=True)
        torch.cuda.synchronize()
        want = torch.where(mask[:, None] != 0, table[t], torch.zeros((), dtype=dt, device=DEV))
        assert torch.equal(got, want)
        assert torch.equal(add, want.float() * 2 + 1)


def test_rows_beyond_32_bit_offsets():
    """Logits and rows of more than 2^32 elements: the last rows give what they give alone."""
    say("[offsets] 90,000 rows of 50,257 bf16; 4,500,000 rows of 1,000 bf16")
    n, V = 90_000, 50_257
    l = torch.zeros((n, V), dtype=torch.bfloat16, device=DEV)
    l[-300:] = randn(30, 300, V, dtype=torch.bfloat16) * 3
    lab = torch.from_numpy(gen(24).integers(0, V, n)).to(DEV)
    u = torch.rand(n, generator=torch.Generator(DEV).manual_seed(31), device=DEV)
    for opt in (dict(), dict(top_k=20, top_p=0.9), dict(temperature=0.0)):
        assert torch.equal(E.eogp_sample_tokens(l, u, **opt)[-300:], E.eogp_sample_tokens(l[-300:].clone(), u[-300:], **opt))
    loss, dl = E.eogp_softmax_xent(l[-300:].clone(), lab[-300:])
    alone = loss.clone(), dl.clone()
    loss, dl = E.eogp_softmax_xent(l, lab, dlogits=l)                    # over the logits
    torch.cuda.synchronize()
    assert torch.equal(loss[-300:], alone[0]) and torch.equal(dl[-300:], alone[1])
    del l, dl
    n, d = 4_500_000, 1000
    table = randn(32, 3000, d, dtype=torch.bfloat16)
    t = torch.from_numpy(gen(25).integers(0, 3000, n)).to(DEV)
    x = E.eogp_embed_tokens(table, t)
    assert torch.equal(x[-200:], table[t[-200:]])
    y, mean, rstd = E.eogp_layer_norm(x)
    y2, mean2, rstd2 = E.eogp_layer_norm(x[-200:].clone())
    assert torch.equal(y[-200:], y2) and torch.equal(mean[-200:], mean2)
    y[:-200] = 0
    dx, dg, db = E.eogp_layer_norm_backward(y, x, None, mean, rstd)
    dx2, dg2, db2 = E.eogp_layer_norm_backward(y2, x[-200:].clone(), None, mean2, rstd2)
    torch.cuda.synchronize()
    assert torch.equal(dx[-200:], dx2)
    # sums of 200 rows in another order
    size = (y2.abs().double() * 8).sum(0).cpu().numpy()
    near(dg, host(dg2), 300 * 2.0 ** -24 * size, "dgamma")
    del y, dx
    dtab = E.eogp_embed_backward(x, t, 3000)
    times = torch.bincount(t, minlength=3000).double()
    want = times[:, None] * table.double()
    torch.cuda.synchronize()
    # equal terms: a chain's error is at most its length times a rounding of its sum
    assert bool(((dtab.double() - want).abs() <= 2.0 ** -24 * 200 * want.abs()).all())


def test_what_shared_memory_held_before_does_not_matter():
    """Before each call every CU's shared memory is filled with NaN (as a norm's weights), at widths that end
    inside a piece of 16 bytes; the results are those of calls after it was filled with ones."""
    say("[shared memory] NaN before every call")
    n = 4000
    wide = torch.zeros((8192, 8192), device=DEV)
    for dt in DT.values():
        for d in (5, 9, 70, 301, 1027, 4099, 8201, 16383):
            x, dy = randn(d, n, d, dtype=dt), randn(d + 1, n, d, dtype=dt)
            tok = torch.from_numpy(gen(26, d).integers(0, d, n)).to(DEV)
            u = torch.rand(n, generator=torch.Generator(DEV).manual_seed(d), device=DEV)
            gam = (1 + 0.1 * randn(d + 2, d)).to(dt)
            both = []
            for value in (1.0, float("nan")):
                fill = torch.full((8192,), value, device=DEV)
                got = []
                def call(f):
                    E.eogp_layer_norm(wide, fill, fill)
                    r = f()
                    got.extend(r if isinstance(r, tuple) else (r,))
                    return r
                y, mean, rstd = call(lambda: E.eogp_layer_norm(x, gam, gam))
                call(lambda: E.eogp_layer_norm_backward(dy, x, gam, mean, rstd))
                call(lambda: E.eogp_softmax_xent(x, tok))
                call(lambda: E.eogp_sample_tokens(x, u))
                call(lambda: E.eogp_sample_tokens(x[:50], u[:50], top_k=40, top_p=0.9))
                call(lambda: E.eogp_embed_backward(dy[:1500], tok[:1500], d))
                call(lambda: E.eogp_embed_backward(dy, tok, d))
                torch.cuda.synchronize()
                both.append(got)
            assert all(torch.equal(a, b) for a, b in zip(*both)), (dt, d)
            assert not torch.isnan(both[1][3]).any()


@pytest.mark.parametrize("n", [2048, 2049, 4095, 4097, 6143, 6144, 6145, 8193])
@pytest.mark.parametrize("V", [1, 40, 30000])
def test_embed_backward_at_the_ends_of_its_sorts(n, V):
    """Whole numbers, so that any order of the sums is exact: small masked and unmasked lists, one token to many."""
    say(f"[embed_backward] n={n} V={V}")
    g = gen(27, n, V)
    tok = torch.from_numpy(g.integers(-1, V + 1, n)).to(DEV)
    do = torch.from_numpy(g.integers(-100, 100, (n, 37)).astype(np.float32)).to(DEV)
    for mask in (None, torch.from_numpy((g.random(n) < 0.7).astype(np.uint8)).to(DEV)):
        got = E.eogp_embed_backward(do, tok, V, token_mask=mask)
        keep = (tok >= 0) & (tok < V) & (True if mask is None else mask != 0)
        want = torch.zeros((V, 37), device=DEV).index_add_(0, tok[keep], do[keep])
        torch.cuda.synchronize()
        assert torch.equal(got, want)
