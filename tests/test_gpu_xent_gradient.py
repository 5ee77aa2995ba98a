"""Every element of the cross-entropy's gradient to its own relative precision, so that a lost, stale or shifted
piece of a row shows also where probabilities are 1e-6 and less.

Tolerances. Logits spread over 40, so an exponent t = (l - max) log2 e of up to 58 carries three roundings of
2^-24 of itself, as does its sum with log2 of the row's sum: under 6 * 60 roundings of 2^-24, relative, in the
probability; the sum's chain of at most V / 256 terms and its logarithm as many; 20 for the exponentials and the
product with the scale; and one rounding to the gradient's type. Only at the label is there a difference (p - 1),
whose absolute error is 2^-23 of the scale. The scale of 4,096 keeps fp16 probabilities down to 1e-8 normal."""
import numpy as np
import pytest
import torch

from paper_2609_37842_amd import eogp as E
from test_gpu_model_ends import DEV, DT, TINY, ULP, VOCABS, gen, say

pytestmark = pytest.mark.gpu
SCALE = 4096.0


def assert_gradient(dl, l, lab):
    """dl of live rows against float64 softmax of the logits l."""
    n, V = l.shape
    rel = (6 * 60 + min(V / 256, 600) + 20) * 2.0 ** -24
    for rows in torch.arange(n, device=DEV).split(max(1, 20_000_000 // V)):
        x = l[rows].double()
        p = torch.exp(x - torch.logsumexp(x, 1, keepdim=True))
        bound = SCALE * rel * p
        at = lab[rows][:, None]
        p.scatter_add_(1, at, torch.full(at.shape, -1.0, dtype=torch.float64, device=DEV))
        bound.scatter_add_(1, at, torch.full(at.shape, SCALE * 2.0 ** -23, dtype=torch.float64, device=DEV))
        ref = SCALE * p
        bound += ULP[dl.dtype] * 1.01 * ref.abs() + TINY[dl.dtype]
        got = dl[rows].double()
        bad = ~((got - ref).abs() <= bound)
        if bad.any():
            r, c = (int(v) for v in bad.nonzero()[0])
            raise AssertionError(f"{int(bad.sum())} of {bad.numel()} beyond the bound, the first at row {int(rows[r])}, "
                                 f"column {c}: {float(got[r, c])} for {float(ref[r, c])} (+- {float(bound[r, c])})")
        assert torch.all(got[x == float("-inf")].abs() == 0)          # (a label has a finite logit here)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V", VOCABS)
def test_gradient_of_each_element(V, dtype):
    dt, g = DT[dtype], gen(50, V)
    for n, pad, shift, over in [(1, 0, 0, False), (6, 1, 1, False), (5, 0, 3, True), (4, 2, 0, True)]:
        say(f"[xent gradient] V={V} {dtype} n={n} pad={pad} shift={shift} in place={over}")
        pad = pad if V > 4 else 0
        l = torch.from_numpy(g.standard_normal((n, V)) * 4 + 10).to(dt).to(DEV)
        if pad:
            l[:, V - pad:] = float("-inf")
        lab = torch.from_numpy(g.integers(0, V - pad, n)).to(DEV)
        ld = V + 3 if shift else V
        buf = torch.full((n * ld + shift + 8,), float("nan"), dtype=dt, device=DEV)
        dl = torch.as_strided(buf, (n, V), (ld, 1), shift)
        if over:
            dl.copy_(l)
        loss, got = E.eogp_softmax_xent(dl if over else l, lab, grad_scale=SCALE, dlogits=dl)
        torch.cuda.synchronize()
        assert got is dl and not torch.isnan(loss).any()
        assert_gradient(dl, l, lab)
        left = torch.ones(buf.shape, dtype=torch.bool, device=DEV)
        torch.as_strided(left, (n, V), (ld, 1), shift).fill_(False)
        assert torch.isnan(buf[left]).all()                           # nothing beside the rows is written


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,V", [(9000, 700), (5000, 1501), (2500, 3001), (1300, 9001), (1300, 20011), (900, 40009),
                                 (600, 70001), (600, 140003)])
def test_gradient_of_rows_in_turn(n, V, dtype):
    """More rows than blocks, masked ones among them: each row's pieces are requested as the row before lets go."""
    say(f"[xent gradient] n={n} V={V} {dtype}")
    dt, g = DT[dtype], gen(51, n, V)
    l = (torch.randn((n, V), generator=torch.Generator(DEV).manual_seed(V), device=DEV) * 4 + 10).to(dt)
    mask = torch.from_numpy((g.random(n) < 0.8).astype(np.uint8)).to(DEV)
    lab = torch.from_numpy(g.integers(0, V, n)).to(DEV)
    live = mask != 0
    l[~live] = float("nan")
    for over in (False, True):
        x = l.clone()
        dl = x if over else torch.full((n, V), float("nan"), dtype=dt, device=DEV)
        E.eogp_softmax_xent(x, lab, mask, SCALE, dlogits=dl)
        torch.cuda.synchronize()
        assert not torch.any(dl[~live])
        assert_gradient(dl[live], l[live], lab[live])
