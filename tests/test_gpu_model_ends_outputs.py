"""The outputs of the operators at the ends of a model that a caller of the C ABI may leave out (NULL): the others are
what they are with them, and nothing is written in their place."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import model_ends as M
from paper_2609_37842_amd import eogp as E
from test_gpu_model_ends import DEV, dev, gen, host, near, say

pytestmark = pytest.mark.gpu


def at(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


@pytest.mark.parametrize("groups,rows,d", [(1, 700, 130), (3, 41, 1100), (5, 7, 768), (1, 300, 5000)])
def test_layer_norm_backward_without_weight_gradients(groups, rows, d):
    """dx alone, then one weight gradient alone: the same bits as with both; without either the workspace stays
    as it was."""
    say(f"[layer_norm_backward] groups={groups} rows={rows} d={d}, outputs left out")
    L, g, n = E.load(), gen(40, d), groups * rows
    x, dy = (dev(g.standard_normal((n, d))) for _ in range(2))
    gam = dev(1 + 0.1 * g.standard_normal(d))
    _, mean, rstd = E.eogp_layer_norm(x, gam)
    need = E.eogp_layer_norm_backward_workspace_size(groups, rows, d, E.F32)

    def call(dg, db):
        dx = torch.full((n, d), 7.0, device=DEV)
        ws = torch.full((need,), 77, dtype=torch.uint8, device=DEV)
        assert L.eogp_layer_norm_backward(at(dy), d, at(x), d, E.F32, at(gam), E.F32, at(mean), at(rstd), None, None, 0,
                                          groups, rows, d, at(dx), d, at(dg), at(db), at(ws), need, stream()) == 0
        torch.cuda.synchronize()
        return dx, ws

    new = lambda: torch.full((groups, d), 7.0, device=DEV)   # noqa: E731
    dg, db, dg1, db1 = new(), new(), new(), new()
    dx, _ = call(dg, db)
    alone, ws = call(None, None)
    assert torch.equal(alone, dx) and torch.all(ws == 77)
    assert torch.equal(call(dg1, None)[0], dx) and torch.equal(dg1, dg)
    assert torch.equal(call(None, db1)[0], dx) and torch.equal(db1, db)
    assert not torch.any(dg == 7.0) and not torch.any(db == 7.0)


@pytest.mark.parametrize("mean_out,rstd_out", [(False, False), (True, False), (False, True)])
def test_layer_norm_without_statistics(mean_out, rstd_out):
    say(f"[layer_norm] mean={mean_out} rstd={rstd_out}")
    L, n, d = E.load(), 70, 1030
    g = gen(41)
    x, gam = dev(g.standard_normal((n, d))), dev(1 + 0.1 * g.standard_normal(d))
    mask = dev((g.random(n) < 0.7).astype(np.uint8), torch.uint8)
    y, mean, rstd = E.eogp_layer_norm(x, gam, token_mask=mask)
    y2 = torch.full((n, d), 7.0, device=DEV)
    stats = [torch.full((n,), 7.0, device=DEV) for _ in range(2)]
    assert L.eogp_layer_norm(at(x), E.F32, d, at(gam), None, E.F32, 1e-5, at(mask), n, d, at(y2), E.F32, d, 0,
                             at(stats[0]) if mean_out else None, at(stats[1]) if rstd_out else None, stream()) == 0
    torch.cuda.synchronize()
    assert torch.equal(y, y2)
    for got, want, asked in zip(stats, (mean, rstd), (mean_out, rstd_out)):
        assert torch.equal(got, want if asked else torch.full_like(want, 7.0))


@pytest.mark.parametrize("V", [5, 700, 9001, 70001])
def test_cross_entropy_gradient_without_loss(V):
    say(f"[xent] V={V}, gradient alone")
    L, n = E.load(), 9
    g = gen(42, V)
    l = dev(g.standard_normal((n, V)) * 3)
    lab = torch.from_numpy(g.integers(-1, V, n)).to(DEV)
    mask = dev((g.random(n) < 0.7).astype(np.uint8), torch.uint8)
    _, dl = E.eogp_softmax_xent(l, lab, mask)
    got = torch.full((n, V), 7.0, device=DEV)
    assert L.eogp_softmax_xent(at(l), E.F32, V, at(lab), at(mask), n, V, 1.0, None, at(got), V, stream()) == 0
    torch.cuda.synchronize()
    assert torch.equal(got, dl)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [5, 64, 769, 1030, 4100, 9000])
def test_norm_weights_in_fp32_beside_rows_of_16_bits(d, dtype):
    """Weights that 16 bits hold give the same bits in either type; others give a backward pass within the
    roundings of the formula, of which every term is at most |dy| (|gamma| + 1) (1 + |xh|) rstd of its row."""
    say(f"[layer_norm_backward] d={d} {dtype}, fp32 weights")
    g, N, T = gen(43, d), 3, 19
    x, dy = (dev(g.standard_normal((N * T, d)) + 0.5, dtype).view(N, T, d) for _ in range(2))
    fine = dev(1 + 0.3 * g.standard_normal(d))
    coarse = fine.to(dtype)
    for per_example in (False, True):
        y, mean, rstd = E.eogp_layer_norm(x, coarse, coarse)
        y32 = E.eogp_layer_norm(x, coarse.float(), coarse.float())[0]
        assert torch.equal(y, y32)
        a = E.eogp_layer_norm_backward(dy, x, coarse, mean, rstd, per_example=per_example)
        b = E.eogp_layer_norm_backward(dy, x, coarse.float(), mean, rstd, per_example=per_example)
        c = E.eogp_layer_norm_backward(dy, x, fine, mean, rstd, per_example=per_example)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(a, b))
        assert torch.equal(a[1], c[1]) and torch.equal(a[2], c[2])    # (weight gradients do not see gamma)
    live = [host(t).reshape(N * T, -1) for t in (dy, x)]
    st = [host(t).reshape(-1) for t in (mean, rstd)]
    ref = M.layer_norm_backward(live[0], live[1], host(fine), st[0], st[1])[0]
    big = (np.abs(live[0]).max(1) * (1 + np.abs(host(fine)).max()) * 6.0 * 6.0 * st[1])[:, None]
    near(c[0].view(N * T, d), ref, 100 * 2.0 ** -24 * big, "dx")
