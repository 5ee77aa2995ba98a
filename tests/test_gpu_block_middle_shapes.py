"""The operators in the middle of a block where their plans take other kernels than at small sizes: waves of two row groups,
two and four heads a lane, keys split over few and many blocks, masks read in parts, long sequences, mixed types."""
import numpy as np
import pytest
import torch

import test_gpu_block_middle as B
from oracle import block_middle as M
from paper_2609_37842_amd import eogp as E

pytestmark = pytest.mark.gpu
DEV, DT, U = B.DEV, B.DT, B.U
say, gen, host, dev, near = B.say, B.gen, B.host, B.dev, B.near
name = lambda c: "-".join(map(str, c))                                  # noqa: E731

# ---- attention: cases as in test_gpu_block_middle
WIDE = [                                                                # 512 blocks of 256 rows and more, heads of up to 64, 16 bits
    (64, 33, 33, 16, 8, 64, True, 0, 0, None, "some", "same", "split", 0),
    (32, 90, 150, 24, 8, 64, True, 0, 0, None, "prefix", "some", "split", 0),
    (32, 90, 150, 24, 8, 40, True, 33, 5, None, "some", "some", "gaps", 3),
    (128, 40, 70, 4, 4, 64, False, 20, 30, None, "none", "some", "heads", 0),
    (3, 300, 300, 90, 86 + 4, 56, True, 0, 0, None, "suffix", "same", "split", 0),
    (172, 260, 12, 3, 3, 64, True, 0, 0, "cache0", "all", "all", "split", 0),
]
SPLIT = [                                                               # tiled rows, keys split over 5 to 20 blocks
    (1, 200, 1500, 4, 2, 64, True, 0, 0, None, "some", "some", "split", 0),
    (1, 200, 1500, 4, 2, 128, True, 300, 40, None, "some", "some", "split", 0),
    (1, 200, 1500, 4, 2, 72, False, 0, 0, None, "all", "some", "gaps", 1),
    (1, 200, 5200, 4, 2, 64, True, 0, 0, None, "all", "some", "split", 0),   # its key mask is read in parts
    (2, 70, 5200, 2, 1, 128, True, 0, 0, "cache", "some", "some", "split", 0),
    (1, 50, 9000, 1, 1, 200, True, 6000, 3, None, "all", "some", "split", 0),
    # few rows in more than 16 splits, each width
    (1, 1, 6000, 4, 2, 64, True, 0, 0, "cache", "all", "some", "split", 0),
    (1, 3, 6000, 10, 2, 128, True, 0, 0, "cache", "all", "all", "heads", 0),
    (1, 2, 6000, 2, 1, 100, True, 5000, 4, None, "some", "some", "split", 0),
]
LONG = [
    (1, 2000, 2000, 2, 1, 64, True, 0, 0, None, "all", "all", "split", 0),
    (1, 1500, 1500, 3, 1, 128, True, 257, 4, None, "suffix", "same", "split", 0),
    (2, 700, 700, 4, 2, 128, True, 0, 0, None, "prefix", "same", "heads", 0),
    (1, 513, 1025, 2, 2, 96, False, 100, 200, None, "some", "some", "gaps", 1),
]


def attend_inputs(case, dt, g):
    """As there; "cache0" starts at position -250 and up, so that most queries come before every key."""
    start = case[9]
    q, k, v, how = B.attend_inputs(case[:9] + (None if start == "cache0" else start,) + case[10:], dt, g)
    if start == "cache0":
        how["q_start"] = np.arange(case[0]) - 250
    return q, k, v, how


def check_forward(case, dt, g, examples=None):
    N, Tq, Tk, Hq, Hkv, D, *_, layout, shift = case
    q, k, v, how = attend_inputs(case, dt, g)
    scale = 1.3 * D ** -0.5
    got, lse = E.eogp_attention(*(B.lay(x, dt, layout, shift) for x in (q, k, v)), scale, **B.device_how(how))
    torch.cuda.synchronize()
    pick = np.arange(N) if examples is None else np.sort(g.permutation(N)[:examples])
    some = {x: y if x not in ("q_start", "q_mask", "k_mask") or y is None else y[pick] for x, y in how.items()}
    ref, rlse = M.attention(q[pick], k[pick], v[pick], scale, **some)
    tol, rel = B.attend_bounds(q[pick], k[pick], v[pick], scale, dt, some)
    near(got[torch.from_numpy(pick)], ref, tol, "out")
    with np.errstate(invalid="ignore"):
        near(lse[torch.from_numpy(pick)], rlse, rel + 8 * U * (np.nan_to_num(np.abs(rlse), posinf=0) + 12), "lse")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("case", WIDE, ids=name)
def test_two_row_groups(case, dtype):
    say(f"[attention] {case} {dtype}")
    check_forward(case, DT[dtype], gen(41, *case[:6]), 24)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("case", SPLIT + LONG, ids=name)
def test_split_keys_and_long_sequences(case, dtype):
    say(f"[attention] {case} {dtype}")
    check_forward(case, DT[dtype], gen(42, *case[:6]))


@pytest.mark.parametrize("dtype,wide_out", [("f32", False), ("bf16", False), ("bf16", True), ("f16", False), ("f16", True)])
@pytest.mark.parametrize("case", LONG + [
    (3, 90, 50, 2, 1, 64, True, 10, 3, "wild", "all", "some", "split", 0),
    (2, 100, 100, 3, 3, 80, True, 17, 3, None, "suffix", "same", "split", 0),
    (4, 1, 300, 5, 1, 128, True, 0, 0, "cache", "all", "all", "split", 0),
    (2, 1, 900, 2, 1, 256, True, 100, 3, "cache", "all", "some", "split", 0),
    (1, 250, 250, 6, 2, 200, True, 0, 0, None, "some", "same", "split", 0),
], ids=name)
def test_gradients(case, dtype, wide_out):
    """wide_out: the forward pass's output is fp32 beside 16-bit inputs, so delta is no less exact."""
    dt = DT[dtype]
    N, Tq, Tk, Hq, Hkv, D, *_, layout, shift = case
    say(f"[attention_backward] {case} {dtype} fp32 out: {wide_out}")
    g = gen(43, *case[:6])
    q, k, v, how = attend_inputs(case, dt, g)
    scale = 1.3 * D ** -0.5
    dout = B.rounded(0.01 * g.standard_normal(q.shape), dt)
    if how["q_mask"] is not None:
        dout[how["q_mask"] == 0] = np.nan
    qd, kd, vd = (B.lay(x, dt, layout, shift) for x in (q, k, v))
    hd = B.device_how(how)
    out = torch.empty(q.shape, device=DEV) if wide_out else None
    out, lse = E.eogp_attention(qd, kd, vd, scale, out=out, **hd)
    dd = B.lay(dout, dt, layout, shift)
    got = E.eogp_attention_backward(dd, qd, kd, vd, out, lse, scale, **hd)
    torch.cuda.synchronize()
    ref = M.attention_backward(dout, q, k, v, scale, **how)
    for x, y, t, what in zip(got, ref, B.back_bounds(dout, q, k, v, scale, dt, how), ("dq", "dk", "dv")):
        near(x, y, t, what)
    for x, y in zip(got, E.eogp_attention_backward(dd, qd, kd, vd, out, lse, scale, **hd)):
        assert torch.equal(x, y)


# ---- rotation
ROWS = [                                                                # a row's norm in one wave: 1, 2 and 4 heads a lane, whole pieces
    (2, 9, 8, 8, 128, 128, "row", False, "some", "split", 0),
    (3, 37, 16, 16, 128, 128, "row", False, "prefix", "split", 0),
    (3, 37, 16, 4, 128, 64, "row", True, "some", "heads", 0),
    (2, 21, 32, 8, 128, 128, "row", False, "some", "split", 0),
    (2, 21, 32, 32, 128, 128, "row", True, "some", "gaps", 0),
    (2, 11, 64, 8, 128, 128, "row", True, "suffix", "split", 0),
    (2, 11, 3, 3, 64, 64, "none", False, "some", "split", 0),           # halves without a norm
    (2, 11, 4, 1, 128, 128, "none", False, "some", "heads", 0),
    (2, 11, 4, 1, 96, 48, "none", False, "some", "gaps", 1),
    (2, 11, 4, 1, 33, 20, "none", False, "some", "gaps", 1),
]


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("case", ROWS, ids=name)
def test_rows_of_one_wave(case, dtype):
    B.test_rotate_heads(case, dtype)
    for per_example in (False, True):
        B.test_rotate_heads_backward(case, per_example, dtype)


# Tokens enough for two heads a lane: (tokens, heads, key heads, D, width, norm, interleaved, dtype)
MANY = [
    (45000, 33, 3, 64, 64, "none", False, "bf16"), (45000, 33, 3, 64, 32, "none", True, "f16"),
    (45000, 33, 3, 57, 26, "none", False, "f16"), (7000, 33, 3, 64, 64, "none", False, "f32"),
    (7000, 33, 3, 63, 40, "none", True, "f32"), (17000, 9, 3, 40, 40, "head", False, "f32"),
    (17000, 9, 3, 40, 24, "head", True, "f32"), (17000, 9, 3, 39, 38, "head", False, "f32"),
    (17000, 9, 0, 40, 40, "head", False, "bf16"),
]


@pytest.mark.parametrize("case", MANY, ids=name)
def test_many_tokens(case):
    """Outputs and gradients of 300 tokens, the first and last ones among them, and the weights' gradients of all. Bounds as
    in test_gpu_block_middle; a weight's gradient is a sum of n values of any sign: fp32 partial sums of 300,000 terms in up to
    8,192 parallel chains, each below the sum of the terms' magnitudes, and n / 8,192 + 80 additions one after another."""
    n, Hq, Hk, D, width, norm, inter, dtype = case
    dt = DT[dtype]
    say(f"[rotate_heads] {case}")
    torch.manual_seed(8)
    T = 500
    N = n // T
    table = E.eogp_rotary_table(T + 7, width, magnitude=1.25)
    pos = torch.randint(0, T + 7, (N, T), device=DEV)
    mask = (torch.rand(N, T, device=DEV) < 0.9).to(torch.uint8)
    heads = [h for h in (Hq, Hk) if h]
    xs, ds = [[torch.randn(N, T, h, D, device=DEV).to(dt) for h in heads] for _ in range(2)]
    for x in xs + ds:
        x[mask == 0] = float("nan")
    ws = [None if norm == "none" else (1 + 0.3 * torch.randn(D, device=DEV)).to(dt) for _ in heads]
    how = dict(norm=norm, q_weight=ws[0], k_weight=ws[1] if Hk else None, interleaved=inter, token_mask=mask)
    two = lambda z: (z[0], z[1] if Hk else None)                        # noqa: E731
    out = E.eogp_rotate_heads(*two(xs), table, pos, **how)
    got = E.eogp_rotate_heads_backward(*two(ds), *(two(xs) if norm != "none" else (None, None)), table, pos, **how)
    torch.cuda.synchronize()
    pick = torch.cat([torch.arange(20), torch.arange(20, n - 20)[torch.randperm(n - 40)[:260]], torch.arange(n - 20, n)])
    p, m, ht = host(pos.flatten()[pick]), host(mask.flatten()[pick]), host(table)
    live = (m != 0)[:, None, None]
    for i, H in enumerate(heads):
        some = lambda t: host(t.flatten(0, 1)[pick.to(DEV)])            # noqa: E731
        x, dy, w = some(xs[i]), some(ds[i]), None if ws[i] is None else host(ws[i])
        ref = M.rotate(x, ht, p, norm, w, 1e-6, inter, m)
        big = np.abs(M.rotate(x, None, p, norm, w, 1e-6, inter, m)).max(2, keepdims=True) * 1.25 * 2
        near(out[i].flatten(0, 1)[pick.to(DEV)], ref, 32 * U * big, "qk"[i])
        ref, _ = M.rotate_backward(dy, x, ht, p, norm, w, 1e-6, inter, m)
        pair = np.nan_to_num(np.abs(dy)).max(2, keepdims=True) * 2.5
        if norm == "none":
            near(got[i].flatten(0, 1)[pick.to(DEV)], ref, 4 * U * pair, "dx")
            continue
        r, gain, size = M._stats(np.nan_to_num(x), norm, w, 1e-6)
        t, xh, ga = 2 * pair, np.abs(np.nan_to_num(x) * r), np.abs(gain)
        mean = (t * ga * xh).sum(2, keepdims=True) / size
        near(got[i].flatten(0, 1)[pick.to(DEV)], ref, r * U * (60 * t * ga + 150 * xh * mean) * live, "dx")
        # the weights' gradients in fp64 on the device, from the same formulas
        x64, d64, keep = xs[i].double(), ds[i].double(), mask.bool()[:, :, None, None]
        x64, d64 = torch.where(keep, x64, 0.0), torch.where(keep, d64, 0.0)
        c, s = (table.double()[pos][:, :, None, :, j] for j in (0, 1))
        a, b = (d64[..., 0:width:2], d64[..., 1:width:2]) if inter else (d64[..., :width // 2], d64[..., width // 2:width])
        a, b = a * c + b * s, b * c - a * s
        turned = torch.stack([a, b], -1).flatten(-2) if inter else torch.cat([a, b], -1)
        terms = torch.cat([turned, d64[..., width:]], -1) * x64 * (x64.square().mean(-1, keepdim=True) + 1e-6).rsqrt()
        near(got[2 + i], host(terms.sum((0, 1, 2))), (n * H / 8192 + 80 + 60) * U * host(terms.abs().sum((0, 1, 2))) * 2.5, "dw")


@pytest.mark.parametrize("dtype", DT)
def test_longest_rows(dtype):
    """The most heads that one norm takes, of every width: none is refused. Ones come out as 1 / (1 + eps)^1/2, with gradients
    of ones near 0: dx = rstd (1 - rstd^2)."""
    dt = DT[dtype]
    say(f"[rotate_heads] longest rows {dtype}")
    for D in range(1, 257):
        H = (2048 if D < 8 else 8192) // D
        x = torch.ones(1, 1, H, D, device=DEV, dtype=dt)
        for width in {0, D // 2 * 2, min(2, D // 2 * 2), D // 4 * 2}:
            table = torch.zeros(1, width // 2, 2, device=DEV)
            table[..., 0] = 1.0
            table = table if width else None
            y, _ = E.eogp_rotate_heads(x, None, table, norm="row", eps=1e-6)
            dx, _, dw, _ = E.eogp_rotate_heads_backward(x, None, x, None, table, norm="row", eps=1e-6)
            assert bool(((y.float() - (1 + 1e-6) ** -0.5).abs() <= B.ULP[dt] + 8 * U).all()), (D, width)
            assert bool((dx.float().abs() <= 1e-6 + 64 * U).all()) and bool(((dw - (1 + 1e-6) ** -0.5).abs() <= 64 * U).all()), (D, width)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("case", [
    (1, 3, 204, 3, 40, 40, "row", False, "some", "split", 0), (1, 3, 102, 2, 80, 80, "row", True, "some", "split", 0),
    (1, 3, 2, 170, 48, 48, "row", False, "some", "split", 0), (1, 3, 682, 1, 12, 10, "row", True, "some", "split", 0)], ids=name)
def test_rows_of_a_block(case, dtype):
    B.test_rotate_heads(case, dtype)
    B.test_rotate_heads_backward(case, False, dtype)


@pytest.mark.parametrize("dtype", DT)
@pytest.mark.parametrize("case", [                                      # up to 128 heads of any width
    (2, 5, 128, 16, 128, 128, "row", False, "some", "split", 0), (1, 4, 128, 3, 256, 256, "row", True, "all", "heads", 0),
    (2, 3, 100, 128, 250, 250, "row", False, "some", "gaps", 1), (1, 3, 128, 128, 256, 250, "row", True, "some", "split", 0),
    (2, 7, 65, 8, 128, 64, "row", False, "prefix", "split", 0), (2, 5, 120, 0, 199, 46, "row", False, "none", "gaps", 3),
    (1, 600, 128, 1, 137, 80, "row", True, "some", "split", 0)], ids=name)
def test_long_rows(case, dtype):
    """Rows that a block goes over twice: a sum's chain is 16 roundings of a lane's head, 8 heads of a lane, 22 over lanes and
    waves, within the 50 that the bounds count."""
    B.test_rotate_heads(case, dtype)
    for per_example in (False, True):
        B.test_rotate_heads_backward(case, per_example, dtype)
