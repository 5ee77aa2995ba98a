"""The C ABI refuses addresses that are no multiple of their elements (no GPU): a value that a whole wave shares comes
by a scalar load, which drops an address's low bits and would read other bytes."""
import ctypes

import pytest

from paper_2609_37842_amd import eogp as E

INVALID = -1
GOOD = {
    "embed_tokens": dict(table=0x1000, tt=0, ldt=8, V=4, d=8, tokens=0x2000, mask=None, n=3, scale=1.0, acc=0,
                         out=0x3000, ot=0, ldo=8, stream=None),
    "embed_backward": dict(d_out=0x1000, t=0, ldd=8, tokens=0x2000, mask=None, n=3, V=4, d=8, scale=1.0, acc=0,
                           d_table=0x3000, ldt=8, ws=0x4000, wsb=1 << 30, stream=None),
    "layer_norm": dict(x=0x1000, xt=0, ldx=8, gamma=0x2000, beta=0x3000, wt=0, eps=1e-5, mask=None, n=3, d=8, y=0x4000,
                       yt=0, ldy=8, ones=0, mean=0x5000, rstd=0x6000, stream=None),
    "layer_norm_backward": dict(dy=0x1000, lddy=8, x=0x2000, ldx=8, t=0, gamma=0x3000, wt=0, mean=0x4000, rstd=0x5000,
                                mask=None, residual=0x6000, ldr=8, groups=2, rows=3, d=8, dx=0x7000, lddx=8,
                                d_gamma=0x8000, d_beta=0x9000, ws=0xa000, wsb=1 << 30, stream=None),
    "softmax_xent": dict(logits=0x1000, t=0, ldl=8, labels=0x2000, mask=None, n=3, V=8, scale=1.0, loss=0x3000,
                         d_logits=0x4000, ldd=8, stream=None),
    "sample_tokens": dict(logits=0x1000, t=0, ldl=8, n=3, V=8, uniforms=0x2000, mask=None, temperature=1.0, top_k=0,
                          top_p=1.0, min_p=0.0, tokens=0x3000, stream=None),
}
POINTERS = {"embed_tokens": dict(table=4, tokens=8, out=4),
            "embed_backward": dict(d_out=4, tokens=8, d_table=4, ws=4),
            "layer_norm": dict(x=4, gamma=4, beta=4, y=4, mean=4, rstd=4),
            "layer_norm_backward": dict(dy=4, x=4, gamma=4, mean=4, rstd=4, residual=4, dx=4, d_gamma=4, d_beta=4, ws=4),
            "softmax_xent": dict(logits=4, labels=8, loss=4, d_logits=4),
            "sample_tokens": dict(logits=4, uniforms=4, tokens=8)}


@pytest.mark.parametrize("call,pointer,element", [(c, p, e) for c, ps in POINTERS.items() for p, e in ps.items()])
def test_addresses_within_an_element_are_refused(call, pointer, element):
    """Every argument is refused before anything is launched: the addresses are no memory."""
    for off in (1, 2, element - 1, element // 2):
        args = dict(GOOD[call], **{pointer: GOOD[call][pointer] + off})
        got = getattr(E.load(), f"eogp_{call}")(*(ctypes.c_void_p(v) if k in POINTERS[call] else v for k, v in args.items()))
        assert got == INVALID, off
        assert f"{pointer} must be aligned".encode() in E.load().eogp_last_error()
