"""One feed-forward block of a language model from token ids to one-bit gradient codes.

The forward pass embeds tokens and positions, normalises (writing the column of ones that stands for the
bias of the next linear module), applies a linear / GELU / linear block on a residual stream, normalises
again and multiplies with the token table. Labels are drawn from the model's own distribution (true-Fisher
labels) or given; the backward pass leaves the inputs and output gradients of the block's first linear
module in the layout the compression path takes, and every weight gradient of the operators, those of the
first norm per example. The module's gradients are then rotated, retained, projected and packed to one bit,
and each sequence's own code has to be the best match of its gradient.

    python examples/block_gradients.py
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2609_37842_amd import eogp as E  # noqa: E402


def random_parameters(V, T, d, f, seed=0, device="cuda:0"):
    """Token and position tables, two norms' weights, W1 [f, d + 1] (its last column the bias), W2 [d, f]."""
    g = torch.Generator().manual_seed(seed)
    r = lambda *shape, scale: (torch.randn(*shape, generator=g) * scale).to(device)   # noqa: E731
    return dict(wte=r(V, d, scale=0.02), wpe=r(T, d, scale=0.01), g1=1 + r(d, scale=0.1), b1=r(d, scale=0.1),
                g2=1 + r(d, scale=0.1), b2=r(d, scale=0.1), W1=r(f, d + 1, scale=d ** -0.5),
                W2=r(d, f, scale=0.02))


def forward_backward(p, tokens, mask, uniforms=None, labels=None, **sampling):
    """Loss and gradients of the block for tokens [N, T] and token mask uint8 [N, T]; labels int64 [N, T], or
    drawn with `uniforms` [N, T]. Returns a dict; acts [N, T, d + 1] and out_grads [N, T, f] are the
    first linear module's."""
    N, T = tokens.shape
    V, d = p["wte"].shape
    flat = lambda t: t.reshape(N * T, t.shape[-1])                                     # noqa: E731
    positions = torch.arange(T, device=tokens.device).expand(N, T).contiguous()
    h0 = E.eogp_embed_tokens(p["wte"], tokens, token_mask=mask)
    E.eogp_embed_tokens(p["wpe"], positions, token_mask=mask, out=h0, accumulate=True)
    acts, m1, r1 = E.eogp_layer_norm(h0, p["g1"], p["b1"], token_mask=mask, ones_column=True)
    z = flat(acts) @ p["W1"].T
    a = torch.nn.functional.gelu(z)
    h1 = h0 + (a @ p["W2"].T).view(N, T, d)
    hf, m2, r2 = E.eogp_layer_norm(h1, p["g2"], p["b2"], token_mask=mask)
    logits = (flat(hf) @ p["wte"].T).view(N, T, V)
    if labels is None:
        labels = E.eogp_sample_tokens(logits, uniforms, token_mask=mask, **sampling)
    loss, dlogits = E.eogp_softmax_xent(logits, labels, mask)
    dhf = (flat(dlogits) @ p["wte"]).view(N, T, d)
    dh1, dg2, db2 = E.eogp_layer_norm_backward(dhf, h1, p["g2"], m2, r2, mask)
    out_grads = torch.ops.aten.gelu_backward(flat(dh1) @ p["W2"], z)
    dacts = (out_grads @ p["W1"][:, :d]).view(N, T, d)
    # the residual stream's gradient is added where the norm's is written
    dh0, dg1, db1 = E.eogp_layer_norm_backward(dacts, h0, p["g1"], m1, r1, mask, residual=dh1, per_example=True)
    dwte = flat(dlogits).T @ flat(hf)                                                  # the head's share
    E.eogp_embed_backward(dh0, tokens, V, token_mask=mask, dtable=dwte, accumulate=True)
    dwpe = E.eogp_embed_backward(dh0, positions, T, token_mask=mask)
    return dict(logits=logits, labels=labels, loss=loss, acts=acts, out_grads=out_grads.view(N, T, -1), dwte=dwte,
                dwpe=dwpe, dg1=dg1, db1=db1, dg2=dg2, db2=db2)


def compress(acts, out_grads, mask, m, k, seed=1):
    """(codes, scales, X) of the module's per-example gradients: eigenbases of the two token covariances,
    corrected eigenvalues, m retained coordinates, k of a randomised Hadamard transform, one bit each."""
    d_in, d_out = acts.shape[2], out_grads.shape[2]
    basis = lambda t: torch.linalg.eigh((t.T @ t).double().cpu())[1].float().contiguous().to(t.device)  # noqa: E731
    QA, QS = basis(acts.reshape(-1, d_in)), basis(out_grads.reshape(-1, d_out))
    eig = E.eogp_ekfac_eigenvalues(acts, out_grads, mask, QA, QS) / acts.shape[0]
    plan = E.eogp_plan_create(eig, 0.1 * float(eig.mean()), m, QA, QS)
    Z = E.eogp_rotate_retain_planned(plan, acts, out_grads, mask, prec=E.PREC_ACCURATE)
    plan.close()
    g = torch.Generator().manual_seed(seed)
    signs = (torch.randint(0, 2, (m,), generator=g) * 2 - 1).to(torch.int8).to(acts.device)
    rows = torch.randperm(1 << (m - 1).bit_length(), generator=g)[:k].to(torch.int32).to(acts.device)
    X = E.eogp_srht_project(Z, signs, rows)
    return (*E.eogp_sign_pack(X), X)


def main(N=64, T=96, V=5003, d=192, f=768, m=4096, k=1024):
    p = random_parameters(V, T, d, f)
    g = torch.Generator().manual_seed(2)
    tokens = torch.randint(0, V, (N, T), generator=g).to("cuda:0")
    lengths = torch.randint(T // 2, T + 1, (N, 1), generator=g)
    mask = (torch.arange(T) < lengths).to(torch.uint8).to("cuda:0")
    uniforms = torch.rand((N, T), generator=g).to("cuda:0")
    out = forward_backward(p, tokens, mask, uniforms)
    codes, scales, X = compress(out["acts"], out["out_grads"], mask, m, k)
    best = E.eogp_score_topk(codes, scales, [k], X, 1)[0][:, 0]
    own = int((best.cpu() == torch.arange(N)).sum())
    print(f"{int(mask.sum())} tokens of {N} sequences: mean loss {float(out['loss'].sum() / mask.sum()):.4f} "
          f"(ln V = {torch.tensor(float(V)).log():.4f}); {own} of {N} sequences are the best match of their own gradient")
    return own, N


if __name__ == "__main__":
    own, N = main()
    sys.exit(0 if own == N else 1)
