"""The example that runs the operators together, against autograd in float64 on the host."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import model_ends as M

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "block_gradients.py")


def example():
    spec = importlib.util.spec_from_file_location("block_gradients", PATH)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def reference(p, tokens, mask, labels):
    """The same block in float64 autograd; the first module's input and output are kept for their gradients."""
    q = {k: v.double().cpu().requires_grad_() for k, v in p.items()}
    tokens, live, labels = tokens.cpu(), mask.cpu().bool(), labels.cpu()
    N, T = tokens.shape
    d = q["wte"].shape[1]
    per_example = [t.detach().expand(N, 1, d).clone().requires_grad_() for t in (q["g1"], q["b1"])]
    norm = torch.nn.functional.layer_norm
    h0 = q["wte"][tokens] + q["wpe"][torch.arange(T)]
    acts = torch.cat([norm(h0, (d,)) * per_example[0] + per_example[1], torch.ones(N, T, 1, dtype=torch.float64)], 2)
    z = acts @ q["W1"].T
    z.retain_grad()
    h1 = h0 + torch.nn.functional.gelu(z) @ q["W2"].T
    logits = norm(h1, (d,), q["g2"], q["b2"]) @ q["wte"].T
    loss = torch.nn.functional.cross_entropy(logits[live], labels[live], reduction="none")
    loss.sum().backward()
    keep = live[..., None]
    return dict(acts=acts.detach() * keep, out_grads=z.grad * keep, logits=logits.detach() * keep, loss=loss.detach(),
                dwte=q["wte"].grad, dwpe=q["wpe"].grad, dg1=per_example[0].grad[:, 0], db1=per_example[1].grad[:, 0],
                dg2=q["g2"].grad, db2=q["b2"].grad, dW1=q["W1"].grad)


def test_block_gradients_match_autograd():
    """Each value passes a few dozen fp32 sums of up to 1,003 terms: relative errors (of the whole array's
    norm) of some 2^-24 sqrt(1003) each, amplified by a norm's 1 / spread of a few; 2e-5 covers them."""
    print("[block] 7 sequences of 40 positions, V = 1003, d = 70, f = 130", flush=True)
    ex = example()
    N, T, V, d, f = 7, 40, 1003, 70, 130
    p = ex.random_parameters(V, T, d, f, seed=3)
    g = torch.Generator().manual_seed(4)
    tokens = torch.randint(0, V, (N, T), generator=g).to("cuda:0")
    mask = (torch.arange(T) < torch.tensor([40, 1, 17, 0, 39, 8, 25])[:, None]).to(torch.uint8).to("cuda:0")
    u = torch.rand((N, T), generator=g).to("cuda:0")
    out = ex.forward_backward(p, tokens, mask, u, temperature=0.8, top_k=50, top_p=0.95)
    torch.cuda.synchronize()
    flat = out["logits"].reshape(N * T, V).cpu().numpy()
    want = M.sample(flat, u.reshape(-1).cpu().numpy(), 0.8, 50, 0.95, mask=mask.reshape(-1).cpu().numpy())
    assert np.array_equal(out["labels"].reshape(-1).cpu().numpy(), want)
    ref = reference(p, tokens, mask, out["labels"])
    live = mask.cpu().bool()
    assert torch.all(out["loss"].cpu()[~live] == 0) and torch.all(out["out_grads"].cpu()[~live] == 0)
    got = dict(out, loss=out["loss"].cpu()[live])
    got["dW1"] = out["out_grads"].reshape(N * T, f).T @ out["acts"].reshape(N * T, d + 1)
    for name, r in ref.items():
        err = float((got[name].double().cpu() - r).norm() / r.norm())
        assert err <= 2e-5, (name, err)
    assert torch.all(out["dg1"][3] == 0) and torch.all(out["db1"][3] == 0)          # a sequence without tokens


def test_every_sequence_finds_its_own_gradient():
    print("[block] from tokens to one-bit codes and back", flush=True)
    own, N = example().main(N=24, T=32, V=700, d=96, f=160, m=1024, k=512)
    assert own == N
