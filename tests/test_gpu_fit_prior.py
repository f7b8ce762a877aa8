"""The example that trains a prior on a flow's latents: it learns, one row gives what the row gives among all, and the network's gradients agree
with autograd's through plain operations as far as eight bits let them."""
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu


def test_prior_learns():
    import fit_prior
    r = fit_prior.fit(model="mini_dense", images=24, width=96, hidden=160, depth=2, steps=40, say=None)
    assert r["last"] < r["first"] - 0.02, (r["first"], r["last"])
    # other sizes take other kernels of the projections' library: equal up to the rounding of 16-bit activations
    assert (r["one_row"] - r["all_rows"][:1]).abs().max() <= 0.05 * r["all_rows"][:1].abs().max()


def test_prior_gradients():
    import fit_prior
    import torch
    gen = torch.Generator("cuda").manual_seed(3)
    prior = fit_prior.Prior(20, 12, 96, 160, 2)
    x = torch.randn((700, 20), generator=gen, device="cuda")
    dy = torch.randn((700, 24), generator=gen, device="cuda")
    params = prior.parameters()
    got = torch.autograd.grad((prior.train_pass(x) * dy).sum(), params)
    wide = [p.detach().double().requires_grad_() for p in params]
    into, out = wide[:2]
    joins = [wide[2 + 4 * k:6 + 4 * k] for k in range(3)]
    blocks = [wide[14 + 2 * k:16 + 2 * k] for k in range(2)]

    def norm(v):
        return v * torch.rsqrt((v * v).mean(1, keepdim=True) + 1e-6)

    alpha, gate, post, pre = joins[0]
    h = alpha * gate * post * norm(x.double() @ into.t())
    u = pre * norm(h)
    for (w1, w2), (alpha, gate, post, pre) in zip(blocks, joins[1:]):
        a, b = (u @ w1.t()).chunk(2, 1)
        h = h + alpha * gate * post * norm((torch.sigmoid(a) * a * b) @ w2.t())
        u = pre * norm(h)
    want = torch.autograd.grad(((u @ out.t()) * dy).sum(), wide)
    for k, (g, w) in enumerate(zip(got, want)):
        # codes are off by half a step at most, a step 1/64 to 1/127 of the largest of 32: about one percent of a value; activations and
        # their gradients in 16 bits by half a percent; three blocks deep
        size = w.norm()
        if w.numel() == 1:  # a residual scale's: the sum over columns of gate * dgate / scale, which cancels; its terms are off by as much each
            size = 3 * (wide[k + 1] * want[k + 1] / wide[k]).norm()
        assert (g.double() - w).norm() <= 0.06 * size
