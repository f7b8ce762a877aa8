"""The example's prior with a table of values for each channel and orthogonalised updates: it runs, one row gives what the row gives among all, and the
gradients of its loss agree with autograd's through plain operations as far as eight bits let them."""
import math
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("loss,optimiser", [("classes", "muon"), ("classes", "adam"), ("logistic", "muon")])
def test_prior_runs(loss, optimiser):
    import fit_prior
    r = fit_prior.fit(model="mini_dense", images=8, width=96, hidden=160, depth=2, steps=3, say=None, loss=loss, optimiser=optimiser)
    assert math.isfinite(r["first"]) and math.isfinite(r["last"]) and r["last"] != r["first"]
    assert all(p.isfinite().all() for p in r["prior"].parameters())
    # other sizes take other kernels: equal up to the rounding of 16-bit activations
    assert (r["one_row"] - r["all_rows"][:1]).abs().max() <= 0.05 * r["all_rows"][:1].abs().max()


def test_prior_gradients():
    import fit_prior
    import torch
    gen = torch.Generator("cuda").manual_seed(4)
    prior = fit_prior.Prior(20, 3, 96, 160, 1, values=50)
    x = torch.randn((700, 20), generator=gen, device="cuda")
    value = torch.randint(0, 50, (700, 3), generator=gen, device="cuda")
    params = [p for p in prior.parameters() if p is not prior.out]
    got = torch.autograd.grad(prior.train_bits(x, value), params)
    wide = [p.detach().double().requires_grad_() for p in params]
    into, first, second, w1, w2, tables = wide[0], wide[1:5], wide[5:9], wide[9], wide[10], wide[11:]

    def norm(v):
        return v * torch.rsqrt((v * v).mean(1, keepdim=True) + 1e-6)

    h = first[0] * first[1] * first[2] * norm(x.double() @ into.t())
    a, b = (first[3] * norm(h) @ w1.t()).chunk(2, 1)
    h = h + second[0] * second[1] * second[2] * norm((torch.sigmoid(a) * a * b) @ w2.t())
    u = second[3] * norm(h)
    total = 0
    for t, v in zip(tables, value.t()):
        s = u @ t.t()
        total = total + (torch.logsumexp(s, 1) - s.gather(1, v[:, None])[:, 0]).mean()
    want = torch.autograd.grad(total / (3 * math.log(2.0)), wide)
    for k, (g, w) in enumerate(zip(got, want)):
        # codes are off by half a step at most, a step 1/64 to 1/127 of the largest of 32: about one percent of a value; activations and their gradients in 16
        # bits by half a percent; two blocks deep. A residual scale's gradient is a sum over columns that cancels: its terms are off by as much each
        size = w.norm() if w.numel() > 1 else 3 * (wide[k + 1] * want[k + 1] / wide[k]).norm()
        assert (g.double() - w).norm() <= 0.06 * size, k
