"""The training example: its gradients against automatic differentiation in binary64, and that it learns."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))


def test_gradients_and_clipping():
    """One worker's gradient norm is put below the limit, the others' above.  A product sums at most 96 terms in
    binary32, layer norm's sums at most 96, six such steps follow one another: (6 x 100) 2^-24 = 4e-5 of the
    gradient's norm, taken twice for the growth through layer norm's division."""
    import clipped_training as example
    model = example.Workers(seed=3)
    x, label = next(example.batches(seed=4))
    model.params += 0.1 * torch.randn(model.params.shape, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    p = {n: t.detach().double().requires_grad_() for n, t in model.p.items()}
    a = torch.bmm(x.double(), p["w1"])
    z = (a - a.mean(-1, keepdim=True)) / torch.sqrt(a.var(-1, unbiased=False, keepdim=True) + 1e-5) * p["ln_w"][:, None] + p["ln_b"][:, None]
    logits = torch.bmm(torch.relu(z), p["w2"])
    loss = torch.nn.functional.cross_entropy(logits.flatten(0, 1), label.flatten(), reduction="none").view(label.shape).mean(1)
    loss.sum().backward()
    want = torch.cat([t.grad.flatten(1) for t in p.values()], 1)
    norm = want.norm(dim=1)
    model.max_norm = float((norm.min() + norm.max()) / 2)
    got = model.gradients(x, label)
    assert torch.allclose(got.double(), loss.detach(), rtol=1e-5, atol=0)
    norms = model.ctx.liec_gather_grads(model.rows, model.max_norm)
    assert ((norms.double() - norm).abs() <= 8e-5 * norm).all()
    want *= torch.clamp(model.max_norm / norm, max=1.0)[:, None]
    assert ((model.rows.double() - want).norm(dim=1) <= 1.6e-4 * want.norm(dim=1)).all()
    assert (norms > model.max_norm).any() and (norms <= model.max_norm).any()


def test_it_learns():
    import clipped_training as example
    losses = example.main(steps=200)
    assert sum(losses[-10:]) < 0.3 * sum(losses[:10])
