"""The example with activations in 8 bits: that it runs, and its gradients against the same formulas in binary64 with the
same restored activations."""
import os
import sys

import pytest
import torch

from activation_helpers import checkpoint64, slope64

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "examples"))


def restored(x):
    return torch.from_numpy(checkpoint64(x)[2].copy()).to(x.device)


def test_gradients():
    """Products of at most 64 terms forward and 576 backward, group norm's sums over 288 entries, six such steps one after
    another: (4 x 64 + 2 x 576 + 2 x 288) 2^-24 = 1.2e-4 of the gradient's norm.  The 8-bit activations are the same on both
    sides: they are made of the example's own."""
    import checkpointed_training as example
    model = example.Workers(seed=3)
    model.params += 0.05 * torch.randn(model.params.shape, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    x, label = next(example.batches(seed=4))
    loss = model.gradients(x, label)
    got = model.rows.double()
    p = {n: t.double() for n, t in model.p.items()}
    # forward in binary64, each layer's input being what the example had there
    inputs, saved = [x], []
    for k in (1, 2):
        inp = inputs[-1]
        a = torch.bmm(inp.double().flatten(1, 2), p[f"c{k}"].transpose(1, 2)).unflatten(1, inp.shape[1:3])
        own = torch.bmm(inp.flatten(1, 2), model.p[f"c{k}"].transpose(1, 2)).unflatten(1, inp.shape[1:3])
        g = a.unflatten(-1, (model.groups, -1))
        m = g.mean((2, 4), keepdim=True)
        r = 1 / torch.sqrt((g - m).square().mean((2, 4), keepdim=True) + 1e-5)
        z = ((g - m) * r).flatten(-2) * p[f"w{k}"][:, None, None] + p[f"b{k}"][:, None, None]
        saved.append((restored(inp.flatten(1, 2)), restored(own), m, r))
        inputs.append(model.layer(inp, k)[0])
    h2 = (z * torch.sigmoid(z))
    pooled = h2.mean(2)
    logp = torch.log_softmax(torch.bmm(pooled, p["out"].transpose(1, 2)), -1)
    assert torch.allclose(loss.double(), -logp.gather(-1, label[..., None]).mean((1, 2)), rtol=1e-5, atol=0)
    dlogit = (logp.exp() - torch.nn.functional.one_hot(label, 10)) / x.shape[1]
    want = {"out": torch.bmm(dlogit.transpose(1, 2), pooled)}
    d = (torch.bmm(dlogit, p["out"])[:, :, None] / x.shape[2]).expand_as(h2)
    for k in (2, 1):
        xr, ar, m, r = saved[k - 1]
        w, b = p[f"w{k}"][:, None, None], p[f"b{k}"][:, None, None]
        xh = ((ar.unflatten(-1, (model.groups, -1)) - m) * r)
        dz = d * slope64(xh.flatten(-2) * w + b, "silu")
        want[f"w{k}"], want[f"b{k}"] = (dz * xh.flatten(-2)).sum((1, 2)), dz.sum((1, 2))
        t = (dz * w).unflatten(-1, (model.groups, -1))
        da = (r * (t - t.mean((2, 4), keepdim=True) - xh * (t * xh).mean((2, 4), keepdim=True))).flatten(-2).flatten(1, 2)
        want[f"c{k}"] = torch.bmm(da.transpose(1, 2), xr)
        d = torch.bmm(da, p[f"c{k}"]).unflatten(1, x.shape[1:3])
    rows = torch.cat([want[n].flatten(1) for n in model.p], 1)
    assert ((got - rows).norm(dim=1) <= 1.2e-4 * rows.norm(dim=1)).all(), float(((got - rows).norm(dim=1) / rows.norm(dim=1)).max())
    # and the 8 bits cost little: against automatic differentiation without them
    q = {n: t.double().detach().requires_grad_() for n, t in model.p.items()}
    h = x.double()
    for k in (1, 2):
        a = torch.einsum("nspc,noc->nspo", h, q[f"c{k}"])
        g = a.unflatten(-1, (model.groups, -1))
        xh = ((g - g.mean((2, 4), keepdim=True)) / torch.sqrt(g.var((2, 4), unbiased=False, keepdim=True) + 1e-5)).flatten(-2)
        z = xh * q[f"w{k}"][:, None, None] + q[f"b{k}"][:, None, None]
        h = z * torch.sigmoid(z)
    logits = torch.bmm(h.mean(2), q["out"].transpose(1, 2))
    torch.nn.functional.cross_entropy(logits.flatten(0, 1), label.flatten(), reduction="sum").div(x.shape[1]).backward()
    full = torch.cat([q[n].grad.flatten(1) for n in model.p], 1)
    # a value is off by 2^(e-1), at most 1/254 of the largest of its 32 channels (about 2.5 of their rms): some 0.3 % rms of
    # independent noise in two factors of every layer, averaged over 576 pixels in every sum; 1 % is far more
    assert ((got - full).norm(dim=1) <= 1e-2 * full.norm(dim=1)).all()


def test_it_runs():
    import checkpointed_training as example
    losses = example.main(steps=30)
    assert len(losses) == 30 and all(v == v and v < 100 for v in losses)
