"""N workers train convolutional models whose activations wait for the backward pass in 8 bits.

Each worker's model is a row of one parameter matrix: two 1 x 1 convolutions, each followed by group normalisation and SiLU, a
mean over the pixels and a classifier.  One iteration:

  forward    products, liec_group_norm_forward (its input's checkpoint comes out of the same read), and
             liec_activation_compress for the inputs of the convolutions; no activation itself is kept
  backward   liec_group_norm_backward from the checkpoint; liec_weight_grad from the checkpoint of a convolution's input,
             straight into the gradient rows
  step       liec_clip_grads and liec_step on the rows

    python examples/checkpointed_training.py [steps]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2402_11857_b200 import liec  # noqa: E402


class Workers:
    """`workers` small models, their gradient rows and the compressed step over them."""

    def __init__(self, workers=4, channels=24, width=64, groups=8, classes=10, seed=0, max_norm=1.0, device="cuda"):
        self.groups, self.max_norm = groups, max_norm
        shapes = {"c1": (width, channels), "w1": (width,), "b1": (width,), "c2": (width, width), "w2": (width,), "b2": (width,), "out": (classes, width)}
        off = [0]
        for s in shapes.values():
            off.append(off[-1] + torch.Size(s).numel())
        gen = torch.Generator(device=device).manual_seed(seed)
        start = torch.cat([torch.ones(s, device=device) if n.startswith("w") else torch.zeros(s, device=device) if n.startswith("b") else
                           torch.randn(s, generator=gen, device=device).flatten() / s[1] ** 0.5 for n, s in shapes.items()])
        self.params = start.repeat(workers, 1)                         # local models: they start equal
        self.rows = torch.zeros_like(self.params)                      # gradient rows
        self.ctx = liec.Context(self.params, torch.zeros(off[-1], device=device), off, liec.COMP_SCALED_SIGN, liec.COMP_SCALED_SIGN)
        self.p = {n: self.params[:, a:b].unflatten(1, s) for (n, s), a, b in zip(shapes.items(), off, off[1:])}
        self.g = {n: self.rows[:, a:b].unflatten(1, s) for (n, s), a, b in zip(shapes.items(), off, off[1:])}

    def layer(self, x, number):
        """SiLU(group norm(convolution)) of x [N, images, pixels, channels], and what its backward pass needs."""
        p, rows = self.p, x.flatten(1, 2)
        kept = liec.liec_activation_compress(rows)
        a = torch.bmm(rows, p[f"c{number}"].transpose(1, 2)).unflatten(1, x.shape[1:3])
        y, mean, rstd, q, scales = liec.liec_group_norm_forward(a, self.groups, p[f"w{number}"], p[f"b{number}"], activation="silu", compress=True)
        return y, (kept, (q, scales), mean, rstd, x.shape[-1])

    def layer_backward(self, dy, number, saved):
        """Leaves the layer's gradients in the rows; returns the gradient of its input."""
        p, g, ((xq, xs), a, mean, rstd, channels) = self.p, self.g, saved
        da, _, _ = liec.liec_group_norm_backward(dy, a, mean, rstd, p[f"w{number}"], p[f"b{number}"], activation="silu",
                                                 dweight=g[f"w{number}"], dbias=g[f"b{number}"])
        da = da.flatten(1, 2)
        liec.liec_weight_grad(da, xq, xs, channels, dweight=g[f"c{number}"])
        return torch.bmm(da, p[f"c{number}"]).unflatten(1, dy.shape[1:3])

    def gradients(self, x, label):
        """Cross entropy of x [workers, images, pixels, channels] per worker; leaves its gradients in self.rows."""
        h1, saved1 = self.layer(x, 1)
        h2, saved2 = self.layer(h1, 2)
        pooled, images, pixels = h2.mean(2), x.shape[1], x.shape[2]
        logp = torch.log_softmax(torch.bmm(pooled, self.p["out"].transpose(1, 2)), -1)
        loss = -logp.gather(-1, label[..., None]).mean((1, 2))
        dlogit = (logp.exp() - torch.nn.functional.one_hot(label, logp.shape[-1])) / images
        self.g["out"].copy_(torch.bmm(dlogit.transpose(1, 2), pooled))
        dh2 = (torch.bmm(dlogit, self.p["out"])[:, :, None] / pixels).expand_as(h2)
        self.layer_backward(self.layer_backward(dh2, 2, saved2), 1, saved1)
        return loss

    def step(self, x, label, lr):
        loss = self.gradients(x, label)
        norms = self.ctx.liec_clip_grads(self.rows, self.max_norm)
        self.ctx.liec_step(self.rows, lr)
        return loss, norms


def batches(workers=4, images=16, pixels=36, channels=24, classes=10, seed=1, device="cuda"):
    """Endless batches: noisy images around one pattern per class."""
    gen = torch.Generator(device=device).manual_seed(seed)
    patterns = torch.randn(classes, pixels, channels, generator=gen, device=device)
    while True:
        label = torch.randint(classes, (workers, images), generator=gen, device=device)
        yield patterns[label] + 0.5 * torch.randn(workers, images, pixels, channels, generator=gen, device=device), label


def main(steps=100, lr=0.05):
    model, losses = Workers(), []
    for i, (x, label) in zip(range(steps), batches()):
        loss, norms = model.step(x, label, lr)
        losses.append(float(loss.mean()))
        if i % 20 == 0 or i == steps - 1:
            print(f"step {i:4d}  loss {losses[-1]:.4f}  gradient norms {norms.min():.3f} to {norms.max():.3f}")
    status = model.ctx.liec_device_status()
    assert status == 0, f"device status {status}"
    return losses


if __name__ == "__main__":
    main(*(int(v) for v in sys.argv[1:2]))
