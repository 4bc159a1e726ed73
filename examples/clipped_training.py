"""N workers train models of their own with layer normalisation, clipped gradients and compressed steps.

Each worker's model is a row of one parameter matrix (first layer, layer norm's weight and bias, second layer), as
the library's step wants it.  One iteration:

  forward    two batched matrix products, liec_layer_norm_forward in between on columns of the parameter rows
  backward   liec_layer_norm_backward leaves the weight's and the bias's gradients beside those of the products,
             one tensor per worker and parameter
  clipping   liec_gather_grads gathers the tensors of each worker into its gradient row and clips the row's norm
  step       liec_step compresses, exchanges and applies the rows

    python examples/clipped_training.py [steps]
"""
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
from paper_2402_11857_b200 import liec  # noqa: E402


class Workers:
    """`workers` two-layer classifiers, their gradients as separate tensors, and the compressed step over them."""

    def __init__(self, workers=4, inputs=32, hidden=96, classes=10, seed=0, max_norm=1.0, device="cuda"):
        self.max_norm = max_norm
        shapes = {"w1": (inputs, hidden), "ln_w": (hidden,), "ln_b": (hidden,), "w2": (hidden, classes)}
        off = [0]
        for s in shapes.values():
            off.append(off[-1] + torch.Size(s).numel())
        gen = torch.Generator(device=device).manual_seed(seed)
        start = torch.cat([torch.randn(inputs * hidden, generator=gen, device=device) / inputs ** 0.5,
                           torch.ones(hidden, device=device), torch.zeros(hidden, device=device),
                           torch.randn(hidden * classes, generator=gen, device=device) / hidden ** 0.5])
        self.params = start.repeat(workers, 1)                         # local models: they start equal
        self.rows = torch.empty_like(self.params)                      # gradient rows
        self.ctx = liec.Context(self.params, torch.zeros(off[-1], device=device), off, liec.COMP_SCALED_SIGN, liec.COMP_SCALED_SIGN)
        self.p = {n: self.params[:, a:b].unflatten(1, s) for (n, s), a, b in zip(shapes.items(), off, off[1:])}
        self.g = {n: torch.empty((workers,) + s, device=device) for n, s in shapes.items()}
        self.ctx.liec_set_tensors([[g[i] for g in self.g.values()] for i in range(workers)])

    def gradients(self, x, label):
        """Cross entropy of x [workers, batch, inputs] per worker; leaves its gradients in self.g."""
        p, g, batch = self.p, self.g, x.shape[1]
        a = torch.bmm(x, p["w1"])
        z, mean, rstd = liec.liec_layer_norm_forward(a, p["ln_w"], p["ln_b"])
        h = torch.relu(z)
        logp = torch.log_softmax(torch.bmm(h, p["w2"]), -1)
        loss = -logp.gather(-1, label[..., None]).mean((1, 2))
        dlogit = (logp.exp() - torch.nn.functional.one_hot(label, logp.shape[-1])) / batch
        torch.bmm(h.transpose(1, 2), dlogit, out=g["w2"])
        dz = torch.bmm(dlogit, p["w2"].transpose(1, 2)) * (z > 0)
        da, _, _ = liec.liec_layer_norm_backward(dz, a, mean, rstd, p["ln_w"], dweight=g["ln_w"], dbias=g["ln_b"])
        torch.bmm(x.transpose(1, 2), da, out=g["w1"])
        return loss

    def step(self, x, label, lr):
        loss = self.gradients(x, label)
        norms = self.ctx.liec_gather_grads(self.rows, self.max_norm)
        self.ctx.liec_step(self.rows, lr)
        return loss, norms


def batches(workers=4, batch=64, inputs=32, classes=10, seed=1, device="cuda"):
    """Endless batches: noisy points around one centre per class, each worker with classes of its own more often."""
    gen = torch.Generator(device=device).manual_seed(seed)
    centres = torch.randn(classes, inputs, generator=gen, device=device)
    taste = torch.randn(workers, classes, generator=gen, device=device).softmax(-1)
    while True:
        label = torch.multinomial(taste, batch, replacement=True, generator=gen)
        yield centres[label] + 0.5 * torch.randn(workers, batch, inputs, generator=gen, device=device), label


def main(steps=200, lr=0.05):
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
