"""What is measured of the operators around activations: their checkpoints in 8 bits (compressed and
restored), group normalisation with an activation over channels-last samples of N local models
(forward, backward from the activations or from their checkpoint, and both in one step), and the
weight gradient of a linear layer from the checkpoint of its input.

N workers are simulated as rows, as everywhere in this package: activations are [N, rows, h] or
[N, samples, pixels, channels], parameters and gradients are rows of [N, d] arrays.  A checkpoint
holds every 32 consecutive channels of a row (the last block of a row is filled up with zeros) as
32 signed bytes and one power of two.
"""
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
BLOCK = 32                               # channels that share a power of two
MAX_ROW_BYTES = 2 * 32 * 4096 * 768      # bytes of x in the largest listed checkpoint
MAX_GN_BYTES = 2 * 8 * 16 * 784 * 512    # bytes of x in the largest listed group normalisation
MAX_GRAD_FLOPS = 2 * 8 * 8192 * 768 * 2304


# ------------------------------------------------------------------------------------ cases

def _checkpoint(name, workers, rows, h, dtype, row_pad=0):
    return {"name": name, "op": "checkpoint", "workers": workers, "rows": rows, "h": h, "dtype": dtype, "row_pad": row_pad}


def _gn(name, op, workers, samples, pixels, channels, groups, dtype, act, grad="f32", compressed=False, row_pad=0, at=0):
    return {"name": name, "op": op, "workers": workers, "samples": samples, "pixels": pixels, "channels": channels,
            "groups": groups, "dtype": dtype, "act": act, "grad": grad, "compressed": compressed, "row_pad": row_pad, "at": at}


def _weight_grad(name, workers, rows, h, out, dtype, grad="f32", row_pad=0, at=0):
    return {"name": name, "op": "weight_grad", "workers": workers, "rows": rows, "h": h, "out": out, "dtype": dtype,
            "grad": grad, "row_pad": row_pad, "at": at}


def listed():
    return [
        # a small model's layer on short micro-batches: four workers, 32 tokens each; launch latency counts
        _checkpoint("checkpoint-small", 4, 32, 256, "f32"),
        # the input of a GPT-2-small layer, 32 workers with four sequences of 1024 tokens
        _checkpoint("checkpoint-768", 32, 4096, 768, "bf16"),
        # odd width, rows that are a slice of a wider buffer
        _checkpoint("checkpoint-odd", 8, 777, 1001, "f32", row_pad=6),
        # an 8 x 8 feature map of a small network, two workers with four samples
        _gn("gn-forward-small", "gn_forward", 2, 4, 64, 64, 8, "f32", "silu"),
        # the first residual stage of the ResNet lists: 56 x 56 pixels of 64 channels, eight workers, 32 images each
        _gn("gn-forward-56", "gn_forward", 8, 32, 3136, 64, 32, "bf16", "relu"),
        # a bottleneck's last normalisation at 28 x 28 with 512 channels, from the checkpoint the forward pass left
        _gn("gn-backward-28", "gn_backward", 8, 16, 784, 512, 32, "bf16", "silu", compressed=True, at=512),
        # channels that are no multiple of anything, 19 x 19 pixels, a slice of a wider buffer, from the activations
        _gn("gn-backward-odd", "gn_backward", 3, 5, 361, 150, 5, "f32", "relu", grad="bf16", row_pad=3, at=1),
        # one model on images of 256 x 256: samples far larger than an SM's memory; forward and backward
        _gn("gn-step-256", "gn_step", 1, 4, 65536, 128, 32, "bf16", "silu", compressed=True),
        # a small model's linear layer, four workers, 32 tokens each
        _weight_grad("weight-grad-small", 4, 32, 256, 256, "f32"),
        # the widest product of a GPT-2-small attention block (768 to three times 768), eight workers, 8192 tokens each
        _weight_grad("weight-grad-768", 8, 8192, 768, 2304, "bf16"),
        # a ResNet-50 bottleneck's 1 x 1 convolution at 7 x 7 pixels, 512 to 2048 channels, 16 workers, 64 images each
        _weight_grad("weight-grad-conv", 16, 3136, 512, 2048, "bf16", grad="bf16", at=64),
        # odd tokens, inputs and outputs, a slice of a wider buffer, gradients in bfloat16
        _weight_grad("weight-grad-odd", 3, 1501, 1333, 515, "bf16", grad="bf16", row_pad=3, at=1),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def _maybe_round(rng, n):
    return n if rng.random() < 0.5 else max(32, n // 32 * 32)


def draw(rng):
    dtype, grad = rng.choice(["f32", "bf16"]), rng.choice(["f32", "bf16"])
    row_pad, at = rng.choice([0, 0, 0, 8, 3]), rng.choice([0, 8 * rng.randrange(64), rng.randrange(512)])
    op = rng.choice(["checkpoint", "gn_forward", "gn_backward", "gn_step", "weight_grad", "weight_grad"])
    if op == "checkpoint":
        workers, h = _log_int(rng, 1, 32), _maybe_round(rng, _log_int(rng, 1, 8192))
        rows = max(1, min(_log_int(rng, 1, 16384), MAX_ROW_BYTES // (workers * h * SIZE[dtype])))
        return _checkpoint(None, workers, rows, h, dtype, row_pad)
    if op == "weight_grad":
        workers, rows = _log_int(rng, 1, 16), _log_int(rng, 1, 16384)
        h, out = _maybe_round(rng, _log_int(rng, 1, 4096)), _maybe_round(rng, _log_int(rng, 1, 4096))
        rows = max(1, min(rows, MAX_GRAD_FLOPS // (2 * workers * h * out), MAX_ROW_BYTES // (workers * max(h, out) * 4)))
        return _weight_grad(None, workers, rows, h, out, dtype, grad, row_pad, at)
    groups, width = _log_int(rng, 1, 64), _log_int(rng, 1, 64)
    if rng.random() < 0.5:
        groups, width = rng.choice([1, 8, 32]), rng.choice([2, 4, 8, 16])
    workers, samples, pixels = _log_int(rng, 1, 32), _log_int(rng, 1, 64), _log_int(rng, 1, 65536)
    limit = max(1, MAX_GN_BYTES // (4 * groups * width))
    workers = min(workers, limit)
    samples = max(1, min(samples, limit // workers))
    pixels = max(1, min(pixels, limit // (workers * samples)))
    act = rng.choice(["none", "relu", "silu"]) if op != "gn_step" else rng.choice(["none", "silu"])
    compressed = op == "gn_step" or (op == "gn_backward" and rng.random() < 0.5)
    return _gn(None, op, workers, samples, pixels, groups * width, groups, dtype, act, grad, compressed, row_pad, at)


# ------------------------------------------------------------------------------------ inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _activations(shape, dtype, row_pad, gen):
    """A residual stream: unit noise, a per-channel offset, a few channels far larger than the rest."""
    h = shape[-1]
    x = torch.randn(shape, generator=gen, device="cuda")
    loud = 1.0 + 19.0 * (torch.rand(h, generator=gen, device="cuda") < 0.005)
    x.mul_(loud).add_(torch.randn(h, generator=gen, device="cuda") * 0.3)
    return _padded(x.to(DTYPES[dtype]), row_pad)


def _padded(t, pad):
    """The same values as a slice of a buffer whose rows are `pad` elements longer."""
    if not pad:
        return t
    wide = torch.zeros(*t.shape[:-1], t.shape[-1] + pad, dtype=t.dtype, device=t.device)
    wide[..., :t.shape[-1]] = t
    return wide[..., :t.shape[-1]]


def _prepare_gn(case, seed):
    gen = _generator(seed)
    N, C, at, dtype = case["workers"], case["channels"], case["at"], case["dtype"]
    shape = (N, case["samples"], case["pixels"], C)
    d = (at + 2 * C + 7) // 8 * 8
    params = torch.randn(N, d, generator=gen, device="cuda") * 0.2
    params[:, at:at + C] += 1.0
    state = {"op": case["op"], "eps": 1e-5, "groups": case["groups"], "act": case["act"], "compressed": case["compressed"],
             "x": _activations(shape, dtype, case["row_pad"], gen),
             "weight": params[:, at:at + C], "bias": params[:, at + C:at + 2 * C]}
    if case["op"] != "gn_forward":
        grads = torch.zeros(N, d, dtype=DTYPES[case["grad"]], device="cuda")
        dy = torch.randn(shape, generator=gen, device="cuda") * 1e-2
        state |= {"dy": _padded(dy.to(DTYPES[dtype]), case["row_pad"]),
                  "dweight": grads[:, at:at + C], "dbias": grads[:, at + C:at + 2 * C]}
    if case["op"] == "gn_backward":   # what the forward pass left
        state["mean"], state["rstd"] = _statistics(state["x"], case["groups"], state["eps"])
        if case["compressed"]:
            state["q"], state["scales"] = _compress(state.pop("x"))
    return state


def prepare(case, seed):
    if case["op"].startswith("gn"):
        return _prepare_gn(case, seed)
    gen = _generator(seed)
    N, rows, h = case["workers"], case["rows"], case["h"]
    x = _activations((N, rows, h), case["dtype"], case["row_pad"], gen)
    if case["op"] == "checkpoint":
        return {"op": "checkpoint", "x": x}
    out, at = case["out"], case["at"]
    grads = torch.zeros(N, (at + out * h + 7) // 8 * 8, dtype=DTYPES[case["grad"]], device="cuda")
    dy = torch.randn(N, rows, out, generator=gen, device="cuda") * 1e-2
    q, scales = _compress(x)
    return {"op": "weight_grad", "dy": _padded(dy.to(DTYPES[case["dtype"]]), case["row_pad"]), "q": q, "scales": scales, "h": h,
            "dweight": grads[:, at:at + out * h].unflatten(1, (out, h))}


# ------------------------------------------------------------------------------------ one pass

def _power(exponent):
    """2^exponent in binary32 for exponents from -126 to 127."""
    return ((exponent + 127) << 23).view(torch.float32)


def _compress(x):
    """Signed bytes [..., 32 ceil(h/32)] and the powers' biased exponents [..., ceil(h/32)]."""
    h = x.shape[-1]
    blocks = torch.nn.functional.pad(x.float(), (0, -h % BLOCK)).unflatten(-1, (-1, BLOCK))
    top = blocks.abs().amax(-1)
    part, exponent = torch.frexp(top)
    exponent = torch.where(part * 128 < 127.5, exponent - 7, exponent - 6).clamp(min=-126)
    exponent = torch.where(top == 0, -126, exponent)
    finite = torch.isfinite(top)
    exponent = torch.where(finite, exponent, 0).int()
    q = torch.where(finite[..., None], torch.round(blocks * _power(-exponent)[..., None]), 0).to(torch.int8)
    return q.flatten(-2), torch.where(finite, exponent + 127, 255).to(torch.uint8)


def _restore(q, scales, h):
    power = (scales.int() << 23).view(torch.float32)
    return (q.unflatten(-1, (-1, BLOCK)).float() * power[..., None]).flatten(-2)[..., :h]


def _grouped(t, groups):
    return t.unflatten(-1, (groups, -1))


def _statistics(x, groups, eps):
    x = _grouped(x.float(), groups)
    mean = x.mean((2, 4))
    var = (x - mean[:, :, None, :, None]).square().mean((2, 4))
    return mean, (var + eps).rsqrt()


def _per_channel(worker_vector, groups):
    return _grouped(worker_vector, groups)[:, None, None]


def _plain_gn_forward(s):
    mean, rstd = _statistics(s["x"], s["groups"], s["eps"])
    xhat = (_grouped(s["x"].float(), s["groups"]) - mean[:, :, None, :, None]) * rstd[:, :, None, :, None]
    z = xhat * _per_channel(s["weight"], s["groups"]) + _per_channel(s["bias"], s["groups"])
    y = z.clamp(min=0) if s["act"] == "relu" else z / (1 + torch.exp(-z)) if s["act"] == "silu" else z
    return y.flatten(-2).to(s["x"].dtype), mean, rstd


def _plain_gn_backward(s, x, mean, rstd):
    G = s["groups"]
    x, dz, mean, rstd = _grouped(x.float(), G), _grouped(s["dy"].float(), G), mean[:, :, None, :, None], rstd[:, :, None, :, None]
    w, b = _per_channel(s["weight"], G), _per_channel(s["bias"], G)
    xhat = (x - mean) * rstd
    if s["act"] == "relu":   # on which side of zero: 64 bits
        dz = dz * ((x.double() - mean.double()) * rstd.double() * w.double() + b.double() > 0)
    elif s["act"] == "silu":
        z = xhat * w + b
        gate = 1 / (1 + torch.exp(-z))
        dz = dz * (gate * (1 + z * (1 - gate)))
    dxhat = dz * w
    dx = (dxhat - dxhat.mean((2, 4), keepdim=True) - xhat * (dxhat * xhat).mean((2, 4), keepdim=True)) * rstd
    grad = s["dweight"].dtype
    return dx.flatten(-2).to(s["dy"].dtype), (dz * xhat).sum((1, 2)).flatten(-2).to(grad), dz.sum((1, 2)).flatten(-2).to(grad)


def _plain(s):
    if s["op"] == "checkpoint":
        return _restore(*_compress(s["x"]), s["x"].shape[-1]).to(s["x"].dtype)
    if s["op"] == "gn_forward":
        return _plain_gn_forward(s)
    if s["op"] == "gn_backward":
        x = _restore(s["q"], s["scales"], s["dy"].shape[-1]) if s["compressed"] else s["x"]
        return _plain_gn_backward(s, x, s["mean"], s["rstd"])
    if s["op"] == "gn_step":
        forward = _plain_gn_forward(s)
        return forward + _plain_gn_backward(s, _restore(*_compress(s["x"]), s["x"].shape[-1]), *forward[1:])
    return torch.bmm(s["dy"].float().transpose(1, 2), _restore(s["q"], s["scales"], s["h"])).to(s["dweight"].dtype)


def run(s):
    if not own:
        return _plain(s)
    from paper_2402_11857_b200 import liec
    if s["op"] == "checkpoint":   # what the backward pass gets back
        q, scales = liec.liec_activation_compress(s["x"])
        return liec.liec_activation_restore(q, scales, s["x"].shape[-1], dtype=s["x"].dtype)
    if s["op"] == "gn_forward":
        return liec.liec_group_norm_forward(s["x"], s["groups"], s["weight"], s["bias"], s["eps"], activation=s["act"])
    if s["op"] == "gn_backward":
        x = (s["q"], s["scales"]) if s["compressed"] else s["x"]
        return liec.liec_group_norm_backward(s["dy"], x, s["mean"], s["rstd"], s["weight"], s["bias"], activation=s["act"],
                                             dweight=s["dweight"], dbias=s["dbias"])
    if s["op"] == "gn_step":
        y, mean, rstd, q, scales = liec.liec_group_norm_forward(s["x"], s["groups"], s["weight"], s["bias"], s["eps"],
                                                                activation=s["act"], compress=True)
        return (y, mean, rstd) + liec.liec_group_norm_backward(s["dy"], (q, scales), mean, rstd, s["weight"], s["bias"],
                                                               activation=s["act"], dweight=s["dweight"], dbias=s["dbias"])
    return liec.liec_weight_grad(s["dy"], s["q"], s["scales"], s["h"], dweight=s["dweight"])


def work(case):
    N, e = case["workers"], SIZE[case["dtype"]]
    if case["op"] == "checkpoint":   # x; bytes and powers written and read; x restored
        rows, h = N * case["rows"], case["h"]
        return {"bytes": rows * (2 * h * e + 2 * (h + -(-h // BLOCK))), "flops": 4 * rows * h}
    if case["op"] == "weight_grad":  # dy; bytes and powers; the gradient
        rows, h, out = N * case["rows"], case["h"], case["out"]
        return {"bytes": rows * (out * e + h + -(-h // BLOCK)) + N * out * h * SIZE[case["grad"]], "flops": 2 * rows * h * out}
    C, images = case["channels"], N * case["samples"]
    pixels = images * case["pixels"]
    held, statistics, weights = pixels * (C + -(-C // BLOCK)), 8 * images * case["groups"], 8 * N * C
    forward, backward = 2 * pixels * C * e + statistics + weights, 2 * pixels * C * e + 2 * N * C * SIZE[case["grad"]]
    if case["op"] == "gn_forward":
        return {"bytes": forward, "flops": 12 * pixels * C}
    if case["op"] == "gn_backward":
        return {"bytes": backward + statistics + weights + (held if case["compressed"] else pixels * C * e), "flops": 24 * pixels * C}
    return {"bytes": forward + backward + 2 * held, "flops": 40 * pixels * C}


# ------------------------------------------------------------------------------------ 64 bits

def _exact_restored(x):
    """x^ = q 2^e of every block: e the least exponent from -126 on for which all |q| are at most 127."""
    h = x.shape[-1]
    wide = torch.zeros(*x.shape[:-1], -(-h // BLOCK) * BLOCK, dtype=torch.float64, device=x.device)
    wide[..., :h] = x
    blocks = wide.view(*x.shape[:-1], -1, BLOCK)
    top = blocks.abs().max(-1, keepdim=True).values
    exponent = torch.frexp(top)[1].long() - 8
    for _ in range(3):
        exponent = torch.where((top * _power64(-exponent)).round() > 127, exponent + 1, exponent)
    exponent = torch.where(top > 0, exponent, -126).clamp(min=-126)
    return ((blocks * _power64(-exponent)).round() * _power64(exponent)).view(wide.shape)[..., :h]


def _power64(exponent):
    return ((exponent + 1023) << 52).view(torch.float64)


def _exact_gn_forward(x, w, b, groups, eps, act):
    """One worker: x [samples, pixels, channels]."""
    B, P, C = x.shape
    n = P * (C // groups)
    g = x.view(B, P, groups, C // groups)
    mean = g.sum(3).sum(1) / n
    centred = g - mean[:, None, :, None]
    rstd = 1.0 / torch.sqrt((centred * centred).sum(3).sum(1) / n + eps)
    z = (centred * rstd[:, None, :, None]).view(B, P, C) * w + b
    y = torch.maximum(z, torch.zeros_like(z)) if act == "relu" else z * torch.special.expit(z) if act == "silu" else z
    return y, mean, rstd


def _exact_gn_backward(dy, x, mean, rstd, w, b, groups, act):
    B, P, C = x.shape
    n = P * (C // groups)
    xhat = ((x.view(B, P, groups, -1) - mean[:, None, :, None]) * rstd[:, None, :, None]).view(B, P, C)
    z = xhat * w + b
    if act == "relu":
        dy = torch.where(z > 0, dy, torch.zeros_like(dy))
    elif act == "silu":
        s = torch.special.expit(z)
        dy = dy * (s + z * s * torch.special.expit(-z))
    level = (dy * w).view(B, P, groups, -1).sum(3).sum(1) / n
    along = (dy * w * xhat).view(B, P, groups, -1).sum(3).sum(1) / n
    inner = (dy * w).view(B, P, groups, -1) - level[:, None, :, None] - xhat.view(B, P, groups, -1) * along[:, None, :, None]
    return (inner * rstd[:, None, :, None]).view(B, P, C), (dy * xhat).sum((0, 1)), dy.sum((0, 1))


def exact(case, seed):
    """The definitions in binary64, worker by worker."""
    s = prepare(case, seed)
    per_worker = [_exact_worker(s, i) for i in range(case["workers"])]
    parts = tuple(torch.stack(p) for p in zip(*per_worker))
    return parts if len(parts) > 1 else parts[0]


def _exact_worker(s, i):
    if s["op"] == "checkpoint":
        return (_exact_restored(s["x"][i].double()),)
    if "q" in s:   # the bytes times their powers
        q, exponent = s["q"][i].double(), s["scales"][i].long() - 127
        restored = q * _power64(exponent).repeat_interleave(BLOCK, -1)
    if s["op"] == "weight_grad":
        return (s["dy"][i].double().t() @ restored[:, :s["h"]],)
    w, b, groups, act = s["weight"][i].double(), s["bias"][i].double(), s["groups"], s["act"]
    if s["op"] == "gn_backward":
        x = restored[..., :w.numel()].contiguous() if "q" in s else s["x"][i].double().contiguous()
        return _exact_gn_backward(s["dy"][i].double(), x, s["mean"][i].double(), s["rstd"][i].double(), w, b, groups, act)
    x = s["x"][i].double().contiguous()
    forward = _exact_gn_forward(x, w, b, groups, s["eps"], act)
    if s["op"] == "gn_forward":
        return forward
    return forward + _exact_gn_backward(s["dy"][i].double(), _exact_restored(x).contiguous(), *forward[1:], w, b, groups, act)
