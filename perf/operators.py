"""What is measured of the operators around the compressed step: layer normalisation for N local
models at once (forward, and backward with the weight's and bias's gradient reduced into the
workers' gradient rows), and the norm of every worker's gradient over all its tensors with
clipping, from gradient rows and from separate tensors.

N workers are simulated as rows, as everywhere in this package: activations are [N, rows, h], the
workers' parameters and gradients are rows of [N, d] arrays, and a layer's weight and bias are two
column ranges of those rows.
"""
import random

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
MAX_LN_ELEMENTS = 32 * 4096 * 768      # elements of x in the largest listed layer normalisation
MAX_ROW_ELEMENTS = 8 * 124_439_808     # N * d of the largest listed clipping


# ------------------------------------------------------------------------------------ tensor lists

def _resnet_sizes(blocks, widths, bottleneck):
    """Parameter tensors of a residual network (convolution weights, scale and shift of every
    normalisation, classifier) as element counts."""
    sizes, inp = [64 * 3 * 49, 64, 64], 64
    for stage, (count, w) in enumerate(zip(blocks, widths)):
        out = 4 * w if bottleneck else w
        for block in range(count):
            sizes += [w * inp, w, w, 9 * w * w, w, w, out * w, out, out] if bottleneck else [9 * w * inp, w, w, 9 * w * w, w, w]
            if block == 0 and (bottleneck or stage > 0):
                sizes += [out * inp, out, out]
            inp = out
    return sizes + [inp * 1000, 1000]


def _gpt2_small_sizes():
    h, sizes = 768, [50257 * 768, 1024 * 768]
    for _ in range(12):
        sizes += [h, h, 3 * h * h, 3 * h, h * h, h, h, h, 4 * h * h, 4 * h, 4 * h * h, h]
    return sizes + [h, h]


def _uneven_sizes(tensors, d, seed):
    """d elements cut into that many tensors, at least one element each, sizes over several magnitudes."""
    rng = np.random.default_rng(seed)
    share = np.exp(rng.normal(0.0, 2.0, tensors))
    sizes = 1 + np.floor(share / share.sum() * (d - tensors)).astype(np.int64)
    sizes[-1] += d - int(sizes.sum())
    return [int(n) for n in sizes]


def _sizes(case):
    kind = case["layout"]
    if kind == "resnet18":
        return _resnet_sizes((2, 2, 2, 2), (64, 128, 256, 512), False)
    if kind == "resnet50":
        return _resnet_sizes((3, 4, 6, 3), (64, 128, 256, 512), True)
    if kind == "gpt2_small":
        return _gpt2_small_sizes()
    return _uneven_sizes(case["tensors"], case["d"], case["layout_seed"])


# ------------------------------------------------------------------------------------ cases

def _ln(name, op, workers, rows, h, dtype, grad="f32", row_pad=0, at=0):
    return {"name": name, "op": op, "workers": workers, "rows": rows, "h": h, "dtype": dtype, "grad": grad,
            "row_pad": row_pad, "at": at}


def _clip(name, op, workers, layout, dtype, row_dtype, tensors=0, d=0, layout_seed=0):
    return {"name": name, "op": op, "workers": workers, "layout": layout, "dtype": dtype, "row_dtype": row_dtype,
            "tensors": tensors, "d": d, "layout_seed": layout_seed}


def listed():
    return [
        # a small model's layer on short micro-batches: four workers, 32 tokens each; launch latency counts
        _ln("ln-forward-small", "ln_forward", 4, 32, 256, "f32"),
        # one of the 25 layer norms of the GPT-2-small list, 32 workers with four sequences of 1024 tokens
        _ln("ln-forward-768", "ln_forward", 32, 4096, 768, "bf16"),
        # odd width, rows that are a slice of a wider buffer, weight at an odd place of the parameter row
        _ln("ln-forward-odd", "ln_forward", 8, 777, 1001, "f32", row_pad=6, at=5),
        _ln("ln-backward-small", "ln_backward", 4, 32, 256, "f32"),
        _ln("ln-backward-768", "ln_backward", 32, 4096, 768, "bf16", grad="bf16", at=768),
        # a wide layer, few workers: the weight's gradient is a sum over many rows
        _ln("ln-backward-4096", "ln_backward", 4, 4096, 4096, "bf16"),
        _ln("ln-backward-odd", "ln_backward", 3, 1501, 1333, "bf16", grad="bf16", row_pad=3, at=1),
        # one flat vector of 65,536 elements for each of four workers: the smallest configuration
        _clip("clip-flat-65536", "clip", 4, "uneven", "f32", "f32", tensors=1, d=65536),
        # the ResNet-18 list, eight workers: every row fits the L2 cache
        _clip("clip-resnet18", "clip", 8, "resnet18", "f32", "f32"),
        # the GPT-2-small list in bfloat16, eight workers: a row is larger than the L2 cache
        _clip("clip-gpt2-small", "clip", 8, "gpt2_small", "bf16", "bf16"),
        # twelve tensors of uneven, odd sizes that a backward pass left in bfloat16, rows in binary32
        _clip("gather-uneven", "gather", 4, "uneven", "bf16", "f32", tensors=12, d=70_001, layout_seed=3),
        # the ResNet-50 list as a backward pass leaves it: 161 separate tensors for each of 16 workers
        _clip("gather-resnet50", "gather", 16, "resnet50", "f32", "f32"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    dtype = rng.choice(["f32", "bf16"])
    if rng.random() < 0.5:
        op = rng.choice(["ln_forward", "ln_backward"])
        workers, h = _log_int(rng, 1, 32), _log_int(rng, 16, 8192)
        if rng.random() < 0.5:
            h = h // 8 * 8
        rows = _log_int(rng, 1, 16384)
        limit = MAX_LN_ELEMENTS // (2 if dtype == "f32" else 1)
        rows = max(1, min(rows, limit // (workers * h)))
        return _ln("", op, workers, rows, h, dtype, grad=rng.choice(["f32", "bf16"]), row_pad=rng.choice([0, 0, 0, 8, 3]),
                   at=rng.choice([0, h, 8 * rng.randrange(64), rng.randrange(512)])) | {"name": None}
    workers, tensors = _log_int(rng, 1, 32), _log_int(rng, 1, 160)
    d = _log_int(rng, 256, 1 << 27)
    row_dtype = dtype if rng.random() < 0.7 else ("f32" if dtype == "bf16" else "bf16")
    op = rng.choice(["clip", "gather"])
    if op == "clip":
        row_dtype = dtype
    limit = MAX_ROW_ELEMENTS * 4 // (SIZE[dtype] + SIZE[row_dtype])
    d = min(d, limit // workers)
    if rng.random() < 0.5:
        d = max(256, d // 8 * 8)
    return _clip("", op, workers, "uneven", dtype, row_dtype, tensors=tensors, d=d, layout_seed=rng.randrange(1 << 20)) | {"name": None}


# ------------------------------------------------------------------------------------ inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _activations(case, gen):
    """A residual stream: unit noise, a per-channel offset, a few channels far larger than the rest."""
    N, rows, h = case["workers"], case["rows"], case["h"]
    x = torch.randn(N, rows, h, generator=gen, device="cuda")
    loud = 1.0 + 19.0 * (torch.rand(h, generator=gen, device="cuda") < 0.005)
    x.mul_(loud).add_(torch.randn(h, generator=gen, device="cuda") * 0.3)
    return _padded(x.to(DTYPES[case["dtype"]]), case["row_pad"])


def _padded(t, pad):
    """The same values as a slice of a buffer whose rows are `pad` elements longer."""
    if not pad:
        return t
    wide = torch.zeros(*t.shape[:-1], t.shape[-1] + pad, dtype=t.dtype, device=t.device)
    wide[..., :t.shape[-1]] = t
    return wide[..., :t.shape[-1]]


def _prepare_ln(case, seed):
    gen = _generator(seed)
    N, h, at = case["workers"], case["h"], case["at"]
    d = (at + 2 * h + 7) // 8 * 8
    params = torch.randn(N, d, generator=gen, device="cuda") * 0.2 + 1.0
    state = {"op": case["op"], "eps": 1e-5, "x": _activations(case, gen),
             "weight": params[:, at:at + h], "bias": params[:, at + h:at + 2 * h]}
    if case["op"] == "ln_backward":
        grads = torch.zeros(N, d, dtype=DTYPES[case["grad"]], device="cuda")
        dy = torch.randn(N, case["rows"], h, generator=gen, device="cuda") * 1e-2
        mean, rstd = _statistics(state["x"], state["eps"])
        state |= {"dy": _padded(dy.to(DTYPES[case["dtype"]]), case["row_pad"]), "mean": mean, "rstd": rstd,
                  "dweight": grads[:, at:at + h], "dbias": grads[:, at + h:at + 2 * h]}
    return state


def _gradient_rows(case, gen):
    """Rows of noise with rare large entries; the workers' norms spread around the clipping norm."""
    N, d = case["workers"], sum(_sizes(case))
    rows = torch.empty(N, d, dtype=DTYPES[case["dtype"]], device="cuda")
    factors = 0.25 * 4.0 ** (2.0 * torch.rand(N, generator=gen, device="cuda"))
    for i in range(N):
        g = torch.randn(d, generator=gen, device="cuda").mul_(0.01)
        g[torch.randint(d, (1 + d // 1000,), generator=gen, device="cuda")] = 0.1
        rows[i] = g.mul_(factors[i])
    return rows, 0.011 * d ** 0.5


def _prepare_clip(case, seed):
    rows, max_norm = _gradient_rows(case, _generator(seed))
    sizes, N = _sizes(case), case["workers"]
    out = torch.empty(rows.shape, dtype=DTYPES[case["row_dtype"]], device="cuda")
    state = {"op": case["op"], "max_norm": max_norm, "out": out}
    if case["op"] == "clip":
        state["grads"] = rows
    else:   # separate tensors, as a backward pass leaves them
        state["tensors"] = [[part.clone() for part in torch.split(rows[i], sizes)] for i in range(N)]
    if own:
        from paper_2402_11857_b200 import liec
        offsets = np.concatenate([[0], np.cumsum(sizes)])
        params = torch.zeros(rows.shape, device="cuda")
        error = torch.zeros(rows.shape[1], device="cuda")
        gdt = liec.BF16 if out.dtype == torch.bfloat16 else liec.F32
        state["ctx"] = liec.Context(params, error, offsets, liec.COMP_SCALED_SIGN, liec.COMP_SCALED_SIGN, grad_dtype=gdt)
        if case["op"] == "gather":
            state["ctx"].liec_set_tensors(state["tensors"])
    return state


def prepare(case, seed):
    return _prepare_ln(case, seed) if case["op"].startswith("ln") else _prepare_clip(case, seed)


# ------------------------------------------------------------------------------------ one pass

def _statistics(x, eps):
    x = x.float()
    mean = x.mean(-1)
    var = (x - mean[..., None]).square().mean(-1)
    return mean, (var + eps).rsqrt()


def _plain_ln_forward(s):
    mean, rstd = _statistics(s["x"], s["eps"])
    xhat = (s["x"].float() - mean[..., None]) * rstd[..., None]
    return (xhat * s["weight"][:, None] + s["bias"][:, None]).to(s["x"].dtype), mean, rstd


def _plain_ln_backward(s):
    dy, mean, rstd = s["dy"].float(), s["mean"][..., None], s["rstd"][..., None]
    xhat = (s["x"].float() - mean) * rstd
    dxhat = dy * s["weight"][:, None]
    dx = (dxhat - dxhat.mean(-1, keepdim=True) - xhat * (dxhat * xhat).mean(-1, keepdim=True)) * rstd
    return dx.to(s["dy"].dtype), (dy * xhat).sum(1).to(s["dweight"].dtype), dy.sum(1).to(s["dbias"].dtype)


def _plain_clip(rows, s):
    rows = rows.float()
    norms = rows.square().sum(1).sqrt()
    factor = torch.where(norms > s["max_norm"], s["max_norm"] / norms, torch.ones_like(norms))
    return (rows * factor[:, None]).to(s["out"].dtype), norms


def run(s):
    if own:
        from paper_2402_11857_b200 import liec
        if s["op"] == "ln_forward":
            return liec.liec_layer_norm_forward(s["x"], s["weight"], s["bias"], s["eps"])
        if s["op"] == "ln_backward":
            return liec.liec_layer_norm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["weight"],
                                                 dweight=s["dweight"], dbias=s["dbias"])
        if s["op"] == "clip":
            return s["out"], s["ctx"].liec_clip_grads(s["grads"], s["max_norm"], out=s["out"])
        return s["out"], s["ctx"].liec_gather_grads(s["out"], s["max_norm"])
    if s["op"] == "ln_forward":
        return _plain_ln_forward(s)
    if s["op"] == "ln_backward":
        return _plain_ln_backward(s)
    if s["op"] == "clip":
        return _plain_clip(s["grads"], s)
    return _plain_clip(torch.cat([t for ts in s["tensors"] for t in ts]).view(s["out"].shape), s)


def work(case):
    if case["op"].startswith("ln"):
        N, rows, h = case["workers"], case["rows"], case["h"]
        e, n = SIZE[case["dtype"]], case["workers"] * case["rows"] * case["h"]
        if case["op"] == "ln_forward":     # x; y; mean and rstd; weight and bias
            return {"bytes": 2 * n * e + 8 * N * rows + 8 * N * h, "flops": 8 * n}
        return {"bytes": 3 * n * e + 8 * N * rows + N * h * (4 + 2 * SIZE[case["grad"]]), "flops": 14 * n}
    n = case["workers"] * sum(_sizes(case))
    return {"bytes": n * (SIZE[case["dtype"]] + SIZE[case["row_dtype"]]) + 4 * case["workers"], "flops": 3 * n}


# ------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    """The definitions in binary64: worker by worker, moments and sums written out."""
    if case["op"].startswith("ln"):
        s = _prepare_ln(case, seed)
        per_worker = [_exact_ln(s, i, case) for i in range(case["workers"])]
        return tuple(torch.stack(parts) for parts in zip(*per_worker))
    rows, max_norm = _gradient_rows(case, _generator(seed))
    out, norms = torch.empty(rows.shape, dtype=torch.float64, device="cuda"), []
    for i in range(case["workers"]):
        g = rows[i].double()
        norm = torch.dot(g, g).sqrt().item()
        out[i] = g * (max_norm / norm) if norm > max_norm else g
        norms.append(norm)
    return out, torch.tensor(norms, dtype=torch.float64, device="cuda")


def _exact_ln(s, i, case):
    x, w = s["x"][i].double(), s["weight"][i].double()
    h = case["h"]
    if case["op"] == "ln_forward":
        mean = x.sum(1) / h
        centred = x - mean[:, None]
        rstd = 1.0 / torch.sqrt((centred * centred).sum(1) / h + s["eps"])
        return centred * rstd[:, None] * w + s["bias"][i].double(), mean, rstd
    dy, mean, rstd = s["dy"][i].double(), s["mean"][i].double(), s["rstd"][i].double()
    xhat = (x - mean[:, None]) * rstd[:, None]
    along, level = (dy * w * xhat).sum(1) / h, (dy * w).sum(1) / h
    dx = rstd[:, None] * (dy * w - level[:, None] - xhat * along[:, None])
    return dx, (dy * xhat).sum(0), dy.sum(0)
