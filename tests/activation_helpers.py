"""Definitions in binary64 of the operators on activations, and error bounds of their binary32 evaluation.

u = 2^-24 is one rounding to binary32, 2^-8 one to bfloat16.  K counts the additions that a term passes through: at most
rows/4 in one thread, 64 where threads meet, a few joins in binary64.
"""
import numpy as np
import torch

U, U_BF = 2.0 ** -24, 2.0 ** -8
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def checkpoint64(x):
    """(q, scale bytes, x^) of [..., h], with numpy on the host, block by block as defined."""
    x = x.detach().float().cpu().numpy().astype(np.float64)
    h = x.shape[-1]
    wide = np.zeros(x.shape[:-1] + (-(-h // 32) * 32,))
    wide[..., :h] = x
    b = wide.reshape(x.shape[:-1] + (-1, 32))
    top = np.abs(b).max(-1)
    bad = ~np.isfinite(top)
    safe = np.where(bad | (top == 0), 1.0, top)
    e = np.floor(np.log2(safe)).astype(np.int64) - 7
    for _ in range(3):
        e = np.where(np.rint(np.ldexp(safe, -e)) > 127, e + 1, e)
    e = np.where(top == 0, -126, np.clip(e, -126, 121))
    with np.errstate(invalid="ignore"):
        q = np.where(bad[..., None], 0.0, np.clip(np.rint(np.ldexp(np.where(bad[..., None], 0.0, b), -e[..., None])), -127, 127))
    back = np.where(bad[..., None], np.nan, np.ldexp(q, e[..., None])).reshape(wide.shape)[..., :h]
    return q.astype(np.int8).reshape(wide.shape), np.where(bad, 255, e + 127).astype(np.uint8), back


def restored64(q, scales, h):
    power = torch.ldexp(torch.ones(scales.shape, dtype=torch.float64), scales.cpu().int() - 127).to(q.device)
    return (q.double().unflatten(-1, (-1, 32)) * power[..., None]).flatten(-2)[..., :h]


def check(got, want, bound, what):
    got = got.double()
    bad = ~((got - want).abs() <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} outside, worst {float(((got - want).abs() / bound).max()):.2f} of the bound"


def out_bound(t, dtype):
    return (U_BF if dtype == "bf16" else U) * t.abs() + 1e-37


def act64(z, act):
    return z.clamp(min=0) if act == "relu" else z * torch.sigmoid(z) if act == "silu" else z


def slope64(z, act):
    s = torch.sigmoid(z)
    return (z > 0).double() if act == "relu" else s * (1 + z * (1 - s)) if act == "silu" else torch.ones_like(z)


def _grouped(t, groups):
    return t.unflatten(-1, (groups, -1))


def _spread(t, width):
    """[N, samples, groups] -> [N, samples, 1, channels]"""
    return t.repeat_interleave(width, -1)[:, :, None]


def _over_group(t, groups, f):
    """f over the pixels and channels of every group of [N, samples, pixels, channels], spread back to channels."""
    g = _grouped(t, groups)
    v = g.amax((2, 4)) if f == "max" else g.mean((2, 4))
    return v, _spread(v, t.shape[-1] // groups)


def check_group_norm_forward(x, w, b, groups, eps, act, dtype, y, mean, rstd):
    """x [N, samples, pixels, C]; w, b [N, C]."""
    x, w, b = x.double(), w.double()[:, None, None], b.double()[:, None, None]
    width, K = x.shape[-1] // groups, 80 + x.shape[2] / 4
    m, mc = _over_group(x, groups, "mean")
    v, vc = _over_group((x - mc).square(), groups, "mean")
    D, Dc = _over_group((x - mc).abs(), groups, "max")
    r = 1 / torch.sqrt(v + eps)
    # sums around a value of the channel, at most D from the mean; the part's mean is rounded once more
    dm = (K + 4) * U * 2 * D + 3 * U * m.abs()
    dv = 3 * (K + 6) * U * (v + 4 * D * D) + 2 * dm * dm
    rel = dv / (v + eps) / 2 + 3 * U
    check(mean, m, dm + 1e-37, "mean")
    check(rstd, r, rel * r, "rstd")
    rc, dmc, relc = (_spread(t, width) for t in (r, dm, rel))
    xw = (x - mc) * rc * w
    dz = rc * w.abs() * dmc * (1 + relc) + xw.abs() * (relc + 4 * U) + 2 * U * (xw.abs() + b.abs())
    z = xw + b
    want = act64(z, act)
    # |silu'| <= 1.1; the gate itself costs 8 u, and the short exponential of bfloat16 results (2 + |z|) 2^-22
    extra = 0 if act != "silu" else want.abs() * (8 * U + (2 ** -22 * (2 + z.abs()) if dtype == "bf16" else 0)) + 1e-26
    check(y, want, 1.1 * dz + extra + out_bound(want, dtype), "y")


def check_group_norm_backward(dy, x, mean, rstd, w, b, act, dtype, gdtype, dx, dw, db, shared=False):
    """x: what the backward pass reads, [N, samples, pixels, C] binary64 or less; mean, rstd as given to it."""
    dy, x, w, b = dy.double(), x.double(), w.double()[:, None, None], b.double()[:, None, None]
    groups = mean.shape[-1]
    width, K = x.shape[-1] // groups, 80 + x.shape[2] / 4
    m, r = _spread(mean.double(), width), _spread(rstd.double(), width)
    xh = (x - m) * r
    z = xh * w + b
    dz = dy * slope64(z, act)
    # silu' has slope 1/2 at most; 24 u its evaluation; the short exponential as in the forward pass
    ez = 0 if act != "silu" else dy.abs() * (U * (24 + 4 * ((xh * w).abs() + b.abs())) + (2 ** -22 * (4 + 2 * z.abs()) if dtype == "bf16" else 0))
    t, et = dz * w, ez * w.abs()
    _, level = _over_group(t, groups, "mean")
    _, along = _over_group(t * xh, groups, "mean")
    _, dl = _over_group((K + 4) * U * t.abs() + et, groups, "mean")
    _, da = _over_group((K + 8) * U * (t * xh).abs() + et * xh.abs(), groups, "mean")
    want = r * (t - level - xh * along)
    bound = r * (8 * U * (t.abs() + level.abs() + (xh * along).abs()) + et + dl + xh.abs() * da)
    check(dx, want, bound + out_bound(want, dtype) + 1e-30, "dx")
    axes = (0, 1, 2) if shared else (1, 2)
    for name, got, term, err, k in (("dweight", dw, dz * xh, ez * xh.abs(), K + 8), ("dbias", db, dz, ez + 0 * dz, K + 4)):
        total = term.sum(axes)
        check(got, total, (k * U * term.abs() + err).sum(axes) + out_bound(total, gdtype), name)


def check_weight_grad(dy, x, gdtype, dweight):
    """dweight[n] = dy[n]^T x[n]; exact products, every addition rounded or cut (2 u), at most rows of them."""
    dy, x = dy.double(), x.double()
    want = dy.transpose(-1, -2) @ x
    bound = 2 * (dy.shape[-2] + 16) * U * (dy.abs().transpose(-1, -2) @ x.abs())
    check(dweight, want, bound + out_bound(want, gdtype), "dweight")
