"""8-bit checkpoints of activations on the GPU: bytes, powers and restored values equal to the definition."""
import numpy as np
import pytest
import torch

from activation_helpers import DT, checkpoint64
from paper_2402_11857_b200 import liec

pytestmark = pytest.mark.gpu
compress, restore = liec.liec_activation_compress, liec.liec_activation_restore


def draw(shape, dtype, seed, pad=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(shape, generator=gen, device="cuda") * torch.exp(3 * torch.randn(shape[:-1] + (1,), generator=gen, device="cuda"))
    wide = torch.full(shape[:-1] + (shape[-1] + pad,), float("nan"), dtype=DT[dtype], device="cuda")
    wide[..., :shape[-1]] = x.to(DT[dtype])
    return wide[..., :shape[-1]]


def same(x, q, scales):
    want_q, want_s, back = checkpoint64(x)
    assert np.array_equal(q.cpu().numpy(), want_q) and np.array_equal(scales.cpu().numpy(), want_s)
    for dtype in ("f32", "bf16"):
        got = restore(q, scales, x.shape[-1], dtype=DT[dtype])
        assert got.dtype == DT[dtype] and np.array_equal(got.double().cpu().numpy(), back, equal_nan=True)
    return back


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,pad", [((1, 1), 0), ((3, 1), 0), ((2, 5, 7), 0), ((4, 33, 31), 0), ((1, 3, 32), 0), ((3, 17, 33), 0), ((2, 40, 256), 0),
                                       ((8, 77, 1001), 6), ((2, 20, 768), 3), ((3, 9, 768), 8), ((2, 3, 4, 50), 1), ((5, 1, 4099), 0),
                                       ((1, 2, 65536), 0), ((300, 2, 96), 0), ((1, 5000, 40), 5)])
def test_bytes_and_restored_values(shape, pad, dtype):
    x = draw(shape, dtype, seed=sum(shape), pad=pad)
    q, scales = compress(x)
    back = same(x, q, scales)
    top = np.abs(x.double().cpu().numpy()).max()
    assert np.abs(back - x.double().cpu().numpy()).max() <= top / 127
    # into a slice of a wider buffer: what lies beside it is left alone
    wide = torch.full(shape[:-1] + (shape[-1] + 5,), 3.0, dtype=DT[dtype], device="cuda")
    restore(q, scales, shape[-1], x=wide[..., 2:2 + shape[-1]])
    assert np.array_equal(wide[..., 2:2 + shape[-1]].double().cpu().numpy(), back) and (wide[..., :2] == 3).all() and (wide[..., -3:] == 3).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_borders_of_the_powers(dtype):
    """Largest magnitudes on both sides of 127.5 times a power, ties, the ends of the range, signed zeros, subnormals."""
    big = torch.finfo(DT[dtype]).max
    tops = [127.0, 127.25, 127.49999, 127.5, 127.50001, 127.75, 128.0, 63.75, 63.5, 64.0, 1.0, 0.0, -0.0, 2.0 ** -126, 2.0 ** -120, 127 * 2.0 ** -126,
            127.5 * 2.0 ** -126, 2.0 ** -127, 2.0 ** -133, 1e-45 if dtype == "f32" else 2.0 ** -133, big, big / 2, 2.0 ** 127, 0.1]
    x = torch.zeros(len(tops), 64, device="cuda")
    for i, t in enumerate(tops):
        x[i, 5], x[i, 7], x[i, 9], x[i, 40] = t, -t / 2, t / 254, -t
    x[:, 11] = -0.0
    x = x.to(DT[dtype])
    same(x, *compress(x))
    ties = (torch.arange(64, device="cuda").float() - 31.5)[None].repeat(2, 1)
    ties[:, 0] = -127.0
    ties[:, 33] = 64.0
    same(ties.to(DT[dtype]), *compress(ties.to(DT[dtype])))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_a_block_that_is_not_finite(value, dtype):
    x = draw((3, 100), dtype, seed=1).clone()
    x[0, 31], x[1, 99], x[2, 64] = value, value, value
    q, scales = compress(x)
    back = same(x, q, scales)
    nan = np.isnan(back)
    assert nan[0, :32].all() and nan[1, 96:].all() and nan[2, 64:96].all() and nan.sum() == 32 + 4 + 32


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_streams_graphs_and_no_rows(dtype):
    x = draw((6, 5, 48), dtype, seed=2)
    inside = x.transpose(0, 1).contiguous().transpose(0, 1)          # workers inside
    want = compress(x)
    for view, ref in ((inside, x), (x[::2], x[::2].contiguous()), (x[:, ::2], x[:, ::2].contiguous()), (x[:, :1].expand(6, 5, 48), x[:, :1].repeat(1, 5, 1)),
                      (x[:1].expand(6, 5, 48), x[:1].repeat(6, 1, 1))):
        assert all(torch.equal(a, b) for a, b in zip(compress(view), compress(ref)))
    out = torch.zeros_like(inside)
    restore(*want, 48, x=out)
    assert torch.equal(out, restore(*want, 48, dtype=DT[dtype]))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = compress(x, stream=s)
    back = restore(*got, 48, dtype=DT[dtype], stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got[0], want[0]) and torch.equal(back, restore(*want, 48, dtype=DT[dtype]))
    graph = torch.cuda.CUDAGraph()
    q, scales = torch.empty_like(want[0]), torch.empty_like(want[1])
    with torch.cuda.graph(graph):
        compress(x, q, scales)
    x.mul_(3)
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip((q, scales), compress(x)))
    for shape in ((0, 32), (3, 0, 32), (0, 3, 5)):
        q, scales = compress(torch.empty(shape, dtype=DT[dtype], device="cuda"))
        assert q.shape == shape[:-1] + (32,) and restore(q, scales, shape[-1], dtype=DT[dtype]).shape == shape


def test_offsets_beyond_32_bits():
    """Rows 2^31 + 8 elements apart."""
    buffer = torch.zeros(2 * (2 ** 31 + 8) + 64, dtype=torch.bfloat16, device="cuda")
    x = buffer.as_strided((3, 64), (2 ** 31 + 8, 1))
    x.copy_(draw((3, 64), "bf16", seed=3))
    q, scales = compress(x)
    back = same(x, q, scales)
    x.zero_()
    restore(q, scales, 64, x=x)
    assert np.array_equal(x.double().cpu().numpy(), back)


def test_many_rows():
    """More than 2^32 bytes of q: the last rows are right."""
    rows = 2 ** 26 + 3
    x = torch.zeros(rows, 40, dtype=torch.bfloat16, device="cuda")
    x[-5:] = draw((5, 40), "bf16", seed=4)
    q, scales = compress(x)
    assert q.numel() > 2 ** 32
    same(x[-5:], q[-5:], scales[-5:])
    assert torch.equal(restore(q, scales, 40, dtype=torch.bfloat16)[-5:], restore(q[-5:].contiguous(), scales[-5:].contiguous(), 40, dtype=torch.bfloat16))


def test_refusals():
    x = torch.randn(4, 64, device="cuda")
    q, scales = compress(x)
    with pytest.raises(ValueError, match="CUDA"):
        compress(x.cpu())
    with pytest.raises(ValueError, match="two axes"):
        compress(x[0])
    with pytest.raises(ValueError, match="contiguous"):
        compress(x.t())
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        compress(x.half())
    for bad in (q[:, :32], q[:2], q.to(torch.uint8)):
        with pytest.raises(ValueError, match="(q|scales) must be"):
            restore(bad, scales, 64)
    with pytest.raises(ValueError, match="scales must be"):
        restore(q, scales[:, :1], 64)
    with pytest.raises(ValueError):
        restore(q, scales, 64, x=torch.empty(4, 63, device="cuda"))
    with pytest.raises(ValueError, match="at most two"):
        compress(torch.zeros(4, 4, 4, 64, device="cuda")[::2, ::2, ::2])
    with pytest.raises(liec.LiecError, match="overlap"):
        restore(q, scales, 64, x=torch.zeros(1, 64, device="cuda").expand(4, 64))
    with pytest.raises(liec.LiecError, match="overlap"):
        compress(x, q=x.view(torch.int8).flatten()[:256].view(4, 64))
    with pytest.raises(liec.LiecError, match="16-byte"):
        compress(x, q=torch.zeros(300, dtype=torch.int8, device="cuda")[1:257].view(4, 64))
