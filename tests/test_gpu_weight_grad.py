"""Weight gradients from 8-bit checkpoints on the GPU against the products in binary64."""
import pytest
import torch

from activation_helpers import DT, U, check_weight_grad, restored64
from paper_2402_11857_b200 import liec

pytestmark = pytest.mark.gpu
weight_grad = liec.liec_weight_grad


def draw(N, rows, h, out, dtype, seed, pad=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(N, rows, h, generator=gen, device="cuda") + torch.randn(h, generator=gen, device="cuda")
    dy = torch.randn(N, rows, out, generator=gen, device="cuda") * 0.1
    wide = torch.full((N, rows, out + pad), float("nan"), dtype=DT[dtype], device="cuda")
    wide[..., :out] = dy.to(DT[dtype])
    return wide[..., :out], *liec.liec_activation_compress(x)


SHAPES = [(1, 1, 1, 1), (3, 4, 2, 5), (2, 32, 32, 32), (1, 33, 31, 65), (2, 64, 128, 256), (2, 100, 257, 129), (4, 32, 256, 256), (1, 2000, 64, 64),
          (3, 151, 133, 515), (1, 1, 768, 768), (2, 300, 768, 1000), (1, 5000, 200, 96), (40, 17, 48, 24), (1, 130, 1500, 40), (1, 20000, 8, 8), (2, 700, 512, 2048)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,rows,h,out", SHAPES)
def test_against_binary64(N, rows, h, out, dtype):
    dy, q, scales = draw(N, rows, h, out, dtype, seed=rows + h)
    got = weight_grad(dy, q, scales, h)
    assert got.shape == (N, out, h) and got.dtype == torch.float32
    check_weight_grad(dy, restored64(q, scales, h), "f32", got)
    assert torch.equal(weight_grad(dy, q, scales, h), got)       # equal calls, equal bits
    rows_of_grads = torch.full((N, out * h + 7), 5.0, dtype=torch.bfloat16, device="cuda")
    got = weight_grad(dy, q, scales, h, dweight=rows_of_grads[:, 3:3 + out * h].unflatten(1, (out, h)))
    check_weight_grad(dy, restored64(q, scales, h), "bf16", got)
    assert (rows_of_grads[:, :3] == 5).all() and (rows_of_grads[:, -4:] == 5).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [1, 3, 8])
def test_strides(pad, dtype):
    N, rows, h, out = 3, 90, 70, 136
    dy, q, scales = draw(N, rows, h, out, dtype, seed=pad, pad=pad)
    want = weight_grad(dy.contiguous(), q, scales, h)
    assert torch.equal(weight_grad(dy, q, scales, h), want)
    inside = dy.transpose(0, 1).contiguous().transpose(0, 1)
    wide = torch.full((out, N, h + 3), 2.0, device="cuda")
    assert torch.equal(weight_grad(inside, q, scales, h, dweight=wide[..., :h].transpose(0, 1)), want) and (wide[..., h:] == 2).all()
    once = dy[:, :1].expand(N, rows, out)                        # one gradient row for all tokens
    check_weight_grad(once, restored64(q, scales, h), "f32", weight_grad(once, q, scales, h))
    single = weight_grad(dy[1], q[1].contiguous(), scales[1].contiguous(), h)
    assert single.shape == (out, h) and torch.equal(single, want[1])


def test_range_of_values():
    """Tiny and large values: products are exact, so only the sum rounds."""
    dy, q, scales = draw(2, 60, 64, 40, "f32", seed=8)
    dy = dy * torch.logspace(-18, 18, 40, device="cuda")
    x = torch.logspace(-18, 15, 64, device="cuda") * torch.randn(2, 60, 64, device="cuda")
    q, scales = liec.liec_activation_compress(x)
    check_weight_grad(dy, restored64(q, scales, 64), "f32", weight_grad(dy, q, scales, 64))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_not_finite_stays_in_its_row_and_column(dtype):
    dy, q, scales = draw(2, 70, 96, 150, dtype, seed=9)
    clean = weight_grad(dy, q, scales, 96)
    dy = dy.clone()
    dy[0, 11, 7], dy[0, 60, 130] = float("nan"), float("inf")
    scales = scales.clone()
    scales[1, 5, 2] = 255                                        # a block that was not finite
    q[1, 5, 64:96] = 0
    got = weight_grad(dy, q, scales, 96)
    bad = torch.zeros_like(got, dtype=torch.bool)
    bad[0, 7], bad[0, 130], bad[1, :, 64:] = True, True, True
    assert not got[bad].isfinite().any() and torch.equal(got[~bad], clean[~bad])
    huge = torch.full_like(dy, torch.finfo(DT[dtype]).max)       # large values are finite
    small = torch.full_like(scales, 60)
    assert weight_grad(huge, q[:1].expand(2, 70, 96).contiguous(), small, 96)[0].isfinite().all()


def test_no_rows_streams_and_graphs():
    dy, q, scales = draw(2, 200, 96, 64, "bf16", seed=5)
    want = weight_grad(dy, q, scales, 96)
    empty = weight_grad(dy[:, :0], q[:, :0].contiguous(), scales[:, :0].contiguous(), 96, dweight=torch.full((2, 64, 96), 3.0, device="cuda"))
    assert (empty == 0).all()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = weight_grad(dy, q, scales, 96, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want)
    graph, out = torch.cuda.CUDAGraph(), torch.zeros(2, 64, 96, device="cuda")
    with torch.cuda.graph(graph):
        weight_grad(dy, q, scales, 96, dweight=out)
    dy.mul_(2)
    graph.replay()
    assert torch.equal(out, 2 * want)


def test_refusals():
    dy, q, scales = draw(2, 20, 40, 24, "f32", seed=6)
    with pytest.raises(ValueError, match="q must be"):
        weight_grad(dy, q[:, :10].contiguous(), scales, 40)
    with pytest.raises(ValueError, match="scales must be"):
        weight_grad(dy, q, scales[:, :10].contiguous(), 40)
    with pytest.raises(ValueError, match="dweight must be"):
        weight_grad(dy, q, scales, 40, dweight=torch.empty(2, 40, 24, device="cuda"))
    with pytest.raises(ValueError, match="contiguous"):
        weight_grad(dy.transpose(1, 2).contiguous().transpose(1, 2), q, scales, 40)
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        weight_grad(dy.half(), q, scales, 40)
    with pytest.raises(ValueError, match="CUDA"):
        weight_grad(dy.cpu(), q, scales, 40)
    with pytest.raises(liec.LiecError, match="overlap"):
        weight_grad(dy, q, scales, 40, dweight=torch.empty(1, 24, 40, device="cuda").expand(2, 24, 40))
    big = torch.zeros(2 * 24 * 40, device="cuda")                # dy within dweight
    with pytest.raises(liec.LiecError, match="overlaps an input"):
        weight_grad(big[:2 * 20 * 24].view(2, 20, 24), q, scales, 40, dweight=big.view(2, 24, 40))


@pytest.mark.parametrize("N,rows,h,out,dtype", [(90, 70, 40, 48, "f32"), (100, 33, 256, 600, "bf16"), (7, 2100, 600, 1300, "bf16"), (160, 200, 30, 20, "bf16"),
                                                (3, 900, 2000, 1700, "f32"), (2, 3300, 700, 300, "bf16")])
def test_more_tiles_than_pairs_of_sms(N, rows, h, out, dtype):
    """Several tiles one after another, whole and cut."""
    dy, q, scales = draw(N, rows, h, out, dtype, seed=N)
    got = weight_grad(dy, q, scales, h)
    check_weight_grad(dy, restored64(q, scales, h), "f32", got)
    assert torch.equal(weight_grad(dy, q, scales, h), got)


def test_copies_that_come_late():
    """All operands from memory and several tiles per pair: copies lag behind the products.  Equal bits over many calls."""
    dy, q, scales = draw(148, 1024, 256, 256, "f32", seed=31)
    want = weight_grad(dy, q, scales, 256)
    check_weight_grad(dy[:3], restored64(q[:3], scales[:3], 256), "f32", want[:3])
    for _ in range(10):
        assert torch.equal(weight_grad(dy, q, scales, 256), want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_sums_keep_their_digits(dtype):
    """Positive terms, so that sums grow evenly.  At most 112 additions (of 16 products each) to a sum in tensor memory, each
    cutting less than 2 u of the part so far: 113 u in all, then a few rounded additions of u each; 120 u."""
    gen = torch.Generator(device="cuda").manual_seed(12)
    dy = (torch.rand(80, 8192, 80, generator=gen, device="cuda") + 0.5).to(DT[dtype])
    q, scales = liec.liec_activation_compress(torch.rand(80, 8192, 96, generator=gen, device="cuda") + 0.5)
    got = weight_grad(dy, q, scales, 96)
    for n in (0, 41, 79):
        want = dy[n].double().t() @ restored64(q[n], scales[n], 96)
        assert ((got[n].double() - want).abs() <= 120 * U * want).all()
