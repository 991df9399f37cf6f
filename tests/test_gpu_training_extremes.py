"""The largest numbers of fp32 and bf16 in 8 bits: finite ones stay finite, within the half unit of three bits (2^-4 of themselves) that holds for all others."""
import math

import pytest
import torch

import training_reference as ref

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16]
TOP = 240.0 * 2.0 ** 120      # the largest number that a code stands for at the largest exponent: the next one, 256 * 2^120, is beyond fp32


@pytest.fixture(scope="module")
def B():
    from paper_2103_08870_amd import binding
    binding.lib()
    assert torch.cuda.is_available()
    return binding


@pytest.fixture(scope="module")
def ctx(B):
    c = B.Context(1, 1, 1)
    B.lgc_reserve_training(c)
    yield c
    c.close()


def codes(x, rows_per):
    """ref.codes, and where the largest exponent would give 256, 240."""
    c, e = ref.codes(x, rows_per)
    over = (ref.spread(e, rows_per, *x.shape) == 247) & (c & 127 == 0x78)
    return torch.where(over, c - 1, c), e


def check(b, x, rows_per):
    want, e = codes(x, rows_per)
    got = b.codes.cpu().long()[:, :x.shape[1]]
    assert torch.equal(torch.where(want == 127, got & 127, got), want) and torch.equal(b.exps.cpu().long()[:, :e.shape[1]], e)
    finite = torch.isfinite(x.double())
    v = ref.blocks_values(b)
    assert torch.equal(v[finite].float().double(), v[finite]) and bool((v[finite].abs() <= TOP).all()) and bool(v[~finite].isnan().all())
    edge = ref.spread(e, rows_per, *x.shape).double()
    assert ((v - x.double()).abs() <= 2.0 ** -4 * x.double().abs() + torch.exp2(edge - 127 - 10))[finite].all()


def top(dtype):
    """Rows whose largest magnitude is every number worth telling apart from 1.75 * 2^127 on, and smaller ones beside it."""
    most = torch.finfo(dtype).max
    steps = [t * 2.0 ** 120 for t in (224, 225, 231, 232, 233, 239, 240, 241, 247, 248, 249, 252, 255)] + [most]
    x = torch.zeros((2 * len(steps) + 2, 300), dtype=torch.float64)
    for i, s in enumerate(steps):
        x[2 * i, :140], x[2 * i, 141] = s, -s                                            # (to the next block, whose only one it is)
        x[2 * i + 1] = torch.linspace(-1, 1, 300, dtype=torch.float64) * s
    x[-2], x[-2, 3], x[-2, 200], x[-1] = most, math.inf, -math.inf, -most
    x[-1, 7] = math.nan
    return x.clamp(-most, most).to(dtype).where(torch.isfinite(x), x.to(dtype))


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_and_back(B, ctx, dtype):
    x = top(dtype)
    b = B.Blocks(*x.shape)
    B.lgc_quantize(ctx, x.cuda(), b)
    check(b, x, 1)
    for out_type in TYPES:
        out = torch.empty(x.shape, dtype=out_type, device="cuda")
        B.lgc_dequantize(ctx, b, out)
        assert torch.equal(out.cpu().double().nan_to_num(7.0), ref.blocks_values(b).nan_to_num(7.0))
        assert torch.equal(torch.isfinite(out.cpu()), torch.isfinite(x))


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_weights(B, ctx, dtype):
    x = top(dtype)
    b, t = B.Blocks(*x.shape, tiles=True), B.Blocks(x.shape[1], x.shape[0], tiles=True)
    B.lgc_quantize_weights(ctx, x.cuda(), b, t)
    check(b, x, 128)
    check(t, x.t().contiguous(), 128)


def test_layer_norm_to_blocks(B, ctx):
    x = torch.ones((3, 256))
    x[:, ::2] = -1.0                                      # its norm is itself, but for eps
    gamma = torch.linspace(0.9, 0.9999, 256) * torch.finfo(torch.float32).max
    y, b = torch.empty_like(x, device="cuda"), B.Blocks(3, 256)
    B.lgc_layer_norm(ctx, x.cuda(), gamma.cuda(), None, 0.0, y=y, blocks=b)
    assert bool(y.isfinite().all()) and float(y.abs().max()) > 250 * 2.0 ** 120
    check(b, y.cpu(), 1)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["relu", "gelu", "silu"])
def test_activate_and_its_gradient(B, ctx, kind, dtype):
    a = top(dtype)
    a8, z8, z = B.Blocks(*a.shape), B.Blocks(*a.shape), torch.empty_like(a, device="cuda")
    B.lgc_activate(ctx, kind, a.cuda(), z=z, a_blocks=a8, z_blocks=z8)
    check(a8, a, 1)
    if dtype == torch.float32:
        check(z8, z.cpu(), 1)
    # far out the slope is 1 or 0; a and dz of the same size, so that da in 8 bits meets the top too
    far = torch.isfinite(a) & (a.double().abs() > 2.0 ** 100)
    dz = torch.where(torch.isfinite(a), a.abs(), torch.ones_like(a)).to(dtype)
    da, da8 = torch.empty_like(a, device="cuda"), B.Blocks(*a.shape)
    B.lgc_activate_grad(ctx, kind, dz.cuda(), a8, da=da, da_blocks=da8)
    da = da.cpu()
    assert torch.equal(da[far], torch.where(a > 0, dz, torch.zeros_like(dz))[far])
    if dtype == torch.float32:
        check(da8, da, 1)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m", [1, 70])
def test_products(B, ctx, m, dtype):
    most = torch.finfo(torch.float32).max
    x, w = torch.full((m, 140), 0.0), torch.zeros((70, 140))
    x[:, 5], w[:, 5] = most, 0.5
    a, b = B.Blocks(m, 140), B.Blocks(70, 140, tiles=True)
    B.lgc_quantize(ctx, x.cuda(), a)
    B.lgc_quantize_weights(ctx, w.cuda(), b)
    y = torch.empty((m, 70), dtype=dtype, device="cuda")
    B.lgc_product(ctx, a, b, None, y)
    assert bool((y.double() == TOP / 2).all())
    x, w = torch.full((m, 140), 0.0), torch.zeros((70, 140))
    x[:, 5], w[:, 5] = 0.5, -most
    B.lgc_quantize(ctx, x.cuda(), a)
    B.lgc_quantize_weights(ctx, w.cuda(), b)
    B.lgc_product(ctx, a, b, None, y)
    assert bool((y.double() == -TOP / 2).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_weight_grad(B, ctx, dtype):
    x, dy = torch.zeros((70, 140)), torch.zeros((70, 40), dtype=dtype)
    x[33, 9], dy[33] = -torch.finfo(torch.float32).max, 0.25
    b, dw = B.Blocks(70, 140), torch.empty((40, 140), device="cuda")
    B.lgc_quantize(ctx, x.cuda(), b)
    B.lgc_weight_grad(ctx, dy.cuda(), b, dw)
    want = torch.zeros((40, 140), dtype=torch.float64)
    want[:, 9] = -TOP / 4
    assert torch.equal(dw.cpu().double(), want)


def test_more_blocks_than_a_launch_s_first_dimension_has(B, ctx):
    """2^26 rows of one column and some: 8.6 GB of codes, in two rows of a launch's blocks; the last rows of the first and all of the second against the same alone."""
    rows, first = (1 << 26) + 70, (1 << 26) - 30
    x = torch.zeros((rows, 1), dtype=torch.bfloat16, device="cuda")
    x[first:] = torch.randn((rows - first, 1), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    last = x[first:].clone()
    big, small = B.Blocks(rows, 1), B.Blocks(rows - first, 1)
    out, z = torch.full_like(x, 7.0), torch.empty_like(last)
    B.lgc_quantize(ctx, last, small)
    check(small, last.cpu(), 1)
    B.lgc_quantize(ctx, x, big)
    assert torch.equal(big.codes[first:], small.codes) and torch.equal(big.exps[first:, 0], small.exps[:, 0]) and bool((big.exps[:first, 0] == 10).all())
    assert not any(bool(part.any()) for part in big.codes[:first].split(1 << 22))
    for large, alone in ((lambda: B.lgc_dequantize(ctx, big, out), lambda: B.lgc_dequantize(ctx, small, z)),
                         (lambda: B.lgc_activate(ctx, "gelu", x, z=out, a_blocks=big), lambda: B.lgc_activate(ctx, "gelu", last, z=z)),
                         (lambda: B.lgc_activate_grad(ctx, "gelu", x, big, da=out), lambda: B.lgc_activate_grad(ctx, "gelu", last, small, da=z))):
        out.fill_(7.0)
        large()
        alone()
        assert torch.equal(out[first:], z) and not out[:first].any()
    assert torch.equal(big.codes[first:], small.codes)
