"""Rotary positions against their definition in 64 bits: layouts, parts of a head, strides, positions far and negative, in place, and the gradient as the inverse and against differences."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
STORE = {torch.float32: U, torch.bfloat16: 2.0 ** -8}


@pytest.fixture(scope="module")
def B():
    from paper_2103_08870_amd import binding
    binding.lib()
    assert torch.cuda.is_available()
    return binding


@pytest.fixture(scope="module")
def ctx(B):
    c = B.Context(1, 1, 1)
    yield c
    c.close()


def rand(rows, cols, seed, dtype):
    return torch.randn((rows, cols), generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def definition(x, heads, freqs, positions, layout, amplitude=1.0, inverse=False):
    """The value, and how far from it: the angle is off by 2^-26 of a turn, sine and cosine by some units, each product and sum by half a unit, the result by its rounding."""
    dims, dim = 2 * freqs.numel(), x.shape[1] // heads
    t = positions.double()[:, None] * freqs.double().cuda() * (-1 if inverse else 1)
    z = x.double().view(x.shape[0], heads, dim).clone()
    a, b = (slice(0, dims // 2), slice(dims // 2, dims)) if layout == "halves" else (slice(0, dims, 2), slice(1, dims, 2))
    c, s = torch.cos(t)[:, None] * amplitude, torch.sin(t)[:, None] * amplitude
    p, q = z[..., a].clone(), z[..., b].clone()
    z[..., a], z[..., b] = p * c - q * s, p * s + q * c
    off = STORE[x.dtype] * z.abs()
    turned = abs(amplitude) * (2 * math.pi * 2.0 ** -26 + 8 * U) * (p.abs() + q.abs())
    off[..., a] += turned
    off[..., b] += turned
    return z.view(x.shape), off.view(x.shape)


def near(got, want, off):
    bad = ~((got.double() - want).abs() <= off)
    assert not bool(bad.any()), (int(bad.sum()), torch.nonzero(bad)[:3].tolist())


SHAPES = [(1, 1, 2, 2), (8, 40, 128, 128), (301, 14, 80, 40), (33, 3, 7, 6), (129, 5, 100, 2), (5000, 8, 64, 64), (17, 2, 300, 256), (1000, 1, 33, 32)]


@pytest.mark.parametrize("layout", ["halves", "neighbours"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,heads,dim,dims", SHAPES)
def test_against_the_definition(B, ctx, rows, heads, dim, dims, dtype, layout):
    x = rand(rows, heads * dim, rows + dim, dtype)
    freqs = B.lgc_rotary_frequencies(dims, factor=4.0, length=8192).cuda()
    positions = torch.randint(-2 ** 31, 2 ** 31 - 1, (rows,), generator=torch.Generator().manual_seed(1), dtype=torch.int64).to(torch.int32).cuda()
    near_by = positions % 4096
    for inverse in (False, True):
        for where, amplitude in ((positions, 1.0), (near_by, 1.25)):
            want, off = definition(x, heads, freqs, where, layout, amplitude, inverse)
            # at 2^31 the product itself, in 64 bits, is off by 2^-53 of up to 2^31 radians
            off = off + 2.0 ** -20 * abs(amplitude) * x.double().abs().amax()
            y = torch.full_like(x, 7.0)
            B.lgc_rotate(ctx, x, heads, freqs, y, positions=where, layout=layout, amplitude=amplitude, inverse=inverse)
            near(y, want, off)
            z = x.clone()
            B.lgc_rotate(ctx, z, heads, freqs, positions=where, layout=layout, amplitude=amplitude, inverse=inverse)
            assert torch.equal(y, z)                        # in place
            wide = torch.full((rows, heads * dim + 5), 7.0, dtype=dtype, device="cuda")
            wide[:, 1:1 + heads * dim] = x                  # other distances, odd addresses
            out = torch.full((rows, heads * dim + 9), 7.0, dtype=dtype, device="cuda")
            B.lgc_rotate(ctx, wide[:, 1:1 + heads * dim], heads, freqs, out[:, 3:3 + heads * dim], positions=where, layout=layout, amplitude=amplitude, inverse=inverse)
            assert torch.equal(out[:, 3:3 + heads * dim], y) and bool((out[:, :3] == 7).all()) and bool((out[:, 3 + heads * dim:] == 7).all())


def test_close_positions_are_exact_to_fp32(B, ctx):
    """Without the allowance for positions of 2^31: up to a million."""
    freqs = B.lgc_rotary_frequencies(128).cuda()
    x = rand(700, 4 * 128, 3, torch.float32)
    positions = torch.randint(0, 1_000_000, (700,), generator=torch.Generator().manual_seed(2), dtype=torch.int32).cuda()
    y = torch.empty_like(x)
    B.lgc_rotate(ctx, x, 4, freqs, y, positions=positions)
    near(y, *definition(x, 4, freqs, positions, "halves"))


def test_positions_by_the_row(B, ctx):
    freqs = B.lgc_rotary_frequencies(64).cuda()
    x = rand(100, 2 * 64, 4, torch.bfloat16)
    for period in (0, 1, 30, 100):
        y, z = torch.empty_like(x), torch.empty_like(x)
        rows = torch.arange(100, dtype=torch.int32, device="cuda")
        B.lgc_rotate(ctx, x, 2, freqs, y, period=period)
        B.lgc_rotate(ctx, x, 2, freqs, z, positions=rows % period if period else rows)
        assert torch.equal(y, z), period


def test_the_gradient(B, ctx):
    """It is the transpose: <dy, rotate(x)> = <inverse(dy), x>; rotating back gives x again; and against differences, which for a linear map are the map itself."""
    freqs = B.lgc_rotary_frequencies(48).cuda()
    x, dy = rand(200, 3 * 64, 5, torch.float32), rand(200, 3 * 64, 6, torch.float32)
    y, dx, back = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    how = dict(layout="neighbours", amplitude=1.5)
    B.lgc_rotate(ctx, x, 3, freqs, y, **how)
    B.lgc_rotate(ctx, dy, 3, freqs, dx, inverse=True, **how)
    both = float((dy.double().abs() * y.double().abs()).sum()) + float((dx.double().abs() * x.double().abs()).sum())
    assert abs(float((dy.double() * y.double()).sum()) - float((dx.double() * x.double()).sum())) <= 32 * U * both
    B.lgc_rotate(ctx, x, 3, freqs, y, layout="neighbours")
    B.lgc_rotate(ctx, y, 3, freqs, back, layout="neighbours", inverse=True)
    size = x.view(200, 3, 64).norm(dim=2, keepdim=True).expand(200, 3, 64).reshape(x.shape)
    assert bool(((back - x).abs() <= 64 * U * size).all())


def test_not_finite(B, ctx):
    freqs = B.lgc_rotary_frequencies(64).cuda()
    x = rand(64, 2 * 96, 7, torch.bfloat16)
    clean = torch.empty_like(x)
    B.lgc_rotate(ctx, x, 2, freqs, clean)
    x[10, 5], x[20, 70] = math.nan, math.inf           # a pair (5, 37) of head 0, and a column that is copied
    y = torch.empty_like(x)
    B.lgc_rotate(ctx, x, 2, freqs, y)
    hit = torch.zeros(x.shape, dtype=torch.bool, device="cuda")
    hit[10, 5] = hit[10, 37] = True
    assert bool(y[hit].isnan().all()) and float(y[20, 70]) == math.inf
    hit[20, 70] = True
    assert torch.equal(y[~hit], clean[~hit])


def test_in_a_graph(B, ctx):
    freqs = B.lgc_rotary_frequencies(64).cuda()
    x = rand(300, 4 * 64, 8, torch.bfloat16)
    y, positions = torch.empty_like(x), torch.arange(300, dtype=torch.int32, device="cuda")
    B.lgc_rotate(ctx, x, 4, freqs, y, positions=positions)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.lgc_rotate(ctx, x, 4, freqs, y, positions=positions)
    for i in range(3):
        x.copy_(rand(300, 4 * 64, 9 + i, torch.bfloat16))
        positions.add_(1000)
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        want = torch.empty_like(y)
        B.lgc_rotate(ctx, x, 4, freqs, want, positions=positions)
        assert torch.equal(y, want)


def test_the_binding_s_checks(B, ctx):
    freqs = B.lgc_rotary_frequencies(64).cuda()
    x = rand(30, 2 * 64, 9, torch.bfloat16)
    for call in (lambda: B.lgc_rotate(ctx, x, 3, freqs), lambda: B.lgc_rotate(ctx, x, 0, freqs), lambda: B.lgc_rotate(ctx, x, 2, freqs.float()), lambda: B.lgc_rotate(ctx, x, 2, freqs.cpu()),
                 lambda: B.lgc_rotate(ctx, x, 2, freqs, x.float()), lambda: B.lgc_rotate(ctx, x, 2, freqs, positions=torch.zeros(29, dtype=torch.int32, device="cuda")),
                 lambda: B.lgc_rotate(ctx, x, 2, freqs, positions=torch.zeros(30, dtype=torch.int64, device="cuda")), lambda: B.lgc_rotate(ctx, x, 2, freqs, layout="pairs"),
                 lambda: B.lgc_rotate(ctx, x, 2, freqs, period=-1), lambda: B.lgc_rotate(ctx, x[:, ::2], 2, freqs)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: B.lgc_rotate(ctx, x, 4, freqs), lambda: B.lgc_rotary_frequencies(7), lambda: B.lgc_rotary_frequencies(0), lambda: B.lgc_rotary_frequencies(8, factor=0.0)):
        with pytest.raises(B.LgcError):
            call()
