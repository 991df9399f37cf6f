"""The product with bias, non-linearity and residual in its epilogue: against the definition in 64 bits, its 8-bit results against what lgc_quantize makes of the same numbers, and its backward pass from
the checkpoint that it leaves, by the operators that were there, against differences."""
import math

import pytest
import torch

import training_reference as ref

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
    B.lgc_reserve_training(c)
    yield c
    c.close()


def rand(shape, seed, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).cuda()


def made(B, ctx, m, n, k, seed):
    """A, B in 8 bits and their values in 64; the bias."""
    a, b = B.Blocks(m, k), B.Blocks(n, k, tiles=True)
    x, w = rand((m, k), seed), rand((n, k), seed + 1, k ** -0.5)
    B.lgc_quantize(ctx, x, a)
    B.lgc_quantize_weights(ctx, w, b)
    B.lgc_dequantize(ctx, a, x)
    B.lgc_dequantize(ctx, b, w)
    return a, b, x.double(), w.double(), rand((n,), seed + 2)


def act(name, t):
    return {None: lambda: t, "relu": lambda: t.clamp(min=0.0), "silu": lambda: t / (1 + torch.exp(-t)), "gelu": lambda: 0.5 * t * torch.erfc(-t / math.sqrt(2))}[name]()


def sum_off(x, w, bias, dtype):
    """How far t may be from its value: exact products added in fp32, or (bf16) eight at a time with 14 bits below the largest."""
    size = x.abs() @ w.abs().t() + bias.abs()
    return size * ((x.shape[1] / 8 + 64) * U + (2.0 ** -13 if dtype is torch.bfloat16 else 0.0))


# few rows, few rows in parts, small tiles, tiles in parts, large tiles, edges of them all
SHAPES = [(1, 4096, 1024), (1, 300, 5000), (5, 130, 100), (16, 700, 300), (33, 8192, 200), (50, 1000, 1000), (64, 129, 129), (100, 300, 200), (257, 1100, 333), (300, 300, 9000), (2100, 4200, 300),
          (130, 33000, 128)]
HOW = [("gelu", False), (None, True), ("silu", True), ("relu", False)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_against_the_definition(B, ctx, m, n, k, dtype):
    a, b, x, w, bias = made(B, ctx, m, n, k, m + n)
    t = x @ w.t() + bias.double()
    t_off = sum_off(x, w, bias.double(), dtype)
    for name, residual in HOW:
        r = rand((m, n), 9).to(dtype) if residual else None
        z = torch.full((m, n + 3), 7.0, dtype=dtype, device="cuda")
        B.lgc_product_activate(ctx, a, b, bias, name, residual=r, z=z[:, 2:2 + n])
        got = z[:, 2:2 + n].double()
        f = act(name, t)
        want = f + r.double() if residual else f
        # the slope of none of them passes 1.13; their own precision is 1e-6 of the result, in the tail some t^2 2^-24
        off = 1.13 * t_off + (0.0 if name is None else f.abs() * (2e-6 + 4 * t * t * U)) + 2 * U * want.abs() + STORE[dtype] * want.abs()
        bad = ~((got - want).abs() <= off + 1e-37)
        assert not bool(bad.any()), (name, int(bad.sum()), float(((got - want).abs() / off)[bad].max()))
        assert bool((z[:, :2] == 7).all()) and bool((z[:, 2 + n:] == 7).all())
        if residual:                                    # the residual in z's own place
            y = torch.empty((m, n), dtype=dtype, device="cuda").copy_(r)
            B.lgc_product_activate(ctx, a, b, bias, name, residual=y, z=y)
            assert torch.equal(y.double(), got)


def holds(b, value, off):
    """b's 8 bits hold numbers as near to value as off, with an exponent that its block's largest asks for, and zeros behind the last column."""
    got = ref.blocks_values(b).cuda()
    e = b.exps[:, :(value.shape[1] + 127) // 128].long()
    size = torch.where(value.isfinite(), value, 0.0).abs()
    pad = torch.nn.functional.pad
    most, least = (pad((size + s * off).clamp(min=0.0), (0, -value.shape[1] % 128)).view(value.shape[0], -1, 128).amax(2) for s in (1, -1))
    top = 448.0 * torch.exp2(e.double() - 127)
    assert bool((least <= top).all()) and bool((most >= top / 2).logical_or(e == 10).all())     # no larger an exponent than needed, and none too small
    step = 2.0 ** -4 * got.abs() + 2.0 ** -10 * top.repeat_interleave(128, 1)[:, :value.shape[1]] / 448 + off
    bad = ~((got - value).abs() <= step)
    assert not bool(bad.any()), (int(bad.sum()),)
    assert int(b.codes[:, value.shape[1]:].count_nonzero()) == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_8_bits(B, ctx, m, n, k, dtype):
    a, b, x, w, bias = made(B, ctx, m, n, k, m + n)
    t = x @ w.t() + bias.double()
    t_off = sum_off(x, w, bias.double(), dtype)
    z, t8, z8 = torch.empty((m, n), dtype=dtype, device="cuda"), B.Blocks(m, n), B.Blocks(m, n)
    for blocks in (t8, z8):
        blocks.codes.fill_(0x55)
    B.lgc_product_activate(ctx, a, b, bias, "gelu", z=z, t_blocks=t8, z_blocks=z8)
    f = act("gelu", t)
    holds(t8, t, t_off)
    holds(z8, f, 1.13 * t_off + f.abs() * (2e-6 + 4 * t * t * U))
    # with fewer outputs, the same bits of those that are asked for (to bf16: a product without z has bf16's precision)
    one, other, plain = B.Blocks(m, n), B.Blocks(m, n), torch.empty_like(z)
    if dtype is torch.bfloat16:
        B.lgc_product_activate(ctx, a, b, bias, "gelu", t_blocks=one)
        B.lgc_product_activate(ctx, a, b, bias, "gelu", z_blocks=other)
        assert torch.equal(one.codes, t8.codes) and torch.equal(other.codes, z8.codes)
        for got, want in ((one, t8), (other, z8)):
            assert torch.equal(got.exps[:, :(n + 127) // 128], want.exps[:, :(n + 127) // 128])
    if dtype is torch.float32:      # z is there, so z8 is what lgc_quantize makes of it
        B.lgc_quantize(ctx, z, other)
        assert torch.equal(other.codes, z8.codes)


@pytest.mark.parametrize("m,n,k", [(1, 256, 128), (100, 300, 200), (2100, 4200, 128)])
def test_not_finite(B, ctx, m, n, k):
    """Infinities and NaNs in the bias: their columns alone; in 8 bits NaNs there, and the block's exponent from what is finite."""
    a, b, x, w, bias = made(B, ctx, m, n, k, 5)
    z, t8 = torch.empty((m, n), dtype=torch.bfloat16, device="cuda"), B.Blocks(m, n)
    B.lgc_product_activate(ctx, a, b, bias, "relu", z=z, t_blocks=t8)
    dirty = bias.clone()
    dirty[7], dirty[200] = math.nan, math.inf
    y, s8 = torch.empty_like(z), B.Blocks(m, n)
    B.lgc_product_activate(ctx, a, b, dirty, "relu", z=y, t_blocks=s8)
    same = torch.ones(n, dtype=torch.bool, device="cuda")
    same[7] = same[200] = False
    assert torch.equal(y[:, same], z[:, same]) and bool(y[:, 7].isnan().all()) and bool((y[:, 200] == math.inf).all())
    got = ref.blocks_values(s8)
    assert bool(got[:, 7].isnan().all()) and bool(got[:, 200].isnan().all()) and bool(got[:, same.cpu()].isfinite().all())


def test_forward_and_backward_of_a_linear_layer(B, ctx):
    """dt from the checkpoint, dx, dw, db and the residual's gradient, by the operators that were there; against differences of the whole in 64 bits without 8-bit rounding of t, which costs f' its part."""
    m, n, k = 40, 256, 128
    a, b, x, w, bias = made(B, ctx, m, n, k, 77)
    bt = B.Blocks(k, n, tiles=True)
    B.lgc_quantize_weights(ctx, w.float(), B.Blocks(n, k, tiles=True), bt)
    r, dz = rand((m, n), 1).to(torch.bfloat16), rand((m, n), 2).to(torch.bfloat16)
    z, t8 = torch.empty((m, n), dtype=torch.bfloat16, device="cuda"), B.Blocks(m, n)
    B.lgc_product_activate(ctx, a, b, bias, "silu", residual=r, z=z, t_blocks=t8)
    dt, dt8, dx = torch.empty_like(z), B.Blocks(m, n), torch.empty((m, k), device="cuda")
    dw, db = torch.empty((n, k), device="cuda"), torch.empty(n, device="cuda")
    B.lgc_activate_grad(ctx, "silu", dz, t8, da=dt, da_blocks=dt8)
    B.lgc_weight_grad(ctx, dt, a, dw, db)
    B.lgc_product(ctx, dt8, bt, None, dx)
    loss = lambda x, w, bias: float(((act("silu", x @ w.t() + bias) + r.double()) * dz.double()).sum())  # noqa: E731
    step = 1e-5
    for got, value, at in ((dx, x, 0), (dw, w, 1), (db, bias.double(), 2)):
        d = rand(value.shape, 30 + at).double()
        args = [x, w, bias.double()]
        up, down = ([v + s * step * d if i == at else v for i, v in enumerate(args)] for s in (1, -1))
        along = (loss(*up) - loss(*down)) / (2 * step)
        # 8 bits move t by 2^-4 of itself, and silu' by at most half of that (its own slope is at most 1/2); dx's factors are in 8 bits too: 2^-4 more of each dt
        t = x @ w.t() + bias.double()
        dt_off = dz.double().abs() * (0.5 * 2.0 ** -4 * t.abs() + 2.0 ** -8 * 1.1)
        grown = dt_off + 2.0 ** -4 * 1.1 * dz.double().abs() if at == 0 else dt_off
        off = {0: lambda: (grown @ w.abs() * d.abs()).sum(), 1: lambda: ((grown.t() @ x.abs()) * d.abs()).sum(), 2: lambda: (grown.sum(0) * d.abs()).sum()}[at]()
        assert abs(float((got.double() * d).sum()) - along) <= float(off), at


def test_strides_streams_graphs_and_bits(B, ctx):
    for m, n, k in ((1, 4096, 1024), (1, 300, 5000), (300, 300, 9000), (100, 300, 200)):
        a, b, _, _, bias = made(B, ctx, m, n, k, 3)
        r = rand((m, n), 1).to(torch.bfloat16)
        z, t8 = torch.empty((m, n), dtype=torch.bfloat16, device="cuda"), B.Blocks(m, n)
        call = lambda: B.lgc_product_activate(ctx, a, b, bias, "gelu", residual=r, z=z, t_blocks=t8)  # noqa: E731
        call()
        torch.cuda.synchronize()
        want = z.clone(), t8.codes.clone()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            z.zero_()
            call()
        side.synchronize()
        assert torch.equal(z, want[0]) and torch.equal(t8.codes, want[1])
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        for i in range(3):
            r.copy_(rand((m, n), 40 + i))
            z.zero_()
            t8.codes.zero_()
            g.replay()
            torch.cuda.synchronize()
            got = z.clone(), t8.codes.clone()
            call()
            assert torch.equal(got[0], z) and torch.equal(got[1], t8.codes)


def test_the_binding_s_checks(B, ctx):
    a, b, _, _, bias = made(B, ctx, 10, 256, 128, 4)
    z, r, same = torch.empty((10, 256), device="cuda"), torch.empty((10, 256), device="cuda"), B.Blocks(10, 256)
    for call in (lambda: B.lgc_product_activate(ctx, a, b, bias, "tanh", z=z), lambda: B.lgc_product_activate(ctx, a, b, bias, z=z[:, :200]), lambda: B.lgc_product_activate(ctx, a, a, bias, z=z),
                 lambda: B.lgc_product_activate(ctx, a, b, bias[:100], z=z), lambda: B.lgc_product_activate(ctx, a, b, bias, residual=r.to(torch.bfloat16), z=z),
                 lambda: B.lgc_product_activate(ctx, a, b, bias, z=z, t_blocks=B.Blocks(10, 128)), lambda: B.lgc_product_activate(ctx, a, b, bias, residual=r[:5], z=z)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: B.lgc_product_activate(ctx, a, b, bias, residual=r.to(torch.bfloat16), t_blocks=B.Blocks(10, 256)),
                 lambda: B.lgc_product_activate(ctx, a, b, bias, residual=r, z=z, z_blocks=B.Blocks(10, 256)), lambda: B.lgc_product_activate(ctx, a, b, bias, t_blocks=same, z_blocks=same)):
        with pytest.raises(B.LgcError):
            call()
    B.lgc_product_activate(ctx, a, b, bias)        # nothing is wanted
