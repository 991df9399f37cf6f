"""The training step's operators against their definitions in 64 bits: matrices in 8 bits bit for bit, the others within bounds that
follow from the format of what is stored and from the length of the fp32 sums (U: half a unit of an fp32 number's last place)."""
import math

import pytest
import torch

import training_reference as ref

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
STORE = {torch.float32: U, torch.bfloat16: 2.0 ** -8}      # rounding of a stored result (bf16: a whole unit)
TYPES = [torch.float32, torch.bfloat16]


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


def rand(shape, seed, scale=1.0, dtype=torch.float32):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=gen) * scale).to(dtype)


def on_gpu(x, pad=0, shift=0):
    """x on the GPU in rows x.shape[1] + pad apart, from an address that is not 16-byte aligned if shift is odd."""
    rows, cols = x.shape
    flat = torch.full((rows * (cols + pad) + shift + 8,), 7.0, dtype=x.dtype, device="cuda")
    view = flat[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(x)
    return view


def check_blocks(b, x, rows_per):
    """b holds x, bit for bit, padding included."""
    want, e = ref.codes(x, rows_per)
    got = b.codes.cpu().long()
    cols = x.shape[1]
    nan = want == 127
    assert torch.equal(torch.where(nan, got[:, :cols] & 127, got[:, :cols]), want)
    assert int(got[:, cols:].count_nonzero()) == 0
    assert torch.equal(b.exps.cpu().long()[:, :e.shape[1]], e)


def awkward(rows, cols, dtype, seed):
    """Blocks of every kind: ordinary, zero, tiny, huge, with infinities and NaNs, at the edge of an exponent, subnormal codes."""
    x = rand((rows, cols), seed) * torch.exp(3 * rand((rows, cols), seed + 1))
    for r in range(rows):
        kind = r % 9
        if kind == 1:
            x[r] = 0.0
        elif kind == 2:
            x[r] *= 1e-36
        elif kind == 3:
            x[r] *= 1e36 / x[r].abs().max()
        elif kind == 4:
            x[r, ::5], x[r, 1::7], x[r, 2::11] = math.inf, -math.inf, math.nan
        elif kind == 5:
            x[r] = torch.round(x[r] * 8).clamp(-7, 7)
            x[r, 0] = 448.0 * 2 ** -3
        elif kind == 6:
            x[r, 0] = 449.0 * 2 ** -3
        elif kind == 7:
            x[r] = math.nan
        elif kind == 8:
            x[r] *= 1e-42
    return x.to(dtype)


SHAPES = [(1, 1), (1, 128), (2, 127), (9, 129), (40, 777), (33, 1000), (130, 512), (3, 8200)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quantize_and_back(B, ctx, rows, cols, dtype):
    x = awkward(rows, cols, dtype, rows + cols)
    for pad, shift in ((0, 0), (3, 1), (8, 0)):
        b = B.Blocks(rows, cols)
        b.codes.fill_(0x55)
        B.lgc_quantize(ctx, on_gpu(x, pad, shift), b)
        check_blocks(b, x, 1)
        for out_type in TYPES:
            out = on_gpu(torch.zeros((rows, cols), dtype=out_type), pad, shift)
            B.lgc_dequantize(ctx, b, out)
            want = ref.blocks_values(b)
            assert torch.equal(out.cpu().double().nan_to_num(1e300), want.nan_to_num(1e300))
            assert float(out.as_strided((rows, cols + pad), (cols + pad, 1))[:-1, cols:].double().sum()) == 7.0 * pad * (rows - 1)   # what lies between rows is let be


@pytest.mark.parametrize("dtype", TYPES)
def test_every_code_comes_back_and_every_tie_goes_to_even(B, ctx, dtype):
    # all codes but NaN as numbers, the numbers half-way between neighbours, and (fp32) those next to half-way
    mids = (ref.NUMBERS[1:] + ref.NUMBERS[:-1]) / 2
    x = torch.cat([ref.NUMBERS, mids, mids * (1 + 2.0 ** -20), mids * (1 - 2.0 ** -20)]).float()
    x = torch.cat([x, -x])
    x = torch.nn.functional.pad(x, (0, -len(x) % 127)).view(-1, 127)
    x = torch.cat([torch.full((x.shape[0], 1), 448.0), x], 1).to(dtype)     # (448 holds the block's exponent at 127)
    for power in (-100, -3, 0, 50):
        b = B.Blocks(*x.shape)
        y = (x.double() * 2.0 ** power).to(dtype)
        B.lgc_quantize(ctx, y.cuda(), b)
        check_blocks(b, y, 1)
        assert int(b.exps[0, 0]) == 127 + power


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (128, 128), (129, 127), (300, 1000), (513, 260)])
def test_quantize_weights_and_their_transpose(B, ctx, rows, cols, dtype):
    w = rand((rows, cols), 5, 0.02, dtype)
    w[0, 0], w[rows // 2, cols // 2] = 3.0, math.inf
    if rows > 256:
        w[256:, :128] = 0.0
    b, t = B.Blocks(rows, cols, tiles=True), B.Blocks(cols, rows, tiles=True)
    B.lgc_quantize_weights(ctx, on_gpu(w, 5, 1), b, t)
    check_blocks(b, w, 128)
    check_blocks(t, w.t(), 128)
    only = B.Blocks(rows, cols, tiles=True)
    B.lgc_quantize_weights(ctx, w.cuda(), only)
    assert torch.equal(only.codes, b.codes)
    out = torch.empty((cols, rows), device="cuda")
    B.lgc_dequantize(ctx, t, out)
    assert torch.equal(out.cpu().double().nan_to_num(1e300), ref.blocks_values(b).t().nan_to_num(1e300))


# ---------------------------------------------------------------- layer norm

NORM_SHAPES = [(1, 1), (5, 2), (3, 8), (7, 511), (6, 512), (5, 513), (9, 1000), (4, 1025), (3, 2048), (5, 2050), (3, 4096), (2, 4099), (3, 8192), (2, 8200),
               (1, 16384), (2, 16390), (2, 32768), (2, 33000), (1000, 64), (2100, 300)]


def norm_inputs(rows, cols, dtype, seed):
    x = rand((rows, cols), seed) * torch.exp(rand((rows, 1), seed + 1)) + 3.0
    return x.to(dtype), 1 + rand((cols,), seed + 2, 0.2), rand((cols,), seed + 3, 0.2)


def norm_bound(x, gamma, mean, rstd, y, dtype):
    """Of y: the sums run through at most 40 additions in a row per thread, 6 in a wavefront and 16 over a block."""
    d = 64 * U
    x = x.double()
    g = 1.0 if gamma is None else gamma.double().abs()
    h = ((x - mean[:, None]) * rstd[:, None]).abs()
    return g * (d * (x.abs().mean(1) * rstd)[:, None] + 3 * d * h) + (STORE[dtype] + 2 * U) * y.abs() + 1e-30


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", NORM_SHAPES)
def test_layer_norm(B, ctx, rows, cols, dtype):
    x, gamma, beta = norm_inputs(rows, cols, dtype, 3 * cols + rows)
    eps = 1e-5
    want, mean, rstd = ref.layer_norm(x, gamma, beta, eps)
    for pad, shift in ((0, 0), (3, 1)):
        y = on_gpu(torch.zeros_like(x), pad, shift)
        m, r, b = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), B.Blocks(rows, cols)
        b.codes.fill_(0x55)
        B.lgc_layer_norm(ctx, on_gpu(x, pad, shift), gamma.cuda(), beta.cuda(), eps, y=y, mean=m, rstd=r, blocks=b)
        assert ((y.cpu().double() - want).abs() <= norm_bound(x, gamma, mean, rstd, want, dtype)).all()
        assert ((m.cpu().double() - mean).abs() <= 64 * U * x.double().abs().mean(1)).all()
        spread = 64 * U * (1 + (x.double().abs().mean(1) * rstd) ** 2) + 8 * U
        assert ((r.cpu().double() / rstd - 1).abs() <= spread).all()
        if dtype == torch.float32:
            check_blocks(b, y.cpu(), 1)               # the 8 bits are those of y, which fp32 holds as it was computed
        else:
            off = (ref.blocks_values(b) - want).abs()
            most = ref.spread(ref.exponents(want, 1), 1, rows, cols)
            assert (off <= 2.0 ** -4 * 1.001 * want.abs() + torch.exp2(most.double() - 127 - 9) + norm_bound(x, gamma, mean, rstd, want, torch.float32)).all()
        only = B.Blocks(rows, cols)
        B.lgc_layer_norm(ctx, on_gpu(x, pad, shift), gamma.cuda(), beta.cuda(), eps, blocks=only)
        assert torch.equal(only.codes, b.codes)


def test_layer_norm_of_rows_that_are_constant_or_not_finite(B, ctx):
    x = rand((5, 300), 9)
    x[0], x[1], x[2, 7], x[3, 8] = 0.0, 1000.0, math.inf, math.nan
    y, m, r = torch.empty_like(x, device="cuda"), torch.empty(5, device="cuda"), torch.empty(5, device="cuda")
    b = B.Blocks(5, 300)
    B.lgc_layer_norm(ctx, x.cuda(), None, None, 1e-5, y=y, mean=m, rstd=r, blocks=b)
    y = y.cpu()
    assert (y[0] == 0).all() and (y[1].abs() <= 300 * U * 1000 / math.sqrt(1e-5)).all()
    assert y[2].isnan().all() and y[3].isnan().all() and (b.codes[2:4, :300] & 127 == 127).all()
    want, mean, rstd = ref.layer_norm(x[4:], None, None, 1e-5)
    assert ((y[4:].double() - want).abs() <= norm_bound(x[4:], None, mean, rstd, want, torch.float32)).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", NORM_SHAPES)
def test_layer_norm_grad(B, ctx, rows, cols, dtype):
    x, gamma, _ = norm_inputs(rows, cols, dtype, 7 * cols + rows)
    dy = rand((rows, cols), cols, 1e-2, dtype)
    _, mean, rstd = ref.layer_norm(x, None, None, 1e-5)
    mean, rstd = mean.float(), rstd.float()
    for g in (gamma, None):
        want, wg, wb = ref.layer_norm_grad(dy, x, g, mean, rstd)
        dx, dg, db = on_gpu(torch.zeros_like(x), 3, 1), torch.full((cols,), 9.0, device="cuda"), torch.full((cols,), 9.0, device="cuda")
        B.lgc_layer_norm_grad(ctx, on_gpu(dy, 1, 1), on_gpu(x, 2, 0), None if g is None else g.cuda(), mean.cuda(), rstd.cuda(), dx, dg, db)
        h = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
        hx = h.abs() + 2 * U * (x.double().abs() * rstd.double()[:, None])
        q = dy.double().abs() * (1.0 if g is None else g.double().abs())
        d = 64 * U
        bound = rstd.double()[:, None] * (4 * U * q + d * q.mean(1, keepdim=True) + d * hx * (q * hx).mean(1, keepdim=True)) \
            + (STORE[dtype] + 4 * U) * want.abs() + 4 * U * rstd.double()[:, None] * (hx * (q * hx).mean(1, keepdim=True) + q) + 1e-30
        assert ((dx.cpu().double() - want).abs() <= bound).all()
        assert ((dg.cpu().double() - wg).abs() <= (rows + 40) * U * (dy.double().abs() * hx).sum(0) + 4 * U * (dy.double().abs() * x.double().abs() * rstd.double()[:, None]).sum(0)).all()
        assert ((db.cpu().double() - wb).abs() <= (rows + 40) * U * dy.double().abs().sum(0)).all()
        alone = torch.empty((cols,), device="cuda")
        B.lgc_layer_norm_grad(ctx, on_gpu(dy, 1, 1), on_gpu(x, 2, 0), None if g is None else g.cuda(), mean.cuda(), rstd.cuda(), dbeta=alone)
        assert torch.equal(alone, db)


def test_layer_norm_grad_against_differences(B, ctx):
    rows, cols = 6, 700
    x, gamma, beta = norm_inputs(rows, cols, torch.float32, 21)
    dy, step = rand((rows, cols), 22), 2.0 ** -7
    to, tg, tb = rand((rows, cols), 23), rand((cols,), 24), rand((cols,), 25)

    def loss(s):
        y = torch.empty((rows, cols), device="cuda")
        B.lgc_layer_norm(ctx, (x + s * to).cuda(), (gamma + s * tg).cuda(), (beta + s * tb).cuda(), 1e-5, y=y)
        return float((y.cpu().double() * dy.double()).sum())

    m, r = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    B.lgc_layer_norm(ctx, x.cuda(), gamma.cuda(), beta.cuda(), 1e-5, mean=m, rstd=r)
    dx, dg, db = torch.empty((rows, cols), device="cuda"), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    B.lgc_layer_norm_grad(ctx, dy.cuda(), x.cuda(), gamma.cuda(), m, r, dx, dg, db)
    slope = sum(float((a.cpu().double() * b.double()).sum()) for a, b in ((dx, to), (dg, tg), (db, tb)))
    up, down = loss(step), loss(-step)
    # what the difference of a step this long is off the slope, from the formula in 64 bits; the rest is the kernels' rounding
    x, gamma, beta, dy, to, tg, tb = (t.double() for t in (x, gamma, beta, dy, to, tg, tb))
    exact = [float((ref.layer_norm(x + s * to, gamma + s * tg, beta + s * tb, 1e-5)[0] * dy).sum()) for s in (step, -step)]
    grads = ref.layer_norm_grad(dy, x, gamma, *ref.layer_norm(x, gamma, beta, 1e-5)[1:])
    off = (exact[0] - exact[1]) / (2 * step) - sum(float((a * b).sum()) for a, b in zip(grads, (to, tg, tb)))
    assert abs((up - down) / (2 * step) - slope - off) <= 64 * U * math.sqrt(rows * cols) / step


# ---------------------------------------------------------------- non-linearities

ACTS = ["relu", "gelu", "silu"]


def act_error(kind, x):
    """Relative: polynomial and roundings, and the exponential's argument rounded at its size."""
    x = x.double().abs()
    return 2e-6 + 2 * U * (x * x if kind == "gelu" else x)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ACTS)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 129), (50, 1000), (70, 4096)])
def test_activate_and_its_gradient(B, ctx, rows, cols, kind, dtype):
    a = rand((rows, cols), 31, 2.0, dtype)
    a.view(-1)[::97] *= 6                      # far into both tails
    dz = rand((rows, cols), 32, 1e-3, dtype)
    z, a8, z8 = on_gpu(torch.zeros_like(a), 3, 1), B.Blocks(rows, cols), B.Blocks(rows, cols)
    B.lgc_activate(ctx, kind, on_gpu(a, 1, 1), z=z, a_blocks=a8, z_blocks=z8)
    want = ref.act(kind, a)
    assert ((z.cpu().double() - want).abs() <= (act_error(kind, a) + STORE[dtype]) * want.abs() + 1e-36).all()
    check_blocks(a8, a, 1)
    if dtype == torch.float32:
        check_blocks(z8, z.cpu(), 1)
    only = B.Blocks(rows, cols)
    B.lgc_activate(ctx, kind, a.cuda(), z_blocks=only)
    assert torch.equal(only.codes, z8.codes)
    da, da8 = on_gpu(torch.zeros_like(a), 3, 1), B.Blocks(rows, cols)
    B.lgc_activate_grad(ctx, kind, on_gpu(dz, 1, 1), a8, da=da, da_blocks=da8)
    k = ref.kept(a)
    slope = ref.act_slope(kind, k)
    # the slope is a sum of two terms of at most 1 and |x| phi(x), |x| p (1 - p), which may cancel
    off = act_error(kind, k) * (ref.act_slope(kind, k.abs()) + 1.2 * torch.exp(-k.abs()) * k.abs()).abs() * (k > -1) + \
        act_error(kind, k) * (1 + k.abs()) * (torch.exp(-k * k / 2) if kind == "gelu" else torch.exp(-k.abs())) * (k <= -1)
    assert ((da.cpu().double() - dz.double() * slope).abs() <= dz.double().abs() * (off + STORE[dtype] * slope.abs()) + 1e-36).all()
    if dtype == torch.float32:
        check_blocks(da8, da.cpu(), 1)


@pytest.mark.parametrize("kind", ACTS)
def test_activate_grad_against_differences(B, ctx, kind):
    rows, cols, step = 4, 256, 2.0 ** -6
    a = ref.kept(rand((rows, cols), 41)).float()       # numbers that 8 bits hold
    a[a == 0] = 0.5                                    # (relu has no slope there)
    a = ref.kept(a).float()
    a8, ones, da = B.Blocks(rows, cols), torch.ones((rows, cols), device="cuda"), torch.empty((rows, cols), device="cuda")
    B.lgc_activate(ctx, kind, a.cuda(), a_blocks=a8)
    B.lgc_activate_grad(ctx, kind, ones, a8, da=da)
    up, down = torch.empty_like(da), torch.empty_like(da)
    B.lgc_activate(ctx, kind, (a + step).cuda(), z=up)
    B.lgc_activate(ctx, kind, (a - step).cuda(), z=down)
    diff = (up.double() - down.double()).cpu() / (2 * step)
    away = (a.abs() > step) if kind == "relu" else torch.ones_like(a, dtype=torch.bool)
    assert ((diff - da.cpu().double()).abs()[away] <= step ** 2 / 6 * 2 + 1e-5 * (1 + a.double().abs()[away]) / step).all()


# ---------------------------------------------------------------- products

def as_blocks(B, ctx, x, tiles=False):
    b = B.Blocks(x.shape[0], x.shape[1], tiles=tiles)
    (B.lgc_quantize_weights if tiles else B.lgc_quantize)(ctx, x.cuda(), b)
    return b


PRODUCTS = [(1, 1, 1), (1, 128, 128), (1, 1000, 4096), (2, 300, 129), (3, 130, 1000), (7, 4096, 260), (16, 257, 512), (17, 128, 4100), (31, 640, 777), (64, 200, 2048),
            (100, 1000, 300), (128, 128, 128), (129, 129, 129), (255, 511, 640), (300, 1300, 1111), (1000, 77, 900), (513, 1025, 1280), (2049, 520, 384)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product(B, ctx, m, n, k, dtype):
    a = as_blocks(B, ctx, rand((m, k), m + n + k) * torch.exp(2 * rand((m, 1), k)))
    b = as_blocks(B, ctx, rand((n, k), n * k % 1000, 0.1), tiles=True)
    bias = rand((n,), 3)
    x, w = ref.blocks_values(a), ref.blocks_values(b)
    size = x.abs() @ w.abs().t()
    for add, pad, shift in ((bias, 0, 0), (None, 3, 1)):
        y = on_gpu(torch.full((m, n), 7.0, dtype=dtype), pad, shift)
        B.lgc_product(ctx, a, b, None if add is None else add.cuda(), y)
        want = x @ w.t() + (0.0 if add is None else add.double())
        # bf16: of eight neighbouring products each may lose 2^-14 of the largest; fp32: k additions at most
        bound = (2.0 ** -11 if dtype == torch.bfloat16 else (k + 16) * U) * size + STORE[dtype] * want.abs() + 4 * U * (1 if add is None else add.abs().double())
        assert ((y.cpu().double() - want).abs() <= bound).all()
        if pad:
            assert float(y.as_strided((m, n + pad), (n + pad, 1))[:-1, n:].double().sum()) == 7.0 * pad * (m - 1)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m", [1, 5, 40, 200])
def test_product_of_whole_numbers_is_exact(B, ctx, m, dtype):
    # numbers of few bits, sums below 2^8: every product and every sum is exact in any order, so a fragment out of its place shows
    n, k = 300, 1500
    gen = torch.Generator().manual_seed(8)
    x, w = (torch.rand((m, k), generator=gen) < 0.05).float(), (torch.rand((n, k), generator=gen) < 0.3).float()
    x *= torch.randint(-2, 3, (m, k), generator=gen)
    a, b = as_blocks(B, ctx, x), as_blocks(B, ctx, w, tiles=True)
    y = torch.empty((m, n), device="cuda", dtype=dtype)
    B.lgc_product(ctx, a, b, None, y)
    want = x.double() @ w.double().t()
    assert float(want.abs().max()) < 256 and torch.equal(y.cpu().double(), want)


@pytest.mark.parametrize("m", [1, 9, 140])
def test_product_meets_nan_and_very_different_scales(B, ctx, m):
    n, k = 140, 640
    x, w = rand((m, k), 1), rand((n, k), 2)
    x[:, 128:256] *= 2.0 ** 60
    w[:, 128:256] *= 2.0 ** -60
    x[:, 256:384] *= 2.0 ** -90
    x[0, 5] = math.inf
    a, b = as_blocks(B, ctx, x), as_blocks(B, ctx, w, tiles=True)
    for dtype in TYPES:
        y = torch.empty((m, n), device="cuda", dtype=dtype)
        B.lgc_product(ctx, a, b, None, y)
        assert y[0].isnan().all()
        xv, wv = ref.blocks_values(a)[1:], ref.blocks_values(b)
        bound = (2.0 ** -11 if dtype == torch.bfloat16 else (k + 16) * U) * (xv.abs() @ wv.abs().t()) + STORE[dtype] * (xv @ wv.t()).abs()
        assert ((y[1:].cpu().double() - xv @ wv.t()).abs() <= bound).all()


WEIGHT_GRADS = [(1, 1, 1), (1, 128, 128), (3, 130, 129), (31, 17, 300), (32, 128, 256), (33, 1000, 500), (64, 257, 511), (500, 64, 64), (1000, 300, 260), (5000, 130, 100),
                (257, 640, 1300), (2048, 512, 513), (40000, 8, 9)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n,k", WEIGHT_GRADS)
def test_weight_grad(B, ctx, rows, n, k, dtype):
    x = as_blocks(B, ctx, rand((rows, k), rows + k) * torch.exp(2 * rand((rows, 1), n)))
    dy = rand((rows, n), n + k, 1e-2, dtype)
    xv = ref.blocks_values(x)
    want, wb = dy.double().t() @ xv, dy.double().sum(0)
    for pad, shift in ((0, 0), (1, 1)):
        dw, db = on_gpu(torch.full((n, k), 7.0), 0, shift), torch.full((n,), 7.0, device="cuda")
        B.lgc_weight_grad(ctx, on_gpu(dy, pad, shift), x, dw, db)
        assert ((dw.cpu().double() - want).abs() <= (rows + 64) * U * (dy.double().abs().t() @ xv.abs()) + 1e-36).all()
        assert ((db.cpu().double() - wb).abs() <= (rows + 64) * U * dy.double().abs().sum(0) + 1e-36).all()
        alone = torch.empty((n, k), device="cuda")
        B.lgc_weight_grad(ctx, on_gpu(dy, pad, shift), x, alone)
        assert torch.equal(alone, dw)


@pytest.mark.parametrize("dtype", TYPES)
def test_weight_grad_of_whole_numbers_is_exact(B, ctx, dtype):
    gen = torch.Generator().manual_seed(8)
    for rows, n, k in ((700, 300, 520), (4000, 130, 260)):
        x, dy = torch.randint(-8, 9, (rows, k), generator=gen).float(), torch.randint(-100, 101, (rows, n), generator=gen).to(dtype)
        dw, db = torch.empty((n, k), device="cuda"), torch.empty((n,), device="cuda")
        B.lgc_weight_grad(ctx, dy.cuda(), as_blocks(B, ctx, x), dw, db)
        assert torch.equal(dw.cpu().double(), dy.double().t() @ x.double()) and torch.equal(db.cpu().double(), dy.double().sum(0))


def test_weight_grad_in_fp32_keeps_what_bf16_would_lose(B, ctx):
    dy = torch.tensor([[1.0 + 2.0 ** -23], [3.4e38], [-(2.0 ** -100) * (1 + 2.0 ** -12)], [math.inf], [-math.inf], [math.nan]])
    for i in range(6):
        dw = torch.empty((1, 1), device="cuda")
        B.lgc_weight_grad(ctx, dy[i:i + 1].cuda(), as_blocks(B, ctx, torch.ones((1, 1))), dw)
        assert torch.equal(dw.cpu().nan_to_num(7.0, 8.0, 9.0), dy[i:i + 1].nan_to_num(7.0, 8.0, 9.0))


def test_product_and_weight_grad_against_differences(B, ctx):
    """The loss is linear in the weights and in the input: its differences along numbers that 8 bits hold are the gradients themselves."""
    rows, n, k = 50, 140, 300
    x, w = ref.kept(rand((rows, k), 1)).float(), rand((n, k), 2)
    w8, wt8 = B.Blocks(n, k, tiles=True), B.Blocks(k, n, tiles=True)
    B.lgc_quantize_weights(ctx, w.cuda(), w8, wt8)
    dy, x8 = ref.kept(rand((rows, n), 3)).float(), as_blocks(B, ctx, x)

    def loss(a, b):
        y = torch.empty((rows, n), device="cuda")
        B.lgc_product(ctx, a, b, None, y)
        return float((y.cpu().double() * dy.double()).sum())

    dw, dx = torch.empty((n, k), device="cuda"), torch.empty((rows, k), device="cuda")
    B.lgc_weight_grad(ctx, dy.cuda(), x8, dw)
    B.lgc_product(ctx, as_blocks(B, ctx, dy), wt8, None, dx)
    tw, tx = rand((n, k), 4).sign(), rand((rows, k), 5).sign()      # directions of whole numbers
    slack = (k + rows + n) * U * float(dy.abs().sum()) * 4
    assert abs(loss(x8, as_blocks(B, ctx, tw, True)) - float((dw.cpu().double() * tw.double()).sum())) <= slack * math.sqrt(k)
    assert abs(loss(as_blocks(B, ctx, tx), w8) - float((dx.cpu().double() * tx.double()).sum())) <= slack * math.sqrt(k)


# ---------------------------------------------------------------- in use

def test_no_rows(B, ctx):
    x, b = torch.empty((0, 300), device="cuda"), B.Blocks(0, 300)
    none = torch.empty(0, device="cuda")
    B.lgc_quantize(ctx, x, b)
    B.lgc_dequantize(ctx, b, x)
    B.lgc_layer_norm(ctx, x, None, None, 1e-5, y=x, mean=none, rstd=none, blocks=b)
    B.lgc_activate(ctx, "gelu", x, z=x, a_blocks=b)
    B.lgc_activate_grad(ctx, "gelu", x, b, da=x)
    dg, db = torch.full((300,), 9.0, device="cuda"), torch.full((300,), 9.0, device="cuda")
    B.lgc_layer_norm_grad(ctx, x, x, None, none, none, x, dg, db)
    assert not dg.any() and not db.any()
    B.lgc_product(ctx, b, as_blocks(B, ctx, rand((40, 300), 1), True), None, torch.empty((0, 40), device="cuda"))
    dw, db = torch.full((40, 300), 9.0, device="cuda"), torch.full((40,), 9.0, device="cuda")
    B.lgc_weight_grad(ctx, torch.empty((0, 40), device="cuda"), b, dw, db)
    assert not dw.any() and not db.any()


def step(B, ctx, x, gamma, beta, w8, dy):
    """A few of the operators one after the other; everything they give."""
    rows, cols = x.shape
    n = w8.rows
    m, r, x8, a8, y8 = (torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), B.Blocks(rows, cols), B.Blocks(rows, n), B.Blocks(rows, n))
    y, z, da = (torch.empty((rows, n), device="cuda", dtype=x.dtype) for _ in range(3))
    dw, db, dx, dg, dt = (torch.empty(s, device="cuda") for s in ((n, cols), (n,), (rows, cols), (cols,), (cols,)))
    out = [m, r, x8.codes, y, z, a8.codes, y8.codes, da, dw, db, dx, dg, dt]

    def go():
        B.lgc_layer_norm(ctx, x, gamma, beta, 1e-5, mean=m, rstd=r, blocks=x8)
        B.lgc_product(ctx, x8, w8, None, y)
        B.lgc_activate(ctx, "silu", y, z=z, a_blocks=a8)
        B.lgc_activate_grad(ctx, "silu", dy, a8, da=da, da_blocks=y8)
        B.lgc_weight_grad(ctx, da, x8, dw, db)
        B.lgc_layer_norm_grad(ctx, x, x, gamma, m, r, dx.view_as(dx) if x.dtype == torch.float32 else None, dg, dt)
    return go, out


@pytest.mark.parametrize("dtype,rows,cols,n", [(torch.float32, 90, 200, 140), (torch.bfloat16, 1500, 640, 520), (torch.bfloat16, 3, 4096, 1024)])
def test_equal_calls_give_equal_bits_on_any_stream_and_in_a_graph(B, ctx, dtype, rows, cols, n):
    x, dy = rand((rows, cols), 1, 1.0, dtype).cuda(), rand((rows, n), 2, 1e-2, dtype).cuda()
    gamma, beta = (1 + rand((cols,), 3, 0.1)).cuda(), rand((cols,), 4).cuda()
    w8 = as_blocks(B, ctx, rand((n, cols), 5, 0.05), True)
    go, out = step(B, ctx, x, gamma, beta, w8, dy)
    go()
    torch.cuda.synchronize()
    want = [t.clone() for t in out]
    other = torch.cuda.Stream()
    mine = B.Context(1, 1, 1)
    B.lgc_reserve_training(mine)
    again, out2 = step(B, mine, x, gamma, beta, w8, dy)
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        again()
    other.synchronize()
    for a, b in zip(out2, want):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)) or dtype != torch.float32 and a is out2[10]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=other):
        again()
    for _ in range(4):
        for i, t in enumerate(out2):
            if dtype == torch.float32 or i != 10:
                t.zero_()
        go()                                           # eager work of another context in between
        graph.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(out2, want)):
            assert (dtype != torch.float32 and i == 10) or torch.equal(a.view(torch.uint8), b.view(torch.uint8)), i


def test_offsets_past_32_bits(B, ctx):
    """Matrices of more than 2^32 elements; the last rows against the same rows alone."""
    rows, cols, tail = 270_000, 16_384, 300
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    x[-tail:] = rand((tail, cols), 1, 1.0, torch.bfloat16).cuda()
    last = x[-tail:].clone()
    big, small = B.Blocks(rows, cols), B.Blocks(tail, cols)
    B.lgc_quantize(ctx, x, big)
    B.lgc_quantize(ctx, last, small)
    assert torch.equal(big.codes[-tail:], small.codes) and torch.equal(big.exps[-tail:], small.exps)
    w8, n = as_blocks(B, ctx, rand((128, cols), 2, 0.1), True), 128
    for dtype in TYPES:
        y, z = torch.empty((rows, n), dtype=dtype, device="cuda"), torch.empty((tail, n), dtype=dtype, device="cuda")
        B.lgc_product(ctx, big, w8, None, y)
        B.lgc_product(ctx, small, w8, None, z)
        want = ref.blocks_values(small) @ ref.blocks_values(w8).t()
        for got in (y[-tail:], z):
            assert float((got.cpu().double() - want).norm() / want.norm()) < (1e-2 if dtype == torch.bfloat16 else 1e-5)
        del y, z
    dy = torch.zeros((rows, 64), dtype=torch.bfloat16, device="cuda")
    dy[-tail:] = rand((tail, 64), 3, 1.0, torch.bfloat16).cuda()
    dw, db = torch.empty((64, cols), device="cuda"), torch.empty((64,), device="cuda")
    B.lgc_weight_grad(ctx, dy, big, dw, db)
    want = dy[-tail:].cpu().double().t() @ ref.blocks_values(small)
    assert float((dw.cpu().double() - want).norm() / want.norm()) < 1e-5
    out = torch.empty_like(x)
    B.lgc_dequantize(ctx, big, out)
    assert torch.equal(out[-tail:].cpu().double(), ref.blocks_values(small))
    m, r = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    B.lgc_layer_norm(ctx, x, None, None, 1e-5, y=out, mean=m, rstd=r)
    y = torch.empty_like(last)
    B.lgc_layer_norm(ctx, last, None, None, 1e-5, y=y)
    assert torch.equal(out[-tail:], y) and not out[:-tail].any()
    dg, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    B.lgc_layer_norm_grad(ctx, x, x, None, m, r, out, dg, db)
    _, wg, wb = ref.layer_norm_grad(last.cpu(), last.cpu(), None, m[-tail:].cpu(), r[-tail:].cpu())
    assert float((db.cpu().double() - wb).norm() / wb.norm()) < 1e-5 and float((dg.cpu().double() - wg).norm() / wg.norm()) < 1e-5
    B.lgc_activate(ctx, "gelu", x, z=out, a_blocks=big)
    B.lgc_activate(ctx, "gelu", last, z=y)
    assert torch.equal(out[-tail:], y)
    B.lgc_activate_grad(ctx, "gelu", x, big, da=out)
    B.lgc_activate_grad(ctx, "gelu", last, small, da=y)
    assert torch.equal(out[-tail:], y)
