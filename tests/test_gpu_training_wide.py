"""Products and weight gradients of widths at which other kernels, or other splits of the sum, serve them than small ones: against their definitions in 64 bits, within
bounds that follow from the format of what is stored and from the length of the fp32 sums (U: half a unit of an fp32 number's last place)."""
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


def as_blocks(B, ctx, x, tiles=False):
    b = B.Blocks(x.shape[0], x.shape[1], tiles=tiles)
    (B.lgc_quantize_weights if tiles else B.lgc_quantize)(ctx, x.cuda(), b)
    return b


def guarded(rows, cols, pad, dtype):
    """Rows cols + pad apart, and the array they lie in, all 7."""
    whole = torch.full((rows, cols + pad), 7.0, dtype=dtype, device="cuda")
    return whole[:, :cols], whole


# A block per compute unit and more of the largest tiles, with rows and columns that end inside one; few rows of many columns; a long sum of few tiles
PRODUCTS = [(4100, 4200, 300), (4133, 4229, 130), (6, 8300, 300), (20, 8421, 1000), (50, 8195, 700), (2, 130, 16000), (150, 700, 16000), (600, 600, 9000)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product(B, ctx, m, n, k, dtype):
    a = as_blocks(B, ctx, rand((m, k), m + n + k) * torch.exp(2 * rand((m, 1), k)))
    b = as_blocks(B, ctx, rand((n, k), n * k % 1000, 0.1), tiles=True)
    bias = rand((n,), 3).cuda()
    x, w = ref.blocks_values(a).cuda(), ref.blocks_values(b).cuda()
    size, exact = x.abs() @ w.abs().t(), x @ w.t()
    for add, pad in ((bias, 0), (None, 3)):
        y, whole = guarded(m, n, pad, dtype)
        B.lgc_product(ctx, a, b, add, y)
        want = exact if add is None else exact + add.double()
        # bf16: of eight neighbouring products each may lose 2^-14 of the largest; fp32: k additions at most
        bound = (2.0 ** -11 if dtype == torch.bfloat16 else (k + 16) * U) * size + STORE[dtype] * want.abs() + 4 * U * (1.0 if add is None else add.abs().double())
        assert ((y.double() - want).abs() <= bound).all()
        assert (whole[:, n:] == 7.0).all()


# One, two and many steps of many tiles; the largest tiles, whole and with edges; tiles that leave compute units idle and a long sum, in parts
WEIGHT_GRADS = [(1, 2100, 2200), (70, 2177, 2201), (130, 8192, 700), (513, 4096, 4096), (650, 4099, 4131), (6200, 1500, 1501), (700, 1500, 1536)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n,k", WEIGHT_GRADS)
def test_weight_grad(B, ctx, rows, n, k, dtype):
    x = as_blocks(B, ctx, rand((rows, k), rows + k) * torch.exp(2 * rand((rows, 1), n)))
    source = rand((rows, n), n + k, 1e-2, dtype).cuda()
    xv, yv = ref.blocks_values(x).cuda(), source.double()
    want, size = yv.t() @ xv, yv.abs().t() @ xv.abs()
    for pad in (0, 1):
        dy, _ = guarded(rows, n, pad, dtype)
        dy.copy_(source)
        dw, db = torch.full((n + 1, k), 7.0, device="cuda"), torch.full((n + 1,), 7.0, device="cuda")
        B.lgc_weight_grad(ctx, dy, x, dw[:n], db[:n])
        assert ((dw[:n].double() - want).abs() <= (rows + 64) * U * size + 1e-36).all()
        assert ((db[:n].double() - yv.sum(0)).abs() <= (rows + 64) * U * yv.abs().sum(0) + 1e-36).all()
        assert (dw[n] == 7.0).all() and db[n] == 7.0
        alone = torch.empty((n, k), device="cuda")
        B.lgc_weight_grad(ctx, dy, x, alone)
        assert torch.equal(alone, dw[:n])


# Sixteen wavefronts for few long rows; over 32 rows that tiles serve; large tiles that a third of the compute units has none of
@pytest.mark.parametrize("m,n,k", [(1, 8200, 8192), (13, 8321, 8300), (60, 2100, 16000), (50, 12100, 2500), (2900, 3000, 200)])
def test_product_between_kernels(B, ctx, m, n, k):
    test_product(B, ctx, m, n, k, torch.bfloat16)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(8200, 1500), (8193, 2048), (8192, 1025), (9000, 700)])
def test_layer_norm_of_many_rows(B, ctx, rows, cols, dtype):
    x = (rand((rows, cols), rows, 2.0) + 1.0).to(dtype).cuda()
    gamma, beta = rand((cols,), 1).cuda(), rand((cols,), 2).cuda()
    y, y8, mean, rstd = torch.empty_like(x), B.Blocks(rows, cols), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    B.lgc_layer_norm(ctx, x, gamma, beta, 1e-5, y=y, blocks=y8, mean=mean, rstd=rstd)
    d = x.double()
    mu = d.mean(1)
    r = ((d - mu[:, None]).square().mean(1) + 1e-5).rsqrt()
    want = (d - mu[:, None]) * r[:, None] * gamma.double() + beta.double()
    # sums of cols numbers about 2 in size, whose mean is off by cols / 4 units at most and their squares' by as much again
    close = cols * U
    assert ((mean.double() - mu).abs() <= close * d.abs().mean(1)).all() and ((rstd.double() - r).abs() <= close * r).all()
    bound = 4 * close * (1 + want.abs() + gamma.abs().double())
    assert ((y.double() - want).abs() <= bound + STORE[dtype] * want.abs()).all()
    out = torch.empty((rows, cols), device="cuda")
    B.lgc_dequantize(ctx, y8, out)
    most = torch.nn.functional.pad(want.abs(), (0, -cols % 128)).view(rows, -1, 128).amax(2).repeat_interleave(128, 1)[:, :cols]
    assert ((out.double() - want).abs() <= bound + want.abs() / 16 + most * 2.0 ** -17).all()   # half a unit of 3 bits; below them, half of 2^-9 of 2^-7 of the largest


# Rows in one launch, with the columns' sums in parts, and by blocks that go on from row to row: either side of where one gives way to another
NORM_GRADS = [(1024, 300), (1025, 300), (2047, 1111), (4096, 515), (4097, 515), (4099, 1000), (4101, 2000), (4097, 4000), (1025, 16000), (600, 16383), (1100, 8192), (4098, 40)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", NORM_GRADS)
def test_layer_norm_grad_of_many_rows(B, ctx, rows, cols, dtype):
    x, dy, gamma = (rand((rows, cols), rows, 2.0) + 1.0).to(dtype), rand((rows, cols), cols, 1e-2, dtype), rand((cols,), 1).cuda()
    x, dy = x.cuda(), dy.cuda()
    d = x.double()
    mean, rstd = d.mean(1).float(), ((d - d.mean(1, keepdim=True)).square().mean(1) + 1e-5).rsqrt().float()
    want, wg, wb = ref.layer_norm_grad(dy, x, gamma, mean, rstd)
    dx, dg, db = torch.full_like(x, 9.0), torch.full((cols,), 9.0, device="cuda"), torch.full((cols,), 9.0, device="cuda")
    B.lgc_layer_norm_grad(ctx, dy, x, gamma, mean, rstd, dx, dg, db)
    r = rstd.double()[:, None]
    hx = ((d - mean.double()[:, None]) * r).abs() + 2 * U * d.abs() * r
    q = dy.double().abs() * gamma.double().abs()
    # a row's sums: 16 additions in a thread and 10 among threads; the rest is a rounding or two of each factor
    bound = r * (8 * U * q + 64 * U * (q.mean(1, keepdim=True) + hx * (q * hx).mean(1, keepdim=True))) + (STORE[dtype] + 4 * U) * want.abs() + 1e-30
    assert ((dx.double() - want).abs() <= bound).all()
    assert ((dg.double() - wg).abs() <= (rows + 40) * U * (dy.double().abs() * hx).sum(0) + 4 * U * (dy.double().abs() * d.abs() * r).sum(0)).all()
    assert ((db.double() - wb).abs() <= (rows + 40) * U * dy.double().abs().sum(0)).all()
    again = [torch.empty_like(t) for t in (dx, dg, db)]
    B.lgc_layer_norm_grad(ctx, dy, x, gamma, mean, rstd, *again)
    assert all(torch.equal(a, b) for a, b in zip(again, (dx, dg, db)))
    alone = torch.empty_like(dg)
    B.lgc_layer_norm_grad(ctx, dy, x, gamma, mean, rstd, dgamma=alone)
    assert torch.equal(alone, dg)
    B.lgc_layer_norm_grad(ctx, dy, x, gamma, mean, rstd, again[0].zero_())
    assert torch.equal(again[0], dx)


# Large tiles: two steps and three, rows in parts; rows of dy so far apart that a step's distances pass 32 bits
@pytest.mark.parametrize("rows,n,k", [(128, 4200, 4100), (140, 4200, 4100), (6200, 1500, 3500)])
def test_weight_grad_by_large_tiles(B, ctx, rows, n, k):
    test_weight_grad(B, ctx, rows, n, k, torch.bfloat16)


@pytest.mark.parametrize("dtype", TYPES)
def test_weight_grad_of_rows_far_apart(B, ctx, dtype):
    rows, n, k, ld = 330, 130, 140, (1 << 24) + 8
    x = as_blocks(B, ctx, rand((rows, k), 1))
    dy = torch.empty(((rows - 1) * ld + n,), dtype=dtype, device="cuda").as_strided((rows, n), (ld, 1))
    dy.copy_(rand((rows, n), 2, 1e-2, dtype))
    xv, yv = ref.blocks_values(x).cuda(), dy.double()
    dw, db = torch.empty((n, k), device="cuda"), torch.empty((n,), device="cuda")
    B.lgc_weight_grad(ctx, dy, x, dw, db)
    assert ((dw.double() - yv.t() @ xv).abs() <= (rows + 64) * U * (yv.abs().t() @ xv.abs()) + 1e-36).all()
    assert ((db.double() - yv.sum(0)).abs() <= (rows + 64) * U * yv.abs().sum(0) + 1e-36).all()
