"""Products of wide outputs with long sums, at the sizes of large models' layers: against 64 bits on the GPU, from codes made there."""
import pytest
import torch

import training_reference as ref

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
STORE = {torch.float32: U, torch.bfloat16: 2.0 ** -8}      # rounding of a stored result (bf16: a whole unit)


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


def made(B, rows, cols, tiles, gen):
    """Blocks with numbers of every size that a code has, and their values in 64 bits."""
    b = B.Blocks(rows, cols, tiles=tiles)
    b.codes.zero_()
    c = torch.randint(0, 127, (rows, cols), generator=gen, device="cuda") + 128 * torch.randint(0, 2, (rows, cols), generator=gen, device="cuda")
    b.codes[:, :cols] = c.to(torch.uint8)
    b.exps.copy_(torch.randint(118, 124, b.exps.shape, generator=gen, device="cuda"))
    v = ref.NUMBERS.cuda()[c & 127] * torch.where(c > 127, -1.0, 1.0).double()
    del c
    per = 128 if tiles else 1
    scale = torch.exp2(b.exps.double() - 127)[:, :(cols + 127) // 128]
    for r in range(0, rows, 4096):      # (a few rows at a time: the scale of every element is as large as the values)
        part = scale[r // per:(min(r + 4096, rows) - 1) // per + 1].repeat_interleave(per, 0)[:min(4096, rows - r)]
        v[r:r + 4096] *= part.repeat_interleave(128, 1)[:, :cols]
    return b, v


# Large tiles on fewer than all compute units, and sums over 60 blocks of columns and more (the last one: 129 tiles of an odd width)
@pytest.mark.parametrize("m,n,k", [(280, 28672, 8192), (700, 11000, 14000), (129, 32801, 12288), (513, 15000, 16384), (900, 8300, 16384)])
def test_product_to_bf16(B, ctx, m, n, k):
    gen = torch.Generator(device="cuda").manual_seed(m)
    a, x = made(B, m, k, False, gen)
    b, w = made(B, n, k, True, gen)
    other, _ = made(B, 600, 9000, True, gen)
    few, _ = made(B, 600, 9000, False, gen)
    wt = w.t().contiguous()
    exact = x @ wt
    size = x.abs_() @ wt.abs_()
    del x, w, wt
    bias = torch.randn(n, generator=gen, device="cuda") * float(exact.std())
    for add, pad in ((bias, 0), (None, 3)):
        # what another call leaves in the scratch must not matter: a product of few tiles puts its parts there
        B.lgc_product(ctx, few, other, None, torch.empty((600, 600), device="cuda"))
        whole = torch.full((m, n + pad), 7.0, dtype=torch.bfloat16, device="cuda")
        y = whole[:, :n]
        B.lgc_product(ctx, a, b, add, y)
        want = exact if add is None else exact + add.double()
        # of eight neighbouring products each may lose 2^-14 of the largest
        bound = 2.0 ** -11 * size + STORE[torch.bfloat16] * want.abs() + 4 * U * (1.0 if add is None else add.abs().double())
        assert ((y.double() - want).abs() <= bound).all()
        assert (whole[:, n:] == 7.0).all()
