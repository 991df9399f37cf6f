"""The training step's kernels where they go on from row to row or end inside a group of blocks, and the tiled weight gradient on numbers that are not finite: sizes that launch
them (test_training_launches.py holds them to that), compared as small ones are."""
import math

import pytest
import torch

import test_gpu_training as small
import test_gpu_training_wide as wide
import training_reference as ref

pytestmark = pytest.mark.gpu

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


# More rows than blocks, so that a block goes on to a second row with the first one's sums still in LDS
NORMS = {(9000, 300): "k_norm 64 1", (5000, 1000): "k_norm 64 2", (3000, 1500): "k_norm 256 1", (2500, 4000): "k_norm 256 2", (2500, 4099): "k_norm 512 2", (2200, 8000): "k_norm 512 2",
         (1500, 16000): "k_norm 1024 2"}
# (the last: columns' sums over several rows of each block)
NORM_GRADS = {(1300, 8192): "k_norm_grad 1024 1", (4100, 5001): "k_norm_grad 1024 1", (4100, 4000): "k_norm_grad 512 1", (200, 16400): "k_norm_grad_columns"}
GROUPS = (4099, 1100)      # 36891 blocks of 128 columns: groups of four, the last of which ends inside


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", NORMS)
def test_layer_norm(B, ctx, rows, cols, dtype):
    wide.test_layer_norm_of_many_rows(B, ctx, rows, cols, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", NORM_GRADS)
def test_layer_norm_grad(B, ctx, rows, cols, dtype):
    wide.test_layer_norm_grad_of_many_rows(B, ctx, rows, cols, dtype)


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_and_back_in_groups(B, ctx, dtype):
    small.test_quantize_and_back(B, ctx, *GROUPS, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", small.ACTS)
def test_activate_and_its_gradient_in_groups(B, ctx, kind, dtype):
    small.test_activate_and_its_gradient(B, ctx, *GROUPS, kind, dtype)


# Tiles of two teams (fp32: of one), several steps of 64 rows, the last not whole; large tiles; the rows in parts
WEIGHT_GRADS = {(330, 130, 140): "k_weight_grad 64 64 4", (300, 4200, 4100): "k_weight_grad", (3001, 300, 260): "k_weight_grad 64 64 4"}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n,k", WEIGHT_GRADS)
def test_weight_grad_of_numbers_that_are_not_finite(B, ctx, rows, n, k, dtype):
    gen = torch.Generator().manual_seed(rows)
    x = torch.randint(-2, 3, (rows, k), generator=gen) * 0.5          # 8 bits hold them; zeros among them, which infinities make NaN
    x[rows // 2, 5], x[rows - 1, 77] = math.nan, math.inf             # both NaN in 8 bits
    x8 = small.as_blocks(B, ctx, x)
    dy = small.rand((rows, n), n, 1e-2, dtype)
    most, tiny = torch.finfo(dtype).max, -(2.0 ** -100) * (1 + 2.0 ** -12)
    special = {3: (0, math.inf), 10: (rows // 2, -math.inf), 33: (rows - 1, math.inf), 64: (70, math.nan), 100: (rows - 2, -math.nan), 129: (64, math.inf)}
    alone = {0: (1, most), 7: (rows - 1, 3.38e38), 31: (rows // 2 + 1, -most), 65: (63, tiny), 127: (rows - 3, 1 + 2.0 ** -23)}
    for c, (t, v) in special.items():
        dy[t, c] = v
    dy[200 % rows, 3] = -math.inf                                      # two infinities of either sign in one sum
    for c, (t, v) in alone.items():
        dy[:, c] = 0.0
        dy[t, c] = v
    for pad in (0, 1):
        given, _ = wide.guarded(rows, n, pad, dtype)
        given.copy_(dy)
        dw, db = torch.full((n, k), 7.0, device="cuda"), torch.full((n,), 7.0, device="cuda")
        B.lgc_weight_grad(ctx, given, x8, dw, db)
        xv, yv = ref.blocks_values(x8).cuda(), given.double()
        lost = xv.isnan().any(0)                                       # columns of x with a NaN: NaN whatever meets it
        assert int(lost.sum()) == 2 and bool(dw[:, lost].isnan().all())
        for c in special:
            want = (yv[:, c:c + 1] * xv).sum(0)
            assert not bool(want.isfinite().any()), c
            assert torch.equal(dw[c].double().nan_to_num(1.0, 2.0, 3.0), want.nan_to_num(1.0, 2.0, 3.0)), c
            assert torch.equal(db[c].double().nan_to_num(1.0, 2.0, 3.0), yv[:, c].sum().nan_to_num(1.0, 2.0, 3.0)), c
        for c, (t, _) in alone.items():                                # one product and zeros: exact, in fp32 all 24 bits of it
            assert torch.equal(dw[c].double()[~lost], (yv[t, c] * xv[t])[~lost]) and float(db[c]) == float(yv[t, c]), c
        rest = torch.ones(n, dtype=torch.bool, device="cuda")
        rest[list(special) + list(alone)] = False
        y, v = yv[:, rest], xv[:, ~lost]
        assert ((dw[rest][:, ~lost].double() - y.t() @ v).abs() <= (rows + 64) * small.U * (y.abs().t() @ v.abs()) + 1e-36).all()
        assert ((db[rest].double() - y.sum(0)).abs() <= (rows + 64) * small.U * y.abs().sum(0) + 1e-36).all()
