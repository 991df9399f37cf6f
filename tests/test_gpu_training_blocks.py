"""The arrays of a Blocks are those that it has when a call is made, and fit it then."""
import pytest
import torch

import training_reference as ref

pytestmark = pytest.mark.gpu


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


def arrays(b):
    return torch.full_like(b.codes, 0x55), torch.full_like(b.exps, 99)


def exchange(how, b, codes, exps):
    if how == "assigned":
        b.codes, b.exps = codes, exps
    elif how == "set":                       # the same tensors, with other memory
        b.codes.set_(codes)
        b.exps.set_(exps)
    else:
        b.codes.data, b.exps.data = codes, exps


@pytest.mark.parametrize("how", ["assigned", "set", "data"])
def test_exchanged_arrays_take_effect(B, ctx, how):
    x = torch.randn((5, 300), generator=torch.Generator().manual_seed(1))
    b, want = B.Blocks(5, 300), ref.kept(x)
    keep = b.codes.view(-1), b.exps.view(-1)                 # (the first arrays live on, and are seen to be left alone)
    for t in keep:
        t.fill_(0x33)
    codes, exps = arrays(b)
    exchange(how, b, codes, exps)
    B.lgc_quantize(ctx, x.cuda(), b)
    assert all(bool((t == 0x33).all()) for t in keep)
    assert b.codes.data_ptr() == codes.data_ptr() and torch.equal(ref.blocks_values(b), want)
    out = torch.empty((5, 300), device="cuda")
    B.lgc_dequantize(ctx, b, out)
    assert torch.equal(out.cpu().double(), want)
    y, w8 = torch.empty((5, 7), device="cuda"), B.Blocks(7, 300, tiles=True)
    w = torch.randn((7, 300), generator=torch.Generator().manual_seed(2)).cuda()
    first = w8.codes.view(-1), w8.exps.view(-1)
    for t in first:
        t.zero_()
    exchange(how, w8, *arrays(w8))
    B.lgc_quantize_weights(ctx, w, w8)
    B.lgc_product(ctx, b, w8, None, y)
    assert float((y.cpu().double() - want @ ref.blocks_values(w8).t()).abs().max()) < 1e-3 and not any(bool(t.any()) for t in first)


def test_arrays_that_do_not_fit_are_refused(B, ctx):
    b, x = B.Blocks(5, 300), torch.zeros((5, 300), device="cuda")
    codes, exps = b.codes, b.exps
    for name, bad in (("codes", codes[:4]), ("codes", codes[:, :256]), ("codes", codes.int()), ("codes", codes.cpu()), ("codes", codes.t()), ("codes", None), ("exps", exps[:4]),
                      ("exps", exps.float()), ("exps", exps[:, :3]), ("rows", 50), ("cols", 301), ("tiles", True)):
        with pytest.raises((ValueError, AttributeError)):
            setattr(b, name, bad)
    assert b.codes is codes and b.exps is exps and (b.rows, b.cols, b.tiles) == (5, 300, False)
    other = torch.empty((4, 384), dtype=torch.uint8, device="cuda")
    codes.set_(other)                                         # smaller, by the tensor's own means: seen by the next call
    with pytest.raises(ValueError):
        B.lgc_quantize(ctx, x, b)
    codes.set_(torch.empty((5, 384), dtype=torch.uint8, device="cuda"))
    B.lgc_quantize(ctx, x, b)
    assert not b.codes.any()


@pytest.mark.parametrize("name", ["codes", "exps"])
def test_arrays_whose_memory_is_gone_are_refused(B, ctx, name):
    b, x = B.Blocks(5, 300), torch.zeros((5, 300), device="cuda")
    getattr(b, name).untyped_storage().resize_(0)
    with pytest.raises(ValueError):
        B.lgc_quantize(ctx, x, b)
