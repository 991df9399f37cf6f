"""What the training step's calls refuse with a context in hand: an error with a message, nothing launched."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2103_08870_amd import binding
    binding.lib()
    assert torch.cuda.is_available()
    return binding


def test_the_calls_refuse_bad_arguments_and_say_why(B):
    ctx = B.Context(1, 1, 1)
    t = torch.full((64, 256), 7.0, device="cuda")
    p, h, lib = t.data_ptr(), ctx.h, B.lib()
    q, far = p + 32768, 1 << 30

    def refused(word, name, *args):
        assert getattr(lib, name)(h, *args) == B.LGC_EINVAL, (name, args)
        assert word in lib.lgc_last_error(h), lib.lgc_last_error(h)

    refused(b"lgc_reserve_training", "lgc_product", p, p, 1, p, p, 128, 128, None, q, 0, 128, None)
    refused(b"lgc_reserve_training", "lgc_weight_grad", p, 0, 1, 128, 128, p, p, 128, q, None, None)
    refused(b"lgc_reserve_training", "lgc_layer_norm_grad", p, 128, p, 128, 0, 1, 128, None, p, p, q, 128, None, None, None)
    B.lgc_reserve_training(ctx)
    B.lgc_reserve_training(ctx)
    for cols in (0, (1 << 20) + 1):
        refused(b"cols", "lgc_quantize", p, 0, 1, cols, far, q, q, None)
        refused(b"cols", "lgc_layer_norm", p, 0, 1, cols, far, None, None, 1e-5, q, far, None, None, None, None, None)
        refused(b"cols", "lgc_activate", 0, p, 0, 1, cols, far, q, far, None, None, None, None, None)
        refused(b"k =", "lgc_product", p, p, 1, p, p, 128, cols, None, q, 0, 128, None)
        refused(b"n =", "lgc_weight_grad", p, 0, 1, cols, far, p, p, 128, q, None, None)
    for rows in (1 << 31, 1 << 30):
        refused(b"rows", "lgc_quantize", p, 0, rows, 128, 128, q, q, None)
        refused(b"rows", "lgc_activate_grad", 0, p, 0, rows, 128, 128, p, p, q, 128, None, None, None)
    refused(b"type", "lgc_quantize", p, 2, 1, 128, 128, q, q, None)
    refused(b"non-linearity", "lgc_activate", 3, p, 0, 1, 128, 128, q, 128, None, None, None, None, None)
    refused(b"x is NULL", "lgc_quantize", None, 0, 1, 128, 128, q, q, None)
    refused(b"codes", "lgc_quantize", p, 0, 1, 128, 128, None, q, None)
    refused(b"codes", "lgc_quantize", p, 0, 1, 128, 128, q + 8, q, None)
    refused(b"exponents", "lgc_quantize", p, 0, 1, 128, 128, q, q + 1, None)
    refused(b"aligned", "lgc_quantize", p + 2, 0, 1, 128, 128, q, q, None)
    refused(b"aligned", "lgc_quantize", p + 1, 1, 1, 128, 128, q, q, None)
    refused(b"apart", "lgc_quantize", p, 0, 2, 128, 127, q, q, None)
    refused(b"exp_rows", "lgc_dequantize", p, p, 2, 1, 128, q, 0, 128, None)
    refused(b"eps", "lgc_layer_norm", p, 0, 1, 128, 128, None, None, -1.0, q, 128, None, None, None, None, None)
    refused(b"eps", "lgc_layer_norm", p, 0, 1, 128, 128, None, None, float("nan"), q, 128, None, None, None, None, None)
    refused(b"mean", "lgc_layer_norm_grad", p, 128, p, 128, 0, 1, 128, None, None, p, q, 128, None, None, None)
    refused(b"y", "lgc_layer_norm", p, 0, 1, 128, 128, None, None, 1e-5, q, 128, None, None, q, None, None)
    refused(b"transpose", "lgc_quantize_weights", p, 0, 128, 128, 128, q, q, q, None, None)
    refused(b"rows", "lgc_quantize_weights", p, 0, 0, 128, 128, q, q, None, None, None)
    refused(b"dw", "lgc_weight_grad", p, 0, 1, 128, 128, p, p, 128, None, None, None)
    refused(b"bias", "lgc_product", p, p, 1, p, p, 128, 128, p + 2, q, 0, 128, None)
    torch.cuda.synchronize()
    assert bool((t == 7.0).all())
    ctx.close()


def test_the_binding_refuses_tensors_that_do_not_fit(B):
    ctx = B.Context(1, 1, 1)
    B.lgc_reserve_training(ctx)
    x, b = torch.zeros((4, 200), device="cuda"), B.Blocks(4, 200)
    w8 = B.Blocks(64, 200, tiles=True)
    v = torch.zeros(200, device="cuda")
    for call in (lambda: B.lgc_quantize(ctx, x.half(), b), lambda: B.lgc_quantize(ctx, x.t(), b), lambda: B.lgc_quantize(ctx, x[:3], b),
                 lambda: B.lgc_quantize(ctx, x, B.Blocks(4, 200, tiles=True)), lambda: B.lgc_quantize(ctx, x.cpu(), b),
                 lambda: B.lgc_quantize_weights(ctx, x, b), lambda: B.lgc_dequantize(ctx, b, x[:, :100]),
                 lambda: B.lgc_layer_norm(ctx, x, v[:100], None, 1e-5, y=x), lambda: B.lgc_layer_norm(ctx, x, v.bfloat16(), None, 1e-5, y=x),
                 lambda: B.lgc_layer_norm(ctx, x, None, None, 1e-5, y=x.bfloat16()), lambda: B.lgc_layer_norm_grad(ctx, x, x, None, v, v),
                 lambda: B.lgc_activate(ctx, "tanh", x, z=x), lambda: B.lgc_product(ctx, b, b, None, torch.zeros((4, 4), device="cuda")),
                 lambda: B.lgc_product(ctx, b, w8, None, torch.zeros((4, 63), device="cuda")),
                 lambda: B.lgc_product(ctx, b, w8, v, torch.zeros((4, 64), device="cuda")),
                 lambda: B.lgc_weight_grad(ctx, torch.zeros((5, 64), device="cuda"), b, torch.zeros((64, 200), device="cuda")),
                 lambda: B.lgc_weight_grad(ctx, torch.zeros((4, 64), device="cuda"), b, torch.zeros((64, 199), device="cuda"))):
        with pytest.raises(ValueError):
            call()
    ctx.close()


def test_a_weight_gradient_laid_out_as_the_transpose_is_refused(B):
    """dw is [n][k], or that many elements in a row: a matrix of another shape with as many elements would get its rows cut in the wrong places."""
    ctx = B.Context(1, 1, 1)
    B.lgc_reserve_training(ctx)
    gen = torch.Generator().manual_seed(1)
    dy, b = torch.randn((4, 64), generator=gen).cuda(), B.Blocks(4, 200)
    B.lgc_quantize(ctx, torch.randn((4, 200), generator=gen).cuda(), b)
    for shape in ((200, 64), (128, 100), (1, 12800), (12800, 1)):
        dw = torch.full(shape, 7.0, device="cuda")
        with pytest.raises(ValueError):
            B.lgc_weight_grad(ctx, dy, b, dw)
        torch.cuda.synchronize()
        assert bool((dw == 7.0).all())
    same = [torch.empty(shape, device="cuda") for shape in ((64, 200), (12800,), (64, 8, 25), (2, 32, 200))]
    for dw in same:
        B.lgc_weight_grad(ctx, dy, b, dw)
        assert torch.equal(dw.view(64, 200), same[0]) and bool(dw.any())
    ctx.close()
