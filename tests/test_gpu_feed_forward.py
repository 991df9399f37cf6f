"""The feed-forward block that runs the training step's operators together: against the same steps in 64 bits, with the numbers
that 8 bits hold in the same places, against the block without 8 bits, and in the loop with the compression."""
import math

import pytest
import torch

import training_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def FF():
    from paper_2103_08870_amd import feed_forward
    assert torch.cuda.is_available()
    return feed_forward


def rand(shape, seed, scale=1.0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale


def tiles(w):
    c, e = ref.codes(w, 128)
    return ref.values(c, e, 128, w.shape[1])


def in_64_bits(block, x, dy, keep, weights):
    """y, dx and the six gradients; keep: what an 8-bit matrix makes of values, weights: of weights."""
    gamma, beta, w1, b1, w2, b2 = (p.double().cpu() for p in block.parts(block.flat))
    x, dy = x.double(), dy.double()
    h, mean, rstd = ref.layer_norm(x, gamma, beta, 1e-5)
    h = keep(h)
    a = h @ weights(w1).t() + b1
    z, kept = keep(ref.act(block.act, a)), keep(a)
    y = x + z @ weights(w2).t() + b2
    da = keep(dy) @ weights(w2) * ref.act_slope(block.act, kept)
    dx, dgamma, dbeta = ref.layer_norm_grad(keep(da) @ weights(w1), x, gamma, mean, rstd)
    return y, dy + dx, [dgamma, dbeta, da.t() @ h, da.sum(0), dy.t() @ z, dy.sum(0)]


@pytest.mark.parametrize("rows,width,hidden,act", [(300, 256, 640, "gelu"), (257, 200, 333, "silu"), (1, 128, 512, "gelu"), (1100, 512, 1024, "relu")])
def test_block(FF, rows, width, hidden, act):
    block = FF.FeedForward(rows, width, hidden, act=act, seed=3)
    with torch.no_grad():
        block.flat.add_(rand(block.flat.shape, 5, 0.02).cuda())
    block.refresh()
    x, dy = rand((rows, width), 1).to(torch.bfloat16), rand((rows, width), 2, 1e-3).to(torch.bfloat16)
    grad = torch.full_like(block.flat, 7.0)
    y = block.forward(x.cuda())
    dx = block.backward(dy.cuda(), grad)
    got = [y, dx] + block.parts(grad)
    # bf16 between the operators: 2^-8 of each value, which may move a value that 8 bits hold by a step of 2^-3 where it lies at the edge of one
    # (of 2^-8 / 2^-3 of them): sqrt(2^-5) 2^-3 of the norm, over four such places; without 8 bits, 2^-4 / sqrt(3) at each of six places
    for keep, weights, bound in ((ref.kept, tiles, 4 * math.sqrt(2.0 ** -5) * 2.0 ** -3), (lambda t: t, lambda t: t, 6 * 2.0 ** -4 / math.sqrt(3))):
        wy, wdx, wg = in_64_bits(block, x, dy, keep, weights)
        for a, b in zip(got, [wy, wdx] + wg):
            assert float((a.cpu().double() - b).norm() / b.norm()) < bound, (a.shape, bound)


def test_the_gradient_s_place_in_a_flat_vector_may_have_any_alignment(FF):
    block = FF.FeedForward(100, 130, 257, seed=1)      # every tensor after the first starts at an odd place
    x, dy = rand((100, 130), 1).to(torch.bfloat16).cuda(), rand((100, 130), 2, 1e-3).to(torch.bfloat16).cuda()
    grads = [torch.empty(block.flat.numel() + 3, device="cuda")[i:i + block.flat.numel()] for i in range(3)]
    for g in grads:
        block.forward(x)
        block.backward(dy, g)
    assert torch.equal(grads[0], grads[1]) and torch.equal(grads[0], grads[2]) and bool(grads[0].isfinite().all())


def test_training_with_sparse_gradients_lowers_the_loss(FF):
    losses = FF.train(nodes=2, rows=512, width=256, hidden=512, iterations=25)
    assert all(math.isfinite(x) for x in losses) and losses[-1] < 0.8 * losses[0], losses
    assert losses == FF.train(nodes=2, rows=512, width=256, hidden=512, iterations=25)      # the same bits again
