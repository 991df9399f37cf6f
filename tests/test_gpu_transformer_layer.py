"""The layer that runs attention, rotary positions and the products with epilogues together: against the same steps in 64 bits, with the numbers that 8 bits hold in the same places; packed sequences
against each by itself; token by token against all at once; in the loop with the compression."""
import math

import pytest
import torch

import training_reference as ref
from attention_reference import visible

pytestmark = pytest.mark.gpu

# bf16 between the operators: 2^-8 of each value, which may move a value that 8 bits hold by a step of 2^-3 where it lies at the edge of one (of 2^-8 / 2^-3 of them): this much of
# the norm at each place where 8 bits hold something (and some tenths of it for bf16 itself)
EDGE = math.sqrt(2.0 ** -5) * 2.0 ** -3


@pytest.fixture(scope="module")
def T():
    from paper_2103_08870_amd import transformer_layer
    assert torch.cuda.is_available()
    return transformer_layer


def rand(shape, seed, scale=1.0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale


class Kept(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x):
        return ref.kept(x)

    @staticmethod
    def backward(ctx, g):
        return g


class Linear(torch.autograd.Function):
    """x W^T + b of 8-bit weights; the input's gradient from the output's in 8 bits, the weights' from all of it."""
    @staticmethod
    def forward(ctx, x, w, b):
        c, e = ref.codes(w, 128)
        w = ref.values(c, e, 128, w.shape[1])
        ctx.save_for_backward(x, w)
        return x @ w.t() + b

    @staticmethod
    def backward(ctx, g):
        x, w = ctx.saved_tensors
        return ref.kept(g) @ w, g.t() @ x, g.sum(0)


class Act(torch.autograd.Function):
    """The slope at what 8 bits hold of the argument."""
    @staticmethod
    def forward(ctx, t, name):
        ctx.save_for_backward(ref.kept(t))
        ctx.name = name
        return ref.act(name, t)

    @staticmethod
    def backward(ctx, g):
        return g * ref.act_slope(ctx.name, ctx.saved_tensors[0]), None


def norm(x, gamma, beta):
    return Kept.apply(torch.nn.functional.layer_norm(x, (x.shape[1],), gamma, beta, 1e-5))


def rotated(x, positions, heads, dim):
    x = x.view(x.shape[0], heads, 2, dim // 2)
    t = positions.double()[:, None] * 10000.0 ** (-torch.arange(dim // 2, dtype=torch.float64) * 2 / dim)
    c, s = torch.cos(t)[:, None], torch.sin(t)[:, None]
    a, b = x.unbind(2)
    return torch.stack([a * c - b * s, a * s + b * c], 2).flatten(1)


def in_64_bits(layer, x, dy, lengths):
    """y, dx and the gradient of `flat`."""
    at, ff = layer.attention, layer.feed_forward
    flat = layer.flat.double().cpu().requires_grad_()
    gamma, beta, w, b, wo, bo = at.parts(flat[:layer.cut])
    x = x.double().cpu().requires_grad_()
    qkv = Linear.apply(norm(x, gamma, beta), w, b)
    wide, both = at.heads * at.dim, (at.heads + at.kv_heads) * at.dim
    positions = torch.cat([torch.arange(n) for n in lengths])
    qk, v = rotated(qkv[:, :both], positions, at.heads + at.kv_heads, at.dim), qkv[:, both:]
    out, first = [], 0
    for n in lengths:
        q, k, u = (t[first:first + n].view(n, -1, at.dim).transpose(0, 1) for t in (qk[:, :wide], qk[:, wide:], v))
        k, u = (t.repeat_interleave(at.heads // at.kv_heads, 0) for t in (k, u))
        s = (q @ k.transpose(1, 2) * at.dim ** -0.5).masked_fill(~visible(n, n, True, at.window), -math.inf)
        out.append((torch.softmax(s, 2) @ u).transpose(0, 1).reshape(n, -1))
        first += n
    y = x + Linear.apply(Kept.apply(torch.cat(out)), wo, bo)
    gamma, beta, w1, b1, w2, b2 = ff.parts(flat[layer.cut:])
    y = y + Linear.apply(Kept.apply(Act.apply(Linear.apply(norm(y, gamma, beta), w1, b1), ff.act)), w2, b2)
    y.backward(dy.double().cpu())
    return y.detach(), x.grad, flat.grad


def made(T, *args, **how):
    layer = T.Layer(*args, **how)
    layer.flat.add_(rand(layer.flat.shape, 5, 0.02).cuda())
    layer.refresh()
    return layer


def far(got, want):
    return float((got.cpu().double() - want).norm() / want.norm())


@pytest.mark.parametrize("rows,width,heads,kv_heads,dim,hidden,how", [(300, 256, 4, 2, 64, 640, dict(sequences=2)), (257, 200, 6, 2, 40, 333, dict(act="silu", window=60)),
                                                                      (70, 131, 3, 1, 8, 77, {}), (1, 128, 2, 1, 64, 512, {}), (512, 512, 4, 4, 128, 1024, dict(act="relu"))])
def test_layer(T, rows, width, heads, kv_heads, dim, hidden, how):
    layer = made(T, rows, width, heads, kv_heads, dim, hidden, seed=3, **how)
    x, dy = rand((rows, width), 1).to(torch.bfloat16).cuda(), rand((rows, width), 2, 1e-3).to(torch.bfloat16).cuda()
    grad = torch.full_like(layer.flat, 7.0)
    y = layer.forward(x)
    dx = layer.backward(dy, grad)
    sequences = how.get("sequences", 1)
    wy, wdx, wg = in_64_bits(layer, x, dy, [rows // sequences] * sequences)
    assert far(y, wy) < 4 * EDGE                                     # h, o, h and z in 8 bits
    assert far(dx, wdx) < 9 * EDGE                                   # and t, dy, dt, dy, dqkv
    at, ff = layer.attention, layer.feed_forward
    for got, want in zip(at.parts(grad[:layer.cut]) + ff.parts(grad[layer.cut:]), at.parts(wg[:layer.cut]) + ff.parts(wg[layer.cut:])):
        assert far(got, want) < 9 * EDGE, got.shape


def test_packed_sequences(T):
    """Sequences of different lengths in one batch: each as by itself, rows of none without influence."""
    lengths, width = [100, 1, 40, 59], 256
    layer = made(T, 220, width, 4, 2, 64, 512, seed=4)
    x, dy = rand((220, width), 1).to(torch.bfloat16).cuda(), rand((220, width), 2, 1e-3).to(torch.bfloat16).cuda()
    starts = torch.tensor([5, 105, 106, 146, 205], dtype=torch.int32, device="cuda")
    grad, other = torch.empty_like(layer.flat), torch.empty_like(layer.flat)
    dy[:5], dy[205:] = 0.0, 0.0
    y = layer.forward(x, starts)
    dx = layer.backward(dy, grad)
    wy, wdx, wg = in_64_bits(layer, x[5:205], dy[5:205], lengths)
    assert far(y[5:205], wy) < 4 * EDGE and far(dx[5:205], wdx) < 9 * EDGE and far(grad, wg) < 9 * EDGE and bool((dx[:5] == 0).all()) and bool((dx[205:] == 0).all())
    x2 = x.clone()
    x2[:5], x2[205:] = 3.0, -2.0
    y2 = layer.forward(x2, starts)
    dx2 = layer.backward(dy, other)
    assert torch.equal(y2[5:205], y[5:205]) and torch.equal(dx2, dx) and far(other, grad.double().cpu()) < 2.0 ** -18


def test_token_by_token(T):
    """A cache with room for more: every token as when all are given at once."""
    sequences, length, more, width = 3, 50, 20, 256
    layer = made(T, sequences * (length + more), width, 4, 2, 64, 512, sequences=sequences, seed=6)
    prompt = T.Layer(sequences * length, width, 4, 2, 64, 512, sequences=sequences, ctx=layer.ctx)
    prompt.flat.copy_(layer.flat)
    prompt.refresh()
    x = rand((sequences, length + more, width), 1).to(torch.bfloat16).cuda()
    want = layer.forward(x.reshape(-1, width)).view(x.shape)
    cache = T.Cache(sequences, length + more + 7, 2 * 64)
    cache.k.fill_(math.nan)
    cache.v.fill_(math.inf)                            # what no token has been put to
    got = [prompt.forward(x[:, :length].reshape(-1, width), cache=cache).view(sequences, length, width)]
    got += [prompt.step(x[:, length + i].contiguous(), cache)[:, None] for i in range(more)]
    assert far(torch.cat(got, 1), want.double().cpu()) < 4 * EDGE
    assert cache.lengths.tolist() == [length + more] * sequences
    with pytest.raises(ValueError):
        prompt.forward(x[:, :length].reshape(-1, width), cache=cache)
    cache.most = cache.capacity
    with pytest.raises(ValueError):
        prompt.step(x[:, 0].contiguous(), cache)


def test_steps_in_a_graph(T):
    """One recorded step, replayed as the cache grows."""
    layer = made(T, 2 * 30, 128, 2, 1, 64, 256, sequences=2, seed=7)
    x = rand((60, 128), 1).to(torch.bfloat16).cuda()
    new = rand((5, 2, 128), 2).to(torch.bfloat16).cuda()
    caches = [T.Cache(2, 64, 64) for _ in range(2)]
    for c in caches:
        layer.forward(x, cache=c)
    want = [layer.step(t, caches[0]) for t in new]
    token = new[0].clone()
    layer.step(token, T.Cache(2, 64, 64))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = layer.step(token, caches[1])
    for t, w in zip(new, want):
        token.copy_(t)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, w)
        layer.forward(x)


def test_the_loop_and_the_continuation_run(T):
    losses = T.train(nodes=2, sequences=2, length=100, width=128, heads=4, kv_heads=2, dim=32, hidden=256, iterations=3)
    assert all(math.isfinite(x) for x in losses)
    assert losses == T.train(nodes=2, sequences=2, length=100, width=128, heads=4, kv_heads=2, dim=32, hidden=256, iterations=3)      # the same bits again
    layer = T.Layer(2 * 30, 128, 2, 1, 64, 256, sequences=2)
    assert bool(T.continued(layer, rand((60, 128), 1).to(torch.bfloat16).cuda(), 4).isfinite().all())
