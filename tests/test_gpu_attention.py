"""Attention and its gradient against their definitions in 64 bits, within bounds that follow from where numbers are rounded (attention_reference.py); gradients against differences; what is hidden
without influence, whatever it is; rows of no sequence let be; strides, far places, streams and graphs."""
import math
import threading

import pytest
import torch

import attention_reference as ref

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
KEEP = 7.0     # what outputs hold before a call


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


def rand(rows, cols, seed, scale=1.0):
    return (torch.randn((rows, cols), generator=torch.Generator().manual_seed(seed)) * scale).to(BF16).cuda()


class Case:
    def __init__(self, lq, lk, heads, kv_heads, dim, sequences=1, starts=None, causal=True, window=0, scale=None, seed=0):
        self.heads, self.kv_heads, self.dim, self.rows, self.keys = heads, kv_heads, dim, lq, lk
        self.q, self.k, self.v = rand(lq, heads * dim, seed, 2.0), rand(lk, kv_heads * dim, seed + 1), rand(lk, kv_heads * dim, seed + 2)
        self.do = rand(lq, heads * dim, seed + 3)
        self.scale = scale if scale is not None else dim ** -0.5
        self.how = dict(sequences=sequences, causal=causal, window=window)
        self.starts = starts

    def shape(self, B):
        starts = {} if self.starts is None else {n: torch.tensor(s, dtype=torch.int32, device="cuda") for n, s in zip(("q_starts", "kv_starts"), self.starts)}
        return B.AttentionShape(self.heads, self.kv_heads, self.dim, scale=self.scale, **self.how, **starts)

    def definition(self):
        starts = {} if self.starts is None else dict(q_starts=self.starts[0], kv_starts=self.starts[1])
        return dict(heads=self.heads, kv_heads=self.kv_heads, dim=self.dim, scale=self.scale, **self.how, **starts)

    def forward(self, B, ctx):
        o, lse = torch.full_like(self.q, KEEP), torch.full((self.rows, self.heads), KEEP, device="cuda")
        B.lgc_attention(ctx, self.shape(B), self.q, self.k, self.v, o, lse)
        return o, lse

    def backward(self, B, ctx, o, lse):
        dq, dk, dv = (torch.full_like(x, KEEP) for x in (self.q, self.k, self.v))
        delta = torch.full_like(lse, KEEP)
        B.lgc_attention_grad(ctx, self.shape(B), self.do, self.q, self.k, self.v, o, lse, dq, dk, dv, delta)
        return dq, dk, dv, delta

    def check(self, B, ctx):
        o, lse = self.forward(B, ctx)
        want_o, want_lse, off_o, off_lse = ref.attention(self.q, self.k, self.v, **self.definition())
        near(o, want_o, off_o, "o")
        near(lse, want_lse, off_lse, "lse")
        o, lse = want_o.nan_to_num(0.0).to(BF16), want_lse.float()
        want, off = ref.attention_grad(self.do, self.q, self.k, self.v, o, lse, **self.definition())
        for got, w, b, name in zip(self.backward(B, ctx, o, lse), want, off, ("dq", "dk", "dv")):
            near(got, w, b, name)


def near(got, want, bound, name):
    """Where the definition has no value (rows of no sequence), what was there; elsewhere the value, or as far from it as bound says."""
    got = got.double()
    none = torch.isnan(want)
    assert bool((got[none] == KEEP).all()), name
    off = torch.where(none | (got == want), 0.0, (got - want).abs())
    bad = ~(off <= bound + 1e-37) & ~none
    assert not bool(bad.any()), (name, int(bad.sum()), float((off / (bound + 1e-37))[bad].max()), torch.nonzero(bad)[:3].tolist())


SHAPES = {
    "one token": (1, 1, 1, 1, 64), "one query": (1, 300, 4, 2, 64), "one key": (40, 1, 2, 1, 128, 1, None, False), "a tile": (64, 64, 1, 1, 128), "ragged": (200, 200, 2, 1, 128),
    "least head": (70, 90, 3, 1, 8), "80": (333, 333, 4, 2, 80), "odd group": (130, 130, 15, 3, 96), "group of 8": (50, 210, 8, 1, 128), "all seen": (130, 517, 3, 3, 32, 1, None, False),
    "window": (500, 500, 4, 4, 64, 1, None, True, 100), "window of one": (100, 100, 2, 2, 64, 1, None, True, 1), "window, not causal": (150, 260, 2, 2, 64, 1, None, False, 40),
    "more queries than keys": (300, 70, 4, 2, 128), "no keys": (30, 0, 2, 2, 64), "no queries": (0, 30, 2, 2, 64), "sequences": (600, 600, 2, 2, 128, 100),
    "starts": (700, 900, 6, 2, 64, 5, ([3, 100, 100, 350, 351, 690], [0, 200, 260, 600, 600, 880])),
    "starts, window": (700, 900, 6, 2, 96, 5, ([3, 100, 100, 350, 351, 690], [0, 200, 260, 600, 600, 880]), False, 50),
    "starts past the end": (300, 300, 2, 2, 64, 3, ([10, 100, 290, 900], [10, 100, 290, 900])), "starts that are all the same": (40, 40, 2, 2, 64, 2, ([40, 40, 40], [7, 7, 7])),
    "64 starts": (640, 640, 2, 1, 64, 64, (list(range(0, 650, 10)), list(range(0, 650, 10)))),
    "65 starts": (900, 900, 2, 1, 64, 65, ([i * (i + 1) // 5 for i in range(66)], [i * (i + 1) // 5 for i in range(66)])),
    "many starts": (3000, 3000, 1, 1, 64, 1500, (list(range(0, 3001, 2)), list(range(0, 3001, 2)))),
    "keys in parts": (4, 8192, 8, 2, 128, 2), "queries in parts": (6000, 100, 4, 2, 128, 1, None, False), "parts of starts": (9, 7000, 2, 2, 64, 3, ([1, 2, 5, 8], [100, 3000, 3001, 6900])),
    "eight wavefronts": (2048, 2048, 64, 64, 128), "half a head": (2048, 2048, 8, 2, 64, 2), "eight wavefronts of 88": (2048, 2048, 64, 64, 88), "many blocks of 72": (1400, 1400, 80, 80, 72, 7), "long": (4096, 4096, 8, 8, 128, 2),
    "many blocks": (1400, 1400, 80, 80, 40, 7), "many blocks, wide heads": (1400, 1400, 80, 80, 104, 7), "many blocks of starts": (1400, 1500, 160, 80, 64, 7, ([0, 3, 400, 400, 800, 1000, 1300, 1399],
                                                                                                                                                              [7, 300, 301, 301, 900, 1000, 1100, 1500]), True, 150),
}


@pytest.mark.parametrize("name", SHAPES)
def test_against_the_definition(B, ctx, name):
    Case(*SHAPES[name], seed=len(name)).check(B, ctx)


def test_extremes(B, ctx):
    """Scores of hundreds, of both signs; all equal; a tiny and a large scale."""
    c = Case(100, 300, 4, 2, 64, seed=5)
    c.q *= 8
    c.k *= 8
    c.check(B, ctx)
    c.q.zero_()
    c.check(B, ctx)
    Case(100, 300, 4, 2, 64, scale=1e-30, seed=6).check(B, ctx)
    Case(100, 300, 4, 2, 64, scale=3.0, seed=7).check(B, ctx)
    c = Case(64, 640, 1, 1, 64, causal=False, seed=8)      # each tile's scores far above the ones before, and the other way round
    c.k *= torch.arange(640, device="cuda", dtype=BF16)[:, None] / 64
    c.check(B, ctx)
    c.k = c.k.flip(0).contiguous()
    c.check(B, ctx)


def test_a_million_keys(B, ctx):
    """Rows enough that nothing is split: a lane adds up 2^14 tiles, whose rounding is at most U / 2 of the whole for each, and within a tile 32 terms."""
    keys, rows = 1 << 20, 1 << 17
    q, k = torch.ones((rows, 8), dtype=BF16, device="cuda"), torch.full((keys, 8), 0.0433, dtype=BF16, device="cuda")
    k[0] = 0.0                                                  # the maximum stays here: the others are 2^0.5 of it
    v = torch.ones_like(k)
    o, lse = torch.full_like(q, KEEP), torch.full((rows, 1), KEEP, device="cuda")
    B.lgc_attention(ctx, B.AttentionShape(1, 1, 8, scale=1.0, causal=False), q, k, v, o, lse)
    want = math.log1p((keys - 1) * math.exp(8 * float(k[1, 0])))
    off = (2 ** 14 / 2 + 32 + 16) * ref.U
    assert float((lse.double() - want).abs().max()) <= off
    # p meets the values in bf16: all of them with one and the same rounding; the products' sums add 16 keys at a time
    p, rounded = math.exp(8 * float(k[1, 0])), float(torch.tensor(math.exp(8 * float(k[1, 0]))).to(BF16))
    assert float((o.double() - (1 + (keys - 1) * rounded) / (1 + (keys - 1) * p)).abs().max()) <= off + 2 ** 16 / 2 * ref.U + ref.H


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("window", [0, 70])
@pytest.mark.parametrize("heads,dim", [(4, 64), (280, 64), (280, 128), (4, 80), (280, 96)])     # (few blocks, many)
def test_what_is_hidden_has_no_influence(B, ctx, bad, window, heads, dim):
    """Infinities and NaNs in keys, values, queries and gradients: what does not see them is as if they were zeros, what does is not finite (where all of it is bad)."""
    n, at = 400, 250
    for which in "kvq":
        c = Case(n, n, heads, heads // 2, dim, window=window, seed=11)
        clean = Case(n, n, heads, heads // 2, dim, window=window, seed=11)
        getattr(c, which)[at] = bad
        getattr(clean, which)[at] = 0.0
        o, lse = c.forward(B, ctx)
        want_o, want_lse = clean.forward(B, ctx)
        seen = ref.visible(n, n, True, window)
        if which == "q":
            rows = torch.arange(n) == at
        else:
            rows = seen[:, at]
        rows = rows.cuda()
        assert torch.equal(o[~rows], want_o[~rows]), which
        if which == "v" or math.isnan(bad):
            assert not bool(o[rows].isfinite().any()), which
        if which != "v":
            assert torch.equal(lse[~rows], want_lse[~rows])
        if which == "v":
            got, want = c.backward(B, ctx, want_o, lse), clean.backward(B, ctx, want_o, want_lse)
            assert torch.equal(got[0][~rows], want[0][~rows]) and not bool(got[0][rows].isfinite().any())
            keys = seen[rows.cpu()].any(0).cuda()      # keys that some of those queries see: their dk hangs on ds
            assert torch.equal(got[1][~keys], want[1][~keys]) and torch.equal(got[2], want[2])
        elif math.isnan(bad):
            got, want = c.backward(B, ctx, want_o, lse), clean.backward(B, ctx, want_o, want_lse)
            assert torch.equal(got[0][~rows], want[0][~rows]) and not bool(got[0][rows].isfinite().any()), which
            keys = seen[rows.cpu()].any(0).cuda()
            for i in (1, 2):
                assert torch.equal(got[i][~keys], want[i][~keys]), (which, i)
                if which == "q":
                    assert not bool(got[i][keys].isfinite().any())
    c, clean = Case(n, n, heads, heads // 2, dim, window=window, seed=12), Case(n, n, heads, heads // 2, dim, window=window, seed=12)
    c.do[at] = bad
    clean.do[at] = 0.0
    o, lse = c.forward(B, ctx)
    got, want = c.backward(B, ctx, o, lse), clean.backward(B, ctx, o, lse)
    others = (torch.arange(n) != at).cuda()
    assert torch.equal(got[0][others], want[0][others]) and not bool(got[0][at].isfinite().any())
    hidden = ~seen_keys(n, window)[at].cuda()
    for i in (1, 2):
        assert torch.equal(got[i][hidden], want[i][hidden]) and not bool(got[i][~hidden].isfinite().any()), i


def seen_keys(n, window):
    return ref.visible(n, n, True, window)


@pytest.mark.parametrize("starts", [None, [0, 3000, 3000, 6000]])
def test_caches_with_room(B, ctx, starts):
    """kv_lengths: of each sequence's rows the first so many, whatever the others hold; a length past the room is the room."""
    lengths, rooms = [1500, 0, 2500], [2000] * 3 if starts is None else [3000, 0, 3000]
    for lengths in ([1500, 0, 2500], [1, 7, 9000]):
        c = Case(6, 6000, 4, 2, 64, 3, None if starts is None else ([0, 2, 4, 6], starts), seed=40)
        real = [min(n, room) for n, room in zip(lengths, rooms)]
        firsts = [0, 2000, 4000] if starts is None else starts[:3]
        for first, n, room in zip(firsts, real, rooms):
            c.k[first + n:first + room] = math.nan
            c.v[first + n:first + room] = math.inf
        how = {} if starts is None else {n: torch.tensor(s, dtype=torch.int32, device="cuda") for n, s in (("q_starts", [0, 2, 4, 6]), ("kv_starts", starts))}
        shape = B.AttentionShape(4, 2, 64, sequences=3, kv_lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"), **how)
        o, lse = torch.full_like(c.q, KEEP), torch.full((6, 4), KEEP, device="cuda")
        B.lgc_attention(ctx, shape, c.q, c.k, c.v, o, lse)
        k, v = (torch.cat([x[first:first + n] for first, n in zip(firsts, real)]) for x in (c.k, c.v))
        packed = [0, real[0], real[0] + real[1], sum(real)]
        want_o, want_lse, off_o, off_lse = ref.attention(c.q, k, v, 4, 2, 64, c.scale, 3, [0, 2, 4, 6], packed)
        near(o, want_o, off_o, "o")
        near(lse, want_lse, off_lse, "lse")


def test_garbage_around_sequences(B, ctx):
    """Rows of no sequence may hold anything, in front, behind and between what is read together."""
    starts = ([5, 90, 200], [8, 100, 260])
    c, clean = (Case(230, 300, 4, 2, 80, 2, starts, seed=13) for _ in range(2))
    for x in (c.q, c.do):
        x[:5] = math.nan
        x[200:] = math.inf
    for x in (c.k, c.v):
        x[:8] = math.nan
        x[260:] = -math.inf
    o, lse = c.forward(B, ctx)
    want, want_lse = clean.forward(B, ctx)
    assert torch.equal(o, want) and torch.equal(lse, want_lse)
    for x, y in zip(c.backward(B, ctx, o, lse), clean.backward(B, ctx, o, lse)):
        assert torch.equal(x, y)


def test_a_query_that_sees_nothing_has_no_part(B, ctx):
    c = Case(200, 60, 2, 2, 64, seed=14)       # queries 0 .. 139 stand before the first key
    c.do[:140] = math.nan
    c.q[:140] = math.inf
    o, lse = c.forward(B, ctx)
    assert bool((o[:140] == 0).all()) and bool((lse[:140] == -math.inf).all()) and bool(o[140:].isfinite().all())
    dq, dk, dv, _ = c.backward(B, ctx, o, lse)
    assert bool((dq[:140] == 0).all()) and bool(dq.isfinite().all()) and bool(dk.isfinite().all()) and bool(dv.isfinite().all())


def test_one_matrix_for_all(B, ctx):
    """q, k and v side by side in the rows of one matrix, gradients in another, o in a wider one: as the three in matrices of their own."""
    rows, heads, kv, dim = 300, 4, 2, 64
    c = Case(rows, rows, heads, kv, dim, seed=15)
    cuts = [0, heads * dim, (heads + kv) * dim, (heads + 2 * kv) * dim]
    fused = torch.cat([c.q, c.k, c.v, rand(rows, 24, 16)], 1)
    q, k, v = (fused[:, a:b] for a, b in zip(cuts, cuts[1:]))
    o, lse = torch.full((rows, heads * dim + 40), KEEP, dtype=BF16, device="cuda"), torch.empty((rows, heads), device="cuda")
    want_o, want_lse = c.forward(B, ctx)
    B.lgc_attention(ctx, c.shape(B), q, k, v, o[:, 16:16 + heads * dim], lse)
    assert torch.equal(o[:, 16:16 + heads * dim], want_o) and torch.equal(lse, want_lse) and bool((o[:, :16] == KEEP).all()) and bool((o[:, 16 + heads * dim:] == KEEP).all())
    B.lgc_attention(ctx, c.shape(B), q, k, v, o[:, 16:16 + heads * dim])        # lse not wanted
    grads = torch.full((rows, cuts[-1] + 8), KEEP, dtype=BF16, device="cuda")
    dq, dk, dv = (grads[:, a:b] for a, b in zip(cuts, cuts[1:]))
    B.lgc_attention_grad(ctx, c.shape(B), c.do, q, k, v, o[:, 16:16 + heads * dim], lse, dq, dk, dv, torch.empty_like(lse))
    for got, want in zip((dq, dk, dv), c.backward(B, ctx, want_o, want_lse)):
        assert torch.equal(got, want)
    assert bool((grads[:, cuts[-1]:] == KEEP).all())


def test_places_past_32_bits(B, ctx):
    """Keys and values whose places pass 2^31 elements and 2^32 bytes, sequences there and at the front."""
    ld, rows = 1 << 15, 70_000
    store = torch.empty(rows * ld, dtype=BF16, device="cuda").view(rows, ld)
    k, v = store[:, :128], store[:, 128:256]
    starts = [0, 100, 69_500, 70_000]
    c = Case(150, 600, 2, 1, 128, 3, ([0, 50, 50, 150], [0, 100, 100, 600]), seed=17)
    for whole, part in ((k, c.k), (v, c.v)):
        whole[:100], whole[69_500:] = part[:100], part[100:]
    want_o, want_lse, off_o, off_lse = ref.attention(c.q, c.k, c.v, **c.definition())
    shape = B.AttentionShape(2, 1, 128, sequences=3, q_starts=torch.tensor([0, 50, 50, 150], dtype=torch.int32, device="cuda"), kv_starts=torch.tensor(starts, dtype=torch.int32, device="cuda"))
    o, lse = torch.full_like(c.q, KEEP), torch.full((150, 2), KEEP, device="cuda")
    B.lgc_attention(ctx, shape, c.q, k, v, o, lse)
    near(o, want_o, off_o, "o")
    near(lse, want_lse, off_lse, "lse")
    want, off = ref.attention_grad(c.do, c.q, c.k, c.v, o, lse, **c.definition())
    grads = torch.empty_like(store)
    dk, dv, dq = grads[:, :128], grads[:, 128:256], torch.empty_like(c.q)
    B.lgc_attention_grad(ctx, shape, c.do, c.q, k, v, o, lse, dq, dk, dv, torch.empty_like(lse))
    near(dq, want[0], off[0], "dq")
    for got, w, bound in zip((dk, dv), want[1:], off[1:]):
        near(torch.cat([got[:100], got[69_500:]]), w, bound, "dk, dv")
        assert bool((got[100:69_500] == 0).all())


def test_gradients_against_differences(B, ctx):
    """The derivative of sum(do * o) along a direction, from differences of the definition in 64 bits."""
    c = Case(90, 130, 4, 2, 64, window=60, seed=18)
    o, lse = c.forward(B, ctx)
    grads = c.backward(B, ctx, o, lse)
    _, off = ref.attention_grad(c.do, c.q, c.k, c.v, o, lse, **c.definition())
    loss = lambda **x: float((c.do.double() * ref.attention(*({"q": c.q.double(), "k": c.k.double(), "v": c.v.double()} | x).values(), **c.definition())[0]).sum())  # noqa: E731
    for name, got, bound in zip("qkv", grads, off):
        x = getattr(c, name).double()
        d = torch.randn(x.shape, generator=torch.Generator().manual_seed(19), dtype=torch.float64).cuda()
        step = 1e-5
        along = (loss(**{name: x + step * d}) - loss(**{name: x - step * d})) / (2 * step)
        # the differences themselves: their third-order term and the rounding of sums of this size, both below 1e-6 here; and o and lse, which are rounded: 2^-8 of each o in delta
        o_off = 2.0 ** -8 * float((got.double().abs() * d.abs()).sum())
        assert abs(float((got.double() * d).sum()) - along) <= float((bound * d.abs()).sum()) + o_off + 1e-5 * abs(along), name


def test_equal_calls_give_equal_bits(B, ctx):
    for args in (SHAPES["starts"], SHAPES["keys in parts"], SHAPES["queries in parts"], SHAPES["eight wavefronts"]):
        c = Case(*args, seed=20)
        first = [*c.forward(B, ctx)]
        first += c.backward(B, ctx, *first)
        for _ in range(2):
            again = [*c.forward(B, ctx)]
            again += c.backward(B, ctx, *again)
            assert all(torch.equal(a.nan_to_num(1e9), b.nan_to_num(1e9)) for a, b in zip(first, again))


def test_on_another_stream_and_another_context(B, ctx):
    c = Case(*SHAPES["keys in parts"], seed=21)
    want = c.forward(B, ctx)
    side, other = torch.cuda.Stream(), B.Context(1, 1, 1)
    B.lgc_reserve_training(other)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = c.forward(B, other)
    mine = c.forward(B, ctx)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) and torch.equal(a, m) for a, b, m in zip(want, got, mine))
    other.close()


def test_one_shape_in_two_threads(B, ctx):
    """The structure of heads and sequences serves calls of other lengths at once, each on a context and stream of its own."""
    cases = [Case(n, n, 2, 2, 64, seed=60 + n) for n in (100, 900)]
    shape = cases[0].shape(B)
    want = [c.forward(B, ctx)[0] for c in cases]
    got, wrong = [torch.full_like(c.q, KEEP) for c in cases], []
    contexts = [B.Context(1, 1, 1) for _ in cases]
    for c in contexts:
        B.lgc_reserve_training(c)
    torch.cuda.synchronize()

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(200):
                    B.lgc_attention(contexts[i], shape, cases[i].q, cases[i].k, cases[i].v, got[i])
        except Exception as e:  # noqa: BLE001
            wrong.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not wrong and all(torch.equal(a, b) for a, b in zip(got, want))
    for c in contexts:
        c.close()


def test_in_graphs(B, ctx):
    """Forward and backward recorded twice on one context, replayed in turn with new inputs and new lengths, eager calls between."""
    names = ("keys in parts", "starts")
    graphs = []
    for i, name in enumerate(names):
        c = Case(*SHAPES[name], seed=30 + i)
        starts = None if c.starts is None else [torch.tensor(s, dtype=torch.int32, device="cuda") for s in c.starts]
        how = {} if starts is None else dict(q_starts=starts[0], kv_starts=starts[1])
        shape = B.AttentionShape(c.heads, c.kv_heads, c.dim, scale=c.scale, **c.how, **how)
        out = [torch.full_like(c.q, KEEP), torch.full((c.rows, c.heads), KEEP, device="cuda"), torch.full_like(c.q, KEEP), torch.full_like(c.k, KEEP), torch.full_like(c.v, KEEP),
               torch.full((c.rows, c.heads), KEEP, device="cuda")]
        calls = lambda c=c, shape=shape, out=out: (B.lgc_attention(ctx, shape, c.q, c.k, c.v, *out[:2]),  # noqa: E731
                                                   B.lgc_attention_grad(ctx, shape, c.do, c.q, c.k, c.v, *out[:2], *out[2:]))
        calls()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            calls()
        graphs.append((g, c, out, starts, calls))
    for round in range(3):
        for g, c, out, starts, calls in graphs:
            for j, x in enumerate((c.q, c.k, c.v, c.do)):
                x.copy_(rand(*x.shape, 50 + 10 * round + j))
            if starts is not None:
                starts[0].copy_(torch.tensor([0, 50 * round, 200, 420, 421, 600], dtype=torch.int32))
            for x in out:
                x.fill_(KEEP)
            g.replay()
            torch.cuda.synchronize()
            got = [x.clone() for x in out]
            for x in out:
                x.fill_(KEEP)
            calls()
            assert all(torch.equal(a, b) for a, b in zip(got, out)), round


def test_the_binding_s_checks(B, ctx):
    c = Case(64, 64, 4, 2, 64)
    o, lse = c.forward(B, ctx)
    wrong = [lambda: B.lgc_attention(ctx, c.shape(B), c.q[:, :128], c.k, c.v, o), lambda: B.lgc_attention(ctx, c.shape(B), c.q.float(), c.k, c.v, o),
             lambda: B.lgc_attention(ctx, c.shape(B), c.q, c.k[:63], c.v, o), lambda: B.lgc_attention(ctx, c.shape(B), c.q, c.k, c.v, o.t().contiguous().t()),
             lambda: B.lgc_attention(ctx, c.shape(B), c.q, c.k, c.v, o, lse.double()), lambda: B.lgc_attention(ctx, c.shape(B), c.q, c.k, c.v, o, lse[:, :3]),
             lambda: B.lgc_attention(ctx, c.shape(B), c.q.cpu(), c.k, c.v, o), lambda: B.AttentionShape(4, 2, 64, q_starts=torch.zeros(2, dtype=torch.int32, device="cuda")),
             lambda: B.AttentionShape(4, 2, 64, q_starts=torch.zeros(3, dtype=torch.int32, device="cuda"), kv_starts=torch.zeros(2, dtype=torch.int32, device="cuda")),
             lambda: B.AttentionShape(4, 2, 64, q_starts=torch.zeros(2, device="cuda"), kv_starts=torch.zeros(2, device="cuda")), lambda: B.AttentionShape(4, 2, -64),
             lambda: B.AttentionShape(4, 2, 64, sequences=2, kv_lengths=torch.zeros(1, dtype=torch.int32, device="cuda")),
             lambda: B.lgc_attention_grad(ctx, c.shape(B), c.do, c.q, c.k, c.v, o, lse, torch.empty_like(c.k), torch.empty_like(c.k), torch.empty_like(c.v), lse.clone())]
    for call in wrong:
        with pytest.raises(ValueError):
            call()
    with pytest.raises(B.LgcError):
        B.lgc_attention(ctx, c.shape(B), c.q, c.k, c.v, c.q)
