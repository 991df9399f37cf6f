"""A layer of attention and feed-forward whose training step, and whose form for one new token at a time, run on the library.

``Attention`` is y = x + Wo attention(rotate(W norm(x) + b)) + bo with its backward pass, over sequences of one length or packed
ones of different lengths; with a ``Cache`` it answers token by token.  ``FusedFeedForward`` is ``FeedForward`` with non-linearity,
8-bit checkpoints and residual in its products' epilogues.  ``Layer`` is one after the other, with all weights and gradients in flat
fp32 vectors for ``lgc_accumulate_topk``.  ``python -m paper_2103_08870_amd.transformer_layer`` trains one from sparse gradients on a
synthetic task, prints the losses, and continues a sequence token by token.
"""
from __future__ import annotations

import argparse
from typing import List, Optional

import torch

from . import binding as B
from .feed_forward import EPS, FeedForward


class Cache:
    """Keys and values of ``sequences`` sequences with room for ``capacity`` tokens each; how many they hold is on the device, and in ``most`` what the fullest can hold at most."""

    def __init__(self, sequences: int, capacity: int, width: int, device: str = "cuda"):
        self.sequences, self.capacity, self.most = sequences, capacity, 0
        self.k, self.v = (torch.zeros((sequences * capacity, width), device=device, dtype=torch.bfloat16) for _ in range(2))
        self.lengths = torch.zeros(sequences, device=device, dtype=torch.int32)
        self.first = torch.arange(sequences, device=device) * capacity


class Attention:
    """One block for up to ``rows`` tokens of ``width`` in bfloat16, ``heads`` query and ``kv_heads`` key heads of ``dim``.  The weights are one flat fp32 vector ``flat``
    (gamma, beta, W [(heads + 2 kv_heads) dim][width], b, Wo [width][heads dim], bo); ``refresh`` makes the 8-bit weights from it, once after every change."""

    def __init__(self, rows: int, width: int, heads: int, kv_heads: int, dim: int, sequences: int = 1, window: int = 0, ctx: Optional[B.Context] = None, seed: int = 0,
                 device: str = "cuda"):
        self.rows, self.heads, self.kv_heads, self.dim, self.sequences, self.window = rows, heads, kv_heads, dim, sequences, window
        self.ctx = ctx if ctx is not None else B.Context(1, 1, 1)
        B.lgc_reserve_training(self.ctx)
        wide, all_heads = heads * dim, (heads + 2 * kv_heads) * dim
        shapes = [(width,), (width,), (all_heads, width), (all_heads,), (width, wide), (width,)]
        self.places, n = [], 0
        for s in shapes:
            size = s[0] * (s[1] if len(s) > 1 else 1)
            self.places.append((n, n + size, s))
            n += size
        self.flat = torch.zeros(n, device=device)
        gen = torch.Generator(device=device).manual_seed(seed)
        gamma, _, w, _, wo, _ = self.parts(self.flat)
        gamma.fill_(1.0)
        w.normal_(0.0, width ** -0.5, generator=gen)
        wo.normal_(0.0, wide ** -0.5, generator=gen)
        blocks = lambda *shape, tiles=False: B.Blocks(*shape, tiles=tiles, device=device)  # noqa: E731
        self.w, self.w_t = blocks(all_heads, width, tiles=True), blocks(width, all_heads, tiles=True)
        self.wo, self.wo_t = blocks(width, wide, tiles=True), blocks(wide, width, tiles=True)
        self.h, self.o8 = blocks(rows, width), blocks(rows, wide)                         # checkpoints, as are qkv, o, lse
        self.dy8, self.dqkv8 = blocks(rows, width), blocks(rows, all_heads)
        half = lambda cols: torch.empty((rows, cols), device=device, dtype=torch.bfloat16)  # noqa: E731
        self.qkv, self.dqkv, self.o, self.do, self.dh = half(all_heads), half(all_heads), half(wide), half(wide), half(width)
        self.lse, self.delta = (torch.empty((rows, heads), device=device) for _ in range(2))
        self.mean, self.rstd = (torch.empty(rows, device=device) for _ in range(2))
        self.freqs = B.lgc_rotary_frequencies(dim).to(device)
        self.x: Optional[torch.Tensor] = None
        self.refresh()

    def parts(self, flat: torch.Tensor) -> List[torch.Tensor]:
        """gamma, beta, W, b, Wo, bo as views of a flat vector of the weights' layout."""
        return [flat[lo:hi].view(shape) for lo, hi, shape in self.places]

    def refresh(self) -> None:
        _, _, w, _, wo, _ = self.parts(self.flat)
        B.lgc_quantize_weights(self.ctx, w, self.w, self.w_t)
        B.lgc_quantize_weights(self.ctx, wo, self.wo, self.wo_t)

    def _split(self, matrix: torch.Tensor) -> List[torch.Tensor]:
        """q, k, v side by side in the rows of one matrix."""
        wide, narrow = self.heads * self.dim, self.kv_heads * self.dim
        return [matrix[:, :wide], matrix[:, wide:wide + narrow], matrix[:, wide + narrow:]]

    def forward(self, x: torch.Tensor, starts: Optional[torch.Tensor] = None, cache: Optional[Cache] = None) -> torch.Tensor:
        """``rows`` tokens: ``sequences`` sequences of one length, or those of which ``starts`` (int32, on the device) has the first rows, and the row behind the last.
        An empty cache takes their keys and values (sequences of one length)."""
        gamma, beta, _, b, _, bo = self.parts(self.flat)
        self.x, self.starts = x, starts
        self.positions = None
        if starts is not None:
            row = torch.arange(x.shape[0], device=x.device, dtype=torch.int32)
            its = (torch.searchsorted(starts, row, right=True) - 1).clamp(0, starts.numel() - 2)
            self.positions = row - starts[its]
        B.lgc_layer_norm(self.ctx, x, gamma, beta, EPS, mean=self.mean, rstd=self.rstd, blocks=self.h)
        B.lgc_product(self.ctx, self.h, self.w, b, self.qkv)
        self._rotate(self.qkv)
        q, k, v = self._split(self.qkv)
        if starts is not None:
            self.shape = B.AttentionShape(self.heads, self.kv_heads, self.dim, sequences=starts.numel() - 1, q_starts=starts, kv_starts=starts, window=self.window)
            self.o.zero_()                                                                # rows of no sequence
        else:
            self.shape = B.AttentionShape(self.heads, self.kv_heads, self.dim, sequences=self.sequences, window=self.window)
        if cache is not None:
            length = x.shape[0] // self.sequences
            if starts is not None or cache.sequences != self.sequences or cache.most or length > cache.capacity:
                raise ValueError(f"an empty cache of {self.sequences} sequences with room for {length} tokens is what takes these")
            for mine, its in ((k, cache.k), (v, cache.v)):
                its.view(self.sequences, cache.capacity, -1)[:, :length] = mine.reshape(self.sequences, length, -1)
            cache.lengths.fill_(length)
            cache.most = length
        B.lgc_attention(self.ctx, self.shape, q, k, v, self.o, self.lse)
        B.lgc_quantize(self.ctx, self.o, self.o8)
        y = torch.empty_like(x)
        B.lgc_product_activate(self.ctx, self.o8, self.wo, bo, None, residual=x, z=y)
        return y

    def _rotate(self, qkv: torch.Tensor, inverse: bool = False) -> None:
        both = self.heads + self.kv_heads                                                 # queries and keys, side by side
        B.lgc_rotate(self.ctx, qkv[:, :both * self.dim], both, self.freqs, positions=self.positions, period=self.rows // self.sequences, inverse=inverse)

    def backward(self, dy: torch.Tensor, grad: torch.Tensor) -> torch.Tensor:
        """Writes the weights' gradient of the last ``forward`` to ``grad`` (laid out like ``flat``); returns the input's."""
        dgamma, dbeta, dw, db, dwo, dbo = self.parts(grad)
        B.lgc_weight_grad(self.ctx, dy, self.o8, dwo, dbo)
        B.lgc_quantize(self.ctx, dy, self.dy8)
        B.lgc_product(self.ctx, self.dy8, self.wo_t, None, self.do)
        if self.starts is not None:
            self.dqkv.zero_()
        B.lgc_attention_grad(self.ctx, self.shape, self.do, *self._split(self.qkv), self.o, self.lse, *self._split(self.dqkv), self.delta)
        self._rotate(self.dqkv, inverse=True)
        B.lgc_weight_grad(self.ctx, self.dqkv, self.h, dw, db)
        B.lgc_quantize(self.ctx, self.dqkv, self.dqkv8)
        B.lgc_product(self.ctx, self.dqkv8, self.w_t, None, self.dh)
        dx = torch.empty_like(dy)
        B.lgc_layer_norm_grad(self.ctx, self.dh, self.x, self.parts(self.flat)[0], self.mean, self.rstd, dx, dgamma, dbeta)
        return dy + dx

    def step(self, x: torch.Tensor, cache: Cache) -> torch.Tensor:
        """One new token of each of the cache's sequences, [sequences][width]: its keys and values go behind the others.  (Recorded into a graph, it is the caller who counts the
        replays: past the capacity a token takes the last one's place.)"""
        if x.shape[0] != cache.sequences or cache.most >= cache.capacity:
            raise ValueError(f"{x.shape[0]} tokens for {cache.sequences} sequences of up to {cache.most} tokens, with room for {cache.capacity}")
        gamma, beta, _, b, _, bo = self.parts(self.flat)
        n, both = x.shape[0], self.heads + self.kv_heads
        h, o8 = B.Blocks(n, x.shape[1], device=x.device), B.Blocks(n, self.heads * self.dim, device=x.device)
        qkv, y = torch.empty((n, self.qkv.shape[1]), device=x.device, dtype=x.dtype), torch.empty_like(x)
        B.lgc_layer_norm(self.ctx, x, gamma, beta, EPS, blocks=h)
        B.lgc_product(self.ctx, h, self.w, b, qkv)
        B.lgc_rotate(self.ctx, qkv[:, :both * self.dim], both, self.freqs, positions=cache.lengths)
        q, k, v = self._split(qkv)
        at = cache.first + cache.lengths.clamp(max=cache.capacity - 1)
        cache.k.index_copy_(0, at, k)
        cache.v.index_copy_(0, at, v)
        cache.lengths.add_(1)
        cache.most += 1
        shape = B.AttentionShape(self.heads, self.kv_heads, self.dim, sequences=n, window=self.window, kv_lengths=cache.lengths)
        o = torch.empty((n, self.heads * self.dim), device=x.device, dtype=x.dtype)
        B.lgc_attention(self.ctx, shape, q, cache.k, cache.v, o)
        B.lgc_quantize(self.ctx, o, o8)
        B.lgc_product_activate(self.ctx, o8, self.wo, bo, None, residual=x, z=y)
        return y


class FusedFeedForward(FeedForward):
    """``FeedForward`` in fewer launches and bytes: its first product leaves only its 8-bit checkpoint and the 8-bit operand of the second, which adds the residual.  (f sees
    the product's fp32 sums, which FeedForward rounds to bfloat16 before.)"""

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        self.x = x
        return self._forward(x, self.h, self.a, self.z, self.mean, self.rstd)

    def _forward(self, x: torch.Tensor, h: B.Blocks, a: Optional[B.Blocks], z: B.Blocks, mean: Optional[torch.Tensor], rstd: Optional[torch.Tensor]) -> torch.Tensor:
        gamma, beta, _, b1, _, b2 = self.parts(self.flat)
        y = torch.empty_like(x)
        B.lgc_layer_norm(self.ctx, x, gamma, beta, EPS, mean=mean, rstd=rstd, blocks=h)
        B.lgc_product_activate(self.ctx, h, self.w1, b1, self.act, t_blocks=a, z_blocks=z)
        B.lgc_product_activate(self.ctx, z, self.w2, b2, None, residual=x, z=y)
        return y

    def step(self, x: torch.Tensor) -> torch.Tensor:
        """Any number of tokens, with nothing kept."""
        blocks = lambda like: B.Blocks(x.shape[0], like.cols, device=x.device)  # noqa: E731
        return self._forward(x, blocks(self.h), None, blocks(self.z), None, None)


class Layer:
    """Attention, then feed-forward; their weights one after another in ``flat``."""

    def __init__(self, rows: int, width: int, heads: int, kv_heads: int, dim: int, hidden: int, sequences: int = 1, window: int = 0, act: str = "gelu",
                 ctx: Optional[B.Context] = None, seed: int = 0, device: str = "cuda"):
        self.ctx = ctx if ctx is not None else B.Context(1, 1, 1)
        self.attention = Attention(rows, width, heads, kv_heads, dim, sequences, window, self.ctx, seed, device)
        self.feed_forward = FusedFeedForward(rows, width, hidden, act, self.ctx, seed + 1, device)
        self.cut = self.attention.flat.numel()
        self.flat = torch.cat([self.attention.flat, self.feed_forward.flat])
        self.attention.flat, self.feed_forward.flat = self.flat[:self.cut], self.flat[self.cut:]

    def refresh(self) -> None:
        self.attention.refresh()
        self.feed_forward.refresh()

    def forward(self, x: torch.Tensor, starts: Optional[torch.Tensor] = None, cache: Optional[Cache] = None) -> torch.Tensor:
        return self.feed_forward.forward(self.attention.forward(x, starts, cache))

    def backward(self, dy: torch.Tensor, grad: torch.Tensor) -> torch.Tensor:
        """Writes the weights' gradient of the last ``forward`` to ``grad`` (laid out like ``flat``); returns the input's."""
        return self.attention.backward(self.feed_forward.backward(dy, grad[self.cut:]), grad[:self.cut])

    def step(self, x: torch.Tensor, cache: Cache) -> torch.Tensor:
        return self.feed_forward.step(self.attention.step(x, cache))


def train(nodes: int = 2, sequences: int = 4, length: int = 256, width: int = 512, heads: int = 8, kv_heads: int = 2, dim: int = 64, hidden: int = 2048, iterations: int = 30,
          ratio: float = 0.01, rate: float = 0.01, momentum: float = 0.5, seed: int = 0, layer: Optional[Layer] = None) -> List[float]:
    """Trains a layer to imitate another one from `nodes` nodes' sparse gradients; returns the nodes' mean loss per iteration."""
    rows = sequences * length
    layer = layer if layer is not None else Layer(rows, width, heads, kv_heads, dim, hidden, sequences, seed=seed)
    goal = Layer(rows, width, heads, kv_heads, dim, hidden, sequences, seed=seed + 2)
    n = layer.flat.numel()
    k = max(1, int(ratio * n))
    ctx = B.Context(n, k, nodes)
    u, v, grads = (torch.zeros((nodes, n), device="cuda") for _ in range(3))
    vals, idx = torch.empty((nodes, k), device="cuda"), torch.empty((nodes, k), device="cuda", dtype=torch.int32)
    dense = torch.empty(n, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(seed)
    losses = []
    for _ in range(iterations):
        loss = torch.zeros((), device="cuda")
        for node in range(nodes):
            x = torch.randn((rows, width), generator=gen, device="cuda").to(torch.bfloat16)
            off = layer.forward(x).float() - goal.forward(x).float()
            loss += off.square().mean() / nodes
            layer.backward((off * (2.0 / rows)).to(torch.bfloat16), grads[node])
        B.lgc_accumulate_topk(ctx, grads, u, v, momentum, k, vals, idx)
        dense.zero_()
        B.lgc_scatter(ctx, vals, idx, 1.0 / nodes, dense)
        layer.flat.sub_(dense, alpha=rate)
        layer.refresh()
        losses.append(loss)
    return [float(x) for x in losses]


def continued(layer: Layer, x: torch.Tensor, tokens: int) -> torch.Tensor:
    """x, sequences of one length, and the `tokens` outputs that follow each when every output is the next input: [sequences][tokens][width]."""
    a = layer.attention
    cache = Cache(a.sequences, x.shape[0] // a.sequences + tokens, a.kv_heads * a.dim, device=x.device)
    y = layer.forward(x, cache=cache).view(a.sequences, -1, x.shape[1])[:, -1].contiguous()
    out = [y]
    for _ in range(tokens - 1):
        out.append(layer.step(out[-1], cache))
    return torch.stack(out, 1)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    names = (("nodes", 2), ("sequences", 4), ("length", 256), ("width", 512), ("heads", 8), ("kv_heads", 2), ("dim", 64), ("hidden", 2048), ("iterations", 30))
    for name, value in names:
        ap.add_argument("--" + name, type=int, default=value)
    how = vars(ap.parse_args())
    made = Layer(how["sequences"] * how["length"], *(how[x] for x in ("width", "heads", "kv_heads", "dim", "hidden", "sequences")))
    for i, x in enumerate(train(**how, layer=made)):
        print(f"iteration {i}: loss {x:.5f}", flush=True)
    prompt = torch.randn((how["sequences"] * how["length"], how["width"]), device="cuda").to(torch.bfloat16)
    print("continued, root mean square of each token:", [round(float(t.float().square().mean().sqrt()), 3) for t in continued(made, prompt, 8).unbind(1)])
