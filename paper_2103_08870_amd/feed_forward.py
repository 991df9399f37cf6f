"""A feed-forward block whose training step runs on the library from the forward pass to the sparse update.

``FeedForward`` is y = x + W2 f(W1 norm(x) + b1) + b2 with its backward pass.  Its products read 8-bit matrices, its backward
pass the same 8-bit matrices as checkpoints, and it leaves its gradient in one flat fp32 vector, which is what
``lgc_accumulate_topk`` takes.  ``train`` is the whole loop for some simulated nodes: gradients, accumulation and top-k,
averaged scatter, update.  ``python -m paper_2103_08870_amd.feed_forward`` runs it on a synthetic regression and prints the
losses.
"""
from __future__ import annotations

import argparse
from typing import List, Optional

import torch

from . import binding as B

EPS = 1e-5


class FeedForward:
    """One block for batches of ``rows`` tokens of ``width`` in bfloat16.  The weights are one flat fp32 vector ``flat`` (gamma, beta,
    W1 [hidden][width], b1, W2 [width][hidden], b2, one after the other); ``refresh`` makes the 8-bit weights from it, once
    after every change.  Everything that ``forward`` keeps for ``backward`` is in 8 bits, but its input."""

    def __init__(self, rows: int, width: int, hidden: int, act: str = "gelu", ctx: Optional[B.Context] = None, seed: int = 0, device: str = "cuda"):
        self.act, self.rows = act, rows
        self.ctx = ctx if ctx is not None else B.Context(1, 1, 1)
        B.lgc_reserve_training(self.ctx)
        shapes = [(width,), (width,), (hidden, width), (hidden,), (width, hidden), (width,)]
        self.places, n = [], 0
        for s in shapes:
            size = s[0] * (s[1] if len(s) > 1 else 1)
            self.places.append((n, n + size, s))
            n += size
        self.flat = torch.zeros(n, device=device)
        gen = torch.Generator(device=device).manual_seed(seed)
        gamma, _, w1, _, w2, _ = self.parts(self.flat)
        gamma.fill_(1.0)
        w1.normal_(0.0, width ** -0.5, generator=gen)
        w2.normal_(0.0, hidden ** -0.5, generator=gen)
        blocks = lambda *shape, tiles=False: B.Blocks(*shape, tiles=tiles, device=device)  # noqa: E731
        self.w1, self.w1_t = blocks(hidden, width, tiles=True), blocks(width, hidden, tiles=True)
        self.w2, self.w2_t = blocks(width, hidden, tiles=True), blocks(hidden, width, tiles=True)
        self.h, self.a, self.z = blocks(rows, width), blocks(rows, hidden), blocks(rows, hidden)      # checkpoints
        self.dy8, self.da8 = blocks(rows, width), blocks(rows, hidden)
        self.wide = torch.empty((rows, hidden), device=device, dtype=torch.bfloat16)
        self.dwide = torch.empty_like(self.wide)
        self.narrow = torch.empty((rows, width), device=device, dtype=torch.bfloat16)
        self.mean, self.rstd = torch.empty(rows, device=device), torch.empty(rows, device=device)
        self.x: Optional[torch.Tensor] = None
        self.refresh()

    def parts(self, flat: torch.Tensor) -> List[torch.Tensor]:
        """gamma, beta, W1, b1, W2, b2 as views of a flat vector of the weights' layout."""
        return [flat[lo:hi].view(shape) for lo, hi, shape in self.places]

    def refresh(self) -> None:
        _, _, w1, _, w2, _ = self.parts(self.flat)
        B.lgc_quantize_weights(self.ctx, w1, self.w1, self.w1_t)
        B.lgc_quantize_weights(self.ctx, w2, self.w2, self.w2_t)

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        gamma, beta, _, b1, _, b2 = self.parts(self.flat)
        self.x = x
        B.lgc_layer_norm(self.ctx, x, gamma, beta, EPS, mean=self.mean, rstd=self.rstd, blocks=self.h)
        B.lgc_product(self.ctx, self.h, self.w1, b1, self.wide)
        B.lgc_activate(self.ctx, self.act, self.wide, a_blocks=self.a, z_blocks=self.z)
        B.lgc_product(self.ctx, self.z, self.w2, b2, self.narrow)
        return x + self.narrow

    def backward(self, dy: torch.Tensor, grad: torch.Tensor) -> torch.Tensor:
        """Writes the weights' gradient of the last ``forward`` to ``grad`` (laid out like ``flat``); returns the input's."""
        dgamma, dbeta, dw1, db1, dw2, db2 = self.parts(grad)
        B.lgc_weight_grad(self.ctx, dy, self.z, dw2, db2)
        B.lgc_quantize(self.ctx, dy, self.dy8)
        B.lgc_product(self.ctx, self.dy8, self.w2_t, None, self.wide)                                       # dz
        B.lgc_activate_grad(self.ctx, self.act, self.wide, self.a, da=self.dwide, da_blocks=self.da8)
        B.lgc_weight_grad(self.ctx, self.dwide, self.h, dw1, db1)
        B.lgc_product(self.ctx, self.da8, self.w1_t, None, self.narrow)                                     # dh
        dx = torch.empty_like(dy)
        B.lgc_layer_norm_grad(self.ctx, self.narrow, self.x, self.parts(self.flat)[0], self.mean, self.rstd, dx, dgamma, dbeta)
        return dy + dx


def train(nodes: int = 2, rows: int = 1024, width: int = 512, hidden: int = 2048, iterations: int = 30, ratio: float = 0.01,
          rate: float = 0.01, momentum: float = 0.5, seed: int = 0) -> List[float]:
    """Trains a block to imitate another one from `nodes` nodes' sparse gradients; returns the nodes' mean loss per iteration."""
    block = FeedForward(rows, width, hidden, seed=seed)
    goal = FeedForward(rows, width, hidden, seed=seed + 1)
    n = block.flat.numel()
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
            target = goal.forward(x)
            off = block.forward(x).float() - target.float()
            loss += off.square().mean() / nodes
            block.backward((off * (2.0 / rows)).to(torch.bfloat16), grads[node])
        B.lgc_accumulate_topk(ctx, grads, u, v, momentum, k, vals, idx)
        dense.zero_()
        B.lgc_scatter(ctx, vals, idx, 1.0 / nodes, dense)
        block.flat.sub_(dense, alpha=rate)
        block.refresh()
        losses.append(loss)
    return [float(x) for x in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("nodes", 2), ("rows", 1024), ("width", 512), ("hidden", 2048), ("iterations", 30)):
        ap.add_argument("--" + name, type=int, default=value)
    for i, x in enumerate(train(**vars(ap.parse_args()))):
        print(f"iteration {i}: loss {x:.5f}", flush=True)
