"""Attention and its gradient from their definitions in 64 bits, one sequence and key head after another, and how far results in fewer bits may be from them.

A lane's score is a sum of `dim` products in fp32, a probability one exponential of it, and p and ds are rounded to bf16 (by at most H of themselves) where they meet the
next matrix, whose sums are fp32 again.  What follows from that for each result is worked out beside the result, from the same magnitudes that its sum has."""
import math

import torch

U, H = 2.0 ** -24, 2.0 ** -8      # half a unit in the last place of fp32 and of bf16
LEAST = 2.0 ** -126


def lengths_of(starts, rows, sequences):
    """[(first, length)] of each sequence."""
    if starts is None:
        return [(i * (rows // sequences), rows // sequences) for i in range(sequences)]
    s = [min(int(x), rows) for x in starts]
    return [(a, max(0, b - a)) for a, b in zip(s, s[1:])]


def visible(lq, lk, causal, window, device="cpu"):
    pos = torch.arange(lq, device=device)[:, None] + lk - lq
    key = torch.arange(lk, device=device)[None, :]
    seen = torch.ones((lq, lk), dtype=torch.bool, device=device)
    if causal:
        seen &= key <= pos
    if window:
        seen &= key > pos - window
    return seen


def _pairs(heads, kv_heads, dim, sequences, q, k, q_starts, kv_starts, causal, window):
    """For each sequence and query head: rows of q, rows of k, head, key head, what is visible."""
    for (q0, lq), (k0, lk) in zip(lengths_of(q_starts, q.shape[0], sequences), lengths_of(kv_starts, k.shape[0], sequences)):
        seen = visible(lq, lk, causal, window, q.device)
        for h in range(heads):
            yield slice(q0, q0 + lq), slice(k0, k0 + lk), h, h // (heads // kv_heads), seen


def _zeroed(x, seen):
    """x where a row sees something of it at all: what nobody sees must not count, whatever it is."""
    return torch.where(seen.any(0)[:, None], x, 0.0)


def attention(q, k, v, heads, kv_heads, dim, scale, sequences=1, q_starts=None, kv_starts=None, causal=True, window=0):
    """o, lse and their bounds; rows that belong to no sequence: NaN."""
    q, k, v = (x.double().view(x.shape[0], x.shape[1] // dim, dim) for x in (q, k, v))
    o, lse = torch.full_like(q, math.nan), torch.full(q.shape[:2], math.nan, dtype=torch.float64, device=q.device)
    off_o, off_lse = torch.zeros_like(o), torch.zeros_like(lse)
    for rq, rk, h, g, seen in _pairs(heads, kv_heads, dim, sequences, q, k, q_starts, kv_starts, causal, window):
        a, b, c = q[rq, h], _zeroed(k[rk, g], seen), _zeroed(v[rk, g], seen)
        s = (scale * a @ b.t()).masked_fill(~seen, -math.inf)
        empty = ~seen.any(1)
        l = torch.where(empty, -math.inf, torch.logsumexp(s, 1) if s.shape[1] else -math.inf)
        p = torch.exp(s - torch.where(empty, 0.0, l)[:, None])
        o[rq, h], lse[rq, h] = p @ c, l
        size = (scale * a.abs() @ b.abs().t()).masked_fill(~seen, 0.0)
        # the score's sum, its rounding when it is scaled and lowered by the row's largest, and the exponential
        wrong = ((dim + 8) * U * size.amax(1) + 4 * U if size.shape[1] else torch.zeros_like(l))[:, None]
        off_o[rq, h] = (H + 4 * wrong + (s.shape[1] + 8) * U) * (p @ c.abs()) + H * o[rq, h].abs()
        off_lse[rq, h] = 2 * wrong[:, 0] + (s.shape[1] + 8) * U + 8 * U * torch.where(empty, 0.0, l).abs()
    return o.flatten(1), lse, off_o.flatten(1), off_lse


def attention_grad(do, q, k, v, o, lse, heads, kv_heads, dim, scale, sequences=1, q_starts=None, kv_starts=None, causal=True, window=0):
    """(dq, dk, dv), and their bounds, with the o and lse that are given; rows that belong to no sequence: NaN."""
    do, q, k, v, o = (x.double().view(x.shape[0], x.shape[1] // dim, dim) for x in (do, q, k, v, o))
    lse = lse.double()
    dq, dk, dv = (torch.full_like(x, math.nan) for x in (q, k, v))
    off = [torch.zeros_like(x) for x in (q, k, v)]
    for x, starts, rows in ((dk, kv_starts, k.shape[0]), (dv, kv_starts, k.shape[0])):
        for first, n in lengths_of(starts, rows, sequences):
            x[first:first + n] = 0.0
    for rq, rk, h, g, seen in _pairs(heads, kv_heads, dim, sequences, q, k, q_starts, kv_starts, causal, window):
        some = seen.any(1)[:, None]
        a, b, c = torch.where(some, q[rq, h], 0.0), _zeroed(k[rk, g], seen), _zeroed(v[rk, g], seen)
        y, out = torch.where(some, do[rq, h], 0.0), torch.where(some, o[rq, h], 0.0)
        l = torch.where(some, lse[rq, h, None], 0.0)
        s = scale * a @ b.t()
        p = torch.where(seen, torch.exp(s - l), 0.0)
        dp, delta = y @ c.t(), (y * out).sum(1, keepdim=True)
        ds = p * (dp - delta)
        dq[rq, h] = scale * ds @ b
        dk[rk, g] += scale * ds.t() @ a
        dv[rk, g] += p.t() @ y
        size = scale * a.abs() @ b.abs().t()
        wrong = (dim + 8) * U * (size + l.abs()) + 4 * U
        # (what is below the least normal number, 2^-126 in fp32 as in bf16, may count as nothing: a probability, and its ds)
        wrong_p = torch.where(seen, p * (H + 2 * wrong) + LEAST, 0.0)
        wrong_ds = ds.abs() * (H + 2 * wrong) + torch.where(seen, LEAST * ((dp - delta).abs() + 1), 0.0) + p * (dim + 4) * U * (y.abs() @ c.abs().t() + (y.abs() * out.abs()).sum(1, keepdim=True))
        n, m = (lk_terms(s.shape[1]), lk_terms(s.shape[0] * heads // kv_heads))
        off[0][rq, h] = scale * (wrong_ds + n * ds.abs()) @ b.abs() + H * dq[rq, h].abs()
        off[1][rk, g] += scale * (wrong_ds + m * ds.abs()).t() @ a.abs()
        off[2][rk, g] += (wrong_p + m * p).t() @ y.abs()
    off[1] += H * dk.abs().nan_to_num(0.0)
    off[2] += H * dv.abs().nan_to_num(0.0)
    return [x.flatten(1) for x in (dq, dk, dv)], [x.flatten(1) for x in off]


def lk_terms(n):
    """fp32 sums of n terms, in whatever order, and the joins of their parts."""
    return (n + 64) * U
