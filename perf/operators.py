"""The operators of a training step that the compressed gradient comes from, each timed as one pass through its public
entry points (`paper_2103_08870_amd.binding`): layer norm and its gradient, activations kept in 8 bits and their use in
the backward pass, products of 8-bit matrices, and the weights' gradient from an 8-bit checkpoint.

A matrix in 8 bits is held as e4m3 codes, one byte an element with the columns padded by zeros to whole blocks of 128, and
one exponent byte E per block: value = code * 2^(E - 127).  A block is 128 columns of one row (activations) or 128 x 128
(weights).  E is the least for which the block's largest finite magnitude does not pass 448, at least 10; infinities and
NaNs become NaN.  Every value is zero or a normal number of few bits, so that it is exact in bfloat16.

Where `own` is false the operators are computed in their plain form, in 32 bits with torch's elementary operations.
"""
import math
import random

import torch

own = False

EPS = 1e-5
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one token of a model that answers: latency
        dict(name="norm_token", kind="norm", rows=1, cols=4096, type="bf16", eight=False),
        # a training batch whose norm feeds a product in 8 bits; the values as a consumer that takes bfloat16 sees them
        dict(name="norm_train", kind="norm", rows=8192, cols=4096, type="bf16", eight=True),
        # a small model in fp32 with sizes that no vector or block divides
        dict(name="norm_grad_ragged", kind="norm_grad", rows=2047, cols=1111, type="fp32"),
        # the longest batch and rows
        dict(name="norm_grad_train", kind="norm_grad", rows=16384, cols=8192, type="bf16"),
        # an activation stored in 8 bits and brought back, last blocks not whole
        dict(name="checkpoint_ragged", kind="checkpoint", rows=3001, cols=777, type="fp32"),
        # one short sequence: non-linearity with its checkpoint, and the gradient through it
        dict(name="activation_ragged", kind="activation", act="silu", rows=509, cols=5000, type="fp32"),
        # the hidden layer of a training batch
        dict(name="activation_train", kind="activation", act="gelu", rows=8192, cols=16384, type="bf16"),
        # one token through a linear layer: the weights are read once
        dict(name="product_token", kind="product", rows=1, n=8192, k=4096, type="bf16"),
        # one sequence through a narrow layer
        dict(name="product_ragged", kind="product", rows=1000, n=2500, k=1777, type="fp32"),
        # a training batch through the first linear layer of a feed-forward block
        dict(name="product_train", kind="product", rows=8192, n=16384, k=4096, type="bf16"),
        # few output tiles and a ragged sum over the tokens
        dict(name="weight_grad_ragged", kind="weight_grad", rows=3001, n=777, k=1300),
        # the second linear layer's weights, from the checkpoint of the hidden layer
        dict(name="weight_grad_train", kind="weight_grad", rows=8192, n=4096, k=16384),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _columns(rng, lo, hi):
    """A width: any, or (as models have them) a multiple of 128."""
    c = _log_uniform(rng, lo, hi)
    return max(lo, c // 128 * 128) if rng.random() < 0.5 else c


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "checkpoint", "activation", "product", "product", "weight_grad", "weight_grad"])
    while True:
        if kind == "product":
            case = dict(kind=kind, rows=_log_uniform(rng, 1, 8192), n=_columns(rng, 256, 16384), k=_columns(rng, 256, 16384),
                        type=rng.choice(["bf16", "bf16", "fp32"]))
        elif kind == "weight_grad":
            case = dict(kind=kind, rows=_log_uniform(rng, 32, 16384), n=_columns(rng, 256, 16384), k=_columns(rng, 256, 16384))
        else:
            case = dict(kind=kind, rows=_log_uniform(rng, 1, 16384), cols=_columns(rng, 64, 16384), type=rng.choice(["bf16", "fp32"]))
            if kind == "norm":
                case["eight"] = rng.random() < 0.5
            if kind == "activation":
                case["act"] = rng.choice(["relu", "gelu", "silu"])
        large = 2 * case["rows"] * case["n"] * case["k"] > 2 * 8192 * 16384 * 4096 if "n" in case else \
            case["rows"] * case["cols"] > 8192 * 16384
        if not large and 3072 not in case.values():
            return case


# ---------------------------------------------------------------------------------------- inputs

def _normal(shape, gen, scale=1.0):
    return torch.randn(shape, generator=gen, device="cuda").mul_(scale)


def _activations(case, gen):
    """Rows of a residual stream: a mean that is not zero, rows of different size, a few columns far larger than the others."""
    rows, cols = case["rows"], case["cols"]
    x = _normal((rows, cols), gen)
    x *= torch.exp(_normal((rows, 1), gen, 0.5))
    x *= torch.where(torch.rand(cols, generator=gen, device="cuda") < 0.01, 15.0, 1.0)
    return x.add_(0.4).to(TYPES[case["type"]])


def _pad(x, rows, cols):
    return torch.nn.functional.pad(x, (0, -x.shape[1] % cols, 0, -x.shape[0] % rows))


def _to_blocks(x, per):
    """Codes and exponents of a matrix with a scale per `per` rows and 128 columns."""
    rows = x.shape[0]
    t = _pad(x.float(), per, 128)
    t = t.view(t.shape[0] // per, per, t.shape[1] // 128, 128)
    most = torch.where(torch.isfinite(t), t.abs(), 0.0).amax(dim=(1, 3), keepdim=True)
    part, power = torch.frexp(most)                       # most = part * 2^power, part in [0.5, 1); 448 = 0.875 * 2^9
    power = torch.where(part > 0.875, power - 8, power - 9).clamp_(min=-117)
    power = torch.where(most > 0, power, -117)
    codes = torch.where(torch.isfinite(t), torch.ldexp(t, -power), math.nan).to(torch.float8_e4m3fn)
    codes = codes.view(torch.uint8).reshape(t.shape[0] * per, -1)[:rows]
    exps = (power + 127).to(torch.uint8).view(t.shape[0], t.shape[2])
    return codes.contiguous(), _pad(exps, 1, 4).contiguous()


def _from_blocks(codes, exps, per, cols):
    """The values, in fp32."""
    t = _pad(codes.view(torch.float8_e4m3fn).float(), per, 128)
    blocks = t.shape[1] // 128
    scale = torch.ldexp(torch.ones((), device=codes.device), exps[:, :blocks].int() - 127)
    t = t.view(-1, per, blocks, 128) * scale.view(-1, 1, blocks, 1)
    return t.view(-1, blocks * 128)[:codes.shape[0], :cols]


_context = None


def _own_context():
    """The one context that a program keeps for its calls."""
    global _context
    if _context is None:
        from paper_2103_08870_amd import binding as B
        _context = B.Context(1, 1, 1)
        B.lgc_reserve_training(_context)
    return _context


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, rows = case["kind"], case["rows"]
    s = dict(case)
    if kind == "product":
        x = _normal((rows, case["k"]), gen) * torch.exp(_normal((rows, 1), gen, 0.5))
        s["a_codes"], s["a_exps"] = _to_blocks(x, 1)
        s["b_codes"], s["b_exps"] = _to_blocks(_normal((case["n"], case["k"]), gen, 0.02), 128)
        s["bias"] = _normal((case["n"],), gen, 0.1)
        s["y"] = torch.empty((rows, case["n"]), device="cuda", dtype=TYPES[case["type"]])
    elif kind == "weight_grad":
        s["x_codes"], s["x_exps"] = _to_blocks(torch.relu(_normal((rows, case["k"]), gen) + 0.5), 1)
        s["dy"] = (_normal((rows, case["n"]), gen, 1e-3) * torch.exp(_normal((rows, 1), gen))).to(torch.bfloat16)
        s["dw"] = torch.empty((case["n"], case["k"]), device="cuda")
        s["db"] = torch.empty((case["n"],), device="cuda")
    else:
        x = _activations(case, gen)
        s["x"] = x
        if kind in ("norm", "norm_grad"):
            s["gamma"], s["beta"] = 1.0 + _normal((case["cols"],), gen, 0.1), _normal((case["cols"],), gen, 0.1)
        if kind in ("norm_grad", "activation"):
            s["dy"] = _normal(x.shape, gen, 1e-3).to(x.dtype)
            s["dx"] = torch.empty_like(x)
        if kind == "norm":
            s["mean"], s["rstd"] = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        if kind == "norm_grad":
            x = x.float()
            s["mean"] = x.mean(1)
            s["rstd"] = torch.rsqrt((x - s["mean"][:, None]).square().mean(1) + EPS)
            s["dgamma"], s["dbeta"] = torch.empty_like(s["gamma"]), torch.empty_like(s["gamma"])
        s["y"] = torch.empty(s["x"].shape, device="cuda", dtype=torch.bfloat16 if s.get("eight") else s["x"].dtype)
    if own:
        from paper_2103_08870_amd import binding as B
        s["ctx"] = _own_context()
        if kind == "product":
            s["a"] = B.Blocks(rows, case["k"], codes=s["a_codes"], exps=s["a_exps"])
            s["b"] = B.Blocks(case["n"], case["k"], tiles=True, codes=s["b_codes"], exps=s["b_exps"])
        elif kind == "weight_grad":
            s["x8"] = B.Blocks(rows, case["k"], codes=s["x_codes"], exps=s["x_exps"])
        elif kind in ("checkpoint", "activation") or s.get("eight"):
            s["x8"] = B.Blocks(rows, case["cols"])
    return s


# ---------------------------------------------------------------------------------------- one pass

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2103_08870_amd import binding as B
    kind, ctx = s["kind"], s["ctx"]
    if kind == "norm":
        if s["eight"]:
            B.lgc_layer_norm(ctx, s["x"], s["gamma"], s["beta"], EPS, mean=s["mean"], rstd=s["rstd"], blocks=s["x8"])
            B.lgc_dequantize(ctx, s["x8"], s["y"])
        else:
            B.lgc_layer_norm(ctx, s["x"], s["gamma"], s["beta"], EPS, y=s["y"], mean=s["mean"], rstd=s["rstd"])
        return s["y"], s["mean"], s["rstd"]
    if kind == "norm_grad":
        B.lgc_layer_norm_grad(ctx, s["dy"], s["x"], s["gamma"], s["mean"], s["rstd"], s["dx"], s["dgamma"], s["dbeta"])
        return s["dx"], s["dgamma"], s["dbeta"]
    if kind == "checkpoint":
        B.lgc_quantize(ctx, s["x"], s["x8"])
        B.lgc_dequantize(ctx, s["x8"], s["y"])
        return s["y"]
    if kind == "activation":
        B.lgc_activate(ctx, s["act"], s["x"], z=s["y"], a_blocks=s["x8"])
        B.lgc_activate_grad(ctx, s["act"], s["dy"], s["x8"], da=s["dx"])
        return s["y"], s["dx"]
    if kind == "product":
        B.lgc_product(ctx, s["a"], s["b"], s["bias"], s["y"])
        return s["y"]
    B.lgc_weight_grad(ctx, s["dy"], s["x8"], s["dw"], s["db"])
    return s["dw"], s["db"]


def _act(act, x):
    if act == "relu":
        return torch.clamp(x, min=0.0)
    if act == "silu":
        return x * torch.sigmoid(x)
    return x * (0.5 + 0.5 * torch.erf(x * math.sqrt(0.5)))


def _act_slope(act, x):
    if act == "relu":
        return (x > 0).to(x.dtype)
    if act == "silu":
        p = torch.sigmoid(x)
        return p + x * p * (1 - p)
    return 0.5 + 0.5 * torch.erf(x * math.sqrt(0.5)) + x * torch.exp(-0.5 * x * x) * (1 / math.sqrt(2 * math.pi))


def _run_plain(s):
    kind = s["kind"]
    if kind == "product":
        a = _from_blocks(s["a_codes"], s["a_exps"], 1, s["k"])
        b = _from_blocks(s["b_codes"], s["b_exps"], 128, s["k"])
        return (a @ b.t() + s["bias"]).to(s["y"].dtype)
    if kind == "weight_grad":
        dy = s["dy"].float()
        return dy.t() @ _from_blocks(s["x_codes"], s["x_exps"], 1, s["k"]), dy.sum(0)
    x = s["x"].float()
    if kind == "norm":
        mean = x.mean(1)
        x = x - mean[:, None]
        rstd = torch.rsqrt(x.square().mean(1) + EPS)
        y = x * rstd[:, None] * s["gamma"] + s["beta"]
        if s["eight"]:
            y = _from_blocks(*_to_blocks(y, 1), 1, s["cols"])
        return y.to(s["y"].dtype), mean, rstd
    if kind == "norm_grad":
        dy = s["dy"].float()
        h = (x - s["mean"][:, None]) * s["rstd"][:, None]
        q = dy * s["gamma"]
        dx = s["rstd"][:, None] * (q - q.mean(1, keepdim=True) - h * (q * h).mean(1, keepdim=True))
        return dx.to(s["x"].dtype), (dy * h).sum(0), dy.sum(0)
    kept = _from_blocks(*_to_blocks(x, 1), 1, s["cols"])
    if kind == "checkpoint":
        return kept.to(s["y"].dtype)
    return _act(s["act"], x).to(s["y"].dtype), (s["dy"].float() * _act_slope(s["act"], kept)).to(s["dx"].dtype)


# ---------------------------------------------------------------------------------------- floors

def work(case):
    kind, rows = case["kind"], case["rows"]
    if kind == "product":
        n, k = case["n"], case["k"]
        return dict(bytes=(rows + n) * k * (1 + 1 / 128) + 4 * n + rows * n * (4 if case["type"] == "fp32" else 2), flops=2 * rows * n * k)
    if kind == "weight_grad":
        n, k = case["n"], case["k"]
        return dict(bytes=2 * rows * n + rows * k * (1 + 1 / 128) + 4 * n * k + 4 * n, flops=2 * rows * n * k)
    cols = case["cols"]
    size, b = rows * cols, 4 if case["type"] == "fp32" else 2
    if kind == "norm":
        return dict(bytes=size * (b + (2 if case["eight"] else b)) + 8 * cols + 8 * rows, flops=8 * size)
    if kind == "norm_grad":
        return dict(bytes=3 * size * b + 12 * cols + 8 * rows, flops=14 * size)
    if kind == "checkpoint":
        return dict(bytes=2 * size * b, flops=4 * size)
    return dict(bytes=4 * size * b, flops=30 * size)


# ---------------------------------------------------------------------------------------- in 64 bits

def _kept64(x):
    """What 8 bits keep of each row's blocks of 128, from the definition: the nearest of the numbers m * 2^(e - 3), |m| < 16, with
    e >= -6 at a scale of one."""
    out = torch.empty_like(x)
    for c in range(0, x.shape[1], 128):
        t = x[:, c:c + 128]
        most = t.abs().amax(1, keepdim=True)
        scale = torch.exp2(torch.ceil(torch.log2(most.clamp(min=1e-300) / 448.0)).clamp(min=-117.0))
        t = t / scale
        step = torch.exp2(torch.floor(torch.log2(t.abs().clamp(min=2.0 ** -6))) - 3)
        out[:, c:c + 128] = torch.round(t / step) * step * scale
    return out


def _values64(codes, exps, per, cols):
    """Values of codes and exponents, from the bits: sign, four of exponent, three of mantissa."""
    c = codes[:, :cols].int()
    e, m = c >> 3 & 15, (c & 7).double()
    v = torch.where(e > 0, (8 + m) * torch.exp2((e - 10).double()), m * 2.0 ** -9)
    v = torch.where(c > 127, -v, v)
    scale = torch.exp2(exps.double() - 127).repeat_interleave(per, 0)[:c.shape[0]].repeat_interleave(128, 1)[:, :cols]
    return v * scale


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "product":
        return _values64(s["a_codes"], s["a_exps"], 1, case["k"]) @ _values64(s["b_codes"], s["b_exps"], 128, case["k"]).t() + s["bias"].double()
    if kind == "weight_grad":
        dy = s["dy"].double()
        return dy.t() @ _values64(s["x_codes"], s["x_exps"], 1, case["k"]), dy.sum(0)
    x, cols = s["x"].double(), case["cols"]
    if kind == "checkpoint":
        return _kept64(x)
    if kind == "activation":
        k, dy = _kept64(x), s["dy"].double()
        if case["act"] == "relu":
            return torch.maximum(x, torch.zeros_like(x)), torch.where(k > 0, dy, 0.0)
        if case["act"] == "silu":
            return x / (1 + torch.exp(-x)), dy * ((1 + torch.exp(-k) + k * torch.exp(-k)) / (1 + torch.exp(-k)).square())
        return 0.5 * x * torch.erfc(-x / math.sqrt(2)), dy * (0.5 * torch.erfc(-k / math.sqrt(2)) + k * torch.exp(-k * k / 2) / math.sqrt(2 * math.pi))
    gamma, beta = s["gamma"].double(), s["beta"].double()
    if kind == "norm":
        mean = x.sum(1) / cols
        rstd = (((x - mean[:, None]) ** 2).sum(1) / cols + EPS) ** -0.5
        y = gamma * (x - mean[:, None]) * rstd[:, None] + beta
        return _kept64(y) if case["eight"] else y, mean, rstd
    mean, rstd, dy = s["mean"].double(), s["rstd"].double(), s["dy"].double()
    h = rstd[:, None] * (x - mean[:, None])
    q = gamma * dy
    dx = (q - q.sum(1, keepdim=True) / cols - h * ((h * q).sum(1, keepdim=True) / cols)) * rstd[:, None]
    return dx, (h * dy).sum(0), dy.sum(0)
