"""What the training step's operators hand from launch to launch, over sweeps of sizes, read from a HIP runtime that only records (recording_hip.cpp): no GPU."""
import json
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
if HERE not in sys.path:
    sys.path.insert(0, HERE)
from test_host_routes import Host, ROOT   # noqa: E402,F401  (puts the repository's root in sys.path)
import test_gpu_training_reach as reach   # noqa: E402
from test_training_routes import AT, BF16, FP32, launches, layer_norm, layer_norm_grad, product, quantize, u64, weight_grad   # noqa: E402

# rows from one to many, widths that models have and others, sums short and long: either side of every rule of launch_product
M = [1, 16, 17, 64, 65, 128, 129, 160, 257, 280, 300, 400, 513, 641, 700, 900, 1100, 2000, 2049, 4100, 8192]
N = [100, 512, 777, 2500, 4096, 8300, 11000, 15000, 18000, 22016, 28672, 32800, 50257]
K = [100, 1000, 4096, 8064, 8192, 12288, 14000, 16384, 40000]
SPLIT = [(280, 28672, 8192), (700, 11000, 14000), (129, 32800, 12288), (513, 15000, 16384), (400, 18000, 12288), (900, 8300, 16384)]   # large tiles that a rule for small ones would split


def lines(h, call, *args):
    """[kernel's mangled name, grid] of each launch of a call."""
    h.log()
    assert call(h.lib, h.train, *args) == 0
    h.log()
    return [[line.split()[1], [int(x) for x in line.split()[2:]]] for line in h.raw.splitlines()]


def output_type(name):
    """A kernel's first template argument: the type of what it stores (products) or reads beside codes (weight gradients)."""
    rest = name[name.index("_GLOBAL__N_1") + len("_GLOBAL__N_1"):]
    length = "".join(c for c in rest[:2] if c.isdigit())
    rest = rest[len(length) + int(length):]
    return "fp32" if rest.startswith("If") else "bf16" if rest.startswith("INS_4Bf16E") else rest


def dequantize(l, ctx, rows, cols, type):
    return l.lgc_dequantize(ctx, AT, AT, 1, u64(rows), u64(cols), AT, type, u64(cols), None)


def activate(l, ctx, rows, cols, type):
    return l.lgc_activate(ctx, 1, AT, type, u64(rows), u64(cols), u64(cols), AT, u64(cols), AT, AT, AT, AT, None)


def activate_grad(l, ctx, rows, cols, type):
    return l.lgc_activate_grad(ctx, 2, AT, type, u64(rows), u64(cols), u64(cols), AT, AT, AT, u64(cols), AT, AT, None)


# blocks of 128 columns: up to the most that the calls take, and either side of where a launch's second dimension begins
BLOCKS = [(rows, cols) for rows in ((1 << 30) - 1, (1 << 30) - 63, (1 << 30) - 64, (1 << 30) - 65, (1 << 26) + 1, 1 << 26) for cols in (1, 128)] + [((1 << 29) - 1, 129), ((1 << 17) - 1, 1 << 20)]


@pytest.fixture(scope="module")
def answers(tmp_path_factory):
    from paper_2103_08870_amd import build
    library = build.build(force=False)
    fake = str(tmp_path_factory.mktemp("hip") / "librecording_hip.so")
    r = subprocess.run([build._hipcc(), "-O1", "-std=c++17", "-shared", "-fPIC", "--offload-arch=gfx950", os.path.join(HERE, "recording_hip.cpp"), "-o", fake],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([sys.executable, os.path.abspath(__file__), fake, library], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stderr
    return json.loads(r.stdout)


def test_parts_of_a_product_are_stored_as_what_their_sum_reads(answers):
    """k_join adds fp32 arrays whatever the product's type: what comes before it stores fp32, for every size; what stores the product itself, its type."""
    split = 0
    for m, n, k, type, got in answers["products"]:
        first, *rest = got
        assert len(rest) <= 1 and (first[1][1] > 1) == bool(rest), (m, n, k, got)      # parts, and their sum, or neither
        if rest:
            split += 1
            assert "k_join" in rest[0][0] and output_type(rest[0][0]) == type and output_type(first[0]) == "fp32", (m, n, k, type, got)
        else:
            assert output_type(first[0]) == type, (m, n, k, type, got)
    assert split > 100


def test_parts_of_a_weight_gradient_are_summed(answers):
    for rows, n, k, type, got in answers["weight_grads"]:
        assert output_type(got[0][0]) == type and (got[0][1][1] > 1) == (len(got) == 2), (rows, n, k, got)
        assert len(got) == 1 or "k_add_parts" in got[1][0]


def test_grids_hold_every_block_and_a_launch_s_threads(answers):
    """A launch's dimension has fewer than 2^32 threads; 64 blocks of 128 columns, one of kernels' 256 threads."""
    for rows, cols, got in answers["blocks"]:
        (_, (x, y, z)), = got
        assert x * 256 < 1 << 32 and y <= 65535 and z == 1, (rows, cols, got)
        assert rows * ((cols + 127) // 128) <= 64 * x * y < rows * ((cols + 127) // 128) + (64 << 20), (rows, cols, got)


def test_sizes_of_the_tests_reach_the_kernels_that_they_are_meant_for(answers):
    for rows, cols, want, got in answers["norms"]:
        (name, (blocks, _, _)), = got
        assert name == want and blocks * (4 if " 64 " in want else 1) < rows, (rows, cols, got)
    for rows, cols, want, got in answers["norm_grads"]:
        blocks = [grid[1 if "columns" in want else 0] for name, grid in got if name.startswith(want)]
        assert len(blocks) == 1 and blocks[0] < rows, (rows, cols, got)
    for rows, n, k, want, got in answers["reach"]:
        assert got[0][0].startswith(want), (rows, n, k, got)
    for got in answers["groups"]:
        (name, (x, y, z)), = got
        assert name.split()[-1] == "4" and 64 * x - 63 <= 36891 < 64 * x, got


if __name__ == "__main__":
    h = Host(sys.argv[1], sys.argv[2])
    h.train = h.ctx(1, 1, 1)
    assert h.lib.lgc_reserve_training(h.train) == 0
    types = (("fp32", FP32), ("bf16", BF16))
    shapes = [(m, n, k) for m in M for n in N for k in K] + SPLIT
    out = {"products": [[m, n, k, name, lines(h, product, m, n, k, type)] for m, n, k in shapes for name, type in types],
           "weight_grads": [[t, n, k, name, lines(h, weight_grad, t, n, k, type)] for t in (8, 100, 1000, 3001, 8192, 40000) for n in N for k in (100, 1000, 4096, 16384)
                            for name, type in types]}
    out["blocks"] = [[rows, cols, lines(h, call, rows, cols, type)] for rows, cols in BLOCKS for call in (quantize, dequantize, activate, activate_grad) for type in (FP32, BF16)]
    out["norms"] = [[rows, cols, want, launches(h, layer_norm, (rows, cols, type))[1]] for (rows, cols), want in reach.NORMS.items() for type in (FP32, BF16)]
    out["norm_grads"] = [[rows, cols, want, launches(h, layer_norm_grad, (rows, cols, type))[1]] for (rows, cols), want in reach.NORM_GRADS.items() for type in (FP32, BF16)]
    out["reach"] = [[*shape, want, launches(h, weight_grad, (*shape, type))[1]] for shape, want in reach.WEIGHT_GRADS.items() for type in (FP32, BF16)]
    out["groups"] = [launches(h, call, (*reach.GROUPS, type))[1] for call in (quantize, dequantize, activate, activate_grad) for type in (FP32, BF16)]
    print(json.dumps(out))
