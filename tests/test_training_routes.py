"""Which kernels the training step's operators launch for which sizes, and how many, read from a HIP runtime that only records (recording_hip.cpp): no GPU, any size."""
import ctypes as C
import json
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
if HERE not in sys.path:
    sys.path.insert(0, HERE)
from test_host_routes import Host, ROOT   # noqa: E402  (puts the repository's root in sys.path)

u64, p, f32 = C.c_uint64, C.c_void_p, C.c_float
AT = p(1 << 40)
FP32, BF16 = 0, 1


def layer_norm(l, ctx, rows, cols, type):
    return l.lgc_layer_norm(ctx, AT, type, u64(rows), u64(cols), u64(cols), AT, AT, f32(1e-5), AT, u64(cols), AT, AT, AT, AT, None)


def layer_norm_grad(l, ctx, rows, cols, type, wants="xgb"):
    dx, dg, db = (p(1 << 41) if w in wants else None for w in "xgb")
    return l.lgc_layer_norm_grad(ctx, AT, u64(cols), AT, u64(cols), type, u64(rows), u64(cols), AT, AT, AT, dx, u64(cols), dg, db, None)


def product(l, ctx, m, n, k, type):
    return l.lgc_product(ctx, AT, AT, u64(m), AT, AT, u64(n), u64(k), AT, AT, type, u64(n), None)


def weight_grad(l, ctx, rows, n, k, type):
    return l.lgc_weight_grad(ctx, AT, type, u64(rows), u64(n), u64(n), AT, AT, u64(k), AT, AT, None)


def quantize(l, ctx, rows, cols, type):
    return l.lgc_quantize(ctx, AT, type, u64(rows), u64(cols), u64(cols), AT, AT, None)


def quantize_weights(l, ctx, rows, cols, type):
    return l.lgc_quantize_weights(ctx, AT, type, u64(rows), u64(cols), u64(cols), AT, AT, AT, AT, None)


# call, arguments; kernels launched, each with its template's numbers in their order
ROUTES = [
    (layer_norm, (1, 500, BF16), ["k_norm 64 1"]), (layer_norm, (1, 1024, FP32), ["k_norm 64 2"]), (layer_norm, (8191, 2048, BF16), ["k_norm 256 1"]),
    (layer_norm, (8192, 2048, BF16), ["k_norm 128 2"]), (layer_norm, (5, 4096, BF16), ["k_norm 256 2"]), (layer_norm, (5, 8192, BF16), ["k_norm 512 2"]),
    (layer_norm, (5, 16384, BF16), ["k_norm 1024 2"]), (layer_norm, (5, 16385, BF16), ["k_norm_long"]), (layer_norm, (0, 16385, BF16), []),
    (layer_norm_grad, (1, 1, FP32), ["k_norm_grad_few 64 1"]), (layer_norm_grad, (1024, 16384, BF16), ["k_norm_grad_few 1024 2"]),
    (layer_norm_grad, (1025, 300, BF16), ["k_norm_grad_few 64 1", "k_norm_columns"]), (layer_norm_grad, (1025, 300, BF16, "x"), ["k_norm_grad_few 64 1"]),
    (layer_norm_grad, (1025, 4096, FP32, "gb"), ["k_norm_grad_few 512 1"]), (layer_norm_grad, (4097, 300, BF16), ["k_norm_grad 64 1", "k_norm_columns"]),
    (layer_norm_grad, (1025, 16384, BF16, "xg"), ["k_norm_grad 1024 2", "k_norm_columns"]),
    (layer_norm_grad, (3, 16385, FP32), ["k_norm_grad_long", "k_norm_grad_columns", "k_norm_columns"]),
    (layer_norm_grad, (3, 16385, FP32, "b"), ["k_norm_grad_columns", "k_norm_columns"]), (layer_norm_grad, (0, 300, FP32), ["k_norm_columns"]),
    (product, (1, 8192, 4096, BF16), ["k_product_few 1 2 8 0"]), (product, (16, 8192, 8192, FP32), ["k_product_few 1 2 16 1"]),
    (product, (16, 4096, 1000, BF16), ["k_product_few 1 1 8 0"]), (product, (2, 100, 16384, BF16), ["k_product_few 1 1 8 0", "k_join"]),
    (product, (17, 4096, 1000, BF16), ["k_product_few 2 1 8 0"]), (product, (64, 4096, 2048, FP32), ["k_product_few 4 1 8 1"]),
    (product, (64, 16384, 2048, BF16), ["k_product 2 2 2 2 0"]), (product, (64, 8300, 1000, BF16), ["k_product_few 4 2 8 0"]),
    (product, (65, 4096, 128, FP32), ["k_product 2 2 2 2 1"]), (product, (2048, 4096, 4096, BF16), ["k_product 2 2 2 2 0"]),
    (product, (2049, 4096, 4096, BF16), ["k_product 4 2 2 4 0"]), (product, (2049, 4096, 4096, FP32), ["k_product 2 2 2 2 1"]),
    (product, (512, 512, 4096, BF16), ["k_product 2 2 2 2 0", "k_join"]), (product, (1000, 1000, 1000, BF16), ["k_product 2 2 2 2 0"]),
    (product, (0, 512, 4096, BF16), []),
    (weight_grad, (0, 100, 100, BF16), ["k_add_parts"]), (weight_grad, (1, 7, 100, BF16), ["k_weight_grad_small"]), (weight_grad, (1, 8, 100, BF16), ["k_weight_grad 64 64 4 2"]),
    (weight_grad, (100, 8, 100, FP32), ["k_weight_grad 64 64 4 1"]), (weight_grad, (128, 8192, 8192, BF16), ["k_weight_grad 64 64 4 1"]),
    (weight_grad, (4096, 32768, 100, BF16), ["k_weight_grad 64 64 4 2"]), (weight_grad, (4096, 131072, 128, BF16), ["k_weight_grad 64 64 4 1"]),
    (weight_grad, (4096, 131072, 129, BF16), ["k_weight_grad 128 64 8 1"]),
    (weight_grad, (129, 8192, 8192, BF16), ["k_weight_grad 128 64 8 1"]), (weight_grad, (3001, 777, 1300, BF16), ["k_weight_grad 64 64 4 2", "k_add_parts"]),
    (weight_grad, (8192, 2000, 2500, BF16), ["k_weight_grad 128 64 8 1", "k_add_parts"]), (weight_grad, (8192, 2048, 4096, BF16), ["k_weight_grad 64 64 4 1"]),
    (weight_grad, (8192, 1500, 1500, BF16), ["k_weight_grad 64 64 4 1", "k_add_parts"]), (weight_grad, (8192, 2000, 2500, FP32), ["k_weight_grad 64 64 4 1"]),
    (quantize, (509, 5000, FP32), ["k_quantize 1"]), (quantize, (8192, 5000, BF16), ["k_quantize 4"]), (quantize_weights, (300, 300, BF16), ["k_quantize_tiles"]),
]

# what memory could hold at most
LARGEST = [(layer_norm, ((1 << 30) - 1, 64, BF16)), (layer_norm_grad, ((1 << 30) - 1, 100, BF16)), (product, ((1 << 30) - 1, 1, 128, BF16)), (product, ((1 << 20) - 1, 1 << 17, 1000, BF16)),
           (weight_grad, (0, 1 << 18, 1 << 18, BF16)), (weight_grad, (1000, 1 << 18, 1 << 18, BF16)), (weight_grad, ((1 << 30) - 1, 30, 64, BF16)),
           (quantize, ((1 << 30) - 65, 100, BF16)), (quantize_weights, (1 << 20, 1 << 16, BF16)), (quantize_weights, (100, 1 << 20, FP32))]


def launches(h, call, args):
    """[kernel and its template's numbers, grid] of each launch of a call."""
    h.log()
    status = call(h.lib, h.train, *args)
    h.log()
    out = []
    for line in h.raw.splitlines():
        _, mangled, *grid = line.split()
        rest = mangled[mangled.index("_GLOBAL__N_1") + len("_GLOBAL__N_1"):]
        digits = "".join(c for c in rest[:2] if c.isdigit())
        length, rest = int(digits), rest[len(digits):]
        name, rest = rest[:length], rest[length:]
        numbers = []
        while "L" in rest and rest.index("L") + 1 < len(rest):   # Li64E, Lb1E, ..
            rest = rest[rest.index("L") + 1:]
            number = rest[1:rest.index("E")] if "E" in rest else ""
            if number.isdigit():
                numbers.append(number)
        out.append([" ".join([name] + numbers), [int(x) for x in grid]])
    return status, out


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


@pytest.mark.parametrize("i", range(len(ROUTES)), ids=lambda i: ROUTES[i][0].__name__ + "-" + "-".join(map(str, ROUTES[i][1])))
def test_kernels(answers, i):
    status, got = answers["routes"][i]
    names = [name if name.split()[0] not in ("k_norm_columns", "k_join", "k_add_parts", "k_norm_long", "k_norm_grad_long", "k_norm_grad_columns", "k_weight_grad_small",
                                             "k_quantize_tiles") else name.split()[0] for name, _ in got]
    assert status == 0 and names == ROUTES[i][2]


@pytest.mark.parametrize("i", range(len(LARGEST)), ids=lambda i: LARGEST[i][0].__name__ + "-" + "-".join(map(str, LARGEST[i][1])))
def test_grids_of_the_largest_sizes(answers, i):
    status, got = answers["largest"][i]
    assert status == 0 and got, (status, got)
    for _, (x, y, z) in got:   # a dimension's threads, 1024 a block at most, are counted in 32 bits where blocks are that large
        assert 1 <= x < 1 << 24 and 1 <= y <= 65535 and z == 1


def test_reservation_is_made_once_and_no_call_allocates(answers):
    assert answers["reserved"] == [["malloc", 64 << 20]] and answers["again"] == [] and answers["allocated by calls"] == 0


def test_a_gradient_in_place_is_refused(answers):
    assert answers["in place"] == [1, 1, 0] and answers["launched in place"] == []


if __name__ == "__main__":
    h = Host(sys.argv[1], sys.argv[2])
    h.train = h.ctx(1, 1, 1)
    h.log()
    assert h.lib.lgc_reserve_training(h.train) == 0
    out = {"reserved": [x for x in h.log() if x[0] == "malloc"]}
    assert h.lib.lgc_reserve_training(h.train) == 0
    out["again"] = h.log()
    out["routes"] = [launches(h, call, args) for call, args, _ in ROUTES]
    out["largest"] = [launches(h, call, args) for call, args in LARGEST]
    h.log()
    dy, x = p(1 << 41), p(1 << 42)
    out["in place"] = [h.lib.lgc_layer_norm_grad(h.train, dy, u64(16), x, u64(16), FP32, rows, u64(16), AT, AT, AT, dx, u64(16), AT, AT, None)
                       for dx, rows in ((dy, u64(8)), (x, u64(8)))]
    out["launched in place"] = h.log()
    out["in place"].append(h.lib.lgc_layer_norm_grad(h.train, dy, u64(16), x, u64(16), FP32, u64(0), u64(16), AT, AT, AT, dy, u64(16), AT, AT, None))
    h.log()
    out["allocated by calls"] = sum("malloc" in str(x) for x in out["routes"] + out["largest"])
    print(json.dumps(out))
