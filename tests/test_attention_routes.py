"""Attention, rotary positions and the product's epilogue on the host: what the calls refuse, which kernels they launch for which sizes, and how large the grids get, read from a HIP runtime
that only records (recording_hip.cpp): no GPU, any size.  And the frequencies of rotary positions, which are worked out on the host."""
import ctypes as C
import json
import math
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
if HERE not in sys.path:
    sys.path.insert(0, HERE)
from test_host_routes import Host, ROOT   # noqa: E402,F401  (puts the repository's root in sys.path)
from test_training_routes import launches   # noqa: E402

u32, u64, p, f32, f64 = C.c_uint32, C.c_uint64, C.c_void_p, C.c_float, C.c_double
FP32, BF16 = 0, 1


def at(i):
    return p((1 << 40) + (i << 36))


class Shape(C.Structure):
    _fields_ = [("q_rows", u64), ("kv_rows", u64), ("sequences", u64), ("q_starts", p), ("kv_starts", p), ("heads", u32), ("kv_heads", u32), ("dim", u32), ("scale", f32),
                ("causal", C.c_int32), ("window", u32), ("kv_lengths", p)]


def shape(q_rows=256, kv_rows=256, sequences=1, heads=4, kv_heads=2, dim=64, scale=0.125, causal=1, window=0, q_starts=None, kv_starts=None, kv_lengths=None):
    return Shape(q_rows, kv_rows, sequences, q_starts, kv_starts, heads, kv_heads, dim, scale, causal, window, kv_lengths)


def attention(l, ctx, s, **change):
    wide, narrow = s.heads * s.dim, s.kv_heads * s.dim
    a = dict(q=at(1), ld_q=wide, k=at(2), ld_k=narrow, v=at(3), ld_v=narrow, o=at(4), ld_o=wide, lse=at(5))
    a.update(change)
    return l.lgc_attention(ctx, C.byref(s), a["q"], u64(a["ld_q"]), a["k"], u64(a["ld_k"]), a["v"], u64(a["ld_v"]), a["o"], u64(a["ld_o"]), a["lse"], None)


def attention_grad(l, ctx, s, **change):
    wide, narrow = s.heads * s.dim, s.kv_heads * s.dim
    a = dict(grad=at(6), ld_grad=wide, q=at(1), ld_q=wide, k=at(2), ld_k=narrow, v=at(3), ld_v=narrow, o=at(4), ld_o=wide, lse=at(5), dq=at(7), ld_dq=wide, dk=at(8), ld_dk=narrow,
             dv=at(9), ld_dv=narrow, delta=at(10))
    a.update(change)
    pair = lambda n: (a[n], u64(a["ld_" + n]))  # noqa: E731
    return l.lgc_attention_grad(ctx, C.byref(s), *pair("grad"), *pair("q"), *pair("k"), *pair("v"), *pair("o"), a["lse"], *pair("dq"), *pair("dk"), *pair("dv"), a["delta"], None)


def rotate(l, ctx, rows=8, heads=4, dim=64, dims=64, type=BF16, pairs=0, ld=None, x=at(1), y=at(2), ld_y=None, positions=None, period=0, freqs=at(3), amplitude=1.0):
    ld = heads * dim if ld is None else ld
    return l.lgc_rotate(ctx, x, type, u64(rows), u64(ld), u32(heads), u32(dim), positions, u64(period), freqs, u32(dims), pairs, f32(amplitude), 0, y, u64(ld if ld_y is None else ld_y), None)


def epilogue(l, ctx, m=100, n=300, k=200, type=BF16, act=1, residual=None, z=at(5), ld=None, t=(None, None), z8=(None, None)):
    return l.lgc_product_activate(ctx, at(1), at(1), u64(m), at(2), at(2), u64(n), u64(k), at(3), act, residual, u64(n if residual else 0), z, type, u64(n if ld is None else ld), *t, *z8, None)


ODD = p((1 << 40) + 2)
TWICE = shape(q_starts=at(11).value, kv_starts=at(12).value)
# what is refused: (call, arguments, a word of the message)
REFUSED = [
    (attention, (shape(dim=0),), "dim"), (attention, (shape(dim=136),), "dim"), (attention, (shape(dim=60),), "dim"),
    (attention, (shape(heads=3),), "heads"), (attention, (shape(heads=0, kv_heads=0),), "heads"), (attention, (shape(kv_heads=0),), "heads"), (attention, (shape(heads=1),), "heads"),
    (attention, (shape(heads=1 << 14, kv_heads=1, dim=128),), "2^20"), (attention, (shape(sequences=0),), "sequences"), (attention, (shape(sequences=(1 << 20) + 1),), "sequences"),
    (attention, (shape(q_rows=1 << 20, kv_rows=1 << 20, sequences=1 << 20, heads=8, kv_heads=8, dim=8),), "sequences"),
    (attention, (shape(q_rows=1 << 28),), "q_rows"), (attention, (shape(q_rows=1 << 40),), "q_rows"), (attention, (shape(kv_rows=1 << 29),), "kv_rows"),
    (attention, (shape(scale=0.0),), "scale"), (attention, (shape(scale=-1.0),), "scale"), (attention, (shape(scale=math.nan),), "scale"), (attention, (shape(scale=math.inf),), "scale"), (attention, (shape(scale=1e-38),), "scale"),
    (attention, (shape(q_starts=at(11).value),), "starts"), (attention, (shape(kv_starts=at(11).value),), "starts"),
    (attention, (shape(q_starts=ODD.value, kv_starts=at(11).value),), "starts"), (attention, (shape(sequences=3),), "equal"),
    (attention, (shape(kv_lengths=ODD.value),), "lengths"), (attention_grad, (shape(kv_lengths=at(11).value),), "cache"),
    (attention, (shape(), dict(q=None)), "q is NULL"), (attention, (shape(), dict(k=None)), "k is NULL"), (attention, (shape(), dict(v=None)), "v is NULL"),
    (attention, (shape(), dict(o=None)), "o is NULL"), (attention, (shape(), dict(q=ODD)), "q is not"), (attention, (shape(), dict(ld_k=127)), "k are"),
    (attention, (shape(), dict(ld_v=132)), "v is not"), (attention, (shape(), dict(ld_q=(1 << 24) + 8)), "q is not"), (attention, (shape(), dict(o=at(2))), "overlap"),
    (attention, (shape(), dict(lse=ODD)), "lse"),
    (attention_grad, (shape(dim=4),), "dim"), (attention_grad, (shape(), dict(grad=None)), "grad is NULL"), (attention_grad, (shape(), dict(lse=None)), "lse"),
    (attention_grad, (shape(), dict(delta=None)), "delta"), (attention_grad, (shape(), dict(delta=at(5))), "delta"), (attention_grad, (shape(), dict(dk=None)), "dk is NULL"),
    (attention_grad, (shape(), dict(dq=at(6))), "overlap"), (attention_grad, (shape(), dict(dk=at(2))), "overlap"), (attention_grad, (shape(), dict(dv=at(8))), "one place"),
    (attention_grad, (shape(), dict(ld_dv=130)), "dv is not"),
    (rotate, ((), dict(heads=0)), "heads"), (rotate, ((), dict(heads=1 << 15)), "heads"), (rotate, ((), dict(rows=1 << 24)), "rows"), (rotate, ((), dict(dims=0)), "dims"),
    (rotate, ((), dict(dims=7)), "dims"), (rotate, ((), dict(dims=66)), "dims"), (rotate, ((), dict(type=2)), "type"), (rotate, ((), dict(pairs=2)), "pairs"),
    (rotate, ((), dict(period=1 << 31)), "period"), (rotate, ((), dict(amplitude=math.nan)), "amplitude"), (rotate, ((), dict(freqs=None)), "freqs"), (rotate, ((), dict(freqs=p(4))), "freqs"),
    (rotate, ((), dict(positions=ODD)), "positions"), (rotate, ((), dict(x=None)), "x is NULL"), (rotate, ((), dict(y=None)), "y is NULL"), (rotate, ((), dict(ld=255)), "apart"),
    (rotate, ((), dict(y=at(1), ld_y=260)), "apart"), (rotate, ((), dict(x=p((1 << 40) + 1))), "aligned"),
    (epilogue, ((), dict(act=4)), "non-linearity"), (epilogue, ((), dict(act=-1)), "non-linearity"), (epilogue, ((), dict(type=5)), "type"), (epilogue, ((), dict(n=0)), "n ="),
    (epilogue, ((), dict(k=(1 << 20) + 1)), "k ="), (epilogue, ((), dict(m=1 << 31)), "m ="), (epilogue, ((), dict(ld=299)), "apart"),
    (epilogue, ((), dict(t=(at(6), None))), "codes"), (epilogue, ((), dict(z8=(p((1 << 40) + 8), at(6)))), "codes"), (epilogue, ((), dict(residual=at(7), z=None, t=(at(6), at(6)))), "residual"),
    (epilogue, ((), dict(residual=at(5), ld=308)), "distance"), (epilogue, ((), dict(t=(at(1), at(6)))), "lies where"), (epilogue, ((), dict(t=(at(6), at(6)), z8=(at(6), at(7)))), "lies where"),
    (epilogue, ((), dict(z8=(at(2), at(7)))), "lies where"),
    (epilogue, ((), dict(residual=at(7), z8=(at(6), at(6)))), "residual"), (epilogue, ((), dict(residual=p((1 << 40) + 1))), "aligned"),
]


def call_of(f, args):
    """(positional, keyword) arguments behind the library and the context."""
    return (args[0] if f in (rotate, epilogue) else args[:1]), (args[1] if len(args) > 1 else {})


# sizes and the kernels that they take, with their template's numbers
BIG = dict(q_rows=16384, kv_rows=16384, sequences=4, heads=32, kv_heads=8, dim=128)
LONG = dict(q_rows=16384, kv_rows=16384, heads=8, kv_heads=8, dim=64)
ROUTES = [
    (attention, (shape(**BIG),), ["k_attention 128 1"]), (attention, (shape(**LONG),), ["k_attention 64 1"]), (attention, (shape(dim=8),), ["k_attention 64 2"]),
    (attention, (shape(dim=72),), ["k_attention 96 2"]), (attention, (shape(dim=96),), ["k_attention 96 2"]), (attention, (shape(dim=104),), ["k_attention 128 2"]), (attention, (shape(q_rows=8, kv_rows=32768, sequences=8, heads=32, kv_heads=8, dim=128),), ["k_attention 128 2", "k_attention_join"]),
    (attention, (shape(q_rows=0),), []), (attention, (shape(kv_rows=0),), ["k_attention 64 1"]), (attention, (shape(q_rows=60, kv_rows=60),), ["k_attention 64 1"]),
    (attention, (shape(q_rows=8192, kv_rows=8192, heads=16, kv_heads=16, sequences=2),), ["k_attention 64 1"]),
    (attention_grad, (shape(**BIG),), ["k_attention_dq 128 1", "k_attention_dkv 128 8 1"]), (attention_grad, (shape(**LONG),), ["k_attention_dq 64 1", "k_attention_dkv 64 4 1"]),
    (attention_grad, (shape(**(BIG | dict(dim=96))),), ["k_attention_dq 96 1", "k_attention_dkv 96 8 1"]), (attention_grad, (shape(dim=80),), ["k_attention_dq 96 2", "k_attention_dkv 96 4 2", "k_attention_add"]),
    (attention_grad, (shape(q_rows=64, kv_rows=64, dim=128),), ["k_attention_dq 128 1", "k_attention_dkv 128 4 2"]), (attention_grad, (shape(q_rows=0),), ["k_attention_dkv 64 4 1"]),
    (attention_grad, (shape(kv_rows=0),), ["k_attention_dq 64 1"]), (attention_grad, (shape(q_rows=0, kv_rows=0),), []),
    (attention_grad, (shape(q_rows=8, kv_rows=32768, sequences=8, heads=32, kv_heads=8, dim=128),), ["k_attention_dq 128 2", "k_attention_add", "k_attention_dkv 128 4 1"]),
    (attention_grad, (shape(q_rows=8192, kv_rows=8192, sequences=2, heads=32, kv_heads=8, dim=128),), ["k_attention_dq 128 1", "k_attention_dkv 128 4 2"]),
    (attention_grad, (shape(q_rows=1, kv_rows=65536, heads=1, kv_heads=1),), ["k_attention_dq 64 2", "k_attention_add", "k_attention_dkv 64 4 1"]),
    (attention_grad, (shape(q_rows=65536, kv_rows=100, heads=1, kv_heads=1, causal=0),), ["k_attention_dq 64 1", "k_attention_dkv 64 4 2", "k_attention_add"]),
    (rotate, ((), dict(rows=8)), ["k_rotate 1 1"]), (rotate, ((), dict(rows=8, pairs=1)), ["k_rotate 0 1"]), (rotate, ((), dict(rows=100000)), ["k_rotate 1 4"]), (rotate, ((), dict(rows=0)), []),
    (epilogue, ((), dict(m=1, n=4096, k=16384)), ["k_product_few 1 1 8 0"]), (epilogue, ((), dict(m=1, n=4096, k=16384, t=(at(6), at(6)))), ["k_product_few 1 1 8 0", "k_epilogue"]),
    (epilogue, ((), dict(m=1, n=300, k=16384)), ["k_product_few 1 1 8 0", "k_epilogue"]), (epilogue, ((), dict(m=8192, n=16384, k=4096)), ["k_product 4 2 2 4 0"]),
    (epilogue, ((), dict(m=2000, n=2000, k=300, t=(at(6), at(6)), z8=(at(7), at(7)))), ["k_product 2 2 2 2 0"]), (epilogue, ((), dict(m=8192, n=16384, k=4096, type=FP32)), ["k_product 2 2 2 2 1"]),
    (epilogue, ((), dict(m=512, n=512, k=4096)), ["k_product 2 2 2 2 0", "k_epilogue"]), (epilogue, ((), dict(m=64, n=1 << 20, k=100, t=(at(6), at(6)))), ["k_product 4 2 2 4 0"]),
    (epilogue, ((), dict(m=0)), []), (epilogue, ((), dict(z=None)), []),
]
LARGEST = [(attention, (shape(q_rows=(1 << 29) - 1, kv_rows=(1 << 29) - 1, heads=1, kv_heads=1, dim=8),)), (attention, (shape(q_rows=1 << 20, kv_rows=1 << 20, sequences=1 << 20, heads=4, kv_heads=4, dim=8),)),
           (attention_grad, (shape(q_rows=1 << 22, kv_rows=1 << 22, sequences=1 << 20, heads=64, kv_heads=4, dim=128, q_starts=at(11).value, kv_starts=at(12).value),)),
           (attention_grad, (shape(q_rows=(1 << 29) - 1, kv_rows=(1 << 29) - 1, heads=1, kv_heads=1, dim=128),)),
           (rotate, ((), dict(rows=(1 << 24) - 1, heads=1, dim=2, dims=2))), (rotate, ((), dict(rows=1 << 16, heads=1 << 19, dim=2, dims=2))), (rotate, ((), dict(rows=1 << 16, heads=1, dim=1 << 20, dims=2))),
           (epilogue, ((), dict(m=(1 << 20) - 1, n=1 << 17, k=1000)))]


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


def test_what_is_refused(answers):
    assert len(answers["refused"]) == len(REFUSED)
    for (f, args, word), (status, message, launched) in zip(REFUSED, answers["refused"]):
        assert status == 1 and word in message and launched == 0, (f.__name__, word, status, message)


def test_scratch_has_to_be_reserved(answers):
    assert [x[0] for x in answers["unreserved"]] == [1, 1, 1] and all("lgc_reserve_training" in x[1] for x in answers["unreserved"])


def test_kernels(answers):
    for (f, args, want), (status, got) in zip(ROUTES, answers["routes"]):
        names = [n if n.split()[0] not in ("k_epilogue", "k_attention_join", "k_attention_add") else n.split()[0] for n, _ in got]
        assert status == 0 and names == want, (f.__name__, want, names)


def test_grids_of_the_largest_sizes(answers):
    for (f, args), (status, got) in zip(LARGEST, answers["largest"]):
        assert status == 0 and got, f.__name__
        for name, (x, y, z) in got:
            assert 1 <= x and x * 512 < 1 << 32 and y <= 65535 and z == 1, (f.__name__, name, x, y)


def test_parts_fit_the_scratch(answers):
    """Partial results are never more than the 16 M floats that are reserved."""
    split = 0
    for rows, keys, heads, kv_heads, dim, got in answers["parts"]:
        for name, (x, parts, _) in got:
            if name.startswith("k_attention_join") or name.startswith("k_attention_add"):
                continue
            results = 2 * keys * kv_heads * dim if "dkv" in name else rows * heads * dim
            assert parts == 1 or parts * results <= 16 << 20, (rows, keys, heads, kv_heads, dim, name, parts)
            split += parts > 1
    assert split > 50


def test_frequencies(answers):
    """f_i = base^(-2 i / dims), lowered as the header says, to a few units of the last place of 64 bits."""
    for (dims, base, factor, length, low, high), got in answers["freqs"]:
        for i, f in enumerate(got):
            want = base ** (-2.0 * i / dims)
            w = min(1.0, max(0.0, (length * want / (2 * math.pi) - low) / (high - low))) if length else 0.0
            want *= w + (1 - w) / factor
            assert abs(f - want) <= 1e-14 * want, (dims, base, factor, length, i)
    assert answers["freqs"][0][1][0] == 1.0 and answers["bad_freqs"] == [1] * len(answers["bad_freqs"])


FREQS = [(128, 10000.0, 1.0, 0.0, 1.0, 4.0), (2, 10000.0, 1.0, 0.0, 1.0, 4.0), (64, 500000.0, 8.0, 8192.0, 1.0, 4.0), (40, 10000.0, 4.0, 0.0, 1.0, 4.0), (96, 1e6, 32.0, 4096.0, 1.0, 32.0)]
BAD_FREQS = [(0, 1e4, 1.0, 0.0, 1.0, 4.0), (7, 1e4, 1.0, 0.0, 1.0, 4.0), (8, 0.0, 1.0, 0.0, 1.0, 4.0), (8, math.inf, 1.0, 0.0, 1.0, 4.0), (8, 1e4, 0.0, 0.0, 1.0, 4.0), (8, 1e4, math.nan, 0.0, 1.0, 4.0),
             (8, 1e4, 1.0, -1.0, 1.0, 4.0), (8, 1e4, 1.0, 100.0, 4.0, 4.0), (8, 1e4, 1.0, 100.0, -1.0, 4.0)]


if __name__ == "__main__":
    h = Host(sys.argv[1], sys.argv[2])
    h.lib.lgc_last_error.restype = C.c_char_p
    h.train = h.ctx(1, 1, 1)
    bare = h.train
    out = {"unreserved": [[f(h.lib, bare, *a), h.lib.lgc_last_error(bare).decode()] for f, a in ((attention, (shape(),)), (attention_grad, (shape(),)), (epilogue, ()))]}
    assert h.lib.lgc_reserve_training(h.train) == 0
    out["refused"] = []
    for f, args, _ in REFUSED:
        positional, named = call_of(f, args)
        h.log()
        status = f(h.lib, h.train, *positional, **named)
        out["refused"].append([status, h.lib.lgc_last_error(h.train).decode(), len(h.log())])

    def run(f, args):
        positional, named = call_of(f, args)
        return launches(h, lambda l, ctx: f(l, ctx, *positional, **named), ())

    out["routes"] = [run(f, args) for f, args, _ in ROUTES]
    out["largest"] = [run(f, args) for f, args in LARGEST]
    out["parts"] = []
    for rows in (1, 16, 300, 5000, 60000):
        for keys in (1, 64, 700, 9000, 200000):
            for heads, kv_heads in ((1, 1), (8, 2), (40, 5)):
                for dim in (64, 128):
                    for causal in (0, 1):
                        s = shape(q_rows=rows, kv_rows=keys, heads=heads, kv_heads=kv_heads, dim=dim, causal=causal)
                        out["parts"].append([rows, keys, heads, kv_heads, dim, run(attention, (s,))[1] + run(attention_grad, (s,))[1]])
    room = (f64 * 64)()
    out["freqs"] = []
    for args in FREQS:
        assert h.lib.lgc_rotary_frequencies(room, u32(args[0]), *(f64(x) for x in args[1:])) == 0
        out["freqs"].append([args, list(room)[:args[0] // 2]])
    out["bad_freqs"] = [h.lib.lgc_rotary_frequencies(room, u32(a[0]), *(f64(x) for x in a[1:])) for a in BAD_FREQS] + [h.lib.lgc_rotary_frequencies(None, u32(8), f64(1e4), f64(1), f64(0), f64(1), f64(4))]
    print(json.dumps(out))
