"""What the training step's calls refuse, before they touch a device (CPU only: no kernel is launched)."""
import ctypes as C
import os

import pytest
import torch

from paper_2103_08870_amd import binding as B
from paper_2103_08870_amd import build

import training_reference as ref


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        build.build()
    return B.lib()


def test_null_context_is_refused(lib):
    p = 1 << 20
    calls = [("lgc_reserve_training", ()), ("lgc_quantize", (p, 0, 1, 128, 128, p, p, None)),
             ("lgc_quantize_weights", (p, 0, 1, 128, 128, p, p, None, None, None)), ("lgc_dequantize", (p, p, 1, 1, 128, p, 0, 128, None)),
             ("lgc_layer_norm", (p, 0, 1, 128, 128, None, None, 1e-5, p, 128, None, None, None, None, None)),
             ("lgc_layer_norm_grad", (p, 128, p, 128, 0, 1, 128, None, p, p, p, 128, None, None, None)),
             ("lgc_activate", (0, p, 0, 1, 128, 128, p, 128, None, None, None, None, None)),
             ("lgc_activate_grad", (0, p, 0, 1, 128, 128, p, p, p, 128, None, None, None)),
             ("lgc_product", (p, p, 1, p, p, 128, 128, None, p, 0, 128, None)), ("lgc_weight_grad", (p, 0, 1, 128, 128, p, p, 128, p, None, None))]
    for name, args in calls:
        assert getattr(lib, name)(None, *args) == B.LGC_EINVAL, name
        assert b"ctx" in lib.lgc_last_error(None)


def test_strides(lib):
    for cols in (0, 1, 127, 128, 129, 512, 513, 5000):
        wide = (cols + 127) // 128
        assert B.lgc_codes_stride(cols) == 128 * wide and B.lgc_exps_stride(cols) == (wide + 3) // 4 * 4


def test_blocks_shapes():
    b = B.Blocks
    with pytest.raises(ValueError):
        b(3, 200, codes=torch.empty((3, 256), dtype=torch.uint8), exps=torch.empty((3, 2), dtype=torch.uint8))
    with pytest.raises(ValueError):
        b(3, 200, codes=torch.empty((3, 200), dtype=torch.uint8), exps=torch.empty((3, 4), dtype=torch.uint8))
    with pytest.raises(ValueError):
        b(3, 200, codes=torch.empty((3, 256), dtype=torch.int8), exps=torch.empty((3, 4), dtype=torch.uint8))
    with pytest.raises(ValueError):                      # host memory
        b(3, 200, device="cpu")


def test_the_reference_s_numbers():
    assert len(ref.NUMBERS) == 127 and float(ref.NUMBERS[-1]) == 448.0 and float(ref.NUMBERS[1]) == 2.0 ** -9 and float(ref.NUMBERS[8]) == 2.0 ** -6
    x = torch.tensor([[448.0, 16.5, 17.5, 0.001, -2.0 ** -10, -448.0]])       # 16.5, 17.5: half-way and half-way less one step of 2
    c, e = ref.codes(x, 1)
    assert int(e[0, 0]) == 127 and ref.values(c, e, 1, 6).tolist() == [[448.0, 16.0, 18.0, 2.0 ** -9 * 1, -0.0, -448.0]]
    assert int(ref.exponents(torch.tensor([[449.0]]), 1)[0, 0]) == 128 and int(ref.exponents(torch.zeros((1, 1)), 1)[0, 0]) == 10
