"""Which forms the linear layer's products take, read from the library's own plan (no GPU needed): the GPU tests' sizes have to reach all of them, also after a change of
the estimates that choose."""
import ctypes
import random

import pytest

from paper_1802_06058_amd import vgc

TILES = ("large", "small", "small, two planes", "cut", "cut, half", "cut, quarter", "few rows", "deep", "narrow")


def form(dtype, backward, B, P, K, C):
    """(tile, whether k is shared out, columns and rows of the kernel for few rows, planes of dz)."""
    out = (ctypes.c_uint32 * 5)()
    assert vgc.load().vgc_form_linear(dtype, int(backward), B, P, K, C, out) == 0, (B, P, K, C)
    return TILES[out[0]], "parts" if out[1] > 1 else "whole", out[2], out[3], out[4] if dtype == vgc.BF16 else 1


def _of_the_tests(dtype, backward):
    import test_gpu_linear as L
    import test_gpu_linear_forms as M
    name = "f32" if dtype == vgc.F32 else "bf16"
    named = {test: [m.args[1] for m in getattr(L, test).pytestmark if "K" in m.args[0]][0] for test in dir(L) if test.endswith("products_of_middle_size")}
    if backward:
        sizes = list(L.BACKWARD) + M.BACKWARD[name] + ([(2, 1100, 1000, 514)] if dtype == vgc.F32 else [(2, 1500, 1024, 1024), (4, 1024, 3000, 520), (1, 2100, 1000, 1029)])
        return sizes + list(named["test_backward_of_float32_products_of_middle_size" if dtype == vgc.F32 else "test_backward_of_bfloat16_products_of_middle_size"])
    sizes = [(n, 1, k, c) for n, k, c in list(L.SIZES) + M.FORWARD[name] + [(2500, 64, 4104), (4096, 128, 4096)]]
    return sizes + [(n, 1, k, c) for n, k, c in named["test_float32_products_of_middle_size" if dtype == vgc.F32 else "test_bfloat16_products_of_middle_size"]]


@pytest.mark.parametrize("dtype", [vgc.F32, vgc.BF16])
@pytest.mark.parametrize("backward", [False, True])
def test_the_tests_reach_every_form(dtype, backward):
    gen, found = random.Random(5), {}
    for _ in range(200000):
        N, K, C = int(2 ** gen.uniform(0, 14.2)), int(2 ** gen.uniform(0, 13.2)), int(2 ** gen.uniform(0, 13.2))
        if gen.random() < 0.5:
            K, C = max(8, K // 8 * 8), max(8, C // 8 * 8)
        found.setdefault(form(dtype, backward, N, 1, K, C), (N, K, C))
    reached = {form(dtype, backward, *size) for size in _of_the_tests(dtype, backward)}
    missing = {f: size for f, size in found.items() if f not in reached}
    assert len(found) > 12 and not missing, missing
