"""Which forms group norm's calls take, read from the library's own plan (no GPU needed): that every compiled form is some call's, and the bounds that the
kernels' comments state."""
import ctypes
import random
import subprocess

import pytest

from paper_1802_06058_amd import vgc


def form(dtype, backward, B, P, C, G):
    out = (ctypes.c_uint32 * 6)()
    assert vgc.load().vgc_form_group_norm(dtype, int(backward), B, P, C, G, out) == 0, (B, P, C, G)
    return dict(zip(("held", "threads", "rows", "groups", "samples", "chunks"), out))


def _sizes(n, seed, longest):
    """(P, w, G): group widths and counts of a workgroup's slab and beyond."""
    gen = random.Random(seed)
    for _ in range(n):
        w, G = int(2 ** gen.uniform(0, 10)), int(2 ** gen.uniform(0, 8))
        yield int(2 ** gen.uniform(0, longest)), w, G


def held_form(dtype, backward, B, P, C, G):
    """(rows a team holds, threads of its launch bounds, how a group's sum is formed or how many moments a lane keeps), as the launches choose them, or None."""
    f, w = form(dtype, backward, B, P, C, G), C // G
    if not f["held"]:
        return None
    if not backward:
        return 2 if f["rows"] <= 2 else 4 if f["rows"] <= 4 else 8, 1024, 2 if f["groups"] == 1 else 1 if w % 8 == 0 else 0
    few = 4 if dtype == vgc.BF16 else 2
    return few // 2 if f["rows"] <= few // 2 else few if f["rows"] <= few else 2 * few, 1024 if f["threads"] == 1024 else 512, 1 if w % 8 == 0 else 8


def _held_forms(dtype, backward):
    return {held_form(dtype, backward, 1, P, w * G, G) for P, w, G in _sizes(60000, 3, 14)} - {None}


@pytest.mark.parametrize("dtype", [vgc.F32, vgc.BF16])
@pytest.mark.parametrize("backward", [False, True])
def test_the_tests_reach_every_held_form(dtype, backward):
    import test_gpu_group_norm as G
    reached = {held_form(dtype, backward, *size) for size in G.SIZES + G.HELD}
    assert _held_forms(dtype, backward) <= reached, _held_forms(dtype, backward) - reached


@pytest.mark.parametrize("name,backward", [("k_group_norm", False), ("k_group_norm_backward", True)])
def test_every_held_form_is_some_calls(name, backward):
    """The launches' host functions are the library's own symbols: <type, rows, ...>."""
    import re
    table = subprocess.run(["nm", "-C", vgc.LIB_PATH], capture_output=True, text=True, check=True).stdout
    built = {"float": set(), "unsigned short": set()}
    for t, a, b, c in re.findall(name + r"<(float|unsigned short), (\d+), (\d+), (\d+)>\(", table):
        built[t].add((int(a), int(b), int(c)) if backward else (int(a), int(c), int(b)))
    for t, dtype in (("float", vgc.F32), ("unsigned short", vgc.BF16)):
        assert built[t] and built[t] == _held_forms(dtype, backward), (t, built[t] ^ _held_forms(dtype, backward))


@pytest.mark.parametrize("dtype", [vgc.F32, vgc.BF16])
@pytest.mark.parametrize("backward", [False, True])
def test_a_sample_has_256_chunks_at_most(dtype, backward):
    """What a group's join has to read, also after a chunk's rows were made whole batches."""
    for B, P, C, G in [(4, 327266, 20, 4), (1, 2 ** 31 - 1, 1, 1), (3, 300007, 4800, 32), (2, 47061, 296, 2)]:
        assert form(dtype, backward, B, P, C, G)["chunks"] <= 256, (B, P, C, G)
    gen = random.Random(9)
    for P, w, G in _sizes(100000, 5, 24):
        assert form(dtype, backward, gen.randint(1, 4), P, w * G, G)["chunks"] <= 256, (P, w, G)
