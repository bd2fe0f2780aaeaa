"""Sizes at the limits of the 8-bit activations' and the softmax loss's entry points, on the host (no pointer here is dereferenced)."""
import pytest

from paper_1802_06058_amd import vgc

SIZE = -2
P = 1 << 20                                          # an aligned address


@pytest.mark.parametrize("R,C", [(1 << 34, 1), (1 << 32, 32), (1 << 36, (1 << 31) - 1), (1 << 40, (1 << 31) - 1), (1 << 30, 1 << 30)])
def test_act8_refuses_what_no_launch_takes(R, C):
    """A launch has fewer than 2^32 threads, each four pieces of eight elements: 2^24 workgroups are one too many, also where the number of
    pieces passes 64 bits."""
    lib = vgc.load()
    assert lib.vgc_act8_encode(vgc.BF16, P, R, C, P, P, None) == SIZE
    assert lib.vgc_act8_decode(vgc.BF16, P, P, R, C, P, None) == SIZE


@pytest.mark.parametrize("N,V", [(1 << 16, 1 << 24), (1 << 20, 1 << 20), (1 << 18, 1 << 22)])
def test_the_loss_of_2_to_the_40_logits_is_a_large_one(N, V):
    """Its working memory is that of its neighbours: a pair a row and 128 classes, not one a row and 16."""
    below, at = (vgc.softmax_loss_workspace_bytes(vgc.BF16, n, 64, V) for n in (N - 256, N))
    assert below < at <= 8 * N * (V // 128) + 4 * N + 512
