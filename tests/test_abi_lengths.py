"""Sizes that pass 32 bits: the library's sizes are uint32, into which ctypes puts any integer modulo 2^32, so the binding has to refuse them.  Tensors of
such sizes here have no memory ("meta"); nothing is launched."""
import ctypes

import pytest
import torch

from paper_1802_06058_amd import vgc

OVER = 1 << 32


def _none(*shape, dtype=torch.bfloat16):
    return torch.empty(*shape, dtype=dtype, device="meta")


@pytest.mark.parametrize("sizes", [(OVER + 4, 3, 40), (4, OVER + 3, 40), (4, 3, OVER + 40), (3 * OVER + 4, 3, 40)])
def test_workspaces_of_a_linear_layer(sizes):
    with pytest.raises(vgc.VgcError, match="32 bits"):
        vgc.linear_workspace_bytes(vgc.F32, *sizes)
    with pytest.raises(vgc.VgcError, match="32 bits"):
        vgc.linear_backward_workspace_bytes(vgc.BF16, 2, *sizes)
    with pytest.raises(vgc.VgcError, match="32 bits"):
        vgc.linear_backward_workspace_bytes(vgc.BF16, *sizes, 24)


@pytest.mark.parametrize("sizes", [(OVER + 2, 5000, 24, 4), (2, OVER + 5000, 24, 4), (2, 5000, OVER + 24, 4), (2, 5000, 24, OVER + 4)])
def test_workspaces_of_group_norm(sizes):
    for bytes_of in (vgc.group_norm_workspace_bytes, vgc.group_norm_backward_workspace_bytes):
        with pytest.raises(vgc.VgcError, match="32 bits"):
            bytes_of(vgc.F32, *sizes)


def test_calls():
    f32, ws = torch.float32, _none(1 << 20, dtype=torch.uint8)
    rng = _none(2, dtype=torch.int64)
    with pytest.raises(vgc.VgcError, match="32 bits"):
        vgc.dropout(_none(OVER + 8), 0.5, rng, _none(OVER + 8))
    with pytest.raises(vgc.VgcError, match="32 bits"):                     # rows
        vgc.linear(_none(OVER + 4, 3), _none(3, 2), _none(OVER + 4, 2), workspace=ws)
    with pytest.raises(vgc.VgcError, match="32 bits"):                     # a row
        vgc.linear(_none(1, OVER + 8), _none(OVER + 8, 1), _none(1, 1), workspace=ws)
    with pytest.raises(vgc.VgcError, match="32 bits"):                     # an output's row
        vgc.linear(_none(1, 1), _none(1, OVER + 8), _none(1, OVER + 8), workspace=ws)
    with pytest.raises(vgc.VgcError, match="32 bits"):
        vgc.linear_backward(_none(1, OVER + 4, 2), None, _none(3, 2), vgc.ACT_NONE, 1.0, _none(1, OVER + 4, 2), workspace=ws)
    with pytest.raises(vgc.VgcError, match="32 bits"):
        vgc.linear_backward(_none(1, 4, 1), None, _none(OVER + 8, 1), vgc.ACT_NONE, 1.0, _none(1, 4, 1), workspace=ws)
    for B, P, C, G in ((2, OVER + 9, 8, 2), (OVER + 2, 1, 8, 2), (1, 1, OVER + 8, 1), (1, 9, 8, OVER + 2)):
        x, v, m = _none(B, P, C), _none(C, dtype=f32), _none(B, G, dtype=f32)
        with pytest.raises(vgc.VgcError, match="32 bits"):
            vgc.group_norm(x, v, v, 1e-5, vgc.ACT_NONE, x, m, m, ws)
        with pytest.raises(vgc.VgcError, match="32 bits"):
            vgc.group_norm_backward(x, x, m, m, v, v, vgc.ACT_NONE, 1.0, x, v, v, workspace=ws)


def test_no_size_of_a_tensor_is_taken_modulo_32_bits():
    """Of any operator, also where the binding does not look at a number first.  (The other calls' 32-bit numbers count entries of lists.)"""
    lib = vgc.load()
    operators = [n for n in vgc.EXPORTS if n.startswith(("vgc_sqgrad", "vgc_act8", "vgc_layer_norm", "vgc_softmax_loss", "vgc_dropout", "vgc_linear", "vgc_group_norm"))]
    assert len(operators) > 20
    for name in operators:
        assert ctypes.c_uint32 not in vgc.EXPORTS[name][1], name
    assert lib.vgc_linear_workspace_bytes(vgc.F32, 4, 3, 40) > 0 and lib.vgc_linear_workspace_bytes(vgc.F32, OVER - 1, 3, 40) == 0
    for n in (OVER, OVER + 4, 5 * OVER):
        with pytest.raises(ctypes.ArgumentError):
            lib.vgc_linear_workspace_bytes(vgc.F32, n, 3, 40)
        with pytest.raises(ctypes.ArgumentError):
            lib.vgc_layer_norm_backward_workspace_bytes(2, n, 8)
