"""How many digits the linear layer's results keep, beyond what the worst cases of its other tests tell.

A bfloat16 result is the nearest one to the formula's value, or its neighbour only where the value lies within its float32 error of the middle between
the two: half a step at value v is 2^(floor(log2 |v|) - 8)."""
import numpy as np
import pytest

import block_checks as T
from oracle import blocks as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return T.device()


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_activations_of_bfloat16_results_are_the_nearest(dev, act):
    """z as given, through a weight of one: every bfloat16 from 2^-6 to 2^3, of both signs."""
    import torch
    from paper_1802_06058_amd import vgc
    bits = torch.arange(int(127 - 6) << 7, int(127 + 3) << 7, dtype=torch.int32)
    z = torch.cat([bits, bits + 0x8000]).to(torch.int16).view(torch.bfloat16).to(dev)
    N = z.numel()
    y, one = torch.empty_like(z), torch.ones(1, 1, dtype=z.dtype, device=dev)
    vgc.linear(z.view(N, 1), one, y.view(N, 1), None, T.ACTS[act], workspace=T.workspace(vgc.linear_workspace_bytes(vgc.BF16, N, 1, 1), dev))
    z64 = T.back(z)
    want = O.act(z64, T.ACTS[act])
    half = np.exp2(np.floor(np.log2(np.abs(want))) - 8)
    tol = T.act_error(z64, want)
    bad = np.abs(T.back(y) - want) > half + tol
    assert not bad.any(), (int(bad.sum()), z64[bad][:5])
