"""The linear layer's backward pass where only dz and the bias's sums are asked for: a first layer's, whose W is not read."""
import pytest

import block_checks as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,P,K,C", [(3, 1, 40, 24), (2, 33, 8, 264), (5, 7, 1000, 131), (2, 300, 96, 1000)])
def test_without_a_weight(B, P, K, C, dtype):
    """What the call with the weight gives, bit for bit: how the sums are formed does not depend on K."""
    import torch
    from paper_1802_06058_amd import vgc
    dev = T.device()
    gen = torch.Generator(device=dev).manual_seed(B + P + K + C)
    dy, z = (torch.randn(B, P, C, device=dev, generator=gen).to(T.dtype_of(dtype)) for _ in range(2))
    W, state = torch.randn(K, C, device=dev, generator=gen).to(dy.dtype), T.rng_state(dev)
    code, out = vgc.F32 if dtype == "f32" else vgc.BF16, []
    for w, k in ((W, K), (None, 1)):
        dz, s, g = torch.empty_like(dy), torch.empty(C, device=dev), torch.empty(C, device=dev)
        ws = T.workspace(vgc.linear_backward_workspace_bytes(code, B, P, k, C), dev)
        vgc.linear_backward(dy, z, w, vgc.ACT_GELU, 1.0 / B, dz, None, s, g, None, 0.25, state, ws)
        out.append((dz, s, g))
    assert all(torch.equal(a, b) for a, b in zip(*out))
    with pytest.raises(vgc.VgcError, match="dX needs W"):
        vgc.linear_backward(dy, z, None, vgc.ACT_GELU, 1.0, out[0][0], torch.empty(B, P, K, dtype=dy.dtype, device=dev), workspace=ws)
    with pytest.raises(vgc.VgcError, match="does not give"):
        vgc.linear_backward(dy, z, W[:, :-1].contiguous(), vgc.ACT_GELU, 1.0, out[0][0], workspace=ws)
