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


# float32.  What a product of planes may be off by, in the root mean square and relative to results whose terms are of either sign (r = sqrt(K) of a term):
#   pairs of planes that are not formed: 2^-25 of a term each, 3e-8 r;
#   sums inside the instructions, 12 of them every 32 k, cut off rather than rounded: on average 0.36 units 2^-23 of what is there, 0.7 of sqrt(32) terms, so 12 0.36 0.7 2^-23 =
#   3.6e-7 of a part, and the parts' errors are independent: 3.6e-7 r;
#   K / 32 rounded additions: sqrt(K / 64 / 3) 2^-24 r, 4e-7 at K = 9000;
# together 5.5e-7, held to 1e-6 (measured: 1.3e-7 to 2.4e-7).  Two planes and three products instead of three and six: 4.4e-6.  (The kernel for few rows, which multiplies floats, has K / 64
# rounded sums a wave: less.)
FORWARD = [(4096, 1000, 4096), (2900, 3000, 3000), (840, 424, 1832), (520, 1210, 1100), (260, 1030, 2050), (845, 427, 1829), (284, 3682, 2918), (128, 784, 1000), (3, 6001, 515), (1, 552, 1)]
BACKWARD = [(4096, 4096, 1000), (2100, 3000, 4000), (1143, 1570, 1680), (600, 2401, 601), (273, 2706, 3989), (700, 1500, 300), (2044, 509, 2045), (128, 1000, 784), (268, 87, 5874), (3, 515, 6001)]


@pytest.mark.parametrize("N,K,C", FORWARD)
def test_float32_products_keep_their_digits(dev, N, K, C):
    import torch
    from paper_1802_06058_amd import vgc
    gen = torch.Generator(device=dev).manual_seed(N + K + C)
    X, W = torch.randn(N, K, device=dev, generator=gen), torch.randn(K, C, device=dev, generator=gen) / K ** 0.5
    y = torch.empty(N, C, device=dev)
    vgc.linear(X, W, y, workspace=T.workspace(vgc.linear_workspace_bytes(vgc.F32, N, K, C), dev))
    want = X.double() @ W.double()
    assert float((y.double() - want).norm() / want.norm()) <= 1e-6


@pytest.mark.parametrize("N,K,C", BACKWARD)
def test_float32_input_gradients_keep_their_digits(dev, N, K, C):
    import torch
    from paper_1802_06058_amd import vgc
    gen = torch.Generator(device=dev).manual_seed(N + K + C)
    dy, W = torch.randn(1, N, C, device=dev, generator=gen), torch.randn(K, C, device=dev, generator=gen) / K ** 0.5
    dz, dX = torch.empty_like(dy), torch.empty(1, N, K, device=dev)
    vgc.linear_backward(dy, None, W, vgc.ACT_NONE, 1.0, dz, dX, workspace=T.workspace(vgc.linear_backward_workspace_bytes(vgc.F32, 1, N, K, C), dev))
    want = dy[0].double() @ W.double().t().contiguous()
    assert float((dX[0].double() - want).norm() / want.norm()) <= 1e-6


@pytest.mark.parametrize("N,K,C", [(4096, 4096, 4096), (1500, 4096, 2048), (260, 5000, 2050), (845, 3333, 1829), (409, 8041, 1126), (40, 4100, 300)])
@pytest.mark.parametrize("backward", [False, True])
def test_sums_of_one_sign_do_not_shrink(dev, N, K, C, backward):
    """Terms between 1 and 4 whose parts are all positive: what rounding a value to bfloat16 leaves of it is.  A sum's parts of 32 k are 12 sums that the instructions may cut off, each by a
    unit 2^-23 of what is there, half of the part on average: 7.2e-7 in no case more.  Their K / 32 additions are rounded: sqrt(K / 96 / 3) 2^-24, 3.2e-7 at K = 8000, of either
    sign.  (Left inside the instructions they come out 1.1e-6 to 1.6e-6 too small.)"""
    import torch
    from paper_1802_06058_amd import vgc
    gen = torch.Generator(device=dev).manual_seed(N + K + C)
    rand = lambda *s: torch.rand(*s, device=dev, generator=gen)
    a, b = (1 + torch.floor(127 * rand(*s)) / 128 + 2.0 ** -8 * 0.98 * rand(*s) for s in ((N, K), (C, K)))
    assert bool((a > a.bfloat16()).float().mean() > 0.99)
    got = torch.empty(N, C, device=dev)
    if backward:
        vgc.linear_backward(a.view(1, N, K), None, b, vgc.ACT_NONE, 1.0, torch.empty(1, N, K, device=dev), got.view(1, N, C),
                            workspace=T.workspace(vgc.linear_backward_workspace_bytes(vgc.F32, 1, N, C, K), dev))
    else:
        vgc.linear(a, b.t().contiguous(), got, workspace=T.workspace(vgc.linear_workspace_bytes(vgc.F32, N, K, C), dev))
    want = a.double() @ b.double().t().contiguous()
    off = (got.double() - want) / want
    assert abs(float(off.mean())) <= 7.2e-7 and float(off.square().mean().sqrt()) <= 1.1e-6
