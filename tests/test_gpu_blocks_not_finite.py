"""Infinities and NaN through the linear layer and group norm: what they reach, and what they do not."""
import numpy as np
import pytest

import block_checks as T

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def dev():
    return T.device()


def _rand(dev, seed, *shape, dtype="f32"):
    import torch
    return torch.randn(*shape, device=dev, generator=torch.Generator(device=dev).manual_seed(seed)).to(T.dtype_of(dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("B,P,K,C", [(3, 4, 40, 72), (2, 400, 300, 264)])
def test_a_nan_that_an_activation_meets(dev, B, P, K, C, act, dtype):
    """Forward it stays one in its row.  Backward relu's slope is 0 at a NaN of z, so that dz, dX and the sums are what z = -1 there gives; the others' is a NaN,
    which reaches dX's row and its channel's sums alone."""
    import torch
    from paper_1802_06058_amd import vgc
    N, code, c = B * P, vgc.F32 if dtype == "f32" else vgc.BF16, 5
    X, W = _rand(dev, 1, B, P, K, dtype=dtype), _rand(dev, 2, K, C, dtype=dtype)
    ws = T.workspace(max(vgc.linear_workspace_bytes(code, N, K, C), vgc.linear_backward_workspace_bytes(code, B, P, K, C)), dev)
    y, z = (torch.empty(B, P, C, dtype=X.dtype, device=dev) for _ in range(2))
    X[1, 2, 7] = NAN
    vgc.linear(X, W, y, None, T.ACTS[act], z, workspace=ws)
    assert torch.isnan(y[1, 2]).all() and torch.isnan(z[1, 2]).all() and torch.isnan(y).sum() == C
    z, dy = _rand(dev, 3, B, P, C, dtype=dtype), _rand(dev, 4, B, P, C, dtype=dtype)

    def run(value):
        z[1, 2, c] = value
        dz, dX, s, g = torch.empty_like(dy), torch.empty_like(X), torch.empty(C, device=dev), torch.empty(C, device=dev)
        vgc.linear_backward(dy, z, W, T.ACTS[act], 1.0, dz, dX, s, g, workspace=ws)
        return dz, dX, s, g
    got, below = run(NAN), run(-1.0)
    if act == "relu":
        assert got[0][1, 2, c] == 0 and all(torch.equal(a, b) for a, b in zip(got, below))
        return
    dz, dX, s, g = got
    assert torch.isnan(dz).nonzero().tolist() == [[1, 2, c]]
    assert torch.isnan(dX[1, 2]).all() and torch.isnan(dX).sum() == K
    assert torch.isnan(s).nonzero().tolist() == [[c]] == torch.isnan(g).nonzero().tolist()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_dropout_drops_is_nothing(dev, dtype):
    import torch
    from paper_1802_06058_amd import vgc
    N, K, C, code = 33, 40, 72, vgc.F32 if dtype == "f32" else vgc.BF16
    X, W, r, state = _rand(dev, 1, N, K, dtype=dtype), _rand(dev, 2, K, C, dtype=dtype), _rand(dev, 3, N, C, dtype=dtype), T.rng_state(dev)
    X[4, 0] = NAN
    ones, keep = torch.ones(N, C, device=dev), torch.empty(N, C, device=dev)
    vgc.dropout(ones, 0.5, state, keep)
    y = torch.empty_like(r)
    vgc.linear(X, W, y, None, vgc.ACT_GELU, None, r, 0.5, state, T.workspace(vgc.linear_workspace_bytes(code, N, K, C), dev))
    assert torch.equal(torch.isnan(y[4]), keep[4] != 0) and torch.equal(y[4][keep[4] == 0], r[4][keep[4] == 0]) and torch.isnan(y).sum() == (keep[4] != 0).sum()


@pytest.mark.parametrize("act", list(T.ACTS))
@pytest.mark.parametrize("P,value", [(40, NAN), (4000, NAN), (40, INF), (4000, -INF)])
def test_a_group_that_is_not_finite(dev, P, value, act):
    """x: the sample's group in y, rstd and dx, and its channels' sums of gamma; beta's sums, which depend on x through the slope alone, where that is a NaN (gelu, silu)."""
    import torch
    from paper_1802_06058_amd import vgc
    B, C, G = 3, 32, 4
    x, dy = _rand(dev, 5, B, P, C), _rand(dev, 6, B, P, C)
    x[1, 7, 9] = value
    gamma, beta = torch.linspace(0.5, 1.5, C, device=dev), torch.linspace(-0.5, 0.5, C, device=dev)
    y, dx, mean, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(B, G, device=dev), torch.empty(B, G, device=dev)
    ws = T.workspace(max(vgc.group_norm_workspace_bytes(vgc.F32, B, P, C, G), vgc.group_norm_backward_workspace_bytes(vgc.F32, B, P, C, G)), dev)
    vgc.group_norm(x, gamma, beta, 1e-5, T.ACTS[act], y, mean, rstd, ws)
    hit = torch.zeros(B, P, C, dtype=torch.bool, device=dev)
    hit[1, :, 8:16] = True
    assert torch.equal(torch.isnan(y), hit) and torch.equal(~torch.isfinite(y), hit)
    assert torch.isnan(rstd).nonzero().tolist() == [[1, 1]] == (~torch.isfinite(mean)).nonzero().tolist()
    s_gamma, s_beta, g_gamma, g_beta = (torch.empty(C, device=dev) for _ in range(4))
    vgc.group_norm_backward(dy, x, mean, rstd, gamma, beta, T.ACTS[act], 1.0, dx, s_gamma, s_beta, g_gamma, g_beta, ws)
    assert torch.equal(~torch.isfinite(dx), hit)
    channels, none = list(range(8, 16)), []
    for v, want in ((s_gamma, channels), (g_gamma, channels), (s_beta, channels if act in ("gelu", "silu") else none), (g_beta, channels if act in ("gelu", "silu") else none)):
        assert (~torch.isfinite(v)).nonzero().flatten().tolist() == want
    if act == "relu":                                                # that sample's group adds nothing to beta's sums
        others = torch.where(y[:, :, 8:16] > 0, dy[:, :, 8:16], 0).double()
        H = others.sum(1)
        assert (H[1] == 0).all() and ((g_beta[8:16].double() - H.sum(0)).abs() <= (P + 64) * T.U * others.abs().sum((0, 1))).all()


@pytest.mark.parametrize("P,value", [(40, NAN), (4000, NAN), (40, INF), (4000, -INF)])
def test_a_gradient_that_is_not_finite(dev, P, value):
    """dy under relu: where the slope is 1 it reaches its group's dx and its channel's sums, where it is 0 nothing."""
    import torch
    from paper_1802_06058_amd import vgc
    B, C, G = 2, 32, 4
    x, dy = _rand(dev, 7, B, P, C), _rand(dev, 8, B, P, C)
    gamma, beta = torch.ones(C, device=dev), torch.zeros(C, device=dev)
    y, mean, rstd = torch.empty_like(x), torch.empty(B, G, device=dev), torch.empty(B, G, device=dev)
    ws = T.workspace(max(vgc.group_norm_workspace_bytes(vgc.F32, B, P, C, G), vgc.group_norm_backward_workspace_bytes(vgc.F32, B, P, C, G)), dev)
    vgc.group_norm(x, gamma, beta, 1e-5, vgc.ACT_RELU, y, mean, rstd, ws)
    for kept in (True, False):
        p = int(((y[1, :, 20] > 0) == kept).nonzero()[0])
        d = dy.clone()
        d[1, p, 20] = value
        dx, out = torch.empty_like(x), [torch.empty(C, device=dev) for _ in range(4)]
        vgc.group_norm_backward(d, x, mean, rstd, gamma, beta, vgc.ACT_RELU, 1.0, dx, *out, workspace=ws)
        hit = torch.zeros(B, P, C, dtype=torch.bool, device=dev)
        hit[1, :, 16:24] = kept
        assert torch.equal(~torch.isfinite(dx), hit)
        for v in out:
            assert (~torch.isfinite(v)).nonzero().flatten().tolist() == ([20] if kept else [])
