"""Dropout, the linear layer and group norm where an element's place passes 32 bits: rows and groups at both ends and about that place, against
the oracle's formulas in 64 bits.

Tolerances.  As in the other tests of these operators: a rounding to bfloat16 is within 2^-8 of the value, a sum of n terms within n units 2^-24 of
the magnitudes summed.  Group norm sums a channel's positions in chunks of 256 at most, each by eight teams or more, then the teams and the chunks:
147 + 8 + 256 terms of one sum here, and a few roundings."""
import numpy as np
import pytest

import block_checks as T
from oracle import blocks as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    import torch
    dev = T.device()
    if torch.cuda.mem_get_info()[0] < 64 << 30:
        pytest.skip("less than 64 GiB of memory are free")
    yield dev
    torch.cuda.empty_cache()


def _filled(shape, dev, seed):
    """bfloat16 in [-1, 1): 2^24 + 3 values over and over, so that places 2^32 apart differ."""
    import torch
    period = (1 << 24) + 3
    one = (torch.rand(period, generator=torch.Generator().manual_seed(seed)) * 2 - 1).bfloat16().to(dev)
    out = torch.empty(int(np.prod(shape)), dtype=torch.bfloat16, device=dev)
    for i in range(0, out.numel(), period):
        out[i:i + period] = one[:min(period, out.numel() - i)]
    return out.view(shape)


def _factor(rows, C, p, state):
    """keep_factor of some rows."""
    t, (key, call) = O.threshold(p), state.tolist()
    q, r = np.meshgrid(np.arange((C + 7) // 8), rows)
    words = O.philox((q, r, np.full_like(r, call & 0xFFFFFFFF), np.full_like(r, call >> 32)), (key & 0xFFFFFFFF, key >> 32))
    kept = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], -1).reshape(len(rows), -1)[:, :C] >= t
    return np.where(kept, 65536 / (65536 - t), 0.0)


def _rows(N, C):
    """The first, the last, and those about place 2^32."""
    at = 2 ** 32 // C
    assert at + 2 < N - 2
    return np.array([0, 1, at - 1, at, at + 1, at + 2, N - 2, N - 1])


@pytest.mark.parametrize("R,C", [(270001, 16000), (268001, 16033), (3, 1500000008)])
def test_dropout(dev, R, C):
    from paper_1802_06058_amd import vgc
    x = _filled((R, C), dev, 1)
    state, some = T.rng_state(dev), slice(None) if C < 1 << 20 else slice(C - 100000 - (C - 100000) % 8, C)
    rows = _rows(R, C) if C < 1 << 20 else np.arange(R)
    before = T.back(x[rows][:, some] if C < 1 << 20 else x[:, some])
    vgc.dropout(x, 0.25, state, x)
    got = T.back(x[rows][:, some] if C < 1 << 20 else x[:, some])
    if C < 1 << 20:
        f = _factor(rows, C, 0.25, state)
    else:
        t, (key, call), q0 = O.threshold(0.25), state.tolist(), some.start // 8
        q, r = np.meshgrid(q0 + np.arange((C + 7) // 8 - q0), rows)
        words = O.philox((q, r, np.full_like(r, call & 0xFFFFFFFF), np.full_like(r, call >> 32)), (key & 0xFFFFFFFF, key >> 32))
        f = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], -1).reshape(len(rows), -1)[:, :C - some.start]
        f = np.where(f >= t, 65536 / (65536 - t), 0.0)
    want = before * f
    assert (np.abs(got - want) <= (T.half_unit("bf16") + 4 * T.U) * np.abs(want)).all()


def test_linear_and_its_backward_pass(dev):
    import torch
    from paper_1802_06058_amd import vgc
    B, P, K, C, p = 9, 30001, 64, 16000, 0.25
    N = B * P
    X, W, y = _filled((B, P, K), dev, 2), _filled((K, C), dev, 3), _filled((B, P, C), dev, 4)
    z, state, rows = torch.empty_like(y), T.rng_state(dev), _rows(N, C)
    bias = torch.rand(C, device=dev)
    residual = T.back(y.view(N, C)[rows])
    vgc.linear(X, W, y, bias, vgc.ACT_RELU, z, y, p, state, T.workspace(vgc.linear_workspace_bytes(vgc.BF16, N, K, C), dev))
    f = _factor(rows, C, p, state)
    want, z64 = O.linear(T.back(X.view(N, K)[rows]), T.back(W), T.back(bias), 1, f, residual)
    err = (K + 16) * 2 * T.U * (np.abs(T.back(X.view(N, K)[rows])) @ np.abs(T.back(W)) + 1)
    assert (np.abs(T.back(z.view(N, C)[rows]) - z64) <= err + T.half_unit("bf16") * (np.abs(z64) + err)).all()
    tol = f * err + 4 * T.U * np.abs(want)
    assert (np.abs(T.back(y.view(N, C)[rows]) - want) <= tol + T.half_unit("bf16") * (np.abs(want) + tol)).all()
    # backward: y's place is its gradient, and dz's
    dX, s = torch.empty(B, P, K, dtype=y.dtype, device=dev), torch.empty(C, device=dev)
    cols = torch.tensor([0, 7, 8, C - 1], device=dev)
    dy, zc = T.back(y.view(N, C)[rows]), T.back(z.view(N, C)[rows])
    ones = T.back((y[:, :, cols].double().abs() * (z[:, :, cols] > 0)).sum(1))
    vgc.linear_backward(y, z, W, vgc.ACT_RELU, 0.5, y, dX, s, None, None, p, state, T.workspace(vgc.linear_backward_workspace_bytes(vgc.BF16, B, P, K, C), dev))
    dz = T.back(y.view(N, C)[rows])
    want = dy * f * (zc > 0)
    assert (np.abs(dz - want) <= (T.half_unit("bf16") + 4 * T.U) * np.abs(want)).all()
    want = dz @ T.back(W).T
    err = (C + 16) * 2 * T.U * (np.abs(dz) @ np.abs(T.back(W)).T)
    assert (np.abs(T.back(dX.view(N, K)[rows]) - want) <= err + T.half_unit("bf16") * (np.abs(want) + err)).all()
    # the sums are of dz before it was rounded, each within half a unit of the dz that is left
    left = y[:, :, cols].double()
    H, size = T.back(left.sum(1)), T.back(left.abs().sum(1))
    off = size * (1.01 * T.half_unit("bf16") + (P + 64) * T.U)
    got = T.back(s[cols])
    assert (size <= ones * 1.4).all() and (np.abs(got - 0.25 * (H * H).sum(0)) <= 0.25 * (2 * np.abs(H) * off + off * off).sum(0) + (B + 4) * T.U * got).all()


def test_group_norm_and_its_backward_pass(dev):
    import torch
    from paper_1802_06058_amd import vgc
    B, P, C, G = 3, 300007, 4800, 32
    w, n = C // G, (147 + 8 + 256 + 32) * T.U
    x, y = _filled((B, P, C), dev, 5), torch.empty(B, P, C, dtype=torch.bfloat16, device=dev)
    gamma, beta = torch.rand(C, device=dev) + 0.5, torch.rand(C, device=dev) - 0.5
    mean, rstd = torch.empty(B, G, device=dev), torch.empty(B, G, device=dev)
    vgc.group_norm(x, gamma, beta, 1e-5, vgc.ACT_RELU, y, mean, rstd, T.workspace(vgc.group_norm_workspace_bytes(vgc.BF16, B, P, C, G), dev))
    dx = torch.empty_like(y)
    sums = [torch.empty(C, device=dev) for _ in range(2)]
    vgc.group_norm_backward(y, x, mean, rstd, gamma, beta, vgc.ACT_RELU, 0.5, dx, *sums, workspace=T.workspace(vgc.group_norm_backward_workspace_bytes(vgc.BF16, B, P, C, G), dev))
    for b, q in ((0, 0), (2, 31), (1, 5)):
        at = slice(q * w, q * w + w)
        v, ga, be = x[b, :, at].double(), gamma[at].double(), beta[at].double()
        m = v.mean()
        r = 1 / ((v - m).square().mean() + 1e-5).sqrt()
        xhat = (v - m) * r
        off = n * (1 + xhat.abs()) * 2                       # mean and rstd within n of the standard deviation
        t = xhat * ga + be
        want, tol = t.clamp(min=0), off * ga + 4 * T.U * (1 + t.abs())
        assert ((y[b, :, at].double() - want).abs() <= tol + T.half_unit("bf16") * (want + tol)).all(), (b, q)
        dy = y[b, :, at].double()
        e = torch.where(t > 0, dy, 0)                        # (where rounding decides the sign, dy is 0 or as small as that)
        d = e * ga
        want = r * (d - d.mean() - xhat * (d * xhat).mean())
        tol = r * (3 * n * (d.abs() + d.abs().mean() + (1 + xhat.abs()) * (d * xhat).abs().mean()) + off * (d * xhat).mean().abs() + 2 * tol)
        assert ((dx[b, :, at].double() - want).abs() <= tol + T.half_unit("bf16") * (want.abs() + tol)).all(), (b, q)
    at = slice(C - w, C)
    g = h = g_off = h_off = 0
    for b in range(B):
        v, t = x[b, :, at].double(), None
        m = v.mean()
        xhat = (v - m) / ((v - m).square().mean() + 1e-5).sqrt()
        t = xhat * gamma[at].double() + beta[at].double()
        e = torch.where(t > 0, y[b, :, at].double(), 0)
        G_z, H_z = (e * xhat).sum(0), e.sum(0)
        eg, eh = 4 * n * (e * (1 + xhat.abs())).sum(0), 4 * n * e.sum(0)
        g, h = g + G_z * G_z, h + H_z * H_z
        g_off, h_off = g_off + 2 * G_z.abs() * eg + eg * eg, h_off + 2 * H_z.abs() * eh + eh * eh
    assert ((sums[0][at].double() - 0.25 * g).abs() <= 0.25 * g_off + 8 * T.U * g).all()
    assert ((sums[1][at].double() - 0.25 * h).abs() <= 0.25 * h_off + 8 * T.U * h).all()
