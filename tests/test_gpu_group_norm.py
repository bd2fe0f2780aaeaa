"""Group norm with an activation and its backward pass with the sums over the samples, against the oracle in 64 bits.

Tolerances.  A sum over a group: a lane adds at most a chunk's rows of its team, then lanes, teams and channels follow; D = 300 + P / 8 + w / 32
roundings of U = 2^-24 of the magnitudes summed cover them (twice that where values are taken relative to their first rows' mean).  The moments' errors reach xhat
as in layer norm's tests; an activation's slope is at most 1.13, and a slope changes by at most the change of its argument.  relu's slope jumps at 0: where gamma xhat + beta
is nearer to it than its own error, the tests' dy is 0."""
import numpy as np
import pytest

from oracle import blocks as O
import block_checks as T

pytestmark = pytest.mark.gpu
U = T.U
EPS = 1e-5


@pytest.fixture(scope="module")
def dev():
    return T.device()


def _case(B, P, C, G, dtype, dev):
    gen = np.random.default_rng(B + 3 * P + 5 * C + 7 * G)
    x = gen.standard_normal((B, P, C)) * np.exp(0.5 * gen.standard_normal(C)) + gen.standard_normal(C) + gen.standard_normal((B, 1, 1))
    gamma, beta = (1 + 0.2 * gen.standard_normal(C)).astype(np.float32), (0.3 * gen.standard_normal(C)).astype(np.float32)
    return gen, T.to(x, dtype, dev), gamma, beta


def _by_channel(v, C):
    return np.repeat(v, C // v.shape[1], 1)[:, None, :]


def _forward(dev, B, P, C, G, act, dtype):
    import torch
    from paper_1802_06058_amd import vgc
    gen, x, gamma, beta = _case(B, P, C, G, dtype, dev)
    y, after_y = T.guarded(x.numel(), x.dtype, dev)
    mean, after_m = T.guarded(B * G, torch.float32, dev)
    rstd, after_r = T.guarded(B * G, torch.float32, dev)
    code = vgc.F32 if dtype == "f32" else vgc.BF16
    ws = T.workspace(vgc.group_norm_workspace_bytes(code, B, P, C, G), dev)
    vgc.group_norm(x, torch.from_numpy(gamma).to(dev), torch.from_numpy(beta).to(dev), EPS, T.ACTS[act], y.view(x.shape), mean.view(B, G), rstd.view(B, G), ws)
    assert T.untouched(after_y, after_m, after_r)
    x64 = T.back(x)
    want, m, r, xhat = O.group_norm(x64, G, gamma, beta, EPS, T.ACTS[act])
    d = 2 * (300 + P / 8 + C // G / 32) * U
    size = np.abs(x64).reshape(B, P, G, -1).mean((1, 3))
    err_m = d * size
    err_r = r * (2 * d + 8 * U + 2 * r * err_m)
    assert (np.abs(T.back(mean).reshape(B, G) - m) <= err_m + U * np.abs(m)).all()
    assert (np.abs(T.back(rstd).reshape(B, G) - r) <= err_r).all()
    rc = _by_channel(r, C)
    err_h = rc * _by_channel(err_m, C) + np.abs(xhat) * _by_channel(err_r / r, C) + 4 * U * np.abs(xhat) + U * rc * np.abs(x64)
    t = xhat * gamma + beta
    tol = 1.13 * (np.abs(gamma) * err_h + 4 * U * (np.abs(xhat * gamma) + np.abs(beta))) + (T.act_error(t, want) if act in ("gelu", "silu") else 0)
    got = T.back(y).reshape(x.shape)
    bad = np.abs(got - want) > tol * (1 + 2.0 ** -8) + (T.half_unit(dtype) * np.abs(want) if dtype == "bf16" else 0)
    assert not bad.any(), np.argwhere(bad)[:5]


#         held by one workgroup: one group, several, odd widths, cut last slabs; then by chunks, of few and many columns
SIZES = [(1, 1, 1, 1), (1, 2, 3, 3), (2, 1, 8, 1), (3, 5, 7, 1), (2, 9, 10, 5), (4, 49, 64, 32), (3, 49, 512, 8), (2, 49, 2048, 32), (1, 100, 130, 2), (2, 33, 99, 9), (5, 16, 24, 8), (2, 7, 520, 1),
         (2, 300, 96, 32), (1, 513, 64, 2), (3, 1000, 40, 5), (2, 784, 72, 9), (1, 1, 4096, 2), (1, 1025, 64, 32),
         (2, 2000, 64, 32), (1, 5000, 3, 1), (2, 3136, 24, 3), (1, 4100, 17, 17), (3, 700, 1056, 1), (1, 900, 4096, 2), (2, 20000, 8, 2), (1, 1500, 264, 11), (70, 600, 512, 1)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,P,C,G", SIZES)
def test_forward(dev, B, P, C, G, dtype):
    _forward(dev, B, P, C, G, list(T.ACTS)[(B + P + C) % 4], dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", list(T.ACTS))
@pytest.mark.parametrize("P", [30, 3000])
def test_forward_activations(dev, P, act, dtype):
    _forward(dev, 2, P, 48, 6, act, dtype)


def _backward(dev, B, P, C, G, act, dtype, with_g=True):
    import torch
    from paper_1802_06058_amd import vgc
    gen, x, gamma, beta = _case(B, P, C, G, dtype, dev)
    x64 = T.back(x)
    _, m, r, _ = O.group_norm(x64, G, gamma, beta, EPS, 0)
    m32, r32 = m.astype(np.float32), r.astype(np.float32)
    rc, mc = _by_channel(r32.astype(float), C), _by_channel(m32.astype(float), C)
    xhat = (x64 - mc) * rc
    t = xhat * gamma + beta
    err_h = 3 * U * np.abs(xhat) + U * rc * np.abs(x64)
    err_t = np.abs(gamma) * err_h + 3 * U * (np.abs(xhat * gamma) + np.abs(beta))
    dy = gen.standard_normal((B, P, C))
    if act == "relu":
        dy = np.where(np.abs(t) <= 4 * err_t, 0, dy)
    dy = T.to(dy, dtype, dev)
    dx, after_dx = T.guarded(x.numel(), x.dtype, dev)
    sums = {k: T.guarded(C, torch.float32, dev) for k in ("s_gamma", "s_beta", "g_gamma", "g_beta")}
    code = vgc.F32 if dtype == "f32" else vgc.BF16
    ws = T.workspace(vgc.group_norm_backward_workspace_bytes(code, B, P, C, G), dev)
    c = 1.0 / B
    vgc.group_norm_backward(dy, x, torch.from_numpy(m32).to(dev), torch.from_numpy(r32).to(dev), torch.from_numpy(gamma).to(dev), torch.from_numpy(beta).to(dev), T.ACTS[act], c,
                            dx.view(x.shape), *(v[0] if k[0] == "s" or with_g else None for k, v in sums.items()), workspace=ws)
    assert T.untouched(after_dx, *(v[1] for v in sums.values()))
    want, Gz, Hz, ref, e = O.group_norm_backward(T.back(dy), xhat, r32, gamma, beta, T.ACTS[act], c)
    d64 = np.abs(T.back(dy))
    err_e = 2 * U * np.abs(e)
    if act in ("gelu", "silu"):
        err_e = err_e + d64 * (err_t + T.act_error(t, 1.13))
    depth = (300 + P / 8) * U
    eH = err_e.sum(1) + depth * np.abs(e).sum(1)
    eG = (err_e * np.abs(xhat) + np.abs(e) * err_h).sum(1) + depth * np.abs(e * xhat).sum(1)
    for name, S, eS in (("gamma", Gz, eG), ("beta", Hz, eH)):
        eg = c * (eS + (B + 64) * U * np.abs(S)).sum(0)
        es = c * c * ((2 * np.abs(S) + eS) * eS + (B + 64) * 2 * U * S * S).sum(0)
        if with_g:
            assert (np.abs(T.back(sums["g_" + name][0]) - ref["g_" + name]) <= eg + 4 * U * np.abs(ref["g_" + name])).all(), name
        assert (np.abs(T.back(sums["s_" + name][0]) - ref["s_" + name]) <= es + 8 * U * ref["s_" + name]).all(), name
    assert with_g or T.untouched(sums["g_gamma"][0], sums["g_beta"][0])
    w, M = C // G, P * (C // G)
    per_group = lambda v: _by_channel(v.reshape(B, G, w).sum(2) / M, C)
    deep = (100 + w / 32) * U
    m1, m2 = per_group(gamma * Hz), per_group(gamma * Gz)
    e1 = per_group(np.abs(gamma) * (eH + deep * np.abs(Hz)))
    e2 = per_group(np.abs(gamma) * (eG + deep * np.abs(Gz)))
    d = e * gamma
    tol = rc * (np.abs(gamma) * err_e + e1 + np.abs(xhat) * e2 + np.abs(m2) * err_h + 8 * U * (np.abs(d) + np.abs(m1) + np.abs(xhat * m2)))
    bad = np.abs(T.back(dx).reshape(x.shape) - want) > tol * (1 + 2.0 ** -8) + T.half_unit(dtype) * np.abs(want)
    assert not bad.any(), np.argwhere(bad)[:5]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,P,C,G", SIZES)
def test_backward(dev, B, P, C, G, dtype):
    _backward(dev, B, P, C, G, list(T.ACTS)[(B + P + C + 1) % 4], dtype, with_g=(P + C) % 3 != 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", list(T.ACTS))
@pytest.mark.parametrize("P", [30, 3000])
def test_backward_activations(dev, P, act, dtype):
    _backward(dev, 2, P, 48, 6, act, dtype)


@pytest.mark.parametrize("P", [40, 4000])
def test_large_means_constant_groups_and_values_that_are_not_finite(dev, P):
    import torch
    from paper_1802_06058_amd import vgc
    B, C, G = 3, 32, 4
    x = torch.randn(B, P, C, device=dev)
    x[0, :, :8] = 3.0                                                # constant: xhat = 0
    x[0, :, 8:16] += 1e4                                             # the squares are of the centred values
    x[1, 5, 9], x[1, P - 1, 31] = float("nan"), float("inf")
    gamma, beta = torch.ones(C, device=dev), torch.full((C,), 0.5, device=dev)
    y, mean, rstd = torch.empty_like(x), torch.empty(B, G, device=dev), torch.empty(B, G, device=dev)
    ws = T.workspace(max(vgc.group_norm_workspace_bytes(vgc.F32, B, P, C, G), vgc.group_norm_backward_workspace_bytes(vgc.F32, B, P, C, G)), dev)
    vgc.group_norm(x, gamma, beta, EPS, vgc.ACT_NONE, y, mean, rstd, ws)
    assert (y[0, :, :8] == 0.5).all()
    v = T.back(x[0, :, 8:16])
    want = (v - v.mean()) / np.sqrt(v.var() + EPS) + 0.5
    assert np.abs(T.back(y[0, :, 8:16]) - want).max() <= (300 + P / 8) * 4 * U * 1e4
    bad = torch.isnan(y).all(1)
    assert torch.equal(bad, ~torch.isfinite(y).all(1))
    assert bad[1].tolist() == [False] * 8 + [True] * 8 + [False] * 8 + [True] * 8 and not bad[0].any() and not bad[2].any()
    dx, out = torch.empty_like(x), [torch.empty(C, device=dev) for _ in range(4)]
    vgc.group_norm_backward(torch.ones_like(x), x, mean, rstd, gamma, beta, vgc.ACT_NONE, 1.0, dx, *out, workspace=ws)
    assert torch.equal(~torch.isfinite(dx).all(1), bad)
    assert (~torch.isfinite(out[0])).tolist() == bad[1].tolist() and torch.equal(out[1], torch.full((C,), 3.0 * P * P, device=dev))


@pytest.mark.parametrize("P", [50, 2500])
def test_images_repeat_bit_for_bit_and_side_by_side(dev, P):
    """[B, height, width, C]; two streams with a workspace each."""
    import torch
    from paper_1802_06058_amd import vgc
    B, C, G = 4, 96, 12
    x = torch.randn(B, P // 10, 10, C, device=dev).to(torch.bfloat16)
    gamma, beta = torch.randn(C, device=dev), torch.randn(C, device=dev)
    need = max(vgc.group_norm_workspace_bytes(vgc.BF16, B, P, C, G), vgc.group_norm_backward_workspace_bytes(vgc.BF16, B, P, C, G))

    def run():
        ws, mean, rstd = T.workspace(need, dev), torch.empty(B, G, device=dev), torch.empty(B, G, device=dev)
        y, dx, out = torch.empty_like(x), torch.empty_like(x), [torch.empty(C, device=dev) for _ in range(4)]
        vgc.group_norm(x, gamma, beta, EPS, vgc.ACT_SILU, y, mean, rstd, ws)
        vgc.group_norm_backward(y, x, mean, rstd, gamma, beta, vgc.ACT_SILU, 0.25, dx, *out, workspace=ws)
        return [y, mean, rstd, dx, *out]

    first = run()
    torch.cuda.synchronize()
    streams, results = [torch.cuda.Stream() for _ in range(2)], []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            results.append(run())
    torch.cuda.synchronize()
    for r in results:
        assert all(torch.equal(a, b) for a, b in zip(first, r))


# what SIZES leaves out of the forms that hold a sample (tests/test_group_norm_forms.py counts them)
HELD = [(2, 500, 64, 1), (1, 300, 32, 2), (2, 800, 96, 12), (3, 400, 60, 12), (2, 250, 75, 3), (2, 200, 512, 4), (2, 790, 40, 8), (3, 200, 75, 3), (2, 130, 40, 1), (4, 110, 99, 9), (3, 60, 96, 12)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,P,C,G", HELD)
def test_forms_that_hold_a_sample(dev, B, P, C, G, dtype):
    _forward(dev, B, P, C, G, "gelu", dtype)
    _backward(dev, B, P, C, G, "silu", dtype)


def test_more_held_samples_than_a_launch_takes(dev):
    """A slab a sample, 2^20 samples a launch: the second one's samples, statistics and sums lie behind the first one's."""
    import ctypes
    import torch
    from paper_1802_06058_amd import vgc
    B, P, C, G = (1 << 20) + 5, 2, 8, 2
    for backward in (0, 1):
        form = (ctypes.c_uint32 * 6)()
        assert vgc.load().vgc_form_group_norm(vgc.BF16, backward, B, P, C, G, form) == 0 and form[0] == 1 and form[4] == 1 << 20
    x = torch.randn(B, P, C, device=dev, generator=torch.Generator(device=dev).manual_seed(3)).to(torch.bfloat16)
    dy = torch.randn(B, P, C, device=dev, generator=torch.Generator(device=dev).manual_seed(4)).to(torch.bfloat16)
    gamma, beta = torch.linspace(0.5, 1.5, C, device=dev), torch.linspace(-0.5, 0.5, C, device=dev)
    some = torch.tensor([0, 1, (1 << 20) - 1, 1 << 20, (1 << 20) + 1, B - 1], device=dev)

    def run(x, dy, s_of_all=True):
        n = x.shape[0]
        y, dx, mean, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(n, G, device=dev), torch.empty(n, G, device=dev)
        out = [torch.empty(C, device=dev) for _ in range(4)]
        vgc.group_norm(x, gamma, beta, EPS, vgc.ACT_SILU, y, mean, rstd, T.workspace(vgc.group_norm_workspace_bytes(vgc.BF16, n, P, C, G), dev))
        vgc.group_norm_backward(dy, x, mean, rstd, gamma, beta, vgc.ACT_SILU, 1.0, dx, *out, workspace=T.workspace(vgc.group_norm_backward_workspace_bytes(vgc.BF16, n, P, C, G), dev))
        return (y, dx, mean, rstd), out

    whole, sums = run(x, dy)
    few, _ = run(x[some].contiguous(), dy[some].contiguous())
    for a, b in zip(whole, few):                                     # (a sample's results do not depend on the others)
        assert torch.equal(a[some], b)
    # the sums over all samples, from their own gradients in 64 bits
    v = x.double().view(B, P, G, C // G)
    m, r = whole[2].double()[:, None, :, None], whole[3].double()[:, None, :, None]
    xhat = ((v - m) * r).view(B, P, C)
    t = xhat * gamma.double() + beta.double()
    sig = torch.sigmoid(t)
    e = dy.double() * (sig + t * sig * (1 - sig))
    for S, g, s in (((e * xhat).sum(1), sums[2], sums[0]), (e.sum(1), sums[3], sums[1])):
        n = 200 * U                                                  # roundings of a sample's terms (as in the other tests, with values of a few units)
        eS = n * (e.abs() * (2 + xhat.abs())).sum(1)
        assert ((g.double() - S.sum(0)).abs() <= (eS + (B / 64 + 64) * U * S.abs()).sum(0)).all()
        assert ((s.double() - (S * S).sum(0)).abs() <= ((2 * S.abs() + eS) * eS + (B / 64 + 64) * U * S * S).sum(0)).all()
