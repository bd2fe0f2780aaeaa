"""Layer norm and its backward pass with the sums over the samples, against the oracle in 64 bits.

Tolerances.  A sum over a row has at most 8 pieces of 8 elements a lane, 6 steps over the wave and 16 over waves in a row:
fewer than 128 roundings of 2^-24 of the magnitudes summed (rows beyond 32768 elements: C / 8192 pieces more a lane); a handful of
roundings for the rest.  An output in bfloat16 adds half a unit, 2^-8 of it covers that.  A column sum over a sample's rows has at most
as many roundings as rows, the sums over teams and samples as many again as there are of them."""
import numpy as np
import pytest

from oracle import operators as O

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def dev():
    import torch
    from paper_1802_06058_amd import vgc
    assert torch.cuda.is_available()
    vgc.load()
    return torch.device("cuda:0")


def _type(dtype):
    import torch
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _np(t):
    return t.double().cpu().numpy()


def _depth(C):
    return 128 + C // 1024


FORWARD = [(1, 1), (5, 1), (3, 2), (7, 7), (4, 8), (9, 33), (130, 64), (1, 512), (3, 513), (2050, 520), (128, 1000), (2100, 1000), (2049, 2048), (2048, 4096),
           (5, 1025), (3, 4097), (1000, 16), (300, 100), (77, 250), (40000, 24), (5, 4100), (2000, 5000), (2, 8192), (2, 8200), (2, 32768), (2, 32776), (3, 40001)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,C", FORWARD)
def test_forward(dev, R, C, dtype):
    import torch
    from paper_1802_06058_amd import vgc
    rng = np.random.default_rng(R * 3 + C)
    x = rng.standard_normal((R, C)) * np.exp(rng.standard_normal((R, 1))) + 3 * rng.standard_normal((R, 1))
    x = torch.from_numpy(x.astype(np.float32)).to(_type(dtype))
    gamma, beta = (1 + 0.2 * rng.standard_normal(C)).astype(np.float32), rng.standard_normal(C).astype(np.float32)
    y = torch.full((R * C + 32,), 7.0, dtype=x.dtype, device=dev)
    mean, rstd = torch.empty(R, device=dev), torch.empty(R, device=dev)
    nb = (C + 31) // 32
    codes, exps = torch.full((R * C + 32,), 9, dtype=torch.int8, device=dev), torch.full((R * nb + 32,), 9, dtype=torch.uint8, device=dev)
    args = (x.to(dev), torch.from_numpy(gamma).to(dev), torch.from_numpy(beta).to(dev), 1e-5)
    vgc.layer_norm(*args, y[:R * C].view(R, C), mean, rstd, (codes, exps))
    x64 = _np(x)
    want, m, r, xhat = O.layer_norm(x64, gamma, beta, 1e-5)
    d, size = _depth(C) * U, np.abs(x64).mean(1)
    err_m = d * size
    err_r = r * (d + 8 * U + r * err_m * 2)          # of the centred squares, and of the mean in them
    err_h = r[:, None] * err_m[:, None] + np.abs(xhat) * (err_r / r)[:, None] + 4 * U * np.abs(xhat) + U * r[:, None] * np.abs(x64)
    out = _np(y[:R * C].view(R, C))
    tol = np.abs(gamma) * err_h + 4 * U * (np.abs(xhat * gamma) + np.abs(beta)) + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0)
    assert (np.abs(_np(mean) - m) <= err_m + U * np.abs(m)).all()
    assert (np.abs(_np(rstd) - r) <= err_r).all()
    assert (np.abs(out - want) <= tol).all()
    kept = O.act8_decode(codes[:R * C].cpu().numpy().reshape(R, C), exps[:R * nb].cpu().numpy().reshape(R, nb))
    unit = np.repeat(np.exp2(exps[:R * nb].cpu().numpy().reshape(R, nb).astype(float) - 127), 32, 1)[:, :C]
    assert (np.abs(kept - xhat) <= unit / 2 + err_h).all()
    assert (y[R * C:] == 7).all() and (codes[R * C:] == 9).all() and (exps[R * nb:] == 9).all()
    y2, m2, r2 = torch.empty_like(y), torch.empty_like(mean), torch.empty_like(rstd)
    vgc.layer_norm(*args, y2[:R * C].view(R, C), m2, r2)                       # without the 8-bit form: the same
    assert torch.equal(y2[:R * C], y[:R * C]) and torch.equal(m2, mean) and torch.equal(r2, rstd)


def test_constant_rows_large_means_and_rows_that_are_not_finite(dev):
    import torch
    from paper_1802_06058_amd import vgc
    R, C = 8, 96
    x = np.random.default_rng(0).standard_normal((R, C)).astype(np.float32)
    x[0] = 3.0                                       # constant: exactly its mean, xhat = 0
    x[1] += 1e4                                      # the sum of squares is of the centred row
    x[2, 5], x[3, 90] = np.nan, np.inf
    x[4] = 0
    gamma, beta = torch.ones(C, device=dev), torch.full((C,), 0.5, device=dev)
    y, mean, rstd = torch.empty(R, C, device=dev), torch.empty(R, device=dev), torch.empty(R, device=dev)
    codes, exps = torch.empty(R, C, dtype=torch.int8, device=dev), torch.empty(R, 3, dtype=torch.uint8, device=dev)
    vgc.layer_norm(torch.from_numpy(x).to(dev), gamma, beta, 1e-5, y, mean, rstd, (codes, exps))
    y = y.cpu().numpy()
    assert (y[0] == 0.5).all() and (y[4] == 0.5).all() and np.isnan(y[2]).all() and np.isnan(y[3]).all()
    assert (exps[2:4] == 255).all() and (codes[2:4] == 0).all()
    ok = [1, 5, 6, 7]
    want = O.layer_norm(x.astype(float)[ok], np.ones(C), np.full(C, 0.5), 1e-5)[0]
    assert np.abs(y[ok] - want).max() < 128 * U * 1e4 * 2 and np.isfinite(y[ok]).all()
    # backward: a row that is not finite reaches its own dx and the sums of its columns
    dy = torch.ones(2, 4, C, device=dev)
    dx = torch.empty_like(dy)
    out = [torch.empty(C, device=dev) for _ in range(4)]
    ws = torch.empty(vgc.layer_norm_backward_workspace_bytes(2, 4, C), dtype=torch.uint8, device=dev)
    vgc.layer_norm_backward(dy, torch.from_numpy(x).to(dev).view(2, 4, C), mean, rstd, gamma, 1.0, dx, *out, ws)
    bad = ~torch.isfinite(dx.view(8, C)).all(1)
    assert bad.tolist() == [False, False, True, True, False, False, False, False]
    assert torch.equal(out[3], torch.full((C,), 8.0, device=dev)) and torch.equal(out[1], torch.full((C,), 32.0, device=dev))


BACKWARD = [(1, 1, 1), (1, 1, 7), (2, 3, 8), (1, 300, 33), (3, 1, 100), (5, 49, 64), (2100, 1, 64), (2050, 3, 40), (2060, 2, 520), (1100, 2, 1030), (520, 2, 4096), (300, 1, 8192),
            (16, 5, 1000), (17, 64, 2048), (1, 1025, 512), (4, 9, 4096), (2, 3, 8192), (2, 5, 8200), (1, 2, 20001),
            (3, 70, 16), (2, 130, 100), (40, 9, 250), (9, 700, 24), (17000, 1, 30), (4200, 1, 200), (600, 8, 128), (70, 33, 300)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("B,P,C", BACKWARD)
def test_backward(dev, B, P, C, kept, dtype):
    import torch
    from paper_1802_06058_amd import vgc
    rng = np.random.default_rng(B + 17 * P + C)
    x = torch.from_numpy((rng.standard_normal((B * P, C)) * 2 + 1).astype(np.float32)).to(_type(dtype))
    dy = torch.from_numpy((rng.standard_normal((B, P, C)) * 1e-2).astype(np.float32)).to(_type(dtype))
    gamma = (1 + 0.2 * rng.standard_normal(C)).astype(np.float32)
    _, m, r, xhat = O.layer_norm(_np(x), gamma, gamma, 1e-5)
    mean, rstd = torch.from_numpy(m.astype(np.float32)), torch.from_numpy(r.astype(np.float32))
    m, r = _np(mean), _np(rstd)                      # (the backward pass's inputs)
    act8 = None
    if kept:
        q, e = O.act8_encode(xhat.astype(np.float32))
        xhat = O.act8_decode(q, e)
        act8 = (torch.from_numpy(q).to(dev), torch.from_numpy(e).to(dev))
    else:
        xhat = (_np(x) - m[:, None]) * r[:, None]
    c = 1.0 / B
    dxw, G, Hb, want = O.layer_norm_backward(_np(dy), xhat.reshape(B, P, C), r.reshape(B, P), gamma, c)
    dx = torch.full((B * P * C + 32,), 7.0, dtype=x.dtype, device=dev)
    s_gamma, s_beta, g_gamma, g_beta = (torch.full((C + 8,), 7.0, device=dev) for _ in range(4))
    nb = vgc.layer_norm_backward_workspace_bytes(B, P, C)
    ws = torch.full((nb + 64,), 0xFF, dtype=torch.uint8, device=dev)
    call = lambda *g: vgc.layer_norm_backward(dy.to(dev), None if kept else x.to(dev).view(B, P, C), None if kept else mean.to(dev), rstd.to(dev),
                                              torch.from_numpy(gamma).to(dev), c, dx[:B * P * C].view(B, P, C), s_gamma, s_beta, *g, workspace=ws[:nb], act8=act8)
    call(g_gamma, g_beta)
    h, dy64 = xhat.reshape(B, P, C), _np(dy)
    # one product's error: the normalised value has two roundings (and the mean's subtraction), then the product
    eh = 0 if kept else 3 * U * np.abs(h) + U * (np.abs(_np(x)) * r[:, None]).reshape(B, P, C)
    d = np.abs(dy64 * gamma)
    mb = (d * np.abs(h)).mean(-1, keepdims=True)
    depth = (_depth(C) + 8) * U
    tol = r.reshape(B, P, 1) * (depth * (d.mean(-1, keepdims=True) + np.abs(h) * mb) + 6 * U * (d + np.abs(h) * mb) + eh * mb +
                                np.abs(h) * (d * (eh + 0 * d)).mean(-1, keepdims=True)) + (2.0 ** -8 * np.abs(dxw) if dtype == "bf16" else 0)
    assert (np.abs(_np(dx[:B * P * C]).reshape(B, P, C) - dxw) <= tol).all()
    for name, S, one, err in (("gamma", G, np.abs(dy64 * h), np.abs(dy64) * eh), ("beta", Hb, np.abs(dy64), 0 * dy64)):
        dS = (P + 8) * U * one.sum(1) + err.sum(1)   # of a sample's sum, roundings in any order
        gs, ss = (g_gamma, s_gamma) if name == "gamma" else (g_beta, s_beta)
        tol_g = c * (dS.sum(0) + (B + 32) * U * np.abs(S).sum(0))
        tol_s = c * c * ((2 * np.abs(S) * dS + dS * dS).sum(0) + (B + 32) * U * (S * S).sum(0))
        assert (np.abs(_np(gs[:C]) - want["g_" + name]) <= tol_g).all(), name
        assert (np.abs(_np(ss[:C]) - want["s_" + name]) <= tol_s).all(), name
        assert (gs[C:] == 7).all() and (ss[C:] == 7).all()
    assert (dx[B * P * C:] == 7).all() and (ws[nb:] == 0xFF).all()
    first = [t.clone() for t in (dx, s_gamma, s_beta)]
    call()                                           # without g, and again: the same bits
    assert all(torch.equal(a, b) for a, b in zip(first, (dx, s_gamma, s_beta)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_that_begin_anywhere(dev, dtype):
    import torch
    from paper_1802_06058_amd import vgc
    B, P, C = 2, 5, 131
    g = torch.Generator().manual_seed(1)
    def off(*shape):                                 # a tensor one element into its storage
        n = int(np.prod(shape))
        t = torch.empty(n + 1, dtype=_type(dtype), device=dev)[1:].view(*shape)
        return t.copy_(torch.randn(*shape, generator=g))
    x, dy, gamma, beta = off(B, P, C), off(B, P, C), torch.ones(C + 1, device=dev)[1:], torch.zeros(C + 1, device=dev)[1:]
    res = []
    for same in (lambda t: t, lambda t: t.clone()):
        y, dx = off(B, P, C), off(B, P, C)
        mean, rstd = torch.empty(B * P, device=dev), torch.empty(B * P, device=dev)
        out = [torch.empty(C, device=dev) for _ in range(4)]
        ws = torch.empty(vgc.layer_norm_backward_workspace_bytes(B, P, C), dtype=torch.uint8, device=dev)
        vgc.layer_norm(same(x), same(gamma), same(beta), 1e-5, y, mean, rstd)
        vgc.layer_norm_backward(same(dy), same(x), mean, rstd, same(gamma), 0.5, dx, *out, ws)
        res.append([y, mean, rstd, dx, *out])
    assert all(torch.equal(a, b) for a, b in zip(*res))


def test_graph_replays_are_the_eager_results(dev):
    import torch
    from paper_1802_06058_amd import vgc
    B, P, C = 6, 40, 384
    x, dy = torch.randn(B, P, C, device=dev), torch.randn(B, P, C, device=dev)
    gamma, beta = torch.rand(C, device=dev), torch.rand(C, device=dev)
    y, dx, mean, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(B * P, device=dev), torch.empty(B * P, device=dev)
    codes, exps = torch.empty(B, P, C, dtype=torch.int8, device=dev), torch.empty(B, P, C // 32, dtype=torch.uint8, device=dev)
    out = [torch.empty(C, device=dev) for _ in range(4)]
    ws = torch.empty(vgc.layer_norm_backward_workspace_bytes(B, P, C), dtype=torch.uint8, device=dev)
    def step():
        vgc.layer_norm(x, gamma, beta, 1e-5, y, mean, rstd, (codes, exps))
        vgc.layer_norm_backward(dy, None, None, rstd, gamma, 0.5, dx, *out, ws, act8=(codes, exps))
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        x.copy_(torch.randn(B, P, C, device=dev) + k)
        step()
        want = [t.clone() for t in (y, dx, *out)]
        for t in (y, dx, *out):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (y, dx, *out)))


def test_refusals(dev):
    import torch
    from paper_1802_06058_amd import vgc
    B, P, C = 2, 3, 40
    f = lambda *s: torch.zeros(*s, device=dev)
    x, gamma, y, mean, rstd = f(B, P, C), f(C), f(B, P, C), f(B * P), f(B * P)
    codes, exps = torch.zeros(B, P, C, dtype=torch.int8, device=dev), torch.zeros(B, P, 2, dtype=torch.uint8, device=dev)
    good = dict(x=x, gamma=gamma, beta=gamma, eps=1e-5, y=y, mean=mean, rstd=rstd, act8=None)
    for change in [dict(x=x.half()), dict(x=x.transpose(0, 1)), dict(gamma=gamma[:-1]), dict(gamma=gamma.to(torch.bfloat16)), dict(y=y.to(torch.bfloat16)), dict(mean=mean[:-1]),
                   dict(eps=-1.0), dict(eps=float("nan")), dict(act8=(codes, exps[:1])), dict(x=x.cpu()), dict(y=y.cpu()), dict(x=f(0, C)), dict(act8=(codes, None))]:
        with pytest.raises(vgc.VgcError):
            vgc.layer_norm(**{**good, **change})
    vgc.layer_norm(**good)
    ws = torch.empty(vgc.layer_norm_backward_workspace_bytes(B, P, C), dtype=torch.uint8, device=dev)
    good = dict(dy=x, x=x, mean=mean, rstd=rstd, gamma=gamma, c=0.5, dx=f(B, P, C), s_gamma=f(C), s_beta=f(C), workspace=ws, act8=None)
    for change in [dict(dy=x.view(B * P, C)), dict(x=None), dict(mean=None), dict(act8=(codes, exps)), dict(x=None, mean=None), dict(workspace=None), dict(workspace=ws[:-1]),
                   dict(c=float("inf")), dict(s_gamma=f(C - 1)), dict(dx=y.to(torch.bfloat16)), dict(x=None, mean=None, act8=(codes.cpu(), exps)), dict(rstd=rstd.double())]:
        with pytest.raises(vgc.VgcError):
            vgc.layer_norm_backward(**{**good, **change})
    vgc.layer_norm_backward(**good)
