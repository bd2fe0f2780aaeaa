"""The softmax loss of a linear layer and its gradients, against the oracle in 64 bits, entry by entry.

Tolerances.  A logit is a float32 sum of H products (exact for bfloat16 pairs; within 2^-22 for float32 ones): H roundings or truncations
of 2^-23 of the magnitudes summed bound it in any order.  An exponential's relative error is that of its argument (the logit's, lse's and
the rounding of their difference) and four roundings.  D is rounded to 2^-8 (bfloat16, for dX) or to 2^-17 (for g and s); float32: 2^-22.
Sums over V, over positions and over samples have as many roundings as terms, of 2^-23 of the magnitudes summed."""
import numpy as np
import pytest

from oracle import operators as O

pytestmark = pytest.mark.gpu
E = 2.0 ** -23


@pytest.fixture(scope="module")
def dev():
    import torch
    from paper_1802_06058_amd import vgc
    assert torch.cuda.is_available()
    vgc.load()
    return torch.device("cuda:0")


def _np(t):
    return t.double().cpu().numpy()


def _inputs(B, P, H, V, dtype, masked=0.2, seed=0):
    import torch
    rng = np.random.default_rng([B, P, H, V, seed])
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    W = torch.from_numpy((rng.standard_normal((V, H)) / np.sqrt(H)).astype(np.float32)).to(t)
    target = rng.integers(0, V, (B, P))
    X = rng.standard_normal((B, P, H)) + 12 * rng.random((B, P, 1)) * _np(W)[target]
    target[rng.random((B, P)) < masked] = -1
    target[0, 0] = V - 1
    return torch.from_numpy(X.astype(np.float32)).to(t), W, torch.from_numpy(target)


def _sides(dev, X, W, target, weight, want_dx=True, want_s=True, want_g=True, c=None):
    """Both calls; every output lies between guards that have to stay."""
    import torch
    from paper_1802_06058_amd import vgc
    B, P, H = X.shape
    V, N = W.shape[0], B * P
    code = vgc.BF16 if X.dtype == torch.bfloat16 else vgc.F32
    guarded = lambda n, t=torch.float32: torch.full((n + 64,), 7.0, dtype=t, device=dev)
    loss, lse, dX, s, g = guarded(N), guarded(N), guarded(N * H, X.dtype), guarded(V * H), guarded(V * H)
    Xd, Wd, td = X.to(dev), W.to(dev), target.to(dev)
    wd = None if weight is None else weight.to(dev)
    n1, n2 = vgc.softmax_loss_workspace_bytes(code, N, H, V), vgc.softmax_loss_backward_workspace_bytes(code, B, P, H, V)
    ws = torch.full((max(n1, n2) + 64,), 0xFF, dtype=torch.uint8, device=dev)
    vgc.softmax_loss(Xd, Wd, td, loss, lse, ws[:n1])
    assert (ws[n1:] == 0xFF).all()
    ws.fill_(0xFF)
    vgc.softmax_loss_backward(Xd, Wd, td, lse, wd, 1.0 / B if c is None else c, dX[:N * H].view(B, P, H) if want_dx else None, s if want_s else None,
                              g if want_g else None, ws[:n2])
    for t, n in ((loss, N), (lse, N), (dX, N * H), (s, V * H), (g, V * H)):
        assert (t[n:] == 7).all()
    assert (ws[n2:] == 0xFF).all()
    return loss[:N], lse[:N], dX[:N * H].view(B, P, H), s[:V * H].view(V, H), g[:V * H].view(V, H)


def _check(X, W, target, weight, got, sums=True):
    import torch
    B, P, H = X.shape
    V, bf16 = W.shape[0], X.dtype == torch.bfloat16
    loss, lse, dX, s, g = [_np(t) for t in got]
    x, w, t = _np(X).reshape(-1, H), _np(W), target.numpy().reshape(-1)
    want, wlse, z = O.softmax_loss(x, w, t)
    ez = (H + 8) * E * (np.abs(x) @ np.abs(w).T)
    el = ez.max(1) + 16 * E * (1 + np.abs(wlse)) + (V // 16 + 64) * E      # (the sum of positive terms: their count a lane and block)
    assert (np.abs(lse - wlse) <= el).all()
    et = np.take_along_axis(ez, np.clip(t, 0, V - 1)[:, None], 1)[:, 0]
    assert (np.abs(loss - want) <= np.where(t < 0, 0, el + et + 4 * E * (np.abs(wlse) + np.abs(wlse - want)))).all()
    c = 1.0 / B
    D, dXw, G, sw, gw = O.softmax_loss_backward(_np(X), w, t, lse, None if weight is None else weight.numpy(), c)
    wt = np.where(t < 0, 0, 1.0 if weight is None else weight.numpy().reshape(-1))[:, None]
    p = np.exp(z - lse[:, None])
    eD = np.abs(wt) * (p * (ez + 4 * E * (1 + np.abs(z) + np.abs(lse)[:, None])) + 2 * E)
    edx = (eD + (2.0 ** -8 if bf16 else 4 * E) * np.abs(D)) @ np.abs(w) + (V + 8) * E * (np.abs(D) @ np.abs(w))
    assert (np.abs(dX.reshape(-1, H) - dXw.reshape(-1, H)) <= edx + (2.0 ** -8 if bf16 else E) * np.abs(dXw.reshape(-1, H))).all()
    if not sums:
        return
    ax = np.abs(np.where((t >= 0)[:, None], x, 0)).reshape(B, P, H)
    e = (eD + (2.0 ** -17 if bf16 else 4 * E) * np.abs(D) + (P + 8) * E * np.abs(D)).reshape(B, P, V)
    eG = np.stack([e[b].T @ ax[b] for b in range(B)])
    assert (np.abs(g - gw) <= c * (eG.sum(0) + (B + 8) * E * np.abs(G).sum(0))).all()
    assert (np.abs(s - sw) <= c * c * ((2 * np.abs(G) * eG + eG ** 2).sum(0) + (B + 8) * E * (G * G).sum(0))).all()


SHAPES = [  # B, P, H, V: one of each; then lengths around a step's ends, odd rows, few and many classes
    (1, 1, 1, 1), (1, 1, 8, 2), (3, 1, 7, 5), (2, 2, 16, 3), (128, 1, 1000, 10), (64, 1, 96, 1000), (1, 7, 33, 40), (5, 8, 64, 31), (3, 9, 40, 33), (2, 24, 72, 65),
    (2, 25, 64, 300), (3, 32, 64, 257), (2, 33, 130, 129), (1, 65, 64, 1000), (4, 100, 128, 517), (70, 3, 24, 90), (2, 31, 1001, 77), (1, 130, 200, 64), (3, 64, 512, 640),
    (130, 1, 512, 300), (40, 1, 640, 7001), (17, 1, 1001, 5003)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,P,H,V", SHAPES)
def test_loss_and_gradients(dev, B, P, H, V, dtype):
    import torch
    X, W, target = _inputs(B, P, H, V, dtype)
    weight = torch.from_numpy(np.random.default_rng(1).random((B, P)).astype(np.float32)) if B % 2 else None
    _check(X, W, target, weight, _sides(dev, X, W, target, weight))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,P,H,V", [(64, 1, 72, 20003), (1, 5, 40, 17000), (3, 20, 16, 17001), (100, 1, 24, 128 * 192 + 5), (4, 75, 40, 256 * 100 + 3), (1, 300, 17, 25700)])
def test_tiles_of_large_vocabularies(dev, B, P, H, V, dtype):
    """Enough tiles for the kernels with 128 and 256 classes a workgroup."""
    X, W, target = _inputs(B, P, H, V, dtype)
    _check(X, W, target, None, _sides(dev, X, W, target, None))


@pytest.mark.parametrize("dtype,B,P,H,V", [("bf16", 4, 1024, 64, 20001), ("bf16", 4, 1024, 64, 150001), ("bf16", 1000, 1, 48, 400001), ("f32", 2, 300, 48, 600011)])
def test_several_pieces_of_the_vocabulary(dev, B, P, H, V, dtype):
    X, W, target = _inputs(B, P, H, V, dtype)
    loss, lse, dX, s, g = got = _sides(dev, X, W, target, None)
    if B * P * V < 10 ** 8:
        _check(X, W, target, None, got)
        return
    # a slice of the classes on each side of the pieces' borders, and a slice of the rows, against the same without the rest
    import torch
    x, t = _np(X).reshape(B * P, H), target.numpy().reshape(-1)
    l = _np(lse)
    rows = np.arange(0, B * P, 97)
    z = x[rows] @ _np(W).T
    wl = np.log(np.exp(z - z.max(1, keepdims=True)).sum(1)) + z.max(1)
    assert np.abs(l[rows] - wl).max() <= (H + 8) * E * (np.abs(x[rows]) @ np.abs(_np(W)).T).max() + (V // 16 + 80) * E
    D = np.exp(z - l[rows, None])
    D[t[rows] < 0] = 0
    ok = np.flatnonzero(t[rows] >= 0)
    D[ok, t[rows][ok]] -= 1
    dXw = D @ _np(W)
    tol = 2.0 ** -8 * (np.abs(D) @ np.abs(_np(W)) + np.abs(dXw)) + (V + H + 32) * E * (np.abs(D) @ np.abs(_np(W)))
    assert (np.abs(_np(dX).reshape(B * P, H)[rows] - dXw) <= tol).all()
    for v0 in range(0, V, 4096):
        v = slice(v0, min(V, v0 + 32))
        D = np.exp(x @ _np(W)[v].T - l[:, None])
        D[t < 0] = 0
        ok = np.flatnonzero((t >= v.start) & (t < v.stop))
        D[ok, t[ok] - v.start] -= 1
        G = np.einsum("bpv,bph->bvh", D.reshape(B, P, -1), x.reshape(B, P, H), optimize=True) / B
        A = np.einsum("bpv,bph->bvh", np.abs(D).reshape(B, P, -1), np.abs(x).reshape(B, P, H), optimize=True) / B
        eG = A * (2.0 ** -17 + (P + H + 64) * E)
        assert (np.abs(_np(g)[v] - G.sum(0)) <= eG.sum(0) + (B + 8) * E * A.sum(0)).all()
        assert (np.abs(_np(s)[v] - (G * G).sum(0)) <= (2 * np.abs(G) * eG + eG ** 2).sum(0) + (B + 8) * E * (G * G).sum(0)).all()


def test_large_tiles_of_the_input_gradient(dev):
    X, W, target = _inputs(4, 1024, 4096, 40, "bf16")
    _check(X, W, target, None, _sides(dev, X, W, target, None, want_s=False, want_g=False), sums=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("P", [1, 5, 40])
def test_rows_that_are_not_asked_for(dev, P, dtype):
    """Their loss is 0, nothing of theirs reaches a gradient, whatever they hold; all of them: all gradients are 0."""
    import torch
    B, H, V = 3, 72, 50
    X, W, target = _inputs(B, P, H, V, dtype, masked=0.0)
    target[1] = -100
    clean = _sides(dev, X, W, target, None)
    X2 = X.clone()
    X2[1, :, ::3], X2[1, :, 1::3] = float("nan"), float("inf")
    dirty = _sides(dev, X2, W, target, None)
    assert (clean[0].view(B, P)[1] == 0).all() and (dirty[0].view(B, P)[1] == 0).all()
    assert (dirty[2][1] == 0).all()
    for a, b in zip(clean[2:], dirty[2:]):
        assert torch.equal(a, b)
    target[:] = -1
    loss, _, dX, s, g = _sides(dev, X2, W, target, None)
    assert not loss.any() and not dX.any() and not s.any() and not g.any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_targets_that_are_no_class(dev, dtype):
    import torch
    X, W, target = _inputs(2, 6, 40, 30, dtype, masked=0.0)
    target[1, 2], target[1, 3] = 30, 2 ** 40
    loss, lse, dX, s, g = _sides(dev, X, W, target, None)
    bad = torch.zeros(2, 6, dtype=torch.bool)
    bad[1, 2:4] = True
    assert torch.equal(torch.isnan(loss.view(2, 6)).cpu(), bad) and torch.isfinite(lse).all()
    assert torch.equal(torch.isnan(dX).all(-1).cpu(), bad) and torch.isfinite(dX.cpu()[~bad]).all()
    assert torch.isnan(s).all() and torch.isnan(g).all()


def test_large_logits_and_equal_ones(dev):
    import torch
    H, V = 8, 70
    X, W = torch.zeros(1, 4, H), torch.zeros(V, H)
    X[0, 0, 0], X[0, 1, 0] = 1e4, -1e4
    W[3, 0] = 1.0                                    # logits 1e4 and -1e4 beside zeros; then all zeros
    target = torch.tensor([[3, 3, 0, 69]])
    loss, lse, dX, s, g = _sides(dev, X, W, target, None)
    want = torch.tensor([0.0, 1e4 + np.log(69), np.log(70), np.log(70)], dtype=torch.float64)
    assert (loss.double().cpu() - want).abs().max() < 4 * E * 1e4
    assert torch.isfinite(dX).all() and torch.isfinite(s).all() and (dX[0, 0] == 0).all()


def test_parts_that_are_not_asked_for(dev):
    import torch
    X, W, target = _inputs(2, 40, 64, 200, "bf16")
    whole = _sides(dev, X, W, target, None)
    for dx, s, g in ((True, False, False), (False, True, False), (False, True, True)):
        part = _sides(dev, X, W, target, None, dx, s, g)
        for want, a, b in zip((dx, s, g), part[2:], whole[2:]):
            assert torch.equal(a, b) if want else (a == 7).all()
    for X, W, target in (_inputs(9, 1, 64, 20, "bf16"), _inputs(9, 1, 33, 20, "f32")):
        whole = _sides(dev, X, W, target, None)
        assert torch.equal(_sides(dev, X, W, target, None, False, True, False)[3], whole[3])


def test_graph_replays_are_the_eager_results(dev):
    import torch
    from paper_1802_06058_amd import vgc
    B, P, H, V = 2, 33, 72, 90
    X, W, target = (t.to(dev) for t in _inputs(B, P, H, V, "bf16"))
    loss, lse = torch.empty(B * P, device=dev), torch.empty(B * P, device=dev)
    dX, s, g = torch.empty_like(X), torch.empty(V, H, device=dev), torch.empty(V, H, device=dev)
    ws = torch.empty(max(vgc.softmax_loss_workspace_bytes(vgc.BF16, B * P, H, V), vgc.softmax_loss_backward_workspace_bytes(vgc.BF16, B, P, H, V)),
                     dtype=torch.uint8, device=dev)
    def step():
        vgc.softmax_loss(X, W, target, loss, lse, ws)
        vgc.softmax_loss_backward(X, W, target, lse, None, 0.5, dX, s, g, ws)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        X.copy_(torch.randn(B, P, H, device=dev) * (k + 1))
        step()
        want = [t.clone() for t in (loss, lse, dX, s, g)]
        for t in (loss, lse, dX, s, g):
            t.zero_()
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (loss, lse, dX, s, g)))


def test_refusals(dev):
    import torch
    from paper_1802_06058_amd import vgc
    B, P, H, V = 2, 3, 40, 30
    f = lambda *s: torch.zeros(*s, device=dev)
    X, W, t, v = f(B, P, H), f(V, H), torch.zeros(B, P, dtype=torch.int64, device=dev), f(B, P)
    ws = torch.empty(vgc.softmax_loss_workspace_bytes(vgc.F32, B * P, H, V), dtype=torch.uint8, device=dev)
    good = dict(X=X, W=W, target=t, loss=v, lse=v.clone(), workspace=ws)
    for change in [dict(X=X.half()), dict(X=X.transpose(0, 1)), dict(W=W.t()), dict(W=W.to(torch.bfloat16)), dict(W=f(V, H + 1)), dict(W=f(0, H)), dict(target=t.int()), dict(target=t[:1]),
                   dict(loss=v[:1]), dict(lse=v.double()), dict(workspace=None), dict(workspace=ws[:-1]), dict(X=X.cpu()), dict(target=t.cpu()), dict(X=f(0, H)),
                   dict(X=f(B * P * H + 1)[1:].view(B, P, H))]:
        with pytest.raises(vgc.VgcError):
            vgc.softmax_loss(**{**good, **change})
    vgc.softmax_loss(**good)
    ws = torch.empty(vgc.softmax_loss_backward_workspace_bytes(vgc.F32, B, P, H, V), dtype=torch.uint8, device=dev)
    good = dict(X=X, W=W, target=t, lse=v, weight=None, c=0.5, dX=f(B, P, H), s_out=f(V, H), g_out=f(V, H), workspace=ws)
    for change in [dict(X=X.view(B * P, H)), dict(weight=v[:1]), dict(weight=v.double()), dict(c=float("nan")), dict(dX=X.to(torch.bfloat16)), dict(s_out=f(V - 1, H)),
                   dict(s_out=None), dict(dX=None, s_out=None, g_out=None), dict(workspace=None), dict(workspace=ws[:-1]), dict(g_out=f(V * H + 1)[1:])]:
        with pytest.raises(vgc.VgcError):
            vgc.softmax_loss_backward(**{**good, **change})
    vgc.softmax_loss_backward(**good)
    assert vgc.softmax_loss_backward_workspace_bytes(vgc.F32, 1 << 11, 1 << 11, H, V) == 0


@pytest.mark.parametrize("P", [38, 57])
def test_weights_that_all_positions_share(dev, P):
    """Rows that miss their classes, each weighted 1 / P, which bfloat16 does not hold: what that rounds to must not be what every position brings.
    Relative to their samples' weight the targets' entries are p - 1 with p about 1 / V, kept to 2^-9 of p in two pieces: 1e-7; a class has a few
    positions, whose products, sums, squares and factors round a dozen times at 2^-24: 1e-6 bounds s.  dX is rounded once, to 2^-9 of itself
    at most, besides the sum of the other entries, each rounded by itself."""
    import torch
    B, H, V = 2, 64, 20011
    X, W, target = _inputs(B, P, H, V, "bf16", masked=0)
    X = torch.from_numpy(np.random.default_rng(3).standard_normal((B, P, H)).astype(np.float32)).to(torch.bfloat16)
    weight = torch.full((B, P), 1.0 / P)
    got = _sides(dev, X, W, target, weight)
    _check(X, W, target, weight, got)
    _, dXw, _, sw, _ = O.softmax_loss_backward(_np(X), _np(W), target.numpy().reshape(-1), _np(got[1]), weight.numpy(), 1.0 / B)
    off = lambda a, b: np.linalg.norm(a - b) / np.linalg.norm(b)
    assert off(_np(got[3]), sw) <= 1e-6 and off(_np(got[2]).reshape(dXw.shape), dXw) <= 2.05e-3


@pytest.mark.parametrize("N,V", [(600, 4000), (3, 7000)])
def test_logits_of_long_float_rows_do_not_shrink(dev, N, V):
    """One class far above the others, so that lse is its logit, 14, a sum of H terms that all point one way.  Float sums that are rounded, in
    whatever order, are off by sqrt(H) 2^-24 of it by chance; cut off instead they would all be too small."""
    import torch
    from paper_1802_06058_amd import vgc
    H, gen = 3000, torch.Generator().manual_seed(1)
    W = torch.randn(V, H, generator=gen) / H ** 0.5
    target = torch.randint(0, V, (N,), generator=gen)
    X = (0.02 * torch.randn(N, H, generator=gen) + 14 * W[target] / (W[target] ** 2).sum(1, keepdim=True)).float()
    want = torch.logsumexp(X.double() @ W.double().t(), 1)
    loss, lse = torch.empty(N, device=dev), torch.empty(N, device=dev)
    ws = torch.empty(vgc.softmax_loss_workspace_bytes(vgc.F32, N, H, V), dtype=torch.uint8, device=dev)
    vgc.softmax_loss(X.to(dev), W.to(dev), target.to(dev), loss, lse, ws)
    assert float((lse.cpu().double() - want).pow(2).mean().sqrt()) <= H ** 0.5 * 2.0 ** -24 * 14


def test_weights_of_every_kind_in_a_sample(dev):
    """Zero throughout, negative, far apart, and infinite or NaN where the row is not asked for."""
    import torch
    B, P, H, V = 5, 20, 40, 300
    for dtype in ("bf16", "f32"):
        X, W, target = _inputs(B, P, H, V, dtype)
        weight = torch.from_numpy(np.random.default_rng(2).standard_normal((B, P)).astype(np.float32))
        weight[1] = 0
        weight[2] *= 1e-20
        weight[3, ::2] *= 1e-10
        clean = weight.clone()
        clean[target < 0] = 1
        weight[target < 0] = torch.where(torch.arange(int((target < 0).sum())) % 2 == 0, float("inf"), float("nan"))
        _check(X, W, target, clean, _sides(dev, X, W, target, weight))
