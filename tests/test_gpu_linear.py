"""The linear layer with its epilogue and its backward pass, against the oracle in 64 bits.

Tolerances.  z: K products and sums, each within a unit 2^-23 of the magnitudes summed (float32: a product of planes is within 2^-22.4 of itself), and
a few roundings more where k is shared out.  An activation's slope is at most 1.13.  dz: act_error of its slope and three roundings.  dX: as z from dz as
the call stored it, or, in the float32 form and for products that read more digits of dz, from the oracle's with what 16 bits leave out, 2^-16.  A sum over a sample's positions has as many
roundings as positions, those over parts and samples as many again."""
import numpy as np
import pytest

from oracle import blocks as O
import block_checks as T

pytestmark = pytest.mark.gpu
E = 2 * T.U


@pytest.fixture(scope="module")
def dev():
    return T.device()


def _case(N, K, C, dtype, dev, seed=0):
    gen = np.random.default_rng(N * 7 + K * 3 + C + seed)
    X, W = T.to(gen.standard_normal((N, K)), dtype, dev), T.to(gen.standard_normal((K, C)) / np.sqrt(K), dtype, dev)
    return gen, X, W, T.to(0.3 * gen.standard_normal(C), "f32", dev)


def _forward(dev, N, K, C, act, dtype, keep=True, residual=True, p=0.25, bias=True):
    import torch
    from paper_1802_06058_amd import vgc
    gen, X, W, b = _case(N, K, C, dtype, dev)
    r = T.to(gen.standard_normal((N, C)), dtype, dev) if residual else None
    state = T.rng_state(dev)
    y, after_y = T.guarded(N * C, X.dtype, dev)
    z, after_z = T.guarded(N * C, X.dtype, dev) if keep else (None, torch.full((1,), 7.0))
    code = vgc.F32 if dtype == "f32" else vgc.BF16
    ws = T.workspace(vgc.linear_workspace_bytes(code, N, K, C), dev)
    vgc.linear(X, W, y.view(N, C), b if bias else None, T.ACTS[act], z.view(N, C) if keep else None, r, p, state, ws)
    assert T.untouched(after_y, after_z)
    X64, W64 = X.double(), W.double()
    size = T.back(X64.abs() @ W64.abs()) + (np.abs(T.back(b)) if bias else 0)
    z64 = T.back(X64 @ W64) + (T.back(b) if bias else 0)
    err = (K + 16) * E * size
    if keep:
        assert (np.abs(T.back(z).reshape(N, C) - z64) <= err + T.half_unit(dtype) * np.abs(z64) + (err * T.half_unit(dtype))).all()
    f = O.keep_factor(N, C, p, *state.tolist())
    a = O.act(z64, T.ACTS[act])
    want = a * f
    tol = f * (1.13 * err + T.act_error(z64, a, act == "gelu" and dtype == "bf16")) + 3 * T.U * np.abs(want)
    if residual:
        want = want + T.back(r)
        tol = tol + T.U * np.abs(want)
    tol = tol + T.half_unit(dtype) * (np.abs(want) + tol)
    bad = np.abs(T.back(y).reshape(N, C) - want) > tol
    assert not bad.any(), np.argwhere(bad)[:5]
    return X, W, b, r, state, y, z, ws


SIZES = [(1, 1, 1), (1, 3, 2), (2, 8, 8), (1, 40, 1000), (1, 1000, 7), (1, 2048, 2048), (3, 1001, 33), (16, 512, 512), (17, 257, 130), (33, 64, 264), (64, 1000, 1000), (65, 784, 129),
         (128, 784, 1000), (100, 5, 300), (129, 96, 128), (200, 4096, 64), (257, 72, 520), (300, 2048, 8), (1030, 256, 256), (700, 513, 261), (5, 8192, 24), (1, 16, 8192), (48, 4100, 96),
         (1, 4096, 4096), (3, 6001, 515), (20, 5001, 1030), (2, 4099, 2050), (130, 4100, 520), (927, 64, 1032), (600, 24, 1416), (257, 2049, 264), (40, 7, 9)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,K,C", SIZES)
def test_forward(dev, N, K, C, dtype):
    act = list(T.ACTS)[(N + K + C) % 4]
    _forward(dev, N, K, C, act, dtype, keep=(N + C) % 3 != 0, residual=(K + C) % 2 == 0, p=[0.25, 0.0, 1.0, 0.5][(N + 2 * K) % 4], bias=(N + K) % 5 != 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", list(T.ACTS))
@pytest.mark.parametrize("N", [1, 40, 300])
def test_forward_activations(dev, N, act, dtype):
    _forward(dev, N, 160, 272, act, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_tiles(dev, dtype):
    """Tiles in all places of several bands, whole and cut."""
    _forward(dev, 2500, 64, 4104, "gelu", dtype, p=0.1)
    _forward(dev, 4096, 128, 4096, "none", dtype, keep=False, p=0.0)


def test_masks_are_those_of_dropout(dev):
    import torch
    from paper_1802_06058_amd import vgc
    for N, K, C in ((5, 24, 70), (300, 64, 513), (1, 9, 1000)):
        _, X, W, b = _case(N, K, C, "f32", dev)
        state = T.rng_state(dev)
        ws = T.workspace(vgc.linear_workspace_bytes(vgc.F32, N, K, C), dev)
        plain, dropped, want = (torch.empty(N, C, device=dev) for _ in range(3))
        vgc.linear(X, W, plain, b, workspace=ws)
        vgc.linear(X, W, dropped, b, p=0.3, rng=state, workspace=ws)
        vgc.dropout(plain, 0.3, state, want)
        assert torch.equal(dropped, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_onto_the_residual_and_twice_the_same(dev, dtype):
    import torch
    from paper_1802_06058_amd import vgc
    for N, K, C in ((3, 300, 65), (130, 520, 264), (600, 1024, 128)):
        X, W, b, r, state, y, z, ws = _forward(dev, N, K, C, "silu", dtype)
        onto = r.clone()
        vgc.linear(X, W, onto, b, T.ACTS["silu"], None, onto, 0.25, state, ws)
        assert torch.equal(onto.view(-1), y)


def _backward(dev, B, P, K, C, act, dtype, add=True, p=0.25, dx=True, sums=True):
    import torch
    from paper_1802_06058_amd import vgc
    N = B * P
    gen, _, W, _ = _case(N, K, C, dtype, dev, 1)
    dy = T.to(gen.standard_normal((B, P, C)), dtype, dev)
    z = T.to(1.5 * gen.standard_normal((B, P, C)), dtype, dev) if act != "none" else None
    extra = T.to(gen.standard_normal((B, P, K)), dtype, dev) if add and dx else None
    state = T.rng_state(dev)
    dz, after_dz = T.guarded(N * C, dy.dtype, dev)
    dX, after_dX = T.guarded(N * K, dy.dtype, dev)
    s, after_s = T.guarded(C, torch.float32, dev)
    g, after_g = T.guarded(C, torch.float32, dev)
    code = vgc.F32 if dtype == "f32" else vgc.BF16
    ws = T.workspace(vgc.linear_backward_workspace_bytes(code, B, P, K, C), dev)
    args = (dy, z, W, T.ACTS[act], 1.0 / B, dz.view(B, P, C), dX.view(B, P, K) if dx else None, s if sums else None, g if sums else None, extra, p, state, ws)
    vgc.linear_backward(*args)
    assert T.untouched(after_dz, after_dX, after_s, after_g) and (dx or T.untouched(dX)) and (sums or T.untouched(s, g))
    f = O.keep_factor(N, C, p, *state.tolist()).reshape(B, P, C)
    z64 = T.back(z) if act != "none" else None
    dz64, dX64, s64, g64, H = O.linear_backward(T.back(dy), z64, T.back(W), T.ACTS[act], 1.0 / B, f)
    d64 = T.back(dy) * f
    tol = 3 * T.U * np.abs(dz64)
    if act in ("gelu", "silu"):                                      # the slope's two terms
        tol = tol + np.abs(d64) * T.act_error(z64, 1.13)
    got = T.back(dz).reshape(B, P, C)
    assert (np.abs(got - dz64) <= tol * (1 + 2.0 ** -8) + T.half_unit(dtype) * np.abs(dz64)).all()
    if sums:
        eH = tol.sum(1) + (P + 64) * T.U * np.abs(dz64).sum(1)
        eg, es = (eH + (B + 64) * T.U * np.abs(H)).sum(0) / B, ((2 * np.abs(H) + eH) * eH + (B + 64) * E * H * H).sum(0) / B ** 2
        assert (np.abs(T.back(g) - g64) <= eg + 4 * T.U * np.abs(g64)).all()
        assert (np.abs(T.back(s) - s64) <= es + 8 * T.U * np.abs(s64)).all()
    if dx:
        one = dtype == "bf16" and N * K * C > 2 ** 31                 # (read as it is stored)
        ref = dz.double().view(N, C) if one else torch.from_numpy(dz64).to(dev).view(N, C)
        W64t = W.double().t().contiguous()
        want, size = T.back(ref @ W64t), T.back(ref.abs() @ W64t.abs())
        err = (C + 16) * E * size + (0 if one else 2.0 ** -16 * size * (dtype == "bf16") + T.back(torch.from_numpy(tol).to(dev).view(N, C) @ W64t.abs()))
        if extra is not None:
            want = want + T.back(extra).reshape(N, K)
            err = err + T.U * np.abs(want)
        bad = np.abs(T.back(dX).reshape(N, K) - want) > err * (1 + 2.0 ** -8) + T.half_unit(dtype) * np.abs(want)
        assert not bad.any(), np.argwhere(bad)[:5]
    return args


BACKWARD = [(1, 1, 1, 1), (1, 1, 2, 3), (2, 1, 8, 8), (1, 5, 33, 40), (3, 1, 1001, 130), (128, 1, 1000, 1000), (2, 33, 64, 264), (5, 13, 129, 784), (1, 300, 8, 2048), (300, 1, 2048, 9),
            (4, 64, 520, 72), (2, 500, 256, 256), (600, 2, 96, 520), (3, 1000, 24, 100), (40, 32, 64, 33), (1, 2000, 16, 16), (2100, 1, 40, 520),
            (1, 1, 2048, 4096), (3, 6, 655, 7513), (129, 1, 131, 4513), (16, 32, 512, 512), (1, 40, 1000, 5000), (7, 3, 83, 2301), (2, 9, 9, 7)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,P,K,C", BACKWARD)
def test_backward(dev, B, P, K, C, dtype):
    _backward(dev, B, P, K, C, list(T.ACTS)[(B + P + K + C) % 4], dtype, add=(B + K) % 2 == 0, p=[0.25, 0.0, 0.5][(P + C) % 3], dx=(B + C) % 7 != 0, sums=(K + C) % 6 != 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", list(T.ACTS))
@pytest.mark.parametrize("B,P", [(6, 1), (3, 50)])
def test_backward_activations(dev, B, P, act, dtype):
    _backward(dev, B, P, 72, 136, act, dtype)


def test_backward_of_large_products(dev):
    """dX reads dz as it is stored, by large and small tiles, and from a padded copy."""
    _backward(dev, 2, 1500, 1024, 1024, "gelu", "bf16")
    _backward(dev, 4, 1024, 3000, 520, "relu", "bf16", p=0.0)
    _backward(dev, 1, 2100, 1000, 1029, "silu", "bf16", add=False)
    _backward(dev, 2, 1100, 1000, 514, "silu", "f32")


def test_backward_in_place_and_twice_the_same(dev):
    import torch
    from paper_1802_06058_amd import vgc
    for dtype in ("f32", "bf16"):
        for size in ((6, 1, 50, 70), (2, 100, 264, 136)):
            dy, z, W, act, c, dz, dX, s, g, extra, p, state, ws = _backward(dev, *size, "gelu", dtype)
            first = [t.clone() for t in (dz, dX, s, g)]
            d2, x2 = dy.clone(), extra.clone()
            vgc.linear_backward(d2, z, W, act, c, d2, x2, s, g, x2, p, state, ws)
            assert all(torch.equal(a, b) for a, b in zip(first, (d2, x2, s, g)))
            z2 = z.clone()
            vgc.linear_backward(dy, z2, W, act, c, z2, dX, s, g, extra, p, state, ws)
            assert torch.equal(z2, first[0]) and torch.equal(dX, first[1])


def test_relu_from_the_output(dev):
    """Without dropout and residual the output has z's signs."""
    import torch
    from paper_1802_06058_amd import vgc
    B, P, K, C = 4, 30, 40, 88
    _, X, W, b = _case(B * P, K, C, "bf16", dev)
    ws = T.workspace(max(vgc.linear_workspace_bytes(vgc.BF16, B * P, K, C), vgc.linear_backward_workspace_bytes(vgc.BF16, B, P, K, C)), dev)
    y, z = (torch.empty(B, P, C, dtype=torch.bfloat16, device=dev) for _ in range(2))
    vgc.linear(X, W, y, b, vgc.ACT_RELU, z, workspace=ws)
    dy = torch.randn_like(y)
    out = [[torch.empty_like(y), torch.empty(B, P, K, dtype=torch.bfloat16, device=dev), torch.empty(C, device=dev), torch.empty(C, device=dev)] for _ in range(2)]
    for o, signs in zip(out, (y, z)):
        vgc.linear_backward(dy, signs, W, vgc.ACT_RELU, 1.0, *o, workspace=ws)
    assert all(torch.equal(a, b) for a, b in zip(*out))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_values_that_are_not_finite_stay_in_their_rows(dev, dtype):
    import torch
    from paper_1802_06058_amd import vgc
    for N, K, C in ((20, 100, 130), (300, 1000, 200)):
        _, X, W, b = _case(N, K, C, dtype, dev)
        X[3, K - 1], X[7, 0], X[N - 1, 5] = float("nan"), float("inf"), float("-inf")
        code = vgc.F32 if dtype == "f32" else vgc.BF16
        ws = T.workspace(max(vgc.linear_workspace_bytes(code, N, K, C), vgc.linear_backward_workspace_bytes(code, N, 1, K, C)), dev)
        y = torch.empty(N, C, dtype=X.dtype, device=dev)
        vgc.linear(X, W, y, b, vgc.ACT_SILU, workspace=ws)
        bad = ~torch.isfinite(y).all(1)
        assert bad.nonzero().flatten().tolist() == [3, 7, N - 1] and torch.isnan(y[3]).all()
        dy = torch.randn(N, 1, C, device=dev).to(X.dtype)
        dy[2, 0, C - 1] = float("inf")
        dz, dX = torch.empty_like(dy), torch.empty(N, 1, K, dtype=X.dtype, device=dev)
        s, g = torch.empty(C, device=dev), torch.empty(C, device=dev)
        vgc.linear_backward(dy, None, W, vgc.ACT_NONE, 1.0, dz, dX, s, g, workspace=ws)
        assert (~torch.isfinite(dX).all(2)).nonzero()[:, 0].tolist() == [2]
        assert (~torch.isfinite(s)).nonzero().flatten().tolist() == [C - 1] == (~torch.isfinite(g)).nonzero().flatten().tolist()


def test_gelu_where_it_is_small_and_large(dev):
    """z as given: one column a value, through a weight of ones."""
    import torch
    from paper_1802_06058_amd import vgc
    z = torch.linspace(-13, 13, 5001, device=dev).view(-1, 1).contiguous()
    one, y = torch.ones(1, 1, device=dev), torch.empty(5001, 1, device=dev)
    ws = T.workspace(vgc.linear_workspace_bytes(vgc.F32, 5001, 1, 1), dev)
    for act in ("gelu", "silu"):
        vgc.linear(z, one, y, None, T.ACTS[act], workspace=ws)
        z64 = T.back(z)
        want = O.act(z64, T.ACTS[act])
        assert (np.abs(T.back(y) - want) <= T.act_error(z64, want)).all()
        short = torch.empty(5001, 1, dtype=torch.bfloat16, device=dev)
        ws16 = T.workspace(vgc.linear_workspace_bytes(vgc.BF16, 5001, 1, 1), dev)
        vgc.linear(z.bfloat16(), one.bfloat16(), short, None, T.ACTS[act], workspace=ws16)
        z64 = T.back(z.bfloat16())
        want = O.act(z64, T.ACTS[act])
        tol = T.act_error(z64, want, act == "gelu")
        assert (np.abs(T.back(short) - want) <= tol + T.half_unit("bf16") * (np.abs(want) + tol)).all()


@pytest.mark.parametrize("N,K,C", [(845, 427, 1829), (701, 301, 3001), (2045, 509, 2043), (520, 1210, 1100), (260, 1030, 2050), (1100, 1030, 515), (1024, 1024, 1024)])
def test_float32_products_of_middle_size(dev, N, K, C):
    """By halves and quarters of the large tiles, k whole and in parts."""
    _forward(dev, N, K, C, "silu", "f32")


@pytest.mark.parametrize("B,P,K,C", [(6, 100, 2401, 601), (4, 511, 509, 2045), (3, 500, 1500, 1500), (7, 100, 1500, 300), (1030, 1, 700, 1100)])
def test_backward_of_float32_products_of_middle_size(dev, B, P, K, C):
    _backward(dev, B, P, K, C, "gelu", "f32")


@pytest.mark.parametrize("N,K,C", [(500, 2056, 2000), (1001, 1031, 1096), (390, 2049, 2051), (1024, 4096, 1024)])
def test_bfloat16_products_of_middle_size(dev, N, K, C):
    """By narrow tiles, k whole and in parts."""
    _forward(dev, N, K, C, "gelu", "bf16")


@pytest.mark.parametrize("B,P,K,C", [(2, 512, 2048, 2048), (7, 100, 1700, 2001)])
def test_backward_of_bfloat16_products_of_middle_size(dev, B, P, K, C):
    _backward(dev, B, P, K, C, "silu", "bf16")
