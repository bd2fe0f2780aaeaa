"""Pins of the oracle's layer norm, softmax loss and 8-bit activations: gradients against differences, the statistic against the
samples taken one by one, the 8-bit form against its own definition."""
import numpy as np
import pytest

from oracle import operators as O
from oracle import vgc_oracle as V

H = 1e-5


def _difference(f, x):
    """Central differences of a scalar function, entry by entry (error of order H^2)."""
    out = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        hi, lo = x.copy(), x.copy()
        hi[i] += H
        lo[i] -= H
        out[i] = (f(hi) - f(lo)) / (2 * H)
    return out


def test_layer_norm_gradients_are_those_of_differences():
    rng = np.random.default_rng(3)
    B, P, C = 3, 2, 5
    x, w = rng.standard_normal((B, P, C)), rng.standard_normal((B, P, C))
    gamma, beta = 1 + 0.3 * rng.standard_normal(C), rng.standard_normal(C)
    f = lambda x, gamma, beta: (O.layer_norm(x.reshape(-1, C), gamma, beta, 1e-3)[0].reshape(x.shape) * w[:x.shape[0]]).sum()
    _, _, rstd, xhat = O.layer_norm(x.reshape(-1, C), gamma, beta, 1e-3)
    dx, G, Hb, sums = O.layer_norm_backward(w, xhat.reshape(B, P, C), rstd.reshape(B, P), gamma, 0.25)
    assert np.allclose(dx, _difference(lambda t: f(t, gamma, beta), x), atol=1e-8)
    for z in range(B):                               # each sample's own gradient
        fz = lambda g, b: (O.layer_norm(x[z], g, b, 1e-3)[0] * w[z]).sum()
        assert np.allclose(G[z], _difference(lambda t: fz(t, beta), gamma), atol=1e-8)
        assert np.allclose(Hb[z], _difference(lambda t: fz(gamma, t), beta), atol=1e-8)
    assert np.allclose(sums["s_gamma"], 0.0625 * sum(G[z] ** 2 for z in range(B)))


@pytest.mark.parametrize("weighted", [False, True])
def test_softmax_loss_gradients_are_those_of_differences(weighted):
    rng = np.random.default_rng(4)
    B, P, Hd, Vc = 2, 3, 4, 6
    X, W = rng.standard_normal((B, P, Hd)), rng.standard_normal((Vc, Hd))
    target = np.array([[0, 5, -1], [2, -7, 2]])
    weight = rng.random((B, P)) if weighted else None
    wt = np.ones((B, P)) if weight is None else weight
    f = lambda X, W, z=slice(None): (O.softmax_loss(X[z].reshape(-1, Hd), W, target[z].reshape(-1))[0] * wt[z].reshape(-1)).sum()
    lse = O.softmax_loss(X.reshape(-1, Hd), W, target.reshape(-1))[1]
    D, dX, G, s, g = O.softmax_loss_backward(X, W, target, lse, weight, 0.5)
    assert np.allclose(dX, _difference(lambda t: f(t, W), X), atol=1e-8)
    for z in range(B):
        assert np.allclose(G[z], _difference(lambda t: f(X, t, slice(z, z + 1)), W), atol=1e-8)
    g64, s64 = V.sqgrad_conv(D.reshape(B, P, Vc), X, 0.5)            # the statistic's own definition with D and X in its places
    assert np.allclose(g, g64) and np.allclose(s, s64)
    assert (D[2] == 0).all() and (dX[0, 2] == 0).all()


def test_rows_that_are_not_asked_for_and_wrong_targets():
    X, W = np.ones((1, 3, 2)), np.eye(2)
    X[0, 1] = np.nan
    target = np.array([0, -1, 2])
    loss, lse, _ = O.softmax_loss(X[0], W, target)
    assert loss[1] == 0 and np.isnan(loss[2]) and np.isfinite(loss[0])
    D, dX, G, s, g = O.softmax_loss_backward(X, W, target[None], lse, None, 1.0)
    assert (D[1] == 0).all() and np.isnan(D[2]).all()
    D, dX, G, s, g = O.softmax_loss_backward(X[:, :2], W, target[None, :2], lse[:2], None, 1.0)
    assert np.isfinite(g).all() and (dX[0, 1] == 0).all()


def test_act8_is_within_half_a_unit_of_the_smallest_unit():
    rng = np.random.default_rng(5)
    x = (rng.standard_normal((64, 70)) * np.exp2(rng.integers(-140, 120, (64, 1)))).astype(np.float32)
    codes, exps = O.act8_encode(x)
    unit = np.repeat(np.exp2(exps.astype(float) - 127), 32, 1)[:, :70]
    top = np.abs(x.astype(float))
    assert (np.abs(O.act8_decode(codes, exps) - x.astype(float)) <= unit / 2).all()
    for b in range(3):
        t, u = top[:, 32 * b:32 * b + 32].max(1), np.exp2(exps[:, b].astype(float) - 127)
        assert (t < 127.5 * u).all()
        assert ((t >= 127.5 * u / 2) | (exps[:, b] == 1) | (t == 0)).all()
    assert np.abs(codes).max() == 127


def test_act8_values_and_special_blocks():
    x = np.zeros((7, 33), np.float32)
    x[0, :3] = 127, 63.5, -0.49                      # unit 1: ties to even
    x[1, 0] = 127.5                                  # no longer below 127.5 units: unit 2
    x[2, 5] = np.inf
    x[3, 32] = np.nan
    x[4, 0] = 2.0 ** -149                            # far below the smallest unit
    x[6, :2] = np.finfo(np.float32).max, -127 * 2.0 ** 121       # the largest value there is
    codes, exps = O.act8_encode(x)
    assert exps[:, 0].tolist() == [127, 128, 255, 120, 1, 120, 248] and exps[:, 1].tolist() == [120, 120, 120, 255, 120, 120, 120]
    assert codes[6, :2].tolist() == [127, -127]
    assert codes[0, :3].tolist() == [127, 64, 0] and codes[1, 0] == 64 and not codes[4].any()
    d = O.act8_decode(codes, exps)
    assert np.isnan(d[2, :32]).all() and d[2, 32] == 0 and np.isnan(d[3, 32]) and (d[3, :32] == 0).all()
