"""Pins of the oracle's dropout, linear layer and group norm: the generator's published words, gradients against differences, sums against
the samples taken one by one."""
import numpy as np
import pytest

from oracle import blocks as O
from oracle import operators as L

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


@pytest.mark.parametrize("counter,key,words", [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))])
def test_the_generator_gives_its_published_words(counter, key, words):
    assert tuple(int(w) for w in O.philox(counter, key)) == words


def test_dropout_keeps_the_mean_and_takes_the_share():
    f = O.keep_factor(500, 1003, 0.25, 77, 3)
    n = f.size
    assert abs((f == 0).mean() - 0.25) < 5 * np.sqrt(0.25 * 0.75 / n) and abs(f.mean() - 1) < 5 * np.sqrt(1 / 3 / n)
    assert set(np.unique(f)) == {0.0, 4 / 3}
    other = O.keep_factor(500, 1003, 0.25, 77, 4)
    assert abs(((f == 0) & (other == 0)).mean() - 0.0625) < 5 * np.sqrt(0.0625 / n)                # another call, another mask
    assert (O.keep_factor(20, 1003, 0.25, 77, 3) == f[:20]).all()                                   # by row and column only
    assert (O.keep_factor(500, 11, 0.25, 77, 3) == f[:, :11]).all()
    assert (O.keep_factor(2, 9, 0.0, 1, 1) == 1).all() and (O.keep_factor(2, 9, 1.0, 1, 1) == 0).all()
    assert O.threshold(0.1) == 6554 and O.threshold(2.0 ** -18) == 0 and O.threshold(1 - 2.0 ** -18) == 65536


@pytest.mark.parametrize("kind", [0, 1, 2, 3])
def test_slopes_are_those_of_differences(kind):
    z = np.array([-6.0, -2.5, -0.75, -0.1, 0.1, 0.3, 1.7, 5.0])
    assert np.allclose(O.slope(z, kind), (O.act(z + H, kind) - O.act(z - H, kind)) / (2 * H), atol=1e-9)


@pytest.mark.parametrize("kind", [0, 1, 2, 3])
def test_linear_gradients_are_those_of_differences(kind):
    rng = np.random.default_rng(5 + kind)
    B, P, K, C = 3, 2, 4, 5
    X, W, b, w = rng.standard_normal((B, P, K)), rng.standard_normal((K, C)), rng.standard_normal(C), rng.standard_normal((B, P, C))
    factor = O.keep_factor(B * P, C, 0.5, 9, 1)
    f = lambda X, b: (O.linear(X.reshape(-1, K), W, b, kind, factor[:X.shape[0] * P])[0].reshape(-1, P, C) * w[:X.shape[0]]).sum() + (0.5 * X).sum()
    z = O.linear(X.reshape(-1, K), W, b)[1].reshape(B, P, C)
    dz, dX, s, g, Hb = O.linear_backward(w, z, W, kind, 0.25, factor, 0.5 * np.ones((B, P, K)))
    assert np.allclose(dX, _difference(lambda t: f(t, b), X), atol=1e-8)
    for q in range(B):
        fq = lambda b: (O.linear(X[q], W, b, kind, factor[q * P:(q + 1) * P])[0] * w[q]).sum()
        assert np.allclose(Hb[q], _difference(fq, b), atol=1e-8)
    assert np.allclose(s, 0.0625 * sum(Hb[q] ** 2 for q in range(B))) and np.allclose(g, 0.25 * Hb.sum(0))


@pytest.mark.parametrize("kind,G", [(0, 1), (1, 2), (2, 3), (3, 6)])
def test_group_norm_gradients_are_those_of_differences(kind, G):
    rng = np.random.default_rng(8 + kind)
    B, P, C = 2, 3, 6
    x, w = rng.standard_normal((B, P, C)), rng.standard_normal((B, P, C))
    gamma, beta = 1 + 0.3 * rng.standard_normal(C), rng.standard_normal(C)
    f = lambda x, gamma, beta, z=slice(None): (O.group_norm(x, G, gamma, beta, 1e-3, kind)[0] * w[z]).sum()
    _, _, rstd, xhat = O.group_norm(x, G, gamma, beta, 1e-3, kind)
    dx, g, b, sums, _ = O.group_norm_backward(w, xhat, rstd, gamma, beta, kind, 0.5)
    assert np.allclose(dx, _difference(lambda t: f(t, gamma, beta), x), atol=1e-8)
    for z in range(B):
        assert np.allclose(g[z], _difference(lambda t: f(x[z:z + 1], t, beta, slice(z, z + 1)), gamma), atol=1e-8)
        assert np.allclose(b[z], _difference(lambda t: f(x[z:z + 1], gamma, t, slice(z, z + 1)), beta), atol=1e-8)
    assert np.allclose(sums["s_gamma"], 0.25 * sum(g[z] ** 2 for z in range(B))) and np.allclose(sums["g_beta"], 0.5 * b.sum(0))


def test_group_norm_of_one_position_and_one_group_is_layer_norm():
    rng = np.random.default_rng(1)
    x, gamma, beta = rng.standard_normal((4, 1, 10)), rng.standard_normal(10), rng.standard_normal(10)
    y, mean, rstd, xhat = O.group_norm(x, 1, gamma, beta, 1e-5, 0)
    want = L.layer_norm(x[:, 0], gamma, beta, 1e-5)
    assert all(np.allclose(a.reshape(b.shape), b) for a, b in zip((y, mean, rstd, xhat), want))
