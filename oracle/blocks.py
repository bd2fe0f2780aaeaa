"""Plain definitions, in 64 bits, of dropout from a counter, a linear layer with what follows it, and group norm.

Like the rest of the oracle: NumPy, no code of the product package, used by tests only."""
import math

import numpy as np

F64 = np.float64
_erfc = np.vectorize(math.erfc, otypes=[F64])


# ---- activations: 0 none, 1 relu, 2 gelu, 3 silu ----
def _sigmoid(z):
    return np.where(z >= 0, 1 / (1 + np.exp(-np.abs(z))), np.exp(-np.abs(z)) / (1 + np.exp(-np.abs(z))))


def act(z, kind):
    z = np.asarray(z, F64)
    return [lambda: z, lambda: np.maximum(z, 0), lambda: z * 0.5 * _erfc(-z / math.sqrt(2)), lambda: z * _sigmoid(z)][kind]()


def slope(z, kind):
    z = np.asarray(z, F64)
    s = _sigmoid(z)
    return [lambda: np.ones_like(z), lambda: (z > 0).astype(F64),
            lambda: 0.5 * _erfc(-z / math.sqrt(2)) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi), lambda: s + z * s * (1 - s)][kind]()


# ---- dropout ----
def philox(counter, key):
    """Four words of Philox 4x32-10: counter four, key two arrays of 32-bit numbers."""
    low = np.uint64(0xFFFFFFFF)
    c = [np.asarray(x, np.uint64) for x in counter]
    k = [np.asarray(x, np.uint64) for x in key]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ k[0], b & low, (a >> np.uint64(32)) ^ c[3] ^ k[1], a & low]
        k = [(k[0] + np.uint64(0x9E3779B9)) & low, (k[1] + np.uint64(0xBB67AE85)) & low]
    return c


def threshold(p):
    return int(math.floor(np.float32(p).astype(F64) * 65536 + 0.5))


def keep_factor(R, C, p, key, call):
    """What dropout multiplies the elements of R rows of C with."""
    t = threshold(p)
    if t == 0:
        return np.ones((R, C))
    if t == 65536:
        return np.zeros((R, C))
    key, call = int(key) & (2 ** 64 - 1), int(call) & (2 ** 64 - 1)
    pieces = (C + 7) // 8
    rows, cols = np.meshgrid(np.arange(R), np.arange(pieces), indexing="ij")
    words = philox((cols, rows, np.full_like(rows, call & 0xFFFFFFFF), np.full_like(rows, call >> 32)), (key & 0xFFFFFFFF, key >> 32))
    out = np.empty((R, pieces, 8), np.int64)
    for j, w in enumerate(words):
        out[:, :, 2 * j] = (w & np.uint64(0xFFFF)).astype(np.int64)
        out[:, :, 2 * j + 1] = (w >> np.uint64(16)).astype(np.int64)
    return np.where(out.reshape(R, -1)[:, :C] >= t, 65536 / (65536 - t), 0.0)


# ---- linear layer ----
def linear(X, W, bias=None, kind=0, factor=1.0, residual=0.0):
    """y and z of X [N, K], W [K, C]; factor: what dropout multiplies act(z) with."""
    z = np.asarray(X, F64) @ np.asarray(W, F64) + (0 if bias is None else np.asarray(bias, F64))
    a = act(z, kind)
    return np.where(np.asarray(factor) == 0, 0, a * factor) + np.asarray(residual, F64), z


def linear_backward(dy, z, W, kind, c, factor=1.0, add=0.0):
    """dz [B, P, C], dX [B, P, K] and s, g of the bias, with the samples' own gradients of it [B, C]."""
    B, P, C = dy.shape
    dz = np.asarray(dy, F64) * np.reshape(factor, (B, P, C) if np.ndim(factor) else ())
    if kind:
        dz = dz * slope(z, kind)
    H = dz.sum(1)
    return dz, np.asarray(add, F64) + dz @ np.asarray(W, F64).T, c * c * (H * H).sum(0), c * H.sum(0), H


# ---- group norm, x [B, P, C] ----
def group_norm(x, G, gamma, beta, eps, kind):
    """y, mean and rstd [B, G], xhat."""
    B, P, C = x.shape
    v = np.asarray(x, F64).reshape(B, P, G, C // G)
    mean = v.mean((1, 3))
    rstd = 1 / np.sqrt(((v - mean[:, None, :, None]) ** 2).mean((1, 3)) + eps)
    xhat = ((v - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(B, P, C)
    return act(xhat * np.asarray(gamma, F64) + np.asarray(beta, F64), kind), mean, rstd, xhat


def group_norm_backward(dy, xhat, rstd, gamma, beta, kind, c):
    """dx, the samples' gradients of gamma and beta [B, C], their sums, and e, the gradient before the activation."""
    B, P, C = xhat.shape
    G = rstd.shape[1]
    gamma, beta = np.asarray(gamma, F64), np.asarray(beta, F64)
    e = np.asarray(dy, F64) * slope(xhat * gamma + beta, kind)
    d, h = (e * gamma).reshape(B, P, G, C // G), xhat.reshape(B, P, G, C // G)
    dx = np.asarray(rstd, F64)[:, None, :, None] * (d - d.mean((1, 3), keepdims=True) - h * (d * h).mean((1, 3), keepdims=True))
    g, b = (e * xhat).sum(1), e.sum(1)
    return dx.reshape(B, P, C), g, b, dict(g_gamma=c * g.sum(0), s_gamma=c * c * (g * g).sum(0), g_beta=c * b.sum(0), s_beta=c * c * (b * b).sum(0)), e
