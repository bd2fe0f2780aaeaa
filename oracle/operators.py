"""Plain definitions, in 64 bits, of activations in 8 bits, layer norm and the softmax loss of a linear layer.

Like the rest of the oracle: NumPy, no code of the product package, used by tests only."""
import numpy as np

F64 = np.float64


def act8_encode(x):
    """codes int8 [R, C] and exps uint8 [R, ceil(C / 32)] of float32 rows: the smallest unit 2^(exp - 127), exp in 1 .. 248, of
    which a block's largest magnitude is less than 127.5; larger magnitudes than 127 of the largest unit count as that."""
    x = np.asarray(x, np.float32).astype(F64)
    R, C = x.shape
    nb = (C + 31) // 32
    codes, exps = np.zeros((R, C), np.int8), np.zeros((R, nb), np.uint8)
    units = np.exp2(np.arange(255) - 127.0)
    for b in range(nb):
        block = x[:, 32 * b:32 * b + 32]
        finite = np.isfinite(block).all(1)
        top = np.where(finite, np.abs(np.where(np.isfinite(block), block, 0)).max(1), 0)
        e = np.maximum(1, np.searchsorted(127.5 * units, top, side="right"))       # first unit with top < 127.5 units
        e = np.minimum(e, 248)
        e = np.where(top == 0, 120, e)
        q = np.clip(np.rint(np.where(finite[:, None], np.where(np.isfinite(block), block, 0) / units[e][:, None], 0)), -127, 127)
        codes[:, 32 * b:32 * b + 32] = q
        exps[:, b] = np.where(finite, e, 255)
    return codes, exps


def act8_decode(codes, exps):
    codes = np.asarray(codes)
    e = np.repeat(np.asarray(exps), 32, axis=-1)[..., :codes.shape[-1]].astype(F64)
    return np.where(e == 255, np.nan, codes * np.exp2(e - 127))


def layer_norm(x, gamma, beta, eps):
    """y, mean, rstd, xhat of rows [R, C]."""
    x = np.asarray(x, F64)
    mean = x.mean(1)
    rstd = 1 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    xhat = (x - mean[:, None]) * rstd[:, None]
    return xhat * np.asarray(gamma, F64) + np.asarray(beta, F64), mean, rstd, xhat


def layer_norm_backward(dy, xhat, rstd, gamma, c):
    """dx [B, P, C] and the samples' gradients of gamma and beta [B, C] with their sums: dict(g_gamma, s_gamma, g_beta, s_beta)."""
    dy, xhat, gamma = np.asarray(dy, F64), np.asarray(xhat, F64), np.asarray(gamma, F64)
    d = dy * gamma
    dx = np.asarray(rstd, F64)[..., None] * (d - d.mean(-1, keepdims=True) - xhat * (d * xhat).mean(-1, keepdims=True))
    G, H = (dy * xhat).sum(1), dy.sum(1)
    return dx, G, H, dict(g_gamma=c * G.sum(0), s_gamma=c * c * (G * G).sum(0), g_beta=c * H.sum(0), s_beta=c * c * (H * H).sum(0))


def softmax_loss(X, W, target):
    """loss, lse [N] and the logits of X [N, H], W [V, H]; target negative: not asked for; V or more: NaN."""
    X, W, target = np.asarray(X, F64), np.asarray(W, F64), np.asarray(target)
    z = X @ W.T
    top = z.max(1, keepdims=True)
    lse = (top + np.log(np.exp(z - top).sum(1, keepdims=True)))[:, 0]
    picked = np.take_along_axis(z, np.clip(target, 0, W.shape[0] - 1)[:, None], 1)[:, 0]
    loss = np.where(target < 0, 0.0, np.where(target < W.shape[0], lse - picked, np.nan))
    return loss, lse, z


def softmax_loss_backward(X, W, target, lse, weight, c):
    """D [B P, V], dX [B, P, H] and the two sums over the samples for W, from X [B, P, H] and the forward pass's lse [B P]."""
    B, P, H = X.shape
    X, W, target = np.asarray(X, F64).reshape(B * P, H), np.asarray(W, F64), np.asarray(target).reshape(-1)
    weight = np.ones(B * P) if weight is None else np.asarray(weight, F64).reshape(-1)
    asked = target >= 0
    D = np.zeros((B * P, W.shape[0]))
    rows = np.flatnonzero(asked)
    D[rows] = np.exp(X[rows] @ W.T - np.asarray(lse, F64).reshape(-1)[rows, None])
    here = rows[target[rows] < W.shape[0]]
    D[here, target[here]] -= 1
    D *= np.where(asked, weight, 0)[:, None]
    D[rows[target[rows] >= W.shape[0]]] = np.nan
    Xa = np.where(asked[:, None], X, 0)
    G = np.einsum("bpv,bph->bvh", D.reshape(B, P, -1), Xa.reshape(B, P, H), optimize=True)
    return D, (D @ W).reshape(B, P, H), G, c * c * (G * G).sum(0), c * G.sum(0)
