"""The token classifier's step: which products it makes, inputs at any address, feed-forward blocks of any number of channels."""
import numpy as np
import pytest

import block_checks as T

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return T.device()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_every_product_is_the_frameworks_own(dev, dtype, monkeypatch):
    import torch
    from paper_1802_06058_amd import token_step
    m = token_step.TokenStep(B=3, P=20, J=48, H=64, V=52, F=96, dropout=0.1, dtype=T.dtype_of(dtype))
    x, target = next(token_step.batches(m))

    def no(*_, **__):
        raise AssertionError("a library product")
    for name in ("matmul", "mm", "addmm", "bmm"):
        monkeypatch.setattr(torch, name, no)
        monkeypatch.setattr(torch.Tensor, name, no)
    monkeypatch.setattr(torch.Tensor, "__matmul__", no)
    W1 = m.p["W1"].to(m.dtype).clone()
    m.step(x, target)
    monkeypatch.undo()
    X, W = x.double().view(-1, 48), W1.double()
    want, size = T.back(X @ W), T.back(X.abs() @ W.abs())
    err = (48 + 16) * 2 * T.U * size
    assert (np.abs(T.back(m.h).reshape(want.shape) - want) <= err + T.half_unit(dtype) * (np.abs(want) + err)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_inputs_at_any_address(dev, dtype):
    """A batch cut out of a longer array: rows of 45 elements begin at any multiple of an element."""
    import torch
    from paper_1802_06058_amd import token_step
    out = []
    for shift in (0, 1):
        m = token_step.TokenStep(B=2, P=9, J=45, H=64, V=52, dtype=T.dtype_of(dtype))
        x, target = next(token_step.batches(m))
        flat = torch.zeros(x.numel() + 1, dtype=x.dtype, device=dev)
        there = flat[shift:shift + x.numel()].view(x.shape)
        there.copy_(x)
        m.step(there, target)
        out.append((m.h, m.g, m.s, m.param))
    assert all(torch.equal(a, b) for a, b in zip(*out))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("F", [1, 101, 130])
def test_a_feed_forward_block_of_any_number_of_channels(dev, F, dtype):
    """Its weights' sums land where the selection reads them: those of the inputs and gradients that the step left.  g's and s's own errors are relative to the sums of
    magnitudes: P terms a sample and B samples, within (P + B + 16) units 2^-23; the inputs are as the call saw them."""
    import torch
    from oracle import vgc_oracle as V
    from paper_1802_06058_amd import token_step
    B, P, H = 3, 20, 64
    m = token_step.TokenStep(B=B, P=P, J=48, H=H, V=52, F=F, dropout=0.1, dtype=T.dtype_of(dtype))
    x, target = next(token_step.batches(m))
    m.step(x, target)
    for k, X, D in (("Wb", m.u, m.dzb), ("Wa", m.y, m.za)):
        X, D = T.back(X), T.back(D)
        g, s = V.sqgrad_conv(X, D, 1.0 / B)
        size, _ = V.sqgrad_conv(np.abs(X), np.abs(D), 1.0 / B)
        by_sample = np.einsum("bpj,bpc->bjc", np.abs(X), np.abs(D)) / B
        e = (P + B + 16) * 2 * T.U
        assert (np.abs(T.back(m.gs[k]) - g) <= e * size + 1e-30).all(), k
        assert (np.abs(T.back(m.ss[k]) - s) <= 2 * e * (by_sample ** 2).sum(0) + 1e-30).all(), k
    for k, D in (("bb", m.dzb), ("ba", m.za)):                       # (of dz before it is rounded)
        D = T.back(D)
        off = (T.half_unit(dtype) + (P + B + 16) * 2 * T.U) * np.abs(D).sum((0, 1)) / B
        assert (np.abs(T.back(m.gs[k]) - D.sum((0, 1)) / B) <= off * (1 + 2.0 ** -7)).all(), k
