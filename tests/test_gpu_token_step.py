"""The operators together, as a worker's step uses them (paper_1802_06058_amd.token_step): the sums that reach the selection are those of
the oracle's chain, training lowers the loss, and a run repeats bit for bit."""
import numpy as np
import pytest

from oracle import operators as O
from oracle import vgc_oracle as V

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ts():
    import torch
    from paper_1802_06058_amd import token_step, vgc
    assert torch.cuda.is_available()
    vgc.load()
    return token_step


def test_the_sums_of_a_step_are_those_of_the_chain(ts):
    """float32; relative to a sum's largest entry: the chain's float32 products and sums of at most 300 terms, normalised and multiplied
    three times over, keep well within 1e-4 of it (300 * 2^-23 * 3 = 1.1e-4 in the worst case), squares within twice that."""
    import torch
    B, P, J, H, Vc = 3, 20, 48, 64, 50
    m = ts.TokenStep(B, P, J, H, Vc, dtype=torch.float32)
    p0 = {k: t.double().cpu().numpy() for k, t in m.p.items()}
    x, target = next(ts.batches(m))
    before = m.param.clone()
    m.step(x, target)
    t = target.cpu().numpy()
    c = 1.0 / B
    x64 = x.double().cpu().numpy().reshape(B * P, J)
    y, mean, rstd, xhat = O.layer_norm(x64 @ p0["W1"], p0["gamma"], p0["beta"], 1e-5)
    loss, lse, _ = O.softmax_loss(y, p0["W"], t.reshape(-1))
    assert np.allclose(m.loss.cpu().numpy(), loss, atol=1e-4)
    w = np.repeat(1.0 / np.maximum((t >= 0).sum(1, keepdims=True), 1), P, 1)
    _, dy, _, s, g = O.softmax_loss_backward(y.reshape(B, P, H), p0["W"], t, lse, w, c)
    want = {"W": (s, g)}
    kept = O.act8_decode(*O.act8_encode(xhat.astype(np.float32)))
    got = O.act8_decode(m.kept_h[0].cpu().numpy().reshape(B * P, H), m.kept_h[1].cpu().numpy().reshape(B * P, -1))
    assert (np.abs(got - kept) <= np.abs(xhat).max() / 64).all() and np.mean(got != kept) < 0.01     # (a tie that the float rounds the other way)
    dh, _, _, sums = O.layer_norm_backward(dy, got.reshape(B, P, H), rstd.reshape(B, P), p0["gamma"], c)
    for k in ("gamma", "beta"):
        want[k] = (sums["s_" + k], sums["g_" + k])
    g, s = V.sqgrad_conv(O.act8_decode(*O.act8_encode(x64.astype(np.float32))).reshape(B, P, J), dh, c)
    want["W1"] = (s, g)
    for k, (s, g) in want.items():
        assert np.abs(m.gs[k].double().cpu().numpy() - g).max() <= 1.1e-4 * np.abs(g).max(), k
        assert np.abs(m.ss[k].double().cpu().numpy() - s).max() <= 2.2e-4 * np.abs(s).max(), k
    assert not torch.equal(before, m.param)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_training_lowers_the_loss_and_repeats(ts, dtype):
    import torch
    runs = []
    for _ in range(2):
        m = ts.TokenStep(B=8, P=32, J=64, H=128, V=40, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, lr=0.1)
        data = ts.batches(m)
        losses = []
        for _ in range(60):
            x, target = next(data)
            losses.append(float(m.step(x, target).sum() / (target >= 0).sum()))
        runs.append((losses, m.param.clone()))
    assert runs[0][0] == runs[1][0] and torch.equal(runs[0][1], runs[1][1])
    first, last = np.mean(runs[0][0][:3]), np.mean(runs[0][0][-5:])
    assert first > 0.9 * np.log(40) and last < 0.5 * first
