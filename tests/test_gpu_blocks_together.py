"""The linear layer, dropout and group norm together, as a step uses them: in the token classifier's step with its feed-forward block, and in a residual block of
1 x 1 convolutions over channels-last images, issued one by one and from a graph.

Tolerance against the oracle's chain, float32, relative to a result's largest entry: products of at most T terms, each sum within T units of 2^-23 of its magnitudes, S of them in a row:
S T 2^-23, and twice that for squares."""
import subprocess
import sys

import block_checks as T
import numpy as np
import pytest

from oracle import blocks as O
from oracle import operators as L
from oracle import vgc_oracle as V

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return T.device()


def _close(got, want, tol, what):
    err, top = np.abs(T.back(got).reshape(np.shape(want)) - want).max(), np.abs(want).max()
    assert err <= tol * top, (what, err / top, tol)


def test_a_token_step_with_a_feed_forward_block(dev):
    import torch
    from paper_1802_06058_amd import token_step
    B, P, J, H, Vc, F = 3, 20, 48, 64, 52, 96
    m = token_step.TokenStep(B, P, J, H, Vc, dtype=torch.float32, F=F, dropout=0.2)
    p0 = {k: T.back(t) for k, t in m.p.items()}
    p0["ba"], p0["bb"] = 0.1 * np.random.default_rng(0).standard_normal(F), 0.1 * np.random.default_rng(1).standard_normal(H)
    m.p["ba"].copy_(torch.from_numpy(p0["ba"]))
    m.p["bb"].copy_(torch.from_numpy(p0["bb"]))
    p0["ba"], p0["bb"] = T.back(m.p["ba"]), T.back(m.p["bb"])
    x, target = next(token_step.batches(m))
    m.step(x, target)
    t, c, N = target.cpu().numpy(), 1.0 / B, B * P
    x64 = T.back(x).reshape(N, J)
    y, mean, rstd, xhat = L.layer_norm(x64 @ p0["W1"], p0["gamma"], p0["beta"], 1e-5)
    u, za = O.linear(y, p0["Wa"], p0["ba"], 2)
    f = O.keep_factor(N, H, 0.2, 0, 1)
    out, _ = O.linear(u, p0["Wb"], p0["bb"], 0, f, y)
    loss, lse, _ = L.softmax_loss(out, p0["W"], t.reshape(-1))
    assert np.allclose(T.back(m.loss), loss, atol=2e-4)
    w = np.repeat(1.0 / np.maximum((t >= 0).sum(1, keepdims=True), 1), P, 1)
    _, dout, _, sW, gW = L.softmax_loss_backward(out.reshape(B, P, H), p0["W"], t, lse, w, c)
    want = {"W": (sW, gW)}
    dzb, du, s, g, _ = O.linear_backward(dout, None, p0["Wb"], 0, c, f)
    want["bb"] = (s, g)
    dza, dy, s, g, _ = O.linear_backward(du, za.reshape(B, P, F), p0["Wa"], 2, c, add=dout)
    want["ba"] = (s, g)
    for k, X, D in (("Wb", u.reshape(B, P, F), dzb), ("Wa", y.reshape(B, P, H), dza)):
        g, s = V.sqgrad_conv(X, D, c)
        want[k] = (s, g)
    kept = L.act8_decode(m.kept_h[0].cpu().numpy().reshape(N, H), m.kept_h[1].cpu().numpy().reshape(N, -1))
    _, _, _, sums = L.layer_norm_backward(dy, kept.reshape(B, P, H), rstd.reshape(B, P), p0["gamma"], c)
    for k in ("gamma", "beta"):
        want[k] = (sums["s_" + k], sums["g_" + k])
    tol = 6 * 300 * 2.0 ** -23
    for k, (s, g) in want.items():
        _close(m.gs[k], g, tol, k)
        _close(m.ss[k], s, 2 * tol, k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_step_with_the_block_repeats_bit_for_bit(dev, dtype):
    import torch
    from paper_1802_06058_amd import token_step
    runs = []
    for _ in range(2):
        m = token_step.TokenStep(B=4, P=32, J=64, H=128, V=40, F=256, dropout=0.1, dtype=T.dtype_of(dtype))
        data = token_step.batches(m)
        losses = []
        for _ in range(4):
            x, target = next(data)
            losses.append(m.step(x, target).clone())
        runs.append((losses, m.param.clone()))
    assert all(torch.equal(a, b) for a, b in zip(runs[0][0], runs[1][0])) and torch.equal(runs[0][1], runs[1][1])
    assert torch.isfinite(runs[0][1]).all()


def test_the_command_runs(dev):
    out = subprocess.run([sys.executable, "-m", "paper_1802_06058_amd.token_step", "--steps", "2", "--feed-forward", "256", "--dropout", "0.1"], capture_output=True, text=True,
                         timeout=100)
    assert out.returncode == 0 and "step 1: loss" in out.stdout, out.stderr[-2000:]


class ImageBlock:
    """x + drop(conv(gelu(conv(silu(group norm(x)))))), 1 x 1 convolutions; x [B, height, width, C]."""

    def __init__(self, dev, dtype, B=3, side=6, C=48, F=80, G=6, seed=0):
        import torch
        from paper_1802_06058_amd import vgc
        self.vgc, self.B, self.P, self.C, self.F, self.G = vgc, B, side * side, C, F, G
        gen = np.random.default_rng(seed)
        t = lambda a, d=dtype: T.to(a, d, dev)
        self.x = t(gen.standard_normal((B, side, side, C)))
        self.gamma, self.beta = t(1 + 0.2 * gen.standard_normal(C), "f32"), t(0.2 * gen.standard_normal(C), "f32")
        self.Wa, self.Wb = t(gen.standard_normal((C, F)) / np.sqrt(C)), t(gen.standard_normal((F, C)) / np.sqrt(F))
        self.ba, self.bb = t(0.2 * gen.standard_normal(F), "f32"), t(0.2 * gen.standard_normal(C), "f32")
        self.dout = t(gen.standard_normal((B, self.P, C)))
        self.rng = T.rng_state(dev)
        e = lambda *s: torch.empty(s, dtype=self.x.dtype, device=dev)
        f = lambda *s: torch.empty(s, device=dev)
        self.n, self.u, self.za, self.y = e(B, self.P, C), e(B, self.P, F), e(B, self.P, F), e(B, self.P, C)
        self.mean, self.rstd = f(B, G), f(B, G)
        self.dzb, self.du, self.dza, self.dn, self.dx = e(B, self.P, C), e(B, self.P, F), e(B, self.P, F), e(B, self.P, C), e(B, side, side, C)
        self.sums = {k: f(n) for k, n in (("s_bb", C), ("g_bb", C), ("s_ba", F), ("g_ba", F), ("s_gamma", C), ("s_beta", C), ("g_gamma", C), ("g_beta", C))}
        self.weights = {k: f(*s) for k, s in (("s_Wb", (F, C)), ("g_Wb", (F, C)), ("s_Wa", (C, F)), ("g_Wa", (C, F)))}
        code = vgc.F32 if dtype == "f32" else vgc.BF16
        N = B * self.P
        self.ws = T.workspace(max(vgc.group_norm_workspace_bytes(code, B, self.P, C, G), vgc.group_norm_backward_workspace_bytes(code, B, self.P, C, G),
                                  *(vgc.linear_workspace_bytes(code, N, *s) for s in ((C, F), (F, C))), *(vgc.linear_backward_workspace_bytes(code, B, self.P, *s) for s in ((C, F), (F, C))),
                                  *(vgc.sqgrad_workspace_bytes(vgc.CONV, code, B, self.P, *s) for s in ((C, F), (F, C)))), dev)

    def run(self):
        vgc, c, S, W = self.vgc, 1.0 / self.B, self.sums, self.weights
        flat = self.x.view(self.B, self.P, self.C)
        vgc.group_norm(self.x, self.gamma, self.beta, 1e-5, vgc.ACT_SILU, self.n, self.mean, self.rstd, self.ws)
        vgc.linear(self.n, self.Wa, self.u, self.ba, vgc.ACT_GELU, z=self.za, workspace=self.ws)
        vgc.linear(self.u, self.Wb, self.y, self.bb, residual=flat, p=0.3, rng=self.rng, workspace=self.ws)
        vgc.linear_backward(self.dout, None, self.Wb, vgc.ACT_NONE, c, self.dzb, self.du, S["s_bb"], S["g_bb"], p=0.3, rng=self.rng, workspace=self.ws)
        vgc.sqgrad(vgc.CONV, self.u, self.dzb, c, W["s_Wb"], W["g_Wb"], self.ws)
        vgc.linear_backward(self.du, self.za, self.Wa, vgc.ACT_GELU, c, self.dza, self.dn, S["s_ba"], S["g_ba"], workspace=self.ws)
        vgc.sqgrad(vgc.CONV, self.n, self.dza, c, W["s_Wa"], W["g_Wa"], self.ws)
        vgc.group_norm_backward(self.dn.view_as(self.x), self.x, self.mean, self.rstd, self.gamma, self.beta, vgc.ACT_SILU, c, self.dx, S["s_gamma"], S["s_beta"], S["g_gamma"], S["g_beta"],
                                workspace=self.ws)

    def results(self):
        return [self.n, self.mean, self.rstd, self.u, self.za, self.y, self.dzb, self.du, self.dza, self.dn, self.dx, *self.sums.values(), *self.weights.values()]


def test_an_image_block_is_the_oracles_chain(dev):
    """float32, and the gradient of x against differences of the chain along a random direction."""
    b = ImageBlock(dev, "f32")
    b.run()
    B, P, C, F, G, c = b.B, b.P, b.C, b.F, b.G, 1.0 / b.B
    x, gamma, beta, Wa, Wb, ba, bb, dout = (T.back(t) for t in (b.x.view(B, P, C), b.gamma, b.beta, b.Wa, b.Wb, b.ba, b.bb, b.dout))
    f = O.keep_factor(B * P, C, 0.3, *b.rng.tolist())

    def forward(x):
        n, mean, rstd, xhat = O.group_norm(x, G, gamma, beta, 1e-5, 3)
        u, za = O.linear(n.reshape(-1, C), Wa, ba, 2)
        return O.linear(u, Wb, bb, 0, f, x.reshape(-1, C))[0].reshape(B, P, C), n, rstd, xhat, u, za

    y, n, rstd, xhat, u, za = forward(x)
    tol = 8 * 108 * 2.0 ** -23                                       # (a group's sums: 288 terms, of which float32's tree makes far fewer roundings)
    for got, want, what in ((b.n, n, "n"), (b.u, u, "u"), (b.y, y, "y")):
        _close(got, want, tol, what)
    dzb, du, s_bb, g_bb, _ = O.linear_backward(dout, None, Wb, 0, c, f)
    dza, dn, s_ba, g_ba, _ = O.linear_backward(du, za.reshape(B, P, F), Wa, 2, c)
    dx, _, _, sums, _ = O.group_norm_backward(dn, xhat, rstd, gamma, beta, 3, c)
    want = dict(s_bb=s_bb, g_bb=g_bb, s_ba=s_ba, g_ba=g_ba, **sums)
    for k, (X, D) in dict(Wb=(u.reshape(B, P, F), dzb), Wa=(n, dza)).items():
        want["g_" + k], want["s_" + k] = V.sqgrad_conv(X, D, c)
    for k, w in want.items():
        _close((b.sums | b.weights)[k], w, 2 * tol if k[0] == "s" else tol, k)
    _close(b.dx, dx, tol, "dx")
    d = np.random.default_rng(5).standard_normal(x.shape)
    h = 1e-5
    slope = ((forward(x + h * d)[0] - forward(x - h * d)[0]) * dout).sum() / (2 * h)
    whole = T.back(b.dx).reshape(B, P, C) + dout                     # the residual path's gradient came past
    assert abs((whole * d).sum() - slope) <= 1e-4 * np.abs(whole * d).sum()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("side", [6, 70])
def test_a_recorded_block_replays_like_eager_calls(dev, dtype, side):
    """Small and large images (groups held by a workgroup, and by chunks); every replay with another mask, eager work and a synchronisation between; then two graphs with one workspace, in turn."""
    import torch
    eager, first, second = (ImageBlock(dev, dtype, side=side) for _ in range(3))
    second.ws = first.ws
    side_stream = torch.cuda.Stream()
    side_stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side_stream):
        first.run()
        second.run()
    torch.cuda.current_stream().wait_stream(side_stream)
    torch.cuda.synchronize()
    graphs = []
    for b in (first, second):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            b.run()
        graphs.append(g)
    for call in range(4):
        for b in (eager, first, second):
            b.rng[1] = call
        for b in (first, second):
            for t in b.results():
                t.fill_(float("nan"))
        eager.run()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        torch.randn(1 << 20, device=dev).sum().item()
        for b in (first, second):
            for k, (want, got) in enumerate(zip(eager.results(), b.results())):
                assert torch.equal(want, got), (call, k)


def test_calls_side_by_side_do_not_share_anything(dev):
    """The same work on two streams at once, a workspace each."""
    import torch
    blocks = [ImageBlock(dev, "bf16", side=40, seed=s) for s in (1, 1, 2, 2)]
    for b in (blocks[0], blocks[2]):
        b.run()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s, b in zip(streams, (blocks[1], blocks[3])):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            for _ in range(3):
                b.run()
    torch.cuda.synchronize()
    for a, b in ((blocks[0], blocks[1]), (blocks[2], blocks[3])):
        assert all(torch.equal(x, y) for x, y in zip(a.results(), b.results()))
