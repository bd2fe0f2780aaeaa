"""The FC statistic of rows kept in 8 bits from bfloat16 planes: outputs beyond the caches, and sums that are not finite or whose squares leave
float32's range on the way."""
import numpy as np
import pytest

from oracle import operators as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    import torch
    from paper_1802_06058_amd import vgc
    assert torch.cuda.is_available()
    vgc.load()
    return torch.device("cuda:0")


def _call(dev, q, e, D):
    import torch
    from paper_1802_06058_amd import vgc
    (B, J), C = q.shape, D.shape[1]
    ws = torch.full((vgc.sqgrad_act8_workspace_bytes(vgc.FC, vgc.BF16, B, 1, J, C),), 0xFF, dtype=torch.uint8, device=dev)
    s, g = (torch.full((J * C + 64,), 7.0, device=dev) for _ in range(2))
    vgc.sqgrad_act8(vgc.FC, torch.from_numpy(q).to(dev), torch.from_numpy(e).to(dev), D, 1.0 / B, s, g, ws)
    assert (s[J * C:] == 7).all() and (g[J * C:] == 7).all()
    only = torch.full_like(s, 7.0)
    vgc.sqgrad_act8(vgc.FC, torch.from_numpy(q).to(dev), torch.from_numpy(e).to(dev), D, 1.0 / B, only, None, ws)
    assert torch.equal(only.view(torch.int32), s.view(torch.int32))
    return g[:J * C].view(J, C), s[:J * C].view(J, C)


def test_sums_beyond_the_caches(dev):
    """More than 256 MiB of g and s, by 1e-5 of the magnitudes summed (24 samples: as many roundings or truncations of 2^-23)."""
    import torch
    B, J, C = 24, 8209, 4133
    rng = np.random.default_rng(0)
    q, e = O.act8_encode(np.maximum(rng.standard_normal((B, J)), 0).astype(np.float32))
    D = torch.from_numpy((1e-3 * rng.standard_normal((B, C))).astype(np.float32)).to(dev).to(torch.bfloat16)
    g, s = _call(dev, q, e, D)
    x, d = torch.from_numpy(O.act8_decode(q, e)).to(dev), D.double()
    xt = x.t().contiguous()
    assert ((g.double() - xt @ d / B).abs() <= 1e-5 * (xt.abs() @ d.abs()) / B).all()
    want = xt.square() @ d.square() / B ** 2
    assert ((s.double() - want).abs() <= 1e-5 * want).all()


@pytest.mark.parametrize("B,J,C", [(5, 70, 40), (40, 300, 200), (70, 133, 135)])
def test_squares_beyond_the_range_and_sums_that_are_not_finite(dev, B, J, C):
    """Each output is what float32 arithmetic makes of its samples' gradients x d: finite where a square of x or d alone leaves the range, infinite
    where a gradient or its square does, NaN where a NaN or 0 times an infinity is among them; the others' values in 64 bits."""
    import torch
    rng = np.random.default_rng(B)
    x = rng.standard_normal((B, J)).astype(np.float32)
    x[rng.random((B, J)) < 0.2] = 0
    d = (1e-3 * rng.standard_normal((B, C))).astype(np.float32)
    x[0, 3] = 3e19                                   # its square is not a float32
    x[1, 36] = 2e38
    d[2, 5] = -2e25                                  # the square of this one neither
    d[1, 7], d[1, 8] = 1e3, 1e-30                    # with x[1, 36]: a gradient beyond the range, and one of 2e8
    d[0, 11], d[3, 11], d[4, 12] = np.inf, -np.inf, np.inf
    d[3, 13] = np.nan
    x[4, 65] = np.nan                                # its block of 32 is not a number
    D = torch.from_numpy(d).to(dev).to(torch.bfloat16)
    q, e = O.act8_encode(x)
    g, s = _call(dev, q, e, D)
    with np.errstate(all="ignore"):
        p = O.act8_decode(q, e)[:, :, None] * D.double().cpu().numpy()[:, None, :]
        p32 = p.astype(np.float32)
        g64, s64 = p.sum(0) / B, (p * p).sum(0) / B ** 2
        inexact = ~np.isfinite(p32).all(0)
        g64 = np.where(inexact, p32.sum(0), g64)
        s64 = np.where(~np.isfinite(p32 * p32).all(0), (p32 * p32).sum(0), s64)
        ga = np.abs(p).sum(0) / B
    assert np.isinf(s64).any() and np.isnan(s64).any() and np.isinf(g64).any() and np.isfinite(s64[3]).any()
    for got, want, size in ((g, g64, ga), (s, s64, s64)):
        got = got.double().cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(want))
        inf = np.isinf(want)
        assert np.array_equal(got[inf], want[inf])
        ok = np.isfinite(want)
        assert (np.abs(got[ok] - want[ok]) <= 1e-5 * size[ok]).all()
