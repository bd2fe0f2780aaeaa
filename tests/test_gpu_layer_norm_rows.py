"""Layer norm's forward pass over many rows that are not kept: other kernels than the kept form's from 520 channels on, so against 64 bits
by itself.  Tolerances as in test_gpu_layer_norm.py: fewer than 128 roundings of 2^-24 of the magnitudes summed in a row's sums, a handful
for the rest, and half a unit of a bfloat16 output."""
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def dev():
    import torch
    from paper_1802_06058_amd import vgc
    assert torch.cuda.is_available()
    vgc.load()
    return torch.device("cuda:0")


def _check(x, gamma, beta, eps, y, mean, rstd, depth=128):
    """Of rows of x, in 64 bits."""
    import torch
    bf16, x, gamma, beta = x.dtype == torch.bfloat16, x.double(), gamma.double(), beta.double()
    m = x.mean(1, keepdim=True)
    r = (((x - m) ** 2).mean(1, keepdim=True) + eps).rsqrt()
    h = (x - m) * r
    err_m = depth * U * x.abs().mean(1, keepdim=True)
    err_r = r * (depth * U + 8 * U + 2 * r * err_m)
    err_h = r * err_m + h.abs() * (err_r / r) + 4 * U * h.abs() + U * r * x.abs()
    want = h * gamma + beta
    tol = gamma.abs() * err_h + 4 * U * ((h * gamma).abs() + beta.abs()) + (2.0 ** -8 * want.abs() if bf16 else 0)
    assert ((mean.double() - m[:, 0]).abs() <= (err_m + U * m.abs())[:, 0]).all()
    assert ((rstd.double() - r[:, 0]).abs() <= err_r[:, 0]).all()
    assert ((y.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,C", [(16384, 513), (16400, 520), (16387, 1001), (20000, 1024), (16391, 2500), (16390, 4096)])
def test_many_rows_that_are_not_kept(dev, R, C, dtype):
    import torch
    from paper_1802_06058_amd import vgc
    gen = torch.Generator(device=dev).manual_seed(R + C)
    randn = lambda *s: torch.randn(s, generator=gen, device=dev)
    x = (randn(R, C) * randn(R, 1).exp() + 3 * randn(R, 1)).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    gamma, beta = 1 + 0.2 * randn(C), randn(C)
    y = torch.full((R * C + 32,), 7.0, dtype=x.dtype, device=dev)
    mean, rstd = torch.full((R + 8,), 7.0, device=dev), torch.full((R + 8,), 7.0, device=dev)
    vgc.layer_norm(x, gamma, beta, 1e-5, y[:R * C].view(R, C), mean, rstd)
    _check(x, gamma, beta, 1e-5, y[:R * C].view(R, C), mean[:R], rstd[:R])
    assert (y[R * C:] == 7).all() and (mean[R:] == 7).all() and (rstd[R:] == 7).all()


@pytest.mark.parametrize("R,C,dtype,kept", [(65536 + 3, 8200, "bf16", False), (65536 + 3, 8200, "bf16", True), (2 * 65536 + 1, 8193, "f32", False), (2 * 65536 + 1, 8193, "f32", True),
                                            (1 << 22, 8194, "bf16", False)])
def test_many_long_rows(dev, R, C, dtype, kept):
    """Rows that a workgroup reads three times, more of them than a launch has workgroups; 2^22 of 1024 threads would be more than one can have."""
    import torch
    from oracle import operators as O
    from paper_1802_06058_amd import vgc
    t, size, nb = (torch.bfloat16, 2, (C + 31) // 32) if dtype == "bf16" else (torch.float32, 4, (C + 31) // 32)
    torch.cuda.empty_cache()
    need = R * (C * (2 * size + kept) + 8) + (8 << 30)
    if torch.cuda.mem_get_info()[0] < need:
        pytest.skip(f"needs {need >> 30} GiB of GPU memory")
    gen = torch.Generator(device=dev).manual_seed(R)
    x = torch.empty(R, C, dtype=t, device=dev)
    for r in range(0, R, 1 << 16):                   # the rows of a later part are a multiple of the first one's, and have another mean
        if r == 0:
            some = torch.randn(1 << 16, C, generator=gen, device=dev)
        n = min(1 << 16, R - r)
        torch.add(some[:n], (r >> 16) % 5, out=x[r:r + n]) if t is torch.float32 else x[r:r + n].copy_(some[:n] + (r >> 16) % 5)
    gamma, beta = 1 + 0.2 * torch.randn(C, generator=gen, device=dev), torch.randn(C, generator=gen, device=dev)
    del some
    y, mean, rstd = torch.empty_like(x), torch.full((R + 8,), -7.0, device=dev), torch.full((R + 8,), -7.0, device=dev)
    act8 = (torch.empty(R, C, dtype=torch.int8, device=dev), torch.empty(R, nb, dtype=torch.uint8, device=dev)) if kept else None
    vgc.layer_norm(x, gamma, beta, 1e-5, y, mean, rstd, act8)
    assert (mean[R:] == -7).all() and (rstd[R:] == -7).all() and (rstd[:R] > 0).all()
    rows = torch.tensor(sorted({0, 1, 65535, 65536, 65537, R // 2, R - 2, R - 1}), device=dev)
    _check(x[rows], gamma, beta, 1e-5, y[rows], mean[rows], rstd[rows])
    if kept:
        h = (x[rows].double() - mean[rows].double()[:, None]) * rstd[rows].double()[:, None]
        q, e = act8[0][rows].cpu().numpy(), act8[1][rows].cpu().numpy()
        unit = torch.from_numpy(O.act8_decode(q * 0 + 1, e)).to(dev)
        assert ((torch.from_numpy(O.act8_decode(q, e)).to(dev) - h).abs() <= unit / 2 + 4 * U * (h.abs() + rstd[rows].double()[:, None] * x[rows].double().abs())).all()
