"""Calls of the softmax loss that are larger than one launch of its kernels can be (2^32 threads)."""
import pytest

pytestmark = pytest.mark.gpu
E = 2.0 ** -23


@pytest.fixture(scope="module")
def dev():
    import torch
    from paper_1802_06058_amd import vgc
    assert torch.cuda.is_available()
    vgc.load()
    return torch.device("cuda:0")


def _room(nbytes):
    import torch
    torch.cuda.empty_cache()
    free = torch.cuda.mem_get_info()[0]
    if free < nbytes:
        pytest.skip(f"needs {nbytes >> 30} GiB of GPU memory, {free >> 30} free")


def test_a_loss_of_many_rows_and_classes(dev):
    """2^15 rows by 2^24 classes: 2^39 logits, 128 a thread.  Tolerance of test_gpu_softmax_loss.py, for lse's sum of a block's terms and of the blocks."""
    import torch
    from paper_1802_06058_amd import vgc
    N, H, V = 1 << 15, 8, 1 << 24
    nbytes = vgc.softmax_loss_workspace_bytes(vgc.BF16, N, H, V)
    assert nbytes < 40 << 30
    _room(nbytes + (8 << 30))
    gen = torch.Generator(device=dev).manual_seed(0)
    W = torch.randn(V, H, generator=gen, device=dev).to(torch.bfloat16)
    X = torch.randn(N, H, generator=gen, device=dev).to(torch.bfloat16)
    target = torch.randint(0, V, (N,), generator=gen, device=dev)
    target[0], target[-1], target[5] = 0, V - 1, -1
    loss, lse = torch.full((N + 8,), 7.0, device=dev), torch.full((N + 8,), 7.0, device=dev)
    vgc.softmax_loss(X, W, target, loss, lse, torch.empty(nbytes, dtype=torch.uint8, device=dev))
    assert (loss[N:] == 7).all() and (lse[N:] == 7).all() and torch.isfinite(lse).all() and float(loss[5]) == 0
    wt = W.double().t().contiguous()
    for row in (0, 5, 255, 256, 4097, 20001, N - 1):
        z = (X[row:row + 1].double() @ wt)[0]
        want, ez = torch.logsumexp(z, 0), (H + 8) * E * float((X[row].double().abs() * wt.abs().amax(1)).sum())
        tol = ez + 16 * E * (1 + float(want.abs())) + (128 + V // (128 * 16) + 64) * E
        assert float((lse[row].double() - want).abs()) <= tol
        if int(target[row]) >= 0:
            assert float((loss[row].double() - (want - z[target[row]])).abs()) <= 2 * tol
