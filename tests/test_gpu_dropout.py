"""Dropout from a counter against the oracle: the mask exactly, the values to their roundings (one of the factor, one of the product, one of the sum with the
residual, one of the result's type)."""
import numpy as np
import pytest

from oracle import blocks as O
import block_checks as T

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    return T.device()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,C,p,residual", [(1, 1, 0.5, True), (1, 7, 0.5, False), (3, 8, 0.1, True), (5, 9, 0.9, True), (300, 3, 0.25, False), (128, 1000, 0.5, False), (77, 1001, 0.1, True),
                                            (1, 100003, 0.3, True), (1023, 33, 0.0, True), (40, 40, 1.0, True), (40, 41, 1.0, False), (2050, 515, 2.0 ** -16, False), (9, 4096, 1 - 2.0 ** -16, True),
                                            (4099, 1030, 0.1, True)])
def test_dropout(dev, R, C, p, residual, dtype):
    import torch
    from paper_1802_06058_amd import vgc
    gen = np.random.default_rng(R + C)
    x = T.to(gen.standard_normal((R, C)) + 3, dtype, dev)
    r = T.to(gen.standard_normal((R, C)), dtype, dev) if residual else None
    state = T.rng_state(dev)
    y, behind = T.guarded(R * C, x.dtype, dev)
    vgc.dropout(x, p, state if p > 0 else None, y.view(R, C), r)
    f = O.keep_factor(R, C, p, *state.tolist())
    want = T.back(x) * f
    tol = 3 * T.U * np.abs(want)
    if residual:
        want = want + T.back(r)
        tol = tol + T.U * np.abs(want)
    tol = tol + (T.half_unit(dtype) * np.abs(want) * (1 + 8 * T.U) if dtype == "bf16" else 0)
    got = T.back(y).reshape(R, C)
    assert (np.abs(got - want) <= tol).all() and T.untouched(behind)
    if not residual:
        assert ((got == 0) == (f == 0)).all()
    same = x.clone()                                                 # in place, and onto the residual
    vgc.dropout(same, p, state, same, r)
    assert torch.equal(same.view(-1), y)
    if residual:
        onto = r.clone()
        vgc.dropout(x, p, state, onto, onto)
        assert torch.equal(onto.view(-1), y)


def test_the_backward_pass_draws_the_same_mask_and_another_call_another(dev):
    import torch
    from paper_1802_06058_amd import vgc
    x = torch.ones(300, 257, device=dev)
    y, dx, z = (torch.empty_like(x) for _ in range(3))
    vgc.dropout(x, 0.3, T.rng_state(dev), y)
    vgc.dropout(x, 0.3, T.rng_state(dev), dx)
    vgc.dropout(x, 0.3, T.rng_state(dev, call=6), z)
    assert torch.equal(y, dx) and not torch.equal(y, z)
    assert abs(float((z == 0).float().mean()) - 0.3) < 0.01


def test_what_is_dropped_does_not_matter(dev):
    import torch
    from paper_1802_06058_amd import vgc
    state = T.rng_state(dev)
    f = torch.from_numpy(O.keep_factor(50, 100, 0.5, *state.tolist())).to(dev)
    for bad in (float("nan"), float("inf"), float("-inf")):
        for dt in (torch.float32, torch.bfloat16):
            x = torch.where(f == 0, bad, 1.0).to(dt)
            y = torch.empty_like(x)
            vgc.dropout(x, 0.5, state, y)
            assert torch.equal(y, f.to(dt))


def test_unaligned_rows_and_another_stream(dev):
    import torch
    from paper_1802_06058_amd import vgc
    state = T.rng_state(dev)
    base = torch.randn(1 + 20 * 37, device=dev).to(torch.bfloat16)
    x = base[1:].view(20, 37)
    want = torch.empty(20, 37, device=dev, dtype=torch.bfloat16)
    vgc.dropout(x, 0.2, state, want)
    out = torch.empty(3 + 20 * 37, device=dev, dtype=torch.bfloat16)[3:].view(20, 37)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        vgc.dropout(x, 0.2, state, out)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, want)


def test_a_recorded_call_draws_anew_when_its_state_changes(dev):
    import torch
    from paper_1802_06058_amd import vgc
    x, state = torch.randn(64, 520, device=dev), T.rng_state(dev)
    y, want = torch.empty_like(x), torch.empty_like(x)
    vgc.dropout(x, 0.4, state, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vgc.dropout(x, 0.4, state, y)
    seen = []
    for call in (1, 2, 1, 9):
        state[1] = call
        graph.replay()
        vgc.dropout(x, 0.4, T.rng_state(dev, call=call), want)
        torch.cuda.synchronize()
        assert torch.equal(y, want)
        seen.append(y.clone())
    assert torch.equal(seen[0], seen[2]) and not torch.equal(seen[0], seen[1])


def test_tensors_of_another_device_than_the_current_one_are_refused(dev, monkeypatch):
    """(Told from the device's number: there is one here.)"""
    import torch
    from paper_1802_06058_amd import vgc
    x, y = torch.randn(4, 8, device=dev), torch.full((4, 8), 7.0, device=dev)
    W, ws, f = torch.randn(8, 8, device=dev), torch.empty(1 << 20, dtype=torch.uint8, device=dev), torch.ones(8, device=dev)
    mean = torch.ones(4, 2, device=dev)
    v, o = x.view(4, 1, 8), y.view(4, 1, 8)
    with monkeypatch.context() as m:
        m.setattr(torch.cuda, "current_device", lambda: 1)
        for call in (lambda: vgc.dropout(x, 0.5, T.rng_state(dev), y), lambda: vgc.linear(x, W, y, workspace=ws), lambda: vgc.linear_backward(v, None, W, 0, 1.0, o, workspace=ws),
                     lambda: vgc.group_norm(v, f, f, 1e-5, 0, o, mean, mean, ws), lambda: vgc.group_norm_backward(v, v, mean, mean, f, f, 0, 1.0, o, f, f, workspace=ws)):
            with pytest.raises(vgc.VgcError, match="current device"):
                call()
    assert (y == 7).all()
