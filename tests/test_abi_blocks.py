"""Argument checks of the linear layer's, dropout's and group norm's entry points: refused on the host, before anything touches a GPU (the
pointers here are never dereferenced)."""
import pytest

from paper_1802_06058_amd import vgc

NULL, SIZE, DTYPE, ALIGN, PARAM = -1, -2, -4, -5, -6
P = 1 << 20                                          # an aligned address
NAN = float("nan")


def _codes(good, changes, call):
    for change, want in changes:
        args = dict(good, **change)
        assert call(*args.values()) == want, change
        assert vgc.load().vgc_last_error()


def test_dropout():
    good = dict(dtype=0, x=P, residual=None, R=4, C=40, p=0.5, rng=P, y=P, stream=None)
    _codes(good, [(dict(dtype=2), DTYPE), (dict(x=None), NULL), (dict(y=None), NULL), (dict(rng=None), NULL), (dict(R=0), SIZE), (dict(C=0), SIZE), (dict(R=1 << 31), SIZE),
                  (dict(R=1 << 40), SIZE), (dict(C=1 << 31), SIZE), (dict(x=P + 2), ALIGN), (dict(residual=P + 1), ALIGN), (dict(y=P + 3), ALIGN), (dict(rng=P + 4), ALIGN),
                  (dict(p=-0.01), PARAM), (dict(p=1.01), PARAM), (dict(p=NAN), PARAM), (dict(p=1.0, rng=None), NULL)], vgc.load().vgc_dropout)


def test_linear():
    need = vgc.linear_workspace_bytes(vgc.F32, 4, 3, 40)              # (a k that is laid out in planes; 24 needs none)
    assert need > 0 and vgc.linear_workspace_bytes(vgc.F32, 4, 24, 40) == 0
    for bad in [(2, 4, 24, 40), (0, 0, 24, 40), (0, 4, 0, 40), (0, 4, 24, 0), (0, (1 << 20) + 1, 24, 40), (0, 4, 1 << 20, 1 << 11), (0, 4, (1 << 20) + 8, 8), (0, 1 << 20, 8, 1 << 15)]:
        assert vgc.linear_workspace_bytes(*bad) == 0, bad
    good = dict(dtype=0, X=P, W=P, bias=None, act=1, p=0.5, rng=P, residual=None, N=4, K=3, C=40, z=None, y=P, ws=P, nb=need, stream=None)
    _codes(good, [(dict(dtype=2), DTYPE), *[(dict([(k, None)]), NULL) for k in ("X", "W", "y", "rng", "ws")], *[(dict([(k, 0)]), SIZE) for k in ("N", "K", "C")],
                  (dict(N=(1 << 20) + 1), SIZE), (dict(K=1 << 15, C=(1 << 15) + 1), SIZE), (dict(X=P + 8), ALIGN), (dict(W=P + 4), ALIGN), (dict(bias=P + 2), ALIGN),
                  (dict(residual=P + 2), ALIGN), (dict(z=P + 1), ALIGN), (dict(y=P + 2), ALIGN), (dict(rng=P + 4), ALIGN), (dict(act=4), PARAM), (dict(act=-1), PARAM), (dict(p=1.5), PARAM),
                  (dict(p=NAN), PARAM), (dict(nb=need - 1), SIZE), (dict(ws=P + 8), ALIGN)], vgc.load().vgc_linear)


def test_linear_backward():
    need = vgc.linear_backward_workspace_bytes(vgc.BF16, 2, 3, 24, 40)
    assert need > 0 and vgc.linear_backward_workspace_bytes(vgc.BF16, 1 << 11, 1 << 10, 24, 40) == 0 and vgc.linear_backward_workspace_bytes(vgc.BF16, 2, 0, 24, 40) == 0
    good = dict(dtype=1, dy=P, z=P, W=P, act=2, p=0.5, rng=P, add=None, B=2, P=3, K=24, C=40, c=0.5, dz=P, dX=P, g=None, s=P, ws=P, nb=need, stream=None)
    _codes(good, [(dict(dtype=7), DTYPE), *[(dict([(k, None)]), NULL) for k in ("dy", "z", "W", "dz", "rng", "ws")], (dict(g=P, s=None), NULL), (dict(add=P, dX=None), NULL),
                  *[(dict([(k, 0)]), SIZE) for k in ("B", "P", "K", "C")], (dict(B=1 << 20, P=2), SIZE), (dict(W=P + 8), ALIGN), (dict(dz=P + 2), ALIGN), (dict(dy=P + 1), ALIGN),
                  (dict(add=P + 1), ALIGN), (dict(dX=P + 1), ALIGN), (dict(s=P + 2), ALIGN), (dict(act=9), PARAM), (dict(p=-1.0), PARAM), (dict(c=float("inf")), PARAM), (dict(nb=need - 1), SIZE),
                  (dict(ws=P + 4), ALIGN)], vgc.load().vgc_linear_backward)


def test_group_norm():
    lib = vgc.load()
    assert vgc.group_norm_workspace_bytes(vgc.F32, 2, 5000, 24, 4) > 0
    for bad in [(2, 2, 9, 24, 4), (0, 0, 9, 24, 4), (0, 2, 0, 24, 4), (0, 2, 9, 24, 0), (0, 2, 9, 24, 5), (0, 1 << 16, 1 << 15, 24, 4), (0, 2, 9, 1 << 21, 4)]:
        assert vgc.group_norm_workspace_bytes(*bad) == 0 and vgc.group_norm_backward_workspace_bytes(*bad) == 0, bad
    need = vgc.group_norm_workspace_bytes(vgc.F32, 2, 5000, 24, 4)
    good = dict(dtype=0, x=P, B=2, P=5000, C=24, G=4, gamma=P, beta=P, eps=1e-5, act=3, y=P, mean=P, rstd=P, ws=P, nb=need, stream=None)
    _codes(good, [(dict(dtype=2), DTYPE), *[(dict([(k, None)]), NULL) for k in ("x", "gamma", "beta", "y", "mean", "rstd", "ws")], *[(dict([(k, 0)]), SIZE) for k in ("B", "P", "C", "G")],
                  (dict(G=5), SIZE), (dict(G=48), SIZE), (dict(x=P + 2), ALIGN), (dict(rstd=P + 2), ALIGN), (dict(gamma=P + 1), ALIGN), (dict(act=4), PARAM), (dict(eps=-1e-6), PARAM),
                  (dict(eps=NAN), PARAM), (dict(nb=need - 1), SIZE), (dict(ws=P + 8), ALIGN)], lib.vgc_group_norm)
    need = vgc.group_norm_backward_workspace_bytes(vgc.BF16, 2, 9, 24, 4)
    good = dict(dtype=1, dy=P, x=P, mean=P, rstd=P, gamma=P, beta=P, act=1, B=2, P=9, C=24, G=4, c=0.5, dx=P, gg=None, sg=P, gb=None, sb=P, ws=P, nb=need, stream=None)
    _codes(good, [(dict(dtype=2), DTYPE), *[(dict([(k, None)]), NULL) for k in ("dy", "x", "mean", "rstd", "gamma", "beta", "dx", "sg", "sb", "ws")], (dict(G=7), SIZE), (dict(P=0), SIZE),
                  (dict(dy=P + 1), ALIGN), (dict(beta=P + 2), ALIGN), (dict(gb=P + 2), ALIGN), (dict(act=-1), PARAM), (dict(c=NAN), PARAM), (dict(nb=need - 1), SIZE)],
           lib.vgc_group_norm_backward)


def test_tensors_that_do_not_belong_together():
    """The binding, which knows sizes and types: host tensors, since nothing may be launched."""
    import torch
    t = torch.zeros
    x, rng = t(4, 24), t(2, dtype=torch.int64)
    with pytest.raises(vgc.VgcError, match="rng"):
        vgc.dropout(x, 0.5, t(2), t(4, 24))
    with pytest.raises(vgc.VgcError, match="y: need"):
        vgc.dropout(x, 0.5, rng, t(4, 23))
    with pytest.raises(vgc.VgcError, match="contiguous"):
        vgc.dropout(t(24, 4).t(), 0.5, rng, t(4, 24))
    with pytest.raises(vgc.VgcError, match="dtype"):
        vgc.dropout(x.half(), 0.5, rng, t(4, 24))
    with pytest.raises(vgc.VgcError, match="GPU|device|cpu"):
        vgc.dropout(x, 0.5, rng, t(4, 24))
    ws = torch.empty(1 << 20, dtype=torch.uint8)
    with pytest.raises(vgc.VgcError, match="does not take"):
        vgc.linear(x, t(25, 8), t(4, 8), workspace=ws)
    with pytest.raises(vgc.VgcError, match="W "):
        vgc.linear(x, t(24, 8, dtype=torch.bfloat16), t(4, 8), workspace=ws)
    with pytest.raises(vgc.VgcError, match="workspace"):
        vgc.linear(t(4, 3), t(3, 8), t(4, 8))                       # (3: laid out, which needs working memory)
    with pytest.raises(vgc.VgcError, match="bias"):
        vgc.linear(x, t(24, 8), t(4, 8), t(7), workspace=ws)
    with pytest.raises(vgc.VgcError, match="does not give"):
        vgc.linear_backward(t(2, 2, 8), None, t(24, 9), vgc.ACT_NONE, 1.0, t(2, 2, 8), workspace=ws)
    with pytest.raises(vgc.VgcError, match="dX"):
        vgc.linear_backward(t(2, 2, 8), None, t(24, 8), vgc.ACT_NONE, 1.0, t(2, 2, 8), t(2, 2, 23), workspace=ws)
    with pytest.raises(vgc.VgcError, match="positions"):
        vgc.group_norm(t(4, 8), t(8), t(8), 1e-5, vgc.ACT_NONE, t(4, 8), t(4, 2), t(4, 2), ws)
    with pytest.raises(vgc.VgcError, match="rstd"):
        vgc.group_norm(t(4, 3, 8), t(8), t(8), 1e-5, vgc.ACT_NONE, t(4, 3, 8), t(4, 2), t(4, 1), ws)
    with pytest.raises(vgc.VgcError, match="s_beta"):
        vgc.group_norm_backward(t(4, 3, 8), t(4, 3, 8), t(4, 2), t(4, 2), t(8), t(8), vgc.ACT_NONE, 1.0, t(4, 3, 8), t(8), t(7), workspace=ws)


def test_a_backward_pass_without_the_weight():
    """W is read for dX alone: without both the binding goes on (to the device check: these are host tensors), with dX it refuses."""
    import torch
    t = torch.zeros
    ws = torch.empty(1 << 20, dtype=torch.uint8)
    with pytest.raises(vgc.VgcError, match="GPU|device|cpu"):
        vgc.linear_backward(t(2, 2, 8), None, None, vgc.ACT_NONE, 1.0, t(2, 2, 8), s_bias=t(8), workspace=ws)
    with pytest.raises(vgc.VgcError, match="dX needs W"):
        vgc.linear_backward(t(2, 2, 8), None, None, vgc.ACT_NONE, 1.0, t(2, 2, 8), t(2, 2, 24), workspace=ws)
