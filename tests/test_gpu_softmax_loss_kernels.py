"""The softmax loss's kernels that only larger problems reach, entry by entry against 64 bits, and the size rules that lead to them.

Tolerances are those of test_gpu_softmax_loss.py: a logit has H roundings of 2^-23 of the magnitudes summed, an exponential the relative error of
its argument, D is rounded to 2^-8 for dX and to 2^-17 for g and s, and sums have as many roundings as terms."""
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


def _inputs(dev, B, P, H, V, dtype, seed=0, masked=0.2):
    import torch
    gen = torch.Generator(device=dev).manual_seed(seed + 7 * B + 11 * P + 13 * H + V)
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    rand = lambda *s: torch.rand(s, generator=gen, device=dev)
    W = (torch.randn(V, H, generator=gen, device=dev) / H ** 0.5).to(t)
    target = (V * rand(B, P)).long().clamp_(max=V - 1)
    X = (torch.randn(B, P, H, generator=gen, device=dev) + 12 * rand(B, P, 1) * W[target].float()).to(t)
    target[rand(B, P) < masked] = -1
    target[0, 0] = V - 1
    return X, W, target


def _calls(X, W, target, weight, want_dx=True, want_s=True):
    """Both calls; every output and the workspace lie before guards that have to stay."""
    import torch
    from paper_1802_06058_amd import vgc
    B, P, H = X.shape
    V, N, dev = W.shape[0], B * P, X.device
    code = vgc.BF16 if X.dtype == torch.bfloat16 else vgc.F32
    guarded = lambda n, t=torch.float32: torch.full((n + 64,), 7.0, dtype=t, device=dev)
    loss, lse, dX, s, g = guarded(N), guarded(N), guarded(N * H, X.dtype), guarded(V * H), guarded(V * H)
    n1, n2 = vgc.softmax_loss_workspace_bytes(code, N, H, V), vgc.softmax_loss_backward_workspace_bytes(code, B, P, H, V)
    ws = torch.full((max(n1, n2) + 64,), 0xFF, dtype=torch.uint8, device=dev)
    vgc.softmax_loss(X, W, target, loss, lse, ws[:n1])
    assert (ws[n1:] == 0xFF).all()
    ws.fill_(0xFF)
    vgc.softmax_loss_backward(X, W, target, lse, weight, 1.0 / B, dX[:N * H].view(B, P, H) if want_dx else None, s if want_s else None,
                              g if want_s else None, ws[:n2])
    for t, n in ((loss, N), (lse, N), (dX, N * H), (s, V * H), (g, V * H)):
        assert (t[n:] == 7).all()
    assert (ws[n2:] == 0xFF).all()
    return loss[:N], lse[:N], dX[:N * H].view(B, P, H), s[:V * H].view(V, H), g[:V * H].view(V, H)


def _check(X, W, target, weight, got, sums=True):
    """Every entry, a sample at a time (samples of one position: all of them)."""
    import torch
    B, P, H = X.shape
    V, bf16 = W.shape[0], X.dtype == torch.bfloat16
    loss, lse, dX, s, g = got
    w, c = W.double(), 1.0 / B
    aw, wt = w.abs(), w.t().contiguous()
    awt = aw.t().contiguous()
    zero = torch.zeros(V, H, dtype=torch.float64, device=X.device) if sums else None
    gw, sw, eg, es = (zero.clone() for _ in range(4)) if sums else [None] * 4
    lse = lse.double().view(B, P)
    for z0 in range(0, B, B if P == 1 else 1):
        z1 = B if P == 1 else z0 + 1
        x, t, l = X[z0:z1].double().reshape(-1, H), target[z0:z1].reshape(-1), lse[z0:z1].reshape(-1, 1)
        z, ez = x @ wt, (H + 8) * E * (x.abs() @ awt)
        wl = torch.logsumexp(z, 1)
        el = ez.amax(1) + 16 * E * (1 + wl.abs()) + (V // 16 + 64) * E
        assert ((l[:, 0] - wl).abs() <= el).all()
        at = t.clamp(min=0)[:, None]
        want = torch.where(t < 0, 0.0, wl - z.gather(1, at)[:, 0])
        tol = torch.where(t < 0, 0.0, el + ez.gather(1, at)[:, 0] + 4 * E * (wl.abs() + el))
        assert ((loss.double().view(B, P)[z0:z1].reshape(-1) - want).abs() <= tol).all()
        asked = (t >= 0)[:, None]
        wz = torch.where(asked, torch.ones_like(l) if weight is None else weight[z0:z1].double().reshape(-1, 1), 0.0)
        p = (z - l).exp()
        eD = wz.abs() * (p * (ez + 4 * E * (1 + z.abs() + l.abs())) + 2 * E)
        D = wz * p.scatter_add(1, at, torch.full_like(l, -1.0))
        aD = D.abs()
        dXw = D @ w
        edx = (eD + (2.0 ** -8 if bf16 else 4 * E) * aD) @ aw + (V + 8) * E * (aD @ aw) + (2.0 ** -8 if bf16 else E) * dXw.abs()
        assert ((dX[z0:z1].double().reshape(-1, H) - dXw).abs() <= edx).all()
        if not sums:
            continue
        x = torch.where(asked, x, 0.0)
        e = eD + ((2.0 ** -17 if bf16 else 4 * E) + (P + 8) * E) * aD
        if P == 1:
            gw += D.t().contiguous() @ x
            sw += D.square().t().contiguous() @ x.square()
            eg += e.t().contiguous() @ x.abs() + (B + 8) * E * (aD.t().contiguous() @ x.abs())
            es += (2 * aD * e + e * e).t().contiguous() @ x.square() + (B + 8) * E * sw
        else:
            G, eG = D.t().contiguous() @ x, e.t().contiguous() @ x.abs()
            gw += G
            sw += G * G
            eg += eG + (B + 8) * E * G.abs()
            es += 2 * G.abs() * eG + eG * eG + (B + 8) * E * G * G
    if sums:
        assert ((g.double() - c * gw).abs() <= c * eg).all()
        assert ((s.double() - c * c * sw).abs() <= c * c * es).all()


def _tiles(V, N, bm, bn):
    return -(-V // bm) * (-(-N // bn))


@pytest.mark.parametrize("B,P,H,V", [(100, 1, 24, 60003), (100, 1, 9, 60003), (2, 160, 40, 20500), (2, 150, 17, 20501)])
def test_small_tiles_of_the_logits(dev, B, P, H, V):
    """128 x 128 tiles: bfloat16, more than 64 rows, enough of these tiles, and no more than 128 rows or too few of the large ones."""
    import torch
    for n in (B * P, B * (P if P == 1 else -(-P // 16) * 16)):
        assert n > 64 and _tiles(V, n, 128, 128) >= 320 and (n <= 128 or _tiles(V, n, 256, 256) < 192)
    X, W, target = _inputs(dev, B, P, H, V, "bf16")
    weight = torch.full((B, P), 1.0 / P, device=dev)
    _check(X, W, target, weight, _calls(X, W, target, weight))


def _dx_splits(B, P, H, V):
    """The number of parts of dX's sum that the workspace has room for, from its size: what tells the two tilings of a bfloat16 dX apart."""
    from paper_1802_06058_amd import vgc
    up = lambda x, m: -(-x // m) * m
    N, Lq, Kp = B * P, B * up(P, 16), up(H, 8)
    planes = 3 if P < 512 or N * V * H <= 9e9 else 2
    most = (2 << 30) // (2 * Kp + 2 * planes * Lq) // 256 * 256
    piece = min(up(-(-V // -(-V // most)), 256), V)
    rows = 0 if H % 8 == 0 else 2 * Kp
    parts = up(N * rows, 256) + up(2 * H * Lq, 256) + up(piece * rows, 256) + up(2 * piece * planes * Lq, 256)
    left = vgc.softmax_loss_backward_workspace_bytes(vgc.BF16, B, P, H, V) - parts
    assert 0 <= left % (4 * N * H) < 4 * (B + N) + 4096, "the workspace is laid out differently"
    return left // (4 * N * H), -(-V // piece)


@pytest.mark.parametrize("B,P,H,V,splits,pieces", [(4, 300, 1500, 30000, 16, 1), (4, 1024, 64, 200001, 16, 2)])
def test_large_tiles_of_the_input_gradient_in_parts(dev, B, P, H, V, splits, pieces):
    """256 x 256 tiles of dX, with remainders in both directions, its sum over the classes in parts (30 and 16 tiles: 16 parts make 256
    workgroups or the most there are; by 128 x 128 tiles there would be 8 parts of the first), and added to from piece to piece."""
    assert _dx_splits(B, P, H, V) == (splits, pieces)
    X, W, target = _inputs(dev, B, P, H, V, "bf16")
    _check(X, W, target, None, _calls(X, W, target, None))


@pytest.mark.parametrize("dtype,B,P,H,V", [("bf16", 3, 40, 515, 60001), ("bf16", 5, 130, 515, 60001), ("bf16", 1, 600, 515, 60001), ("bf16", 20, 1, 701, 50001), ("f32", 3, 40, 515, 60001), ("bf16", 33, 1, 701, 50001),
                                            ("bf16", 70, 1, 72, 90001)])
def test_sums_beyond_the_caches(dev, dtype, B, P, H, V):
    """g and s of more than 192 MiB (samples of one position: 256) are stored past the caches: from three planes of D, from two, by the FC
    form from planes (33 samples, and 70 with sums that the caches hold) and from floats, and from float32 planes."""
    import torch
    assert V * H * 8 > (256 << 20 if P == 1 else 192 << 20) or H == 72
    if dtype == "bf16" and P > 1:
        assert (P >= 512 and B * P * V * H > 9e9) == (B == 1)
    X, W, target = _inputs(dev, B, P, H, V, dtype)
    weight = torch.rand(B, P, device=dev)
    _check(X, W, target, weight, _calls(X, W, target, weight))


@pytest.mark.parametrize("B,P,H,V", [(4, 100, 512, 8000), (2, 20, 129, 3001), (9, 33, 65, 2500), (3, 7, 264, 900), (64, 1, 512, 3001), (20, 1, 1001, 9000), (256, 1, 40, 1001), (4, 1024, 64, 200001),
                                     (4, 300, 1500, 30000)])
@pytest.mark.parametrize("sums", [False, True])
def test_dx_is_rounded_once(dev, B, P, H, V, sums):
    """bfloat16: rows that miss their classes by anything, so that the target's entry of D is what dX mostly consists of.  Besides the rounding of
    dX itself, whose size is that of the exact dX's rounding (to 1 % in the root mean square over thousands of entries), every other
    entry of D may be off by 2^-9 of itself, each by its own: in the root mean square at most 2^-9 sqrt(sum of (D W)^2); 2e-5 covers the float32
    sums and exponentials.  (With the target's entry rounded too: 1.1 to 1.3 times the rounding.)"""
    import torch
    X, W, target = _inputs(dev, B, P, H, V, "bf16", seed=5)
    weight = torch.full((B, P), 1.0 / P, device=dev)
    _, lse, dX, _, _ = _calls(X, W, target, weight, want_s=sums)
    w = W.double()
    wt, want, others = w.t().contiguous(), [], 0.0
    for z in range(0, B, B if P == 1 else 1):
        n = B if P == 1 else 1
        x, t, l = X[z:z + n].double().reshape(-1, H), target[z:z + n].reshape(-1), lse.double().view(B, P)[z:z + n].reshape(-1, 1)
        D = torch.where((t >= 0)[:, None], weight[z:z + n].double().reshape(-1, 1), 0.0) * (x @ wt - l).exp_()
        p = D.scatter(1, t.clamp(min=0)[:, None], 0.0)
        others += float((p.square() @ w.square()).sum())
        D = torch.where((t >= 0)[:, None], D.scatter_add(1, t.clamp(min=0)[:, None], -weight[z:z + n].double().reshape(-1, 1)), 0.0)
        want.append(D @ w)
    want = torch.cat(want)
    size, got = want.norm(), dX.double().reshape(-1, H)
    rounding = (want.to(torch.bfloat16).double() - want).norm() / size
    assert float((got - want).norm() / size) <= float(1.01 * rounding + 2.0 ** -9 * others ** 0.5 / size) + 2e-5


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,P,H,V", [(20, 1, 72, 50), (70, 1, 72, 3000), (3, 7, 33, 40), (4, 100, 64, 6000), (300, 1, 520, 9000), (67, 1, 520, 13001)])
@pytest.mark.parametrize("where", ["x", "weight"])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_values_that_are_not_finite_stay_with_their_row(dev, where, value, B, P, H, V, dtype):
    """In a row that is asked for they reach its own results (a weight: not its loss) and the sums; the other rows keep their bits, and where
    the value is a weight, which the rounding of its sample's other rows goes by, stay finite."""
    import torch
    X, W, target = _inputs(dev, B, P, H, V, dtype, masked=0.0)
    weight = torch.rand(B, P, device=dev) + 0.5
    clean = _calls(X, W, target, weight)
    z, p = B // 2, P // 2
    (X if where == "x" else weight.unsqueeze(-1))[z, p, 0] = value
    loss, lse, dX, s, g = _calls(X, W, target, weight)
    hit = torch.zeros(B, P, dtype=torch.bool, device=dev)
    hit[z, p] = True
    for a, b in ((loss, clean[0]), (lse, clean[1])):
        a, b = a.view(B, P), b.view(B, P)
        assert torch.equal(a[~hit], b[~hit]) and (torch.equal(a, b) if where == "weight" else not torch.isfinite(a[hit]).any())
    assert not torch.isfinite(dX[hit]).any() and torch.isfinite(dX[~hit]).all()
    others = ~hit if where == "x" else ~hit & (torch.arange(B, device=dev) != z)[:, None]
    assert torch.equal(dX[others], clean[2][others])
    assert not torch.isfinite(s).any() and not torch.isfinite(g).any()


@pytest.mark.parametrize("N,H,V", [(2048, 120, 20000), (2048, 2048, 20000)])
def test_logits_of_floats_are_not_too_small(dev, N, H, V):
    """float32 by planes, rows whose logit of one class, 16, is a sum of products that point one way.  Planes that were cut off instead of rounded
    would leave each product 2^-24.3 of itself too small on average, by the pairs that are not formed, and the logits 7.5e-7; rounded ones err to
    either side.  Half of that is the bound of the mean: chance leaves 2e-6 / sqrt(N) of it at most, 4e-8.  In the root mean square: sums of 32
    from zero and H / 32 of them rounded by 2^-24 of 16 at most, 2.8e-7 in the root mean square each, beside logsumexp's own rounding."""
    import torch
    from paper_1802_06058_amd import vgc
    gen = torch.Generator(device=dev).manual_seed(H)
    W = torch.randn(V, H, generator=gen, device=dev) / H ** 0.5
    t = torch.randint(0, V, (N,), generator=gen, device=dev)
    X = torch.randn(N, H, generator=gen, device=dev) + 16 * W[t]
    want = torch.logsumexp(X.double() @ W.double().t().contiguous(), 1)
    loss, lse = torch.empty(N, device=dev), torch.empty(N, device=dev)
    ws = torch.empty(vgc.softmax_loss_workspace_bytes(vgc.F32, N, H, V), dtype=torch.uint8, device=dev)
    vgc.softmax_loss(X, W, t, loss, lse, ws)
    off = lse.double() - want
    assert abs(float(off.mean())) <= 3.7e-7
    assert float(off.square().mean().sqrt()) <= 2.8e-7 * (H / 32 + 9) ** 0.5


@pytest.mark.parametrize("N,H,V", [(10, 1703, 21092), (60, 2048, 8000), (128, 2048, 20000)])
def test_logits_of_few_rows(dev, N, H, V):
    """bfloat16, logits of 16 in a row: in the root mean square lse is off by H / 128 roundings, each half a step of its sum over sqrt 3 (2^-20.8 above
    16, half of it below), and a few more of logsumexp.  (16 k at a time, as the instructions add them, there are eight times as many: 1.3 to 2 times this bound.)"""
    import torch
    from paper_1802_06058_amd import vgc
    gen = torch.Generator(device=dev).manual_seed(N)
    W = (torch.randn(V, H, generator=gen, device=dev) / H ** 0.5).to(torch.bfloat16)
    t = torch.randint(0, V, (N,), generator=gen, device=dev)
    X = (torch.randn(N, H, generator=gen, device=dev) + 16 * W[t].float()).to(torch.bfloat16)
    want = torch.logsumexp(X.double() @ W.double().t().contiguous(), 1)
    loss, lse = torch.empty(N, device=dev), torch.empty(N, device=dev)
    ws = torch.empty(vgc.softmax_loss_workspace_bytes(vgc.BF16, N, H, V), dtype=torch.uint8, device=dev)
    vgc.softmax_loss(X, W, t, loss, lse, ws)
    assert float((lse.double() - want).square().mean().sqrt()) <= 2.0 ** -20.9 * (H / 128 + 2) ** 0.5


def _s_off(dev, B, P, H, V, dtype="bf16"):
    """How far s is off in the root mean square, for rows that lean to their classes by anything and samples that weight their positions alike."""
    import torch
    X, W, target = _inputs(dev, B, P, H, V, dtype, seed=9)
    weight = torch.full((B, P), 1.0 / P, device=dev)
    _, lse, _, s, _ = _calls(X, W, target, weight)
    w, want = W.double().t().contiguous(), torch.zeros(V, H, dtype=torch.float64, device=dev)
    for z in range(B):
        x, t = X[z].double(), target[z]
        D = (x @ w - lse.double().view(B, P)[z][:, None]).exp_()
        D = D.scatter_add_(1, t.clamp(min=0)[:, None], torch.full((P, 1), -1.0, dtype=torch.float64, device=dev)) * torch.where(t >= 0, weight[z].double(), 0.0)[:, None]
        want += (D.t().contiguous() @ torch.where((t >= 0)[:, None], x, 0.0)).square()
    return float((s.double() * B * B - want).norm() / want.norm())


@pytest.mark.parametrize("B,H,V", [(33, 192, 40001), (64, 105, 60505), (40, 704, 14413), (128, 512, 20011)])
def test_sums_of_samples_of_one_position_keep_all_digits(dev, B, H, V):
    """bfloat16, outputs large enough for the FC form from planes.  D is a float32 there: its target entry, p - 1, is off by p (1 - p) times the logit's
    error, 1.5e-6 at most, of either sign and in the rows between missed and certain; the products, their sum and the scale round half a dozen
    times at 2^-24 at most.  1e-6 covers both.  (D and its square in 16 bits: 1.3e-6 to 2.0e-6.)"""
    assert B >= 32 and V * H >= 6 << 20
    assert _s_off(dev, B, 1, H, V) <= 1e-6


@pytest.mark.parametrize("B,P,H,V", [(16, 48, 512, 40000), (2, 300, 512, 40000), (4, 256, 256, 50001), (2, 20, 128, 9000)])
def test_sums_of_few_positions_keep_all_digits(dev, B, P, H, V):
    """bfloat16, samples of fewer than 512 positions: as above, a class's gradient being that of a few of the sample's positions.  (D in 16
    bits: 1.3e-6 to 2.7e-6.)"""
    assert P < 512
    assert _s_off(dev, B, P, H, V) <= 1e-6
