"""The operators of a residual block around the statistic's layers, as measured cases.

What a worker computes between two weights whose sums `vgc.sqgrad` and `vgc.sqgrad_conv2d` form: a linear layer with its bias,
activation, dropout and residual in one call and the gradients that belong to it (`vgc.linear`, `vgc.linear_backward`), dropout
whose mask is drawn again instead of stored (`vgc.dropout`), and group norm with an activation over channels-last positions, which
unlike a batch's norm leaves every sample a gradient of its own (`vgc.group_norm`, `vgc.group_norm_backward`).  Bias, scale and shift
end in the two sums over the samples that the compression reads.

`own` chooses between the plain form in elementary 32-bit operations and the calls of the package.
"""
import math

import torch

own = False

EPS = 1e-5
ACTS = ("none", "relu", "gelu", "silu")


# ---------------------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------------------
def listed():
    return [
        # the first hidden layer of a 784-1000-1000-10 perceptron at batch 128: the call's own time counts
        dict(name="linear_f32_hidden", kind="linear", N=128, K=784, C=1000, dtype="f32", act="relu", keep=False, residual=False, p=0.0),
        # one token through a layer of 4096 channels: the weight is what has to be read
        dict(name="linear_bf16_token", kind="linear", N=1, K=4096, C=4096, dtype="bf16", act="gelu", keep=False, residual=True, p=0.0),
        # the first half of a feed-forward block on 16 sequences of 1024 positions; z is kept for the backward pass
        dict(name="linear_bf16_up", kind="linear", N=16384, K=2048, C=8192, dtype="bf16", act="gelu", keep=True, residual=False, p=0.0),
        # its second half, back onto the residual stream
        dict(name="linear_bf16_down", kind="linear", N=16384, K=8192, C=2048, dtype="bf16", act="none", keep=False, residual=True, p=0.1),
        # the backward pass of a perceptron's second hidden layer, every sample one position
        dict(name="linear_backward_f32_hidden", kind="linear_backward", B=128, P=1, K=1000, C=1000, dtype="f32", act="relu", add=False, p=0.0),
        # the backward pass of the third case; the gradient that came past the block is added to dX
        dict(name="linear_backward_bf16_up", kind="linear_backward", B=16, P=1024, K=2048, C=8192, dtype="bf16", act="gelu", add=True, p=0.0),
        # a perceptron's hidden units at batch 128
        dict(name="dropout_f32_hidden", kind="dropout", R=128, C=1000, dtype="f32", residual=False, p=0.5),
        # 16 sequences of 1024 positions back onto a residual stream of 4096 channels
        dict(name="dropout_bf16_residual", kind="dropout", R=16384, C=4096, dtype="bf16", residual=True, p=0.1),
        # a ResNet-50's last stage at batch 32: 7 x 7 positions of 2048 channels
        dict(name="group_norm_f32_49", kind="group_norm", B=32, P=49, C=2048, G=32, dtype="f32", act="relu"),
        # the widest activations of a VGG-16 at batch 64: two channels a group
        dict(name="group_norm_bf16_vgg_conv1", kind="group_norm", B=64, P=224 * 224, C=64, G=32, dtype="bf16", act="relu"),
        # a ResNet-50's first stage at batch 32: 56 x 56 positions of 256 channels
        dict(name="group_norm_backward_f32_3136", kind="group_norm_backward", B=32, P=3136, C=256, G=32, dtype="f32", act="relu"),
        # a VGG-16's fourth stage at batch 64: 28 x 28 positions of 512 channels
        dict(name="group_norm_backward_bf16_784", kind="group_norm_backward", B=64, P=784, C=512, G=32, dtype="bf16", act="silu"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear_backward", "linear_backward", "dropout", "group_norm", "group_norm_backward"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    wide = 2 if dtype == "f32" else 1
    if kind == "dropout":
        C = _log(rng, 3, 16384)
        R = _log(rng, 1, max(1, 16384 * 4096 // (C * wide)))
        return dict(kind=kind, R=R, C=C, dtype=dtype, residual=rng.random() < 0.5, p=rng.choice([0.0, 0.1, 0.25, 0.5, 0.9]))
    act = rng.choice(ACTS)
    if kind in ("group_norm", "group_norm_backward"):
        G = rng.choice([1, 2, 3, 8, 16, 32, 32])
        C = G * _log(rng, 1 if G >= 8 else 8, max(8, min(256, 4096 // G)))
        most = 64 * 224 * 224 * 64 // wide // (4 if kind == "group_norm_backward" else 1)
        P = _log(rng, max(1, 16 * G // C), 224 * 224)
        return dict(kind=kind, B=_log(rng, 1, max(1, min(64, most // (P * C)))), P=min(P, most // C), C=C, G=G, dtype=dtype, act=act)
    step = rng.choice([1, 1, 8, 64])                                 # odd sizes, whole pieces of 16 bytes, whole tiles

    def length(lo, hi):
        return min(hi, (_log(rng, lo, hi) // step | 1) * step)

    most = 16384 * 2048 * 8192 // (8 if dtype == "f32" else 1)
    K, C = length(16, 8192), length(16, 8192)
    N = rng.choice([_log(rng, 1, 64), _log(rng, 1, 16384), _log(rng, 64, 16384)])
    N = max(1, min(N, most // (K * C)))
    p = rng.choice([0.0, 0.0, 0.1, 0.5])
    if kind == "linear":
        return dict(kind=kind, N=N, K=K, C=C, dtype=dtype, act=act, keep=rng.random() < 0.5, residual=rng.random() < 0.5, p=p)
    P = rng.choice([1, _log(rng, 1, N)])
    return dict(kind=kind, B=max(1, N // P), P=P, K=K, C=C, dtype=dtype, act=act, add=rng.random() < 0.5, p=p)


# ---------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------
def _randn(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _empty(*shape, dtype=torch.float32):
    return torch.empty(shape, device="cuda", dtype=dtype)


def _weight(gen, K, C, dt):
    return (_randn(gen, K, C) / math.sqrt(K)).to(dt)


def _rng(seed):
    """The generator's state: a key, and the number of the call under it."""
    return torch.tensor([(seed * 0x9E3779B97F4A7C15 + 0x1234567) & 0x7FFFFFFFFFFFFFFF, seed + (5 << 32)], device="cuda")


def prepare(case, seed):
    gen, kind, dt = torch.Generator(device="cuda").manual_seed(seed), case["kind"], _dtype(case)
    st = dict(case=case)
    if case.get("p", 0.0) > 0 or kind == "dropout":
        st.update(rng=_rng(seed))
    if kind == "dropout":
        R, C = case["R"], case["C"]
        st.update(x=_randn(gen, R, C).to(dt), y=_empty(R, C, dtype=dt))
        if case["residual"]:
            st.update(residual=_randn(gen, R, C).to(dt))
    elif kind == "linear":
        N, K, C = case["N"], case["K"], case["C"]
        st.update(X=_randn(gen, N, K).to(dt), W=_weight(gen, K, C, dt), bias=0.1 * _randn(gen, C), y=_empty(N, C, dtype=dt))
        if case["keep"]:
            st.update(z=_empty(N, C, dtype=dt))
        if case["residual"]:
            st.update(residual=_randn(gen, N, C).to(dt))
    elif kind == "linear_backward":
        B, P, K, C = case["B"], case["P"], case["K"], case["C"]
        st.update(W=_weight(gen, K, C, dt), dy=(1e-3 * _randn(gen, B, P, C)).to(dt), dz=_empty(B, P, C, dtype=dt), dX=_empty(B, P, K, dtype=dt),
                  s_bias=_empty(C), g_bias=_empty(C))
        if case["act"] != "none":
            st.update(z=_randn(gen, B, P, C).to(dt))
        if case["add"]:
            st.update(add=(1e-3 * _randn(gen, B, P, K)).to(dt))
    else:
        B, P, C, G = case["B"], case["P"], case["C"], case["G"]
        # channels of different scale and offset, brighter and darker samples
        x = _randn(gen, B, P, C).mul_(_randn(gen, C).mul_(0.5).exp_()).add_(_randn(gen, C)).mul_(_randn(gen, B, 1, 1).mul_(0.3).exp_()).to(dt)
        st.update(x=x, gamma=1 + 0.1 * _randn(gen, C), beta=0.1 * _randn(gen, C))
        if kind == "group_norm":
            st.update(y=_empty(B, P, C, dtype=dt), mean=_empty(B, G), rstd=_empty(B, G))
        else:
            mean, rstd = _moments(x.float().view(B, P, G, C // G))
            st.update(mean=mean, rstd=rstd, dy=(1e-3 * _randn(gen, B, P, C)).to(dt), dx=_empty(B, P, C, dtype=dt))
            st.update({k: _empty(C) for k in ("s_gamma", "s_beta", "g_gamma", "g_beta")})
    return st


# ---------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------
def _act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return 0.5 * z * torch.erfc(-z * math.sqrt(0.5))
    if act == "silu":
        return z / (1 + (-z).exp())
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "gelu":
        return 0.5 * torch.erfc(-z * math.sqrt(0.5)) + z * (-0.5 * z * z).exp() * (1 / math.sqrt(2 * math.pi))
    if act == "silu":
        s = 1 / (1 + (-z).exp())
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def _threshold(p):
    """A 16-bit number below this drops an element: p to 16 bits."""
    return int(math.floor(p * 65536 + 0.5))


def _dropped(x, rng, p):
    """x [R, C], every element with probability p dropped, the others scaled so that the mean stays.  Philox with 4 words and 10 rounds (Salmon et al.,
    SC 2011), keyed by rng[0], of the counter (piece of eight columns, row, rng[1]): its four words are the eight columns' 16-bit numbers."""
    t = _threshold(p)
    if t == 0:
        return x
    if t == 65536:
        return torch.zeros_like(x)
    R, C = x.shape
    low = 0xFFFFFFFF
    pieces = (C + 7) // 8
    c0 = torch.arange(pieces, device="cuda").expand(R, pieces)
    c1 = torch.arange(R, device="cuda")[:, None].expand(R, pieces)
    c2, c3 = rng[1] & low, (rng[1] >> 32) & low
    k0, k1 = rng[0] & low, (rng[0] >> 32) & low
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    numbers = torch.stack([half.expand(R, pieces) for w in (c0, c1, c2, c3) for half in (w & 0xFFFF, w >> 16)], -1).reshape(R, -1)[:, :C]
    return torch.where(numbers >= t, x * (65536 / (65536 - t)), 0.0)


def _sums(G, c):
    """The two sums over the samples of their gradients G."""
    return c * c * (G * G).sum(0), c * G.sum(0)


def _moments(x):
    """Mean and 1 / standard deviation of every sample's groups, x [B, P, G, channels]."""
    mean = x.mean((1, 3))
    d = x - mean[:, None, :, None]
    return mean, 1 / ((d * d).mean((1, 3)) + EPS).sqrt()


def _plain(st):
    case = st["case"]
    kind, dt, p = case["kind"], _dtype(case), case.get("p", 0.0)
    if kind == "dropout":
        y = _dropped(st["x"].float(), st["rng"], p)
        return dict(y=(y + st["residual"].float() if case["residual"] else y).to(dt))
    if kind == "linear":
        z = st["X"].float() @ st["W"].float() + st["bias"]
        y = _act(z, case["act"])
        if p > 0:
            y = _dropped(y, st["rng"], p)
        if case["residual"]:
            y = y + st["residual"].float()
        return dict(y=y.to(dt), z=z.to(dt)) if case["keep"] else dict(y=y.to(dt))
    if kind == "linear_backward":
        B, P, C = case["B"], case["P"], case["C"]
        dz = st["dy"].float()
        if p > 0:
            dz = _dropped(dz.view(B * P, C), st["rng"], p).view(B, P, C)
        if case["act"] != "none":
            dz = dz * _act_slope(st["z"].float(), case["act"])
        dX = dz @ st["W"].float().t()
        if case["add"]:
            dX = dX + st["add"].float()
        s, g = _sums(dz.sum(1), 1.0 / B)
        return dict(dz=dz.to(dt), dX=dX.to(dt), s_bias=s, g_bias=g)
    B, P, C, G = case["B"], case["P"], case["C"], case["G"]
    x, gamma, beta = st["x"].float().view(B, P, G, C // G), st["gamma"].view(G, C // G), st["beta"].view(G, C // G)
    if kind == "group_norm":
        mean, rstd = _moments(x)
        xhat = (x - mean[:, None, :, None]) * rstd[:, None, :, None]
        return dict(y=_act(xhat * gamma + beta, case["act"]).to(dt).view(B, P, C), mean=mean, rstd=rstd)
    mean, rstd = st["mean"][:, None, :, None], st["rstd"][:, None, :, None]
    xhat = (x - mean) * rstd
    dt_ = st["dy"].float().view(x.shape)
    if case["act"] != "none":
        dt_ = dt_ * _act_slope(xhat * gamma + beta, case["act"])
    d = dt_ * gamma
    dx = rstd * (d - d.mean((1, 3), keepdim=True) - xhat * (d * xhat).mean((1, 3), keepdim=True))
    out, c = dict(dx=dx.to(dt).view(B, P, C)), 1.0 / B
    out["s_gamma"], out["g_gamma"] = _sums((dt_ * xhat).sum(1).view(B, C), c)
    out["s_beta"], out["g_beta"] = _sums(dt_.sum(1).view(B, C), c)
    return out


# ---------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------
def _workspace(st, nbytes):
    """A program makes the working memory of a call once and keeps it."""
    if "workspace" not in st:
        st["workspace"] = _empty(nbytes, dtype=torch.uint8) if nbytes else None
    return st["workspace"]


def run(st):
    if not own:
        return _plain(st)
    from paper_1802_06058_amd import vgc

    case = st["case"]
    kind, code, p = case["kind"], vgc.BF16 if case["dtype"] == "bf16" else vgc.F32, case.get("p", 0.0)
    if kind == "dropout":
        vgc.dropout(st["x"], p, st["rng"], st["y"], st.get("residual"))
        return dict(y=st["y"])
    act = dict(none=vgc.ACT_NONE, relu=vgc.ACT_RELU, gelu=vgc.ACT_GELU, silu=vgc.ACT_SILU)[case["act"]]
    if kind == "linear":
        ws = _workspace(st, vgc.linear_workspace_bytes(code, case["N"], case["K"], case["C"]))
        vgc.linear(st["X"], st["W"], st["y"], st["bias"], act, z=st.get("z"), residual=st.get("residual"), p=p, rng=st.get("rng"), workspace=ws)
        return dict(y=st["y"], z=st["z"]) if case["keep"] else dict(y=st["y"])
    if kind == "linear_backward":
        B, P, K, C = case["B"], case["P"], case["K"], case["C"]
        ws = _workspace(st, vgc.linear_backward_workspace_bytes(code, B, P, K, C))
        vgc.linear_backward(st["dy"], st.get("z"), st["W"], act, 1.0 / B, st["dz"], st["dX"], st["s_bias"], st["g_bias"], add=st.get("add"), p=p,
                            rng=st.get("rng"), workspace=ws)
        return {k: st[k] for k in ("dz", "dX", "s_bias", "g_bias")}
    B, P, C, G = case["B"], case["P"], case["C"], case["G"]
    if kind == "group_norm":
        ws = _workspace(st, vgc.group_norm_workspace_bytes(code, B, P, C, G))
        vgc.group_norm(st["x"], st["gamma"], st["beta"], EPS, act, st["y"], st["mean"], st["rstd"], ws)
        return {k: st[k] for k in ("y", "mean", "rstd")}
    ws = _workspace(st, vgc.group_norm_backward_workspace_bytes(code, B, P, C, G))
    vgc.group_norm_backward(st["dy"], st["x"], st["mean"], st["rstd"], st["gamma"], st["beta"], act, 1.0 / B, st["dx"], st["s_gamma"], st["s_beta"],
                            st["g_gamma"], st["g_beta"], ws)
    return {k: st[k] for k in ("dx", "s_gamma", "s_beta", "g_gamma", "g_beta")}


# ---------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------
def work(case):
    kind, size = case["kind"], 2 if case["dtype"] == "bf16" else 4
    if kind == "dropout":
        n = case["R"] * case["C"]
        return {"bytes": size * n * (3.0 if case["residual"] else 2.0), "flops": 2.0 * n}
    if kind == "linear":
        N, K, C = case["N"], case["K"], case["C"]
        return {"bytes": size * (N * K + K * C + N * C * (1.0 + case["keep"] + case["residual"])) + 4.0 * C, "flops": 2.0 * N * K * C}
    if kind == "linear_backward":
        N, K, C = case["B"] * case["P"], case["K"], case["C"]
        return {"bytes": size * (N * C * (2.0 + (case["act"] != "none")) + K * C + N * K * (1.0 + case["add"])) + 8.0 * C, "flops": 2.0 * N * K * C}
    n = case["B"] * case["P"] * case["C"]
    if kind == "group_norm":
        return {"bytes": 2.0 * size * n + 8.0 * case["B"] * case["G"] + 8.0 * case["C"], "flops": 8.0 * n}
    return {"bytes": 3.0 * size * n + 8.0 * case["B"] * case["G"] + 24.0 * case["C"], "flops": 16.0 * n}


# ---------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------
def _numbers(R, C, rng):
    """The generator's 16-bit numbers, its products formed from halves of 16 bits."""
    key, call = (int(v) for v in rng.tolist())

    def product(x, m):
        xl, xh, ml, mh = x & 65535, x >> 16, m & 65535, m >> 16
        mid = xl * mh + (xl * ml >> 16)
        rest = xh * ml + (mid & 65535)
        return xh * mh + (mid >> 16) + (rest >> 16), (rest & 65535) * 65536 + (xl * ml & 65535)

    rows, pieces = torch.meshgrid(torch.arange(R, device="cuda"), torch.arange(-(-C // 8), device="cuda"), indexing="ij")
    x = [pieces, rows, torch.full_like(rows, call % 2 ** 32), torch.full_like(rows, call // 2 ** 32)]
    for i in range(10):
        h0, l0 = product(x[0], 0xD2511F53)
        h1, l1 = product(x[2], 0xCD9E8D57)
        x = [h1 ^ x[1] ^ (key + i * 0x9E3779B9) % 2 ** 32, l1, h0 ^ x[3] ^ (key // 2 ** 32 + i * 0xBB67AE85) % 2 ** 32, l0]
    words = torch.stack(x, -1)
    return torch.stack([words % 65536, words // 65536], -1).flatten(1)[:, :C]


def _kept(R, C, rng, p):
    """What every element is multiplied with."""
    t = _threshold(p)
    if t == 65536:
        return torch.zeros(R, C, device="cuda", dtype=torch.float64)
    return (_numbers(R, C, rng) >= t).double() * (65536 / (65536 - t))


def _phi(z):
    """The share of a normal distribution below z."""
    return torch.special.ndtr(z)


def _value(z, act):
    return {"none": lambda: z, "relu": lambda: torch.maximum(z, torch.zeros_like(z)), "gelu": lambda: z * _phi(z),
            "silu": lambda: z * torch.sigmoid(z)}[act]()


def _slope(z, act):
    if act == "silu":
        s = torch.sigmoid(z)
        return s + z * s * torch.sigmoid(-z)
    return {"none": lambda: torch.ones_like(z), "relu": lambda: (z > 0).double(),
            "gelu": lambda: _phi(z) + z * torch.exp(-z.square() / 2) / math.sqrt(2 * math.pi)}[act]()


def exact(case, seed):
    st = prepare(case, seed)
    kind, p = case["kind"], case.get("p", 0.0)
    if kind == "dropout":
        y = st["x"].double() * _kept(case["R"], case["C"], st["rng"], p)
        return dict(y=y + st["residual"].double() if case["residual"] else y)
    if kind == "linear":
        z = torch.addmm(st["bias"].double(), st["X"].double(), st["W"].double())
        y = _value(z, case["act"])
        if p > 0:
            y = y * _kept(case["N"], case["C"], st["rng"], p)
        if case["residual"]:
            y = y + st["residual"]
        return dict(y=y, z=z) if case["keep"] else dict(y=y)
    if kind == "linear_backward":
        B, P, K, C = case["B"], case["P"], case["K"], case["C"]
        dz = st["dy"].double().view(B * P, C)
        if p > 0:
            dz = dz * _kept(B * P, C, st["rng"], p)
        if case["act"] != "none":
            dz = dz * _slope(st["z"].double().view(B * P, C), case["act"])
        dX = torch.mm(dz, st["W"].double().t().contiguous())
        if case["add"]:
            dX += st["add"].view(B * P, K)
        H = dz.view(B, P, C).sum(1) / B
        return dict(dz=dz.view(B, P, C), dX=dX.view(B, P, K), s_bias=H.square().sum(0), g_bias=H.sum(0))
    B, P, C, G = case["B"], case["P"], case["C"], case["G"]
    M, channel = P * (C // G), torch.arange(C, device="cuda") // (C // G)
    gamma, beta, act = st["gamma"].double(), st["beta"].double(), case["act"]
    if kind == "group_norm":
        out = dict(y=torch.empty(B, P, C, device="cuda", dtype=torch.float64), mean=torch.empty(B, G, device="cuda", dtype=torch.float64),
                   rstd=torch.empty(B, G, device="cuda", dtype=torch.float64))
        for z in range(B):
            x = st["x"][z].double()
            groups = x.view(P, G, C // G).transpose(0, 1).reshape(G, M)
            var, mean = torch.var_mean(groups, 1, unbiased=False)
            out["mean"][z], out["rstd"][z] = mean, (var + EPS).rsqrt()
            out["y"][z] = _value((x - mean[channel]) * out["rstd"][z][channel] * gamma + beta, act)
        return out
    dx = torch.empty(B, P, C, device="cuda", dtype=torch.float64)
    of_gamma, of_beta = (torch.empty(B, C, device="cuda", dtype=torch.float64) for _ in range(2))
    for z in range(B):
        rstd = st["rstd"][z].double()[channel]
        xhat = (st["x"][z].double() - st["mean"][z].double()[channel]) * rstd
        d = st["dy"][z].double() * _slope(xhat * gamma + beta, act)
        of_gamma[z], of_beta[z] = (d * xhat).sum(0), d.sum(0)
        a = (gamma * of_beta[z]).view(G, -1).sum(1)[channel]
        b = (gamma * of_gamma[z]).view(G, -1).sum(1)[channel]
        dx[z] = (M * gamma * d - a - xhat * b) * (rstd / M)
    return dict(dx=dx, s_gamma=(of_gamma / B).square().sum(0), s_beta=(of_beta / B).square().sum(0), g_gamma=of_gamma.mean(0), g_beta=of_beta.mean(0))
