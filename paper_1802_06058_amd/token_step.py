"""One worker's training step of a small token classifier, from its activations to the updated parameters, on the GPU:

    h = x W1            a linear layer; its input x is kept in 8 bits       (linear, act8_encode)
    y = layer norm(h)   the normalised rows are kept in 8 bits              (layer_norm)
    u = gelu(y Wa + ba) a residual feed-forward block, if asked for: its    (linear)
    y += drop(u Wb + bb)    dropout's mask is drawn again in the backward pass
    loss of y W^T       over the classes, without the logits                (softmax_loss)
    backward            dy and the sums for W                               (softmax_loss_backward)
                        through the block, with the sums for ba and bb      (linear_backward)
                        the sums for Wa and Wb                              (sqgrad)
                        dh and the sums for gamma and beta, from what is kept (layer_norm_backward)
                        the sums for W1, from what is kept                  (sqgrad_act8)
    exchange            accumulate and select, pack, decode with the update (accumulate_select, pack, unpack_apply)

The sums g and s of every parameter land in the flat arrays that the selection reads.  Run it:

    python -m paper_1802_06058_amd.token_step --steps 40
    python -m paper_1802_06058_amd.token_step --steps 40 --feed-forward 2048 --dropout 0.1
"""
from __future__ import annotations

import argparse

import torch

from . import vgc, workloads


class TokenStep:
    """Parameters, optimizer and worker state, and the working memory of a step on batches of B sequences of P positions.  F: channels of the
    feed-forward block (0: none); dropout: of what the block adds."""

    def __init__(self, B=8, P=64, J=256, H=512, V=1000, dtype=torch.bfloat16, alpha=1.0, zeta=0.999, lr=0.05, momentum=0.9, seed=0, device="cuda", F=0,
                 dropout=0.0):
        self.B, self.P, self.J, self.H, self.V, self.dtype, self.F, self.dropout = B, P, J, H, V, dtype, F, dropout
        self.alpha, self.zeta, self.lr, self.momentum = alpha, zeta, lr, momentum
        f32 = dict(dtype=torch.float32, device=device)
        shapes = dict(W1=(J, H), gamma=(H,), beta=(H,), W=(V, H))
        if F:
            shapes.update(Wa=(H, F), Wb=(F, H), ba=(F,), bb=(H,))        # (weights first: where they lie is then aligned for any F)
        sizes = [torch.Size(s).numel() for s in shapes.values()]
        groups = workloads.groups_from_sizes(sizes)
        self.plan = vgc.Plan(groups, device)
        n = self.plan.n
        self.g, self.s, self.r, self.v = (torch.zeros(n, **f32) for _ in range(4))
        self.param, self.velocity = torch.empty(n, **f32), torch.zeros(n, **f32)
        at = lambda flat: {k: flat[o:o + m].view(shape) for (k, shape), (o, m) in zip(shapes.items(), groups)}
        self.p, self.gs, self.ss = at(self.param), at(self.g), at(self.s)
        gen = torch.Generator(device=device).manual_seed(seed)
        self.p["W1"].normal_(0, J ** -0.5, generator=gen)
        self.p["W"].normal_(0, H ** -0.5, generator=gen)
        self.p["gamma"].fill_(1)
        self.p["beta"].zero_()
        if F:
            self.p["Wa"].normal_(0, H ** -0.5, generator=gen)
            self.p["Wb"].normal_(0, F ** -0.5, generator=gen)
            self.p["ba"].zero_()
            self.p["bb"].zero_()
        self.scratch, self.hdrs, self.status = self.plan.new_scratch(), self.plan.new_headers(), self.plan.new_status()
        self.words = torch.zeros(n, dtype=torch.int32, device=device)
        rows = lambda C, t=dtype: torch.empty(B, P, C, dtype=t, device=device)
        kept = lambda C: (rows(C, torch.int8), rows((C + 31) // 32, torch.uint8))
        self.kept_x, self.kept_h = kept(J), kept(H)
        self.h, self.y, self.dy, self.dh = rows(H), rows(H), rows(H), rows(H)
        if F:
            self.za, self.u, self.du, self.out, self.dout, self.dzb = rows(F), rows(F), rows(F), rows(H), rows(H), rows(H)
            self.rng = torch.tensor([seed, 0], device=device)          # the dropout's key and the number of the step, which lives on the device too
        self.mean, self.rstd, self.loss, self.lse = (torch.empty(B * P, **f32) for _ in range(4))
        code = vgc.F32 if dtype == torch.float32 else vgc.BF16
        # the calls of a step follow each other on one stream: one workspace serves them all
        need = [vgc.softmax_loss_workspace_bytes(code, B * P, H, V), vgc.softmax_loss_backward_workspace_bytes(code, B, P, H, V),
                vgc.layer_norm_backward_workspace_bytes(B, P, H), vgc.sqgrad_act8_workspace_bytes(vgc.CONV, code, B, P, J, H),
                vgc.linear_workspace_bytes(code, B * P, J, H)]
        if F:
            for K, C in ((H, F), (F, H)):
                need += [vgc.linear_workspace_bytes(code, B * P, K, C), vgc.linear_backward_workspace_bytes(code, B, P, K, C),
                         vgc.sqgrad_workspace_bytes(vgc.CONV, code, B, P, K, C)]
        self.workspace = torch.empty(max(need), dtype=torch.uint8, device=device)

    def step(self, x, target):
        """x [B, P, J], target [B, P] (negative: not asked for).  Enqueues one step; returns the losses [B, P] of before the update."""
        c, ws = 1.0 / self.B, self.workspace
        asked = (target >= 0).sum(1, keepdim=True).clamp(min=1)
        weight = (1.0 / asked).expand(self.B, self.P).contiguous().float()     # a sequence's own loss: the mean over what it is asked for
        W1, W = self.p["W1"].to(self.dtype), self.p["W"].to(self.dtype)
        vgc.act8_encode(x, *self.kept_x)
        vgc.linear(x if x.data_ptr() % 16 == 0 else x.clone(), W1, self.h, workspace=ws)
        vgc.layer_norm(self.h, self.p["gamma"], self.p["beta"], 1e-5, self.y, self.mean, self.rstd, self.kept_h)
        out, dout = (self.out, self.dout) if self.F else (self.y, self.dy)
        if self.F:
            Wa, Wb = self.p["Wa"].to(self.dtype), self.p["Wb"].to(self.dtype)
            self.rng[1] += 1
            vgc.linear(self.y, Wa, self.u, self.p["ba"], vgc.ACT_GELU, z=self.za, workspace=ws)
            vgc.linear(self.u, Wb, self.out, self.p["bb"], residual=self.y, p=self.dropout, rng=self.rng, workspace=ws)
        vgc.softmax_loss(out, W, target, self.loss, self.lse, ws)
        vgc.softmax_loss_backward(out, W, target, self.lse, weight, c, dout, self.ss["W"], self.gs["W"], ws)
        if self.F:                                                   # dzb and dza (in za's place) are the D of their weights' statistic
            vgc.linear_backward(dout, None, Wb, vgc.ACT_NONE, c, self.dzb, self.du, self.ss["bb"], self.gs["bb"], p=self.dropout, rng=self.rng, workspace=ws)
            vgc.sqgrad(vgc.CONV, self.u, self.dzb, c, self.ss["Wb"], self.gs["Wb"], ws)
            vgc.linear_backward(self.du, self.za, Wa, vgc.ACT_GELU, c, self.za, self.dy, self.ss["ba"], self.gs["ba"], add=dout, workspace=ws)
            vgc.sqgrad(vgc.CONV, self.y, self.za, c, self.ss["Wa"], self.gs["Wa"], ws)
        vgc.layer_norm_backward(self.dy, None, None, self.rstd, self.p["gamma"], c, self.dh, self.ss["gamma"], self.ss["beta"], self.gs["gamma"],
                                self.gs["beta"], ws, act8=self.kept_h)
        vgc.sqgrad_act8(vgc.CONV, *self.kept_x, self.dh, c, self.ss["W1"], self.gs["W1"], ws)
        vgc.accumulate_select(self.g, self.s, self.r, self.v, self.plan, self.alpha, self.zeta, self.scratch)
        vgc.pack(self.plan, self.scratch, self.words, self.hdrs, self.status)
        vgc.unpack_apply([self.words], [self.words.numel()], [self.hdrs], self.plan, 1.0, self.param, self.velocity, lr=self.lr,
                         momentum=self.momentum)
        return self.loss.view(self.B, self.P)


def batches(model, seed=1, noise=0.5, unasked=0.1):
    """Positions whose inputs are noisy copies of their class's own vector; a tenth of them is not asked for."""
    dev = model.param.device
    gen = torch.Generator(device=dev).manual_seed(seed)
    centres = torch.randn(model.V, model.J, generator=gen, device=dev)
    while True:
        target = torch.randint(0, model.V, (model.B, model.P), generator=gen, device=dev)
        x = centres[target] + noise * torch.randn(model.B, model.P, model.J, generator=gen, device=dev)
        target[torch.rand(model.B, model.P, generator=gen, device=dev) < unasked] = -1
        yield x.to(model.dtype), target


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--alpha", type=float, default=1.0)
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    ap.add_argument("--feed-forward", type=int, default=0, help="channels of a residual feed-forward block before the classes (0: none)")
    ap.add_argument("--dropout", type=float, default=0.0, help="of what the block adds")
    a = ap.parse_args()
    model = TokenStep(alpha=a.alpha, dtype=torch.bfloat16 if a.dtype == "bf16" else torch.float32, F=a.feed_forward, dropout=a.dropout)
    data = batches(model)
    for k in range(a.steps):
        x, target = next(data)
        loss = model.step(x, target)
        if k % 10 == 0 or k == a.steps - 1:
            sent, _ = vgc.read_status(model.status)
            print(f"step {k}: loss {float(loss.sum() / (target >= 0).sum()):.4f}, {sent} of {model.plan.n} parameters sent", flush=True)


if __name__ == "__main__":
    main()
