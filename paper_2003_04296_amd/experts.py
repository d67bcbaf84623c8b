"""A block of gated experts, trained in 16 bits, and adapters of many requests
beside a shared 4-bit projection: moe_sort once a batch, moe_gather, the experts'
products, moe_combine and their gradients in a training step; q4_linear and
lora_forward for every batch of requests.

  python -m paper_2003_04296_amd.experts          trains a small block towards
                                                  another's outputs and serves
                                                  requests with adapters
"""
from __future__ import annotations

import torch

from . import (ACT_SILU, aqe_clip_grads, aqe_sgd_clip, lora_forward, moe_combine, moe_combine_backward, moe_gated_backward,
               moe_gated_forward, moe_gather, moe_gather_backward, moe_linear_backward, moe_linear_forward, moe_sort, q4_linear,
               q4_pack)


class ExpertBlock:
    """y[t] = sum_s w[t, s] W_e h_e(x[t]), h_e = act(x Wg_e^T) * (x Wu_e^T), e the
    token's s-th best expert by a linear router and w the softmax of those scores.
    Weights: fp32 masters in [-1, 1] (what aqe_sgd_clip keeps them in) and the
    16-bit copies the products use: gate and up [experts][f][k], down
    [experts][k][f]; the router [experts][k] in fp32."""

    def __init__(self, k: int, f: int, experts: int, slots: int, act: int = ACT_SILU, dtype=torch.bfloat16,
                 device="cuda:0", seed: int = 0):
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        draw = lambda *s: torch.randn(s, generator=gen, device=device).mul_(s[-1] ** -0.5).clamp_(-1, 1)
        self.act, self.slots = act, slots
        self.masters = [draw(experts, f, k), draw(experts, f, k), draw(experts, k, f), draw(experts, k)]
        self.weights = [w.to(dtype) for w in self.masters[:3]]

    def route(self, x):
        """(ids, weights) [tokens][slots] of each token's best experts."""
        top = torch.topk(x.float() @ self.masters[3].t(), self.slots, dim=1)
        return top.indices, torch.softmax(top.values, dim=1)

    def forward_train(self, x):
        """-> (y, what gradients needs of this forward)."""
        ids, weights = self.route(x)
        offsets, _, place = moe_sort(ids, len(self.masters[3]))
        wg, wu, wd = self.weights
        xs = moe_gather(x, place)
        h, pre = moe_gated_forward(xs, wg, wu, offsets, self.act, keep_pre=True)
        ys = moe_linear_forward(h, wd, offsets)
        return moe_combine(ys, place, weights), (x, ids, weights, offsets, place, xs, h, pre, ys)

    def forward(self, x):
        return self.forward_train(x)[0]

    def gradients(self, gy, saved):
        """From the gradient gy of y -> (that of x, those of the four weights)."""
        x, ids, weights, offsets, place, xs, h, pre, ys = saved
        wg, wu, wd = self.weights
        gys, gw = moe_combine_backward(gy, ys, place, weights)
        gh, gwd = moe_linear_backward(h, wd, offsets, gys)
        gxs, gwg, gwu = moe_gated_backward(xs, wg, wu, offsets, pre, gh, self.act)
        # of the scores, through their softmax; the others have none
        gs = weights * (gw - (weights * gw).sum(1, keepdim=True))
        scores = torch.zeros((len(x), len(self.masters[3])), device=x.device).scatter_(1, ids, gs)
        gx = moe_gather_backward(gxs, place).float() + scores @ self.masters[3]
        return gx.to(x.dtype), [gwg, gwu, gwd, scores.t() @ x.float()]

    def step(self, gy, saved, lr: float, max_norm: float):
        """The weights one SGD step on, the gradients' joint norm held to max_norm
        -> (gradient of x, norm before clipping)."""
        gx, grads = self.gradients(gy, saved)
        grads = [g.float() for g in grads]
        norm = aqe_clip_grads(grads, max_norm)
        for master, g in zip(self.masters, grads):
            aqe_sgd_clip(master, g, lr)
        for w, master in zip(self.weights, self.masters):
            w.copy_(master)
        return gx, norm


class AdaptedProjection:
    """y = x W^T with W in 4 bits for all requests, plus the adapter of each token's
    request: a [adapters][rank][k], b [adapters][n][rank], scale [adapters]."""

    def __init__(self, w, a, b, scale=None, group: int = 64):
        self.packed = q4_pack(w, group)
        self.a, self.b, self.scale = a, b, scale

    def plan(self, ids):
        """What forward needs of a batch's adapters (ids [tokens], -1: none); one serves all layers."""
        return moe_sort(ids, len(self.a))[:2]

    def forward(self, x, plan):
        y = q4_linear(x, *self.packed)
        return lora_forward(y, x, self.a, self.b, *plan, self.scale)[0]


def train(steps: int = 120, m: int = 256, k: int = 64, f: int = 96, experts: int = 8, slots: int = 2, lr: float = 1.0,
          max_norm: float = 1.0, device="cuda:0", seed: int = 0):
    """Trains a block towards another one's outputs on random tokens -> (block, the mean squared errors)."""
    teacher, block = (ExpertBlock(k, f, experts, slots, device=device, seed=seed + s) for s in (1, 2))
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    losses = []
    for _ in range(steps):
        x = torch.randn((m, k), generator=gen, device=device).to(torch.bfloat16)
        want, (y, saved) = teacher.forward(x), block.forward_train(x)
        diff = y.float() - want.float()
        losses.append(diff.square().mean())
        block.step((diff * (2.0 / m)).to(y.dtype), saved, lr, max_norm)
    return block, torch.stack(losses).tolist()


def main():
    _, losses = train()
    print(f"mean squared error {losses[0]:.4f} -> {losses[-1]:.4f} in {len(losses)} steps")
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(0)
    draw = lambda *s: torch.randn(s, generator=gen, device="cuda:0")
    adapters, rank, k, n = 5, 8, 256, 192
    layer = AdaptedProjection(draw(n, k) * k ** -0.5, (draw(adapters, rank, k) * k ** -0.5).bfloat16(),
                              draw(adapters, n, rank).bfloat16(), torch.full((adapters,), 0.5, device="cuda:0"))
    ids = torch.tensor([3, -1, 0, 3, 4, 1], device="cuda:0")
    y = layer.forward(draw(len(ids), k).bfloat16(), layer.plan(ids))
    print(f"{len(ids)} requests of {adapters} adapters: outputs of mean size {float(y.float().abs().mean()):.3f}")


if __name__ == "__main__":
    main()
