"""A gated feed-forward block, trained in 16 bits and served with 4-bit
weights: ffn_forward, ffn_backward, aqe_clip_grads and aqe_sgd_clip in a
training step, q4_pack once, then q4_gated for every token.

  python -m paper_2003_04296_amd.gated            trains a small block towards
                                                  another's outputs, packs it
                                                  and serves single tokens
"""
from __future__ import annotations

import torch

from . import ACT_SILU, aqe_clip_grads, aqe_sgd_clip, ffn_backward, ffn_forward, q4_gated, q4_pack


class GatedBlock:
    """h = act(x w_gate^T) * (x w_up^T) with trainable weights [f][k]: fp32
    masters in [-1, 1] (what aqe_sgd_clip keeps them in) and the 16-bit copies
    the products use."""

    def __init__(self, k: int, f: int, act: int = ACT_SILU, dtype=torch.bfloat16, device="cuda:0", seed: int = 0):
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        self.act = act
        self.masters = [torch.randn((f, k), generator=gen, device=device).mul_(k ** -0.5).clamp_(-1, 1)
                        for _ in range(2)]
        self.weights = [w.to(dtype) for w in self.masters]

    def forward(self, x):
        return ffn_forward(x, *self.weights, self.act)[0]

    def forward_train(self, x):
        """-> (h, what step needs of this forward)."""
        return ffn_forward(x, *self.weights, self.act, keep_pre=True)

    def step(self, x, gh, lr: float, max_norm: float, pre=None):
        """From the gradient gh of h at x: the weights one SGD step on, with the
        gradients' joint norm held to max_norm -> (gradient of x, norm before
        clipping).  pre: from forward_train(x) with the present weights;
        without it the forward is computed again."""
        if pre is None:
            pre = self.forward_train(x)[1]
        gx, *grads = ffn_backward(x, *self.weights, pre, gh, self.act)
        grads = [g.float() for g in grads]
        norm = aqe_clip_grads(grads, max_norm)
        for w, master, g in zip(self.weights, self.masters, grads):
            w.copy_(aqe_sgd_clip(master, g, lr))
        return gx, norm

    def packed(self, group: int = 64, top: int = 6):
        return PackedGatedBlock([q4_pack(w, group, top) for w in self.masters], self.act)


class PackedGatedBlock:
    """The same block on 4-bit weights (q4_pack), for inference."""

    def __init__(self, weights, act: int):
        self.act = act
        self.weights = weights

    def forward(self, x, out=None):
        return q4_gated(x, *self.weights[0], *self.weights[1], self.act, out=out)


def train(steps: int = 150, m: int = 256, k: int = 128, f: int = 192, lr: float = 1.0, max_norm: float = 1.0,
          device="cuda:0", seed: int = 0):
    """Trains a block towards another one's outputs on random tokens ->
    (block, its teacher, the mean squared errors)."""
    teacher, block = (GatedBlock(k, f, device=device, seed=seed + s) for s in (1, 2))
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    losses = []
    for _ in range(steps):
        x = torch.randn((m, k), generator=gen, device=device).to(torch.bfloat16)
        want, (h, pre) = teacher.forward(x), block.forward_train(x)
        diff = h.float() - want.float()
        losses.append(diff.square().mean())
        block.step(x, (diff * (2.0 / m)).to(h.dtype), lr, max_norm, pre)
    return block, teacher, torch.stack(losses).tolist()


def main():
    block, teacher, losses = train()
    print(f"mean squared error {losses[0]:.4f} -> {losses[-1]:.4f} in {len(losses)} steps")
    packed = block.packed()
    x = torch.randn((8, block.masters[0].shape[1]), device=block.masters[0].device).to(torch.bfloat16)
    served = torch.cat([packed.forward(x[i:i + 1]) for i in range(len(x))])
    full = block.forward(x)
    off = float((served.float() - full.float()).norm() / full.float().norm())
    print(f"served token by token on 4-bit weights: {off:.3f} relative to the 16-bit block")


if __name__ == "__main__":
    main()
