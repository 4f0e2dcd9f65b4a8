"""Merge, then run what the merge made: python examples/feed_forward.py

A Qwen2.5-1.5B-shaped family of one layer is merged (TIES, a quarter of the
expert reads).  The merged checkpoint's feed-forward block then takes a prompt
(mp_norm, mp_linear), a few training steps on it (mp_linear_backward,
mp_norm_backward) and single tokens (mp_moe with the merged checkpoint as its
only expert).  Last, the experts are served unmerged, two of them per token
(mp_moe over the K checkpoints).
"""

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2605_29489_amd as mp  # noqa: E402
from workloads import family_spec, make_family_device  # noqa: E402


class FeedForward:
    """x + down(silu(gate n) * (up n)), n = RMS norm of x, over a flat checkpoint's own storage."""

    def __init__(self, spec, flat, layer=0):
        self.off, at = {}, 0
        for name, shape in spec.tensors:
            n = torch.Size(shape).numel()
            self.off[name] = at
            if name.startswith(f"layers.{layer}."):
                view = flat[at:at + n].view(shape)
                for part, key in (("gate_proj", "gate"), ("up_proj", "up"), ("down_proj", "down"),
                                  ("post_attention_layernorm", "norm")):
                    if part in name:
                        setattr(self, key, view)
                        setattr(self, key + "_off", at)
            at += n
        self.ffn, self.hidden = self.gate.shape
        self.flat = flat

    def layer(self, top_k, renorm=True):
        return mp.MoeLayer(self.hidden, self.ffn, top_k, self.gate_off, self.up_off, self.down_off, mp.MP_ACT_SILU,
                           renorm)

    def normed(self, x):
        n = torch.empty_like(x)
        rstd = torch.empty(x.shape[0], device=x.device)
        mp.mp_norm(x, n, weight=self.norm, rms=True, rstd=rstd)
        return n, rstd

    def forward(self, x):
        """y, and what the backward pass needs."""
        n, rstd = self.normed(x)
        wide = lambda: x.new_empty(x.shape[0], self.ffn)  # noqa: E731
        g, z, u, y = wide(), wide(), wide(), torch.empty_like(x)
        mp.mp_linear(n, self.gate, g, act=mp.MP_ACT_SILU, z=z)
        mp.mp_linear(n, self.up, u)
        h = g * u
        mp.mp_linear(h, self.down, y, residual=x)
        return y, (x, n, rstd, g, z, u, h)

    def backward(self, dy, kept):
        """Gradients of x and of the four tensors."""
        x, n, rstd, g, z, u, h = kept
        new = torch.empty_like
        dh, ddown = new(h), new(self.down)
        mp.mp_linear_backward(dy, x=h, w=self.down, dx=dh, dw=ddown)
        dn, du, dgate, dup = new(n), new(n), new(self.gate), new(self.up)
        mp.mp_linear_backward(dh * u, x=n, w=self.gate, z=z, act=mp.MP_ACT_SILU, dx=dn, dw=dgate)
        mp.mp_linear_backward(dh * g, x=n, w=self.up, dx=du, dw=dup)
        dx, dnorm = new(x), new(self.norm)
        mp.mp_norm_backward(dn + du, x, rstd, weight=self.norm, rms=True, dx=dx, dweight=dnorm)
        return dx + dy, dict(gate=dgate, up=dup, down=ddown, norm=dnorm)


def merge(spec, base, experts, budget=0.25):
    lay = spec.layout
    L = mp.Layout(lay.numel, lay.block_elems, mp.MP_BF16)
    K, G = len(experts), len(lay.block_lengths())
    sumsq = torch.empty(G * K, device="cuda")
    tau = torch.empty(G * K, dtype=torch.int32, device="cuda")
    mask = torch.empty(G, dtype=torch.int32, device="cuda")
    out = torch.empty_like(base)
    mp.mp_index_ties(L, base, experts, 0.2, tau, sumsq)
    mp.mp_plan(L, K, sumsq, [1.0] * K, int(budget * lay.ckpt_bytes * K), mask)
    mp.mp_merge_ties_tau(L, base, experts, mask, tau, 1.0, out)
    return out


def main(tokens=512, steps=4, seed=0, say=print):
    spec = family_spec("qwen2.5-1.5b", n_layers=1, vocab=256)
    base, experts = make_family_device(spec, seed=seed)
    block = FeedForward(spec, merge(spec, base, experts))
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    x = torch.randn(tokens, block.hidden, generator=gen, device="cuda", dtype=torch.bfloat16)

    # single tokens through the merged checkpoint: the layer of experts with one expert
    y, _ = block.forward(x)
    n, _ = block.normed(x)
    one = torch.empty_like(x[:4])
    mp.mp_moe(block.layer(1), n[:4], torch.zeros_like(block.norm)[None], [block.flat], one, residual=x[:4])
    apart = float((one.float() - y[:4].float()).abs().max())
    say(f"prompt of {tokens} tokens, and its first 4 as single tokens: {apart:.4f} apart at most")

    # the experts unmerged, two per token
    router = torch.randn(len(experts), block.hidden, generator=gen, device="cuda", dtype=torch.bfloat16) * 0.02
    ids = torch.empty(4, 2, dtype=torch.int32, device="cuda")
    mixed = torch.empty_like(one)
    mp.mp_moe(block.layer(2), n[:4], router, experts, mixed, ids=ids, residual=x[:4])
    say(f"unmerged, experts {ids.tolist()}: {float((mixed.float() - one.float()).abs().max()):.4f} from the merge")

    # training on from the merge: towards the base checkpoint's answers
    want, _ = FeedForward(spec, base).forward(x)
    losses = []
    for step in range(steps):
        y, kept = block.forward(x)
        d = y - want
        losses.append(float(d.float().square().mean()))
        _, grads = block.backward(d, kept)
        for name, grad in grads.items():
            getattr(block, name).sub_(grad, alpha=0.02 / tokens)
        say(f"step {step}: loss {losses[-1]:.3e}")
    return apart, losses


if __name__ == "__main__":
    main()
