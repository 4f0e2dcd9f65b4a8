"""Merge, then serve what the merge made token by token: python examples/decode.py

A Qwen2.5-1.5B-shaped family of one layer is merged as in feed_forward.py.  The
merged checkpoint's whole block then takes a prompt and single tokens of
several sequences: mp_norm and mp_linear into a packed projection, mp_kv_append
(rotary positions, keys and values into pages), mp_kv_attend, mp_linear with the
residual, and the feed-forward part.  A step of single tokens is captured in a
HIP graph and replayed; positions, slots and lengths are device data.  Last, the
rotary positions alone and their gradient (mp_rope, mp_rope_backward).
"""

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2605_29489_amd as mp  # noqa: E402
from examples.feed_forward import FeedForward, merge  # noqa: E402
from workloads import family_spec, make_family_device  # noqa: E402

HEAD, PAGE = 128, 16


class Block:
    """One layer over a flat checkpoint's own storage, with a cache of `pages` pages."""

    def __init__(self, spec, flat, pages, base=1e6, layer=0):
        self.ff, at = FeedForward(spec, flat, layer), 0
        for name, shape in spec.tensors:
            n = torch.Size(shape).numel()
            if name.startswith(f"layers.{layer}.self_attn.") or name.startswith(f"layers.{layer}.input_layernorm"):
                key = name.split(".")[-2] + ("_b" if name.endswith("bias") else "")
                setattr(self, key, flat[at:at + n].view(shape))
            at += n
        self.q_heads, self.heads = self.q_proj.shape[0] // HEAD, self.k_proj.shape[0] // HEAD
        page = lambda: torch.zeros(pages, PAGE, self.heads, HEAD, dtype=flat.dtype, device=flat.device)  # noqa: E731
        self.cache = mp.KvCache(page(), page())
        freqs, self.amplitude = mp.mp_rope_frequencies(HEAD, base)
        self.freqs = freqs.to(flat.device)

    def project(self, x):
        """Queries, keys and values [tokens, heads, HEAD], parts of one packed buffer."""
        n, cuts = torch.empty_like(x), (self.q_heads, self.heads, self.heads)
        mp.mp_norm(x, n, weight=self.input_layernorm, rms=True)
        qkv = x.new_empty(x.shape[0], sum(cuts) * HEAD)
        for name, part in zip("qkv", qkv.split([c * HEAD for c in cuts], 1)):
            mp.mp_linear(n, getattr(self, name + "_proj"), part, bias=getattr(self, name + "_proj_b", None))
        return qkv.unflatten(1, (-1, HEAD)).split(cuts, 1)

    def forward(self, x, positions, table):
        """Tokens at `positions` of the sequences whose pages the rows of `table` hold."""
        q, k, v = self.project(x)
        page = table.gather(1, (positions // PAGE)[:, None])[:, 0].long()
        mp.mp_kv_append(self.cache, k, v, page * PAGE + positions % PAGE, positions=positions, freqs=self.freqs, q=q,
                        amplitude=self.amplitude)
        out = x.new_empty(q.shape)
        mp.mp_kv_attend(self.cache, q, table, (positions + 1).int(), out)
        y = torch.empty_like(x)
        mp.mp_linear(out.flatten(1), self.o_proj, y, residual=x)
        return self.ff.forward(y)[0]


def main(prompt=96, steps=8, sequences=4, seed=0, say=print):
    spec = family_spec("qwen2.5-1.5b", n_layers=1, vocab=256)
    base, experts = make_family_device(spec, seed=seed)
    width = -(-(prompt + steps) // PAGE)
    block = Block(spec, merge(spec, base, experts), pages=(sequences + 1) * width)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda", dtype=torch.bfloat16)  # noqa: E731
    table = torch.randperm((sequences + 1) * width, generator=gen, device="cuda").int().view(sequences + 1, width)

    # a prompt: its tokens are rows of one sequence, each with the keys up to its own
    hidden = block.o_proj.shape[0]
    x = rand(prompt, hidden)
    at = torch.arange(prompt, device="cuda")
    whole = block.forward(x, at, table[:1].expand(prompt, -1).contiguous())

    # the same tokens one by one in another sequence's pages
    single = torch.cat([block.forward(x[i:i + 1], at[i:i + 1], table[1:2]) for i in range(prompt)])
    apart = float((single.float() - whole.float()).norm() / whole.float().norm())
    say(f"prompt of {prompt} tokens, at once and one by one: {apart:.1e} of their norm apart")

    # single tokens of all sequences, captured once and replayed
    tokens, positions = rand(sequences, hidden), torch.zeros(sequences, dtype=torch.long, device="cuda")
    positions[0] = prompt  # after the tokens that went in one by one; the others begin
    rows = table[1:].contiguous()
    first = block.forward(tokens, positions, rows).clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = block.forward(tokens, positions, rows)
    graph.replay()
    same = torch.equal(y, first)
    for _ in range(1, steps):
        tokens.copy_(y)
        positions.add_(1)
        graph.replay()
    torch.cuda.synchronize()
    say(f"{steps} steps of {sequences} sequences, to position {int(positions.max())}: replays "
        f"{'equal' if same else 'differ from'} the eager step")

    # rotary positions alone, as training takes them: <turned q, d> = <q, d turned back>
    q = block.project(x)[0].contiguous()
    turned, back = torch.empty_like(q), torch.empty_like(q)
    mp.mp_rope(q, turned, at, block.freqs)
    d = turned + rand(*q.shape)  # so that both sides are of the products' size
    mp.mp_rope_backward(d, back, at, block.freqs)
    dots = [float((a.double() * b.double()).sum()) for a, b in ((turned, d), (q, back))]
    scale = float((q.double() * d.double()).abs().sum())
    say(f"rotary gradient: {abs(dots[0] - dots[1]) / scale:.1e} of the products' size apart")
    return y, same, apart, dots, scale


if __name__ == "__main__":
    main()
