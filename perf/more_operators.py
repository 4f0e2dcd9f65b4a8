"""Timing cases of the operators that put attention beside a checkpoint's
feed-forward part: rotary positions, a paged cache of keys and values, and the
attention of new tokens over it.

  rope       each pair of a head's first `rot` values turned by its token's
             position times the pair's frequency
  rope_back  the gradient: turned back
  append     new tokens' keys, turned, and values into the pages of a cache,
             and their queries turned
  attend     one new token per sequence over the sequence's pages; groups of
             query heads share a head of keys and values

``run`` computes them with the library's entry points where ``own`` is true, and
else in their plain form: elementary operations in 32 bits (angles in 64),
rounded once.  Queries and keys are N(0, 1) with a few channels that are
larger, as the projections of the checkpoint families give them.
"""

import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
OPS = ("rope", "rope_back", "append", "attend", "attend")
SCALINGS = ("none", "linear", "parts", "yarn")
MOST_VALUES = 5.0e7  # tokens x heads x dim of a drawn rotation or append; f32 cases half of each
MOST_CACHE = 5.0e8   # values that a drawn attention reads, fewer for groups of more than 8 heads


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # one token's queries and keys, side by side in a row of the packed projection of a 1.5B-parameter model
        dict(name="rope-1-token", op="rope", dtype="bf16", tokens=1, heads=14, dim=128, rot=128, interleaved=False,
             scaling="none", base=1e6, start=30011, restart=1, pad=256),
        # a training batch of sequences through a 7B-parameter model's queries and keys
        dict(name="rope-batch", op="rope", dtype="bf16", tokens=16384, heads=32, dim=128, rot=128, interleaved=False,
             scaling="none", base=1e6, start=0, restart=4096, pad=512),
        # the same of an 8B-parameter model with a context extended by parts, backward
        dict(name="rope-back", op="rope_back", dtype="bf16", tokens=8192, heads=40, dim=128, rot=128,
             interleaved=False, scaling="parts", base=5e5, start=0, restart=8192, pad=0),
        # an fp32 model that turns adjacent values of part of an odd head, far out, in rows of wider buffers
        dict(name="rope-back-f32-odd", op="rope_back", dtype="f32", tokens=777, heads=5, dim=101, rot=52,
             interleaved=True, scaling="yarn", base=1e4, start=1000003, restart=500, pad=7),
        # one new token for each of 64 sequences of a 7B-parameter model
        dict(name="append-64-tokens", op="append", dtype="bf16", tokens=64, heads=4, group=7, dim=128, rot=128,
             interleaved=False, scaling="none", base=1e6, start=0, restart=0, page=16, heads_first=False, skip=0),
        # a chunk of prompts of an 8B-parameter model, a few tokens of padding among them
        dict(name="append-prompt", op="append", dtype="bf16", tokens=8192, heads=8, group=4, dim=128, rot=128,
             interleaved=False, scaling="parts", base=5e5, start=4096, restart=2048, page=64, heads_first=True,
             skip=37),
        # an fp32 model of odd sizes, pages of ten tokens
        dict(name="append-f32-odd", op="append", dtype="f32", tokens=333, heads=3, group=3, dim=72, rot=36,
             interleaved=True, scaling="linear", base=1e4, start=17, restart=111, page=10, heads_first=False, skip=5),
        # the first tokens of a dialogue with a 1.5B-parameter model
        dict(name="attend-short", op="attend", dtype="bf16", seqs=1, longest=37, ragged=False, heads=2, group=6,
             dim=128, page=16, heads_first=False, window=0, lse=False),
        # one sequence of a 7B-parameter model at the end of a long context
        dict(name="attend-long", op="attend", dtype="bf16", seqs=1, longest=131072, ragged=False, heads=4, group=7,
             dim=128, page=16, heads_first=False, window=0, lse=False),
        # a server's batch of ragged dialogues, 8B-parameter shape
        dict(name="attend-batch", op="attend", dtype="bf16", seqs=64, longest=8192, ragged=True, heads=8, group=4,
             dim=128, page=64, heads_first=True, window=0, lse=False),
        # many short sequences, every query head with keys of its own
        dict(name="attend-many", op="attend", dtype="bf16", seqs=256, longest=700, ragged=True, heads=16, group=1,
             dim=64, page=32, heads_first=False, window=0, lse=False),
        # an fp32 model of odd sizes with a sliding window, pages of ten tokens
        dict(name="attend-f32-odd", op="attend", dtype="f32", seqs=7, longest=3001, ragged=True, heads=3, group=3,
             dim=72, page=10, heads_first=False, window=2000, lse=True),
    ]


def _log(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm; a third of them multiples of 16."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if n > 16 and rng.random() < 1 / 3:
        n = n // 16 * 16
    return min(max(n, lo), hi)


def _dims(rng):
    """Head size and the part of it that is turned."""
    dim = rng.choice((64, 128, 128, 128, 256, 8 * rng.randrange(1, 33), rng.randrange(2, 257)))
    rot = dim // 2 * 2 if rng.random() < 0.6 else 2 * rng.randrange(1, dim // 2 + 1)
    return dim, rot


def draw(rng):
    op = rng.choice(OPS)
    dtype = "bf16" if rng.random() < 0.75 else "f32"
    coin = lambda p=0.5: rng.random() < p  # noqa: E731
    share = 1.0 if dtype == "bf16" else 0.5
    if op == "attend":
        group = rng.choice((1, 2, 4, 7, 8, rng.randrange(1, 17), rng.randrange(17, 49)))
        while True:
            seqs, longest, heads = _log(rng, 1, 256), _log(rng, 1, 131072), _log(rng, 1, 32)
            dim, _ = _dims(rng)
            if 2.0 * seqs * longest * heads * dim * max(1.0, group / 8) <= MOST_CACHE * share:
                break
        return dict(op=op, dtype=dtype, seqs=seqs, longest=longest, ragged=coin(0.7), heads=heads, group=group, dim=dim,
                    page=rng.choice((16, 16, 32, 64, 128, 1, rng.randrange(2, 100))), heads_first=coin(),
                    window=0 if coin(0.75) else _log(rng, 1, 2 * longest), lse=coin(0.3))
    while True:
        tokens, heads = _log(rng, 1, 32768), _log(rng, 1, 64 if op != "append" else 32)
        group = rng.choice((1, 4, 7, rng.randrange(1, 9)))
        dim, rot = _dims(rng)
        if tokens * heads * (group + 2 if op == "append" else 1) * dim <= MOST_VALUES * share:
            break
    case = dict(op=op, dtype=dtype, tokens=tokens, heads=heads, dim=dim, rot=rot, interleaved=coin(),
                scaling=rng.choice(SCALINGS), base=rng.choice((1e4, 5e5, 1e6)),
                start=rng.choice((0, _log(rng, 1, 10 ** 7))), restart=rng.choice((0, _log(rng, 1, 32768))))
    if op == "append":
        return dict(case, group=group, page=rng.choice((16, 16, 32, 64, 128, 1, rng.randrange(2, 100))),
                    heads_first=coin(), skip=rng.choice((0, rng.randrange(0, tokens + 1))))
    return dict(case, pad=rng.choice((0, 0, dim, rng.randrange(1, 64))))


# ----------------------------------------------------------------- the inputs
def _frequencies(case):
    """Radians per position of each pair, and the factor that the turned values take."""
    half, scaling = case["rot"] // 2, case["scaling"]
    f = case["base"] ** (-torch.arange(half, dtype=torch.float64) / half)
    if scaling == "linear":
        return f / 4, 1.0
    if scaling == "parts":  # slow pairs slowed by 8, fast ones kept, between them by their turns in 8192 tokens
        turns = 8192 * f / (2 * math.pi)
        keep = ((turns - 1) / (4 - 1)).clamp(0, 1)
        return f * keep + f / 8 * (1 - keep), 1.0
    if scaling == "yarn":  # the same between pair numbers, over 4096 tokens and by 16
        at = lambda turns: half * math.log(4096 / (turns * 2 * math.pi)) / math.log(case["base"])  # noqa: E731
        lo, hi = max(math.floor(at(32)), 0), min(math.ceil(at(1)), case["rot"] - 1)
        slow = ((torch.arange(half, dtype=torch.float64) - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
        return f / 16 * slow + f * (1 - slow), 0.1 * math.log(16) + 1
    return f, 1.0


def _lens(case):
    """Lengths of the sequences, spread evenly over [1, longest]."""
    n, longest = case["seqs"], case["longest"]
    if not case["ragged"]:
        return [longest] * n
    return [longest if i == 0 else 1 + int((longest - 1) * (i * 0.6180339887498949 % 1.0)) for i in range(n)]


def _reach(case):
    """Keys that each sequence's token reads."""
    return [min(n, case["window"]) if case["window"] else n for n in _lens(case)]


def prepare(case, seed):
    """Inputs, and the buffers that the outputs go to."""
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    dt = DTYPES[case["dtype"]]
    dim = case["dim"]

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda", dtype=dt)

    def projected(rows, heads, pad=0):
        """rows x heads x dim values, each row `pad` values before the next."""
        t = torch.zeros(rows, heads * dim + pad, dtype=dt, device="cuda")[:, :heads * dim].unflatten(1, (heads, dim))
        t.copy_(normal(rows, heads, dim))
        t[:, :, torch.randint(0, dim, (max(1, dim // 64),), generator=g, device="cuda")] *= 3
        return t

    def cache(pages):
        """keys or values: pages x page x heads x dim, in memory so or with the heads before a page's tokens."""
        p, h = case["page"], case["heads"]
        return normal(pages, h, p, dim).transpose(1, 2) if case["heads_first"] else normal(pages, p, h, dim)

    s = dict(case)
    if case["op"] == "attend":
        order = list(range(case["seqs"]))
        random.Random(int(seed)).shuffle(order)
        lens = [_lens(case)[i] for i in order]
        need = [-(-n // case["page"]) for n in lens]
        pages = sum(need) + 3
        at = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        table = torch.zeros(len(lens), max(need) + 1, dtype=torch.int32, device="cuda")
        row = torch.repeat_interleave(torch.arange(len(lens)), torch.tensor(need))
        first = torch.cumsum(torch.tensor(need), 0) - torch.tensor(need)
        col = torch.arange(sum(need)) - first[row]
        table[row.cuda(), col.cuda()] = at[:sum(need)]
        q = projected(len(lens), case["heads"] * case["group"])
        s.update(host_lens=lens, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), table=table, q=q,
                 k=cache(pages), v=cache(pages), scale=dim ** -0.5, out=torch.zeros_like(q),
                 stat=torch.zeros(q.shape[:2], device="cuda") if case["lse"] else None)
        return s
    n = case["tokens"]
    f, amplitude = _frequencies(case)
    if case["op"] == "append" and case["restart"] == 0:  # one new token of each sequence
        pos = torch.randint(0, case["start"] + 32768, (n,), generator=g, device="cuda")
    else:
        pos = case["start"] + torch.arange(n, device="cuda") % (case["restart"] or n)
    s.update(freqs=f.cuda(), amplitude=amplitude, positions=pos)
    if case["op"] != "append":
        s.update(x=projected(n, case["heads"], case["pad"]), y=projected(n, case["heads"], case["pad"]))
        return s
    pages = -(-n // case["page"]) + 2
    slots = torch.randperm(pages * case["page"], generator=g, device="cuda")[:n]
    slots[torch.randperm(n, generator=g, device="cuda")[:case["skip"]]] = -1
    qkv = projected(n, case["heads"] * (case["group"] + 2))
    cut = (case["heads"] * case["group"], case["heads"], case["heads"])
    q, k, v = torch.split(qkv, cut, 1)
    s.update(q=q, k_new=k, v_new=v, slots=slots, q_out=torch.zeros_like(q.contiguous()), k=cache(pages), v=cache(pages))
    return s


# ------------------------------------------------------------- the plain form
def _plain_turn(s, x, back=False):
    t = s["positions"].double()[:, None] * s["freqs"][None]
    t = t - 2 * math.pi * torch.round(t / (2 * math.pi))
    c, n = torch.cos(t).float()[:, None] * s["amplitude"], torch.sin(t).float()[:, None] * s["amplitude"]
    if back:
        n = -n
    rot = s["rot"]
    y = x.float().clone()
    if s["interleaved"]:
        a, b = slice(0, rot, 2), slice(1, rot, 2)
    else:
        a, b = slice(0, rot // 2), slice(rot // 2, rot)
    xa, xb = x[:, :, a].float(), x[:, :, b].float()
    y[:, :, a] = xa * c - xb * n
    y[:, :, b] = xa * n + xb * c
    return y.to(x.dtype)


def _plain_append(s):
    kept = torch.nonzero(s["slots"] >= 0)[:, 0]
    slot = s["slots"][kept]
    page, at = torch.div(slot, s["page"], rounding_mode="floor"), slot % s["page"]
    s["k"][page, at] = _plain_turn(s, s["k_new"])[kept]
    s["v"][page, at] = s["v_new"][kept]
    return {"q": _plain_turn(s, s["q"]), "k": s["k"], "v": s["v"]}


def _plain_attend(s):
    h, p = s["heads"], s["page"]
    for i, n in enumerate(s["host_lens"]):
        lo = max(0, n - s["window"]) if s["window"] else 0
        pages = s["table"][i, lo // p:-(-n // p)].long()
        cut = slice(lo - lo // p * p, n - lo // p * p)
        k = s["k"][pages].flatten(0, 1)[cut].float().transpose(0, 1).contiguous()
        v = s["v"][pages].flatten(0, 1)[cut].float().transpose(0, 1).contiguous()
        score = torch.matmul(s["q"][i].float().view(h, -1, s["dim"]), k.transpose(1, 2).contiguous()) * s["scale"]
        top = score.amax(2, keepdim=True)
        e = torch.exp(score - top)
        total = e.sum(2, keepdim=True)
        s["out"][i] = (torch.matmul(e, v) / total).view(-1, s["dim"]).to(s["out"].dtype)
        if s["stat"] is not None:
            s["stat"][i] = (top + torch.log(total)).view(-1)
    return {"out": s["out"], "lse": s["stat"]}


# ------------------------------------------------------ the library's kernels
def _own(s):
    import paper_2605_29489_amd as mp

    if s["op"] == "attend":
        kv = mp.KvCache(s["k"], s["v"])
        if "workspace" not in s:
            need = mp.mp_kv_attend_workspace(kv, s["q"].shape[0], s["q"].shape[1], s["table"].shape[1], s["window"])
            s["workspace"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
        mp.mp_kv_attend(kv, s["q"], s["table"], s["lens"], s["out"], scale=s["scale"], window=s["window"],
                        lse=s["stat"], workspace=s["workspace"])
        return {"out": s["out"], "lse": s["stat"]}
    turn = dict(interleaved=s["interleaved"], amplitude=s["amplitude"])
    if s["op"] == "append":
        mp.mp_kv_append(mp.KvCache(s["k"], s["v"]), s["k_new"], s["v_new"], s["slots"], positions=s["positions"],
                        freqs=s["freqs"], q=s["q"], q_out=s["q_out"], **turn)
        return {"q": s["q_out"], "k": s["k"], "v": s["v"]}
    call = mp.mp_rope if s["op"] == "rope" else mp.mp_rope_backward
    call(s["x"], s["y"], s["positions"], s["freqs"], **turn)
    return {"y": s["y"]}


def run(state):
    if own:
        return _own(state)
    if state["op"] == "attend":
        return _plain_attend(state)
    if state["op"] == "append":
        return _plain_append(state)
    return {"y": _plain_turn(state, state["x"], state["op"] == "rope_back")}


# ------------------------------------------------------------------- the work
def work(case):
    """Bytes and operations of one pass: every input read once, every output written once."""
    es, dim = BYTES[case["dtype"]], case["dim"]
    if case["op"] == "attend":
        keys, hq = sum(_reach(case)), case["heads"] * case["group"]
        return {"bytes": es * dim * (2 * keys * case["heads"] + 2 * case["seqs"] * hq) +
                4 * case["seqs"] * (hq * case["lse"] + 1) + 4 * sum(-(-n // case["page"]) for n in _reach(case)),
                "flops": 4 * keys * hq * dim}
    n, h = case["tokens"], case["heads"]
    if case["op"] == "append":
        kept = n - case["skip"]
        return {"bytes": 2 * es * dim * h * (n * case["group"] + 2 * kept) + 16 * n + 4 * case["rot"],
                "flops": 3 * case["rot"] * h * (n * case["group"] + kept)}
    return {"bytes": 2 * es * n * h * dim + 8 * n + 4 * case["rot"], "flops": 3 * case["rot"] * n * h}


# ---------------------------------------------------- the definition, 64 bits
def _exact_turn(s, x, sign):
    """Pairs as complex numbers, multiplied by amplitude e^(i sign t)."""
    rot = s["rot"]
    x = x.double()
    pairs = x[:, :, :rot].unflatten(2, (rot // 2, 2) if s["interleaved"] else (2, rot // 2))
    if not s["interleaved"]:
        pairs = pairs.transpose(2, 3)
    angle = torch.outer(s["positions"].double(), s["freqs"]) * sign
    turn = torch.polar(torch.full_like(angle, s["amplitude"]), angle)
    turned = torch.view_as_complex(pairs.contiguous()) * turn[:, None]
    pairs = torch.view_as_real(turned)
    if not s["interleaved"]:
        pairs = pairs.transpose(2, 3)
    return torch.cat((pairs.flatten(2), x[:, :, rot:]), 2)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("rope", "rope_back"):
        return {"y": _exact_turn(s, s["x"], 1 if case["op"] == "rope" else -1)}
    if case["op"] == "append":
        k, v = s["k"].double(), s["v"].double()
        new_k, new_v = _exact_turn(s, s["k_new"], 1), s["v_new"].double()
        for i, slot in enumerate(s["slots"].tolist()):
            if slot >= 0:
                k[slot // case["page"], slot % case["page"]] = new_k[i]
                v[slot // case["page"], slot % case["page"]] = new_v[i]
        return {"q": _exact_turn(s, s["q"], 1), "k": k, "v": v}
    out, stat = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda"), None
    if case["lse"]:
        stat = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    for i, n in enumerate(s["host_lens"]):
        at = torch.arange(max(0, n - case["window"]) if case["window"] else 0, n, device="cuda")
        page, slot = s["table"][i][at // case["page"]].long(), at % case["page"]
        for h in range(case["heads"]):
            heads = slice(h * case["group"], (h + 1) * case["group"])
            score = torch.mm(s["k"][page, slot, h].double(), s["q"][i, heads].double().T.contiguous()) * s["scale"]
            total = torch.logsumexp(score, 0)
            out[i, heads] = torch.mm(torch.exp(score - total).T.contiguous(), s["v"][page, slot, h].double())
            if case["lse"]:
                stat[i, heads] = total
    return {"out": out, "lse": stat}
