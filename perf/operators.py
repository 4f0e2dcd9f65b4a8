"""Timing cases of the operators that run a checkpoint's feed-forward part: what
follows a merge.

  linear       y = act(x w^T + b) + r over a checkpoint's weight matrix, from
               single tokens to long prompts; with keep, the pre-activations
               z = x w^T + b are stored for a backward pass
  linear_back  the gradients of x, w and b
  norm         layer norm or RMS norm with its per-row statistics
  norm_back    the gradients of x, the weight and the bias
  moe          a few tokens through a router and the feed-forward tensors of E
               experts, read where their checkpoints hold them

``run`` computes them with the library's entry points where ``own`` is true, and
else in their plain form: elementary operations in 32 bits, rounded once.
Weights are N(0, 0.02^2) and norm weights about 1, as in the checkpoint
families; activations are N(0, 1) with a few channels that are much larger.
"""

import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
OPS = ("linear", "linear_back", "norm", "norm_back", "moe")
MOST_FLOPS = 5.0e11   # of a drawn case; f32 cases a tenth
MOST_VALUES = 5.5e7   # rows x columns of a drawn norm
MOST_WEIGHTS = 1.5e9  # values of a drawn case's experts


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # one token through the down projection of a 1.5B-parameter model, added to the residual stream
        dict(name="linear-1-token", op="linear", dtype="bf16", m=1, n=1536, k=8960, act="none", bias=False,
             residual=True, keep=False, pad=0),
        # a small batch of tokens through the same model's gate projection
        dict(name="linear-13-tokens", op="linear", dtype="bf16", m=13, n=8960, k=1536, act="silu", bias=False,
             residual=False, keep=False, pad=0),
        # a long prompt, or a training batch, through the up projection of a 7B-parameter model
        dict(name="linear-prompt", op="linear", dtype="bf16", m=4096, n=18944, k=3584, act="gelu_tanh", bias=True,
             residual=False, keep=True, pad=0),
        # an fp32 model of odd sizes, rows inside wider buffers
        dict(name="linear-f32-odd", op="linear", dtype="f32", m=777, n=515, k=1029, act="gelu", bias=True,
             residual=True, keep=True, pad=3),
        # a training step's backward pass through the 1.5B-parameter model's gate projection
        dict(name="linear-back", op="linear_back", dtype="bf16", m=8192, n=8960, k=1536, act="silu", bias=True, pad=0),
        # a short ragged batch, odd sizes
        dict(name="linear-back-odd", op="linear_back", dtype="bf16", m=509, n=1001, k=777, act="gelu", bias=True, pad=1),
        # a training batch through a norm of a 7B-parameter model's width
        dict(name="norm", op="norm", dtype="bf16", rows=16384, cols=3584, rms=False, bias=True, pad=0),
        # and back, at the 1.5B-parameter model's width
        dict(name="norm-back", op="norm_back", dtype="bf16", rows=16384, cols=1536, rms=False, bias=True, pad=0),
        # few fp32 rows of an odd length
        dict(name="norm-back-f32-odd", op="norm_back", dtype="f32", rows=1001, cols=8961, rms=True, bias=False, pad=0),
        # one token, two of eight experts of the 1.5B-parameter shape
        dict(name="moe-1-token", op="moe", dtype="bf16", tokens=1, hidden=1536, ffn=8960, experts=8, top=2, gated=True,
             act="silu", renorm=True, bias=False, residual=True),
        # a batch of tokens that reaches every expert of the 7B-parameter shape
        dict(name="moe-24-tokens", op="moe", dtype="bf16", tokens=24, hidden=3584, ffn=18944, experts=8, top=2,
             gated=True, act="silu", renorm=True, bias=False, residual=True),
        # many small fp32 experts of odd sizes, no gate
        dict(name="moe-f32-odd", op="moe", dtype="f32", tokens=7, hidden=515, ffn=1030, experts=21, top=3, gated=False,
             act="gelu", renorm=False, bias=True, residual=False),
    ]


def _log(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm; a third of them multiples of 64."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if n > 64 and rng.random() < 1 / 3:
        n = n // 64 * 64
    n = min(max(n, lo), hi)
    return n + 1 if n == 3072 else n


def draw(rng):
    op = rng.choice(OPS)
    dtype = "bf16" if rng.random() < 0.75 else "f32"
    coin = lambda: rng.random() < 0.5  # noqa: E731
    if op in ("linear", "linear_back"):
        most = MOST_FLOPS * (1.0 if dtype == "bf16" else 0.1) / (2 if op == "linear" else 4)
        while True:
            m, n, k = _log(rng, 1, 8192), _log(rng, 64, 20000), _log(rng, 64, 20000)
            if m * n * k <= most:
                break
        pad = rng.choice((0, 0, 8, rng.randrange(1, 64)))
        case = dict(op=op, dtype=dtype, m=m, n=n, k=k, act=rng.choice(ACTS), bias=coin(), pad=pad)
        return case if op == "linear_back" else dict(case, residual=coin(), keep=coin())
    if op in ("norm", "norm_back"):
        while True:
            rows, cols = _log(rng, 1, 32768), _log(rng, 1, 18944)
            if rows * cols <= MOST_VALUES:
                break
        return dict(op=op, dtype=dtype, rows=rows, cols=cols, rms=coin(), bias=coin(),
                    pad=rng.choice((0, 0, 8, rng.randrange(1, 64))))
    while True:
        hidden, ffn, experts = _log(rng, 64, 4096), _log(rng, 64, 18944), rng.randrange(1, 33)
        gated = coin()
        if hidden * ffn * experts * (3 if gated else 2) <= MOST_WEIGHTS * (1.0 if dtype == "bf16" else 0.5):
            break
    return dict(op="moe", dtype=dtype, tokens=_log(rng, 1, 64), hidden=hidden, ffn=ffn, experts=experts,
                top=rng.randrange(1, min(experts, 8) + 1), gated=gated, act=rng.choice(ACTS), renorm=coin(),
                bias=coin(), residual=coin())


# ----------------------------------------------------------------- the inputs
def prepare(case, seed):
    """Inputs, and the buffers that the outputs go to."""
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    dt = DTYPES[case["dtype"]]
    pad = int(case.get("pad", 0))

    def normal(*shape, std=1.0, mean=0.0):
        t = torch.randn(*shape, generator=g, device="cuda", dtype=dt)
        return t.mul_(std).add_(mean) if mean else t.mul_(std)

    def wide(rows, cols):
        """A buffer of rows x cols values, each row `pad` values before the next."""
        return torch.zeros(rows, cols + pad, dtype=dt, device="cuda")[:, :cols]

    def activations(rows, cols):
        t = wide(rows, cols)
        t.copy_(normal(rows, cols))
        big = torch.randint(0, cols, (max(1, cols // 512),), generator=g, device="cuda")
        t[:, big] *= 8
        return t

    s = dict(case)
    op = case["op"]
    if op in ("linear", "linear_back"):
        m, n, k = case["m"], case["n"], case["k"]
        s.update(x=activations(m, k), w=normal(n, k, std=0.02))
        if op == "linear":
            s.update(b=normal(n, std=0.1) if case["bias"] else None,
                     r=activations(m, n) if case["residual"] else None,
                     y=wide(m, n), z=wide(m, n) if case["keep"] else None)
        else:
            z = None
            if case["act"] != "none":
                z = wide(m, n)
                z.copy_(normal(m, n))
            dy = wide(m, n)
            dy.copy_(normal(m, n, std=1e-2))
            s.update(dy=dy, z=z, dx=wide(m, k), dw=torch.zeros_like(s["w"]),
                     db=torch.zeros(n, dtype=dt, device="cuda") if case["bias"] else None)
    elif op in ("norm", "norm_back"):
        rows, cols = case["rows"], case["cols"]
        x = activations(rows, cols)
        s.update(x=x, w=normal(cols, std=0.02, mean=1.0), eps=1e-6)
        if op == "norm":
            s.update(b=normal(cols, std=0.02) if case["bias"] else None, y=wide(rows, cols),
                     mean=torch.zeros(rows, device="cuda"), rstd=torch.zeros(rows, device="cuda"))
        else:
            mean, rstd = _statistics(x.float(), case["rms"], s["eps"])
            dy = wide(rows, cols)
            dy.copy_(normal(rows, cols, std=1e-2))
            s.update(dy=dy, mean=mean, rstd=rstd, dx=wide(rows, cols), dw=torch.zeros_like(s["w"]),
                     db=torch.zeros_like(s["w"]) if case["bias"] else None)
    else:
        t, d, f, e = case["tokens"], case["hidden"], case["ffn"], case["experts"]
        # E checkpoints; each holds gate (F x D), up (F x D, if gated) and down (D x F) back to back
        flat = normal(e, (3 if case["gated"] else 2) * d * f, std=0.02)
        s.update(x=activations(t, d), router=normal(e, d, std=0.02), flat=flat, experts_list=list(flat.unbind(0)),
                 rb=normal(e, std=0.1) if case["bias"] else None,
                 r=activations(t, d) if case["residual"] else None, y=torch.zeros(t, d, dtype=dt, device="cuda"),
                 ids=torch.zeros(t, case["top"], dtype=torch.int32, device="cuda"),
                 gates=torch.zeros(t, case["top"], device="cuda"))
    return s


# ------------------------------------------------------------- the plain form
def _act(z, name):
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _slope(z, name):
    """d act / d z."""
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * math.sqrt(0.5 / math.pi)
    if name == "gelu_tanh":
        c = math.sqrt(2 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    if name == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 + z * (1 - p))
    return torch.ones_like(z)


def _statistics(x, rms, eps):
    mean = torch.zeros_like(x[:, 0]) if rms else x.mean(1)
    var = (x - mean[:, None]).square().mean(1)
    return mean, 1 / torch.sqrt(var + eps)


def _plain_linear(s):
    z = s["x"].float() @ s["w"].float().t()
    if s["b"] is not None:
        z = z + s["b"].float()
    y = _act(z, s["act"])
    if s["r"] is not None:
        y = y + s["r"].float()
    dt = s["x"].dtype
    return {"y": y.to(dt), "z": z.to(dt) if s["keep"] else None}


def _plain_linear_back(s):
    dt = s["x"].dtype
    dz = s["dy"].float()
    if s["z"] is not None:
        dz = dz * _slope(s["z"].float(), s["act"])
    return {"dx": (dz @ s["w"].float()).to(dt), "dw": (dz.t() @ s["x"].float()).to(dt),
            "db": dz.sum(0).to(dt) if s["db"] is not None else None}


def _plain_norm(s):
    x = s["x"].float()
    mean, rstd = _statistics(x, s["rms"], s["eps"])
    y = (x - mean[:, None]) * rstd[:, None] * s["w"].float()
    if s["b"] is not None:
        y = y + s["b"].float()
    return {"y": y.to(s["x"].dtype), "mean": None if s["rms"] else mean, "rstd": rstd}


def _plain_norm_back(s):
    dt = s["x"].dtype
    dy = s["dy"].float()
    xhat = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    g = dy * s["w"].float()
    dx = g - xhat * (g * xhat).mean(1, keepdim=True)
    if not s["rms"]:
        dx = dx - g.mean(1, keepdim=True)
    return {"dx": (dx * s["rstd"][:, None]).to(dt), "dw": (dy * xhat).sum(0).to(dt),
            "db": dy.sum(0).to(dt) if s["db"] is not None else None}


def _plain_moe(s):
    t, d, f, e, top, gated = (s[n] for n in ("tokens", "hidden", "ffn", "experts", "top", "gated"))
    x = s["x"].float()
    logits = x @ s["router"].float().t()
    if s["rb"] is not None:
        logits = logits + s["rb"].float()
    best, order = torch.sort(logits, dim=1, descending=True, stable=True)
    ids = order[:, :top]
    p = torch.exp(best - best[:, :1])
    gates = p[:, :top] / (p[:, :top] if s["renorm"] else p).sum(1, keepdim=True)
    flat, df = s["flat"], d * f
    if t * top < e:  # the chosen experts' weights, one copy for each choice
        at = ids.reshape(-1)
        part = lambda lo, rows, cols: flat[at, lo:lo + df].view(-1, rows, cols).float()  # noqa: E731
        xs = x.repeat_interleave(top, 0)[:, :, None]
        h = _act(torch.matmul(part(0, f, d), xs), s["act"])
        if gated:
            h = h * torch.matmul(part(df, f, d), xs)
        out = torch.matmul(part((2 if gated else 1) * df, d, f), h).view(t, top, d)
        y = (out * gates[:, :, None]).sum(1)
    else:  # every expert for every token, with a weight of 0 where it was not chosen
        part = lambda lo: flat[:, lo:lo + df].float()  # noqa: E731
        h = _act(x @ part(0).reshape(e * f, d).t(), s["act"])
        if gated:
            h = h * (x @ part(df).reshape(e * f, d).t())
        c = torch.zeros(t, e, device=x.device).scatter_(1, ids, gates)
        h = (h.view(t, e, f) * c[:, :, None]).view(t, e * f)
        down = part((2 if gated else 1) * df).view(e, d, f).transpose(1, 2).reshape(e * f, d)
        y = h @ down
    if s["r"] is not None:
        y = y + s["r"].float()
    return {"y": y.to(s["x"].dtype), "ids": ids.to(torch.int32), "gates": gates}


PLAIN = {"linear": _plain_linear, "linear_back": _plain_linear_back, "norm": _plain_norm,
         "norm_back": _plain_norm_back, "moe": _plain_moe}


# ------------------------------------------------------ the library's kernels
def _own(s):
    import paper_2605_29489_amd as mp

    op = s["op"]
    act = getattr(mp, "MP_ACT_" + s["act"].upper()) if "act" in s else 0
    if op == "linear":
        mp.mp_linear(s["x"], s["w"], s["y"], bias=s["b"], residual=s["r"], act=act, z=s["z"])
        return {"y": s["y"], "z": s["z"]}
    if op == "linear_back":
        mp.mp_linear_backward(s["dy"], s["x"], s["w"], z=s["z"], act=act, dx=s["dx"], dw=s["dw"], dbias=s["db"])
        return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}
    if op == "norm":
        mp.mp_norm(s["x"], s["y"], weight=s["w"], bias=s["b"], eps=s["eps"], rms=s["rms"],
                   mean=None if s["rms"] else s["mean"], rstd=s["rstd"])
        return {"y": s["y"], "mean": None if s["rms"] else s["mean"], "rstd": s["rstd"]}
    if op == "norm_back":
        mp.mp_norm_backward(s["dy"], s["x"], s["rstd"], mean=None if s["rms"] else s["mean"], weight=s["w"],
                            rms=s["rms"], dx=s["dx"], dweight=s["dw"], dbias=s["db"])
        return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}
    df = s["hidden"] * s["ffn"]
    layer = mp.MoeLayer(hidden=s["hidden"], ffn=s["ffn"], top_k=s["top"], gate_off=0,
                        up_off=df if s["gated"] else None, down_off=2 * df if s["gated"] else df, act=act,
                        renorm=s["renorm"])
    mp.mp_moe(layer, s["x"], s["router"], s["experts_list"], s["y"], ids=s["ids"], gates=s["gates"],
              router_bias=s["rb"], residual=s["r"])
    return {"y": s["y"], "ids": s["ids"], "gates": s["gates"]}


def run(state):
    return _own(state) if own else PLAIN[state["op"]](state)


# ------------------------------------------------------------------- the work
def work(case):
    """Bytes and operations of one pass: every input read once, every output written once."""
    es, op = BYTES[case["dtype"]], case["op"]
    if op == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": es * (m * k + n * k + m * n * (1 + case["residual"] + case["keep"]) + n * case["bias"]),
                "flops": 2 * m * n * k}
    if op == "linear_back":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": es * (2 * m * k + 2 * n * k + m * n * (1 + (case["act"] != "none")) + n * case["bias"]),
                "flops": 4 * m * n * k}
    if op in ("norm", "norm_back"):
        r, c = case["rows"], case["cols"]
        back = op == "norm_back"
        return {"bytes": es * ((3 if back else 2) * r * c + (2 if back else 1) * c * (1 + case["bias"])) +
                4 * r * (1 if case["rms"] else 2),
                "flops": (11 if back else 8) * r * c}
    t, d, f, e, top = (case[n] for n in ("tokens", "hidden", "ffn", "experts", "top"))
    mats = 3 if case["gated"] else 2
    reached = e * (1 - (1 - top / e) ** t)  # experts that a token reaches, were the choices even
    return {"bytes": es * (reached * mats * d * f + e * d + t * d * (2 + case["residual"])) + 8 * t * top,
            "flops": 2 * mats * d * f * t * top + 2 * t * d * e}


# ---------------------------------------------------- the definition, 64 bits
def _exact_act(z, name, slope=False):
    """act(z) or its derivative from the normal distribution's and the logistic function."""
    if name == "none":
        return torch.ones_like(z) if slope else z
    if name == "relu":
        return torch.heaviside(z, torch.zeros_like(z)) if slope else z.clamp(min=0)
    if name == "gelu":
        cdf = torch.special.ndtr(z)
        return cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi) if slope else z * cdf
    # x sigmoid(a(x)): silu has a(x) = x, and (1 + tanh u) / 2 = sigmoid(2 u)
    a = z if name == "silu" else math.sqrt(8 / math.pi) * (z + 0.044715 * z ** 3)
    da = 1.0 if name == "silu" else math.sqrt(8 / math.pi) * (1 + 0.134145 * z ** 2)
    p = torch.sigmoid(a)
    return p + z * p * (1 - p) * da if slope else z * p


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    up = lambda n: s[n].double() if s[n] is not None else 0.0  # noqa: E731
    if op == "linear":
        z = torch.mm(up("x"), up("w").T.contiguous()) + up("b")
        return {"y": _exact_act(z, case["act"]) + up("r"), "z": z if case["keep"] else None}
    if op == "linear_back":
        dz = up("dy") if s["z"] is None else up("dy") * _exact_act(up("z"), case["act"], True)
        return {"dx": torch.mm(dz, up("w")), "dw": torch.mm(dz.T.contiguous(), up("x")),
                "db": dz.sum(0) if case["bias"] else None}
    if op == "norm":
        x = up("x")
        mean = x.sum(1) / x.shape[1] * (0 if case["rms"] else 1)
        power = (x * x).sum(1) / x.shape[1] - mean ** 2
        rstd = (power + s["eps"]) ** -0.5
        return {"y": torch.addcmul(up("b") * torch.ones_like(x), x.sub(mean[:, None]).mul(rstd[:, None]), up("w")),
                "mean": None if case["rms"] else mean, "rstd": rstd}
    if op == "norm_back":
        # y_j = w_j n_j with n = c rstd, c = x - mean: the chain rule through rstd, then through the mean
        c, r, n = up("x") - up("mean")[:, None], up("rstd")[:, None], case["cols"]
        dn = up("dy") * up("w")
        dc = dn * r - c * r ** 3 * torch.sum(dn * c, 1, keepdim=True) / n
        # the centred row sums to nothing, so that only the first term of dc reaches the mean
        return {"dx": dc if case["rms"] else dc - torch.sum(dn, 1, keepdim=True) * r / n,
                "dw": torch.sum(up("dy") * c * r, 0), "db": up("dy").sum(0) if case["bias"] else None}
    d, f, top = case["hidden"], case["ffn"], case["top"]
    x = up("x")
    logits = torch.mm(x, up("router").T.contiguous()) + up("rb")
    prob = torch.softmax(logits, 1)
    value, ids = torch.topk(prob, top, 1)
    gates = value / value.sum(1, keepdim=True) if case["renorm"] else value
    y = torch.zeros_like(x) + up("r")
    for e, flat in enumerate(s["experts_list"]):
        row, slot = torch.nonzero(ids == e, as_tuple=True)
        if row.numel() == 0:
            continue
        mats = list(flat.split(d * f))
        h = _exact_act(torch.mm(x[row], mats[0].view(f, d).double().T.contiguous()), case["act"])
        if case["gated"]:
            h = h * torch.mm(x[row], mats[1].view(f, d).double().T.contiguous())
        y.index_add_(0, row, torch.mm(h, mats[-1].view(d, f).double().T.contiguous()) * gates[row, slot][:, None])
    return {"y": y, "ids": None, "gates": gates}
