"""The attention entry points (mp_rope, mp_kv_append, mp_kv_attend) against
their definitions in 64 bits.

Tolerances come from the arithmetic, not from runs.
  rotation: the angle is right to 2^-25 of a half turn, so cos and sin are off by
    pi 2^-25 < 2^-23 for the angle, 4 units of 2^-23 for the function and half a
    unit for the amplitude's product: TURN = 5.5 * 2^-23 of the amplitude; the
    two products and their sum add 3 roundings of 2^-24.
  attention: a score is off by (dim + 16) * EPS * |scale| * sum |q k| + 4 EPS |s|
    (EPS = 2^-23, twice the unit roundoff: matrix cores may truncate), which
    changes p by that factor, as does the exponential (8 EPS); a difference
    from the running maximum is rounded (EPS times the largest difference), and
    the sums over n keys add (n + 64) EPS.  In bf16, p enters as two bf16
    values: 2^-16.  All of it counts against sum p |v|; numerator and
    denominator both carry it.
  Outputs are rounded once: U times the result (bf16 2^-8, fp32 2^-24).
"""

import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -23
TURN = 5.5 * EPS
U = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


@pytest.fixture(scope="module")
def mp():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2605_29489_amd as m
    return m


def _dt(name):
    import torch
    return {"bf16": torch.bfloat16, "f32": torch.float32}[name]


def _dev(a, dtype):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).to(_dt(dtype)).cuda()


def _host(t):
    return t.double().cpu().numpy()


def _near(got, want, tol, what):
    got = _host(got)
    assert got.shape == want.shape, what
    with np.errstate(invalid="ignore"):
        bad = ~((np.abs(got - want) <= tol) | (got == want) | (np.isnan(got) & np.isnan(want)))
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.size} outside, first at {np.argwhere(bad)[0]}: "
                           f"{got[bad][0]} for {want[bad][0]}, tolerance {np.broadcast_to(tol, bad.shape)[bad][0]}")


def _equal(a, b):
    """The same bits (NaN included)."""
    import torch
    w = torch.int16 if a.element_size() == 2 else torch.int32
    return torch.equal(a.contiguous().view(w), b.contiguous().view(w))


# ------------------------------------------------------------------ rotary positions
def _turn(x, pos, freqs, interleaved, amp, back=False):
    """y and its tolerance without the final rounding; angles in extended precision."""
    half = len(freqs)
    t = pos.astype(np.longdouble)[:, None] * freqs.astype(np.longdouble)[None]
    two_pi = np.longdouble("6.28318530717958647692528676655900577")
    t = (t - two_pi * np.rint(t / two_pi)).astype(float)
    c, s = np.cos(t)[:, None] * amp, np.sin(t)[:, None] * amp * (-1 if back else 1)
    p, q = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    y, tol = x.copy(), np.zeros_like(x)
    a, b = x[:, :, p], x[:, :, q]
    y[:, :, p], y[:, :, q] = a * c - b * s, a * s + b * c
    tol[:, :, p] = tol[:, :, q] = abs(amp) * (np.abs(a) + np.abs(b)) * (TURN + 3 * 2.0 ** -24)
    return y, tol


def _buffer(rng, tokens, heads, dim, dtype, pad, tokens_inside):
    """tokens x heads x dim inside a buffer of NaN; its values; what of it lies between."""
    import torch
    if tokens_inside:  # heads x tokens x dim
        buf = torch.full((heads, tokens * dim + pad), float("nan"), dtype=_dt(dtype), device="cuda")
        t = buf[:, :tokens * dim].unflatten(1, (tokens, dim)).transpose(0, 1)
        between = buf[:, tokens * dim:]
    else:
        buf = torch.full((tokens, heads * dim + pad), float("nan"), dtype=_dt(dtype), device="cuda")
        t = buf[:, :heads * dim].unflatten(1, (heads, dim))
        between = buf[:, heads * dim:]
    t.copy_(torch.from_numpy(rng.standard_normal((tokens, heads, dim))))
    return t, _host(t), between


ROPE = [  # tokens, heads, dim, rot, interleaved, pad, tokens inside, first position, amplitude
    (1, 1, 2, 2, False, 0, False, 0, 1.0),
    (1, 14, 128, 128, False, 256, False, 30011, 1.0),
    (3, 2, 128, 128, True, 0, False, 5, 1.25),
    (5, 3, 64, 64, False, 8, True, 1000, 1.0),
    (33, 4, 128, 64, False, 8, False, 131071, 1.0),
    (33, 4, 128, 64, True, 0, False, 131071, 1.0),
    (70, 5, 101, 52, True, 7, False, 1000003, 1.277),
    (70, 5, 101, 52, False, 7, False, 1000003, 1.277),
    (17, 7, 80, 80, False, 0, False, 99, 1.0),
    (17, 7, 96, 48, False, 1, False, 99, 1.0),
    (19, 3, 72, 36, True, 0, True, 3, 0.5),
    (300, 40, 128, 128, False, 0, False, 0, 1.0),
    (300, 9, 256, 256, True, 3, False, -150, 1.0),
    (8, 3, 13, 0, False, 1, False, 4, 1.0),
    (9, 2, 1, 0, True, 0, False, 4, 2.0),
    (6, 2, 520, 514, False, 5, False, 7, 1.0),
    (6, 2, 4096, 4096, True, 0, False, 7, 1.0),
    (2, 70, 24, 24, False, 0, False, 2 ** 31 + 7, 1.0),
    (4, 1, 128, 128, False, 9, False, 2 ** 40, 1.0),
    (40, 3, 134, 110, False, 1, False, 77, 1.0),
    (40, 3, 140, 134, True, 0, True, 77, 1.0),
    (2000, 1, 6, 4, False, 0, False, 0, 1.0),
    (5, 300, 64, 64, False, 0, False, 9, 1.0),
]


def _freqs(rot, base=1e6):
    return base ** (-2.0 * np.arange(rot // 2) / max(rot, 1))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,heads,dim,rot,inter,pad,inside,first,amp", ROPE)
def test_rope(mp, dtype, tokens, heads, dim, rot, inter, pad, inside, first, amp):
    import torch
    rng = np.random.default_rng(tokens * 131 + dim * 7 + rot)
    x, X, _ = _buffer(rng, tokens, heads, dim, dtype, pad, inside)
    y, _, between = _buffer(rng, tokens, heads, dim, dtype, 2 * pad, False)
    pos = first + rng.permutation(tokens).astype(np.int64)
    f = _freqs(rot)
    P, F = torch.from_numpy(pos).cuda(), torch.from_numpy(f).cuda()
    # angles of positions past 2^31 carry pos f 2^-53 of the product in 64 bits, 2 pi in turns
    far = float(np.abs(pos).max()) * 2.0 ** -51
    for back in (False, True):
        call = mp.mp_rope_backward if back else mp.mp_rope
        call(x, y, P, F, interleaved=inter, amplitude=amp)
        torch.cuda.synchronize()
        want, tol = _turn(X, pos, f, inter, np.float64(np.float32(amp)), back)
        _near(y, want, tol * (1 + far / TURN) + U[dtype] * 1.01 * np.abs(want), "y")
        if rot < dim:
            assert _equal(y[:, :, rot:], x[:, :, rot:])
        assert torch.isnan(between).all()
        z = x.clone()  # keeps a dense permutation's strides
        call(z, z, P, F, interleaved=inter, amplitude=amp)
        assert _equal(z, y)
        call(x, y, P, F, interleaved=inter, amplitude=amp)
        assert _equal(z, y)  # the same bits again


def test_rope_gradient_against_the_formula_and_differences(mp):
    import torch
    rng = np.random.default_rng(5)
    pos = torch.tensor([0, 9, 70001], device="cuda")
    for inter in (False, True):
        f, amp = mp.mp_rope_frequencies(6, 1e4, mp.MP_ROPE_YARN, 16.0, 4096.0, 1.0, 32.0)
        f = f.cuda()
        x, dy = (_dev(rng.standard_normal((3, 2, 8)), "f32") for _ in range(2))
        y, dx = torch.empty_like(x), torch.empty_like(x)
        mp.mp_rope(x, y, pos, f, interleaved=inter, amplitude=amp)
        mp.mp_rope_backward(dy, dx, pos, f, interleaved=inter, amplitude=amp)
        # a linear map: <y(x), dy> = <x, dx>; each of the 48 products off by TURN and a few roundings
        a, b = (_host(y) * _host(dy)).sum(), (_host(x) * _host(dx)).sum()
        size = np.abs(_host(y)).sum() * np.abs(_host(dy)).max() + np.abs(_host(x)).sum() * np.abs(_host(dx)).max()
        assert abs(a - b) <= 2 * (TURN + 4 * EPS) * amp * size
        # differences of each input, with a step of 1 the map being linear
        for t in range(3):
            for j in range(8):
                e = torch.zeros_like(x)
                e[t, 1, j] = 1.0
                up, down = torch.empty_like(x), torch.empty_like(x)
                mp.mp_rope(x + e, up, pos, f, interleaved=inter, amplitude=amp)
                mp.mp_rope(x - e, down, pos, f, interleaved=inter, amplitude=amp)
                got = ((_host(up) - _host(down)) / 2 * _host(dy)).sum()
                mag = (np.abs(_host(x[t, 1])).sum() + 1) * amp
                assert abs(got - _host(dx[t, 1, j])) <= 4 * (TURN + 4 * EPS) * mag * np.abs(_host(dy[t, 1])).sum()


@pytest.mark.parametrize("inter", [False, True])
def test_rope_small_cosines_and_sines_keep_their_bits(mp, inter):
    """Angles near a quarter and a half turn that lie between two fp32 values: of a pair (1, 0), cos and sin themselves.
    Each is right to 4 units of 2^-23 for the function and half a unit for each of its two roundings, relative to it;
    what is added to first order leaves 2^-48 + 2^-25 pi (4.5 2^-23 + 2^-23), less than 2^-43."""
    import torch
    half = 64
    j = np.arange(1, half + 1)
    for centre in (0.5, 1.0):  # half turns
        for sign in (1, -1):
            turns = sign * (centre - j * 2.0 ** -20 - 0.45 * 2.0 ** -24)
            f = turns * math.pi
            x = torch.zeros(2, 1, 2 * half, device="cuda")
            a, b = (slice(0, None, 2), slice(1, None, 2)) if inter else (slice(0, half), slice(half, None))
            x[:, :, a] = 1.0
            y = torch.empty_like(x)
            mp.mp_rope(x, y, torch.tensor([1, -1], device="cuda"), torch.from_numpy(f).cuda(), interleaved=inter)
            for t, pos in enumerate((1, -1)):
                w = (np.longdouble(pos) * f.astype(np.longdouble))
                for got, want in ((y[t, 0, a], np.cos(w)), (y[t, 0, b], np.sin(w))):
                    want = want.astype(float)
                    _near(got, want, 5 * EPS * np.abs(want) + 2.0 ** -43, f"centre {centre}, position {pos}")


def test_rope_non_finite_values_stay_in_their_pairs(mp):
    import torch
    for dtype in ("bf16", "f32"):
        x = torch.ones(4, 3, 16, dtype=_dt(dtype), device="cuda")
        x[1, 2, 3], x[2, 0, 9] = float("nan"), float("inf")
        y = torch.empty_like(x)
        pos, f = torch.arange(1, 5, device="cuda"), torch.from_numpy(_freqs(12)).cuda()
        mp.mp_rope(x, y, pos, f)
        bad = torch.zeros(x.shape, dtype=torch.bool)
        bad[1, 2, 3] = bad[1, 2, 9] = bad[2, 0, 3] = bad[2, 0, 9] = True
        assert torch.equal(~torch.isfinite(y).cpu(), bad)


@pytest.mark.parametrize("outer", ["tokens", "heads"])
def test_rope_past_four_gib(mp, outer):
    """Tokens, or heads, far apart: offsets past 32 bits, in bytes and in elements."""
    import torch
    rng = np.random.default_rng(4)
    T, H, dim, stride = 3, 3, 64, 2 ** 31 + 8  # elements: the third is 8 GiB away
    far = (stride, dim, 1) if outer == "tokens" else (dim, stride, 1)
    try:
        x = torch.zeros(2 * stride + 3 * dim, dtype=torch.bfloat16, device="cuda").as_strided((T, H, dim), far)
    except torch.OutOfMemoryError:
        pytest.skip("not enough device memory")
    x.copy_(_dev(rng.standard_normal((T, H, dim)), "bf16"))
    near, pos, f = x.clone(memory_format=torch.contiguous_format), torch.arange(5, 5 + T, device="cuda"), _freqs(dim)
    f = torch.from_numpy(f).cuda()
    want, y = torch.empty_like(near), torch.empty_like(near)
    mp.mp_rope(near, want, pos, f)
    mp.mp_rope(x, y, pos, f)
    assert _equal(y, want)
    back = torch.empty_like(near)
    mp.mp_rope_backward(near, back, pos, f)
    mp.mp_rope_backward(x, x, pos, f)
    assert _equal(x, back)


def test_more_tokens_than_workgroups(mp):
    """A million tokens of many heads, for workgroups that take several: as in calls of a part of them each."""
    import torch
    T, heads, dim = (1 << 20) + 777, 127, 2
    x = torch.randn(T, heads + 2, dim, device="cuda").bfloat16()
    pos, f = torch.arange(T, device="cuda") * 3, torch.tensor([0.7], dtype=torch.float64, device="cuda")
    y, want = torch.empty_like(x), torch.empty_like(x)
    mp.mp_rope(x, y, pos, f)
    for a in range(0, T, 1 << 18):
        b = min(a + (1 << 18), T)
        mp.mp_rope(x[a:b], want[a:b], pos[a:b], f)
    assert _equal(y, want)
    q, k, v = torch.split(x, (heads, 1, 1), 1)
    pages, page = T // 7 + 1, 7
    c = mp.KvCache(*(torch.full((pages, page, 1, dim), float("nan"), dtype=torch.bfloat16, device="cuda")
                     for _ in range(2)))
    slots = torch.randperm(pages * page, device="cuda")[:T]
    slots[::1000] = -1
    q_out = torch.empty(T, heads, dim, dtype=torch.bfloat16, device="cuda")
    mp.mp_kv_append(c, k, v, slots, positions=pos, freqs=f, q=q, q_out=q_out)
    assert _equal(q_out, want[:, :heads])
    kept = slots >= 0
    for got, new in ((c.k, want[:, heads:heads + 1]), (c.v, v)):
        flat = got.view(pages * page, 1, dim)
        assert _equal(flat[slots[kept]], new[kept])
        assert int((~torch.isnan(flat)).sum()) == int(kept.sum()) * dim


# ------------------------------------------------------------------ the cache
def _new_cache(mp, dtype, pages, page, heads, dim, layout, rng=None):
    """A cache of NaN (or values) in one of the layouts."""
    import torch
    full = lambda *s: torch.full(s, float("nan"), dtype=_dt(dtype), device="cuda")  # noqa: E731
    if layout == "tokens":
        k, v = full(pages, page, heads, dim), full(pages, page, heads, dim)
    elif layout == "heads":
        k, v = full(pages, heads, page, dim).transpose(1, 2), full(pages, heads, page, dim).transpose(1, 2)
    elif layout == "together":  # pages x 2 x ...: keys and values of a page side by side
        kv = full(pages, 2, page, heads, dim)
        k, v = kv[:, 0], kv[:, 1]
    elif layout == "braided":  # a head's key beside its value
        kv = full(pages, page, heads, 2, dim)
        k, v = kv[:, :, :, 0], kv[:, :, :, 1]
    else:  # gaps behind heads and pages
        k, v = (full(pages, page + 1, heads, dim + 3)[:, :page, :, :dim] for _ in range(2))
    if rng is not None:
        for t in (k, v):
            t.copy_(torch.from_numpy(rng.standard_normal((pages, page, heads, dim))))
    return mp.KvCache(k, v)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,heads,group,dim,rot,inter,page,layout,skip,place", [
    (1, 1, 1, 1, 0, False, 1, "tokens", 0, "packed"),
    (1, 2, 6, 128, 128, False, 16, "tokens", 0, "packed"),
    (64, 4, 7, 128, 128, False, 16, "together", 0, "in place"),
    (37, 3, 3, 72, 36, True, 10, "gaps", 5, "apart"),
    (37, 3, 3, 72, 72, False, 10, "braided", 5, "in place"),
    (130, 2, 2, 101, 52, True, 7, "heads", 30, "packed"),
    (130, 2, 2, 101, 100, False, 64, "gaps", 130, "packed"),
    (257, 8, 4, 128, 128, True, 64, "heads", 3, "in place"),
    (41, 5, 0, 64, 64, False, 32, "tokens", 1, "packed"),
    (23, 2, 5, 256, 0, False, 16, "heads", 2, "apart"),
    (1000, 1, 1, 24, 24, False, 16, "together", 10, "apart"),
])
def test_append(mp, dtype, tokens, heads, group, dim, rot, inter, page, layout, skip, place):
    import torch
    rng = np.random.default_rng(tokens + dim)
    pages = -(-tokens // page) + 2
    c = _new_cache(mp, dtype, pages, page, heads, dim, layout)
    slots = rng.permutation(pages * page)[:tokens].astype(np.int64)
    out = rng.permutation(tokens)[:skip]
    slots[out] = rng.choice([-1, -2 ** 62, pages * page, 2 ** 62], skip)
    pos = rng.integers(0, 200000, tokens)
    S, P = torch.from_numpy(slots).cuda(), torch.from_numpy(pos).cuda()
    F = torch.from_numpy(_freqs(rot)).cuda() if rot else None
    hq = heads * group
    qkv = _dev(rng.standard_normal((tokens, hq + 2 * heads, dim)), dtype)
    q, k, v = torch.split(qkv, (hq, heads, heads), 1)
    if place == "apart":
        q, k, v = q.clone(), k.clone(), v.clone()
    q0, k0, v0 = q.clone(), k.clone(), v.clone()
    q_out = q if place == "in place" else torch.full_like(q, float("nan"), memory_format=torch.contiguous_format)
    kw = dict(interleaved=inter, amplitude=1.5)
    if group:
        mp.mp_kv_append(c, k, v, S, positions=P, freqs=F, q=q, q_out=q_out, **kw)
    else:
        mp.mp_kv_append(c, k, v, S, positions=P, freqs=F, **kw)
    torch.cuda.synchronize()
    # what is stored and returned is what mp_rope makes of it, bit for bit
    turned = []
    for t in (q0, k0):
        y = t.clone()
        if rot and t.numel():
            mp.mp_rope(y, y, P, F, **kw)
        turned.append(y)
    if group:
        assert _equal(q_out, turned[0])
    assert _equal(k, k0) and _equal(v, v0)
    kept = torch.from_numpy(np.flatnonzero((slots >= 0) & (slots < pages * page))).cuda()
    at = S[kept]
    for got, want in ((c.k, turned[1]), (c.v, v0)):
        assert _equal(got[at // page, at % page], want[kept])
        rest = got.clone()
        rest[at // page, at % page] = float("nan")
        assert torch.isnan(rest).all()
    for t in (c.k, c.v):  # gaps of the array as well
        whole = t._base if t._base is not None else t
        both = 2 if layout in ("together", "braided") else 1
        assert int((~torch.isnan(whole)).sum()) == len(kept) * heads * dim * both


def test_append_slots_named_twice(mp):
    """Of tokens with one slot each value is one of theirs, key and value alike, and nothing else is written."""
    import torch
    rng = np.random.default_rng(8)
    pages, page, heads, dim, tokens = 5, 7, 3, 72, 400
    for dtype in ("bf16", "f32"):
        c = _new_cache(mp, dtype, pages, page, heads, dim, "gaps")
        at = rng.integers(0, 20, tokens)
        k, v = (_dev(rng.standard_normal((tokens, heads, dim)), dtype) for _ in range(2))
        mp.mp_kv_append(c, k, v, torch.from_numpy(at).cuda())
        for got, new in ((_host(c.k), _host(k)), (_host(c.v), _host(v))):
            flat = got.reshape(pages * page, heads, dim)
            for slot in range(pages * page):
                if (at == slot).any():
                    assert (flat[slot] == new[at == slot]).any(0).all()
                else:
                    assert np.isnan(flat[slot]).all()


# ------------------------------------------------------------------ attention
def _attention(q, k, v, keys, scale, dtype):
    """One row: q [heads, group, dim], k and v [n, heads, dim] in 64 bits; out, lse and their tolerances."""
    h, g, d = q.shape
    n = len(keys)
    out, lse = np.zeros((h, g, d)), np.full((h, g), -np.inf)
    t_out, t_lse = np.zeros((h, g, d)), np.zeros((h, g))
    if n == 0:
        return out, lse, t_out, t_lse
    k, v = k[keys], v[keys]
    for i in range(h):
        s = scale * (q[i] @ k[:, i].T)
        ds = (d + 16) * EPS * abs(scale) * (np.abs(q[i]) @ np.abs(k[:, i]).T) + 4 * EPS * np.abs(s)
        top = s.max(1, keepdims=True)
        p = np.exp(s - top)
        total = p.sum(1, keepdims=True)
        lse[i] = (top + np.log(total))[:, 0]
        p /= total
        out[i] = p @ v[:, i]
        # keys whose p is nothing do not count: a relative error of each term, weighed by it
        rel = ds + 8 * EPS + EPS * np.abs(s - top) * 4 + (2.0 ** -16 if dtype == "bf16" else 0.0) + (n + 64) * EPS
        av = np.abs(v[:, i])
        t_out[i] = 1.05 * ((p * rel) @ av + (p * rel).sum(1, keepdims=True) * (p @ av))
        t_out[i] += U[dtype] * 1.02 * np.abs(out[i])
        t_lse[i] = 1.05 * (p * rel).sum(1) + 4 * EPS * np.abs(lse[i]) + 1e-30
    return out, lse, t_out + 1e-30, t_lse


def _paged(rng, lens, page, spare=2):
    """Pages of each row's sequence: a table whose unused places are nonsense."""
    need = [-(-n // page) for n in lens]
    pages = sum(need) + spare
    perm = rng.permutation(pages)
    table = rng.choice([-5, 0, pages, 2 ** 31 - 1], (len(lens), max(need + [0]) + 2)).astype(np.int32)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = perm[at:at + n]
        at += n
    return table, pages


def _fill(rng, cache, table, lens, page):
    """Keys and values of the rows' tokens into a cache of NaN; what it holds in 64 bits, by slot."""
    import torch
    heads, dim = cache.k.shape[2:]
    for i, n in enumerate(lens):
        j = np.arange(n)
        at = torch.from_numpy(table[i, j // page].astype(np.int64)).cuda(), torch.from_numpy(j % page).cuda()
        for t in (cache.k, cache.v):
            t[at] = _dev(rng.standard_normal((n, heads, dim)), "f32").to(t.dtype)
    flat = lambda t: _host(t).reshape(-1, heads, dim)  # noqa: E731
    return flat(cache.k), flat(cache.v)


def _slots(table_row, n, page, window, pages):
    """Slots of a row's keys."""
    j = np.arange(max(0, n - window) if window else 0, max(n, 0))
    p = table_row[j // page].astype(np.int64)
    ok = (p >= 0) & (p < pages)
    return (p * page + j % page)[ok]


ATTEND = [  # lengths, heads, group, dim, page, layout, window
    ([1], 1, 1, 1, 1, "tokens", 0),
    ([37], 2, 6, 128, 16, "tokens", 0),
    ([0, 1, 2, 15, 16, 17, 31, 32, 33], 2, 4, 128, 16, "tokens", 0),
    ([0, 0], 1, 7, 64, 16, "heads", 0),
    ([63, 64, 65, 127, 128, 129, 130], 3, 2, 64, 32, "heads", 0),
    ([500, 3, 257], 2, 7, 128, 64, "together", 0),
    ([700, 12], 4, 1, 64, 16, "braided", 0),
    ([300, 299], 1, 16, 128, 48, "tokens", 0),
    ([300, 1, 40], 1, 17, 128, 16, "gaps", 0),
    ([260, 31], 2, 33, 64, 16, "tokens", 0),
    ([200, 5], 1, 48, 256, 16, "heads", 0),
    ([2500, 1, 1023], 2, 3, 128, 16, "tokens", 0),
    ([5000], 1, 4, 128, 256, "heads", 0),
    ([3000], 2, 1, 32, 16, "tokens", 0),
    ([100, 7], 2, 3, 72, 10, "tokens", 0),
    ([100, 7], 2, 3, 101, 10, "gaps", 0),
    ([333, 1, 90], 3, 5, 80, 16, "gaps", 0),
    ([129, 4], 2, 2, 256, 7, "tokens", 0),
    ([129, 4], 1, 2, 250, 16, "heads", 0),
    ([77], 2, 8, 23, 1, "tokens", 0),
    ([65, 3], 2, 2, 13, 16, "gaps", 0),
    ([700, 40, 5, 0, 1], 2, 4, 128, 16, "tokens", 33),
    ([700, 40, 5, 0, 1], 2, 4, 96, 16, "heads", 1),
    ([1700, 600, 599], 2, 3, 72, 10, "tokens", 600),
    ([40], 1, 1, 128, 16, "tokens", 2 ** 40),
    ([90] * 300, 1, 2, 64, 16, "tokens", 0),
    ([40, 3, 200, 1, 0, 17] * 200, 1, 1, 64, 16, "tokens", 0),     # more rows than threads
    ([40, 3, 0, 1, 150] * 130, 1, 3, 128, 16, "heads", 0),
    ([9, 130] * 300, 1, 2, 72, 10, "tokens", 0),
    ([300, 2, 90, 0] * 20, 16, 1, 64, 32, "tokens", 0),            # a head a wave
    ([260, 31, 700, 5] * 10, 8, 2, 128, 16, "tokens", 0),
    ([5, 140, 33], 15, 2, 128, 16, "heads", 0),                    # sets with a wave to spare
    ([5, 340, 33, 90], 13, 3, 96, 16, "tokens", 50),
    ([5, 140, 33], 3, 20, 256, 16, "heads", 0),
    ([3, 1], 31, 38, 256, 16, "tokens", 0),
    ([4000] + [1] * 40, 8, 1, 64, 16, "heads", 0),                 # one long row among short ones
    ([1500, 20] + [3] * 290, 2, 2, 64, 16, "heads", 0),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,heads,group,dim,page,layout,window", ATTEND)
def test_attend(mp, dtype, lens, heads, group, dim, page, layout, window):
    import torch
    rng = np.random.default_rng(sum(lens) + dim)
    R, H, scale = len(lens), heads * group, 0.7 / math.sqrt(dim)
    table, pages = _paged(rng, lens, page)
    c = _new_cache(mp, dtype, pages, page, heads, dim, layout)
    K, V = _fill(rng, c, table, lens, page)
    buf = torch.full((R, H * dim + 5), float("nan"), dtype=_dt(dtype), device="cuda")
    q = _dev(rng.standard_normal((R, H, dim)) * 2, dtype)
    out = buf[:, :H * dim].unflatten(1, (H, dim))
    T, L = torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda")
    lse = torch.full((R, H), float("nan"), device="cuda")
    need = mp.mp_kv_attend_workspace(c, R, H, T.shape[1], window)
    ws = torch.full((need + 16,), 255, dtype=torch.uint8, device="cuda")  # NaN: nothing of it is taken as it comes
    mp.mp_kv_attend(c, q, T, L, out, scale=scale, window=window, lse=lse, workspace=ws[:need] if need else None)
    torch.cuda.synchronize()
    assert (ws[need:] == 255).all()
    assert torch.isnan(buf[:, H * dim:]).all()
    Q = _host(q).reshape(R, heads, group, dim)
    want = [_attention(Q[i], K, V, _slots(table[i], n, page, window, pages), scale, dtype) for i, n in enumerate(lens)]
    stack = lambda j, *s: np.stack([w[j] for w in want]).reshape(R, H, *s)  # noqa: E731
    _near(out, stack(0, dim), stack(2, dim), "out")
    _near(lse, stack(1), stack(3), "lse")
    # without lse, in place and without a workspace of the caller: the same bits
    first = out.contiguous()
    mp.mp_kv_attend(c, q, T, L, q, scale=scale, window=window)
    torch.cuda.synchronize()
    assert _equal(q, first)


ATTEND_FORMS = [  # the same: groups of more than 16 heads in every kind of page and head size, heads of few values
    ([300, 5], 2, 17, 72, 10, "tokens", 0),
    ([2500, 1], 1, 33, 48, 10, "gaps", 0),
    ([300, 31], 2, 20, 96, 16, "heads", 0),
    ([300, 31], 1, 24, 24, 16, "tokens", 0),
    ([2100, 40, 0], 2, 40, 112, 48, "gaps", 0),
    ([700, 90, 1], 3, 19, 128, 7, "together", 200),
    ([40, 3, 0, 150] * 70, 8, 17, 64, 5, "tokens", 0),
    ([260, 31] * 20, 8, 18, 80, 16, "heads", 0),
    ([3000, 17], 2, 3, 3, 10, "tokens", 0),
    ([700, 5], 1, 20, 3, 16, "tokens", 0),
    ([90] * 300, 8, 1, 7, 16, "tokens", 0),
    ([260, 0, 200] * 25, 8, 1, 3, 16, "heads", 0),
    ([2000], 3, 2, 2, 16, "braided", 0),
    ([1500, 3], 2, 5, 5, 7, "gaps", 300),
    ([900, 0, 1], 1, 33, 1, 16, "tokens", 0),
    ([1200, 77], 2, 40, 7, 10, "gaps", 0),
    ([96, 5, 90, 33], 2, 4, 128, 16, "tokens", 127),  # a window of almost all the table's four tiles
    ([96, 5, 90, 33], 2, 4, 128, 16, "tokens", 70),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,heads,group,dim,page,layout,window", ATTEND_FORMS)
def test_attend_every_form(mp, dtype, lens, heads, group, dim, page, layout, window):
    test_attend(mp, dtype, lens, heads, group, dim, page, layout, window)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page,group", [(16, 4), (10, 4), (64, 17)])
def test_attend_pages_outside_the_cache_and_lengths_out_of_range(mp, dtype, page, group):
    import torch
    rng = np.random.default_rng(page)
    heads, dim, width = 2, 64, 700 // page
    pages = 3 * width + 1
    c = _new_cache(mp, dtype, pages, page, heads, dim, "tokens", rng)
    K, V = (_host(t).reshape(-1, heads, dim) for t in (c.k, c.v))
    table = np.stack([rng.permutation(pages)[:width] for _ in range(6)]).astype(np.int32)
    table[0, ::2] = -1
    table[1, :] = pages          # no page of it is there
    table[2, 1:] = -2 ** 31
    table[3, -1] = 2 ** 31 - 1
    most = width * page
    lens = [most - 3, most, most, most, 2 ** 31 - 1, -7]
    H = heads * group
    q = _dev(rng.standard_normal((6, H, dim)), dtype)
    out, lse = torch.empty_like(q), torch.empty(6, H, device="cuda")
    L = torch.tensor(lens, dtype=torch.int32, device="cuda")
    wide = torch.full((6, width + 3), 1, dtype=torch.int32, device="cuda")  # rows of a wider table
    wide[:, :width] = torch.from_numpy(table).cuda()
    mp.mp_kv_attend(c, q, wide[:, :width], L, out, lse=lse)
    torch.cuda.synchronize()
    Q = _host(q).reshape(6, heads, group, dim)
    for i, n in enumerate(lens):
        w = _attention(Q[i], K, V, _slots(table[i], min(n, most), page, 0, pages), dim ** -0.5, dtype)
        _near(out[i], w[0].reshape(H, dim), w[2].reshape(H, dim), f"out {i}")
        _near(lse[i], w[1].reshape(H), w[3].reshape(H), f"lse {i}")
    assert (out[[1, 5]] == 0).all() and torch.isneginf(lse[[1, 5]]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_pages_named_twice(mp, dtype):
    """A page counts as often as a row names it, and rows may share pages."""
    import torch
    rng = np.random.default_rng(31)
    pages, page, heads, group, dim = 6, 16, 2, 3, 64
    lens = [150, 150, 40, 0, 97]
    table = np.array([[2] * 10, [0, 1, 2, 3, 4, 5, 0, 1, 2, 3], [2, 2, 0, 0, 0, 0, 0, 0, 0, 0], [5] * 10,
                      [4, 4, 4, 1, 1, 1, 4, 0, 0, 0]], np.int32)
    c = _new_cache(mp, dtype, pages, page, heads, dim, "heads")
    K, V = _fill(rng, c, np.arange(pages, dtype=np.int32)[None], [pages * page], page)
    q = _dev(rng.standard_normal((len(lens), heads * group, dim)), dtype)
    out, lse = torch.empty_like(q), torch.empty(len(lens), heads * group, device="cuda")
    mp.mp_kv_attend(c, q, torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), out,
                    lse=lse)
    Q = _host(q).reshape(len(lens), heads, group, dim)
    for i, n in enumerate(lens):
        w = _attention(Q[i], K, V, _slots(table[i], n, page, 0, pages), dim ** -0.5, dtype)
        _near(out[i], w[0].reshape(-1, dim), w[2].reshape(-1, dim), f"row {i}")
        _near(lse[i], w[1].reshape(-1), w[3].reshape(-1), f"row {i}")


@pytest.mark.parametrize("heads,dim,rows,n", [(16, 64, 20, 500), (8, 128, 40, 300), (2, 128, 1, 9000),
                                              (3, 256, 3, 800)])
def test_attend_infinite_values_among_exact_ones(mp, heads, dim, rows, n):
    """An infinite value reaches its own dim of the heads that read it, and changes nothing else by a bit."""
    import torch
    rng = np.random.default_rng(heads)
    page, group = 16, 2
    table, pages = _paged(rng, [n] * rows, page)
    c = _new_cache(mp, "bf16", pages, page, heads, dim, "tokens")
    _fill(rng, c, table, [n] * rows, page)
    q = _dev(rng.standard_normal((rows, heads * group, dim)), "bf16")
    T, L = torch.from_numpy(table).cuda(), torch.full((rows,), n, dtype=torch.int32, device="cuda")
    want = torch.empty_like(q)
    mp.mp_kv_attend(c, q, T, L, want)
    for row, j, h, d, x in ((0, 0, 0, 3, "inf"), (rows - 1, n - 1, heads - 1, dim - 1, "-inf"),
                            (rows // 2, n // 2, 1, 9, "nan")):
        c.v[int(table[row, j // page]), j % page, h, d] = float(x)
        want[row, h * group:(h + 1) * group, d] = float(x)
    out = torch.empty_like(q)
    mp.mp_kv_attend(c, q, T, L, out)
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(out), nan)
    assert torch.equal(out[~nan], want[~nan])


def test_attend_many_rows_of_one_sequence(mp):
    """A million rows share a table row: more workgroups than a launch holds threads for."""
    import torch
    rng = np.random.default_rng(4)
    rows, heads, dim, page = 1 << 20, 7, 64, 16
    c = _new_cache(mp, "bf16", 9, page, heads, dim, "tokens", rng)
    K, V = (_host(t).reshape(-1, heads, dim) for t in (c.k, c.v))
    table = np.array([[3, 8]], np.int32)
    q = torch.randn(rows, heads, dim, dtype=torch.bfloat16, device="cuda")
    lens = (torch.arange(rows, device="cuda") % 33).int()
    out, lse = torch.full_like(q, float("nan")), torch.full((rows, heads), float("nan"), device="cuda")
    mp.mp_kv_attend(c, q, torch.from_numpy(table).cuda().expand(rows, -1), lens, out, lse=lse)
    torch.cuda.synchronize()
    for i in [0, 1, 32, 33, 4095, 4096, 65537, rows // 2 + 5, rows - 2, rows - 1]:
        n = i % 33
        w = _attention(_host(q[i])[:, None], K, V, _slots(table[0], n, page, 0, 9), dim ** -0.5, "bf16")
        _near(out[i], w[0][:, 0], w[2][:, 0], f"out {i}")
        _near(lse[i], w[1][:, 0], w[3][:, 0], f"lse {i}")
    assert not torch.isnan(out).any() and torch.equal(torch.isneginf(lse).all(1), lens == 0)


def test_attend_short_rows_of_a_very_wide_table(mp):
    """A table row of 2^25 pages for 2^14 rows: room for so many keys that rows are not split."""
    import torch
    rng = np.random.default_rng(6)
    rows, width, group, dim, page = 1 << 14, 1 << 25, 3, 128, 16
    c = _new_cache(mp, "bf16", 300, page, 1, dim, "tokens")
    named = rng.integers(0, 300, 320).astype(np.int32)
    table = torch.full((1, width), -1, dtype=torch.int32, device="cuda")
    table[0, :320] = torch.from_numpy(named).cuda()
    K, V = _fill(rng, c, np.arange(300, dtype=np.int32)[None], [300 * page], page)
    q = torch.randn(rows, group, dim, dtype=torch.bfloat16, device="cuda")
    lens = (torch.arange(rows, device="cuda") % 71).int()
    lens[5], lens[9000] = 5000, 4113
    assert mp.mp_kv_attend_workspace(c, rows, group, width) == 0
    out, lse = torch.full_like(q, float("nan")), torch.full((rows, group), float("nan"), device="cuda")
    mp.mp_kv_attend(c, q, table.expand(rows, -1), lens, out, lse=lse)
    torch.cuda.synchronize()
    for i in [0, 1, 5, 70, 71, 4095, 9000, rows - 1]:
        w = _attention(_host(q[i])[None], K, V, _slots(named, int(lens[i]), page, 0, 300), dim ** -0.5, "bf16")
        _near(out[i], w[0][0], w[2][0], f"out {i}")
        _near(lse[i], w[1][0], w[3][0], f"lse {i}")
    assert not torch.isnan(out).any() and torch.equal(torch.isneginf(lse).all(1), lens == 0)


def test_attend_splits_do_not_change_what_a_row_is(mp):
    """A row alone, among others and cut in two that lse joins: within the tolerance of each other."""
    import torch
    rng = np.random.default_rng(12)
    page, heads, group, dim, n = 16, 2, 3, 128, 5000
    table, pages = _paged(rng, [n, 40, 900], page)
    c = _new_cache(mp, "f32", pages, page, heads, dim, "tokens")
    K, V = _fill(rng, c, table, [n, 40, 900], page)
    q = _dev(rng.standard_normal((3, heads * group, dim)), "f32")
    T = torch.from_numpy(table).cuda()

    def attend(rows, table, lens):
        out, lse = torch.empty(len(rows), heads * group, dim, device="cuda"), torch.empty(len(rows), 6, device="cuda")
        mp.mp_kv_attend(c, q[rows], table, torch.tensor(lens, dtype=torch.int32, device="cuda"), out, lse=lse)
        return out, lse
    together, alone = attend([0, 1, 2], T, [n, 40, 900]), attend([0], T[:1], [n])
    cut = 2000
    a = attend([0], T[:1, :cut // page].contiguous(), [cut])
    b = attend([0], T[:1, cut // page:].contiguous(), [n - cut])
    la, lb = _host(a[1])[..., None], _host(b[1])[..., None]
    lse = np.logaddexp(la, lb)
    joined = np.exp(la - lse) * _host(a[0]) + np.exp(lb - lse) * _host(b[0])
    slots = _slots(table[0], n, page, 0, pages)
    w = _attention(_host(q[0]).reshape(heads, group, dim), K, V, slots, dim ** -0.5, "f32")
    want, tol = w[0].reshape(1, 6, dim), w[2].reshape(1, 6, dim)
    _near(together[0][:1], want, tol, "together")
    _near(alone[0], want, tol, "alone")
    # a part is off by no more than the whole may be, having fewer keys, and the parts' weights sum to 1; the error of
    # either lse moves those weights by that much of sum p |v| again
    assert (np.abs(joined - want) <= 3 * tol).all()
    assert (np.abs(lse[..., 0] - w[1].reshape(1, 6)) <= 3 * w[3].reshape(1, 6)).all()


def test_attend_empty_tables_and_caches(mp):
    import torch
    for dtype in ("bf16", "f32"):
        c = mp.KvCache(*(torch.empty(0, 16, 2, 64, dtype=_dt(dtype), device="cuda") for _ in range(2)))
        q = torch.ones(3, 4, 64, dtype=_dt(dtype), device="cuda")
        lens = torch.tensor([0, 5, 100], dtype=torch.int32, device="cuda")
        for width in (0, 1, 300):
            out, lse = torch.full_like(q, float("nan")), torch.full((3, 4), float("nan"), device="cuda")
            mp.mp_kv_attend(c, q, torch.zeros(3, width, dtype=torch.int32, device="cuda"), lens, out, lse=lse)
            assert (out == 0).all() and torch.isneginf(lse).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [20, 3000])
def test_attend_non_finite_values_stay_in_their_rows(mp, dtype, n):
    import torch
    rng = np.random.default_rng(n)
    page, heads, group, dim = 16, 2, 3, 64
    table, pages = _paged(rng, [n] * 4, page)
    c = _new_cache(mp, dtype, pages, page, heads, dim, "tokens")
    _fill(rng, c, table, [n] * 4, page)
    at = lambda i, j: (int(table[i, j // page]), j % page)  # noqa: E731
    c.k[at(0, n - 2)][0, 5] = float("nan")    # row 0, first head of keys
    c.v[at(1, 3)][1, 7] = float("inf")        # row 1, second head: value 7 alone
    for j in range(n):                        # row 2, first head: no score above -inf
        c.k[at(2, j)][0, 9] = float("-inf")
    q = _dev(np.abs(rng.standard_normal((4, 6, dim))) + 0.1, dtype)
    q[3, 4, 0] = float("nan")                 # one query head
    out, lse = torch.empty_like(q), torch.empty(4, 6, device="cuda")
    L = torch.full((4,), n, dtype=torch.int32, device="cuda")
    mp.mp_kv_attend(c, q, torch.from_numpy(table).cuda(), L, out, lse=lse)
    torch.cuda.synchronize()
    bad = torch.zeros(out.shape, dtype=torch.bool)
    bad[0, :3] = True
    bad[1, 3:, 7] = True
    bad[3, 4] = True
    assert torch.equal(~torch.isfinite(out).cpu(), bad)
    assert torch.isnan(out[0, :3]).all() and torch.isposinf(out[1, 3:, 7]).all() and torch.isnan(out[3, 4]).all()
    assert (out[2, :3] == 0).all() and torch.isneginf(lse[2, :3]).all()
    assert torch.isnan(lse[0, :3]).all() and torch.isnan(lse[3, 4]) and torch.isfinite(lse[1]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_large_scores(mp, dtype):
    """Scores of +-1000 and more, in increasing and decreasing order: the running maximum."""
    import torch
    rng = np.random.default_rng(8)
    page, dim, n = 16, 64, 1200
    table, pages = _paged(rng, [n, n], page)
    c = _new_cache(mp, dtype, pages, page, 1, dim, "tokens")
    _fill(rng, c, table, [n, n], page)
    for i, order in enumerate((np.arange(n), np.arange(n)[::-1])):
        for j in range(n):
            c.k[int(table[i, j // page]), j % page, 0, 0] = float(order[j] - n // 2) * 2
    q = torch.zeros(2, 3, dim, dtype=_dt(dtype), device="cuda")
    q[:, 0, 0], q[:, 1, 0], q[:, 2, 1] = 1.0, -1.0, 3.0
    out, lse = torch.empty_like(q), torch.empty(2, 3, device="cuda")
    mp.mp_kv_attend(c, q, torch.from_numpy(table).cuda(), torch.full((2,), n, dtype=torch.int32, device="cuda"), out,
                    scale=1.0, lse=lse)
    K, V = (_host(t).reshape(-1, 1, dim) for t in (c.k, c.v))
    for i in range(2):
        slots = _slots(table[i], n, page, 0, pages)
        w = _attention(_host(q[i])[None], np.nan_to_num(K), V, slots, 1.0, dtype)
        _near(out[i], w[0][0], w[2][0], "out")
        _near(lse[i], w[1][0], w[3][0], "lse")


def test_attend_and_append_past_four_gib(mp):
    """Pages far apart: offsets past 32 bits, in bytes and in elements."""
    import torch
    rng = np.random.default_rng(3)
    page, heads, dim = 16, 2, 128
    stride = 3 * 2 ** 30 // 2  # elements: two pages reach 3 GiB, four 9
    try:
        arrays = [torch.zeros(3 * stride + page * heads * dim, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    except torch.OutOfMemoryError:
        pytest.skip("not enough device memory")
    k, v = (a.as_strided((4, page, heads, dim), (stride, heads * dim, dim, 1)) for a in arrays)
    c = mp.KvCache(k, v)
    n = 4 * page - 3
    order = np.array([3, 0, 2, 1])
    slots = torch.from_numpy((order[:, None] * page + np.arange(page)).reshape(-1)[:n]).cuda()
    new = [_dev(rng.standard_normal((n, heads, dim)), "bf16") for _ in range(2)]
    mp.mp_kv_append(c, new[0], new[1], slots)
    assert _equal(k[slots // page, slots % page], new[0]) and _equal(v[slots // page, slots % page], new[1])
    q = _dev(rng.standard_normal((1, 8, dim)), "bf16")
    out = torch.empty_like(q)
    mp.mp_kv_attend(c, q, torch.from_numpy(order.astype(np.int32))[None].cuda(),
                    torch.tensor([n], dtype=torch.int32, device="cuda"), out)
    w = _attention(_host(q).reshape(heads, 4, dim), _host(new[0]), _host(new[1]), np.arange(n), dim ** -0.5, "bf16")
    _near(out[0], w[0].reshape(8, dim), w[2].reshape(8, dim), "out")


# ------------------------------------------------------------------ together
def _serve(mp, dtype, rng, steps, page, prompt):
    """Tokens of three sequences, one a step, through append and attend after a prompt of the first sequence whose
    tokens are rows of their own; yields what is needed to check each."""
    import torch
    heads, group, dim = 2, 4, 64
    H, width = heads * group, -(-(prompt + steps) // page)
    c = _new_cache(mp, dtype, 3 * width, page, heads, dim, "heads")
    table = torch.from_numpy(rng.permutation(3 * width).reshape(3, width).astype(np.int32)).cuda()
    freqs = mp.mp_rope_frequencies(dim, 1e6)[0].cuda()

    def call(qkv, rows, pos):
        q, k, v = torch.split(qkv, (H, heads, heads), 1)
        slots = table[rows, pos // page].long() * page + pos % page
        mp.mp_kv_append(c, k, v, slots, positions=pos, freqs=freqs, q=q)
        out = torch.empty(q.shape, dtype=q.dtype, device="cuda")
        if len(rows) == prompt:  # rows of one sequence share its pages
            mp.mp_kv_attend(c, q, table[rows[0]].expand(len(rows), -1), (pos + 1).int(), out)
        else:
            mp.mp_kv_attend(c, q, table[rows], (pos + 1).int(), out)
        return q, k, v, out
    history = [([], []) for _ in range(3)]
    starts = [prompt, 0, 0]
    batches = [(torch.zeros(prompt, dtype=torch.long, device="cuda"), torch.arange(prompt, device="cuda"))]
    batches += [(torch.arange(3, device="cuda"), torch.tensor([s + i for s in starts], device="cuda"))
                for i in range(steps)]
    for rows, pos in batches:
        qkv = _dev(rng.standard_normal((len(rows), H + 2 * heads, dim)), dtype)
        k0 = qkv[:, H:H + heads].clone()
        q, k, v, out = call(qkv, rows, pos)
        turned = torch.empty_like(k0)
        mp.mp_rope(k0, turned, pos, freqs)
        assert _equal(k, k0)
        for t, (i, p) in enumerate(zip(rows.tolist(), pos.tolist())):
            history[i][0].append(_host(turned[t]))
            history[i][1].append(_host(v[t]))
            assert len(history[i][0]) == p + 1
            w = _attention(_host(q[t]).reshape(heads, group, dim), np.stack(history[i][0]), np.stack(history[i][1]),
                           np.arange(p + 1), dim ** -0.5, dtype)
            _near(out[t], w[0].reshape(H, dim), w[2].reshape(H, dim), f"sequence {i}, token {p}")


@pytest.mark.parametrize("dtype,steps,page,prompt", [("bf16", 20, 16, 50), ("f32", 12, 5, 33)])
def test_a_prompt_and_tokens_after_it(mp, dtype, steps, page, prompt):
    _serve(mp, dtype, np.random.default_rng(steps), steps, page, prompt)


def _step(mp, rng, dtype="bf16", longest=2000):
    """One decoding step over fixed buffers, as a program captures it; what it writes."""
    import torch
    page, heads, group, dim, rows, width = 16, 2, 4, 128, 5, 128
    c = _new_cache(mp, dtype, rows * width, page, heads, dim, "tokens", rng)
    table = torch.from_numpy(rng.permutation(rows * width).reshape(rows, width).astype(np.int32)).cuda()
    lens = torch.tensor([1, longest, 700, 64, 1999], dtype=torch.int32, device="cuda")
    H = heads * group
    qkv = _dev(rng.standard_normal((rows, H + 2 * heads, dim)), dtype)
    q, k, v = torch.split(qkv, (H, heads, heads), 1)
    slots, pos = torch.zeros(rows, dtype=torch.long, device="cuda"), torch.zeros(rows, dtype=torch.long, device="cuda")
    freqs = mp.mp_rope_frequencies(dim, 1e6)[0].cuda()
    turned = torch.empty(rows, H, dim, dtype=_dt(dtype), device="cuda")
    out, lse = torch.empty_like(turned), torch.empty(rows, H, device="cuda")
    ws = torch.empty(max(mp.mp_kv_attend_workspace(c, rows, H, width), 16), dtype=torch.uint8, device="cuda")

    def aim():
        p = (lens - 1).long()
        pos.copy_(p)
        slots.copy_(table.gather(1, (p // page)[:, None])[:, 0].long() * page + p % page)

    def run(stream=None):
        mp.mp_kv_append(c, k, v, slots, positions=pos, freqs=freqs, q=q, q_out=turned, stream=stream)
        mp.mp_kv_attend(c, turned, table, lens, out, lse=lse, workspace=ws, stream=stream)
    return run, aim, lens, qkv, (turned, out, lse, c.k, c.v)


def test_another_stream(mp):
    import torch
    run, aim, lens, qkv, outs = _step(mp, np.random.default_rng(1))
    aim()
    run()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    for t in outs[:3]:
        t.fill_(-1)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    run(stream=s)
    s.synchronize()
    assert all(_equal(a, b) for a, b in zip(outs, want))
    for t in outs[:3]:
        t.fill_(-1)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run()
    s.synchronize()
    assert all(_equal(a, b) for a, b in zip(outs, want))


def test_two_streams_at_once(mp):
    import torch
    steps = [_step(mp, np.random.default_rng(s), longest=1000 * s + 7) for s in (1, 2)]
    for run, aim, *_ in steps:
        aim()
        run()
    torch.cuda.synchronize()
    want = [[t.clone() for t in outs] for *_, outs in steps]
    streams = [torch.cuda.Stream() for _ in steps]
    for *_, outs in steps:
        for t in outs[:3]:
            t.fill_(-1)
    torch.cuda.synchronize()
    for _ in range(5):
        for (run, *_), s in zip(steps, streams):
            run(stream=s)
    torch.cuda.synchronize()
    for (*_, outs), w in zip(steps, want):
        assert all(_equal(a, b) for a, b in zip(outs, w))


def test_no_rows_and_a_cache_without_pages(mp):
    import torch
    z = lambda *s, d=torch.bfloat16: torch.zeros(*s, dtype=d, device="cuda")  # noqa: E731
    c, e = mp.KvCache(z(2, 16, 2, 64), z(2, 16, 2, 64)), mp.KvCache(z(0, 16, 2, 64), z(0, 16, 2, 64))
    none = z(0, d=torch.int64)
    f = mp.mp_rope_frequencies(64)[0].cuda()
    mp.mp_rope(z(0, 2, 64), z(0, 2, 64), none, f)
    mp.mp_rope(z(3, 0, 64), z(3, 0, 64), z(3, d=torch.int64), f)
    mp.mp_kv_append(c, z(0, 2, 64), z(0, 2, 64), none, positions=none, freqs=f, q=z(0, 4, 64))
    mp.mp_kv_attend(c, z(0, 4, 64), z(0, 5, d=torch.int32), z(0, d=torch.int32), z(0, 4, 64))
    # new tokens beside a cache that holds none: queries are turned, nothing is stored
    q, at = torch.randn(3, 4, 64, device="cuda").bfloat16(), torch.arange(3, device="cuda")
    want = torch.empty_like(q)
    mp.mp_rope(q, want, at, f)
    mp.mp_kv_append(e, q[:, :2].contiguous(), q[:, 2:].contiguous(), at, positions=at, freqs=f, q=q)
    assert _equal(q, want)


def test_graph_capture_and_replays_at_other_lengths(mp):
    import torch
    rng = np.random.default_rng(2)
    run, aim, lens, qkv, outs = _step(mp, rng)
    aim()
    run()  # loads the kernels
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for i, n in enumerate(([1, 2000, 700, 64, 1999], [2, 1, 1, 1, 1], [1500, 17, 16, 2048, 900], [2048] * 5)):
        lens.copy_(torch.tensor(n, dtype=torch.int32))
        qkv.copy_(_dev(rng.standard_normal(qkv.shape), "bf16"))
        aim()
        before = [t.clone() for t in outs[3:]]
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        for t, b in zip(outs[3:], before):
            t.copy_(b)
        for t in outs[:3]:
            t.fill_(-1)
        run()
        torch.cuda.synchronize()
        assert all(_equal(a, b) for a, b in zip(outs, got)), i


def test_two_graphs_that_share_a_workspace(mp):
    """Captured on one stream and replayed in turn, with other lengths and eager calls between: each call leaves the
    workspace to the next."""
    import torch
    rng = np.random.default_rng(12)
    page, heads, group, dim, H = 16, 2, 4, 128, 8
    pages = 700
    c = _new_cache(mp, "bf16", pages, page, heads, dim, "tokens")
    c.k.copy_(torch.randn(c.k.shape, device="cuda"))
    c.v.copy_(torch.randn(c.v.shape, device="cuda"))
    calls = []
    for rows, width in ((5, 120), (1, 600)):
        table = torch.from_numpy(rng.integers(0, pages, (rows, width)).astype(np.int32)).cuda()
        q = _dev(rng.standard_normal((rows, H, dim)), "bf16")
        calls.append((q, table, torch.full((rows,), 9, dtype=torch.int32, device="cuda"), torch.empty_like(q)))
    ws = torch.empty(max(mp.mp_kv_attend_workspace(c, len(q), H, t.shape[1]) for q, t, *_ in calls),
                     dtype=torch.uint8, device="cuda")
    graphs = []
    for q, table, lens, out in calls:
        mp.mp_kv_attend(c, q, table, lens, out, workspace=ws)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            mp.mp_kv_attend(c, q, table, lens, out, workspace=ws)
    for turn in range(4):
        for (q, table, lens, out) in calls:
            lens.copy_(torch.from_numpy(rng.integers(0, table.shape[1] * page + 1, len(q)).astype(np.int32)))
            out.fill_(-1)
        torch.cuda.synchronize()
        for g in graphs if turn % 2 else graphs[::-1]:
            g.replay()
        torch.cuda.synchronize()
        for q, table, lens, out in calls:
            want = torch.empty_like(out)
            mp.mp_kv_attend(c, q, table, lens, want)
            assert _equal(out, want), turn


def test_refusals_of_device_buffers(mp):
    import torch
    z = lambda *s, d=torch.bfloat16: torch.zeros(*s, dtype=d, device="cuda")  # noqa: E731
    kv = z(2, 512, 16, 2, 64)
    c = mp.KvCache(kv[0], kv[1])
    pos, f = z(4, d=torch.int64), z(32, d=torch.float64)
    x, big = z(4, 2, 64), z(4, 10, 64)

    def refused(call, word, **kw):
        with pytest.raises(mp.MPError) as e:
            call(**kw)
        assert e.value.code == mp.MP_E_ARG and word in str(e.value)
    refused(mp.mp_rope, "overlaps", x=big[:, :4], y=big[:, 2:6], positions=pos, freqs=f)
    refused(mp.mp_rope, "y is NULL", x=x, y=_Null(x), positions=pos, freqs=f)
    mp.mp_rope(big[:, :4], big[:, 4:8], pos, f)  # rows that pass between each other
    refused(mp.mp_rope, "not device memory", x=x, y=x, positions=pos.cpu().pin_memory(), freqs=f)
    app = dict(cache=c, k=x, v=x.clone(), slots=pos, positions=pos, freqs=f)
    refused(mp.mp_kv_append, "overlaps", **dict(app, v=kv[0, 0, :4]))
    refused(mp.mp_kv_append, "overlaps", **dict(app, q=big[:, :4], q_out=big[:, 2:6]))
    refused(mp.mp_kv_append, "overlaps", **dict(app, k=big[:, 4:6], q=big[:, :4], q_out=big[:, 3:7]))
    refused(mp.mp_kv_append, "share memory", **dict(app, cache=mp.KvCache(kv[0], kv[0])))
    flat = kv.view(-1)
    shifted = [flat[s:s + 4 * 16 * 2 * 64].view(4, 16, 2, 64) for s in (0, 32)]
    refused(mp.mp_kv_append, "share memory", **dict(app, cache=mp.KvCache(*shifted)))
    mp.mp_kv_append(**app)
    q, table, lens = z(4, 4, 64), z(4, 700, d=torch.int32), z(4, d=torch.int32)
    att = dict(cache=c, q=q, table=table, lens=lens, out=z(4, 4, 64))
    refused(mp.mp_kv_attend, "overlaps", **dict(att, out=kv[0, 0, :8].view(4, 4, 64)))
    refused(mp.mp_kv_attend, "overlaps", **dict(att, lse=table.view(-1)[:16].view(torch.float32).view(4, 4)))
    refused(mp.mp_kv_attend, "multiple", **dict(att, q=z(4, 3, 64), out=z(4, 3, 64)))
    need = mp.mp_kv_attend_workspace(c, 4, 4, 700)
    if need:
        refused(mp.mp_kv_attend, "workspace", **dict(att, workspace=z(need - 1, d=torch.uint8)))
        refused(mp.mp_kv_attend, "overlaps", **dict(att, workspace=kv.view(-1).view(torch.uint8)))
    mp.mp_kv_attend(**att)
    torch.cuda.synchronize()


def test_rope_between_the_heads_of_its_input(mp):
    """An output whose heads lie between the input's, of one token and of several, tokens outside heads and inside."""
    import torch
    rng = np.random.default_rng(2)
    f = torch.from_numpy(_freqs(16)).cuda()
    for T in (1, 5):
        pos = torch.arange(3, 3 + T, device="cuda")
        for inside in (False, True):
            buf = _dev(rng.standard_normal((6, T, 16) if inside else (T, 6, 16)), "bf16")
            x, y = (buf[0::2], buf[1::2]) if inside else (buf[:, 0::2], buf[:, 1::2])
            if inside:
                x, y = x.transpose(0, 1), y.transpose(0, 1)
            kept, want = x.clone(), torch.empty(T, 3, 16, dtype=torch.bfloat16, device="cuda")
            mp.mp_rope(kept.contiguous(), want, pos, f)
            mp.mp_rope(x, y, pos, f)
            assert _equal(y, want) and _equal(x, kept)
            mp.mp_rope_backward(kept.contiguous(), want, pos, f)
            mp.mp_rope_backward(x, y, pos, f)
            assert _equal(y, want) and _equal(x, kept)
    flat = torch.zeros(200, dtype=torch.bfloat16, device="cuda")
    for shift in (15, 33, 47):  # by 32 elements from head to head, 16 of them values: these share some
        with pytest.raises(mp.MPError, match="overlaps"):
            mp.mp_rope(*(flat[s:].as_strided((1, 3, 16), (96, 32, 1)) for s in (0, shift)), pos[:1], f)


def test_one_page_beside_an_array_of_many(mp):
    """Keys in an array of their own, values in a page of a larger one whose stride differs."""
    import torch
    rng = np.random.default_rng(9)
    k = torch.zeros(1, 16, 2, 64, device="cuda")
    v = torch.zeros(3, 2, 16, 2, 64, device="cuda")[1:2, 1]
    assert k.stride() != v.stride()
    c = mp.KvCache(k, v)
    new = [_dev(rng.standard_normal((16, 2, 64)), "f32") for _ in range(2)]
    mp.mp_kv_append(c, new[0], new[1], torch.arange(16, device="cuda"))
    assert _equal(k[0], new[0]) and _equal(v[0], new[1])
    q = _dev(rng.standard_normal((1, 4, 64)), "f32")
    out = torch.empty_like(q)
    mp.mp_kv_attend(c, q, torch.zeros(1, 1, dtype=torch.int32, device="cuda"),
                    torch.tensor([13], dtype=torch.int32, device="cuda"), out)
    w = _attention(_host(q).reshape(2, 2, 64), _host(new[0]), _host(new[1]), np.arange(13), 64 ** -0.5, "f32")
    _near(out[0], w[0].reshape(4, 64), w[2].reshape(4, 64), "out")


class _Null:
    """A tensor of another's shape at address 0."""

    def __init__(self, like):
        self.shape, self.dtype, self._stride = like.shape, like.dtype, like.stride()

    def stride(self):
        return self._stride

    def data_ptr(self):
        return 0


def test_example_serves_a_merge(mp):
    """The example runs, its graph replays the eager step's bits, and its rotary gradient is the transpose."""
    import torch
    from examples import decode
    y, same, apart, dots, scale = decode.main(prompt=40, steps=4, say=lambda s: None)
    assert same and torch.isfinite(y).all()
    # each of the two sums of products of bf16 values carries the roundings of its turned factor, 2^-8 at most, and of
    # the turn itself; a pair's products are at most twice those of the untouched values
    assert abs(dots[0] - dots[1]) <= 2 * 2 * (2.0 ** -8 + 2 * TURN) * 2 * scale


def test_example_attends_to_its_own_tokens(mp, monkeypatch):
    """Every append and attention of the example's eager steps against the tokens that its sequences have had: where a
    position, slot, page or length were wrong, a row would be attended to other keys.  And the gradient of its rotary
    positions value by value."""
    import torch
    from examples import decode
    append, attend, backward = mp.mp_kv_append, mp.mp_kv_attend, mp.mp_rope_backward
    tokens, calls, backs = [], [], []

    def eager():
        return not torch.cuda.is_current_stream_capturing()

    def on_append(cache, k, v, slots, positions, freqs, q, **kw):
        if eager():
            tokens.append([t.clone() for t in (k, v, q, positions)] + [freqs, kw])
        append(cache, k, v, slots, positions=positions, freqs=freqs, q=q, **kw)

    def on_attend(cache, q, table, lens, out, **kw):
        assert not kw  # the head's scale, every key
        attend(cache, q, table, lens, out)
        if eager():
            calls.append([t.clone() for t in (q, table, lens, out)])

    def on_backward(dy, dx, positions, freqs):
        backward(dy, dx, positions, freqs)
        backs.append((dy, dx, positions, freqs))
    for name, f in (("mp_kv_append", on_append), ("mp_kv_attend", on_attend), ("mp_rope_backward", on_backward)):
        monkeypatch.setattr(decode.mp, name, f)
    prompt, sequences = 40, 3
    decode.main(prompt=prompt, steps=2, sequences=sequences, say=lambda s: None)
    assert len(tokens) == len(calls) == 1 + prompt + 1
    history = {}
    for (k, v, q0, pos, freqs, kw), (q, table, lens, out) in zip(tokens, calls):
        assert set(kw) <= {"amplitude"}
        keys, turned = torch.empty_like(k), torch.empty_like(q)
        mp.mp_rope(k, keys, pos, freqs, **kw)
        mp.mp_rope(q0, turned, pos, freqs, **kw)
        assert _equal(q, turned)
        H, heads, dim = q.shape[1], *k.shape[1:]
        rows = [tuple(r) for r in table.tolist()]  # a sequence is known by its pages
        for t, row in enumerate(rows):
            past = history.setdefault(row, ([], []))
            assert int(pos[t]) == len(past[0]) and int(lens[t]) == len(past[0]) + 1
            past[0].append(_host(keys[t]))
            past[1].append(_host(v[t]))
        for t, row in enumerate(rows):
            n = int(lens[t])
            w = _attention(_host(q[t]).reshape(heads, H // heads, dim), np.stack(history[row][0][:n]),
                           np.stack(history[row][1][:n]), np.arange(n), dim ** -0.5, "bf16")
            _near(out[t], w[0].reshape(H, dim), w[2].reshape(H, dim), f"sequence {row}, token {n - 1}")
    assert sorted(len(p[0]) for p in history.values()) == [1] * (sequences - 1) + [prompt, prompt + 1]
    (dy, dx, pos, freqs), = backs
    want, tol = _turn(_host(dy), _host(pos).astype(np.int64), _host(freqs), False, 1.0, back=True)
    _near(dx, want, tol + U["bf16"] * 1.01 * np.abs(want), "the rotary gradient")
