"""Refusals of the attention entry points on their host arguments, before any device work, their structs' layouts and
the rotary frequencies (runs on the CPU)."""

import ctypes as C
import math

import pytest


@pytest.fixture(scope="module")
def mp():
    import paper_2605_29489_amd as m
    return m


def test_struct_layouts(mp):
    assert C.sizeof(mp.mp_rope_shape) == 8 + 8 * 8 + 8
    assert C.sizeof(mp.mp_rope_scaling) == 8 + 5 * 8
    assert C.sizeof(mp.mp_kv_cache) == 8 + 7 * 8 + 16
    assert C.sizeof(mp.mp_kv_rows) == 3 * 8 + 8 + 4 * 8
    assert C.sizeof(mp.mp_kv_attend_shape) == 7 * 8 + 8


ONE = C.c_void_p(16)  # never reached


def _rope(mp, **over):
    f = dict(dtype=1, flags=0, tokens=5, heads=3, head_dim=8, rot_dim=8, ldx=24, hdx=8, ldy=24, hdy=8, amplitude=1.0)
    f.update(over)
    return mp.mp_rope_shape(**f)


@pytest.mark.parametrize("over", [
    dict(dtype=2), dict(flags=2), dict(tokens=-1), dict(tokens=1 << 31), dict(heads=-1), dict(heads=65537),
    dict(head_dim=0), dict(head_dim=4097), dict(rot_dim=7), dict(rot_dim=10), dict(rot_dim=-2),
    dict(amplitude=float("inf")), dict(amplitude=float("nan")), dict(ldx=23), dict(hdx=7), dict(ldy=0), dict(hdy=-8),
    dict(ldx=8, hdx=39), dict(ldx=(1 << 40) + 1), dict(ldx=1 << 40, hdx=1 << 40)])
def test_rope_shapes_refused(mp, over):
    s = _rope(mp, **over)
    for call in (mp.lib.mp_rope, mp.lib.mp_rope_backward):
        assert call(C.byref(s), ONE, ONE, ONE, ONE, None) == mp.MP_E_ARG
        assert mp.mp_last_error() != ""


def test_rope_with_nothing_to_do(mp):
    for over in (dict(tokens=0), dict(heads=0)):
        s = _rope(mp, **over)
        assert mp.lib.mp_rope(C.byref(s), None, None, None, None, None) == mp.MP_OK
    assert mp.lib.mp_rope(None, ONE, ONE, ONE, ONE, None) == mp.MP_E_ARG
    s = _rope(mp)
    assert mp.lib.mp_rope(C.byref(s), None, None, None, None, None) == mp.MP_E_ARG


def _want_frequencies(kind, rot, base, factor, original, low, high):
    """Pair by pair, from each formula."""
    out, amp = [], 0.1 * math.log(factor) + 1 if kind == 4 else 1.0
    for i in range(rot // 2):
        f = math.exp(-2 * i / rot * math.log(base))
        if kind == 1:
            f /= factor
        elif kind == 2 and rot > 2:
            f = math.exp(-2 * i / rot * (math.log(base) + rot / (rot - 2) * math.log(factor)))
        elif kind == 3:
            wave = 2 * math.pi / f
            if wave > original / low:
                f /= factor
            elif wave >= original / high:
                s = (original / wave - low) / (high - low)
                f = (1 - s) * f / factor + s * f
        elif kind == 4:
            at = lambda r: rot * math.log(original / (r * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
            lo, hi = max(math.floor(at(high)), 0), min(math.ceil(at(low)), rot - 1)
            s = min(max((i - lo) / max(hi - lo, 1e-3), 0.0), 1.0)
            f = f / factor * s + f * (1 - s)
        out.append(f)
    return out, amp


@pytest.mark.parametrize("rot", [0, 2, 4, 52, 128, 256])
@pytest.mark.parametrize("kind,base,factor,original,low,high", [
    (0, 10000.0, 1.0, 0.0, 0.0, 0.0), (1, 10000.0, 4.0, 0.0, 0.0, 0.0), (2, 1e6, 8.0, 0.0, 0.0, 0.0),
    (3, 5e5, 8.0, 8192.0, 1.0, 4.0), (4, 1e4, 16.0, 4096.0, 1.0, 32.0), (4, 1e6, 1.0, 32768.0, 1.0, 32.0)])
def test_frequencies(mp, rot, kind, base, factor, original, low, high):
    f, amp = mp.mp_rope_frequencies(rot, base, kind, factor, original, low, high)
    want, want_amp = _want_frequencies(kind, rot, base, factor, original, low, high)
    assert f.dtype.is_floating_point and f.element_size() == 8 and f.tolist() == pytest.approx(want, rel=1e-13)
    assert amp == pytest.approx(want_amp, rel=2.0 ** -24)  # it is a float


@pytest.mark.parametrize("over", [
    dict(kind=5), dict(kind=-1), dict(rot_dim=3), dict(rot_dim=-2), dict(rot_dim=4098), dict(base=1.0), dict(base=0.0),
    dict(base=float("nan")), dict(base=float("inf")), dict(kind=1, factor=0.5), dict(kind=2, factor=float("nan")),
    dict(kind=3, factor=8.0), dict(kind=3, factor=8.0, original=8192.0, low=4.0, high=4.0),
    dict(kind=4, factor=8.0, original=-1.0), dict(kind=4, factor=8.0, original=8192.0, low=0.0)])
def test_frequencies_refused(mp, over):
    with pytest.raises(mp.MPError) as e:
        mp.mp_rope_frequencies(**dict(dict(rot_dim=8), **over))
    assert e.value.code == mp.MP_E_ARG


def _cache(mp, **over):
    f = dict(dtype=1, flags=0, pages=10, page_size=16, heads=2, head_dim=8, page_stride=256, slot_stride=16,
             head_stride=8, k=1 << 20, v=1 << 21)
    f.update(over)
    return mp.mp_kv_cache(**f)


def _rows(mp, **over):
    f = dict(tokens=4, q_heads=6, rot_dim=8, flags=0, amplitude=1.0, ldk=16, ldv=16, ldq=48, ldqo=48)
    f.update(over)
    return mp.mp_kv_rows(**f)


def _attend(mp, **over):
    f = dict(rows=4, q_heads=6, width=5, ldq=48, ldo=48, ldt=5, window=0, scale=0.5)
    f.update(over)
    return mp.mp_kv_attend_shape(**f)


BAD_CACHES = [
    (dict(dtype=7), -1), (dict(flags=1), -1), (dict(pages=-1), -1), (dict(pages=(1 << 40) + 1), -1),
    (dict(pages=1 << 37), -1), (dict(page_size=0), -1), (dict(page_size=(1 << 30) + 1), -1), (dict(heads=0), -1),
    (dict(heads=4097), -1), (dict(head_dim=0), -1), (dict(head_dim=257), -2), (dict(page_stride=0), -1),
    (dict(page_stride=255), -1), (dict(slot_stride=15), -1), (dict(slot_stride=(1 << 24) + 1), -1),
    (dict(head_stride=7), -1), (dict(slot_stride=8, head_stride=8), -1), (dict(head_stride=0), -1),
    (dict(slot_stride=8, head_stride=127), -1)]


@pytest.mark.parametrize("over,code", BAD_CACHES)
def test_caches_refused(mp, over, code):
    c, r, s, n = _cache(mp, **over), _rows(mp), _attend(mp), C.c_uint64(7)
    assert mp.lib.mp_kv_append(C.byref(c), C.byref(r), ONE, ONE, ONE, ONE, ONE, ONE, ONE, None) == code
    assert mp.lib.mp_kv_attend(C.byref(c), C.byref(s), ONE, ONE, ONE, ONE, None, ONE, 1 << 40, None) == code
    assert mp.lib.mp_kv_attend_workspace(C.byref(c), C.byref(s), C.byref(n)) == code and n.value == 7


@pytest.mark.parametrize("over", [
    dict(tokens=-1), dict(tokens=1 << 31), dict(q_heads=-1), dict(q_heads=65537, ldq=1 << 30, ldqo=1 << 30),
    dict(rot_dim=9), dict(rot_dim=10), dict(flags=2), dict(amplitude=float("nan")), dict(ldk=15), dict(ldv=15),
    dict(ldq=47), dict(ldqo=47)])
def test_rows_refused(mp, over):
    c, r = _cache(mp), _rows(mp, **over)
    assert mp.lib.mp_kv_append(C.byref(c), C.byref(r), ONE, ONE, ONE, ONE, ONE, ONE, ONE, None) == mp.MP_E_ARG
    assert mp.lib.mp_kv_append(C.byref(c), None, ONE, ONE, ONE, ONE, ONE, ONE, ONE, None) == mp.MP_E_ARG


@pytest.mark.parametrize("over", [
    dict(rows=-1), dict(rows=(1 << 20) + 1), dict(q_heads=0), dict(q_heads=7), dict(q_heads=-2), dict(width=-1),
    dict(width=1 << 27), dict(ldq=47), dict(ldo=47), dict(ldt=4), dict(ldt=-1), dict(window=-1),
    dict(scale=float("inf")), dict(scale=float("nan")), dict(scale=-2e30), dict(width=(1 << 25) + 1), dict(rows=1 << 20, q_heads=10, ldq=80, ldo=80)])
def test_attend_shapes_refused(mp, over):
    c, s = _cache(mp), _attend(mp, **over)
    assert mp.lib.mp_kv_attend(C.byref(c), C.byref(s), ONE, ONE, ONE, ONE, None, ONE, 1 << 40, None) == mp.MP_E_ARG
    assert mp.lib.mp_kv_attend(C.byref(c), None, ONE, ONE, ONE, ONE, None, ONE, 1 << 40, None) == mp.MP_E_ARG
    assert mp.lib.mp_kv_attend(None, C.byref(s), ONE, ONE, ONE, ONE, None, ONE, 1 << 40, None) == mp.MP_E_ARG
    assert mp.lib.mp_kv_attend_workspace(C.byref(c), C.byref(s), None) == mp.MP_E_ARG


@pytest.mark.parametrize("dtype,rows,q_heads,width", [
    ("MP_BF16", 1 << 14, 1, 1 << 25), ("MP_F32", 1 << 13, 1, 1 << 25), ("MP_BF16", 1 << 20, 8, 1 << 19),
    ("MP_F32", 1 << 18, 16, 1 << 20)])
def test_tables_with_room_for_more_tiles_than_a_share_counts(mp, dtype, rows, q_heads, width):
    """2^38 tiles (of 32 keys, fp32 16) would be 256 shares of 2^30: rows are not split then, and need no workspace."""
    def need(rows, width):
        n = C.c_uint64(7)
        c = _cache(mp, dtype=getattr(mp, dtype), heads=1, head_dim=128, page_stride=2048, slot_stride=128)
        s = _attend(mp, rows=rows, q_heads=q_heads, width=width, ldq=2048, ldo=2048, ldt=0)
        assert mp.lib.mp_kv_attend_workspace(C.byref(c), C.byref(s), C.byref(n)) == mp.MP_OK
        return n.value
    assert need(rows, width) == 0
    assert need(rows - 1, width) > 0 and need(rows, width - 2) > 0


def _need(mp, rows, q_heads, width, window, **cache):
    n = C.c_uint64(7)
    c, s = _cache(mp, **cache), _attend(mp, rows=rows, q_heads=q_heads, width=width, window=window)
    assert mp.lib.mp_kv_attend_workspace(C.byref(c), C.byref(s), C.byref(n)) == mp.MP_OK
    return n.value


@pytest.mark.parametrize("dtype,tile", [("MP_BF16", 32), ("MP_F32", 16)])
@pytest.mark.parametrize("page", [1, 10, 16, 64])
@pytest.mark.parametrize("rows,q_heads", [(1, 2), (4, 8), (64, 14), (5000, 2)])
def test_a_window_takes_no_more_workspace_than_every_key(mp, dtype, tile, page, rows, q_heads):
    """A window counts no more tiles than the table has room for: four tiles are not split, with or without one."""
    cache = dict(dtype=getattr(mp, dtype), page_size=page, page_stride=16 * page)
    for most in (page, 3 * tile, 4 * tile - 1, 4 * tile, 4 * tile + 1, 9 * tile, 300 * tile):
        width = max(1, most // page)
        most = width * page
        whole = _need(mp, rows, q_heads, width, 0, **cache)
        assert (whole == 0) == (most <= 4 * tile)
        for window in {1, 2, most // 2, most - tile, most - 2, most - 1, most, most + 1, 2 * most, 1 << 40}:
            if window > 0:
                assert _need(mp, rows, q_heads, width, window, **cache) <= whole, (most, window)


def test_no_rows_no_tokens(mp):
    c, r, s = _cache(mp), _rows(mp, tokens=0), _attend(mp, rows=0)
    assert mp.lib.mp_kv_append(C.byref(c), C.byref(r), None, None, None, None, None, None, None, None) == mp.MP_OK
    assert mp.lib.mp_kv_attend(C.byref(c), C.byref(s), None, None, None, None, None, None, 0, None) == mp.MP_OK


def test_a_cache_of_one_page_or_head_takes_any_strides_there(mp):
    """Strides of a dimension of one place are no strides: a part of a larger array beside an array of its own."""
    import torch
    z = torch.zeros
    for k, v in ((z(1, 16, 2, 8), z(3, 16, 2, 16)[1:2, :, :, :8].contiguous().as_strided((1, 16, 2, 8), (7, 16, 8, 1))),
                 (z(4, 16, 1, 8), z(4, 16, 1, 8).as_strided((4, 16, 1, 8), (128, 8, 3, 1))),
                 (z(4, 1, 2, 8), z(4, 1, 2, 8).as_strided((4, 1, 2, 8), (16, 99, 8, 1)))):
        mp.KvCache(k, v)
    with pytest.raises(ValueError):
        mp.KvCache(z(2, 16, 2, 8), z(2, 16, 4, 8)[:, :, :2])


def test_binding_refuses_shapes_and_types(mp):
    import torch
    z = torch.zeros
    k = z(4, 16, 2, 8)
    with pytest.raises(ValueError):
        mp.KvCache(k, z(4, 16, 2, 4))
    with pytest.raises(ValueError):
        mp.KvCache(k, k.bfloat16())
    with pytest.raises(ValueError):
        mp.KvCache(k.half(), k.half())
    with pytest.raises(ValueError):
        mp.KvCache(k, z(4, 2, 16, 8).transpose(1, 2))  # strides differ
    with pytest.raises(ValueError):
        mp.KvCache(z(4, 16, 8, 2).transpose(2, 3), z(4, 16, 8, 2).transpose(2, 3))
    c = mp.KvCache(k, z(4, 16, 2, 8))
    x, pos, f = z(3, 2, 8), z(3, dtype=torch.int64), z(4, dtype=torch.float64)
    for bad in (dict(k=z(3, 3, 8)), dict(v=z(3, 2, 8).bfloat16()), dict(slots=pos.int()), dict(positions=None),
                dict(positions=z(2, dtype=torch.int64)), dict(freqs=f.float()), dict(q=z(2, 4, 8)), dict(q=z(3, 4, 9)),
                dict(q=z(3, 8, 4).transpose(1, 2)), dict(k=z(2, 3, 8).transpose(0, 1))):
        with pytest.raises(ValueError):
            mp.mp_kv_append(c, **dict(dict(k=x, v=x, slots=pos, positions=pos, freqs=f, stream=0), **bad))
    table, lens, q = z(3, 5, dtype=torch.int32), z(3, dtype=torch.int32), z(3, 4, 8)
    for bad in (dict(table=table.long()), dict(table=table[:2]), dict(table=z(5, 3, dtype=torch.int32).t()),
                dict(lens=lens.long()), dict(lens=lens[:2]), dict(out=z(3, 4, 7)), dict(q=q.bfloat16()),
                dict(lse=z(3, 5)), dict(lse=z(3, 4).double())):
        with pytest.raises(ValueError):
            mp.mp_kv_attend(c, **dict(dict(q=q, table=table, lens=lens, out=z(3, 4, 8), stream=0), **bad))
    for bad in (dict(y=z(3, 2, 9)), dict(y=x.bfloat16()), dict(x=z(3, 8, 2).transpose(1, 2)), dict(positions=pos.int()),
                dict(freqs=f.float())):
        with pytest.raises(ValueError):
            mp.mp_rope(**dict(dict(x=x, y=z(3, 2, 8), positions=pos, freqs=f, stream=0), **bad))
