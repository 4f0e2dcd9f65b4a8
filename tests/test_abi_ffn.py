"""Refusals of the feed-forward entry points on their host arguments, before any
device work (runs on the CPU), and their structs' layouts."""

import ctypes as C
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def mp():
    import paper_2605_29489_amd as m
    return m


def test_struct_layouts(mp):
    assert C.sizeof(mp.mp_linear_shape) == 8 + 8 * 8
    assert C.sizeof(mp.mp_norm_shape) == 8 + 4 * 8 + 8  # float eps + tail padding
    assert C.sizeof(mp.mp_moe_layer) == 16 + 5 * 8


def _linear(mp, **over):
    f = dict(dtype=1, act=0, m=4, n=6, k=8, ldx=8, ldw=8, ldy=6, ldz=6, ldr=6)
    f.update(over)
    return mp.mp_linear_shape(**f)


@pytest.mark.parametrize("over", [dict(dtype=2), dict(act=5), dict(act=-1), dict(m=-1), dict(n=1 << 31),
                                  dict(k=-1), dict(ldx=7), dict(ldw=7), dict(ldy=5), dict(ldz=5), dict(ldr=5),
                                  dict(ldx=(1 << 40) + 1)])
def test_linear_shapes_refused(mp, over):
    one = C.c_void_p(16)  # never reached
    s = _linear(mp, **over)
    assert mp.lib.mp_linear(C.byref(s), one, one, None, one, one, one, None, 0, None) == mp.MP_E_ARG
    assert mp.mp_last_error() != ""


def test_linear_null_arguments(mp):
    n = C.c_uint64(77)
    assert mp.lib.mp_linear(None, None, None, None, None, None, None, None, 0, None) == mp.MP_E_ARG
    assert mp.lib.mp_linear_workspace(None, 0, C.byref(n)) == mp.MP_E_ARG
    s = _linear(mp)
    assert mp.lib.mp_linear_workspace(C.byref(s), 2, C.byref(n)) == mp.MP_E_ARG
    assert mp.lib.mp_linear_workspace(C.byref(s), 0, None) == mp.MP_E_ARG
    assert n.value == 77
    assert mp.lib.mp_linear(C.byref(s), None, None, None, None, None, None, None, 0, None) == mp.MP_E_ARG
    # nothing to do: no pointer is looked at
    s = _linear(mp, m=0)
    assert mp.lib.mp_linear(C.byref(s), None, None, None, None, None, None, None, 0, None) == mp.MP_OK
    # a backward pass that needs a workspace gets none
    s = _linear(mp, act=4)
    assert mp.lib.mp_linear_workspace(C.byref(s), 1, C.byref(n)) == mp.MP_OK and n.value > 0
    assert mp.lib.mp_linear_backward(C.byref(s), None, None, None, None, None, 8, None, 8, None, None, 0,
                                     None) == mp.MP_E_ARG
    assert "workspace" in mp.mp_last_error()


@pytest.mark.parametrize("over", [dict(dtype=9), dict(flags=2), dict(rows=-1), dict(cols=1 << 31), dict(ldx=7),
                                  dict(ldy=7), dict(eps=-1.0), dict(eps=float("inf")), dict(eps=float("nan"))])
def test_norm_shapes_refused(mp, over):
    f = dict(dtype=1, flags=0, rows=4, cols=8, ldx=8, ldy=8, eps=1e-6)
    f.update(over)
    s = mp.mp_norm_shape(**f)
    one = C.c_void_p(16)
    assert mp.lib.mp_norm(C.byref(s), one, None, None, one, None, None, None) == mp.MP_E_ARG
    assert mp.lib.mp_norm_backward(C.byref(s), one, one, None, one, one, one, 8, None, None, one, 1 << 40,
                                   None) == mp.MP_E_ARG


@pytest.mark.parametrize("over,E,residency,code", [
    (dict(dtype=3), 4, 0, -1), (dict(act=7), 4, 0, -1), (dict(top_k=0), 4, 0, -1), (dict(top_k=9), 32, 0, -1),
    (dict(top_k=3), 2, 0, -1), (dict(flags=4), 4, 0, -1), (dict(hidden=0), 4, 0, -1), (dict(ffn=0), 4, 0, -1),
    (dict(gate_off=-1), 4, 0, -1), (dict(down_off=(1 << 48) + 1), 4, 0, -1), ({}, 0, 0, -1), ({}, 33, 0, -1),
    ({}, 4, 2, -2), ({}, 4, 3, -2), ({}, 4, 16, -1),
])
def test_moe_layers_refused(mp, over, E, residency, code):
    f = dict(dtype=1, act=4, top_k=2, flags=0, hidden=8, ffn=6, gate_off=0, up_off=48, down_off=96)
    f.update(over)
    s = mp.mp_moe_layer(**f)
    ptrs = (C.c_void_p * 33)()
    one = C.c_void_p(16)
    rc = mp.lib.mp_moe(C.byref(s), 2, one, 8, one, None, ptrs, E, residency, None, 0, one, 8, None, None, one, 1 << 40,
                       None)
    assert rc == code


def test_moe_token_limit(mp):
    s = mp.mp_moe_layer(1, 4, 2, 0, 8, 6, 0, 48, 96)
    n = C.c_uint64(0)
    assert mp.lib.mp_moe_workspace(C.byref(s), 64, C.byref(n)) == mp.MP_OK and n.value > 0
    assert mp.lib.mp_moe_workspace(C.byref(s), 65, C.byref(n)) == mp.MP_E_UNSUPPORTED
    assert mp.lib.mp_moe_workspace(C.byref(s), -1, C.byref(n)) == mp.MP_E_ARG


def test_sizes_that_no_launch_holds_are_refused(mp):
    one, n = C.c_void_p(16), C.c_uint64(0)
    for over in (dict(m=(1 << 26) + 1), dict(n=(1 << 26) + 1, ldy=1 << 27), dict(k=(1 << 26) + 1, ldx=1 << 27)):
        s = _linear(mp, **over)
        assert mp.lib.mp_linear(C.byref(s), one, one, None, None, one, None, None, 0, None) == mp.MP_E_ARG
        assert mp.lib.mp_linear_workspace(C.byref(s), 1, C.byref(n)) == mp.MP_E_ARG
    s = mp.mp_norm_shape(1, 0, 4, (1 << 26) + 1, 1 << 27, 1 << 27, 1e-6)
    assert mp.lib.mp_norm_workspace(C.byref(s), C.byref(n)) == mp.MP_E_ARG
    for over in (dict(hidden=(1 << 24) + 1), dict(ffn=(1 << 24) + 1)):
        f = dict(dtype=1, act=4, top_k=2, flags=0, hidden=8, ffn=6, gate_off=0, up_off=48, down_off=96)
        f.update(over)
        s = mp.mp_moe_layer(**f)
        assert mp.lib.mp_moe_workspace(C.byref(s), 4, C.byref(n)) == mp.MP_E_ARG


def test_linear_workspace_of_empty_sizes(mp):
    """Sizes of zero have a workspace size, both ways; asked in a process of its own, which a host exception
    would end."""
    import subprocess
    import sys
    ask = """
import itertools
import paper_2605_29489_amd as mp
for dtype, act, m, n, k in itertools.product((0, 1), (0, 4), (0, 4, 70), (0, 6), (0, 8)):
    print(dtype, act, m, n, k, *(mp.mp_linear_workspace(dtype, act, m, n, k, b) for b in (False, True)), flush=True)
"""
    r = subprocess.run([sys.executable, "-c", ask], capture_output=True, text=True, cwd=ROOT)
    lines = [tuple(map(int, line.split())) for line in r.stdout.splitlines()]
    assert r.returncode == 0 and len(lines) == 48, f"status {r.returncode} after {lines[-1:]}: {r.stderr}"
    for dtype, act, m, n, k, forward, backward in lines:
        assert forward == 0 and (n > 0 or backward == 0)
