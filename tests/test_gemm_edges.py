"""Which K tiles of a tiled product may be read in whole chunks (gemm_edge.h): no chunk of them passes the
operand's end, and no tile is held back without need.  Runs on the CPU: the rule is compiled as host code, and the
bytes that a K tile's chunks touch are listed here."""

import ctypes as C
import shutil
import subprocess

import pytest

from paper_2605_29489_amd import build

TILE = 64  # columns of the smallest tile


@pytest.fixture(scope="module")
def whole(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    d = tmp_path_factory.mktemp("edges")
    src = d / "edges.cpp"
    src.write_text('#include "gemm_edge.h"\n'
                   'extern "C" int64_t whole(int64_t p, int64_t cols, int64_t ld, int v, int bk)\n'
                   '{ return mp::whole_k_tiles(p, cols, ld, v, bk); }\n')
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", "-I", build.CSRC, str(src), "-o", str(d / "edges.so")], check=True)
    f = C.CDLL(str(d / "edges.so")).whole
    f.restype, f.argtypes = C.c_int64, [C.c_int64] * 3 + [C.c_int, C.c_int]
    return f


def _chunk_ends(cols, V):
    """Ends of the chunks that the tiles along a p-row read, in elements from the row's first."""
    return [j0 + (c + 1) * V for j0 in range(0, cols, TILE) for c in range(min(TILE // V, -(-(cols - j0) // V)))]


@pytest.mark.parametrize("V,BK", [(8, 64), (4, 32)])  # bf16, fp32: elements of 16 bytes, rows of a K tile
def test_whole_chunks_stay_inside_the_operand(whole, V, BK):
    for cols in [*range(1, 20), 63, 64, 65, 71, 130]:
        most = max(_chunk_ends(cols, V))
        for ld in sorted({cols, cols + 1, cols + 2, cols + 5, cols + 8, cols + 100}):
            for P in [*range(1, 2 * BK + 10), 3 * BK, 3 * BK + 1, 50 * BK + 3]:
                end = (P - 1) * ld + cols  # of the operand, in elements
                tiles = -(-P // BK)
                # the rows of a tile read furthest at its last one; the last tile is never read whole, for its
                # rows past P have to be zeros
                fits = [t < tiles - 1 and ((t + 1) * BK - 1) * ld + most <= end for t in range(tiles)]
                n = whole(P, cols, ld, V, BK)
                assert 0 <= n < tiles and all(fits[:n]), (cols, ld, P, n)
                assert not fits[n], (cols, ld, P, n)  # none held back
                assert n >= tiles - 2, (cols, ld, P, n)
