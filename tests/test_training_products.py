"""The 4-bit product's large tiles in every form: both output types, rows of C on any element, batches."""
import ctypes
import os
import subprocess

import pytest
import torch

from test_training_ops import B, DTYPES, U, codes4, values

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2504_20437_amd", "csrc")
TILES = {0: 256, 1: 128, 2: 64}

SHIM = """
#include "dispatch.hpp"
extern "C" int tile_(long M, long N, long b) { return galore::mx4_tile(M, N, b); }
"""


@pytest.fixture(scope="module")
def tile(tmp_path_factory):
    d = tmp_path_factory.mktemp("tiles")
    src, out = str(d / "shim.cpp"), str(d / "libtiles.so")
    with open(src, "w") as f:
        f.write(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, src, "-o", out], check=True)
    lib = ctypes.CDLL(out)
    return lambda m, n, b=1: TILES[lib.tile_(ctypes.c_long(m), ctypes.c_long(n), ctypes.c_long(b))]


@pytest.fixture(scope="module")
def gl():
    import paper_2504_20437_amd
    return paper_2504_20437_amd


def check(gl, C, a, b, k):
    """C against the product of the decoded operands in 64 bits"""
    ad, bd = (gl.galore_mx4_dequantize(*q, k, dtype=torch.float32).double() for q in (a, b))
    want, size = ad @ bd.t().contiguous(), ad.abs() @ bd.abs().t().contiguous()
    tol = (k + 4) * U * size
    if C.dtype == torch.bfloat16:
        tol = tol + B * (want.abs() + tol)
    assert ((C.double() - want).abs() <= tol).all()


@pytest.mark.gpu
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k,size", [(4096, 4096, 256, 256), (4096, 4104, 300, 256), (4301, 4099, 777, 256),
                                        (2048, 2048, 512, 128), (2100, 1930, 520, 128), (2051, 2049, 33, 128),
                                        (500, 701, 300, 64)])
def test_large_tiles(gl, tile, m, n, k, size, out):
    assert tile(m, n) == size
    a, b = codes4(values(m, k, "f32", 1)), codes4(values(n, k, "f32", 2))
    C = gl.galore_mx4_matmul(*a, *b, k, dtype=DTYPES[out])
    check(gl, C, a, b, k)
    # rows of C of an odd and of an even pitch, from an odd and from an even element on
    for pitch, first in ((n + 1, 1), (n + 2, 1), (n + 2, 2), (n + 3, 0)):
        room = torch.full((m, pitch), 5.0, dtype=DTYPES[out], device="cuda")
        gl.galore_mx4_matmul(*a, *b, k, C=room[:, first:first + n])
        assert torch.equal(room[:, first:first + n], C)
        assert (room[:, :first] == 5).all() and (room[:, first + n:] == 5).all()


@pytest.mark.gpu
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("nb,m,n,k,size", [(6, 2048, 2100, 300, 256), (3, 1200, 1300, 256, 128), (5, 300, 200, 130, 64)])
def test_batched_tiles(gl, tile, nb, m, n, k, size, out):
    """another matrix in every slot, in rows of a longer pitch, the slots apart from each other"""
    assert tile(m, n, nb) == size
    sets = [(codes4(values(m, k, "f32", i)), codes4(values(n, k, "f32", 50 + i))) for i in range(nb)]

    def slots(which, part):
        rows, width = sets[0][which][part].shape
        room = torch.full((nb, rows + 3, width + 16), 255, dtype=torch.uint8, device="cuda")
        for i in range(nb):
            room[i, :rows, :width] = sets[i][which][part]
        return room[:, :rows, :width]

    a, b = (slots(0, 0), slots(0, 1)), (slots(1, 0), slots(1, 1))
    room = torch.full((nb, m + 1, n + 2), 5.0, dtype=DTYPES[out], device="cuda")
    C = gl.galore_mx4_matmul(*a, *b, k, C=room[:, :m, 1:n + 1])
    for i in range(nb):
        check(gl, C[i], *sets[i], k)
    assert (room[:, m] == 5).all() and (room[:, :, 0] == 5).all() and (room[:, :, n + 1] == 5).all()
