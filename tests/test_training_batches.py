"""Batches whose tiles do not fit one launch: its work-items along x are a 32-bit number."""
import ctypes
import os
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2504_20437_amd", "csrc")

SHIM = """
#include "dispatch.hpp"
extern "C" int matrices_(long tiles, int batch) { return galore::matrices_a_launch(tiles, batch); }
"""


@pytest.fixture(scope="module")
def matrices(tmp_path_factory):
    d = tmp_path_factory.mktemp("batches")
    src, out = str(d / "shim.cpp"), str(d / "libbatches.so")
    with open(src, "w") as f:
        f.write(SHIM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, src, "-o", out], check=True)
    lib = ctypes.CDLL(out)
    return lambda tiles, batch: lib.matrices_(ctypes.c_long(tiles), batch)


@pytest.mark.parametrize("tiles,batch,want", [
    (1, 1, 1), (1, 65535, 65535), (256, 65535, 65535), (257, 65535, 65280), ((1 << 24) - 1, 3, 1), ((1 << 23) - 1, 3, 2),
    (1 << 23, 3, 1), (1 << 24, 1, 0), (1 << 40, 1, 0)])
def test_matrices_of_a_launch(matrices, tiles, batch, want):
    """as many as keep 256 work-items for each tile below 2^32; none where a single matrix does not"""
    got = matrices(tiles, batch)
    assert got == want
    assert got * tiles * 256 < 1 << 32


@pytest.mark.gpu
@pytest.mark.parametrize("accumulate", [False, True])
def test_weight_grad_of_a_long_batch(accumulate):
    """65535 gradients of 32769 x 1, 257 tiles each: 4 GB in and 4 GB out"""
    import paper_2504_20437_amd as gl
    b, m = 65535, 32769
    dy = torch.empty((b, 1, m), dtype=torch.bfloat16, device="cuda")
    dy[:] = (torch.arange(m, device="cuda") % 200).bfloat16()
    x = (torch.arange(b, device="cuda") % 3 - 1).bfloat16().reshape(b, 1, 1)
    q = gl.galore_checkpoint_pack(x)
    G = torch.ones((b, m, 1), dtype=torch.bfloat16, device="cuda") if accumulate else None
    G = gl.galore_checkpoint_weight_grad(dy, *q, 1, G=G, accumulate=accumulate)
    for i in range(0, b, 4096):                       # small integers: exact in bf16 in any order
        assert torch.equal(G[i:i + 4096, :, 0], dy[i:i + 4096, 0] * x[i:i + 4096, 0] + (1 if accumulate else 0))
