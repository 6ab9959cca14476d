"""Vector accesses of the training operators: rows that start on 16 bytes and whose
width is no multiple of eight values."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import test_training_ops as ops
import training_oracle as ora
from test_training_ops import DTYPES, host, norm_inputs, values

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2504_20437_amd", "csrc")

# The row readers of mx.hpp as host code. On x86 a load past the caches whose type
# promises 16 bytes of alignment traps at any other address.
HOST = """
#include <hip/hip_runtime.h>
#include <stdio.h>
#undef __device__
#define __device__ __attribute__((host)) __attribute__((device))
#include "mx.hpp"
using namespace galore;

static void set(float& to, int v) { to = static_cast<float>(v); }
static void set(bf16_t& to, int v) {   // exact: v < 256
    const float f = static_cast<float>(v);
    unsigned u;
    __builtin_memcpy(&u, &f, 4);
    to.bits = static_cast<unsigned short>(u >> 16);
}
template <typename T>
static float at(const Eight<T>& x, int i);
template <>
float at(const Eight<float>& x, int i) { return x.v[i]; }
template <>
float at(const Eight<bf16_t>& x, int i) {
    const unsigned u = i & 1 ? x.w[i >> 1] & 0xffff0000u : x.w[i >> 1] << 16;
    float f;
    __builtin_memcpy(&f, &u, 4);
    return f;
}

template <typename T>
static int check() {
    alignas(64) static T row[64];
    for (int i = 0; i < 64; ++i) set(row[i], i + 1);
    for (int n = 8; n <= 40; ++n)
        for (int e = 0; e + 8 <= n || e < n; e += 8) {
            Eight<T> x;
            x.load(row, e, n, true);
            // the row's last eight where the group crosses its end
            const int from = e + 8 <= n ? e : n - 8;
            for (int i = 0; i < 8; ++i)
                if (at(x, i) != static_cast<float>(from + i + 1)) {
                    printf("n %d e %d i %d\\n", n, e, i);
                    return 1;
                }
        }
    return 0;
}
int main() { return check<float>() || check<bf16_t>(); }
"""


def test_row_reads_promise_no_more_than_the_elements_alignment(tmp_path):
    hipcc = os.environ.get("HIPCC") or shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    src, exe = str(tmp_path / "rows.hip"), str(tmp_path / "rows")
    with open(src, "w") as f:
        f.write(HOST)
    res = subprocess.run([hipcc, "--offload-arch=gfx950", "--offload-host-only", "-std=c++17", "-O0", "-msse4.1", "-I", CSRC,
                          src, "-o", exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    res = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert res.returncode == 0, (res.returncode, res.stdout)


RULE = """
#include "dispatch.hpp"
extern "C" int past_(int bytes, int on16) { return galore::norm_past_caches(bytes, on16 != 0); }
"""


@pytest.mark.parametrize("bytes_,on16,past", [(2, 1, 1), (2, 0, 0), (4, 1, 0), (4, 0, 0)])
def test_backward_norms_past_the_caches(tmp_path, bytes_, on16, past):
    """bf16 rows on 16 bytes alone: a thread's eight fp32 values are two pieces of lines that it shares"""
    src, out = str(tmp_path / "shim.cpp"), str(tmp_path / "librule.so")
    with open(src, "w") as f:
        f.write(RULE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC, src, "-o", out], check=True)
    assert ctypes.CDLL(out).past_(bytes_, on16) == past


def padded(x, fill=float("nan")):
    """x on the GPU in rows that start on 16 bytes, the pitch longer than the width"""
    per = 16 // x.element_size()
    pitch = (x.shape[1] + per) // per * per
    big = torch.full((x.shape[0], pitch), fill, dtype=x.dtype, device="cuda")
    big[:, :x.shape[1]] = x.cuda()
    v = big[:, :x.shape[1]]
    assert v.data_ptr() % 16 == 0 and v.stride(0) * x.element_size() % 16 == 0 and v.stride(0) > x.shape[1]
    return v


@pytest.fixture(scope="module")
def gl():
    import paper_2504_20437_amd
    return paper_2504_20437_amd


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(5, 9), (33, 63), (130, 131), (64, 257), (200, 1021), (40, 2731)])
def test_mx4_codes_of_padded_rows(gl, rows, cols, dtype):
    x = values(rows, cols, dtype, rows + cols)
    both = gl.galore_mx4_quantize(padded(x), columns=True)
    only = gl.galore_mx4_quantize(padded(x), rows=False, columns=True)
    want = ora.mx4_encode(host(x)) + ora.mx4_encode(host(x).T)
    for got, w in zip((*both, *only), want + want[2:]):
        assert np.array_equal(host(got), w)


@pytest.mark.gpu
@pytest.mark.parametrize("gate", ["none", "vector", "tokens"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("t,d", [(5, 9), (9, 511), (6, 1021), (5, 2047), (3, 2731), (3, 5461), (2, 8193), (530, 1100)])
def test_norm_backward_of_padded_rows(gl, t, d, dtype, gate):
    """inputs and outputs alike on 16 bytes, so that the call moves them past the caches"""
    x, y, wo, wp, gt = norm_inputs(t, d, dtype, gate, t + d)
    dz, dh = values(t, d, dtype, 5, "gradients"), values(t, d, dtype, 6, "gradients")
    h, _, rstd = ora.norms(host(x), host(y), host(wo), host(wp), 1.0 if gt is None else host(gt), ops.ALPHA, ops.EPS)
    h, R = torch.from_numpy(h).to(DTYPES[dtype]), torch.from_numpy(rstd).float()
    gate_in = gt if gt is None or gt.dim() == 1 else padded(gt)
    room = [padded(torch.zeros((t, d), dtype=DTYPES[dtype]), 7.0) for _ in range(3)]
    got = gl.galore_norm_block_backward(
        *(padded(v) for v in (dz, dh, h, y)), R.cuda(), wo.cuda(), wp.cuda(), gate_in if gt is None or gt.dim() == 2 else gt.cuda(),
        alpha=ops.ALPHA, dX=room[0], dY=room[1], dgate=room[2] if gate == "tokens" else None)
    ops.check_backward(got, host(dz), host(dh), host(h), host(y), host(R), host(wo), host(wp), gt, t, d)
    for v in room:
        whole = v.as_strided((t, v.stride(0)), v.stride())
        assert (whole[:, d:] == 7).all()
