"""Which outputs of the 8-bit products are stored past the caches: those of the 256-row tiles whose rows are whole 64-byte
pieces; both ways to the same results."""
import ctypes
import functools
import os
import subprocess
import tempfile

import pytest
import torch

from paper_2502_17728_amd import build as B
from tests import test_linear_fp8 as L
from tests.test_fp8_kernels import kernel

BF16, F32 = torch.bfloat16, torch.float32
# tile 3, tile 4 (256 x 128, 256 x 256); rows of whole 64-byte pieces in bf16 and fp32, in neither, in fp32 alone
PLAIN = [(200, 400, 16640), (200, 400, 16648), (200, 400, 16656), (200, 144, 33216), (200, 144, 33224), (200, 144, 33232)]
GATED = [(200, 400, 8384), (200, 400, 8392), (200, 400, 8400), (200, 144, 16640), (200, 144, 16648), (200, 144, 16656)]

SHIM = r"""
#include "fp8_rules.hpp"
using namespace dn;
extern "C" int streams(int64_t M, int64_t K, int64_t N, int gated, int f32, uint64_t out) {
    return fp8_streams_out(plan_fp8(M, K, fp8_layout(K, N, gated).blocks, gated, f32, kMaxSplits), N, f32, out);
}
"""


@functools.lru_cache(None)
def rule():
    with tempfile.TemporaryDirectory() as d:
        src, so = os.path.join(d, "shim.cpp"), os.path.join(d, "shim.so")
        open(src, "w").write(SHIM)
        subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fPIC", "-shared", "-I", B.CSRC, src, "-o", so])
        f = ctypes.CDLL(so).streams
        f.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_int] * 2 + [ctypes.c_uint64]
        return f


@pytest.mark.parametrize("f32", [0, 1])
@pytest.mark.parametrize("gated", [0, 1])
def test_whole_pieces_alone(gated, f32):
    reached = set()
    for M, K, N in GATED if gated else PLAIN:
        got = rule()(M, K, N, gated, f32, 1 << 20)
        assert got == (N * (4 if f32 else 2) % 64 == 0)
        assert not rule()(M, K, N, gated, f32, (1 << 20) + 16) and got == rule()(M, K, N, gated, f32, (1 << 20) + 64)
        reached.add((kernel(M, K, N, gated, f32)[0], got))
    assert reached == {(tile, s) for tile in ((3,) if f32 else (3, 4)) for s in (0, 1)}
    for M, K, N in ((1, 4096, 4096), (32, 14336, 4096), (65, 784, 64), (65, 784, 8320), (129, 784, 5504)):  # smaller tiles
        assert kernel(M, K, N, gated, f32)[0] < 3 and not rule()(M, K, N, gated, f32, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("gated", [0, 1])
@pytest.mark.parametrize("which", range(6))
def test_results(which, gated, dtype):
    from paper_2502_17728_amd import ops
    M, K, N = (GATED if gated else PLAIN)[which]
    c = L.case(M, K, N, which, bool(gated), True, dtype)
    w = L.prepared(ops, c)
    step = 16 // torch.finfo(dtype).bits * 8  # elements to 16 bytes
    outs = []
    for offset in (0, step, 4 * step):
        flat = torch.full((M * N + 8 * step,), -7.0, dtype=dtype, device="cuda")
        out = flat[offset:offset + M * N].view(M, N)
        outs.append(ops.linear_fp8(c["x"], c["xs"], w, "silu" if gated else "none", c["r"], out=out))
        assert (flat[:offset] == -7).all() and (flat[offset + M * N:] == -7).all()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    L.check(c, "silu" if gated else "none", outs[0])
