"""The 8-bit products, rows and log probabilities on the host: every refusal of the C entry points (nothing is launched),
the sizes they ask for, and the launch rules, compiled with the host compiler."""
import ctypes
import functools
import itertools
import os
import subprocess
import tempfile

import pytest
import torch

from paper_2502_17728_amd import build as B
from paper_2502_17728_amd import ops

INVALID, UNSUPPORTED, MISALIGNED = 1, 2, 3
P = [0x7F0000000000 + (i << 36) for i in range(10)]  # aligned fake device addresses, far apart
lib = ops._lib
INF, NAN = float("inf"), float("nan")


def norm(x=P[0], res=P[1], gamma=P[2], M=4, K=64, eps=1e-5, dt=1, sm=P[3], y=P[4]):
    return lib.residual_rmsnorm(x, res, gamma, M, K, eps, dt, sm, y, None)


def norm8(x=P[0], res=P[1], gamma=P[2], M=4, K=64, eps=1e-5, dt=1, sm=P[3], y=P[4], s=P[5]):
    return lib.residual_rmsnorm_fp8(x, res, gamma, M, K, eps, dt, sm, y, s, None)


def rows(x=P[0], M=4, K=64, dt=1, y=P[4], s=P[5]):
    return lib.rows_fp8(x, M, K, dt, y, s, None)


def test_rows_refusals():
    for f in (norm, norm8):
        for bad in (dict(x=None), dict(y=None), dict(M=0), dict(K=0), dict(eps=-1.0), dict(eps=NAN), dict(eps=INF), dict(dt=2),
                    dict(res=None), dict(sm=None), dict(M=1 << 62)):
            assert f(**bad) == INVALID, bad
        for bad in (dict(K=60), dict(K=65544 if f is norm else 65552), dict(K=32784, dt=0), dict(M=1 << 31)):  # (too many threads)
            assert f(**bad) == UNSUPPORTED, bad
        for name in ("x", "res", "gamma", "sm", "y"):
            assert f(**{name: P[9] + 8}) == MISALIGNED, name
        for name in ("x", "res", "gamma", "sm"):  # y over each of the others
            assert f(**{name: P[4] + 16}) == INVALID, name
        assert f(sm=P[0] + 16) == INVALID and f(sm=P[1] - 16) == INVALID and f(sm=P[2]) == INVALID
    assert norm8(s=None) == INVALID and norm8(s=P[0]) == INVALID and norm8(s=P[3]) == INVALID and norm8(s=P[4]) == INVALID
    assert norm8(s=P[9] + 2) == MISALIGNED and norm8(K=72) == UNSUPPORTED
    for bad in (dict(x=None), dict(y=None), dict(s=None), dict(M=0), dict(dt=3), dict(y=P[0]), dict(s=P[0])):
        assert rows(**bad) == INVALID, bad
    assert rows(K=24) == UNSUPPORTED and rows(x=P[0] + 2) == MISALIGNED


def prep(W=P[0], s=None, gamma=P[2], b=P[3], U=None, us=None, ub=None, K=64, N=32, dt=1, packed=P[7], n=1 << 20, out=True):
    d = ops.LinearFp8Weights()
    return lib.linear_fp8_prepare(W, s, gamma, b, U, us, ub, K, N, dt, packed, n, ctypes.byref(d) if out else None, None)


def test_prepare_refusals():
    for bad in (dict(W=None), dict(packed=None), dict(out=False), dict(dt=3), dict(dt=-1), dict(s=P[1]), dict(us=P[1]), dict(ub=P[1]),
                dict(dt=2), dict(dt=2, s=P[1]), dict(dt=2, s=P[1], gamma=None, U=P[4]), dict(dt=2, s=P[1], gamma=None, us=P[5]),
                dict(n=100), dict(K=0), dict(N=0), dict(W=P[7]), dict(gamma=P[7] + 256), dict(b=P[7]), dict(U=P[7])):
        assert prep(**bad) == INVALID, bad
    for bad in (dict(K=72), dict(N=12), dict(K=1 << 23), dict(N=1 << 24)):
        assert prep(**bad) == UNSUPPORTED, bad
    for bad in (dict(W=P[0] + 8), dict(gamma=P[2] + 8), dict(b=P[3] + 4), dict(U=P[4] + 2), dict(packed=P[7] + 128)):
        assert prep(**bad) == MISALIGNED, bad


def test_packed_bytes():
    f = ops.linear_fp8_packed_bytes
    assert f(128, 16) == 128 * 16 + 2 * 64 and f(16, 8) == 128 * 16 + 2 * 64      # K padded to 128, N to 16
    assert f(144, 24) == 256 * 32 + 4 * 64 and f(144, 24, True) == 2 * f(144, 24)
    assert f(4096, 12288) == 4096 * 12288 + 12288 * 8
    assert f(0, 8) == f(16, 0) == f(24, 8) == f(16, 12) == f(1 << 23, 8) == f(16, 1 << 24) == 0


def weights(K=64, N=32, gated=0, version=1, packed=P[7]):
    return ops.LinearFp8Weights(K, N, gated, version, packed)


def linear(x=P[0], s=P[1], w=None, M=4, act=0, res=P[2], dt=1, ws=P[3], n=1 << 30, out=P[4], none=False):
    return lib.linear_fp8(x, s, None if none else ctypes.byref(w or weights()), M, act, res, dt, ws, n, out, None)


def test_linear_refusals():
    for bad in (dict(x=None), dict(s=None), dict(none=True), dict(out=None), dict(M=0), dict(act=-1), dict(act=5), dict(dt=2),
                dict(w=weights(version=0)), dict(w=weights(packed=None)), dict(w=weights(gated=2)), dict(w=weights(K=0)),
                dict(M=1 << 56), dict(out=P[0]), dict(out=P[1]), dict(out=P[7] + 256), dict(out=P[2] + 16), dict(res=P[4] + 16)):
        assert linear(**bad) == INVALID, bad
    for bad in (dict(w=weights(K=72)), dict(w=weights(N=12)), dict(M=1 << 40)):
        assert linear(**bad) == UNSUPPORTED, bad
    for bad in (dict(x=P[0] + 8), dict(s=P[1] + 2), dict(res=P[2] + 8), dict(out=P[4] + 2), dict(ws=P[3] + 16),
                dict(w=weights(packed=P[7] + 16))):
        assert linear(**bad) == MISALIGNED, bad
    # a workspace that is used must not lie over anything
    w = weights(K=14336, N=4096)
    assert lib.linear_fp8_workspace_bytes(100, ctypes.byref(w)) > 0
    for at in (P[0], P[1], P[2], P[4], P[7]):
        assert linear(w=w, M=100, ws=at) == INVALID, hex(at)


def test_linear_workspace():
    f = lambda M, w: lib.linear_fp8_workspace_bytes(M, ctypes.byref(w))
    assert f(1, weights(4096, 12288)) == 0 and f(8192, weights(8192, 28672)) == 0
    n = f(100, weights(14336, 4096))
    assert n > 0 and n % (100 * 4096 * 4) == 0
    assert f(0, weights()) == 0 and f(4, weights(version=3)) == 0 and f(4, weights(K=72)) == 0


def logprobs(x=P[0], stride=100, T=4, V=100, dt=1, scale=1.0, t=P[1], n=2, top=5, lp=P[2], e=P[3], tl=P[4], ti=P[5], ws=P[6],
             nb=1 << 30):
    return lib.token_logprobs(x, stride, T, V, dt, scale, t, n, top, lp, e, tl, ti, ws, nb, None)


def test_logprobs_refusals():
    for bad in (dict(x=None), dict(stride=99), dict(T=0), dict(V=0), dict(V=1 << 30, stride=1 << 30), dict(dt=2), dict(scale=0.0),
                dict(scale=-1.0), dict(scale=NAN), dict(scale=INF), dict(scale=3e38), dict(t=None), dict(lp=None), dict(n=-1),
                dict(n=0), dict(top=-1), dict(top=0), dict(top=65), dict(top=101), dict(tl=None), dict(ti=None),
                dict(t=None, lp=None, n=0, e=None, tl=None, ti=None, top=0), dict(lp=P[0]), dict(e=P[0]), dict(tl=P[3]), dict(ti=P[4]),
                dict(lp=P[1]), dict(T=1 << 60)):
        assert logprobs(**bad) == INVALID, bad
    for bad in (dict(x=P[0] + 1), dict(x=P[0] + 2, dt=0), dict(t=P[1] + 2), dict(lp=P[2] + 1), dict(e=P[3] + 2), dict(tl=P[4] + 3),
                dict(ti=P[5] + 2)):
        assert logprobs(**bad) == MISALIGNED, bad
    big = dict(T=1, V=131072, stride=131072)
    need = lib.token_logprobs_workspace_bytes(1, 131072, 5)
    assert need > 0
    assert logprobs(**big, ws=None, nb=0) == INVALID and logprobs(**big, nb=need - 1) == INVALID
    assert logprobs(**big, ws=P[6] + 16) == MISALIGNED and logprobs(**big, ws=P[0]) == INVALID and logprobs(**big, ws=P[5]) == INVALID
    f = lib.token_logprobs_workspace_bytes
    assert f(0, 10, 0) == f(1, 0, 0) == f(1, 10, 11) == f(1, 100, 65) == f(4096, 8192, 5) == f(1, 8192, 5) == 0


def test_launches_past_the_devices_limit_are_refused():
    """2^32 threads and more in one launch, where the device would refuse it; one row less is past validation."""
    far = [0x7F0000000000 + (i << 46) for i in range(10)]
    # 256 threads to a row of 4096, 64 to one of 512
    for K, most in ((4096, (1 << 24) - 1), (512, (1 << 26) - 4)):
        assert lib.rows_fp8(far[0], most + 1 + 4 * (K == 512), K, 1, far[1], far[2], None) == UNSUPPORTED
        assert lib.rows_fp8(far[0] + 2, most, K, 1, far[1], far[2], None) == MISALIGNED
    w = weights(K=16, N=8)
    # 256 x 256 or 256 x 128 tiles of 512 threads, one column of them
    f = lambda M, x=far[0]: lib.linear_fp8(x, far[1], ctypes.byref(w), M, 0, None, 1, None, 0, far[2], None)
    assert f(1 << 32) == UNSUPPORTED
    f = lambda T, x=far[0]: lib.token_logprobs(x, 8, T, 8, 1, 1.0, None, 0, 0, None, far[1], None, None, None, 0, None)
    assert f(1 << 26) == UNSUPPORTED and f((1 << 26) - 1, far[0] + 1) == MISALIGNED


def test_binding_refuses_cpu_tensors():
    x = torch.zeros((2, 64), dtype=torch.bfloat16)
    for f in (lambda: ops.residual_rmsnorm(x), lambda: ops.residual_rmsnorm_fp8(x), lambda: ops.rows_fp8(x),
              lambda: ops.token_logprobs(x), lambda: ops.linear_fp8_prepare(torch.zeros((64, 64)))):
        with pytest.raises(ValueError):
            f()


# ------------------------------------------------------------------------------- launch rules
SHIM = r"""
#include "fp8_rules.hpp"
using namespace dn;
extern "C" {
void plan(int64_t M, int64_t K, int64_t blocks, int gated, int f32, int64_t fit, int64_t* out) {
    const Fp8Plan p = plan_fp8(M, K, blocks, gated, f32, fit);
    out[0] = p.tile; out[1] = p.rf; out[2] = p.nc; out[3] = p.splits;
    out[4] = fp8_workgroups(p, M, blocks); out[5] = fp8_threads(p);
}
uint64_t space(int64_t M, int64_t K, int64_t blocks, int gated) { return fp8_workspace(M, K, blocks, gated); }
void rows(int64_t M, int64_t K, int64_t* out) { const RowPlan p = plan_rows(M, K); out[0] = p.threads; out[1] = p.pieces; }
void lp(int64_t T, int64_t V, int64_t top, int64_t* out) { const LogprobPlan p = plan_logprobs(T, V, top); out[0] = p.threads; out[1] = p.segments; }
}
"""


@functools.lru_cache(None)
def rules():
    with tempfile.TemporaryDirectory() as d:
        src, so = os.path.join(d, "shim.cpp"), os.path.join(d, "shim.so")
        open(src, "w").write(SHIM)
        subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fPIC", "-shared", "-I", B.CSRC, src, "-o", so])
        return ctypes.CDLL(so)


def call(name, *args, n):
    out = (ctypes.c_int64 * n)()
    getattr(rules(), name)(*[ctypes.c_int64(a) if name != "plan" or i not in (3, 4) else ctypes.c_int(a)
                             for i, a in enumerate(args)], out)
    return list(out)


SIZES = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 128, 129, 256, 257, 500, 1000, 2047, 4096, 8192, 100000]


@pytest.mark.parametrize("gated", [0, 1])
@pytest.mark.parametrize("f32", [0, 1])
def test_product_plans_are_ones_that_exist(gated, f32):
    rules().space.restype = ctypes.c_uint64
    for M, K, N in itertools.product(SIZES, (16, 128, 768, 4096, 14336, 1 << 20), (8, 768, 4096, 12288, 28672, 1 << 20)):
        blocks = (N + 15) // 16 * (1 + gated)
        space = rules().space(ctypes.c_int64(M), ctypes.c_int64(K), ctypes.c_int64(blocks), gated)
        for fit in (1, 2, 3, 5, 16):
            tile, rf, nc, splits, wgs, threads = call("plan", M, K, blocks, gated, f32, fit, n=6)
            if tile < 0:
                assert M <= 64 and splits == 1 and (rf, nc) in [(1, c) for c in (1, 2, 3, 4, 6, 7, 8)] + [(2, c) for c in (1, 2, 3, 4, 6, 7)]
                assert not gated or nc % 2 == 0
                assert wgs == -(-M // (16 * rf)) * -(-blocks // nc) and threads == (256 if rf == 2 and nc > 2 else 512)
            else:
                assert 0 <= tile <= (3 if f32 else 4) and M > 16
                # every split has a stage, and its sums fit what the caller was asked for
                assert 1 <= splits <= min(fit, 16) and splits <= (K + 127) // 128
                assert splits == 1 or splits * M * blocks * 64 <= space
                bm, bn, t = [(64, 64, 128), (64, 128, 256), (128, 128, 256), (256, 128, 512), (256, 256, 512)][tile]
                assert threads == t and wgs == -(-M // bm) * -(-blocks * 16 // bn) * splits


def test_row_plans_hold_the_row():
    for M, K in itertools.product(SIZES, list(range(8, 2048, 8)) + [4096, 8192, 14336, 28672, 32768, 65536]):
        threads, pieces = call("rows", M, K, n=2)
        assert threads in (64, 256, 1024) and pieces in (1, 2, 4, 8) and threads * pieces * 8 >= K


def test_logprob_plans():
    for T, V, top in itertools.product(SIZES, (1, 8, 1000, 8192, 32000, 50257, 131072, 1 << 20, (1 << 30) - 1), (0, 1, 64)):
        threads, segments = call("lp", T, V, top, n=2)
        assert threads in (64, 128, 256, 512) and 1 <= segments <= 16
        assert segments == 1 or (V + 14) // 8 >= segments  # every segment but the last has tokens
