"""Every kernel that the launch rule of the 8-bit products can choose, run: sizes for each, ragged in M, N and K, their choice
checked on the CPU, so that a change of the rule cannot leave a kernel untested."""
import functools
import itertools

import pytest
import torch

from tests import test_linear_fp8 as L
from tests.test_fp8_rules import call

BF16, F32 = torch.bfloat16, torch.float32
# (M, K, N): few rows with 1 to 8 column blocks to a workgroup, streamed and through rings; tiles of 64 x 64 to 256 x 256 with K whole and
# with K split.  K ends inside a stage of 128 (four stages and more), N inside a block of 16.
PLAIN = [(13, 784, 24), (16, 784, 4136), (13, 784, 8344), (16, 784, 12568), (13, 784, 16600), (13, 1296, 28056), (16, 784, 28760),
         (49, 784, 1032), (49, 784, 2088), (33, 784, 4136), (33, 784, 6280), (33, 784, 8344), (13, 784, 24776),
         (65, 784, 72), (65, 784, 8344), (129, 784, 11064), (257, 784, 13224), (257, 784, 21864),
         (65, 4112, 72), (65, 8208, 1032), (1363, 8208, 136), (8197, 14352, 72), (4099, 14352, 200), (257, 14352, 13224)]
GATED = [(13, 784, 24), (16, 784, 4136), (13, 784, 8344), (16, 784, 12568), (49, 784, 1032), (49, 784, 2088), (33, 784, 4136),
         (65, 784, 40), (65, 784, 4136), (129, 784, 5512), (257, 784, 6616), (257, 784, 11064),
         (65, 4112, 40), (65, 4112, 1032), (1363, 8208, 72), (8193, 14320, 40), (4099, 14352, 104), (257, 14352, 6616)]


# (M, N) that reach each tile with one to five stages, fewer than their copies run ahead and more
SHALLOW = {0: [(65, 72), (65, 8344), (65, 16648), (129, 16648), (129, 21864), (65, 33192), (129, 33192)],
           1: [(65, 72), (65, 4104), (65, 8344), (129, 8344), (129, 11064), (65, 16648), (129, 16648)]}
DEPTHS = [16, 144, 272, 400, 528]


@functools.lru_cache(None)
def kernel(M, K, N, gated, f32):
    """(tile, rows, column blocks, is K split): tile < 0 for few rows."""
    tile, rf, nc, splits, _, _ = call("plan", M, K, (N + 15) // 16 * (1 + gated), gated, f32, 16, n=6)
    return tile, rf, nc, splits > 1


@pytest.mark.parametrize("gated", [0, 1])
@pytest.mark.parametrize("f32", [0, 1])
def test_sizes_reach_every_kernel(gated, f32):
    rows = list(range(1, 65, 3)) + [16, 32, 64, 65, 97, 129, 160, 193, 257, 320, 385, 513, 700, 1025, 1363, 2049, 4099, 8192, 8197, 20000]
    widths = [8, 72, 136, 200, 520, 768, 1032, 2048, 2088, 4096, 4136, 6280, 8192, 8344, 10240, 11064, 12288, 12568, 13224, 14336,
              16600, 20480, 21864, 24776, 28056, 28672, 28760, 34000, 65536, 131072]
    depths = [16, 128, 784, 1296, 2064, 4096, 8192, 14336, 28672, 65536]
    chosen = {kernel(M, K, N, gated, f32) for M, K, N in itertools.product(rows, depths, widths)}
    run = {kernel(M, K, N, gated, f32) for M, K, N in (GATED if gated else PLAIN)}
    assert chosen <= run, chosen - run


@pytest.mark.parametrize("gated", [0, 1])
@pytest.mark.parametrize("f32", [0, 1])
@pytest.mark.parametrize("K", DEPTHS)
def test_shallow_sizes_reach_every_tile(K, gated, f32):
    assert {kernel(M, K, N, gated, f32)[0] for M, N in SHALLOW[gated]} == set(range(4 if f32 else 5))


def _run(ops, M, K, N, gated, dtype):
    c = L.case(M, K, N, M + N, gated, True, dtype)
    w = L.prepared(ops, c)
    space = torch.full((ops.linear_fp8_workspace_bytes(M, w),), 255, dtype=torch.uint8, device="cuda")
    act = "silu" if gated else "gelu"
    outs = []
    for _ in range(2):
        around = torch.full((M + 2, N), -7.0, dtype=dtype, device="cuda")
        got = ops.linear_fp8(c["x"], c["xs"], w, act, c["r"], out=around[1:-1], workspace=space)
        assert (around[0] == -7).all() and (around[-1] == -7).all()
        outs.append(got)
    assert torch.equal(*outs)
    L.check(c, act, outs[0])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,K,N", PLAIN)
def test_plain(M, K, N, dtype):
    from paper_2502_17728_amd import ops
    _run(ops, M, K, N, False, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,K,N", GATED)
def test_gated(M, K, N, dtype):
    from paper_2502_17728_amd import ops
    _run(ops, M, K, N, True, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("gated", [0, 1])
@pytest.mark.parametrize("K", DEPTHS)
def test_shallow(K, gated, dtype):
    from paper_2502_17728_amd import ops
    for M, N in SHALLOW[gated]:
        _run(ops, M, K, N, bool(gated), dtype)


def test_rows_take_no_more_pieces_than_their_kernels_have():
    most = {64: 2, 256: 4, 1024: 8}
    seen = set()
    for M in (1, 2, 255, 256, 257, 5000):
        for K in range(8, 65537, 8):
            threads, pieces = call("rows", M, K, n=2)
            assert pieces <= most[threads] and (pieces <= 4 or K > 32768), (M, K)
            seen.add((threads, pieces))
    assert seen == {(t, p) for t in most for p in (1, 2, 4, 8) if p <= most[t]}


def test_no_plan_for_fp32_outputs_streams_seven_blocks():
    for M, K, blocks, gated in itertools.product((1, 5, 16, 17, 33, 64), (16, 784, 4096, 14336), range(1, 6000, 3), (0, 1)):
        assert call("plan", M, K, blocks, gated, 1, 16, n=6)[:3] != [-1, 1, 7]


def test_rows_without_ranks_take_64_128_or_512_threads():
    seen = {call("lp", T, V, 0, n=2)[0] for T in (1, 5, 255, 256, 500, 511, 512, 1000, 1999, 2000, 4000, 5000, 100000)
            for V in (1, 100, 1000, 8191, 8192, 16383, 16384, 32000, 131072, 1 << 25)}
    assert seen == {64, 128, 512}
