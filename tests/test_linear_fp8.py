"""Products of e4m3 codes and their epilogue against plain 64-bit forms (tests/fp8_reference.py)."""
import math

import pytest
import torch

from tests import fp8_reference as R

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2502_17728_amd import ops as _ops
    return _ops


def case(M, K, N, seed, gated=False, bias=True, residual=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *shape: torch.randn(shape, generator=g, device="cuda")
    x = rnd(M, K)
    x[:, ::101] *= 10
    c = {}
    v, s, _ = R.quantised(x.double())
    c["x"], c["xs"] = v.float().to(R.F8), s.float()
    for w, ws, b in (("w", "ws", "b"), ("up", "us", "ub"))[: 2 if gated else 1]:
        v, s, _ = R.quantised((rnd(K, N) * K ** -0.5).t().double())
        c[w], c[ws] = v.t().float().to(R.F8).contiguous(), s.float()
        if bias:
            c[b] = rnd(N)
    if residual is not None:
        c["r"] = rnd(M, N).to(residual)
    return c


def prepared(ops, c):
    return ops.linear_fp8_prepare(c["w"], scales=c["ws"], bias=c.get("b"), up=c.get("up"), up_scales=c.get("us"),
                                  up_bias=c.get("ub"))


def check(c, act, got):
    ref, e = R.linear(c["x"], c["xs"], c["w"], c["ws"], c.get("b"), act, c.get("up"), c.get("us"), c.get("ub"), c.get("r"),
                      got.dtype == F32)
    R.assert_within(got, ref, e + (ref.abs() + e) * R.HALF[got.dtype])
    # and as a whole: the output's rounding, and what sums of random signs leave of the bound above (fp32: sqrt(K)
    # roundings of a sum that is sqrt(K) of the result's parts; 8-bit sums: 15 2^-13 of a group's largest product,
    # four times a typical one, and a group's sum is four times a typical product too: 2^-9 at most, with signs that
    # cancel over the group's 16, 2^-11)
    K = c["x"].shape[1]
    sums = 4 * math.sqrt(K) * 2.0 ** -24 + (0.0 if got.dtype == F32 else 2.0 ** -11)
    assert ((got.double() - ref).norm() / ref.norm()).item() <= R.HALF[got.dtype] + 2 * sums


SIZES = [(1, 16, 8), (1, 4096, 4096), (2, 128, 16), (3, 144, 24), (16, 272, 136), (17, 1040, 264), (33, 2064, 1000),
         (64, 512, 64), (65, 112, 72), (100, 4096, 520), (128, 1024, 1024), (129, 640, 2056), (257, 1296, 776),
         (300, 14336, 256), (513, 768, 768), (1000, 256, 512), (1, 14336, 64), (5, 8192, 48)]


@pytest.mark.parametrize("M,K,N", SIZES)
def test_sizes(ops, M, K, N):
    for gated, act, bias, res, dtype in ((False, "none", True, None, BF16), (False, "gelu", False, BF16, BF16),
                                         (True, "silu", True, F32, F32), (True, "gelu_tanh", False, None, BF16)):
        c = case(M, K, N, M + K + N, gated, bias, res)
        got = ops.linear_fp8(c["x"], c["xs"], prepared(ops, c), act, c.get("r"), out_dtype=dtype)
        assert got.dtype == dtype and got.shape == (M, N)
        check(c, act, got)


@pytest.mark.parametrize("M", [1, 40, 300, 1025])
@pytest.mark.parametrize("act", sorted(R.ACT))
@pytest.mark.parametrize("gated", [False, True])
def test_activations(ops, M, act, gated):
    c = case(M, 320, 264, 7, gated)
    c["ws"] = c["ws"] * 4  # arguments from -20 to 20
    for dtype in (BF16, F32):
        check(c, act, ops.linear_fp8(c["x"], c["xs"], prepared(ops, c), act, out_dtype=dtype))


@pytest.mark.parametrize("M", [1, 16, 31, 128, 600])
@pytest.mark.parametrize("gated", [False, True])
def test_every_split_and_none(ops, M, gated):
    c = case(M, 8192, 96, 8, gated, True, F32)
    w = prepared(ops, c)
    n = ops.linear_fp8_workspace_bytes(M, w)
    for size in {0, 1024, n // 3, n // 2, n, 2 * n + 512}:
        space = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
        check(c, "none", ops.linear_fp8(c["x"], c["xs"], w, residual=c["r"], workspace=space))
        if size > n:
            assert (space[n:] == 255).all()


@pytest.mark.parametrize("M", [1, 70, 400])
def test_onto_the_residual_itself(ops, M):
    for K, N in ((256, 136), (8192, 64)):
        c = case(M, K, N, 9, residual=BF16)
        w = prepared(ops, c)
        ref = ops.linear_fp8(c["x"], c["xs"], w, residual=c["r"])
        stream = c["r"].clone()
        assert ops.linear_fp8(c["x"], c["xs"], w, residual=stream, out=stream) is stream
        assert torch.equal(stream, ref)


@pytest.mark.parametrize("M", [1, 50, 500])
def test_rows_and_columns_that_are_not_numbers(ops, M):
    c = case(M, 400, 72, 10)
    c["xs"][M // 2] = math.nan
    c["ws"][5] = math.nan
    c["b"][9] = math.inf
    codes = c["w"].view(torch.uint8).clone()
    codes[399, 20] = 0x7F  # a NaN code in the last row of W
    c["w"] = codes.view(R.F8)
    got = ops.linear_fp8(c["x"], c["xs"], prepared(ops, c))
    other = torch.ones((M, 72), dtype=torch.bool, device="cuda")
    other[M // 2] = False
    other[:, [5, 9, 20]] = False
    assert torch.isnan(got[M // 2]).all() and torch.isnan(got[:, 5]).all() and torch.isnan(got[:, 20]).all()
    inf = torch.arange(M, device="cuda") != M // 2
    assert (got[inf, 9] == math.inf).all() and torch.isfinite(got[other]).all()
    # a NaN code in a row's last piece stays in its row, where K ends inside a stage as well
    x = c["x"].view(torch.uint8).clone()
    x[0, 399] = 0x7F
    got = ops.linear_fp8(x.view(R.F8), torch.ones_like(c["xs"]), prepared(ops, case(M, 400, 72, 10)))
    assert torch.isnan(got[0]).all() and torch.isfinite(got[1:]).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("K,N", [(16, 8), (144, 24), (1040, 200), (4096, 520)])
def test_weights_quantised_by_prepare(ops, dtype, K, N):
    g = torch.Generator(device="cuda").manual_seed(K)
    W, U = (torch.randn((K, N), generator=g, device="cuda").to(dtype) for _ in range(2))
    W[:, 3] = 0
    gamma = (0.5 + torch.rand(K, generator=g, device="cuda")).to(dtype)
    eye = torch.eye(K, device="cuda")[: min(K, 200)]
    x, xs = eye.to(R.F8), torch.ones(len(eye), device="cuda")  # the product reads the weights back
    for kw in ({}, {"gamma": gamma}):
        a = W.float() * kw["gamma"].float()[:, None] if kw else W.float()
        v, s, _ = R.quantised(a.t().double())
        back = ops.linear_fp8(x, xs, ops.linear_fp8_prepare(W, **kw), out_dtype=F32)
        # codes by the rule from the fp32 product: scale 1 rounding, quotient 1, product with the scale 1
        codes = (back / s.float()).t()
        assert ((codes.double() - v[:, : len(eye)]).abs() <= R.half_step_e4m3(v[:, : len(eye)]) * (1 + 1e-4)).all()
    both = ops.linear_fp8_prepare(W, gamma=gamma, up=U)
    assert both.gated and both.N == N
    one = ops.linear_fp8(x, xs, ops.linear_fp8_prepare(W, gamma=gamma), out_dtype=F32)
    two = ops.linear_fp8(x, xs, ops.linear_fp8_prepare(U, gamma=gamma), out_dtype=F32)
    got = ops.linear_fp8(x, xs, both, "relu", out_dtype=F32)
    assert torch.equal(got, torch.where(one < 0, torch.zeros_like(one), one) * two)


def test_columns_that_are_not_numbers(ops):
    W = torch.randn((64, 24), device="cuda").to(BF16)
    W[5, 2], W[63, 7] = math.nan, -math.inf
    got = ops.linear_fp8(*ops.rows_fp8(torch.randn((3, 64), device="cuda")), ops.linear_fp8_prepare(W))
    assert torch.isnan(got[:, [2, 7]]).all() and torch.isfinite(got[:, [c for c in range(24) if c not in (2, 7)]]).all()


def test_given_codes_and_quantised_weights_agree(ops):
    W = torch.randn((512, 264), device="cuda")
    v, s, _ = R.quantised(W.t().double())
    s = s.float()
    codes = (W / s).to(R.F8)
    a, b = ops.linear_fp8_prepare(W), ops.linear_fp8_prepare(codes, scales=s)
    n = 17 * 16 * 512
    assert torch.equal(a.packed[:n], b.packed[:n])


def test_refusals(ops):
    c = case(4, 64, 32, 11, residual=BF16)
    w = prepared(ops, c)
    x, xs = c["x"], c["xs"]
    with pytest.raises(TypeError):
        ops.linear_fp8(x, xs, c["w"])
    with pytest.raises(ValueError):
        ops.linear_fp8(x, xs, w, "swish")
    for bad in (x.cpu(), x[0], x[:, :32], x.view(torch.uint8), x.float()):
        with pytest.raises(ValueError):
            ops.linear_fp8(bad, xs, w)
    for bad in (xs[:3], xs.double(), None, xs.cpu()):
        with pytest.raises(ValueError):
            ops.linear_fp8(x, bad, w)
    with pytest.raises(ValueError):
        ops.linear_fp8(x, xs, w, residual=c["r"].float(), out_dtype=BF16)
    with pytest.raises(ValueError):
        ops.linear_fp8(x, xs, w, out=torch.empty((4, 16), device="cuda"))
    with pytest.raises((ValueError, TypeError)):
        ops.linear_fp8(x, xs, w, out_dtype=torch.float16)
    with pytest.raises(ops.DNError):
        ops.linear_fp8_prepare(c["w"])  # codes without scales
    with pytest.raises(ops.DNError):
        ops.linear_fp8_prepare(torch.randn((64, 32), device="cuda"), scales=c["ws"])
    with pytest.raises(ops.DNError):
        ops.linear_fp8_prepare(torch.randn((72, 32), device="cuda"))
    with pytest.raises(ops.DNError):
        ops.linear_fp8_prepare(torch.randn((64, 12), device="cuda"))
    with pytest.raises(ValueError):
        ops.linear_fp8_prepare(c["w"], scales=c["ws"], bias=torch.zeros(32, dtype=BF16, device="cuda"))
    with pytest.raises(ValueError):
        ops.linear_fp8_prepare(c["w"], scales=c["ws"], up=c["w"][:, :16].contiguous(), up_scales=c["ws"][:16])
