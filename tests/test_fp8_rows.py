"""Residual sums, RMSNorm and e4m3 rows against plain 64-bit forms (tests/fp8_reference.py)."""
import math

import pytest
import torch

from tests import fp8_reference as R

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
# roundings of 1 / rms: a thread's chain of up to 64 squares, 6 + 16 sums of partial sums (all halved by the
# root), the division by K, eps, root and quotient; then gamma and the product with it
R_NORM = (0.5 * 90 + 4 + 3) * 2.0 ** -24


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2502_17728_amd import ops as _ops
    return _ops


def rows(M, K, dtype, seed, outliers=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((M, K), generator=g, device="cuda")
    if outliers:
        x[:, ::97] *= 20
    return x.to(dtype)


SIZES = [(1, 16), (1, 8192), (3, 64), (5, 768), (7, 1040), (2, 1024 + 16), (300, 512), (257, 2064), (260, 8192), (2, 14336),
         (1, 16384), (2, 28672), (1, 32768)]


def check_norm(ops, x, residual, gamma, eps):
    h, r, a = R.rmsnorm(x, residual, gamma, eps)
    y, total = ops.residual_rmsnorm(x, residual, gamma, eps)
    codes, scales, total8 = ops.residual_rmsnorm_fp8(x, residual, gamma, eps)
    ref = a * r[:, None]
    half = R.HALF[x.dtype]
    assert y.dtype == x.dtype and codes.dtype == R.F8 and scales.dtype == F32
    R.assert_within(y, ref, ref.abs() * (half + R_NORM))
    if residual is None:
        assert total is None and total8 is None
    else:
        assert torch.equal(total, total8)
        R.assert_within(total, h, h.abs() * (half + 2.0 ** -24))
    v, s, bad = R.quantised(a)
    assert not bad.any()
    R.assert_codes(codes, v)
    R.assert_within(scales, s * r, s * r * (R_NORM + 3 * 2.0 ** -24))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,K", SIZES + [(1, 65536), (40, 40000)])
def test_sizes(ops, M, K, dtype):
    if dtype == F32 and K > 32768:
        with pytest.raises(ops.DNError):
            ops.residual_rmsnorm(rows(M, K, dtype, 1))
        return
    x, res = rows(M, K, dtype, 1), rows(M, K, dtype, 2, False)
    gamma = (0.5 + torch.rand(K, device="cuda")).to(dtype)
    check_norm(ops, x, res, gamma, 1e-5)
    check_norm(ops, x, None, None, 1e-6)
    check_norm(ops, x, res, None, 0.0)
    check_norm(ops, x, None, gamma, 1.0)
    codes, scales = ops.rows_fp8(x)
    v, s, _ = R.quantised(x.double())
    R.assert_codes(codes, v)
    R.assert_within(scales, s, s * 2.0 ** -23)


def test_rows_of_eight(ops):
    # K a multiple of 8 but not of 16: rows of values, and no codes
    x = rows(9, 72, BF16, 5)
    h, r, a = R.rmsnorm(x, None, None, 1e-5)
    y, _ = ops.residual_rmsnorm(x)
    R.assert_within(y, a * r[:, None], (a * r[:, None]).abs() * (2.0 ** -8 + R_NORM))
    for f in (ops.residual_rmsnorm_fp8, ops.rows_fp8):
        with pytest.raises(ops.DNError):
            f(x)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("K", [64, 4096, 20480])
def test_the_stream_is_updated_in_place(ops, dtype, K):
    x, res = rows(6, K, dtype, 3), rows(6, K, dtype, 4)
    y, total = ops.residual_rmsnorm(x, res)
    codes, scales, _ = ops.residual_rmsnorm_fp8(x, res)
    for which in (0, 1):
        a, b = x.clone(), res.clone()
        y2, t2 = ops.residual_rmsnorm(a, b, total=(a, b)[which])
        assert t2 is (a, b)[which] and torch.equal(t2, total) and torch.equal(y2, y)
        a, b = x.clone(), res.clone()
        c2, s2, t2 = ops.residual_rmsnorm_fp8(a, b, total=(a, b)[which])
        assert torch.equal(t2, total) and torch.equal(s2, scales) and torch.equal(c2.view(torch.uint8), codes.view(torch.uint8))
    a = x.clone()  # a row added to itself, in place
    y3, t3 = ops.residual_rmsnorm(a, a, total=a)
    assert torch.equal(t3, (2 * x.double()).to(dtype))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("K", [64, 1040, 12288])
def test_rows_that_are_not_numbers(ops, dtype, K):
    x = rows(8, K, dtype, 6)
    x[1, 3], x[2, K - 1], x[4, 0] = math.nan, math.inf, -math.inf
    x[5] = 0
    x[6] = torch.finfo(dtype).tiny
    codes, scales = ops.rows_fp8(x)
    v, s, bad = R.quantised(x.double())
    assert bad.tolist() == [False, True, True, False, True, False, False, False]
    R.assert_codes(codes, v)
    assert (codes[bad].double() == 0).all() and torch.isnan(scales[bad]).all()
    R.assert_within(scales[~bad], s[~bad], s[~bad] * 2.0 ** -23)
    assert (codes[5].double() == 0).all() and scales[5] == 2.0 ** -120
    codes, scales, _ = ops.residual_rmsnorm_fp8(x)
    assert (codes[bad].double() == 0).all() and torch.isnan(scales[bad]).all() and torch.isfinite(scales[~bad]).all()
    y, _ = ops.residual_rmsnorm(x)
    assert torch.isfinite(y[~bad]).all() and torch.isnan(y[1]).all()
    # an all-zero row without eps is 0 / 0, as RMSNorm of it is
    assert torch.isnan(ops.residual_rmsnorm_fp8(x, eps=0.0)[1][5])
    gamma = torch.ones(K, dtype=dtype, device="cuda")
    gamma[2] = math.inf
    assert torch.isnan(ops.residual_rmsnorm_fp8(x, gamma=gamma)[1]).all()


def test_outputs_given(ops):
    x, res = rows(3, 256, BF16, 7), rows(3, 256, BF16, 8)
    out, total = torch.empty_like(x), torch.empty_like(x)
    y, t = ops.residual_rmsnorm(x, res, out=out, total=total)
    assert y is out and t is total
    codes, scales = torch.empty((3, 256), dtype=R.F8, device="cuda"), torch.empty(3, device="cuda")
    c, s, t = ops.residual_rmsnorm_fp8(x, res, total=total, codes=codes, scales=scales)
    assert c is codes and s is scales and t is total
    c2, s2 = ops.rows_fp8(x, codes=codes, scales=scales)
    assert c2 is codes and s2 is scales


def test_refusals(ops):
    x, res = rows(4, 64, BF16, 9), rows(4, 64, BF16, 10)
    for bad in (x.cpu(), x[0], x[:, ::2], x.half()):
        with pytest.raises((ValueError, TypeError)):
            ops.residual_rmsnorm(bad)
    with pytest.raises(ValueError):
        ops.residual_rmsnorm(x, res.float())
    with pytest.raises(ValueError):
        ops.residual_rmsnorm(x, res[:3])
    with pytest.raises(ValueError):
        ops.residual_rmsnorm(x, total=res)
    with pytest.raises(ValueError):
        ops.residual_rmsnorm(x, gamma=torch.ones(64, device="cuda"))
    with pytest.raises(ValueError):
        ops.rows_fp8(x, codes=torch.empty((4, 64), dtype=torch.uint8, device="cuda"))
    with pytest.raises(ops.DNError):
        ops.residual_rmsnorm(x, res, out=x)
    with pytest.raises(ops.DNError):
        ops.residual_rmsnorm(x, eps=-1.0)
    both = torch.randn((8, 64), device="cuda").to(BF16)
    with pytest.raises(ops.DNError):  # half of x
        ops.residual_rmsnorm(both[:4], res, total=both[2:6])
