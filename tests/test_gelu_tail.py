"""GELU relative to itself: its left tail falls to 1e-35 and keeps its digits there (GPU).  The products are zero, so the
argument is the bias, exactly."""
import math

import pytest
import torch

from tests import fp8_reference as R

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
N = 4104


def arguments():
    z = torch.cat([torch.linspace(-12.5, 8.0, N - 40, dtype=torch.float64),
                   torch.logspace(-20, 0, 20, dtype=torch.float64), -torch.logspace(-20, 0, 20, dtype=torch.float64)])
    return z.float().cuda()


# one row, a ring's 32, tiles of 64 and more
@pytest.mark.parametrize("M", [1, 32, 130, 600])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_relative_error(M, gated, dtype):
    from paper_2502_17728_amd import ops
    z = arguments()
    zero = lambda *s: torch.zeros(s, dtype=torch.uint8, device="cuda").view(R.F8)
    one = torch.ones(N, device="cuda")
    kw = dict(up=zero(32, N), up_scales=one, up_bias=one) if gated else {}
    w = ops.linear_fp8_prepare(zero(32, N), scales=one, bias=z, **kw)
    got = ops.linear_fp8(zero(M, 32), torch.ones(M, device="cuda"), w, "gelu", out_dtype=dtype)
    assert (got == got[0]).all()
    ref = 0.5 * z.double() * torch.special.erfc(z.double() * -math.sqrt(0.5))  # (1 + erf would cancel, in 64 bits too)
    # q(a) = t P(t) e^(-a^2 / 2), t = 1 / (1 + p a), of half steps 2^-24: P's own error 2.2; t 4 (p, p a + 1, the reciprocal's 2), by
    # which q moves 2.7 times as much at most; P's evaluation 5; the power's exponent three roundings of z^2 / 2, the power itself 2, its
    # products 2; the last sum and the output's rounding.  With a bf16 output P's own error is 3.6e-5.
    bound = (2.2 + 4 * 2.7 + 5 + 1.5 * z.double() ** 2 + 2 + 2 + 2) * 2.0 ** -24
    if dtype == BF16:
        bound = bound + 3.6e-5 + 2.0 ** -8
    R.assert_within(got[0], ref, bound * ref.abs())


def test_the_ends():
    from paper_2502_17728_amd import ops
    z = torch.tensor([float("inf"), -float("inf"), float("nan"), 0.0, -0.0, 1e30, -1e30, 40.0, -40.0, 3e38, -3e38] + [0.0] * 5).cuda()
    zero = lambda *s: torch.zeros(s, dtype=torch.uint8, device="cuda").view(R.F8)
    w = ops.linear_fp8_prepare(zero(16, 16), scales=torch.ones(16, device="cuda"), bias=z)
    for dtype in (BF16, F32):
        for M in (1, 200):
            got = ops.linear_fp8(zero(M, 16), torch.ones(M, device="cuda"), w, "gelu", out_dtype=dtype)
            want = torch.where(z > 0, z, torch.zeros_like(z))
            want[2] = float("nan")
            assert torch.equal(got.float().nan_to_num(nan=-7.0), want.to(dtype).float().nan_to_num(nan=-7.0).expand(M, 16))
