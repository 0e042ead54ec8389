"""The rule of e4m3 rows to the bit: the code of a value is the fp32 quotient by the row's scale to the nearest, which is
the rule of the weights too (GPU; the expected codes are computed on the CPU)."""
import pytest
import torch

from tests import fp8_reference as R

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
# 1, 2 and 8 pieces of 8 values to a thread, 64 to 1024 threads to a row
SIZES = [(1, 64), (2000, 512), (300, 1040), (300, 4096), (260, 8192), (2, 14336), (3, 32768)]


def rule(a):
    """(codes, scales) of the fp32 rows a."""
    scale = (a.abs().amax(-1) / 448.0).clamp(min=R.LEAST)
    return (a / scale[:, None]).to(R.F8), scale


def same(got, want):
    return torch.equal(got.cpu().view(torch.uint8), want.view(torch.uint8))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,K", SIZES)
def test_rows(M, K, dtype):
    from paper_2502_17728_amd import ops
    x = torch.randn((M, K), generator=torch.Generator().manual_seed(M + K)).to(dtype)
    codes, scales = ops.rows_fp8(x.cuda())
    want, scale = rule(x.float())
    assert torch.equal(scales.cpu(), scale) and same(codes, want)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,K", SIZES)
def test_rows_of_the_norm(M, K, dtype):
    from paper_2502_17728_amd import ops
    g = torch.Generator().manual_seed(M + K + 1)
    x, res = (torch.randn((M, K), generator=g).to(dtype) for _ in range(2))
    gamma = (0.5 + torch.rand(K, generator=g)).to(dtype)
    codes, _, total = ops.residual_rmsnorm_fp8(x.cuda(), res.cuda(), gamma.cuda())
    h = x.float() + res.float()
    assert torch.equal(total.cpu(), h.to(dtype)) and same(codes, rule(h * gamma.float())[0])
    codes, _, _ = ops.residual_rmsnorm_fp8(x.cuda())
    assert same(codes, rule(x.float())[0])


@pytest.mark.parametrize("size", [2.0 ** -126, 1e-36, 1e-30, 8e-26, 1e-25, 1e-20, 1e20, 1e38])
def test_the_ends_of_the_range(size):
    from paper_2502_17728_amd import ops
    x = torch.empty((64, 1024)).uniform_(-1, 1, generator=torch.Generator().manual_seed(5)) * size
    codes, scales = ops.rows_fp8(x.cuda())
    want, scale = rule(x)
    assert torch.equal(scales.cpu(), scale) and same(codes, want)


def test_every_tie():
    """Quotients half way between neighbouring codes, and one fp32 step to either side of that."""
    from paper_2502_17728_amd import ops
    v = torch.arange(0x7F, dtype=torch.uint8).view(R.F8).float()
    tie = (v[1:] + v[:-1]) / 2
    for scale in (1.0, 3.0 / 7.0, 1.1):
        x = torch.zeros((3, 256))
        x[0, :126], x[1, :126], x[2, :126] = tie, torch.nextafter(tie, torch.tensor(1e9)), torch.nextafter(tie, torch.tensor(0.0))
        x[:, 128:254] = -x[:, :126]
        x[:, 127] = 448.0
        x = x * torch.tensor(scale)
        codes, _ = ops.rows_fp8(x.cuda())
        assert same(codes, rule(x)[0])


def test_a_column_of_weights_has_the_codes_of_the_same_row():
    from paper_2502_17728_amd import ops
    x = torch.randn((16, 1024), generator=torch.Generator().manual_seed(9)).cuda()
    codes, scales = ops.rows_fp8(x)
    w = x.t().contiguous()
    a, b = ops.linear_fp8_prepare(w), ops.linear_fp8_prepare(codes.t().contiguous(), scales=scales)
    assert torch.equal(a.packed, b.packed)
