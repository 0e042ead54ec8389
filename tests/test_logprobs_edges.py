"""Token log probabilities at the edges of their numbers: ranks beside NaNs of either kind, logits whose difference has
no room in fp32."""
import math

import pytest
import torch

from tests import fp8_reference as R

BF16, F32 = torch.bfloat16, torch.float32
# bits of a signalling and of a quiet NaN
NANS = {BF16: (torch.int16, (0x7F81, 0x7FC0)), F32: (torch.int32, (0x7F800001, 0x7FC00000))}


def ranked(logits, top):
    """The ids of the `top` largest numbers of each row, the lowest first among equals; -1 where there are no more."""
    x = logits.double()
    none = torch.isnan(x)
    key = torch.where(none, torch.full_like(x, -math.inf), x)
    # NaNs behind every number, -inf included
    order = torch.argsort(none.long(), dim=1, stable=True)
    order = order.gather(1, torch.sort(key.gather(1, order), dim=1, descending=True, stable=True)[1])
    ids = order[:, :top]
    return torch.where(none.gather(1, ids), torch.full_like(ids, -1), ids)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [0, 1])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,V", [(8, 40), (8, 3000), (8, 50001), (600, 4099), (2100, 1000), (4100, 264)])
def test_a_nan_costs_no_other_token_its_rank(T, V, dtype, kind):
    from paper_2502_17728_amd import ops
    g = torch.Generator(device="cuda").manual_seed(T + V)
    logits = torch.randn((T, V), generator=g, device="cuda").to(dtype)
    as_int, nans = NANS[dtype]
    bits = logits.view(as_int)
    top = 5
    for row in range(T):
        # row r: the likeliest tokens share their group of 8 with a NaN in every place in turn
        if row < 64:
            at = (V // 2) // 8 * 8
            logits[row, at:at + 8] = torch.arange(20.0, 28.0, device="cuda").to(dtype)
            bits[row, at + row % 8] = nans[kind]
    bits[-1, ::3] = nans[kind]  # many of them
    got = ops.token_logprobs(logits, None, top)
    assert torch.equal(got["top_ids"].long(), ranked(logits, top))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", [0, 1])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V", [64, 5000, 70001])
def test_rows_of_little_but_nans(V, dtype, kind):
    from paper_2502_17728_amd import ops
    as_int, nans = NANS[dtype]
    logits = torch.empty((4, V), dtype=dtype, device="cuda")
    logits.view(as_int).fill_(nans[kind])
    logits[1, V - 1] = 2.0
    logits[2, ::7] = -math.inf
    logits[3, 5], logits[3, 6] = -1.0, 1.0
    got = ops.token_logprobs(logits, None, 3)
    assert torch.equal(got["top_ids"].long(), ranked(logits, 3))
    assert torch.isnan(got["entropy"]).all() and torch.isnan(got["top_logprobs"]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V", [6, 40000])
def test_logits_further_apart_than_their_type_reaches(V, dtype):
    """x - m passes fp32's range where scale (x - m) does not."""
    from paper_2502_17728_amd import ops
    most = torch.finfo(dtype).max
    logits = torch.zeros((2, V), dtype=dtype, device="cuda")
    logits[:, 3], logits[0, 4], logits[1, V - 1] = most, -most, -0.75 * most
    targets = torch.tensor([[3, 4], [V - 1, 0]], dtype=torch.int32, device="cuda")
    for scale in (0.5, 0.25, 2.0 ** -40, 2.0 ** -96):
        got, ref = ops.token_logprobs(logits, targets, 6, scale), R.logprobs(logits, targets, 6, scale)
        # the difference, its product with the scale, ln l's sum and the result's rounding
        for name in ("logprobs", "top_logprobs"):
            fits = ref[name].abs() <= torch.finfo(F32).max
            assert fits.all()
            R.assert_within(got[name][fits], ref[name][fits], ref[name][fits].abs() * 4 * 2.0 ** -24)
    top = torch.sort(logits[:, :6].double() if V == 6 else logits.double(), dim=1, descending=True, stable=True)[1][:, :6]
    assert torch.equal(got["top_ids"].long(), top)


def test_scales_that_bring_such_logits_together_are_refused():
    # below 2^-96 a difference past fp32's range would count in the sums
    from paper_2502_17728_amd import ops
    far = [0x7F0000000000 + (i << 36) for i in range(2)]  # not touched: the entropy's address is misaligned, which is seen later
    call = lambda s: ops._lib.token_logprobs(far[0], 100, 4, 100, 0, s, None, 0, 0, None, far[1] + 1, None, None, None, 0, None)
    assert call(2.0 ** -97) == 2 and call(1e-40) == 2 and call(2.0 ** -96) == 3 and call(1.0) == 3
