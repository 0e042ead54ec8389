"""Token log probabilities at the edges of their numbers: ranks beside NaNs of either kind (GPU)."""
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
