"""Token log probabilities, entropy and the likeliest tokens against a plain 64-bit form."""
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


def make(T, V, dtype, seed, row=None, offset=0, spread=3.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    row = row or V
    flat = torch.randn(T * row + offset, generator=g, device="cuda").mul_(spread).to(dtype)
    targets = torch.randint(0, V, (T, 3), generator=g, device="cuda", dtype=torch.int32)
    return flat[offset:].view(T, row)[:, :V], targets


def check(ops, logits, targets, top, scale=1.0, **kw):
    got = ops.token_logprobs(logits, targets, top, scale, **kw)
    ref = R.logprobs(logits, targets, top, scale)
    # ln p = d - ln l, d = scale (x - m).  d is 2 roundings off; an exponent to base 2 takes a third and is then
    # off by 3 2^-24 of itself, at most 40 where its power counts in a sum (2^-40 V is past fp32 else): l and ln l
    # are off by 3 * 40 * 2^-24 * ln 2, the powers' and logarithm's own 2 steps, and a chain of sums: a lane's
    # share of at most V / 64 values (64 threads to a row) and rescalings, 6 + 2 + 6 joins.
    V = logits.shape[1]
    l = (3 * 40 * 0.7 + 4 + (V / 64 + 80)) * 2.0 ** -24
    for name in ("logprobs", "top_logprobs"):
        if ref[name] is None:
            assert got[name] is None
        else:
            R.assert_within(got[name], ref[name], ref[name].abs() * 4 * 2.0 ** -24 + l)
    # the entropy's terms p d are off by the same shares of p |d|, whose sum is at most entropy + ln V
    if kw.get("entropy", True):
        fine = torch.isfinite(ref["entropy"])
        R.assert_within(got["entropy"], ref["entropy"], torch.where(fine, 2 * l * (1 + ref["entropy"] + math.log(V)), 0.0))
    if top:
        ok = ~torch.isnan(ref["entropy"]) | ~torch.isnan(logits.float()).any(1)
        assert torch.equal(got["top_ids"][ok].long(), ref["top_ids"][ok])
    return got


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,V", [(1, 1), (3, 5), (2, 8), (5, 63), (2, 64), (4, 65), (1, 1000), (2, 2049), (1, 8192), (3, 8200),
                                 (700, 1003), (1, 100003), (33, 50001), (2, 131072), (1100, 9000)])
def test_sizes(ops, T, V, dtype):
    logits, targets = make(T, V, dtype, T + V)
    for top in (0, 1, 5, 20, 64):
        if top <= V:
            check(ops, logits, targets, top)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("offset", range(9))
def test_rows_that_start_at_any_element(ops, dtype, offset):
    for V, row in ((37, 41), (4099, 4101), (9001, 9003)):
        logits, targets = make(5, V, dtype, offset, row, offset)
        check(ops, logits, targets, 7)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,V", [(600, 3000), (600, 20003), (2100, 11), (2100, 1023), (2003, 5001), (2001, 8200), (4003, 257),
                                 (4003, 4500)])
def test_many_rows(ops, T, V, dtype):
    for top in (0, 1, 20, 64):
        logits, targets = make(T, V, dtype, T + V + top)
        check(ops, logits, targets, min(top, V))


def test_what_lies_around_the_rows_is_not_read(ops):
    # NaN and large values before, between and after the rows
    for dtype in (BF16, F32):
        for V, row, offset in ((5, 8, 3), (8191, 8200, 5), (20001, 20011, 1)):
            flat = torch.full((4 * row + 16,), math.nan, dtype=dtype, device="cuda")
            flat[::2] = 1e30
            logits = flat[offset:offset + 4 * row].view(4, row)[:, :V]
            clean, targets = make(4, V, dtype, V)
            logits.copy_(clean)
            a, b = check(ops, logits, targets, 5), check(ops, clean, targets, 5)
            assert torch.equal(a["top_ids"], b["top_ids"])


@pytest.mark.parametrize("scale", [0.25, 1.0, 1.7, 30.0])
def test_scales(ops, scale):
    for V in (500, 40000):
        logits, targets = make(6, V, F32, 3)
        check(ops, logits, targets, 9, scale)


@pytest.mark.parametrize("V", [64, 1000, 70001])
@pytest.mark.parametrize("kind", ["equal", "rising", "falling", "two", "zeros"])
def test_ties_and_orders(ops, V, kind):
    x = torch.arange(V, device="cuda", dtype=torch.float32)
    row = {"equal": torch.ones_like(x), "rising": x / V, "falling": -x / V, "two": (x % 2), "zeros": x * -0.0}[kind]
    if kind == "zeros":
        row[::3] = 0.0  # +0 and -0 are equal
    targets = torch.zeros((2, 1), dtype=torch.int32, device="cuda")
    for dtype in (F32, BF16):
        check(ops, torch.stack([row, row.flip(0)]).to(dtype).contiguous(), targets, 64)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V", [40, 3000, 90000])
def test_masks(ops, V, dtype):
    logits, targets = make(9, V, dtype, 11)
    logits = logits.clone()
    logits[0, : V // 2] = -math.inf
    logits[1] = -math.inf
    logits[2, 1:] = -math.inf                        # one token left: p = 1, entropy 0
    logits[3] = torch.finfo(dtype).min               # the type's lowest value everywhere: even odds
    logits[4, ::2] = torch.finfo(dtype).min
    logits[5, V // 3] = math.inf
    logits[6, V - 1] = math.nan
    logits[7] = torch.finfo(dtype).max
    logits[8, 0] = torch.finfo(dtype).max
    logits[8, 1] = torch.finfo(dtype).min
    targets[2, 0] = 0
    got = check(ops, logits, targets, 20)
    assert got["entropy"][2] == 0 and got["logprobs"][2, 0] == 0
    assert torch.isnan(got["logprobs"][1]).all() and torch.isnan(got["logprobs"][5]).all() and torch.isnan(got["entropy"][6])
    # NaN logits have no rank
    assert V - 1 not in got["top_ids"][6].tolist()
    logits[6] = math.nan
    logits[6, 3] = 1.0
    assert ops.token_logprobs(logits, None, 4)["top_ids"][6].tolist() == [3, -1, -1, -1]


def test_targets_outside(ops):
    for V in (100, 30000):
        logits, targets = make(4, V, BF16, 12)
        targets[0, 0], targets[1, 1], targets[2, 2], targets[3, 0] = -1, V, 2 ** 31 - 1, -(2 ** 31)
        got = check(ops, logits, targets, 0)
        assert got["logprobs"][0, 0] == 0 and got["logprobs"][3, 0] == 0
        logits = logits.clone()
        logits[0] = math.nan
        assert ops.token_logprobs(logits, targets)["logprobs"][0, 0] == 0  # padding drops out of a sum


def test_what_is_asked_for(ops):
    logits, targets = make(3, 2000, BF16, 13)
    got = ops.token_logprobs(logits)
    assert got["logprobs"] is None and got["top_ids"] is None and got["entropy"].shape == (3,)
    got = ops.token_logprobs(logits, targets, entropy=False)
    assert got["entropy"] is None and got["logprobs"].shape == (3, 3)
    check(ops, logits, targets[:, :0], 2)
    with pytest.raises(ops.DNError):
        ops.token_logprobs(logits, entropy=False)


def test_runs_agree_bit_for_bit(ops):
    for T, V in ((1, 131072), (40, 33333)):
        logits, targets = make(T, V, BF16, 14)
        a = ops.token_logprobs(logits, targets, 20)
        for _ in range(3):
            b = ops.token_logprobs(logits, targets, 20)
            assert all(torch.equal(a[k], b[k]) for k in a)


def test_refusals(ops):
    logits, targets = make(3, 100, BF16, 15)
    for bad in (logits.cpu(), logits[0], logits.half(), logits.t()):
        with pytest.raises((ValueError, TypeError)):
            ops.token_logprobs(bad, None, 1)
    for bad in (targets.long(), targets[:2], targets[:, 0], targets.cpu()):
        with pytest.raises(ValueError):
            ops.token_logprobs(logits, bad)
    for kw in (dict(top=101), dict(top=65), dict(scale=0.0), dict(scale=math.nan), dict(scale=math.inf), dict(top=-1, entropy=False)):
        with pytest.raises(ops.DNError):
            ops.token_logprobs(logits, None, **kw)
    with pytest.raises(ops.DNError):  # rows that lie on one another
        ops.token_logprobs(logits[:1].expand(3, 100))
    big, _ = make(1, 131072, BF16, 16)
    n = ops.token_logprobs_workspace_bytes(1, 131072, 5)
    assert n > 0 and ops.token_logprobs_workspace_bytes(1, 100, 101) == 0
    with pytest.raises(ops.DNError):
        ops.token_logprobs(big, None, 5, workspace=torch.empty(n - 1, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        ops.token_logprobs(big, None, 5, workspace=torch.empty(n, device="cuda"))
