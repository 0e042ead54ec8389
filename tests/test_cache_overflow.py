"""Turned keys at the end of bfloat16's range (GPU)."""
import pytest
import torch

import kv_reference as R
from paper_2502_17728_amd import ops

pytestmark = pytest.mark.gpu
MOST = 3.3895313892515355e38  # (2 - 2^-7) 2^127, the largest bfloat16; half a step on, x (1 + 2^-8 / (2 - 2^-7)), rounds to infinity


@pytest.mark.parametrize("amplitude,fits", [(1.0, True), (1.0019, True), (1.0021, False), (1.003, False), (1.01, False)])
@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128])
def test_turned_keys_past_the_largest_bf16(d, fmt, amplitude, fits):
    """A bf16 row whose turned value rounds to an infinity is held as NaN; e4m3 holds whatever fp32 does, and
    the rows beside it are as they are."""
    heads, rot = 2, 16
    rows = torch.randn((3, 4 * heads, d), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    k = rows[:, 2 * heads:3 * heads]
    k[1, 0, 3] = -MOST
    cache = ops.kv_cache_create(1, heads, d, fmt)
    table = ops.rotary_table(ops.rotary_frequencies(rot)[0], 4, amplitude)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    ops.kv_cache_append(cache, rows.cuda().view(3, -1), ints([5, 6, 7]), ints([0, 0, 0]), table)
    K, V, ks, vs = R.held(cache.data, d, fmt)
    held = fits if fmt == "bf16" else amplitude < 1.0039  # fp32's largest is 1.0039 times bf16's
    bad = torch.zeros(heads, 3, dtype=torch.bool)
    bad[0, 1] = not held
    assert torch.equal(ks[0, :, 5:8].isnan(), bad) and not vs[0, :, 5:8].isnan().any()
    codes = K[0, :, 5:8]
    assert codes.isfinite().all() and bool((codes[bad] == 0).all()) and bool((codes[~bad].abs().amax(-1) > 0).all())
