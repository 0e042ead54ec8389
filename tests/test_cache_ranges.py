"""The paged cache and attention over it at the ends of their ranges: many ragged sequences in every
tile size, work cut many times, caches past 4 GiB, and what the binding refuses (GPU)."""
import pytest
import torch

from paper_2502_17728_amd import ops
from test_attention_cache import KINDS, Batch, ints
from test_cache_rules import plan

pytestmark = pytest.mark.gpu


def ragged(count, most_new, most_keys):
    """Sequences with and without new tokens, some with fewer keys than new tokens."""
    return [((7 * i * i + 3 * i) % (most_new + 1), (31 * i + i * i) % (most_keys + 1)) for i in range(1, count + 1)]


@pytest.mark.parametrize("fmt,d", KINDS)
@pytest.mark.parametrize("rows,group,new", [(16, 4, 6), (64, 8, 14), (128, 16, 20), (256, 16, 40)])
def test_many_ragged_sequences(rows, group, new, fmt, d):
    seqs = ragged(130, new, 200)
    b = Batch(seqs, group, 1, d, fmt)
    assert plan(int(b.q_start[-1]), len(seqs), 1, group, d, b.table.shape[1])[0]["rows"] == rows
    b.check(b.run())


@pytest.mark.parametrize("fmt,d", KINDS)
@pytest.mark.parametrize("seqs", [[(300, 6000), (0, 40), (257, 257), (90, 2000)], [(700, 700)], [(200, 130), (150, 4100)]])
def test_wide_tiles_in_runs(seqs, fmt, d):
    b = Batch(seqs, 8, 2, d, fmt)
    own, _, _ = plan(int(b.q_start[-1]), len(seqs), 2, 4, d, b.table.shape[1])
    assert own["rows"] == 256 and own["in_runs"]
    first = b.run()
    b.check(first)
    assert torch.equal(first.view(torch.int16), b.run().view(torch.int16))  # no order is left to chance


@pytest.mark.parametrize("fmt,d", KINDS)
@pytest.mark.parametrize("seqs,prefix,own_rows,rows", [([(1, 30)] * 10, 5000, 16, 64), ([(1, 70), (0, 9), (2, 2)] * 9, 2500, 16, 128),
                                                       ([(1, 64)] * 80, 1300, 16, 128), ([(16, 70)] * 3, 700, 64, 128),
                                                       ([(40, 50)] * 5, 700, 128, 256), ([(100, 200), (70, 65)], 700, 256, 256)])
def test_shared_prefix_tiles(seqs, prefix, own_rows, rows, fmt, d):
    b = Batch(seqs, 8, 2, d, fmt, prefix=prefix)
    own, shared, _ = plan(int(b.q_start[-1]), len(seqs), 2, 4, d, b.table.shape[1], -(-prefix // 64))
    assert (own["rows"], shared["rows"]) == (own_rows, rows)
    first = b.run()
    b.check(first)
    assert torch.equal(first.view(torch.int16), b.run().view(torch.int16))


@pytest.mark.parametrize("n", [1, 20, 40, 100])
def test_rows_of_no_sequence_are_left_alone(n):
    """q_start may end before T: padding, which is neither read nor written."""
    b = Batch([(n, 900), (n, 70)], 4, 1, 64, "fp8")
    Q = torch.cat([b.Q, torch.full((9, 4, 64), float("nan"), dtype=torch.bfloat16)]).cuda()
    out = torch.full_like(Q, 7.0)
    b.run(Q=Q, out=out)
    b.check(out[:2 * n])
    assert (out[2 * n:] == 7.0).all()


@pytest.mark.parametrize("fmt,pages", [("fp8", 40000), ("bf16", 20500)])
def test_cache_past_32_bit_offsets(fmt, pages):
    """The same tokens in the last pages of a cache over 5 GB and in a small one: the same bits."""
    heads, d, n = 8, 128, 150
    big = ops.kv_cache_create(pages, heads, d, fmt)
    assert big.data.numel() > 5 << 30
    small = ops.kv_cache_create(3, heads, d, fmt)
    g = torch.Generator().manual_seed(5)
    qkv = torch.randn((n, (16 + 2 * heads) * d), generator=g).to(torch.bfloat16).cuda()
    at = [pages - 1, pages - 7, pages // 2 + 3]
    slots = [at[t // 64] * 64 + t % 64 for t in range(n)]
    q = ops.kv_cache_append(big, qkv, ints(slots))
    assert torch.equal(q, ops.kv_cache_append(small, qkv, ints(range(n))))
    for x, y in zip(ops.kv_cache_read(big, ints(slots)), ops.kv_cache_read(small, ints(range(n)))):
        assert torch.equal(x, y)
    for new in (1, 20, 70, 150):
        args = (ints([0, new]), ints([n]))
        x = ops.attention_cache_deferred(q[:new], big, ints([at]), *args)
        assert torch.equal(x, ops.attention_cache_deferred(q[:new], small, ints([[0, 1, 2]]), *args))
        assert x.isfinite().all()


def test_strided_queries_out_of_qkv_rows():
    """Queries taken straight from QKV rows (their stride is the rows'), in every tile size."""
    for n in (1, 9, 30, 90):
        b = Batch([(n, 100), (n, 300)], 8, 2, 64, "bf16")
        rows = torch.randn((2 * n, 12 * 64)).to(torch.bfloat16).cuda()
        rows[:, :512] = b.Q.cuda().view(2 * n, 512)
        b.check(b.run(Q=rows[:, :512].view(2 * n, 8, 64)))


def test_refusals_on_the_device():
    c = ops.kv_cache_create(4, 2, 64, "fp8")
    f, amplitude = ops.rotary_frequencies(64)
    table = ops.rotary_table(f, 16, amplitude)
    x, i = torch.zeros((4, 2, 64), device="cuda"), ints([0, 1, 2, 3])
    rows = torch.zeros((4, 8 * 64), dtype=torch.bfloat16, device="cuda")
    Q = torch.zeros((4, 4, 64), dtype=torch.bfloat16, device="cuda")
    bt, qs, kl = ints([[0, 1], [2, 3]]), ints([0, 2, 4]), ints([70, 70])
    few = torch.empty(16, dtype=torch.uint8, device="cuda")
    good = ops.attention_cache_deferred(Q, c, bt, qs, kl)
    calls = [lambda: ops.rotary_table(f.float(), 16), lambda: ops.rotary_table(f[:4], 16), lambda: ops.rotary_table(f, 0),
             lambda: ops.rotary_apply(x.double(), i, table), lambda: ops.rotary_apply(x, i.long(), table),
             lambda: ops.rotary_apply(x, i[:3], table), lambda: ops.rotary_apply(x, i, table.double()),
             lambda: ops.rotary_apply(x[:1].expand(4, 2, 64), i, table),           # tokens on one another
             lambda: ops.rotary_apply(x.transpose(1, 2), i, table),                # a head's values apart
             lambda: ops.rotary_apply(x[:, :, :48], i, table), lambda: ops.rotary_apply(x[:0], i[:0], table),
             lambda: ops.rotary_apply(x, i, table, out=x.bfloat16()), lambda: ops.rotary_apply(x, i, table, out=x[1:]),
             lambda: ops.kv_cache_append(c, rows.float(), i), lambda: ops.kv_cache_append(c, rows, i.long()),
             lambda: ops.rotary_apply(x, None, table), lambda: ops.rotary_apply(x, i, None),
             lambda: ops.kv_cache_append(c, rows, None), lambda: ops.kv_cache_append(c, rows, i[:2]), lambda: ops.kv_cache_append(c, rows, i, None, table),
             lambda: ops.kv_cache_append(c, rows[:1].expand(4, 512), i),
             lambda: ops.kv_cache_append(c, rows, i, q_out=Q.float()),
             lambda: ops.kv_cache_append(c, rows[:, :256].contiguous(), i, q_out=Q),
             lambda: ops.kv_cache_append(c, rows, i, q_out=rows[:, :256].view(4, 4, 64)),
             lambda: ops.kv_cache_read(c, i.long()), lambda: ops.kv_cache_read(c, i, K=torch.zeros(4, 2, 64, device="cuda")),
             lambda: ops.kv_cache_read(c, i.cpu()),
             lambda: ops.attention_cache_deferred(Q.float(), c, bt, qs, kl),
             lambda: ops.attention_cache_deferred(Q, c, bt.long(), qs, kl),
             lambda: ops.attention_cache_deferred(Q, c, bt, qs[:2], kl), lambda: ops.attention_cache_deferred(Q, c, bt, qs, kl[:1]),
             lambda: ops.attention_cache_deferred(Q, c, bt.t(), qs, kl), lambda: ops.attention_cache_deferred(Q, c, bt.cpu(), qs, kl),
             lambda: ops.attention_cache_deferred(Q, c, bt, qs, kl, scale=0.0),
             lambda: ops.attention_cache_deferred(Q, c, bt, qs, kl, out=Q),
             lambda: ops.attention_cache_deferred(Q, c, bt, qs, kl, out=good[:2]),
             lambda: ops.attention_cache_deferred(Q, c, bt, qs, kl, workspace=few),
             lambda: ops.attention_cache_deferred(Q[:1].expand(4, 4, 64), c, bt, qs, kl),
             lambda: ops.attention_shared_prefix_deferred(Q, c, ints([0]), 65, bt, qs, kl),
             lambda: ops.attention_shared_prefix_deferred(Q, c, ints([0]), 0, bt, qs, kl),
             lambda: ops.attention_shared_prefix_deferred(Q, c, ints([0]).long(), 10, bt, qs, kl)]
    for k, call in enumerate(calls):
        with pytest.raises((ValueError, TypeError, ops.DNError)):
            call()
            print("not refused:", k)  # shown if the call goes through
