"""The deal of 256-row tiles in equal runs, on the host with the code that the device runs: every tile is
written whole by one run, or by the merge from pieces that hold each of its pages once."""
import ctypes
import functools
import os
import random
import subprocess
import tempfile

import pytest

from paper_2502_17728_amd import build as B
from test_cache_rules import plan

SHIM = r"""
#include "kv_layout.hpp"
using namespace dn;
// pieces: 6 numbers each, by place; tiles: first piece and pieces of each; runs: likewise.  The number of tiles.
extern "C" int64_t deal(int64_t B, const int* n, const int* len, int heads, int group, int rows, int64_t target, int64_t least,
                        int64_t tiles_most, int* pieces, int* tile_lists, int* run_lists) {
    auto sequence = [&](int64_t b) { return Seq{0, n[b], len[b], (len[b] + kKvPage - 1) / kKvPage}; };
    int64_t total = 0, tiles = 0;
    for (int64_t b = 0; b < B; ++b) {
        const Seq s = sequence(b);
        total += weights(s, group, rows).before(tiles_of(s, group, rows)) * heads;
        tiles += (int64_t)tiles_of(s, group, rows) * heads;
    }
    const Line line{B, heads, target, total, run_length(total, target, least, group), group, rows, tiles_most};
    for (int64_t run = 0; run < target; ++run) {
        int64_t at = -1, start = 0, before = 0, x = 0, t = 0;
        for (int64_t b = 0; b < B; ++b) {  // the first sequence that ends past the run's start
            const Seq s = sequence(b);
            const int64_t sum = weights(s, group, rows).before(tiles_of(s, group, rows)) * heads;
            if (at < 0 && x + sum > run * line.per) at = b, start = x, before = t;
            x += sum;
            t += (int64_t)tiles_of(s, group, rows) * heads;
        }
        deal_run(
            line, run, at, start, before, sequence,
            [&](int64_t i, const Piece& p) {
                const int v[6] = {p.b, p.head, p.tile, p.lo, p.hi, p.slot};
                std::copy(v, v + 6, pieces + 6 * i);
            },
            [&](int64_t i, int first, int count) {
                tile_lists[2 * i] = first;
                tile_lists[2 * i + 1] = count;
            },
            run_lists[2 * run], run_lists[2 * run + 1]);
    }
    return tiles;
}
extern "C" int64_t divide(int64_t a, int64_t b) { return quotient(a, b); }
"""
WHOLE, NONE = -1, -2
UNWRITTEN = -9


@functools.lru_cache(None)
def deal():
    with tempfile.TemporaryDirectory() as d:
        src, lib = os.path.join(d, "shim.cpp"), os.path.join(d, "shim.so")
        open(src, "w").write(SHIM)
        subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-fPIC", "-shared", "-I", B.CSRC, src, "-o", lib])
        lib = ctypes.CDLL(lib)
    i64, i32, p = ctypes.c_int64, ctypes.c_int, ctypes.POINTER(ctypes.c_int)
    lib.deal.argtypes, lib.deal.restype = [i64, p, p, i32, i32, i32, i64, i64, i64, p, p, p], i64
    lib.divide.argtypes, lib.divide.restype = [i64, i64], i64
    return lib


def check(seqs, heads, group):
    """The lists of a batch of (new tokens, cached tokens); False where the launch rule deals it otherwise."""
    T = sum(n for n, _ in seqs)
    width = max(8, max(-(-k // 64) for _, k in seqs))  # a table may be wider than its sequences need
    own, _, _ = plan(T, len(seqs), heads, group, 128, width)
    if not own["in_runs"]:
        return False
    target, most = own["target"], own["tiles"]
    ints = lambda v: (ctypes.c_int * len(v))(*v)
    pieces, tiles, runs = ints([UNWRITTEN] * 6 * (target + most)), ints([UNWRITTEN] * 2 * most), ints([0] * 2 * target)
    count = deal().deal(len(seqs), ints([n for n, _ in seqs]), ints([k for _, k in seqs]), heads, group, 256, target,
                        own["least"], most, pieces, tiles, runs)
    assert count <= most
    # what each run works through, and what it leaves
    done, held, slots = {}, {}, set()
    for run in range(target):
        for at in range(runs[2 * run], runs[2 * run] + runs[2 * run + 1]):
            b, head, tile, lo, hi, slot = pieces[6 * at:6 * at + 6]
            assert b >= 0, "a piece that no run listed"
            if slot == WHOLE:
                done[b, head, tile] = done.get((b, head, tile), 0) + 1
            elif slot != NONE:
                assert 0 <= slot < own["slots"] and slot not in slots and lo < hi
                slots.add(slot)
            held.setdefault((b, head, tile), []).append((lo, hi, slot))
    ordinal = 0
    for b, (n, k) in enumerate(seqs):
        for head in range(heads):
            for tile in range(-(-n * group // 256)):
                first, parts = tiles[2 * ordinal:2 * ordinal + 2]
                ordinal += 1
                keys = max(0, min(k, k - n + min(n, (tile * 256 + 255) // group + 1)))
                pages = -(-keys // 64)
                if parts == 0:
                    assert done.get((b, head, tile)) == 1, (seqs, heads, group, (b, head, tile))
                    assert [(lo, hi) for lo, hi, slot in held[b, head, tile] if slot == WHOLE] == [(0, pages)]
                    continue
                assert (b, head, tile) not in done
                at = 0
                for i in range(first, first + parts):
                    where, lo, hi, slot = tuple(pieces[6 * i:6 * i + 3]), *pieces[6 * i + 3:6 * i + 6]
                    assert where == (b, head, tile) and lo == at
                    assert (slot == NONE) == (lo == hi)
                    at = hi
                assert at == pages
    assert ordinal == count
    return True


@pytest.mark.parametrize("seqs,heads,group", [([(2048, 300)], 1, 4), ([(1057, 217)], 4, 5), ([(4096, 500), (4096, 4096)], 8, 4),
                                              ([(4096, 1)], 2, 1), ([(4096, 0)], 1, 8), ([(3000, 2999)], 1, 1),
                                              ([(1, 8192)] * 31 + [(2048, 8192)], 8, 4), ([(2000, 100000)], 8, 4)])
def test_named_batches(seqs, heads, group):
    assert check(seqs, heads, group)


@pytest.mark.parametrize("seed", range(40))
def test_random_batches(seed):
    """Sequences with all of their keys before the new tokens, some of them, or far fewer keys than new tokens."""
    rng = random.Random(seed)
    log = lambda a, b: int(round(a * (b / a) ** rng.random()))
    dealt = 0
    for _ in range(40):
        heads, group = rng.choice((1, 2, 4, 8)), rng.choice((1, 3, 4, 5, 16))
        seqs = []
        for _ in range(log(1, 12)):
            n = rng.choice((0, 1, log(1, 5000), log(300, 5000)))
            kind = rng.random()
            seqs.append((n, log(1, max(1, n)) if kind < 0.5 else n + log(1, 20000) if kind < 0.9 else 0))
        if sum(n for n, _ in seqs):
            dealt += check(seqs, heads, group)
    assert dealt >= 5


def test_quotients():
    rng = random.Random(1)
    for _ in range(20000):
        b = rng.randrange(1, 1 << rng.randrange(1, 41))
        a = rng.choice((rng.randrange(1 << 61), b * rng.randrange(1 << 20), b * rng.randrange(1, 1 << 20) - 1))
        if a // b < 1 << 52:
            assert deal().divide(a, b) == a // b


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,d", [("bf16", 64), ("fp8", 128)])
@pytest.mark.parametrize("seqs,Hq,Hkv", [([(2048, 300)], 4, 1), ([(1057, 217)], 20, 4), ([(900, 100), (1, 5000), (700, 290)], 8, 2),
                                         ([(1, 4000), (600, 4000), (1, 1), (1, 64), (1, 0), (1, 129)], 8, 2)])
def test_tiles_of_runs_on_the_device(seqs, Hq, Hkv, fmt, d):
    """Queries before their first key (zeros), those behind them, and single new tokens beside chunks:
    every row is written, with what the plain form gives."""
    import torch
    from test_attention_cache import Batch
    b = Batch(seqs, Hq, Hkv, d, fmt)
    width = max(8, b.table.shape[1])
    b.table = torch.nn.functional.pad(b.table, (0, width - b.table.shape[1]), value=-7)
    assert plan(int(b.q_start[-1]), len(seqs), Hkv, Hq // Hkv, d, width)[0]["in_runs"]
    out = torch.full(b.Q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    first = b.run(out=out).clone()
    b.check(first)
    assert torch.equal(first, b.run(out=out.fill_(float("nan"))))


# ------------------------------------------------------------------------------- launches past what HIP takes
def test_launches_past_the_devices_limit_are_refused():
    """2^32 threads and more in one launch: refused before anything is launched, where the device would refuse it;
    the largest that fits is taken."""
    from paper_2502_17728_amd import ops
    wb = ops._lib.attention_cache_workspace_bytes
    # one new token of a million sequences, 16-row tiles of 256 threads: 2^20 heads + 2^16 heads + 768 of them
    assert wb(1 << 20, 1 << 20, 15, 15, 64, 8, 0) > 0 == wb(1 << 20, 1 << 20, 16, 16, 64, 8, 0)
    # behind a prefix both kinds of tile share the launch
    assert wb(986000, 986000, 17, 17, 64, 8, 0) > 0 == wb(986000, 986000, 17, 17, 64, 8, 6400)
    # the merge: 2^28 rows of d = 128, 8 threads each; behind a prefix 16
    assert wb(1 << 13, 1, 1 << 15, 1, 128, 64, 0) > 0
    assert wb(1 << 13, 1, 1 << 15, 1, 128, 64, 64) == 0 < wb(1 << 12, 1, 1 << 15, 1, 128, 64, 64)
    P = 0x7F0000000000
    UNSUPPORTED = 2
    far = lambda k: P + (k << 42)
    desc = ops.KVCacheDesc(64, 64, 64, 2, 1, P)
    big = 1 << 28
    assert ops._lib.kv_cache_append(ctypes.byref(desc), far(1), 128 * 64, far(2), None, None, 0, 0, 0, big, 0, 1, None, None) == UNSUPPORTED
    assert ops._lib.kv_cache_read(ctypes.byref(desc), far(1), big, 1, far(2), far(3), None) == UNSUPPORTED
    assert ops._lib.rotary_apply(far(1), 1 << 14, far(2), far(3), 4, 1 << 24, 256, 64, 64, 0, 0, 1, far(4), 1 << 14, None) == UNSUPPORTED
    assert ops._lib.rotary_table(far(1), 256, 1 << 26, 1.0, far(2), None) == UNSUPPORTED
