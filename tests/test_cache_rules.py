"""Rotary positions, the paged cache and attention over it, on the host: every refusal of the C entry
points and of the binding, the block layout, and the rules that pick kernels, chunks and scratch."""
import ctypes
import functools
import os
import random
import subprocess
import tempfile

import pytest
import torch

import kv_reference as R
from paper_2502_17728_amd import build as B
from paper_2502_17728_amd import ops

OK, INVALID, UNSUPPORTED, MISALIGNED = 0, 1, 2, 3
P = 0x7F0000000000  # aligned addresses of nothing: validation never reads them
P2, P3, P4, P5, P6, P7 = (P + (k << 36) for k in range(1, 7))
FAR = P + (1 << 43)
NAN, INF = float("nan"), float("inf")

SHIM = r"""
#include "kv_layout.hpp"
using namespace dn;
extern "C" {
int at(int fmt, int d, int o, int x, int is_v) {
#define CASE(F, D) if (fmt == F && d == D) return is_v ? KvBlock<F, D>::PART + KvBlock<F, D>::v_at(o, x) : KvBlock<F, D>::k_at(o, x)
    CASE(1, 64); CASE(1, 128); CASE(2, 64); CASE(2, 128);
    return -1;
}
int rows(int64_t T, int64_t B, int64_t group) { return cache_rows(T, B, group); }
int append(int64_t tokens, int64_t heads, int64_t group, int64_t d) { return append_tile(tokens, heads, group, d); }
// rows, in_runs, target, least, tiles, grid, slots of the sequences' own keys and of the prefix, total bytes
void plan(int64_t T, int64_t B, int64_t heads, int64_t group, int64_t d, int64_t width, int64_t prefix_pages, int64_t* out) {
    const CacheWorkspace w = cache_workspace(T, B, heads, group, d, width, prefix_pages);
    for (const CachePlan* p : {&w.own, &w.prefix}) {
        const int64_t v[7] = {p->rows, p->in_runs, p->target, p->least, p->tiles, p->grid, p->slots};
        out = std::copy(v, v + 7, out);
    }
    *out = (int64_t)w.total;
}
}
"""


@functools.lru_cache(None)
def rules():
    with tempfile.TemporaryDirectory() as d:
        src, lib = os.path.join(d, "shim.cpp"), os.path.join(d, "shim.so")
        open(src, "w").write(SHIM)
        subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-fPIC", "-shared", "-I", B.CSRC, src, "-o", lib])
        lib = ctypes.CDLL(lib)
    i64, i32 = ctypes.c_int64, ctypes.c_int
    lib.at.argtypes = [i32] * 5
    lib.rows.argtypes = [i64] * 3
    lib.append.argtypes = [i64] * 4
    lib.plan.argtypes = [i64] * 7 + [ctypes.POINTER(i64)]
    return lib


def plan(T, seqs, heads, group, d=128, width=8, prefix_pages=0):
    out = (ctypes.c_int64 * 15)()
    rules().plan(T, seqs, heads, group, d, width, prefix_pages, out)
    names = ("rows", "in_runs", "target", "least", "tiles", "grid", "slots")
    return dict(zip(names, out[:7])), dict(zip(names, out[7:14])), out[14]


# ------------------------------------------------------------------------------- refusals of the library
def refuse(f, good, cases):
    """Each case changes some arguments of a call whose every argument is right."""
    names = list(good)
    for want, change in cases:
        args = dict(good, **change)
        assert list(args) == names, change
        got = f(*[ctypes.byref(v) if isinstance(v, ctypes.Structure) else v for v in args.values()])
        assert got == want, (change, got)


def cache(pages=64, heads=2, d=64, format=2, version=1, data=P):
    return ops.KVCacheDesc(pages, heads, d, format, version, data)


BAD_CACHES = [(INVALID, dict(cache=None)), (INVALID, dict(cache=cache(data=None))), (INVALID, dict(cache=cache(version=0))),
              (INVALID, dict(cache=cache(pages=0))), (INVALID, dict(cache=cache(heads=0))), (INVALID, dict(cache=cache(d=96))),
              (INVALID, dict(cache=cache(format=3))), (MISALIGNED, dict(cache=cache(data=P + 128)))]


def test_rotary_table_refusals():
    good = dict(inv=P, rot=64, positions=100, amplitude=1.0, table=P2, stream=None)
    refuse(ops._lib.rotary_table, good, [
        (INVALID, dict(inv=None)), (INVALID, dict(table=None)), (INVALID, dict(rot=0)), (INVALID, dict(positions=0)),
        (INVALID, dict(positions=-5)), (INVALID, dict(amplitude=NAN)), (INVALID, dict(amplitude=INF)),
        (INVALID, dict(table=P)), (INVALID, dict(positions=1 << 62)),
        (UNSUPPORTED, dict(rot=24)), (UNSUPPORTED, dict(positions=1 << 32)),
        (MISALIGNED, dict(inv=P + 4)), (MISALIGNED, dict(table=P2 + 8))])


def test_rotary_apply_refusals():
    good = dict(x=P, x_stride=256, positions=P2, table=P3, table_rows=100, T=10, H=4, d=64, rot=32, interleaved=0,
                inverse=0, dtype=1, out=P4, out_stride=256, stream=None)
    refuse(ops._lib.rotary_apply, good, [
        *[(INVALID, {k: None}) for k in ("x", "positions", "table", "out")],
        *[(INVALID, {k: 0}) for k in ("table_rows", "T", "H", "d", "rot", "x_stride", "out_stride")],
        (INVALID, dict(rot=80)), (INVALID, dict(interleaved=2)), (INVALID, dict(inverse=-1)), (INVALID, dict(dtype=2)),
        (INVALID, dict(x_stride=255)), (INVALID, dict(out_stride=248)), (INVALID, dict(x_stride=1 << 62)),
        (INVALID, dict(out=P + 16)), (INVALID, dict(x_stride=512, out=P)),      # in place only with one stride
        (INVALID, dict(out=P3 + 64)), (INVALID, dict(out=P2)),                  # out over the table, the positions
        (UNSUPPORTED, dict(rot=24)), (UNSUPPORTED, dict(d=72, x_stride=288, out_stride=288)),
        (UNSUPPORTED, dict(x_stride=260)), (UNSUPPORTED, dict(out_stride=257)),
        (UNSUPPORTED, dict(T=1 << 32, out=FAR)),
        (MISALIGNED, dict(x=P + 8)), (MISALIGNED, dict(out=P4 + 2)), (MISALIGNED, dict(table=P3 + 4)),
        (MISALIGNED, dict(positions=P2 + 2))])


def test_cache_sizes_and_description():
    nb = ops._lib.kv_cache_bytes
    assert nb(3, 2, 128, 1) == 3 * 2 * (2 * 64 * 128 * 2 + 512) and nb(3, 2, 64, 2) == 3 * 2 * (2 * 64 * 64 + 512)
    assert [nb(*a) for a in ((0, 2, 64, 1), (2, 0, 64, 1), (2, 2, 96, 1), (2, 2, 64, 0), (1 << 26, 1, 64, 1),
                             (1 << 24, 1 << 30, 128, 1))] == [0] * 6
    desc = ops.KVCacheDesc()
    good = dict(data=P, bytes=nb(4, 2, 64, 2), pages=4, heads=2, d=64, format=2, out=desc)
    refuse(ops._lib.kv_cache_describe, good, [
        (INVALID, dict(data=None)), (INVALID, dict(out=None)), (INVALID, dict(bytes=nb(4, 2, 64, 2) - 1)),
        (INVALID, dict(pages=0)), (INVALID, dict(heads=-1)), (INVALID, dict(d=0)), (INVALID, dict(format=0)),
        (UNSUPPORTED, dict(d=96)), (UNSUPPORTED, dict(pages=1 << 25)), (MISALIGNED, dict(data=P + 64))])
    assert desc.layout_version == 0 and not desc.data  # untouched by a refusal
    refuse(ops._lib.kv_cache_describe, good, [(OK, {})])
    assert (desc.pages, desc.heads, desc.d, desc.format, desc.layout_version, desc.data) == (4, 2, 64, 2, 1, P)


def test_append_refusals():
    good = dict(cache=cache(), qkv=P2, stride=512, slots=P3, positions=P4, table=P5, table_rows=100, rot=32,
                interleaved=0, T=10, q_heads=4, dtype=1, q_out=P6, stream=None)
    refuse(ops._lib.kv_cache_append, good, BAD_CACHES + [
        *[(INVALID, {k: None}) for k in ("qkv", "slots", "positions", "table", "q_out")],
        (INVALID, dict(T=0)), (INVALID, dict(table_rows=0)), (INVALID, dict(rot=-16)), (INVALID, dict(rot=80)),
        (INVALID, dict(interleaved=2)), (INVALID, dict(q_heads=3)), (INVALID, dict(q_heads=-2)),
        (INVALID, dict(q_heads=0)), (INVALID, dict(stride=504)), (INVALID, dict(dtype=7)),
        (INVALID, dict(qkv=P + 4096)), (INVALID, dict(slots=P + 4096)), (INVALID, dict(positions=P)),
        (INVALID, dict(table=P)), (INVALID, dict(q_out=P)), (INVALID, dict(q_out=P2 + 1024)), (INVALID, dict(q_out=P3)),
        (UNSUPPORTED, dict(dtype=0)), (UNSUPPORTED, dict(rot=24)), (UNSUPPORTED, dict(stride=516)),
        (UNSUPPORTED, dict(T=1 << 30, qkv=P7, q_out=FAR)),
        (MISALIGNED, dict(qkv=P2 + 8)), (MISALIGNED, dict(q_out=P6 + 8)), (MISALIGNED, dict(slots=P3 + 2)),
        (MISALIGNED, dict(table=P5 + 8)), (MISALIGNED, dict(positions=P4 + 1))])


def test_read_refusals():
    good = dict(cache=cache(), slots=P2, T=10, dtype=1, K=P3, V=P4, stream=None)
    refuse(ops._lib.kv_cache_read, good, BAD_CACHES + [
        *[(INVALID, {k: None}) for k in ("slots", "K", "V")], (INVALID, dict(T=0)), (INVALID, dict(dtype=9)),
        (INVALID, dict(K=P4 + 256)), (INVALID, dict(K=P)), (INVALID, dict(V=P + 512)), (INVALID, dict(V=P2)),
        (UNSUPPORTED, dict(dtype=0)), (UNSUPPORTED, dict(T=1 << 30, K=P6, V=FAR)),
        (MISALIGNED, dict(K=P3 + 8)), (MISALIGNED, dict(V=P4 + 4)), (MISALIGNED, dict(slots=P2 + 2))])


@pytest.mark.parametrize("shared", [False, True])
def test_attention_refusals(shared):
    wb = ops._lib.attention_cache_workspace_bytes
    prefix = dict(prefix_table=P7, prefix=100) if shared else {}
    need = wb(10, 3, 4, 2, 64, 8, 100 if shared else 0)
    good = dict(Q=P2, q_stride=256, T=10, q_heads=4, cache=cache(), **prefix, table=P3, width=8, q_start=P4, kv_len=P4 + 4096,
                B=3, scale=0.125, dtype=1, workspace=P5, bytes=need, out=P6, stream=None)
    cases = BAD_CACHES + [
        *[(INVALID, {k: None}) for k in ("Q", "table", "q_start", "kv_len", "workspace", "out")],
        *[(INVALID, {k: 0}) for k in ("T", "B", "width", "q_heads", "q_stride")],
        (INVALID, dict(q_heads=3)), (INVALID, dict(q_stride=248)), (INVALID, dict(bytes=need - 1)), (INVALID, dict(dtype=4)),
        *[(INVALID, dict(scale=v)) for v in (0.0, -1.0, NAN, INF)],
        *[(INVALID, dict(out=v)) for v in (P2 + 1024, P, P3, P4, P4 + 4096, P5)],
        *[(INVALID, dict(workspace=v)) for v in (P2 + 256, P, P3, P4)],
        (UNSUPPORTED, dict(dtype=0)), (UNSUPPORTED, dict(q_stride=260)), (UNSUPPORTED, dict(width=1 << 26)),
        (UNSUPPORTED, dict(B=1 << 21)), (UNSUPPORTED, dict(T=1 << 25)),
        (MISALIGNED, dict(Q=P2 + 8)), (MISALIGNED, dict(out=P6 + 8)), (MISALIGNED, dict(workspace=P5 + 128)),
        (MISALIGNED, dict(table=P3 + 2)), (MISALIGNED, dict(q_start=P4 + 1)), (MISALIGNED, dict(kv_len=P4 + 4097))]
    if shared:
        cases += [(INVALID, dict(prefix_table=None)), (INVALID, dict(prefix=0)), (INVALID, dict(prefix_table=P6)),
                  (MISALIGNED, dict(prefix_table=P7 + 2)), (UNSUPPORTED, dict(prefix=(1 << 31) - 1))]
    refuse(ops._lib.attention_shared_prefix_deferred if shared else ops._lib.attention_cache_deferred, good, cases)
    bad = [(0, 3, 4, 2, 64, 8, 0), (10, 0, 4, 2, 64, 8, 0), (10, 3, 3, 2, 64, 8, 0), (10, 3, 4, 2, 96, 8, 0),
           (10, 3, 4, 2, 64, 0, 0), (10, 3, 4, 2, 64, 8, -1), (1 << 25, 3, 4, 2, 64, 8, 0)]
    assert [wb(*a) for a in bad] == [0] * len(bad)
    assert wb(1 << 13, 1, 1 << 16, 1, 64, 1 << 24, 0) == 0 < wb(1 << 13, 1, 1 << 16, 1, 64, 1 << 10, 0)


# ------------------------------------------------------------------------------- refusals of the binding
def host_cache(heads=2, d=64):
    """A cache whose memory is the host's: enough for what is checked before any launch."""
    n = ops.kv_cache_bytes(2, heads, d, "fp8")
    return ops.KVCache(torch.zeros((2, heads, n // (2 * heads)), dtype=torch.uint8), cache(2, heads, d))


def test_binding_refusals():
    x, i, t = torch.zeros(4, 2, 64), torch.zeros(4, dtype=torch.int32), torch.zeros(8, 32, 2)
    rows = torch.zeros(4, 8 * 64, dtype=torch.bfloat16)
    c, table = host_cache(), torch.zeros(4, 2, dtype=torch.int32)
    Q = torch.zeros(4, 4, 64, dtype=torch.bfloat16)
    for f in (lambda: ops.rotary_apply(x[0], i, t), lambda: ops.rotary_apply(x, i, t),
              lambda: ops.rotary_table(torch.zeros(2, 2), 8), lambda: ops.rotary_table(torch.zeros(8), 8),
              lambda: ops.rotary_frequencies(0), lambda: ops.rotary_frequencies(17),
              lambda: ops.rotary_frequencies(64, scaling="other"), lambda: ops.rotary_frequencies(64, factor=0.0),
              lambda: ops.rotary_frequencies(64, scaling="parts", low=4.0, high=1.0),
              lambda: ops.kv_cache_wrap(torch.zeros(2, 2), 64), lambda: ops.kv_cache_wrap(torch.zeros(2, 2, 9), 64),
              lambda: ops.kv_cache_append(c, rows[0], i), lambda: ops.kv_cache_append(c, rows, i),
              lambda: ops.kv_cache_append(c, rows[:, :500], i), lambda: ops.kv_cache_append(c, rows[:, :128], i),
              lambda: ops.kv_cache_append(c, rows[:, :7 * 64], i), lambda: ops.kv_cache_read(c, table),
              lambda: ops.attention_cache_deferred(Q[0], c, table, i, i),
              lambda: ops.attention_cache_deferred(Q[:, :3], c, table, i, i),
              lambda: ops.attention_cache_deferred(Q[:, :, :32], c, table, i, i),
              lambda: ops.attention_cache_deferred(Q, c, i, i, i), lambda: ops.attention_cache_deferred(Q, c, table, i, i),
              lambda: ops.attention_shared_prefix_deferred(Q, c, i, 257, table, i, i),
              lambda: ops.attention_shared_prefix_deferred(Q, c, table, 64, table, i, i)):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: ops.kv_cache_append(None, rows, i), lambda: ops.kv_cache_read(c.desc, i),
              lambda: ops.attention_cache_deferred(Q, c.data, table, i, i)):
        with pytest.raises(TypeError):
            f()
    for a in ((0, 2, 64, "fp8"), (2, 2, 96, "bf16"), (2, 2, 64, "int4")):
        assert ops.kv_cache_bytes(*a) == 0
        with pytest.raises(ops.DNError):
            ops.kv_cache_create(*a, device="cpu")


# ------------------------------------------------------------------------------- layout
@pytest.mark.parametrize("fmt,name,d", [(1, "bf16", 64), (1, "bf16", 128), (2, "fp8", 64), (2, "fp8", 128)])
def test_block_layout(fmt, name, d):
    """Every element has a place of its own, the documented one, and scales follow the codes."""
    e = 2 if fmt == 1 else 1
    seen = set()
    for o in range(64):
        for x in range(d):
            k, v = rules().at(fmt, d, o, x, 0), rules().at(fmt, d, o, x, 1)
            assert (k, v) == (R.k_byte(o, x, d, e), 64 * d * e + R.v_byte(o, x, d, e))
            seen |= {k, v}
    assert seen == set(range(0, 2 * 64 * d * e, e))
    assert ops.kv_cache_bytes(1, 1, d, name) == 2 * 64 * d * e + 2 * 64 * 4


# ------------------------------------------------------------------------------- launch rules
def test_row_classes():
    """Which tile the sizes of the GPU tests and of their neighbours reach."""
    assert [rules().rows(n * 8, 8, 4) for n in (1, 4, 5, 16, 17, 64, 65, 1000)] == [16, 16, 64, 64, 128, 128, 256, 256]
    assert rules().rows(1, 8, 32) == 16      # most sequences idle
    assert rules().rows(300, 2, 1) == 128 and rules().rows(1000, 3, 1) == 256


def test_append_tiles():
    assert [rules().append(t, 8, 4, 128) for t in (1, 32, 1000, 1520, 1521, 4096)] == [4, 4, 4, 4, 16, 16]
    assert [rules().append(t, 12, 1, 64) for t in (1, 1000, 1024, 1040)] == [16, 16, 16, 16]
    assert rules().append(100, 8, 1, 128) == 8 and rules().append(100, 1, 0, 128) == 16


def chunks_of(p, seqs, heads, group, prefix):
    """The device's deal of tiles in chunks, in plain integers: items, partial slots, and each tile's pages."""
    tiles = [-(-n * group // p["rows"]) for n, _ in seqs]
    pages = [-(-k // 64) for _, k in seqs]
    cost = sum(t * g for t, g in zip(tiles, pages)) * heads
    per = max(p["least"], -(-cost // p["target"]))
    items = slots = 0
    for t, g in zip(tiles, pages):
        chunks = max(1, -(-g // per))
        items += t * chunks * heads
        slots += t * chunks * heads if prefix or chunks > 1 else 0
    return items, slots


@pytest.mark.parametrize("seed", range(40))
def test_grid_and_slots_hold_every_deal(seed):
    rng = random.Random(seed)
    log = lambda a, b: int(round(a * (b / a) ** rng.random()))
    for _ in range(25):
        heads, group, width = rng.choice((1, 2, 8, 32)), rng.choice((1, 3, 4, 16)), log(1, 2000)
        most = log(1, 2000)
        seqs = [(rng.choice((0, 1, log(1, most))), rng.randrange(0, 64 * width + 1)) for _ in range(log(1, 150))]
        T = sum(n for n, _ in seqs)
        if T == 0:
            continue
        prefix_pages = rng.choice((0, 0, log(1, 3000)))
        own, shared, total = plan(T, len(seqs), heads, group, 128, width, prefix_pages)
        assert own["rows"] == rules().rows(T, len(seqs), group)
        if own["in_runs"]:
            assert own["rows"] == 256 and own["slots"] == 2 * own["target"] and own["grid"] == own["target"]
        else:
            items, slots = chunks_of(own, seqs, heads, group, prefix_pages > 0)
            assert items <= own["grid"] and slots <= own["slots"], (seqs, heads, group, width)
        parts = own["slots"] * own["rows"]
        if prefix_pages:
            items, slots = chunks_of(shared, [(T, 64 * prefix_pages)], heads, group, True)
            assert items <= shared["grid"] and slots <= shared["slots"]
            parts += shared["slots"] * shared["rows"]
            assert own["rows"] > 16 or shared["rows"] <= 128
        assert total >= 4 * (128 + 4) * parts + 16 * (len(seqs) + 1)
        assert total == ops.attention_cache_workspace_bytes(T, len(seqs), heads * group, heads, 128, width, 64 * prefix_pages)
