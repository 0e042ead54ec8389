"""Calls on a stream of their own: what a call makes for itself (outputs, scratch, copies) belongs to the stream
that it launches on, and its scratch is held until the kernels are launched."""
import contextlib
import weakref

import pytest
import torch

from paper_2502_17728_amd import ops
from test_cache_rules import host_cache

BF16 = torch.bfloat16


class Launch:
    """The library replaced by a recorder, tensors of the host in place of the device's."""

    def __init__(self, monkeypatch):
        self.calls, self.made, self.on = 0, [], None
        m = monkeypatch
        for name in ops.SYMBOLS:
            if name.endswith("_bytes") or name in ("dn_status_string", "dn_version"):
                continue
            m.setattr(ops._lib, name, self.call)
        m.setattr(ops, "_dev", lambda t, name: None if t is None else t.data_ptr())
        m.setattr(ops, "_rows", lambda t, name: (t.data_ptr(), t.numel() // t.shape[0]))
        m.setattr(ops, "_stream_of", lambda stream, x: 77 if stream is None else stream)
        m.setattr(ops, "_stream", lambda stream: 77 if stream is None else stream)
        m.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: handle)
        m.setattr(torch.cuda, "default_stream", lambda device=None: 0)
        m.setattr(torch.cuda, "stream", self.current)
        empty, new_empty, empty_like, reshape = torch.empty, torch.Tensor.new_empty, torch.empty_like, torch.Tensor.reshape
        m.setattr(torch, "empty", lambda *a, **k: self.seen(empty(*a, **k)))
        m.setattr(torch, "empty_like", lambda *a, **k: self.seen(empty_like(*a, **k)))
        m.setattr(torch.Tensor, "new_empty", lambda *a, **k: self.seen(new_empty(*a, **k)))
        m.setattr(torch.Tensor, "reshape", lambda t, *a: t if (r := reshape(t, *a)).data_ptr() == t.data_ptr() else self.seen(r))

    @contextlib.contextmanager
    def current(self, stream):
        self.on = stream
        yield
        self.on = None

    def seen(self, t):
        self.made.append((weakref.ref(t), self.on, t.numel()))
        return t

    def call(self, *args):
        self.calls += 1
        gone = [n for ref, _, n in self.made if ref() is None]
        assert not gone, f"tensors of {gone} elements were given back before the launch"
        return 0


def prepared(K, N):
    return ops.PreparedLinear(torch.zeros(64, dtype=torch.uint8), ops.LnLinearWeights(K, N, ops.DN_BF16, 2, 4096))


def calls():
    x, w, one = torch.zeros(4, 64, dtype=BF16), prepared(64, 32), torch.ones(64, dtype=BF16)
    W, S, V = torch.zeros(64, 32, dtype=BF16), torch.zeros(2, 4, 8, dtype=BF16), torch.zeros(2, 8, 64, dtype=BF16)
    q, k = torch.zeros(4, 3, 64, dtype=BF16), torch.zeros(2, 700, 64, dtype=BF16)
    c, i = host_cache(), torch.zeros(4, dtype=torch.int32)
    r, Q, t = torch.zeros(4, 2, 64, dtype=BF16), torch.zeros(4, 4, 64, dtype=BF16), torch.zeros(8, 32, 2)
    bt, qs, kl = torch.zeros(3, 9, dtype=torch.int32), i, i[:3]
    return {
        "ln_linear_prepare": lambda **s: ops.ln_linear_prepare(W, one, **s),
        "ln_linear_deferred": lambda **s: ops.ln_linear_deferred(x, w, **s),
        "ln_linear_serial": lambda **s: ops.ln_linear_serial(x, w, **s),
        "ln_linear_norm_on_load": lambda **s: ops.ln_linear_norm_on_load(x, w, **s),
        "linear_deferred_post": lambda **s: ops.linear_deferred_post(x, w, one, **s),
        "rms_linear_deferred": lambda **s: ops.rms_linear_deferred(x, w, **s),
        "swiglu_prepare": lambda **s: ops.swiglu_prepare(W, W, one, **s),
        "rms_swiglu_deferred": lambda **s: ops.rms_swiglu_deferred(x, w, **s),
        "softmax_pv_deferred": lambda **s: ops.softmax_pv_deferred(S, V, **s),
        "attention_deferred": lambda **s: ops.attention_deferred(q, k, k, **s),
        "attention_decode_deferred": lambda **s: ops.attention_decode_deferred(q, k, k, **s),
        "attention_decode_deferred, strided": lambda **s: ops.attention_decode_deferred(q.transpose(0, 1).contiguous().transpose(0, 1), k, k, out=q, **s),
        "attention_decode_deferred_noalloc": lambda **s: ops.attention_decode_deferred_noalloc(q, k, k, **s),
        "layernorm": lambda **s: ops.layernorm(x, one, **s),
        "rmsnorm": lambda **s: ops.rmsnorm(x, one, **s),
        "silu_mul": lambda **s: ops.silu_mul(x, x, **s),
        "softmax": lambda **s: ops.softmax(S, **s),
        "gemm": lambda **s: ops.gemm(x, W, **s),
        "rotary_table": lambda **s: ops.rotary_table(torch.zeros(8, dtype=torch.float64), 9, **s),
        "rotary_apply": lambda **s: ops.rotary_apply(r, i, t, **s),
        "kv_cache_append": lambda **s: ops.kv_cache_append(c, torch.zeros(4, 8 * 64, dtype=BF16), i, **s),
        "kv_cache_read": lambda **s: ops.kv_cache_read(c, i, **s),
        "kv_cache_read, K given": lambda **s: ops.kv_cache_read(c, i, K=r, **s),
        "attention_cache_deferred": lambda **s: ops.attention_cache_deferred(Q, c, bt, qs, kl, **s),
        "attention_shared_prefix_deferred": lambda **s: ops.attention_shared_prefix_deferred(Q, c, i, 200, bt, qs, kl, **s),
    }


@pytest.mark.parametrize("name", sorted(calls()))
def test_scratch_is_held_until_the_launch(name, monkeypatch):
    launch = Launch(monkeypatch)
    calls()[name]()
    assert launch.calls == 1


@pytest.mark.parametrize("name", sorted(calls()))
def test_what_a_call_makes_belongs_to_its_stream(name, monkeypatch):
    call = calls()[name]
    launch = Launch(monkeypatch)
    call()
    assert launch.calls == 1 and launch.made and all(on is None for _, on, _ in launch.made)
    for stream in (5, 0):  # a handle; the default stream's
        launch.made.clear()
        call(stream=stream)
        assert launch.made and all(on == stream for _, on, _ in launch.made), launch.made
    assert launch.calls == 3 and launch.on is None


def test_the_current_stream_given_by_name(monkeypatch):
    """No switch of streams where the one given is the current one."""
    launch = Launch(monkeypatch)
    calls()["attention_cache_deferred"](stream=77)
    assert launch.calls == 1 and len(launch.made) == 2 and all(on is None for _, on, _ in launch.made)


# ------------------------------------------------------------------------------- on the device
def stream_of(t):
    """The stream that the allocator holds a tensor's memory for."""
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= t.data_ptr() < s["address"] + s["total_size"]:
            return s["stream"]


@pytest.mark.gpu
@pytest.mark.parametrize("as_handle", [False, True])
@pytest.mark.parametrize("seqs,prefix", [([(1, 5000), (1, 900)], 0), ([(20, 3000)], 0), ([(300, 3000)], 0), ([(1, 50)] * 6, 3000)])
def test_attention_over_the_cache_on_a_stream_given(seqs, prefix, as_handle):
    """Scratch of the call's own, while the current stream takes and writes memory of the same sizes."""
    from test_attention_cache import Batch
    b = Batch(seqs, 4, 1, 64, "fp8", prefix=prefix)
    want = b.run()
    b.check(want)
    n = ops.attention_cache_workspace_bytes(b.Q.shape[0], len(seqs), 4, 1, 64, b.table.shape[1], prefix)
    side = torch.cuda.Stream()
    Q = b.Q.cuda()
    torch.cuda.synchronize()
    held = []
    for _ in range(4):
        got = b.run(Q=Q, stream=side.cuda_stream if as_handle else side)
        assert stream_of(got) == side.cuda_stream
        held.append(got)
        for size in (n, got.numel() * 2):
            torch.empty(size, dtype=torch.uint8, device="cuda").fill_(0xFF)
    torch.cuda.synchronize()
    assert all(torch.equal(want, got) for got in held)


@pytest.mark.gpu
def test_decode_attention_on_a_stream_given():
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn((2, 5000, 64), generator=g).to(BF16).cuda() for _ in range(2))
    q = torch.randn((3, 4, 64), generator=g).to(BF16).cuda().transpose(0, 1)  # heads apart: copied by the call
    want = ops.attention_decode_deferred(q.contiguous(), k, v)
    n = ops.attention_decode_workspace_bytes(2, 6, 5000, 64)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    held = []
    for _ in range(4):
        got = ops.attention_decode_deferred(q, k, v, stream=side)
        assert stream_of(got) == side.cuda_stream
        held.append(got)
        for size in (n, q.numel() * 2):
            torch.empty(size, dtype=torch.uint8, device="cuda").fill_(0xFF)
    torch.cuda.synchronize()
    assert all(torch.equal(want, got) for got in held)
