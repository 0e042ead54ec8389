"""The 8-bit products together, as a decoder layer uses them: each step against its plain 64-bit form on what it was given,
recorded in a graph, on streams of their own, and in the serving example (GPU)."""
import importlib.util
import os

import pytest
import torch

from paper_2502_17728_amd import ops
from tests import fp8_reference as R

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
HIDDEN, FFN, VOCABULARY = 1024, 2560, 4104


class Layer:
    """norm -> gated product -> rows -> product onto the stream -> norm -> head -> log probabilities, with what each
    step was given and gave."""

    def __init__(self, M, seed=1):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(s, generator=g, device="cuda")
        self.x, self.d = rnd(M, HIDDEN).to(BF16), rnd(M, HIDDEN).to(BF16)
        self.gamma = (0.5 + torch.rand(HIDDEN, generator=g, device="cuda")).to(BF16)

        def weight(K, N):
            v, s, _ = R.quantised((rnd(K, N) * K ** -0.5).t().double())
            return v.t().float().to(R.F8).contiguous(), s.float()

        (self.w, self.ws), (self.u, self.us) = weight(HIDDEN, FFN), weight(HIDDEN, FFN)
        self.down, self.downs = weight(FFN, HIDDEN)
        self.head, self.heads = weight(HIDDEN, VOCABULARY)
        self.bias = rnd(VOCABULARY)
        self.W = ops.linear_fp8_prepare(self.w, scales=self.ws, up=self.u, up_scales=self.us)
        self.D = ops.linear_fp8_prepare(self.down, scales=self.downs)
        self.H = ops.linear_fp8_prepare(self.head, scales=self.heads, bias=self.bias)
        self.targets = torch.randint(0, VOCABULARY, (M, 2), generator=g, device="cuda", dtype=torch.int32)
        space = lambda w: torch.empty(max(256, ops.linear_fp8_workspace_bytes(M, w)), dtype=torch.uint8, device="cuda")
        self.spaces = [space(w) for w in (self.W, self.D, self.H)]

    def __call__(self, **kw):
        s = {}
        s["codes"], s["scales"], s["sum"] = ops.residual_rmsnorm_fp8(self.x, self.d, self.gamma, **kw)
        s["h"] = ops.linear_fp8(s["codes"], s["scales"], self.W, "silu", workspace=self.spaces[0], **kw)
        s["hc"], s["hs"] = ops.rows_fp8(s["h"], **kw)
        s["x2"] = ops.linear_fp8(s["hc"], s["hs"], self.D, residual=s["sum"], workspace=self.spaces[1], **kw)
        s["y"], _ = ops.residual_rmsnorm(s["x2"], None, self.gamma, **kw)
        s["yc"], s["ys"] = ops.rows_fp8(s["y"], **kw)
        s["logits"] = ops.linear_fp8(s["yc"], s["ys"], self.H, out_dtype=F32, workspace=self.spaces[2], **kw)
        s.update(ops.token_logprobs(s["logits"], self.targets, 3, **kw))
        return s


def same(a, b):
    return all(torch.equal(a[k].view(torch.uint8), b[k].view(torch.uint8)) for k in a)


@pytest.mark.parametrize("M", [1, 7, 33, 130, 520])
def test_each_step_on_what_it_was_given(M):
    L = Layer(M)
    s = L()
    norm = (0.5 * 90 + 7) * 2.0 ** -24
    h, r, a = R.rmsnorm(L.x, L.d, L.gamma, 1e-5)
    v, sc, _ = R.quantised(a)
    R.assert_codes(s["codes"], v)
    R.assert_within(s["scales"], sc * r, sc * r * (norm + 3 * 2.0 ** -24))
    R.assert_within(s["sum"], h, h.abs() * (2.0 ** -8 + 2.0 ** -24))
    ref, e = R.linear(s["codes"], s["scales"], L.w, L.ws, None, "silu", L.u, L.us, None, f32=False)
    R.assert_within(s["h"], ref, e + (ref.abs() + e) * 2.0 ** -8)
    v, sc, _ = R.quantised(s["h"].double())
    R.assert_codes(s["hc"], v)
    R.assert_within(s["hs"], sc, sc * 2.0 ** -23)
    ref, e = R.linear(s["hc"], s["hs"], L.down, L.downs, None, "none", residual=s["sum"], f32=False)
    R.assert_within(s["x2"], ref, e + (ref.abs() + e) * 2.0 ** -8)
    _, r, a = R.rmsnorm(s["x2"], None, L.gamma, 1e-5)
    R.assert_within(s["y"], a * r[:, None], (a * r[:, None]).abs() * (2.0 ** -8 + norm))
    ref, e = R.linear(s["yc"], s["ys"], L.head, L.heads, L.bias, "none")
    R.assert_within(s["logits"], ref, e + (ref.abs() + e) * 2.0 ** -24)
    ref = R.logprobs(s["logits"], L.targets, 3)
    assert torch.equal(s["top_ids"].long(), ref["top_ids"])
    for k in ("logprobs", "top_logprobs", "entropy"):
        # logits of a few units: the bounds of the log probabilities' own tests are below 2e-5 there
        R.assert_within(s[k], ref[k], ref[k].abs() * 4 * 2.0 ** -24 + 2e-5)


@pytest.mark.parametrize("M", [1, 40, 300])
def test_a_graph_replays_with_what_its_inputs_hold(M):
    L = Layer(M)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        L()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = L()
    for k in range(4):
        L.x.normal_()
        L.d.normal_().mul_(k + 1)
        L.targets.random_(0, VOCABULARY)
        graph.replay()
        torch.cuda.synchronize()
        got = {n: t.clone() for n, t in held.items()}
        assert same(got, L()), k
    torch.cuda.synchronize()


def test_on_streams_of_their_own():
    layers = [Layer(40, 5), Layer(40, 6)]
    want = [L() for L in layers]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in layers]
    for _ in range(5):
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
        got = [L(stream=s) for L, s in zip(layers, streams)]  # side by side
        torch.cuda.synchronize()
        assert all(same(a, b) for a, b in zip(got, want))
    with torch.cuda.stream(streams[0]):
        got = layers[0]()
    torch.cuda.synchronize()
    assert same(got, want[0])


def test_a_part_of_a_batch():
    """Rows from any one on, with what belongs to them; the rows around are left as they were."""
    L = Layer(70)
    s = L()
    for a, b in ((1, 4), (3, 70), (5, 6)):
        codes, scales = torch.zeros_like(s["codes"]), torch.full_like(s["scales"], -1.0)
        ops.residual_rmsnorm_fp8(L.x[a:b], L.d[a:b], L.gamma, codes=codes[a:b], scales=scales[a:b])
        R.assert_codes(codes[a:b], s["codes"][a:b].double())
        assert torch.equal(scales[a:b], s["scales"][a:b]) and (scales[:a] == -1).all() and (scales[b:] == -1).all()
        assert (codes[:a].view(torch.uint8) == 0).all() and (codes[b:].view(torch.uint8) == 0).all()
        ref, e = R.linear(s["codes"][a:b], s["scales"][a:b], L.w, L.ws, None, "silu", L.u, L.us, None, f32=False)
        h = torch.full_like(s["h"], 7.0)
        ops.linear_fp8(s["codes"][a:b], s["scales"][a:b], L.W, "silu", out=h[a:b])
        R.assert_within(h[a:b], ref, e + (ref.abs() + e) * 2.0 ** -8)
        assert (h[:a] == 7).all() and (h[b:] == 7).all()
        targets = torch.cat([L.targets, L.targets[:, :1]], 1)  # rows of 12 bytes
        got, ref = ops.token_logprobs(s["logits"][a:b], targets[a:b], 3), R.logprobs(s["logits"][a:b], targets[a:b], 3)
        assert torch.equal(got["top_ids"].long(), ref["top_ids"])
        R.assert_within(got["logprobs"], ref["logprobs"], ref["logprobs"].abs() * 4 * 2.0 ** -24 + 2e-5)


def test_long_offsets():
    """Rows whose last bytes lie past 4 GiB."""
    K = 16384
    M = 2 ** 32 // K + 3
    x = torch.zeros((M, K), dtype=torch.uint8, device="cuda").view(R.F8)
    tail = torch.randn((5, K), device="cuda")
    codes, scales = ops.rows_fp8(tail)
    x[-5:] = codes
    xs = torch.ones(M, device="cuda")
    xs[-5:] = scales
    W = torch.randn((K, 16), device="cuda") * K ** -0.5
    w = ops.linear_fp8_prepare(W)
    few = ops.linear_fp8(codes, scales, w, out_dtype=F32)
    many = ops.linear_fp8(x, xs, w, out_dtype=F32)
    assert (many[:-5] == 0).all()
    assert torch.allclose(many[-5:], few, rtol=0, atol=K * 2.0 ** -24 * float(few.abs().max()))
    del x, many
    logits = torch.zeros((2 ** 31 // 131072 + 2, 131072), dtype=BF16, device="cuda")
    logits[-1] = torch.randn(131072, device="cuda").to(BF16)
    a, b = ops.token_logprobs(logits, None, 5), ops.token_logprobs(logits[-1:].clone(), None, 5)
    assert torch.equal(a["top_ids"][-1], b["top_ids"][0]) and a["top_ids"][0].tolist() == [0, 1, 2, 3, 4]


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_the_longest_row(dtype):
    V = 2 ** 30 - 1
    logits = torch.zeros((1, V), dtype=dtype, device="cuda")
    ids = [V - 1, 2 ** 29 + 7, 3]
    for i, at in enumerate(ids):
        logits[0, at] = 50.0 - 5 * i
    got = ops.token_logprobs(logits, torch.tensor([ids], dtype=torch.int32, device="cuda"), 5)
    assert got["top_ids"][0].tolist() == ids + [0, 1]
    # the zeros' share is 2^30 e^-50, 2e-13 of the sum
    d = torch.tensor([0.0, -5.0, -10.0], dtype=torch.float64, device="cuda")
    want = d - d.exp().sum().log()
    bound = 16 * 2.0 ** -24 * (1 + want.abs())
    R.assert_within(got["logprobs"][0], want, bound)
    R.assert_within(got["top_logprobs"][0, :3], want, bound)


PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_layers.py")
spec = importlib.util.spec_from_file_location("serve_layers", PATH)
serve = importlib.util.module_from_spec(spec)
spec.loader.exec_module(serve)
TEXTS = [70, 3, 1, 130, 64]


def server(products):
    torch.manual_seed(3)
    s = serve.Server(layers=2, hidden=256, q_heads=4, heads=2, d=64, ffn=512, vocabulary=512, sequences=5, prompt=192, room=256,
                     fmt="fp8", products=products)
    s.read_prompt(torch.randint(0, 512, (192,), device="cuda"), chunk=100)
    return s, [torch.randint(0, 512, (n,), device="cuda") for n in TEXTS]


def test_served_steps_replay():
    runs = []
    for graphed in (False, True):
        s, texts = server("fp8")
        tokens = s.read_texts(texts)
        step = serve.record(s, tokens).replay if graphed else lambda: s.step(tokens)
        made = []
        for _ in range(20):
            step()
            made.append(tokens.clone())
            torch.cuda.synchronize()
        runs.append(torch.stack(made))
    assert torch.equal(runs[0], runs[1])


@pytest.mark.parametrize("products", ["bf16", "fp8"])
def test_scores(products):
    s, texts = server(products)
    logprobs, entropy = s.score(texts)
    assert s.kv_len.tolist() == TEXTS and len(logprobs) == sum(TEXTS)
    last = torch.tensor(TEXTS, device="cuda").cumsum(0) - 1
    assert (logprobs[last] == 0).all() and (entropy >= 0).all()
    s.kv_len.zero_()
    x, _ = s._read(texts)
    ref = torch.log_softmax(ops.rms_linear_deferred(x, s.head).double(), 1)
    follows = torch.cat([torch.cat(texts)[1:], texts[0][:1]])
    want = ref.gather(1, follows[:, None])[:, 0]
    want[last] = 0
    R.assert_within(logprobs, want, want.abs() * 4 * 2.0 ** -24 + 2e-5)
