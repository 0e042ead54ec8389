"""examples/serve_layers.py at small sizes: the operators run together give what they give apart (GPU)."""
import importlib.util
import os

import pytest
import torch

from paper_2502_17728_amd import ops

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serve_layers.py")
spec = importlib.util.spec_from_file_location("serve_layers", PATH)
serve = importlib.util.module_from_spec(spec)
spec.loader.exec_module(serve)


def server(fmt, prompt=192):
    torch.manual_seed(3)
    s = serve.Server(layers=2, hidden=256, q_heads=4, heads=2, d=64, ffn=512, vocabulary=512, sequences=5, prompt=prompt,
                     room=256, fmt=fmt)
    s.read_prompt(torch.randint(0, 512, (prompt,), device="cuda"), chunk=100)
    return s


TEXTS = [70, 3, 1, 130, 64]


def texts():
    return [torch.randint(0, 512, (n,), device="cuda") for n in TEXTS]


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
def test_shared_prefix_is_the_same_as_tables_that_name_it(fmt):
    """Every attention call of texts and steps, against one whose tables hold the prompt's pages too.  Each is
    within (2^-8 + 2^-9) of the sum over |V| (at most its largest value) and 2^-8 + 2^-15 of the result."""
    s = server(fmt)
    whole = torch.cat([s.shared.expand(s.sequences, -1), s.own], 1)
    seen = []

    def behind(q_start, kv_len, workspace=None):
        def attend(q, cache):
            a = ops.attention_shared_prefix_deferred(q, cache, s.shared, s.prompt, s.own, q_start, kv_len, workspace=workspace)
            b = ops.attention_cache_deferred(q, cache, whole, q_start, kv_len + s.prompt)
            # every slot that was written; a page's unwritten slots hold anything
            used = torch.cat([torch.arange(s.prompt, device="cuda").int()] + [
                s.slots_of(torch.full((n,), i, device="cuda"), torch.arange(n, device="cuda"))
                for i, n in enumerate(kv_len.tolist())])
            top = ops.kv_cache_read(cache, used)[1].float().abs().amax(0).repeat_interleave(2, 0)
            bound = 2 * ((2.0 ** -8 + 2.0 ** -9) * top + (2.0 ** -8 + 2.0 ** -15) * a.float().abs())
            seen.append(float(((a.float() - b.float()).abs() / bound).max()))
            return a
        return attend

    s.attend_behind_prompt = behind
    tokens = s.read_texts(texts())
    for _ in range(3):
        s.step(tokens)
    assert len(seen) == 2 * 4 and max(seen) <= 1.0, seen


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
def test_replayed_steps_are_the_eager_ones(fmt):
    runs = []
    for graphed in (False, True, True):
        s = server(fmt)
        tokens = s.read_texts(texts())
        step = serve.record(s, tokens).replay if graphed else lambda: s.step(tokens)
        made = []
        for _ in range(70):  # past the end of a page
            step()
            made.append(tokens.clone())
            torch.cuda.synchronize()
        assert s.kv_len.tolist() == [n + 70 for n in TEXTS]
        runs.append(torch.stack(made))
    assert torch.equal(runs[0], runs[1]) and torch.equal(runs[0], runs[2])


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
def test_moved_tokens(fmt):
    """Moved keys are the cached ones turned by the distance, values the cached ones: one rounding to bf16 of
    the turned keys (2^-8), then the format's (bf16: the same value; e4m3: 2^-4 of a value, or half of
    its least step 2^-9 where the row's largest is 448, and 2^-8 more as it is read back)."""
    s = server(fmt)
    n, distance = 90, 37
    slots = torch.arange(5, 5 + n, device="cuda").int()
    to = s.slots_of(torch.full((n,), 2, device="cuda"), torch.arange(n, device="cuda"))
    before = [[t.double().cpu() for t in ops.kv_cache_read(layer.cache, slots)] for layer in s.layers]
    s.move(slots, to, distance)
    c, sn = (s.table[distance, :, k].double().cpu() for k in (0, 1))
    for layer, (K, V) in zip(s.layers, before):
        a, b = K[..., :32], K[..., 32:]
        want = torch.cat([a * c - b * sn, b * c + a * sn], -1)
        for got, w in zip(ops.kv_cache_read(layer.cache, to), (want, V)):
            top = w.abs().amax(-1, keepdim=True)
            bound = (2.0 ** -8) * w.abs() * 1.01 if fmt == "bf16" else \
                (2.0 ** -4 + 2 * 2.0 ** -8) * 1.05 * w.abs() + top / 448 * 2.0 ** -10 * 1.05
            bound = bound + 2.0 ** -22 * top  # fp32 products and sums of a pair
            assert bool(((got.double().cpu() - w).abs() <= bound).all())
