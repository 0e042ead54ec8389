"""Decoder layers served from a paged key/value cache, with the package's entry points alone.

A prompt that all sequences share is cached once, chunk by chunk; the sequences' own texts follow in one
ragged call; then every sequence generates, one token a step, the step recorded once as a HIP graph that
replays while lengths, slots and positions move on the device.  A document that was cached by itself is
moved behind a sequence without running the layers again: read, turned by the distance, written.

    python examples/serve_layers.py                        # 8B-class layers, 32 sequences, an e4m3 cache
    python examples/serve_layers.py --layers 4 --format bf16

Weights and tokens are random: what runs is the arithmetic of such a model, not its text.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2502_17728_amd import ops  # noqa: E402

PAGE = ops.DN_KV_PAGE


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


class Layer:
    """RMSNorm -> QKV -> attention over the cache -> output product, RMSNorm -> SwiGLU -> down product."""

    def __init__(self, hidden, q_heads, heads, d, ffn, pages, fmt, g):
        w = lambda K, N: (torch.randn((K, N), generator=g, device="cuda") * K ** -0.5).to(torch.bfloat16)
        ones = lambda n: torch.ones(n, dtype=torch.bfloat16, device="cuda")
        self.qkv = ops.ln_linear_prepare(w(hidden, (q_heads + 2 * heads) * d), ones(hidden))
        self.out = ops.ln_linear_prepare(w(q_heads * d, hidden), ones(q_heads * d))
        self.mlp = ops.swiglu_prepare(w(hidden, ffn), w(hidden, ffn), ones(hidden))
        self.down = ops.ln_linear_prepare(w(ffn, hidden), ones(ffn))
        self.cache = ops.kv_cache_create(pages, heads, d, fmt)

    def __call__(self, x, attend, slots, positions, table):
        q = ops.kv_cache_append(self.cache, ops.rms_linear_deferred(x, self.qkv), slots, positions, table)
        x = x + ops.gemm(attend(q, self.cache).view(x.shape[0], -1), self.out)
        return x + ops.gemm(ops.rms_swiglu_deferred(x, self.mlp), self.down)


class Server:
    def __init__(self, layers=2, hidden=4096, q_heads=32, heads=8, d=128, ffn=14336, vocabulary=8192, sequences=32,
                 prompt=4096, room=512, fmt="fp8", seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.sequences, self.prompt = sequences, prompt
        own = -(-room // PAGE)
        self.room = own * PAGE  # tokens of a sequence behind the prompt at most
        self.prefix_pages = -(-prompt // PAGE)
        pages = self.prefix_pages + sequences * own
        self.layers = [Layer(hidden, q_heads, heads, d, ffn, pages, fmt, g) for _ in range(layers)]
        self.table = ops.rotary_table(ops.rotary_frequencies(d)[0], prompt + self.room)
        self.embed = torch.randn((vocabulary, hidden), generator=g, device="cuda").to(torch.bfloat16)
        self.head = ops.ln_linear_prepare(self.embed.t().contiguous() * hidden ** -0.5,
                                          torch.ones(hidden, dtype=torch.bfloat16, device="cuda"))
        self.shared = torch.arange(self.prefix_pages, dtype=torch.int32, device="cuda")
        self.own = self.prefix_pages + torch.arange(sequences * own, dtype=torch.int32, device="cuda").view(sequences, own)
        self.kv_len = ints([0] * sequences)  # tokens of each sequence behind the prompt
        self.one_each = ints(range(sequences + 1))
        need = ops.attention_cache_workspace_bytes
        self.workspace = torch.empty(need(sequences, sequences, q_heads, heads, d, own, prompt) + 256, dtype=torch.uint8,
                                     device="cuda")

    def run(self, tokens, attend, slots, positions):
        x = self.embed[tokens]
        for layer in self.layers:
            x = layer(x, attend, slots, positions, self.table)
        return x

    def next_tokens(self, x):
        return ops.rms_linear_deferred(x, self.head).argmax(-1)

    def read_prompt(self, tokens, chunk=1024):
        """The shared prompt, `chunk` tokens at a time, each against all before it."""
        for at in range(0, self.prompt, chunk):
            n = min(chunk, self.prompt - at)
            slots = ints(range(at, at + n))  # its pages come first, in order
            q_start, kv_len = ints([0, n]), ints([at + n])
            attend = lambda q, cache: ops.attention_cache_deferred(q, cache, self.shared[None], q_start, kv_len)
            self.run(tokens[at:at + n], attend, slots, slots)

    def attend_behind_prompt(self, q_start, kv_len, workspace=None):
        return lambda q, cache: ops.attention_shared_prefix_deferred(q, cache, self.shared, self.prompt, self.own, q_start,
                                                                     kv_len, workspace=workspace)

    def slots_of(self, sequence, at):
        """Where tokens `at` of the sequences lie; -1 (written nowhere) past a sequence's room."""
        page = self.own[sequence.long(), (at // PAGE).long().clamp(max=self.own.shape[1] - 1)]
        return torch.where(at < self.room, page * PAGE + at % PAGE, -1).int()

    def read_texts(self, texts):
        """Each sequence's own tokens, all in one ragged call; the tokens that follow."""
        if len(texts) != self.sequences or min(map(len, texts)) < 1:
            raise ValueError(f"a text of one token at least is needed for each of {self.sequences} sequences")
        lengths = ints([len(t) for t in texts])
        if int((self.kv_len + lengths).max()) > self.room:
            raise ValueError(f"a sequence has room for {self.room} tokens")
        q_start = torch.cat([lengths.new_zeros(1), lengths.cumsum(0, dtype=torch.int32)])
        sequence = torch.repeat_interleave(torch.arange(self.sequences, device="cuda"), lengths.long())
        at = (torch.arange(len(sequence), device="cuda") - q_start[sequence] + self.kv_len[sequence]).int()
        self.kv_len += lengths
        x = self.run(torch.cat(texts), self.attend_behind_prompt(q_start, self.kv_len), self.slots_of(sequence, at),
                     (self.prompt + at).int())
        return self.next_tokens(x[q_start[1:].long() - 1])

    def step(self, tokens):
        """One token of every sequence: the lengths move on the device, so the step can be replayed.  A sequence
        whose room is full stays as it is: its further tokens see it, and are not kept."""
        at = self.kv_len.clone()
        self.kv_len.add_(1).clamp_(max=self.room)
        attend = self.attend_behind_prompt(self.one_each, self.kv_len, self.workspace)
        x = self.run(tokens, attend, self.slots_of(self.one_each[:-1], at), (self.prompt + at).clamp(max=len(self.table) - 1))
        tokens.copy_(self.next_tokens(x))

    def move(self, slots, to, distance):
        """The keys and values at `slots` of every layer, put at slots `to` as if they were `distance` tokens
        further on: a rotation by p, then by the distance, is the rotation by their sum."""
        if not 0 <= distance < len(self.table):
            raise ValueError(f"the table turns by less than {len(self.table)} positions")
        by = torch.full_like(slots, distance)
        for layer in self.layers:
            K, V = ops.kv_cache_read(layer.cache, slots)
            K = ops.rotary_apply(K, by, self.table)
            ops.kv_cache_append(layer.cache, torch.cat([K, V], 1).flatten(1), to)


def record(server, tokens):
    """The step as a graph; what the recording's warm-up moved is put back."""
    kept = tokens.clone(), server.kv_len.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        server.step(tokens)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        server.step(tokens)
    tokens.copy_(kept[0])
    server.kv_len.copy_(kept[1])
    return graph


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--layers", type=int, default=2)
    p.add_argument("--sequences", type=int, default=32)
    p.add_argument("--prompt", type=int, default=4096)
    p.add_argument("--steps", type=int, default=64)
    p.add_argument("--format", choices=sorted(ops.KV_FORMATS), default="fp8")
    a = p.parse_args()
    if min(a.layers, a.sequences, a.prompt, a.steps) < 1:
        p.error("--layers, --sequences, --prompt and --steps are at least 1")
    room = 256 + a.steps
    s = Server(layers=a.layers, sequences=a.sequences, prompt=a.prompt, room=room, fmt=a.format)
    draw = lambda n: torch.randint(0, s.embed.shape[0], (n,), device="cuda")

    def timed(what, tokens, f):
        torch.cuda.synchronize()
        t = time.perf_counter()
        result = f()
        torch.cuda.synchronize()
        t = time.perf_counter() - t
        print(f"{what}: {t * 1e3:.2f} ms, {tokens / t:.0f} tokens/s", flush=True)
        return result

    s.read_prompt(draw(a.prompt))  # first calls load kernels; the timed ones write the same slots again
    timed(f"prompt of {a.prompt} tokens", a.prompt, lambda: s.read_prompt(draw(a.prompt)))
    texts = [draw(20 + 29 * b % 100) for b in range(a.sequences)]
    s.read_texts(texts)
    s.kv_len.zero_()
    tokens = timed("ragged texts", sum(map(len, texts)), lambda: s.read_texts(texts))
    n = min(100, a.prompt)  # the prompt's first tokens once more, behind sequence 0: 100 tokens that no layer runs
    at = s.kv_len[0] + torch.arange(n, device="cuda", dtype=torch.int32)
    distance = a.prompt + int(s.kv_len[0])
    timed(f"{n} cached tokens moved", n, lambda: s.move(ints(range(n)), s.slots_of(torch.zeros_like(at), at), distance))
    s.kv_len[0] += n
    graph = record(s, tokens)
    timed(f"{a.steps} steps of {a.sequences} sequences", a.steps * a.sequences,
          lambda: [graph.replay() for _ in range(a.steps)])


if __name__ == "__main__":
    main()
