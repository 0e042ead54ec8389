"""examples/serve_layers.py at the end of a sequence's room, and what it refuses (GPU)."""
import pytest
import torch

from test_serving_example import serve

pytestmark = pytest.mark.gpu


def server(room, sequences=3):
    torch.manual_seed(4)
    s = serve.Server(layers=2, hidden=256, q_heads=4, heads=2, d=64, ffn=512, vocabulary=512, sequences=sequences, prompt=100,
                     room=room, fmt="fp8")
    s.read_prompt(torch.randint(0, 512, (100,), device="cuda"))
    return s


def draw(*lengths):
    return [torch.randint(0, 512, (n,), device="cuda") for n in lengths]


@pytest.mark.parametrize("graphed", [False, True])
def test_a_full_sequence_leaves_the_others_as_they_are(graphed):
    """Steps past one sequence's room: its length and cached tokens stay, and the others go on as with more room."""
    made, lens = [], []
    for room in (64, 256):
        s = server(room)
        tokens = s.read_texts(draw(60, 5, 30))
        step = serve.record(s, tokens).replay if graphed else lambda: s.step(tokens)
        steps = []
        for _ in range(12):
            step()
            torch.cuda.synchronize()
            steps.append(tokens.clone())
            assert bool((tokens[1:] >= 0).all()) and bool((tokens < 512).all())
        made.append(torch.stack(steps))
        lens.append(s.kv_len.tolist())
    assert lens == [[64, 17, 42], [72, 17, 42]]
    assert torch.equal(made[0][:, 1:], made[1][:, 1:]) and torch.equal(made[0][:4, 0], made[1][:4, 0])


def test_slots_past_the_room():
    s = server(64, sequences=2)
    at = torch.tensor([0, 63, 64, 100000], device="cuda")
    first = int(s.own[1, 0]) * 64
    assert s.slots_of(torch.ones(4, device="cuda"), at).tolist() == [first, first + 63, -1, -1]


def test_texts_that_do_not_fit_are_refused():
    s = server(64)
    for texts in (draw(5, 5), draw(5, 0, 5), draw(65, 1, 1)):
        with pytest.raises(ValueError):
            s.read_texts(texts)
    s.read_texts(draw(64, 1, 1))
    with pytest.raises(ValueError):
        s.read_texts(draw(1, 1, 1))
    assert s.kv_len.tolist() == [64, 1, 1]
    with pytest.raises(ValueError):
        s.move(torch.zeros(1, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda"), 10000)
