"""The decoding loop at the end of its room."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2502_15572_b200 import speculate
from tests.test_speculate_gpu import logits64

pytestmark = pytest.mark.gpu


def check_text(model, quantised, prompt, text):
    """The bound of tests/test_speculate_gpu.py."""
    x = logits64(model, np.array(prompt + text[:-1]), quantised, "f16")[len(prompt) - 1:]
    gap = x.max(-1) - x[np.arange(len(text)), text]
    assert gap.max() <= 16 * np.sqrt(20) * (2.0 ** -8 if quantised else 2.0 ** -11) * x.std()


@pytest.mark.parametrize("room", [0, 1, 12])
def test_texts_longer_than_their_room_are_refused(room):
    model, prompts = speculate.Decoder(seed=5), [[3, 5, 7], [11] * 20]
    spec = speculate.Speculator(model, prompts, room, page_size=16)
    with pytest.raises(ValueError):
        spec.run(room + 2)
    texts, steps = spec.run(room + 1)                         # the first token stands behind the prompt already
    assert steps == room
    for prompt, text in zip(prompts, texts):
        check_text(model, False, prompt, text)
    with pytest.raises(ValueError):
        spec.step()
    with pytest.raises(ValueError):
        spec.run(2)


def test_texts_in_several_pieces():
    """A second piece begins with the last token of the first one, and is refused where it does not fit."""
    model, prompts, room = speculate.Decoder(seed=5), [[3, 5, 7], [11] * 20], 20
    whole = speculate.Speculator(model, prompts, room).run(room + 1)[0]
    spec = speculate.Speculator(model, prompts, room)
    first, _ = spec.run(9)
    with pytest.raises(ValueError):
        spec.run(14)
    second, _ = spec.run(13)
    assert [a + b[1:] for a, b in zip(first, second)] == whole


def test_a_sequence_ahead_does_not_go_on_beyond_its_room():
    """The first sequence's drafts are accepted, the second one's are not: the next piece would begin beyond the first one's room."""
    model, prompts = speculate.Decoder(seed=5), [[3, 5, 7], [11] * 20]
    store = speculate.make_datastore(model, [prompts[0] + speculate.Speculator(model, prompts, 121).run(120)[0][0]], 9)
    spec = speculate.Speculator(model, prompts, 30, store, 2, 8, page_size=16)
    texts, _ = spec.run(16)
    assert int(spec.ctx[0]) - len(prompts[0]) == 30 and int(spec.ctx[1]) - len(prompts[1]) < 30
    for prompt, text in zip(prompts, texts):
        check_text(model, False, prompt, text)
    with pytest.raises(ValueError):
        spec.run(5)
