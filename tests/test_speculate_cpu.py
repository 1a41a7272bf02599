"""Refusals of the decoding example that need no GPU."""
import pytest

pytest.importorskip("torch")

from paper_2502_15572_b200 import speculate


@pytest.mark.parametrize("prompts", [[], [[]], [[1, 2], []]])
def test_sequences_without_a_prompt_are_refused(prompts):
    """There is no last token whose successor could be asked for (the row of another sequence was taken for it)."""
    model = speculate.Decoder(vocab=11, width=16, layers=1, device="cpu")
    with pytest.raises(ValueError):
        speculate.Speculator(model, prompts, 4)
