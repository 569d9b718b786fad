"""Generation from prompts and to lengths at the ends of their ranges."""
import pytest
import torch

from paper_2412_07752_amd import language_model as lm

pytestmark = pytest.mark.gpu


def test_generation_of_no_words_of_one_and_of_several():
    model = lm.LanguageModel(40, 2, 32, dtype=torch.float32, seed=5)
    prompt = lm.chain_text(40, 6, 3, seed=2)[0]
    several = model.generate(prompt, 4)
    assert several.shape == (4, 3) and several.dtype == torch.int64
    none = model.generate(prompt, 0)
    assert none.shape == (0, 3) and none.dtype == torch.int64
    for n in (1, 2):
        assert torch.equal(model.generate(prompt, n), several[:n])
    assert torch.equal(model.generate(torch.cat([prompt, several[:2]]), 2), several[2:])
    assert model.generate(prompt[:1], 2).shape == (2, 3)
    assert torch.equal(model.generate(prompt.int(), 4), several)
    with pytest.raises(ValueError, match="0 words"):
        model.generate(prompt[:0], 2)
    with pytest.raises(ValueError, match="by -1"):
        model.generate(prompt, -1)
