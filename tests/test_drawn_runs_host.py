"""Arguments of drawn runs, no GPU needed: refused before either model is touched."""
from types import SimpleNamespace

import numpy as np
import pytest


@pytest.mark.parametrize("numbers", [None, np.zeros((2, 4)), np.zeros((3, 5)), np.zeros(12), 0.5])
def test_a_number_for_every_position(numbers):
    from paper_2504_07878_amd import joint, sampling
    model = SimpleNamespace(shape=dict(vocab=10), device="cuda:0")
    with pytest.raises(ValueError, match="numbers"):
        joint.generate(model, model, [[1], [2], [3]], 4, draw=sampling.Draw(), numbers=numbers)


def test_numbers_are_on_the_device_of_each_model(monkeypatch):
    from paper_2504_07878_amd import joint, sampling
    monkeypatch.setattr(sampling, "Sampler", lambda rows, vocab, device: None)
    small, large = (SimpleNamespace(shape=dict(vocab=10), device=d) for d in ("cpu", "meta"))
    for chooser, model in zip(joint._choosers(small, large, 3, 4, sampling.Draw(), np.zeros((3, 4))), (small, large)):
        assert chooser.numbers.device.type == model.device
