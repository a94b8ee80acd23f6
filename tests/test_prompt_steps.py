"""Steps of a text layer that are refused (no GPU: the layer's own work is left out)."""

import pytest
import torch

from paper_2608_09231_gb300 import prompt


@pytest.fixture(autouse=True)
def on_the_host(monkeypatch):
    monkeypatch.setattr(prompt, "DEV", "cpu")


class Layer(prompt.TextAttention):
    """Writes down the lengths of the steps it runs; refuses any whose rows are not h's."""

    def __init__(self, cache):
        self.texts, self.room, self.log = cache.texts, cache.room, []

    def _run(self, h, step):
        if h.shape[0] != step["rows"]:
            raise ValueError("rows")
        self.log.append(step["k_len"].tolist())


def h(n):
    return torch.zeros(n, 8)


@pytest.mark.parametrize("texts, room", [(3, 10), (2, 11), (1, 10)])
def test_steps_of_texts_that_lie_elsewhere(texts, room):
    layer, other = Layer(prompt.TextCache(2, 10)), prompt.TextCache(texts, room)
    with pytest.raises(ValueError, match="a layer for 2 of 10"):
        layer.step(h(texts), other.extend([1] * texts))
    assert layer.log == []
