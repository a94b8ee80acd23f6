"""Steps of a text layer that are refused, taken back, given again or run twice (no GPU: the layer's own work is left
out)."""

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


def test_a_refused_step_is_taken_back():
    cache = prompt.TextCache(2, 10)
    layer = Layer(cache)
    layer.step(h(5), cache.extend([2, 3]))
    with pytest.raises(ValueError, match="rows"):
        layer.step(h(3), cache.extend([1, 1]))
    assert cache.lens == [2, 3]
    s = cache.extend([1, 0])
    assert s["pos"].tolist() == [2] and s["slots"].tolist() == [2] and s["k_len"].tolist() == [3, 3]
    layer.step(h(1), s)
    assert layer.log == [[2, 3], [3, 3]] and cache.lens == [3, 3]


def test_given_again():
    cache = prompt.TextCache(2, 10)
    layer = Layer(cache)
    s = cache.extend([2, 3])
    for _ in range(2):
        with pytest.raises(ValueError, match="rows"):
            layer.step(h(1), s)
        assert cache.lens == [0, 0]
    layer.step(h(5), s)
    assert cache.lens == [2, 3] and layer.log == [[2, 3]]
    t, u = cache.extend([1, 1]), cache.extend([2, 0])
    with pytest.raises(ValueError, match="rows"):
        layer.step(h(1), t)
    assert cache.lens == [2, 3]
    with pytest.raises(ValueError, match="taken back"):  # not before the one it follows
        layer.step(h(2), u)
    layer.step(h(2), t)
    layer.step(h(2), u)
    assert cache.lens == [5, 4] and layer.log[1:] == [[3, 4], [5, 4]]


def test_not_again_behind_another():
    cache = prompt.TextCache(1, 10)
    layer = Layer(cache)
    s = cache.extend([4])
    cache.take_back(s)
    cache.take_back(s)
    t = cache.extend([2])
    with pytest.raises(ValueError, match="taken back"):
        layer.step(h(4), s)
    assert cache.lens == [2]
    layer.step(h(2), t)
    assert cache.lens == [2] and layer.log == [[2]]
    cache.take_back(t)  # also of a step that has run
    assert cache.lens == [0]


def test_several_layers_and_steps_that_run_twice():
    cache = prompt.TextCache(1, 10)
    one, two = Layer(cache), Layer(prompt.TextCache(1, 10))
    s = cache.extend([4])
    one.step(h(4), s)
    with pytest.raises(ValueError, match="rows"):
        two.step(h(3), s)
    assert cache.lens == [0]  # the second layer does not have it
    for _ in range(3):
        for layer in (one, two):
            layer.step(h(4), s)
    t = cache.extend([1])
    for layer in (one, two):
        layer.step(h(1), t)
    with pytest.raises(ValueError, match="rows"):
        one.step(h(2), s)  # a step that the layer has had stays
    assert cache.lens == [5]
    one.step(h(4), s)
    assert cache.lens == [5]


@pytest.mark.parametrize("texts, room", [(3, 10), (2, 11), (1, 10)])
def test_steps_of_texts_that_lie_elsewhere(texts, room):
    layer, other = Layer(prompt.TextCache(2, 10)), prompt.TextCache(texts, room)
    with pytest.raises(ValueError, match="a layer for 2 of 10"):
        layer.step(h(texts), other.extend([1] * texts))
    assert other.lens == [0] * texts and layer.log == []


def test_lengths_set_by_hand():
    """A step keeps the lengths that it was made for."""
    cache = prompt.TextCache(2, 10)
    s = cache.extend([1, 2])
    cache.lens[0] = 7
    assert s["after"] == [1, 2] and s["before"] == [0, 0]
    assert cache.extend([1, 0])["pos"].tolist() == [7]


def test_taken_back_and_given_again_many_times():
    """A later step and then the one before it; both again; what they are does not depend on how often."""
    cache = prompt.TextCache(1, 10)
    layer = Layer(cache)
    s, t = cache.extend([2]), cache.extend([3])
    for _ in range(3):
        cache.take_back(t)
        assert cache.lens == [2]
        cache.take_back(s)
        assert cache.lens == [0]
        layer.step(h(2), s)
        layer.step(h(3), t)
        layer.step(h(3), t)
        assert cache.lens == [5]
    assert len(cache.gone) == 1
    u = cache.extend([1])
    layer.step(h(1), u)
    assert cache.lens == [6] and layer.log[-1] == [6]
