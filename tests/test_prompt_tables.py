"""Rotary tables and the bookkeeping of texts in a cache (no GPU)."""

import math

import numpy as np
import pytest
import torch

from paper_2608_09231_gb300 import prompt


def test_plain_frequencies():
    f, s = prompt.rope_frequencies(64, 10000.0)
    assert s == 1.0 and f[0] == 1.0 and abs(f[-1] - 10000.0 ** (-63 / 64)) < 1e-18
    assert np.allclose(f[1:] / f[:-1], 10000.0 ** (-1 / 64), rtol=1e-14)


@pytest.mark.parametrize("factor", [2.0, 8.0])
def test_long_contexts(factor):
    f, _ = prompt.rope_frequencies(64)
    lin, s = prompt.rope_frequencies(64, factor=factor, scaling="linear")
    assert s == 1.0 and np.allclose(lin * factor, f, rtol=1e-15)
    base, s = prompt.rope_frequencies(64, factor=factor, scaling="base")
    assert s == 1.0 and base[0] == 1.0 and abs(base[-1] * factor / f[-1] - 1) < 1e-12
    parts, s = prompt.rope_frequencies(64, factor=factor, original=8192)
    assert abs(s - 0.1 * math.log(factor) - 1) < 1e-15
    turns = 8192 * f / (2 * math.pi)
    assert np.allclose(parts[turns > 32], f[turns > 32], rtol=1e-15)
    assert np.allclose(parts[turns < 1] * factor, f[turns < 1], rtol=1e-15)
    assert (turns > 32).any() and (turns < 1).any() and (np.diff(parts) < 0).all()


def test_bad_tables():
    for args in (dict(pairs=0), dict(pairs=4, theta=1.0), dict(pairs=4, factor=0.5), dict(pairs=4, factor=2.0, scaling="none"),
                 dict(pairs=4, factor=2.0, slow=3.0, fast=3.0)):
        with pytest.raises(ValueError):
            prompt.rope_frequencies(**args)


def test_places_of_texts(monkeypatch):
    monkeypatch.setattr(prompt, "DEV", "cpu")
    c = prompt.TextCache(3, 10)
    s = c.extend([4, 0, 7])
    assert s["rows"] == 11 and s["max_q"] == 7 and s["max_k"] == 7
    assert s["q_start"].tolist() == [0, 4, 4, 11] and s["k_start"].tolist() == [0, 10, 20] and s["k_len"].tolist() == [4, 0, 7]
    assert s["pos"].tolist() == [0, 1, 2, 3, 0, 1, 2, 3, 4, 5, 6]
    assert s["slots"].tolist() == [0, 1, 2, 3, 20, 21, 22, 23, 24, 25, 26]
    s = c.extend([1, 1, 1])
    assert s["pos"].tolist() == [4, 0, 7] and s["slots"].tolist() == [4, 10, 27] and s["k_len"].tolist() == [5, 1, 8]
    assert all(s[n].dtype == torch.int32 for n in ("q_start", "k_start", "k_len", "pos", "slots"))
    before = list(c.lens)
    for bad in ([6, 0, 0], [0, 0], [-1, 0, 0]):
        with pytest.raises(ValueError):
            c.extend(bad)
    assert c.lens == before
