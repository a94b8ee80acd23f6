"""The restatements that the low-precision GPU tests compare with, against torch's own conversions
and closed forms (CPU)."""

import numpy as np
import torch

import lowbit_ref as R


def test_e4m3_values_and_rounding_are_torchs():
    codes = torch.arange(256, dtype=torch.uint8)
    assert np.array_equal(codes.view(torch.float8_e4m3fn).float().numpy(), R.E4M3.astype(np.float32), equal_nan=True)
    x = torch.cat([torch.randn(4000), torch.randn(4000) * 100, torch.randn(2000) * 2.0 ** -8]).clamp(-448, 448)
    mid = torch.from_numpy((R.E4M3[:126] + R.E4M3[1:127]) / 2).float()  # ties
    x = torch.cat([x, mid, -mid])
    want = x.to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(R.e4m3_code(x.numpy().astype(np.float64)), want)


def test_scale_is_the_least_that_fits():
    x = np.zeros((4, 128), np.float32)
    x[0, 0], x[1, 0], x[2, 0] = 448.0, np.nextafter(np.float32(448), np.float32(500)), 1.75
    codes, scales = R.quant(x)
    assert list(scales[:, 0]) == [127, 128, 119, 0]
    assert R.decode(codes, scales)[0, 0] == 448.0 and R.decode(codes, scales)[2, 0] == 1.75


def test_bf16_rounding_is_torchs():
    x = np.random.default_rng(0).standard_normal(1000).astype(np.float32)
    assert np.array_equal(R.bf16(x), torch.from_numpy(x).bfloat16().float().numpy())


def test_selection_takes_the_lower_index_of_equal_scores():
    k = np.ones((1, 5, 128), np.int8)
    s = np.array([[1.0, 2.0, 1.0, 2.0, 1.0]], np.float32)
    assert R.select(np.ones((1, 1, 128), np.int8), k, s, 3).tolist() == [[[0, 1, 3]]]


def test_pooled_mean_of_a_short_block():
    x = np.zeros((130, 128), np.float32)
    x[128:] = 3.0
    x[:128, 0] = 1.0
    codes, scales = R.pool(x, 1)
    assert codes[0, 0, 0] == 127 and (codes[0, 0, 1:] == 0).all() and (codes[0, 1] == 127).all()
    assert scales[0, 1] == np.float32(3.0) * (np.float32(1) / np.float32(127))
