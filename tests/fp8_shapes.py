"""Shapes of the 8-bit product that reach its few-row kernel's passes: (M, N, K) by (rows of a tile,
CTAs that share K).  test_fp8_plan.py holds them against the library's rule on the
CPU, test_gpu_fp8_sums.py runs them."""

# sums longer than a pass in a CTA's part of K
LONG = {
    (16, 8): (3, 5000, 70000), (32, 8): (17, 500, 69000), (64, 8): (64, 300, 70016), (128, 8): (250, 500, 68000),
}
