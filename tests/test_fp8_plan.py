"""The 8-bit product's choice of kernel, tile and split (plan_fp8, compiled for the host) at 152 SMs."""

import itertools

import pytest

import source_parts
from fp8_shapes import FORMS, LONG

KINDS = {"f32": 0, "bf16": 1, "fp8": 2, "resid": 3}
LIMIT = {"f32": 32, "bf16": 64, "fp8": 20, "resid": 32}  # K blocks of one sum on the tensor core

CODE = """
#include <algorithm>
#include <cmath>
#include <cstdio>
#define __host__
#define __device__
enum { BAG_FP8_F32 = 0, BAG_FP8_BF16 = 1, BAG_FP8_CODES = 2, BAG_FP8_RESID = 3 };
static int sm_count() { return 152; }
constexpr int F8_BK = 128, F8_GROUP = 4;
"""

MAIN = """
// for each shape: rows of a tile, CTAs that share K, K blocks of the longest part, and the K blocks of
// the longest of the sums that the tensor core takes at once
int main() {
  long M, N, K;
  int kind;
  while (std::scanf("%ld %ld %ld %d", &M, &N, &K, &kind) == 4) {
    const Fp8Plan p = plan_fp8(M, N, K, kind);
    const int nkb = (int)((K + F8_BK - 1) / F8_BK), S = 1 << p.logS, most = pass_blocks(kind);
    int sum = 0, part = nkb;
    if (p.BN) {
      part = few_longest(S, nkb);
      for (int r = 0; r < S; ++r) {
        const int kb0 = few_cut(r, S, nkb), kb1 = few_cut(r + 1, S, nkb), kg0 = kb0 & ~(F8_GROUP - 1);
        if (kb1 <= kb0) return 1;  // a CTA without work
        const int step = part > most ? pass_length(kb1 - kg0, most) : kb1 - kg0;
        for (int kg = kg0; kg < kb1; kg += step) sum = std::max(sum, std::min(kb1, kg + step) - std::max(kb0, kg));
      }
    } else {
      sum = nkb > most ? pass_length(nkb, most) : nkb;
    }
    std::printf("%d %d %d %d\\n", p.BN, S, part, sum);
  }
}
"""

PARTS = ["static long cluster_sms(int logS) {", "__host__ __device__ constexpr int pass_blocks(int kind) {",
         "__host__ __device__ constexpr int pass_length(int n, int most) {",
         "__host__ __device__ constexpr int few_cut(int r, int S, int nkb) {", "static int few_longest(int S, int nkb) {",
         "static long whole_tiles(", "struct Fp8Plan {", "static Fp8Plan plan_fp8("]


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    code = CODE + "\n".join(source_parts.part("gemm_fp8.cu", p) for p in PARTS) + MAIN
    path = tmp_path_factory.mktemp("fp8_plan")

    def ask(shapes):
        text = "".join("%d %d %d %d\n" % s for s in shapes)
        out = [int(v) for v in source_parts.run(code, path, text=text).split()]
        assert len(out) == 4 * len(shapes)
        return [tuple(out[i:i + 4]) for i in range(0, len(out), 4)]

    return ask


@pytest.mark.parametrize("kind", KINDS)
def test_shapes_of_the_tests_reach_every_form(kind, plan):
    got = plan([s + (KINDS[kind],) for s in FORMS.values()])
    assert {g[:2]: s for g, s in zip(got, FORMS.values())} == FORMS
    got = plan([s + (KINDS[kind],) for s in LONG.values()])
    assert {g[:2]: s for g, s in zip(got, LONG.values())} == LONG and all(g[2] > LIMIT[kind] for g in got)


@pytest.mark.parametrize("kind", KINDS)
def test_no_sum_on_the_tensor_core_is_longer_than_its_limit(kind, plan):
    M = (1, 2, 9, 16, 17, 33, 77, 128, 200, 400, 1000, 2048, 4608)
    N = (1, 128, 300, 1536, 5120, 13824, 27648)
    K = [128 * b for b in (*range(1, 180, 3), 224, 225, 416, 512, 1021, 2048, 16384)]
    shapes = [s + (KINDS[kind],) for s in itertools.product(M, N, K)]
    for s, (rows, ctas, part, longest) in zip(shapes, plan(shapes)):
        assert longest <= LIMIT[kind], (s, rows, ctas, part, longest)
