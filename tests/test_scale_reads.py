"""Which bytes the 8-bit product reads of an operand's scales: ScaleRun::fetch, compiled for the host
with loads that are written down.  Every aligned load holds a scale byte of the operand's own K blocks
(so none can leave the operand's memory), and the words of all of them are fetched."""

import pytest

import source_parts

SHIM = """
#include <cstdint>
#include <cstdio>
#include <set>
#define BAG_DEV inline
#define __restrict__
struct uint4 { uint32_t x, y, z, w; };
static uint4 make_uint4(uint32_t x, uint32_t y, uint32_t z, uint32_t w) { return uint4{x, y, z, w}; }
static struct { unsigned x; } threadIdx;
static const uint8_t* memory;
static std::set<std::pair<long, int>> loads;  // (offset, bytes)
static uint4 __ldg(const uint4* p) { loads.insert({(const uint8_t*)p - memory, 16}); return uint4{1, 1, 1, 1}; }
static uint32_t __ldg(const uint32_t* p) { loads.insert({(const uint8_t*)p - memory, 4}); return 1; }
"""

MAIN = """
int main() {
  alignas(16) static uint8_t buffer[1 << 16];
  memory = buffer;
  // rows of nkb scale bytes from byte `first` on, in rows of lds
  const struct { int lds, first, nkb, rows; } cases[] = {
    {16, 4, 4, 5}, {16, 4, 1, 1}, {16, 8, 5, 3}, {16, 12, 3, 128}, {20, 0, 20, 40}, {20, 4, 13, 33}, {64, 4, 17, 7},
    {64, 36, 28, 2}, {108, 0, 108, 3}, {112, 4, 107, 3}, {4, 0, 1, 1}, {48, 20, 20, 130}};
  int bad = 0;
  for (const auto& c : cases) {
    for (int row0 : {0, 128}) {
      loads.clear();
      const uint8_t* s = buffer + c.first;
      std::set<long> held;
      for (int run = 0; run * 16 < c.nkb; ++run)
        for (threadIdx.x = 0; threadIdx.x < 32; ++threadIdx.x) {
          ScaleRun r;
          r.fetch(s, c.lds, false, row0, c.rows, run, c.nkb);
        }
      for (const auto& l : loads) {
        bool own = false;
        for (long b = l.first; b < l.first + l.second; ++b) {
          const long at = b - c.first, row = at / c.lds, col = at % c.lds;
          held.insert(b);
          own |= at >= 0 && row >= row0 && row < c.rows && col < c.nkb;
        }
        bad += !own || l.first % l.second;
      }
      for (int row = row0; row < c.rows && row < row0 + 128; ++row)
        for (int b = 0; b < c.nkb; ++b) bad += !held.count((long)c.first + (long)row * c.lds + b);
      if (bad) {
        std::printf("lds %d first %d blocks %d rows %d from %d: %d\\n", c.lds, c.first, c.nkb, c.rows, row0, bad);
        return 0;
      }
    }
  }
  std::puts("ok");
}
"""


@pytest.fixture(scope="module")
def result(tmp_path_factory):
    code = SHIM + source_parts.part("gemm_fp8.cu", "struct ScaleRun {") + MAIN
    return source_parts.run(code, tmp_path_factory.mktemp("scale_reads"))


def test_loads_stay_in_the_operand(result):
    assert result == "ok\n"
