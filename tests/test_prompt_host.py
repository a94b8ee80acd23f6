"""Rotary positions and attention of packed sequences without a GPU: a null context, arguments that the
binding refuses, and the host's own arithmetic (compiled from its source)."""

import ctypes
from fractions import Fraction

import numpy as np
import pytest
import torch

import source_parts
from paper_2608_09231_gb300 import bag


@pytest.fixture(scope="module")
def lib():
    from paper_2608_09231_gb300 import build
    build.build()
    return bag.load()


def test_null_context(lib):
    assert lib.bag_rope(None, None) == 1
    assert lib.bag_attention_packed(None, None) == 1
    assert lib.bag_attention_prefix(None, None, None, 0, None, 0, 0) == 1
    assert lib.bag_attention_work(None, 1, 1, 1, 128, 1, 1, 1, 0, None) == 1


def test_structures_match_the_header(tmp_path):
    """Offsets of every field, as the C compiler lays them out."""
    import os
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    code = f'#include "{include}/bag.h"\n#include <cstdio>\n#include <cstddef>\nint main() {{\n'
    want = []
    for name, cls in (("bag_rope_args", bag.RopeArgs), ("bag_packed_args", bag.PackedArgs)):
        for f, _ in cls._fields_:
            code += f'  printf("%zu\\n", offsetof({name}, {f}));\n'
            want.append(getattr(cls, f).offset)
        code += f'  printf("%zu\\n", sizeof({name}));\n'
        want.append(ctypes.sizeof(cls))
    assert [int(x) for x in source_parts.run(code + "}\n", tmp_path).split()] == want


def test_packed_bytes_are_the_structures():
    """The bytes handed to the library hold every field where the structure has it."""
    for cls, pack in ((bag.RopeArgs, bag._pack_rope), (bag.PackedArgs, bag._pack_packed)):
        values = [i + 1 for i in range(len(cls._fields_))]
        got = cls.from_buffer_copy(pack(*values))
        assert [getattr(got, f) for f, _ in cls._fields_] == values


def test_host_tensors_are_refused():
    ctx = bag.Context.__new__(bag.Context)  # refused before the library is reached
    x = torch.zeros(3, 128)
    with pytest.raises(ValueError, match="device matrix"):
        ctx.rope(x, x, [1.0], 128)
    h = x.half()
    with pytest.raises(ValueError, match="device matrix"):
        ctx.attention_packed(h, h, h, h, torch.zeros(2, dtype=torch.int32), 1)
    with pytest.raises(ValueError, match="none of"):
        ctx.rope(x, x, [1.0], 128, layout="quarter")
    with pytest.raises(ValueError, match="needs q, k or v"):
        ctx.rope(None, None, [1.0], 128)


# 1 / (2 pi) to 70 digits
TURN = Fraction("0.1591549430918953357688837633725143620344596457404564487476673440588967")


def test_turns_of_a_frequency(tmp_path):
    """A frequency as a 64-bit fraction of a turn: within a unit of the exact one (half of it the rounding to
    a whole number; the two parts of 1 / 2 pi are good to 2^-110, 2^-16 units at 2^30)."""
    rng = np.random.default_rng(0)
    freqs = [0.0, 1.0, -1.0, 0.5, 1e-8, 2.0 ** -60, 3.0, 2.0 ** 30, -(2.0 ** 29), 6.283185307179586]
    freqs += list(10000.0 ** -rng.uniform(0, 1, 200)) + list(rng.uniform(-1000, 1000, 50))
    code = "#include <cmath>\n#include <cstdint>\n#include <cstdio>\n" + source_parts.part("bag_api.cu", "static uint64_t turn_fraction(") + \
        '\nint main() { double f; while (scanf("%lf", &f) == 1) printf("%llu\\n", (unsigned long long)turn_fraction(f)); }\n'
    got = source_parts.run(code, tmp_path, "\n".join(repr(float(f)) for f in freqs)).split()
    assert len(got) == len(freqs)
    for f, g in zip(freqs, got):
        exact = Fraction(float(f)) * TURN
        off = (Fraction(int(g), 1 << 64) - exact) % 1
        off = min(off, 1 - off) * (1 << 64)
        assert off <= 1, (f, float(off))


def test_shared_memory_of_two_matrices(tmp_path):
    """Never says apart of two matrices that share a byte; and says apart of plain columns side by side, of
    ranges that do not meet and of empty ones."""
    code = "#include <cstdint>\n#include <cstdio>\n" + source_parts.part("bag_api.cu", "static bool share(") + """
int main() {
  long a, la, ra, wa, b, lb, rb, wb;
  while (scanf("%ld %ld %ld %ld %ld %ld %ld %ld", &a, &la, &ra, &wa, &b, &lb, &rb, &wb) == 8)
    printf("%d\\n", share((void*)(1000 + a), la, ra, wa, (void*)(1000 + b), lb, rb, wb));
}
"""
    rng = np.random.default_rng(1)
    cases = [(0, 16, 4, 8, 8, 16, 4, 8), (0, 16, 4, 8, 7, 16, 4, 8), (0, 16, 4, 8, 64, 16, 4, 8), (0, 16, 0, 8, 0, 16, 4, 8),
             (8, 16, 4, 8, 0, 16, 4, 8), (8, 16, 4, 8, 16, 16, 9, 8), (0, 16, 4, 16, 0, 16, 4, 16)]
    for _ in range(3000):
        la = int(rng.integers(4, 20))
        lb = la if rng.random() < 0.7 else int(rng.integers(4, 20))
        cases.append((int(rng.integers(0, 60)), la, int(rng.integers(0, 5)), int(rng.integers(1, la + 1)),
                      int(rng.integers(0, 60)), lb, int(rng.integers(0, 5)), int(rng.integers(1, lb + 1))))
    got = source_parts.run(code, tmp_path, "\n".join(" ".join(map(str, c)) for c in cases)).split()
    apart = 0
    for c, g in zip(cases, got):
        a, la, ra, wa, b, lb, rb, wb = c
        one = {a + r * la + i for r in range(ra) for i in range(wa)}
        two = {b + r * lb + i for r in range(rb) for i in range(wb)}
        if one & two:
            assert g == "1", c
        elif la == lb or not one or not two:
            apart += g == "0"
            assert g == "0" or (one and two and not (max(one) < min(two) or max(two) < min(one))), c
    assert apart > 300 and got[:7] == ["0", "1", "0", "0", "0", "0", "1"]
