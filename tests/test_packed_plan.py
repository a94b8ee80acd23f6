"""How attention of packed sequences is cut into parts (plan_of of csrc/attn_packed.cu, compiled for the host): over
many sizes and workspaces, that what it keeps fits the workspace, that parts cover all keys, and that a
bound of the workspace's size is one."""

import random
import re

import pytest

import source_parts

FIELDS = ("parts1", "parts2", "chunk1", "chunk2", "few", "split", "ctas", "fused", "rows", "together", "need", "work")


def program():
    src = open(source_parts.CSRC + "/attn_packed.cu").read()
    consts = "\n".join(re.search(rf"^constexpr int {n} = [^;]*;", src, re.M).group(0)
                       for n in ("F_KEYS", "F_ROWS", "PT"))
    consts = consts.replace("constexpr int F_ROWS", "constexpr int F_WARPS = 4, F_TILE = F_WARPS * F_KEYS;\nconstexpr int F_ROWS")
    assert re.search(r"F_WARPS = 4,", src)
    return f"""
#include <algorithm>
#include <cstddef>
#include <cstdint>
#include <cstdio>
{consts}
template <int DH>
{source_parts.part("attn_packed.cu", "constexpr int few_ctas()")}
static long g_sms = 152;
static long sm_count() {{ return g_sms; }}
struct PackedArgs {{ long nq, k_rows, n_prefix, seqs, max_q, max_k; int heads, kv_heads, dh; }};
{source_parts.part("attn_packed.cu", "struct Plan {")}
{source_parts.part("attn_packed.cu", "long cdiv(long a, long b)")}
{source_parts.part("attn_packed.cu", "size_t part_bytes(const PackedArgs& a)")}
{source_parts.part("attn_packed.cu", "size_t piece_bytes(const PackedArgs& a, const Plan& t)")}
{source_parts.part("attn_packed.cu", "long parts_of(const Plan& t)")}
{source_parts.part("attn_packed.cu", "Plan plan_of(const PackedArgs& a, size_t bytes)")}
int main() {{
  PackedArgs a;
  size_t bytes;
  while (scanf("%ld %ld %ld %ld %ld %ld %d %d %d %zu", &a.nq, &a.k_rows, &a.n_prefix, &a.seqs, &a.max_q, &a.max_k, &a.heads,
               &a.kv_heads, &a.dh, &bytes) == 10) {{
    const Plan t = plan_of(a, bytes), w = plan_of(a, ~(size_t)0 >> 1);
    printf("%d %d %d %d %d %d %d %d %d %d %zu %zu\\n", t.parts1, t.parts2, t.chunk1, t.chunk2, t.few, t.split, t.ctas, t.fused,
           t.rows, t.together, parts_of(t) * part_bytes(a) + piece_bytes(a, t), parts_of(w) * part_bytes(a) + piece_bytes(a, w));
  }}
}}
"""


def cases():
    r = random.Random(0)
    log = lambda lo, hi: int(round(lo * (hi / lo) ** r.random()))  # noqa: E731
    out = []
    for _ in range(4000):
        kv = r.choice([1, 2, 3, 8, 40])
        g = r.choice([1, 2, 4, 5, 7, 8, 13, 28, 40, 128, 131])
        seqs = log(1, 3000)
        nq = r.choice([seqs, log(1, 200000)])
        k_rows = r.choice([0, log(1, 10 ** 7)])
        prefix = r.choice([0, 0, log(1, 200000)])
        max_q, max_k = log(1, nq + 1), log(1, 10 ** 6)
        bytes_ = r.choice([0, 16, log(100, 10 ** 6), log(10 ** 5, 10 ** 11), 2 ** 62])
        out.append((nq, k_rows, prefix, seqs, max_q, max_k, kv * g, kv, r.choice([64, 128]), bytes_))
    return out


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    cs = cases()
    text = source_parts.run(program(), tmp_path_factory.mktemp("plan"), "\n".join(" ".join(map(str, c)) for c in cs))
    return list(zip(cs, (dict(zip(FIELDS, map(int, line.split()))) for line in text.splitlines())))


def test_plans(plans):
    kinds = set()
    assert len(plans) == 4000
    for (nq, k_rows, prefix, seqs, max_q, max_k, heads, kv, dh, bytes_), t in plans:
        G = heads // kv
        assert t["need"] <= bytes_                       # what is kept fits
        assert t["chunk1"] > 0 and t["chunk1"] % 128 == 0 and t["chunk2"] > 0 and t["chunk2"] % 128 == 0
        assert t["parts2"] >= 1 and t["rows"] in (128, 256) and G % t["together"] == 0 and t["together"] <= 128
        assert 128 // t["together"] * t["together"] >= 64   # a tile has some rows
        if prefix:                                       # the prefix is met in exactly one way
            assert (t["parts1"] > 0) != (t["fused"] > 0)
            if t["parts1"]:
                assert t["parts1"] * t["chunk1"] >= prefix > (t["parts1"] - 1) * t["chunk1"]
                assert t["need"] > 0
            else:
                assert t["fused"] * 128 >= prefix > (t["fused"] - 1) * 128
        else:
            assert t["parts1"] == 0 and t["fused"] == 0
        if t["few"]:
            assert t["fused"] == 0 and t["ctas"] >= 1 and max_q * G <= 16 or nq * G <= 16
        if t["split"]:
            assert t["few"] and t["need"] > 0
        kinds.add((bool(t["few"]), bool(t["split"]), t["parts1"] > 0, t["fused"] > 0, t["parts2"] > 1, t["rows"]))
    assert len(kinds) >= 12


def test_a_workspace_of_the_told_size_serves_fewer_keys(plans, tmp_path):
    """The size is told for any number of rows of k; a call with fewer rows may not need more."""
    cs = [c[:1] + (0x7fffff00,) + c[2:9] + (2 ** 62,) for c, _ in plans]
    told = [int(line.split()[-1]) for line in
            source_parts.run(program(), tmp_path, "\n".join(" ".join(map(str, c)) for c in cs)).splitlines()]
    for (c, t), size in zip(plans, told):
        assert t["work"] <= size, c
