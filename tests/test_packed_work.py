"""The workspace that attention of packed sequences asks for (attention_packed_work of csrc/attn_packed.cu and
bag_attention_work, compiled for the host): with it every call up to the sizes it was told for is cut as with memory
without end, the steps of a text layer among them."""

import os
import random
import re

import pytest

import source_parts
import test_packed_plan as plan

INCLUDE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")


def program():
    api = open(source_parts.CSRC + "/bag_api.cu").read()
    limits = "\n".join(re.search(rf"^(static )?constexpr (long|int) {n} = [^;]*;", api, re.M).group(0) for n in ("kMaxRows", "kMaxHeads"))
    parts = plan.program().split("int main()")[0]
    return f"""
#include "{INCLUDE}/bag.h"
{parts}
{source_parts.part("attn_packed.cu", "size_t attention_packed_work(const PackedArgs& a)")}
{limits}
static bag_status fail(bag_ctx*, bag_status s, const char*) {{ return s; }}
#define CKS(x) do {{ const bag_status st = (x); if (st != BAG_OK) return st; }} while (0)
{source_parts.part("bag_api.cu", "static bag_status check_packed(")}
{source_parts.part("bag_api.cu", "static bag_status bag_attention_work_impl(")}
// a call's own sizes, with 0 for what it does not know: as bag_attention_packed_impl takes them
static PackedArgs call(long nq, long k_rows, long n_prefix, long seqs, long max_q, long max_k, int heads, int kv_heads, int dh) {{
  PackedArgs g{{}};
  g.nq = nq, g.k_rows = k_rows, g.n_prefix = n_prefix, g.seqs = seqs, g.heads = heads, g.kv_heads = kv_heads, g.dh = dh;
  g.max_q = max_q ? std::min(max_q, nq) : nq;
  g.max_k = max_k ? std::min(max_k, kMaxRows) : k_rows;
  return g;
}}
int main() {{
  long sms, nq, n_prefix, seqs, max_q, max_k, c[6];
  int heads, kv_heads, dh;
  while (scanf("%ld %d %d %d %ld %ld %ld %ld %ld %ld %ld %ld %ld %ld %ld", &sms, &heads, &kv_heads, &dh, &nq, &n_prefix, &seqs, &max_q,
               &max_k, c, c + 1, c + 2, c + 3, c + 4, c + 5) == 15) {{
    g_sms = sms;
    size_t told = 0;
    if (bag_attention_work_impl(nullptr, nq, heads, kv_heads, dh, seqs, max_q, max_k, n_prefix, &told) != BAG_OK) return 1;
    const PackedArgs a = call(c[0], c[1], c[2], c[3], c[4], c[5], heads, kv_heads, dh);
    const Plan t = plan_of(a, told), w = plan_of(a, ~(size_t)0 >> 1);
    const bool same = t.parts1 == w.parts1 && t.parts2 == w.parts2 && t.chunk1 == w.chunk1 && t.chunk2 == w.chunk2 && t.few == w.few &&
                      t.split == w.split && t.ctas == w.ctas && t.fused == w.fused && t.rows == w.rows && t.together == w.together;
    printf("%d %zu %zu %d %d\\n", same, told, parts_of(w) * part_bytes(a) + piece_bytes(a, w), w.parts1, w.parts2);
  }}
}}
"""


def run(tmp_path, cases):
    out = source_parts.run(program(), tmp_path, "\n".join(" ".join(map(str, c)) for c in cases))
    lines = [tuple(map(int, line.split())) for line in out.splitlines()]
    assert len(lines) == len(cases)
    return lines


def test_calls_up_to_the_told_sizes(tmp_path):
    r = random.Random(3)
    log = lambda lo, hi: int(round(lo * (hi / lo) ** r.random()))  # noqa: E731
    cases = []
    for _ in range(3000):
        kv = r.choice([1, 2, 4, 5, 8, 40])
        head = (r.choice([152, 152, 148, 20]), kv * r.choice([1, 2, 4, 5, 7, 8, 13, 28, 130]), kv, r.choice([64, 128]))
        seqs, nq = log(1, 3000), log(1, 100000)
        prefix = r.choice([0, log(1, 200000)])
        max_q, max_k = r.choice([0, 1, log(1, nq + 1)]), r.choice([0, log(1, 10 ** 6)])
        for _ in range(20):
            s = r.choice([seqs, log(1, seqs)])
            q = r.choice([0, log(1, max_q)]) if max_q and max_q >= nq else (log(1, max_q) if max_q else r.choice([0, log(1, nq)]))
            n = min(nq, log(1, nq), s * q if q else nq)
            k = log(1, max_k) if max_k else r.choice([0, log(1, 10 ** 6)])
            p = r.choice([0, prefix, log(1, prefix)]) if prefix else 0
            cases.append(head + (nq, prefix, seqs, max_q, max_k, n, log(1, 10 ** 7), p, s, q, k))
    cut = 0
    for c, (same, told, need, p1, p2) in zip(cases, run(tmp_path, cases)):
        assert same and need <= told, (c, told, need)
        cut += need > 0
    assert cut > 10000


LAYERS = [  # sequences, room, rows, prefix, heads, key heads
    (8, 32768, 4096, 0, 32, 8), (1, 131072, 4096, 0, 28, 4), (1, 32768, 4096, 1024, 28, 4), (32, 320, 8192, 1024, 32, 8),
    (64, 8192, 512, 5000, 40, 40), (3, 400, 600, 130, 4, 2),
]


@pytest.mark.parametrize("layer", LAYERS)
@pytest.mark.parametrize("dh", [64, 128])
def test_steps_of_a_layer(layer, dh, tmp_path):
    """Every step of a layer, from one token to all of its rows, in one text or spread over all, early and late in the
    texts; and the prefix itself."""
    texts, room, rows, prefix, heads, kv = layer
    head = (152, heads, kv, dh)
    limits = (rows, prefix, texts, min(rows, room), room)
    cases = []
    for n in sorted({*range(1, 130), *range(130, rows, 37), rows}):
        for q in {min(n, room), -(-n // texts)}:
            for k in {q, min(room, q + room // 2), room}:
                if n <= texts * q and q <= room:
                    cases.append(head + limits + (n, texts * room, prefix, texts, q, k))
    parts = set()
    for c, (same, told, need, p1, p2) in zip(cases, run(tmp_path, cases)):
        assert same and need <= told, (c, told, need)
        parts.add((p1, p2))
    assert len(parts) > 1 or room < 2000


@pytest.mark.parametrize("heads,kv,dh,seqs,max_q,rows", [(28, 4, 128, 1, 1, 131072), (28, 4, 128, 1, 64, 600000), (8, 8, 64, 30, 1, 9000)])
def test_keys_that_nobody_knows(heads, kv, dh, seqs, max_q, rows, tmp_path):
    """Without max_k a call goes by the cache's rows, and so has the size to."""
    n = seqs * max_q
    (same, told, need, _, p2), = run(tmp_path, [(152, heads, kv, dh, n, 0, seqs, max_q, 0, n, rows, 0, seqs, max_q, 0)])
    assert same and told >= need > 0


def test_nothing_where_no_call_shares(tmp_path):
    """Short sequences want no workspace, and sizes are of an order that a program has beside its cache."""
    (_, told, _, _, _), = run(tmp_path, [(152, 12, 12, 64, 84, 0, 2, 77, 77, 84, 84, 0, 2, 77, 77)])
    assert told == 0
    for layer in LAYERS:
        texts, room, rows, prefix, heads, kv = layer
        (_, told, _, _, _), = run(tmp_path, [(152, heads, kv, 128, rows, prefix, texts, rows, room, 1, 1, 0, 1, 1, 1)])
        assert told < 250e6, (layer, told)


def test_sizes_that_no_memory_holds(tmp_path):
    """The largest sizes that are accepted: the size told is that of the formula, whatever it is."""
    rows, kv = 0x7fffff00, 65535
    cases = [(152, kv, kv, 128, rows, p, rows, q, 0, 1, 1, 0, 1, 1, 1) for p in (0, rows) for q in (0, 1, 1000)]
    for c, (_, told, _, _, _) in zip(cases, run(tmp_path, cases)):
        cap, few = 13 * 152 * 256 // 3, 304 * 2 * 16 * 520 + (rows + 1) * 8
        if c[5] == 0:
            assert told == (0 if c[7] == 1 else cap * 520) + few
        else:
            assert told >= 2 * rows * kv * 520 + few and told < 2 ** 62
