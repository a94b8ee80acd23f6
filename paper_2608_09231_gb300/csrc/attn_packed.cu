// Attention of packed sequences over their own rows of a key-value cache, behind a prefix that all of
// them share (heads of 64 or 128, 16-bit operands, grouped heads).
//
//   o_t = sum_j w_tj v_j / sum_j w_tj,  w_tj = exp(c q_t . k_j),
//
// over the prefix's keys and the own keys j <= t + lk - lq.  Sums over parts of the keys are kept as
// (m, l, O) with l = sum 2^(s - m), O = sum 2^(s - m) v, s in log2 units; parts are joined by
// m = max m_i, l = sum 2^(m_i - m) l_i, O likewise.  l = 0: no key is seen; l = 1 with m of minus infinity: keys are
// seen, but all scores are minus infinity, which weighs nothing beside other parts and makes a row without them NaN.
//
// A sequence's rows of a key head are its query tokens times the heads that share it.  At most 16 of them: the
// keys are what there is to read, and attn_few_kernel streams them.  More: attn_packed_kernel, on the tensor
// cores.  A prefix that all sequences share is met by the rows of all of them together, where they have few each,
// or goes ahead of each sequence's own keys.  attn_join_* add up where keys were cut.
#include <algorithm>

#include "attn_common.cuh"
#include "kernels.h"

namespace bag {

namespace {
struct PackedParams {
  const uint16_t *q, *k, *v, *pk, *pv;
  uint16_t* o;
  long ldq, ldk, ldv, ldpk, ldpv, ldo;
  float* lse;
  const int *q_start, *k_start, *k_len;
  int nq, k_rows, n_prefix, seqs;
  int heads, kv_heads, group, causal;
  float scale_log2;
  // The prefix is met by the rows of all sequences together (parts1 parts of chunk1 keys, whose sums are joined
  // with those over own keys), or comes before each sequence's own keys (fused key tiles; then parts1 = 0).
  // own_parts() parts of a sequence, chunk2 keys (those of the fused tiles among them) each.
  // Part i of row t and head h: part_o[((i * nq + t) * heads + h) * dh ...], part_ml likewise.
  int parts1, parts2, chunk1, chunk2;
  int fused;
  float* part_o;
  float2* part_ml;
  // tensor-core kernel: a tile's rows are `tokens` query tokens x `together` heads of a group; units over the
  // tokens of all sequences and of each
  int together, tokens, slots1, slots2;
  int by_head;  // order of the units: a head after the other, or all heads of a slot
  int beside;   // the kernel before is attn_few_kernel of the same call, which it has nothing to wait for from
  int* err;
  // few-row kernel: whether a unit's keys may be shared among CTAs, their sums (see attn_few_kernel)
  int few, split;
  float* piece_o;      // [CTA][2][16][dh]
  float2* piece_ml;    // [CTA][2][16]
  long* place;         // [0]: tiles of a CTA, [1 + sequence]: its first tile
};

// A sequence's rows of q and of k and v, clipped to the tensors' own.
struct Span {
  int q0, lq, k0, lk;
};
BAG_DEV Span span_of(const PackedParams& p, int i) {
  Span s;
  s.q0 = min(max(__ldg(p.q_start + i), 0), p.nq);
  s.lq = min(max(__ldg(p.q_start + i + 1), s.q0), p.nq) - s.q0;
  s.k0 = p.k_start ? min(max(__ldg(p.k_start + i), 0), p.k_rows) : s.q0;
  s.lk = p.k_start ? min(max(__ldg(p.k_len + i), 0), p.k_rows - s.k0) : s.lq;
  return s;
}
// All sequences' rows of q.
BAG_DEV Span span_all(const PackedParams& p) {
  Span s;
  s.q0 = min(max(__ldg(p.q_start), 0), p.nq);
  s.lq = min(max(__ldg(p.q_start + p.seqs), s.q0), p.nq) - s.q0;
  s.k0 = 0;
  s.lk = p.n_prefix;
  return s;
}
// Parts that hold a sequence's own keys; the last of parts2 takes all that the others leave (their sizes
// come from the caller's estimate of the longest sequence).
BAG_DEV int own_parts(const PackedParams& p, int lk) {
  return (int)min(((long)p.fused * 128 + lk + p.chunk2 - 1) / p.chunk2, (long)p.parts2);
}

// 2^(m - top) of a part with (m, l) where the parts' largest maximum is top, and what a row's joined sums are
// multiplied by: zero where no key is seen, NaN where there are only scores of minus infinity.
BAG_DEV float part_weight(float2 ml, float top) { return ml.y == 0.f ? 0.f : (ml.x == top ? 1.f : ex2(ml.x - top)); }
BAG_DEV float inverse_sum(float top, float l) {
  return l == 0.f ? 0.f : (top == -INFINITY ? __int_as_float(0x7fffffff) : 1.f / l);
}

// fp16 weights: m is kept this much below the largest score, so that a row's largest weight is 2^7 to 2^15 (65504 is
// the type's end) and weights keep all their bits down to 2^-21 of it, and some down to 2^-32; with the largest at 1,
// many keys of weights below 2^-25 would vanish from O and stay in l.  bf16 has the range of fp32.
template <bool F16>
constexpr float kWeightsUp = F16 ? 7.f : 0.f;

template <bool F16>
BAG_DEV uint32_t pack16(float a, float b) {
  return F16 ? pack_f16x2(a, b) : pack_bf16x2(a, b);
}

template <bool F16>
BAG_DEV void mma16816(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (F16)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// 16 bytes that are read once
BAG_DEV uint4 ld_stream(const uint16_t* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}

constexpr int F_WARPS = 4, F_TH = 32 * F_WARPS;
template <int DH>
constexpr int few_ctas() { return (DH == 64 ? 16 : 8) / F_WARPS; }  // on an SM
constexpr int F_KEYS = 16;               // of a warp's step
constexpr int F_TILE = F_WARPS * F_KEYS;  // of the CTA's
constexpr int F_ROWS = 16;               // query rows of a unit
template <int DH>
constexpr int few_smem() {
  return F_WARPS * F_ROWS * (DH + 4) * 4 + F_WARPS * F_ROWS * 8;
}

// Units of a sequence (16 rows, a key head), and the length of one where they lie in a row: its key tiles, and
// F_COST for what a unit costs besides them.
BAG_DEV long few_units(const PackedParams& p, int lq) { return (long)((lq * p.group + F_ROWS - 1) / F_ROWS) * p.kv_heads; }
constexpr int F_COST = 1;
BAG_DEV int few_length(int lk) { return (lk + F_TILE - 1) / F_TILE + F_COST; }
}  // namespace

// Up to 16 rows (query token, head of the group) of a sequence and key head, a unit, against keys in registers: a
// warp takes 16 keys a step.  A key's 16-byte pieces go from global memory straight into the B operands of
// mma.m16n8k16: the order of a contraction is free, so lane (n, c) holds head columns 32 j + 8 c .. + 7 of
// key n for Q K^T (the rows of Q are loaded in the same order), and columns 64 u + 8 n .. + 7 of keys 2 c,
// 2 c + 1, 2 c + 8 and 2 c + 9 for P V, whose pairs of keys a byte permutation makes; its column n of
// product t is then head column 64 u + 8 n + t, and a lane ends with runs of 8 columns of the output.
// Keys past the last are loaded as zeros (whatever lies there, NaN included).
// Units lie in a row, of which each CTA takes an equal share, and finds the next one from the last.  Split: their key
// tiles do, so that lengths need not be alike and one wave of CTAs does it all; every CTA adds the lengths up
// for itself.  A unit that lies in one CTA's share is finished there; of the others a CTA holds at most two
// pieces, one that starts its unit (piece 1) and one that does not (piece 0), which attn_join_kernel adds up.
// The next unit's first loads are in flight while the warps' sums are joined.
// Bound: HBM.  64 tokens over 512 to 32,767 keys each (32 heads, 8 key heads, 2.3 GB) 360 us, 6.4 TB/s or 95 % of the
// copy rate (a grid of sequences, heads and parts of up to 8192 keys: 392 to 546); one token over 131,071
// keys 51 us (floor 40, the rest a launch's start and the join).  Few keys a unit: latency, a unit's loads, the join
// of its warps; 128 tokens over 10 to 400 keys 20 us, floor 8.  Four warps a CTA and two CTAs on an SM
// instead of eight and one: 376 -> 363 us, 128 tokens over short own keys 85 -> 65.  bf16 weights enter P V in
// two parts, whose rounding would otherwise be the largest error (2-norm 1.9e-3 against 1.7e-3, the
// output's own).  With at most eight rows the second parts are rows 8 to 15 of the same product, added up at
// the end (two products: 16 tokens over 4097 keys 51.7 us, so 50.4), and the softmax takes half.
template <bool F16, int DH>
__global__ void __launch_bounds__(F_TH, few_ctas<DH>()) attn_few_kernel(const PackedParams p) {
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ long before[F_TH], warp_sum[F_WARPS];
  __shared__ Span spans[F_TH];  // of the sequences in `before`
  constexpr int LD = DH + 4, U = DH / 64, J = DH / 32;
  float* so = reinterpret_cast<float*>(smem);                                      // [F_WARPS][16][LD]
  float2* sml = reinterpret_cast<float2*>(smem + F_WARPS * F_ROWS * LD * 4);       // [F_WARPS][16]
  grid_dep_sync();
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, n = lane >> 2, c = lane & 3;
  const int G = p.group;

  // sequences [first, first + F_TH): what lies before each of them (of these), and their sum
  auto add_up = [&](int first) {
    long w = 0;
    const int i = first + (int)threadIdx.x;
    Span s{};
    if (i < p.seqs) {
      s = span_of(p, i);
      w = few_units(p, s.lq) * (p.split ? few_length(s.lk) : 1);
    }
    long sum = w;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const long y = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += y;
    }
    __syncthreads();  // the last call's values have been read
    if (lane == 31) warp_sum[warp] = sum;
    __syncthreads();
    long all = 0, mine = 0;
#pragma unroll
    for (int v = 0; v < F_WARPS; ++v) {
      if (v < warp) mine += warp_sum[v];
      all += warp_sum[v];
    }
    before[threadIdx.x] = mine + sum - w;
    spans[threadIdx.x] = s;
    __syncthreads();
    return all;
  };
  int first = 0;          // of the sequences in `before`
  long base = 0;          // what lies before them
  long here = add_up(0), total = here;
  for (int i = F_TH; i < p.seqs; i += F_TH) total += add_up(i);
  if (p.seqs > F_TH) add_up(0);
  const long share = (total + gridDim.x - 1) / gridDim.x;
  long pos = (long)blockIdx.x * share;
  const long stop = min(pos + share, total);
  if (p.split && blockIdx.x == 0 && threadIdx.x == 0) p.place[0] = share;

  // what is done next: a unit, or some tiles of one
  struct Work {
    int q0, rows, head, r0;      // the sequence's first query row and rows, the key head, the unit's first row
    int k_lo, k_hi;              // keys
    int shift, last;             // token t sees keys before t + shift; the sequence's last token
    int k0;
    int length;                  // of it (split)
    bool starts, ends;           // the unit's keys do
  };
  int lo = -1;  // the sequence that holds pos, among those of `before` (-1: not known)
  auto find = [&]() {
    while (pos >= base + here) {
      base += here;
      first += F_TH;
      here = add_up(first);
      lo = -1;
    }
    if (lo < 0) {
      lo = 0;
#pragma unroll
      for (int o = F_TH / 2; o > 0; o /= 2)
        if (first + lo + o < p.seqs && before[lo + o] <= pos - base) lo += o;
    } else {  // the same one mostly, or the next
      while (lo + 1 < F_TH && first + lo + 1 < p.seqs && before[lo + 1] <= pos - base) ++lo;
    }
    const Span s = spans[lo];
    const int all = p.split ? few_length(s.lk) : 1, blocks = (s.lq * G + F_ROWS - 1) / F_ROWS;
    const long off = pos - base - before[lo];
    const long unit = off <= 0x7fffffffL ? (long)((unsigned)off / (unsigned)all) : off / all;
    const int at = (int)(off - unit * all);
    if (p.split && off == 0 && threadIdx.x == 0) p.place[1 + first + lo] = pos;
    Work w;
    w.q0 = s.q0;
    w.rows = s.lq * G;
    w.head = blocks == 1 ? (int)unit : (int)(unit / blocks);
    w.r0 = blocks == 1 ? 0 : (int)(unit - (long)w.head * blocks) * F_ROWS;
    w.length = (int)min((long)(all - at), stop - pos);
    w.starts = at == 0;
    w.ends = at + w.length == all;
    w.k_lo = max(at - F_COST, 0) * F_TILE;
    w.k_hi = w.ends ? s.lk : max(at + w.length - F_COST, 0) * F_TILE;
    w.shift = 1 + s.lk - s.lq;
    w.last = s.lq - 1;
    w.k0 = s.k0;
    return w;
  };
  // token and head (of the group) of row r = r0 + i; of the rows that a thread has to do with in a sequence's first
  // unit (mostly the only one) worked out once
  struct Row {
    int tok, g;
  };
  auto row_of = [&](int r) {
    const int t = (unsigned)r / (unsigned)G;
    return Row{t, r - t * G};
  };
  constexpr int ITEMS = F_ROWS * (DH / 8) / F_TH;  // of a thread where the sums are stored: rows F_TH / (DH / 8) apart
  const Row first_rows[2] = {row_of(n), row_of(n + 8)};
  const Row last_rows[2] = {row_of(threadIdx.x / (DH / 8)), row_of(threadIdx.x / (DH / 8) + F_TH / (DH / 8))};
  static_assert(ITEMS <= 2 && F_ROWS * (DH / 8) == ITEMS * F_TH, "a thread's items");
  const Row end_row = row_of(F_ROWS - 1);
  // keys that row r (token tok of the sequence) of the unit sees end before
  auto limit = [&](const Work& w, int r, int tok) {
    if (r >= w.rows) return w.k_lo;
    return min(max(p.causal ? tok + w.shift : w.k_hi, w.k_lo), w.k_hi);
  };
  uint4 qa[2][J], kf[2][J], vf[4][U];
  const uint16_t *kb = nullptr, *vb = nullptr;
  int end = 0;  // of the keys that the unit's last row sees
  auto load_k = [&](int k0) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int key = k0 + 8 * t + n;
#pragma unroll
      for (int j = 0; j < J; ++j)
        kf[t][j] = key < end ? ld_stream(kb + key * p.ldk + 32 * j + 8 * c) : make_uint4(0, 0, 0, 0);
    }
  };
  auto load_v = [&](int k0) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int key = k0 + 2 * c + (t & 1) + 8 * (t >> 1);
#pragma unroll
      for (int u = 0; u < U; ++u)
        vf[t][u] = key < end ? ld_stream(vb + key * p.ldv + 64 * u + 8 * n) : make_uint4(0, 0, 0, 0);
    }
  };
  auto begin = [&](const Work& w) {
    kb = p.k + w.k0 * p.ldk + w.head * DH;
    vb = p.v + w.k0 * p.ldv + w.head * DH;
    // the last row sees most
    end = w.r0 + F_ROWS <= w.rows ? limit(w, 0, w.r0 == 0 ? end_row.tok : row_of(w.r0 + F_ROWS - 1).tok)
                                  : limit(w, 0, w.last);
    const int k0 = w.k_lo + warp * F_KEYS;
    if (k0 < end) load_k(k0);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = w.r0 + n + 8 * i;
      const Row t = w.r0 == 0 ? first_rows[i] : row_of(r);
      const uint16_t* at = p.q + (w.q0 + t.tok) * p.ldq + (w.head * G + t.g) * DH;
#pragma unroll
      for (int j = 0; j < J; ++j)
        qa[i][j] = r < w.rows ? __ldg(reinterpret_cast<const uint4*>(at + 32 * j + 8 * c)) : make_uint4(0, 0, 0, 0);
    }
    if (k0 < end) load_v(k0);
  };
  if (pos >= stop) return;
  Work w = find();
  begin(w);
  while (true) {
    const bool eight = w.rows - w.r0 <= 8;  // rows, whose weights' second parts take the place of the other eight
    int lim[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = w.r0 + n + 8 * i;
      lim[i] = limit(w, r, w.r0 == 0 ? first_rows[i].tok : row_of(r).tok);
    }
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, o[U * 8][4];
#pragma unroll
    for (int i = 0; i < U * 8; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i][e] = 0.f;
    for (int k0 = w.k_lo + warp * F_KEYS; k0 < end; k0 += F_TILE) {
      float sc[2][4];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int e = 0; e < 4; ++e) sc[t][e] = 0.f;
#pragma unroll
        for (int j = 0; j < J; ++j) {
          mma16816<F16>(sc[t], qa[0][j].x, qa[1][j].x, qa[0][j].y, qa[1][j].y, kf[t][j].x, kf[t][j].y);
          mma16816<F16>(sc[t], qa[0][j].z, qa[1][j].z, qa[0][j].w, qa[1][j].w, kf[t][j].z, kf[t][j].w);
        }
      }
      if (k0 + F_TILE < end) load_k(k0 + F_TILE);
      bool moved = false;
      float alpha[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (i == 1 && eight) {
          alpha[1] = alpha[0];
          break;
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            if (k0 + 8 * t + 2 * c + e >= lim[i]) sc[t][2 * i + e] = -INFINITY;
        float mx = fmaxf(fmaxf(sc[0][2 * i], sc[0][2 * i + 1]), fmaxf(sc[1][2 * i], sc[1][2 * i + 1]));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaf(fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2)), p.scale_log2, -kWeightsUp<F16>);
        alpha[i] = 1.f;
        if (mx > m[i] + 8.f) {  // the maximum moves only by more than 2^8, which P's type holds
          alpha[i] = ex2(m[i] - mx);
          m[i] = mx;
          l[i] *= alpha[i];
          moved = true;
        }
        const float neg = m[i] == -INFINITY ? 0.f : -m[i];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float x = ex2(fmaf(sc[t][2 * i + e], p.scale_log2, neg));
            l[i] += x;
            sc[t][2 * i + e] = x;
          }
      }
      if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
        for (int i = 0; i < U * 8; ++i) {
          o[i][0] *= alpha[0];
          o[i][1] *= alpha[0];
          o[i][2] *= alpha[1];
          o[i][3] *= alpha[1];
        }
      }
      const uint32_t a0 = pack16<F16>(sc[0][0], sc[0][1]), a2 = pack16<F16>(sc[1][0], sc[1][1]);
      // bf16: what its eight bits leave of a weight
      auto rest = [](uint32_t w, float a, float b) {
        return F16 ? 0u : pack_bf16x2(a - __uint_as_float(w << 16), b - __uint_as_float(w & 0xffff0000u));
      };
      // P V; both: with a second operand for what is left of the weights
      auto products = [&](auto both, uint32_t a1, uint32_t a3, uint32_t r0, uint32_t r1, uint32_t r2, uint32_t r3) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
          for (int t = 0; t < 8; ++t) {
            auto word = [&](const uint4& v) { return t < 2 ? v.x : (t < 4 ? v.y : (t < 6 ? v.z : v.w)); };
            const uint32_t sel = t & 1 ? 0x7632u : 0x5410u;
            const uint32_t b0 = __byte_perm(word(vf[0][u]), word(vf[1][u]), sel),
                           b1 = __byte_perm(word(vf[2][u]), word(vf[3][u]), sel);
            mma16816<F16>(o[u * 8 + t], a0, a1, a2, a3, b0, b1);
            if constexpr (decltype(both)::value) mma16816<F16>(o[u * 8 + t], r0, r1, r2, r3, b0, b1);
          }
        }
      };
      const uint32_t r0 = rest(a0, sc[0][0], sc[0][1]), r2 = rest(a2, sc[1][0], sc[1][1]);
      if (eight) {
        products(std::false_type{}, r0, r2, 0, 0, 0, 0);
      } else {
        const uint32_t a1 = pack16<F16>(sc[0][2], sc[0][3]), a3 = pack16<F16>(sc[1][2], sc[1][3]);
        products(std::bool_constant<!F16>{}, a1, a3, r0, rest(a1, sc[0][2], sc[0][3]), r2, rest(a3, sc[1][2], sc[1][3]));
      }
      if (k0 + F_TILE < end) load_v(k0 + F_TILE);
    }
    if (!F16 && eight) {
#pragma unroll
      for (int i = 0; i < U * 8; ++i) {
        o[i][0] += o[i][2];
        o[i][1] += o[i][3];
      }
    }
    // where the sums go, then the next unit's loads
    const Work done = w;
    pos += w.length;
    const bool more = pos < stop;
    if (more) {
      w = find();
      begin(w);
    }
    // the warps' parts
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
      l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
      if (c == 0) sml[warp * F_ROWS + n + 8 * i] = make_float2(m[i], l[i]);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if (done.r0 + n + 8 * i >= done.rows) continue;  // no such row
      float top = -INFINITY;
#pragma unroll
      for (int v = 0; v < F_WARPS; ++v) top = fmaxf(top, sml[v * F_ROWS + n + 8 * i].x);
      const float f = m[i] == -INFINITY ? 0.f : ex2(m[i] - top);
      float* row = so + (warp * F_ROWS + n + 8 * i) * LD;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int t = 0; t < 8; t += 4)
            *reinterpret_cast<float4*>(row + 64 * u + 16 * c + 8 * e + t) =
                make_float4(o[u * 8 + t][2 * i + e] * f, o[u * 8 + t + 1][2 * i + e] * f,
                            o[u * 8 + t + 2][2 * i + e] * f, o[u * 8 + t + 3][2 * i + e] * f);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int lr = threadIdx.x / (DH / 8) + i * (F_TH / (DH / 8)), col = threadIdx.x % (DH / 8) * 8;
      const int r = done.r0 + lr;
      if (r >= done.rows) continue;
      float top = -INFINITY, den = 0.f, v[8];
#pragma unroll
      for (int k = 0; k < F_WARPS; ++k) top = fmaxf(top, sml[k * F_ROWS + lr].x);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = 0.f;
#pragma unroll
      for (int k = 0; k < F_WARPS; ++k) {
        const float2 f = sml[k * F_ROWS + lr];
        den += part_weight(f, top) * f.y;
        const float4* row = reinterpret_cast<const float4*>(so + (k * F_ROWS + lr) * LD + col);
        const float4 a = row[0], b = row[1];
        v[0] += a.x, v[1] += a.y, v[2] += a.z, v[3] += a.w;
        v[4] += b.x, v[5] += b.y, v[6] += b.z, v[7] += b.w;
      }
      const Row t = done.r0 == 0 ? last_rows[i] : row_of(r);
      if (den == 0.f && limit(done, r, t.tok) > done.k_lo) den = 1.f;  // all scores are minus infinity
      const long tok = done.q0 + t.tok;
      const int h = done.head * G + t.g;
      const bool whole = done.starts && done.ends;
      if (whole && p.parts1 == 0) {
        const float inv = inverse_sum(top, den);
        uint4 x;
        x.x = pack16<F16>(v[0] * inv, v[1] * inv);
        x.y = pack16<F16>(v[2] * inv, v[3] * inv);
        x.z = pack16<F16>(v[4] * inv, v[5] * inv);
        x.w = pack16<F16>(v[6] * inv, v[7] * inv);
        *reinterpret_cast<uint4*>(p.o + tok * p.ldo + (long)h * DH + col) = x;
        if (p.lse && col == 0) p.lse[tok * p.heads + h] = (top + log2f(den)) * 0.6931471805599453f;
      } else {
        const long at = whole ? ((long)p.parts1 * p.nq + tok) * p.heads + h
                              : (long)(blockIdx.x * 2 + (done.starts ? 1 : 0)) * F_ROWS + lr;
        float4* d = reinterpret_cast<float4*>((whole ? p.part_o : p.piece_o) + at * DH + col);
        d[0] = make_float4(v[0], v[1], v[2], v[3]);
        d[1] = make_float4(v[4], v[5], v[6], v[7]);
        if (col == 0) (whole ? p.part_ml : p.piece_ml)[at] = make_float2(top, den);
      }
    }
    if (!more) break;
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// many rows: tensor cores
// ---------------------------------------------------------------------------
namespace {
constexpr int PT = 128;                    // rows and keys of a tile
constexpr int PT_CHUNK = PT * 64 * 2;      // 128 rows x 64 columns: one 128-byte swizzle column
constexpr int PT_LD = 80;                  // bytes a row in the output transpose (16 against bank conflicts)
constexpr int PT_OUT = 4 * 32 * PT_LD;     // bytes of a tile's
// A CTA of NT tiles: threads, tensor memory (the scores' NT * 128 columns, then the outputs'), registers (168
// a thread at launch with two tiles, 128 with one: 128 * 88 + 256 * 208 and 128 * 64 + 128 * 192 of them)
// and shared memory (two CTAs on an SM with one tile).
template <int DH, int NT>
struct Pt {
  static constexpr int THREADS = 128 + NT * 128, TMEM_COLS = NT * 256;
  static constexpr int REGS_ISSUE = NT == 2 ? 88 : 64, REGS_SOFTMAX = NT == 2 ? 208 : 192;
  static constexpr int STAGES = NT == 1 && DH == 128 ? 1 : 2;  // of the K ring and of the V ring
  static constexpr int TILE = DH / 64 * PT_CHUNK;
  static constexpr int Q = 0, K = NT * TILE, V = K + STAGES * TILE, OUT = V + STAGES * TILE;
  static constexpr int ROWS = OUT + NT * PT_OUT;  // where a row's output goes
  static constexpr int BAR = ROWS + NT * PT * 8;
  static constexpr int BYTES = BAR + 384 + 1024;
};
static_assert(2 * (Pt<128, 1>::BYTES + 1024) <= 228 * 1024 && 2 * (Pt<64, 1>::BYTES + 1024) <= 228 * 1024, "two CTAs on an SM");
static_assert(Pt<128, 2>::BYTES <= 227 * 1024, "shared memory of a CTA");

// Another CTA's work: the launch hands over the index of one that has not started, which then never does
// (16 bytes to `response`, signalled on bar), until none is left.
BAG_DEV void next_cta_request(void* response, uint64_t* bar) {
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(
                   smem_u32(response)),
               "r"(smem_u32(bar))
               : "memory");
}
BAG_DEV bool next_cta(const void* response, int* x) {
  uint32_t there, at;
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b128 r;\n\t"
      "ld.shared.b128 r, [%2];\n\t"
      "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t"
      "mov.u32 %1, 0;\n\t"
      "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, r;\n\t}"
      : "=r"(there), "=r"(at)
      : "r"(smem_u32(response))
      : "memory");
  *x = (int)at;
  return there != 0;
}

// Shared-memory descriptors (as sw128_desc) by their lower words: the upper one (1024 bytes from eight rows to
// the next, version, 128-byte swizzle) is the same for all, and a register less for each.  _mn: of a tile whose
// rows run along the contraction (V: a row a key), 64-column chunks PT_CHUNK apart.
constexpr uint32_t PT_DESC_HI = (1024 >> 4) | 1u << 14 | 2u << 29;
BAG_DEV uint32_t desc_k(uint32_t saddr) { return (saddr & 0x3ffffu) >> 4 | 1u << 16; }
BAG_DEV uint32_t desc_mn(uint32_t saddr) { return (saddr & 0x3ffffu) >> 4 | (uint32_t)(PT_CHUNK >> 4) << 16; }
// D (TMEM) (+)= A (shared memory) * B (shared memory), and with A in TMEM
BAG_DEV void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\t"
      "mov.b64 a, {%1, %5};\n\tmov.b64 b, {%2, %5};\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n\t}" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "n"(PT_DESC_HI)
      : "memory");
}
BAG_DEV void mma_ts(uint32_t d, uint32_t a_tmem, uint32_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 b;\n\t"
      "mov.b64 b, {%2, %5};\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n\t}" ::"r"(d),
      "r"(a_tmem), "r"(b), "r"(idesc), "r"(accumulate), "n"(PT_DESC_HI)
      : "memory");
}

// The sequence of the units' slot `slot` (units of `per` tokens, a key head), and the unit's index in it (-1: none).
// Up to 32 sequences: in order of their keys, most first (units that take long go first), each with as many
// slots as it has units.  More: as they come, the last first, sequence i's slots from q_start[i] / per + i on
// (as many as its units, or one more).  A sequence's last unit sees most keys, and goes first.  Called by a
// whole warp.
BAG_DEV Span span_of_slot(const PackedParams& p, int per, int slot, int* index) {
  const int lane = threadIdx.x % 32;
  Span s;
  int first, units, src;
  if (p.seqs <= 32) {
    s = span_of(p, min(lane, p.seqs - 1));
    units = lane < p.seqs ? (s.lq + per - 1) / per : 0;
    first = 0;
    for (int i = 0; i < p.seqs; ++i) {
      const int lk = __shfl_sync(0xffffffffu, s.lk, i), n = __shfl_sync(0xffffffffu, units, i);
      if (lk > s.lk || (lk == s.lk && i < lane)) first += n;
    }
    const uint32_t at = __ballot_sync(0xffffffffu, slot >= first && slot < first + units);
    src = at ? __ffs(at) - 1 : 0;
  } else {
    auto start = [&](int i) { return (int)((unsigned)max(__ldg(p.q_start + i), 0) / (unsigned)per) + i; };
    slot = p.slots2 - 1 - slot;
    int lo = 0, n = p.seqs;
    while (n > 32) {
      const int step = (n + 31) / 32, i = lane * step;
      const uint32_t at = __ballot_sync(0xffffffffu, i < n && start(lo + i) <= slot);
      const int skip = max(__popc(at) - 1, 0) * step;
      lo += skip;
      n = min(step, n - skip);
    }
    s = span_of(p, lo + min(lane, n - 1));
    units = (s.lq + per - 1) / per;
    first = start(lo + min(lane, n - 1));
    src = max(__popc(__ballot_sync(0xffffffffu, lane < n && first <= slot)) - 1, 0);
    // the same order as above: the highest slot is the last unit
    slot = first + units - 1 - (slot - first);
  }
  s.q0 = __shfl_sync(0xffffffffu, s.q0, src);
  s.lq = __shfl_sync(0xffffffffu, s.lq, src);
  s.k0 = __shfl_sync(0xffffffffu, s.k0, src);
  s.lk = __shfl_sync(0xffffffffu, s.lk, src);
  units = __shfl_sync(0xffffffffu, units, src);
  const int i = units - 1 - (__shfl_sync(0xffffffffu, slot, src) - __shfl_sync(0xffffffffu, first, src));
  *index = i >= 0 && i < units ? i : -1;
  return s;
}

// mbar_wait_warp for the hand-over of units: a role without work in a unit waits as long as the others take for it,
// which for very many keys in one part may pass a wait's usual limit.  A failure elsewhere still ends it at once.
BAG_DEV bool wait_unit(uint64_t* bar, uint32_t parity, volatile int* abort) {
  bool there = mbar_try_wait(bar, parity);
  const uint64_t t0 = global_ns();
  for (uint32_t i = 1; !there; ++i) {
    there = mbar_try_wait(bar, parity);
    if (!there && (i & 63) == 0) {
      if (*abort) break;
      if (global_ns() - t0 > 30 * kWaitLimitNs) {
        *abort = 1;
        break;
      }
    }
  }
  return __all_sync(0xffffffffu, there);
}

// What a CTA works on at a time.
struct Unit {
  int q0, tokens;        // its first query row, and how many (0: nothing to do, -1: no unit is left)
  int head0;             // first query head of its rows
  int sees;              // own keys that its first token sees (below zero: none; of all with no mask)
  int k0, lk;            // the sequence's keys
  int fused;             // key tiles of the prefix, before them
  int part, j0;          // the part of the keys, and its first tile
  int n[2];              // key tiles of each tile of rows
  int direct;            // the part is the only one: the output is final
};
// own keys that the unit's token i sees
BAG_DEV int sees_of(const PackedParams& p, const Unit& u, int i) {
  return p.causal ? min(max(u.sees + i, 0), u.lk) : u.lk;
}
BAG_DEV Unit unit_of(const PackedParams& p, int nt, int at) {
  Unit u{};
  const int per_head = p.slots1 * p.parts1 + p.slots2 * p.parts2, units1 = p.slots1 * p.parts1, per = nt * p.tokens;
  int hu;
  if (p.by_head) {  // a head at a time, so that its keys stay in L2
    hu = at / per_head;
    at -= hu * per_head;
  } else {  // all heads of a slot
    const int groups = p.heads / p.together, i = at / groups;
    hu = at - i * groups;
    at = i;
  }
  u.head0 = hu * p.together;
  int most;  // tiles that the part may have
  if (at < units1) {  // the prefix with the tokens of all sequences
    const Span s = span_all(p);
    const int slot = at / p.parts1;
    u.part = at - slot * p.parts1;
    u.q0 = s.q0 + slot * per;
    u.tokens = max(min(s.lq - slot * per, per), 0);
    most = p.chunk1 / PT;
    u.j0 = u.part * most;
    u.fused = (p.n_prefix + PT - 1) / PT;
  } else {
    at -= units1;
    const int back = at / p.parts2, own = at - back * p.parts2;
    int index;
    const Span s = span_of_slot(p, per, back, &index);
    if (index < 0) return u;
    const int parts = own_parts(p, s.lk), t0 = index * per;
    if (own >= (p.parts1 ? parts : max(parts, 1))) return u;
    u.q0 = s.q0 + t0;
    u.tokens = min(s.lq - t0, per);
    u.sees = p.causal ? t0 + 1 + s.lk - s.lq : s.lk;
    u.k0 = s.k0, u.lk = s.lk;
    u.fused = p.fused;
    u.part = p.parts1 + own;
    u.j0 = own * (p.chunk2 / PT);
    most = own == p.parts2 - 1 ? 0x7fffffff : p.chunk2 / PT;
    u.direct = p.parts1 == 0 && parts <= 1;
  }
  for (int x = 0; x < nt; ++x) {
    const int end = min((x + 1) * p.tokens, u.tokens);
    if (end > x * p.tokens) u.n[x] = min(max(u.fused + (sees_of(p, u, end - 1) + PT - 1) / PT - u.j0, 0), most);
  }
  return u;
}
}  // namespace

// A CTA takes units of NT tiles of up to 128 rows (row r: query token r / together, head r % together of those that
// share the key head), one after the other, and walks the tiles of 128 keys that the last of their rows sees:
//   warp 0        finds the units (its own, then those of CTAs that have not started, each asked for when the
//                 last loads of the one before are due) and loads by TMA: the queries, then K and V tiles
//                 into rings of their own
//   warp 1        MMA issuer, in turn between the tiles: S_A,0 S_B,0 | PV_A,j S_A,j+1 | PV_B,j S_B,j+1 | ...
//                 It zeros the rows of V past a sequence's (or the prefix's) last key: whatever lies there would
//                 meet weights of zero, and may be NaN
//   warps 4..     the softmax of tile A (4..7) and B (8..11), a row a thread, as in the dense kernel: P goes
//                 back over the scores in 16 bits and enters the second product from TMEM; O stays in
//                 TMEM and is rescaled only when the maximum has grown by more than 8
// So the loads and scores of a unit run beside the output of the one before, and what a CTA costs to launch
// (tensor memory, barriers, the launch itself, some 5,000 cycles) comes once for each that is resident.
// V is read as it lies, a row a key: as an operand whose rows run along the contraction (as fast as the other way).
// P is rounded to the operands' type, as in the dense kernel: both operands of an MMA are of one type (2-norm error
// bf16 1.8e-3 to 2.2e-3 where the output's own rounding gives 1.6e-3 to 1.7e-3, fp16 2.2e-4 to 2.7e-4 for 1.9e-4 to 2.1e-4).
// Two tiles and one CTA on an SM, or one tile and two CTAs: the first reads each K and V tile once for 256 rows
// (16,384 tokens, 32 heads 1300 against 1480 us, 16 x 512 tokens 62 against 72), the second has more CTAs for
// few rows (77 tokens, 32 heads 7.1 against 8.3, 512 tokens 11.9 against 12.9).
// Bound: a step of both tiles takes some 2,600 cycles for 2,048 of products: a tile's scores, softmax and P V
// follow each other, and the hand-overs between the warps (about 1,200 cycles a step) are only partly hidden
// by the other tile.  A unit costs some 6,000 cycles besides, mostly its output.  16,384 causal tokens, 32 heads 1300 to
// 1474 us (1690 to 1490 TFLOP/s: back to back, or between other work, by what clock the card holds), 4608 x 24 heads 103, 4 x 2048 x 32 115, 16 x 512 x 32 61 (query and output bytes 25); heads of
// 64: 16,384 x 32 1150, where the softmax has twice the work for each product.
// Not kept: two threads a row (4 x 2048 124 -> 188 us: the issuing warp loses its slots), an MMA warp whose issue branches on
// the last tile (16,384 tokens 1380 -> 1480), 64-bit descriptors in registers (spills in the issuing warp).
template <bool F16, int DH, int NT>
__global__ void __launch_bounds__(Pt<DH, NT>::THREADS, 3 - NT)
    attn_packed_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                       const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmPK,
                       const __grid_constant__ CUtensorMap tmPV, const PackedParams p) {
  using M = Pt<DH, NT>;
  constexpr int PT_STAGES = M::STAGES;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  uint8_t *sQ = smem + M::Q, *sK = smem + M::K, *sV = smem + M::V;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + M::BAR);
  uint64_t* q_full = bars + 0;
  uint64_t* q_empty = bars + 1;
  uint64_t* k_full = bars + 2;    // [2]
  uint64_t* k_empty = bars + 4;   // [2]
  uint64_t* v_full = bars + 6;    // [2]
  uint64_t* v_empty = bars + 8;   // [2]
  uint64_t* s_full = bars + 10;   // [2] per query tile
  uint64_t* p_full = bars + 12;   // [2]
  uint64_t* o_done = bars + 14;   // [2]
  uint64_t* u_full = bars + 16;   // [2] of the ring of units
  uint64_t* u_empty = bars + 18;  // [2]
  uint64_t* asked = bars + 20;
  uint64_t* drain = bars + 21;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 22);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  uint8_t* response = reinterpret_cast<uint8_t*>(bars + 24);  // 16 bytes
  Unit* units = reinterpret_cast<Unit*>(bars + 26);           // [2]
  static_assert(26 * 8 + 2 * sizeof(Unit) <= 384 && M::BAR % 16 == 0, "barriers and units");
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;

  if (threadIdx.x == 0) {
    mbar_init(q_full, 1);
    mbar_init(q_empty, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(k_full + i, 1);
      mbar_init(k_empty + i, 1);
      mbar_init(v_full + i, 1);
      mbar_init(v_empty + i, 1);
      mbar_init(s_full + i, 1);
      mbar_init(p_full + i, 4);  // one arrival per softmax warp of the tile
      mbar_init(o_done + i, 1);
      mbar_init(u_full + i, 1);
      mbar_init(u_empty + i, 1 + 4 * NT);  // the issuer and the softmax warps
    }
    mbar_init(asked, 1);
    mbar_init(drain, 1);
    *abort_flag = 0;
    fence_mbar_init();
    tma_prefetch_desc(&tmQ);
    tma_prefetch_desc(&tmK);
    tma_prefetch_desc(&tmV);
  }
  __syncwarp();
  if (warp == 1) {
    tmem_alloc(tmem_slot, M::TMEM_COLS);
    tmem_relinquish();
  }
  // Beside the few-row kernel of a call, whose sums only the join reads: it let this one start when all of its CTAs
  // had waited for what came before the call, so this one has CTAs wherever an SM is done with those, and waits
  // for it at the end, for the kernels that follow.
  if (p.beside)
    grid_dep_launch();
  else
    grid_dep_sync();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = uniform(*tmem_slot);
  auto wait = [&](uint64_t* bar, uint32_t ph) {
    const bool w = mbar_wait_warp(bar, ph, abort_flag);
    tc_fence_after();
    return w;
  };

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(M::REGS_ISSUE));
    if (warp == 0) {
      // ---------------- units and TMA ----------------
      int at = blockIdx.x, c = 0, qn = 0, kn = 0, vn = 0, asks = 0;  // unit; units, Q, K and V tiles, requests so far
      bool ok = true, left = true;
      while (ok && left) {
        bool ask = true;  // for the next unit, once
        auto request = [&]() {
          if (lane == 0) {
            fence_proxy_async_smem();  // the last answer has been read
            mbar_arrive_expect_tx(asked, 16);
            next_cta_request(response, asked);
          }
          ask = false;
        };
        if (!(ok = wait_unit(u_empty + (c & 1), ((c >> 1) & 1) ^ 1, abort_flag))) break;
        const Unit& u = units[c & 1];
        {
          const Unit found = unit_of(p, NT, at);
          if (lane == 0) units[c & 1] = found;
        }
        __syncwarp();
        if (u.tokens > 0) {
          if (lane == 0) mbar_arrive(u_full + (c & 1));
          ++c;
          const int nkb = max(u.n[0], u.n[1]), head = u.head0 / p.group;
          if (nkb > 0) {
            if (!(ok = wait(q_empty, (qn & 1) ^ 1))) break;
            if (lane == 0) {
              const int tiles = (u.n[0] > 0) + (u.n[1] > 0);
              mbar_arrive_expect_tx(q_full, tiles * (DH / 64) * p.tokens * p.together * 128);
              for (int x = 0; x < NT; ++x)
                for (int d = 0; d < DH / 64 && u.n[x] > 0; ++d)
                  tma_load_3d(sQ + x * M::TILE + d * PT_CHUNK, &tmQ, d * 64, u.head0, u.q0 + x * p.tokens, q_full);
            }
            ++qn;
          }
          for (int j = 0; j < nkb; ++j) {
            const int t = u.j0 + j;
            const bool pre = t < u.fused;
            const int row = pre ? t * PT : u.k0 + (t - u.fused) * PT;
            const CUtensorMap *mk = pre ? &tmPK : &tmK, *mv = pre ? &tmPV : &tmV;
            if (ask && j >= nkb - 3) request();
            const int ks = kn % PT_STAGES, vs = vn % PT_STAGES;
            if (!(ok = wait(k_empty + ks, ((kn / PT_STAGES) & 1) ^ 1))) break;
            if (lane == 0) {
              mbar_arrive_expect_tx(k_full + ks, M::TILE);
              for (int d = 0; d < DH / 64; ++d)
                tma_load_2d(sK + ks * M::TILE + d * PT_CHUNK, mk, head * DH + d * 64, row, k_full + ks);
            }
            ++kn;
            if (!(ok = wait(v_empty + vs, ((vn / PT_STAGES) & 1) ^ 1))) break;
            if (lane == 0) {
              mbar_arrive_expect_tx(v_full + vs, M::TILE);
              for (int d = 0; d < DH / 64; ++d)
                tma_load_2d(sV + vs * M::TILE + d * PT_CHUNK, mv, head * DH + d * 64, row, v_full + vs);
            }
            ++vn;
          }
        }
        if (ok && ask) request();
        if (!ask) {
          // also after an abort: the answer may not come when the CTA has gone
          const uint64_t t0 = global_ns();
          while (!mbar_try_wait(asked, asks & 1) && global_ns() - t0 < kWaitLimitNs) {
          }
          if (!__all_sync(0xffffffffu, mbar_try_wait(asked, asks & 1))) {
            *abort_flag = 1;
            ok = false;
          }
          ++asks;
          __syncwarp();
          left = ok && next_cta(response, &at);
          __syncwarp();
        }
      }
      if (ok && (ok = wait_unit(u_empty + (c & 1), ((c >> 1) & 1) ^ 1, abort_flag)) && lane == 0) {
        units[c & 1].tokens = -1;
        mbar_arrive(u_full + (c & 1));
      }
      if (!ok) {
        // wait (bounded) for copies still in flight before the CTA may exit
        const uint64_t t0 = global_ns();
        auto landed = [&](uint64_t* bar, uint32_t ph) {
          while (!mbar_try_wait(bar, ph) && global_ns() - t0 < kWaitLimitNs) {
          }
        };
        if (qn > 0) landed(q_full, (qn - 1) & 1);
        for (int j = max(0, kn - PT_STAGES); j < kn; ++j) landed(k_full + j % PT_STAGES, (j / PT_STAGES) & 1);
        for (int j = max(0, vn - PT_STAGES); j < vn; ++j) landed(v_full + j % PT_STAGES, (j / PT_STAGES) & 1);
      }
    } else if (warp == 1) {
      // ---------------- MMA issuer (converged warp, one elected lane issues) ----------------
      constexpr uint32_t idesc_s = F16 ? idesc_f16_f32(PT, PT) : idesc_bf16_f32(PT, PT);
      constexpr uint32_t idesc_o = (F16 ? idesc_f16_f32(PT, DH) : idesc_bf16_f32(PT, DH)) | 1u << 16;  // B along its rows
      const uint32_t q_addr = smem_u32(sQ), k_addr = smem_u32(sK), v_addr = smem_u32(sV);
      // K step kk of a tile: 64-column chunk kk / 4, 32 bytes per step inside it (16-byte units)
      auto koff = [](int kk) { return (uint32_t)(((kk >> 2) * PT_CHUNK + (kk & 3) * 32) >> 4); };
      int base = 0, qn = 0;  // key tiles of the units before; units with any
      int done0 = 0, done1 = 0;  // those of each tile of rows
      bool ok = true;
      for (int c = 0; ok; ++c) {
        if (!(ok = wait_unit(u_full + (c & 1), (c >> 1) & 1, abort_flag))) break;
        const Unit& u = units[c & 1];
        const int n0 = u.n[0], n1 = NT == 2 ? u.n[1] : 0, nkb = max(n0, n1), fused = u.fused, j0 = u.j0, lk = u.lk;
        if (u.tokens < 0) break;
        int scores = n0 + n1;  // products that still need the queries
        // S of tile x and key tile j; release: the tile's K is no longer needed
        auto issue_s = [&](int x, int j, bool release) {
          const int st = (base + j) % PT_STAGES;
          const uint32_t qd = desc_k(q_addr + x * M::TILE);
          const uint32_t kd = desc_k(k_addr + st * M::TILE);
          const bool last = --scores == 0;
          if (elect_one()) {
#pragma unroll
            for (int kk = 0; kk < DH / 16; ++kk)
              mma_ss(tmem + x * 128, qd + koff(kk), kd + koff(kk), idesc_s, kk > 0 ? 1u : 0u);
            mma_commit(s_full + x);
            if (release) mma_commit(k_empty + st);
            if (last) mma_commit(q_empty);
          }
          __syncwarp();
        };
        // release: the tile's V is no longer needed; last: no other product follows for tile x
        auto issue_pv = [&](int x, int j, bool release, bool last) {
          const int st = (base + j) % PT_STAGES;
          const uint32_t vd = desc_mn(v_addr + st * M::TILE);
          if (elect_one()) {
#pragma unroll
            for (int kk = 0; kk < PT / 16; ++kk)
              mma_ts(tmem + NT * 128 + x * 128, tmem + x * 128 + kk * 8, vd + kk * (2048 >> 4), idesc_o,
                     (j > 0 || kk > 0) ? 1u : 0u);
            if (release) mma_commit(v_empty + st);
            if (last) mma_commit(o_done + x);
          }
          __syncwarp();
        };
        auto k_there = [&](int j) { return wait(k_full + (base + j) % PT_STAGES, ((base + j) / PT_STAGES) & 1); };
        auto p_there = [&](int x, int j) { return wait(p_full + x, ((x ? done1 : done0) + j) & 1); };
        // V of tile j, zeros past its last key: only the prefix's last tile and the sequence's can end early
        const int ends0 = fused - 1 - j0, ends1 = fused + (lk + PT - 1) / PT - 1 - j0;
        auto v_there = [&](int j) {
          const int st = (base + j) % PT_STAGES;
          if (!wait(v_full + st, ((base + j) / PT_STAGES) & 1)) return false;
          if (j == ends0 || j == ends1) {
            const int t = j0 + j, keys = t < fused ? p.n_prefix - t * PT : lk - (t - fused) * PT;
            for (int i = keys * 128 + lane * 16; i < PT_CHUNK; i += 512)  // a chunk's rows lie together
#pragma unroll
              for (int d = 0; d < DH / 64; ++d)
                *reinterpret_cast<uint4*>(sV + st * M::TILE + d * PT_CHUNK + i) = make_uint4(0u, 0u, 0u, 0u);
            fence_proxy_async_smem();
            __syncwarp();
          }
          return true;
        };
        auto last_user = [&](int j) { return j < n1 ? 1 : 0; };
        if (nkb > 0) {
          if (!(ok = wait(q_full, qn & 1))) break;
          ++qn;
          // PV_j of a tile, then its S_{j+1} into the columns P_j came from (in issue order): first the S_0 alone,
          // then steps after which all tiles go on, then those where one ends
          const int both = max((NT == 2 ? min(n0, n1) : n0) - 1, 0);
          int j = -1;
#pragma unroll 1
          for (int end = 0; ok; end = nkb) {
#pragma unroll 1
            for (; j < end && ok; ++j) {
              if (j >= 0 && !(ok = v_there(j))) break;
              bool next = false;  // the next K tile is there
#pragma unroll 1
              for (int x = 0; x < NT; ++x) {
                const int nx = x ? n1 : n0;
                if (j >= nx) continue;
                if (j >= 0) {
                  if (!(ok = p_there(x, j))) break;
                  issue_pv(x, j, x == last_user(j), j == nx - 1);
                }
                if (j + 1 < nx) {
                  if (!next && !(ok = k_there(j + 1))) break;
                  next = true;
                  issue_s(x, j + 1, x == last_user(j + 1));
                }
              }
            }
            if (end == nkb) break;
            for (; j < both && ok; ++j) {
              if (!(ok = v_there(j) && p_there(0, j))) break;
              issue_pv(0, j, NT == 1, false);
              if (!(ok = k_there(j + 1))) break;
              issue_s(0, j + 1, NT == 1);
              if constexpr (NT == 2) {
                if (!(ok = p_there(1, j))) break;
                issue_pv(1, j, true, false);
                issue_s(1, j + 1, true);
              }
            }
          }
          if (!ok) break;
          base += nkb;
          done0 += n0;
          done1 += n1;
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(u_empty + (c & 1));
      }
      if (elect_one()) {
        mma_commit(drain);
        const uint64_t t0 = global_ns();
        while (!mbar_try_wait(drain, 0) && global_ns() - t0 < kWaitLimitNs) {
        }
      }
    }
    __syncwarp();
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(M::REGS_SOFTMAX));
    // ---------------- softmax warpgroups (warps 4..7: tile A, 8..11: tile B) ----------------
    const int x = NT == 2 ? (warp - 4) >> 2 : 0;
    const int quad = warp & 3;
    const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
    const uint32_t s_addr = tmem + lane_base + x * 128;
    const uint32_t o_addr = tmem + lane_base + NT * 128 + x * 128;
    const int row = quad * 32 + lane, of = (unsigned)row / (unsigned)p.together;
    long* at = reinterpret_cast<long*>(smem + M::ROWS) + x * PT + quad * 32;
    uint8_t* buf = smem + M::OUT + x * PT_OUT + quad * 32 * PT_LD;
    int steps = 0, outputs = 0;  // key tiles, and units with any, so far
    bool ok = true;
    for (int c = 0; ok; ++c) {
      if (!(ok = wait_unit(u_full + (c & 1), (c >> 1) & 1, abort_flag))) break;
      const Unit& u = units[c & 1];
      if (u.tokens < 0) break;
      const int tiles = u.n[x];
      // the thread's row: its token of the unit, and how many keys from the part's first tile on it sees (those
      // of a last prefix tile that is not full counted as 128)
      auto token = [&]() { return of < p.tokens && x * p.tokens + of < u.tokens ? x * p.tokens + of : -1; };
      const int own = sees_of(p, u, token() < 0 ? u.tokens - 1 : token());
      const int limit = own + (u.fused - u.j0) * PT;
      // tiles with keys that a row of the warp does not see: that last one of the prefix, and all from the first
      // on that ends behind the keys of the warp's first row
      const int cut0 = p.n_prefix % PT ? u.fused - 1 - u.j0 : -1;
      const int cut1 = u.fused - u.j0 + (int)__reduce_min_sync(0xffffffffu, (unsigned)own) / PT;
      float m_use = -INFINITY, l = 0.f;
      for (int j = 0; j < tiles; ++j) {
        const bool w = mbar_wait(s_full + x, (steps + j) & 1, abort_flag);
        if (!__all_sync(0xffffffffu, w)) {
          ok = false;
          break;
        }
        tc_fence_after();
        // the whole S row in registers: four loads, one wait
        uint32_t r[PT];
#pragma unroll
        for (int i = 0; i < PT / 32; ++i) tmem_ld32_nowait(s_addr + i * 32, r + i * 32);
        tmem_ld_wait();
        if (j == cut0 || j >= cut1) {
          const int kvalid = j == cut0 ? p.n_prefix % PT : limit - j * PT;  // keys that the row sees
#pragma unroll
          for (int i = 0; i < PT; ++i)
            if (i >= kvalid) r[i] = __float_as_uint(-INFINITY);
        }
        // row maximum: four independent chains of three-input maxima
        float mq[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) mq[i] = fmaxf(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1]));
#pragma unroll
        for (int i = 8; i < PT; i += 8)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            mq[k] = max3(mq[k], __uint_as_float(r[i + 2 * k]), __uint_as_float(r[i + 2 * k + 1]));
        const float mx2 = fmaf(fmaxf(fmaxf(mq[0], mq[1]), fmaxf(mq[2], mq[3])), p.scale_log2, -kWeightsUp<F16>);
        float alpha = 1.f;
        if (mx2 > m_use + 8.f) {
          alpha = ex2(m_use - mx2);
          m_use = mx2;
          l *= alpha;
        }
        const float neg_m = m_use == -INFINITY ? 0.f : -m_use;
        float ls0 = 0.f, ls1 = 0.f;
#pragma unroll
        for (int b = 0; b < PT / 32; ++b) {
          uint32_t pk[16];
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            float x0, x1;
            fma2(x0, x1, __uint_as_float(r[b * 32 + i]), __uint_as_float(r[b * 32 + i + 1]), p.scale_log2, neg_m);
            const float a0 = ex2(x0), a1 = ex2(x1);
            add2(ls0, ls1, a0, a1);
            pk[i / 2] = pack16<F16>(a0, a1);
          }
          tmem_st16(s_addr + b * 16, pk);
        }
        l += ls0 + ls1;
        // O_x holds PV of every earlier key tile (the S of this tile was issued after it);
        // rescale it before this tile's PV is issued
        if (j > 0 && __any_sync(0xffffffffu, alpha != 1.f)) {
#pragma unroll 1
          for (int b = 0; b < DH / 32; ++b) {
            float o[32];
            tmem_ld32(o_addr + b * 32, o);
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] *= alpha;
            tmem_st32(o_addr + b * 32, o);
          }
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full + x);
      }
      if (!ok) break;
      steps += tiles;
      // while the last product is on its way: the row's maximum and sum, and where its output goes, for the lanes
      // that store it
      if (l == 0.f && tiles > 0 && limit > 0) l = 1.f;  // the row sees keys, but all scores are minus infinity
      const bool any = l > 0.f || l != l;  // the row sees a key (or NaN)
      const float f = inverse_sum(m_use, l);
      const bool direct = u.direct;
      {
        const int mine = token(), h = u.head0 + row - of * p.together;
        const long i = (long)(u.q0 + mine) * p.heads + h;
        at[lane] = mine < 0 ? -1 : (direct ? (u.q0 + mine) * p.ldo + h * DH : ((long)u.part * p.nq * p.heads + i) * DH);
        if (mine >= 0) {
          if (!direct)
            p.part_ml[(long)u.part * p.nq * p.heads + i] = make_float2(any ? m_use : -INFINITY, l);
          else if (p.lse)
            p.lse[i] = any ? (m_use + log2f(l)) * 0.6931471805599453f : -INFINITY;
        }
      }
      __syncwarp();
      long to[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) to[i] = at[8 * i + (lane >> 2)];
      if (tiles > 0 && !(ok = wait(o_done + x, outputs++ & 1))) break;
      if (x * p.tokens < u.tokens) {
        const bool seen = any && tiles > 0;
        uint32_t o[32];
        auto load = [&](int b) {
          if (tiles > 0) tmem_ld32_nowait(o_addr + b, o);
        };
        load(0);
        tmem_ld_wait();
        // through shared memory, so that a store covers whole runs of a few rows: 64 bytes a row at a time, 32
        // columns in 16 bits or 16 of a part in fp32
        auto turn = [&](const uint32_t* w, auto* out, int col) {
#pragma unroll
          for (int i = 0; i < 16; i += 4)
            *reinterpret_cast<uint4*>(buf + lane * PT_LD + i * 4) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
          __syncwarp();
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint4 v = *reinterpret_cast<const uint4*>(buf + (8 * i + (lane >> 2)) * PT_LD + (lane & 3) * 16);
            if (to[i] >= 0) *reinterpret_cast<uint4*>(out + to[i] + col + (lane & 3) * (16 / sizeof(*out))) = v;
          }
          __syncwarp();
        };
        if (direct) {
#pragma unroll 1
          for (int b = 0; b < DH; b += 32) {
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i)
              w[i] = seen ? pack16<F16>(__uint_as_float(o[2 * i]) * f, __uint_as_float(o[2 * i + 1]) * f) : 0u;
            if (b + 32 < DH) load(b + 32);
            turn(w, p.o, b);
            tmem_ld_wait();
          }
        } else {
#pragma unroll 1
          for (int b = 0; b < DH; b += 32) {
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = seen ? o[i] : 0u;
            turn(o, p.part_o, b);
            turn(o + 16, p.part_o, b + 16);
            if (b + 32 < DH) load(b + 32);
            tmem_ld_wait();
          }
        }
        tc_fence_before();  // the next unit's products into O come after these loads
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(u_empty + (c & 1));
    }
  }
  tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag && p.err) atomicOr(p.err, 1);
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, M::TMEM_COLS);
  }
  if (p.beside) grid_dep_wait();
}

namespace {
constexpr int JN_TH = 256, JR_TH = 256;

// The sequence of query row t, the last one that starts at or before it, and its span.  Called by a whole warp.
BAG_DEV int sequence_of(const PackedParams& p, int t, Span* s) {
  if (p.seqs == p.nq) {  // a token each, mostly
    *s = span_of(p, t);
    if (t >= s->q0 && t < s->q0 + s->lq) return t;
  }
  const int lane = threadIdx.x % 32;
  int lo = 0, n = p.seqs;
  while (n > 1) {
    const int step = (n + 31) / 32, i = lane * step;
    const uint32_t at = __ballot_sync(0xffffffffu, i < n && __ldg(p.q_start + lo + i) <= t);
    const int skip = max(__popc(at) - 1, 0) * step;
    lo += skip;
    n = min(step, n - skip);
  }
  *s = span_of(p, lo);
  return lo;
}
}  // namespace

namespace {
// Where the sums of a row's and head's parts lie.
struct Parts {
  long regular;    // of part 0 among part_ml (times dh: among part_o)
  long piece;      // of the few-row kernel's first piece among piece_ml, -1: none
  int parts1, n;   // parts of the prefix; of all (none: the output is there already)
  long step;       // from part to part
  BAG_DEV long at(int i, bool* whole) const {
    const int k = i - parts1;
    *whole = k < 0 || piece < 0;  // of pieces, the first CTA's starts the unit (1), the others' do not
    return *whole ? regular + i * step : piece + (long)k * 2 * F_ROWS + (k == 0 ? F_ROWS : 0);
  }
};
BAG_DEV Parts parts_of(const PackedParams& p, int seq, const Span& s, int tok, int h) {
  Parts a;
  a.regular = (long)tok * p.heads + h;
  a.step = (long)p.nq * p.heads;
  a.piece = -1;
  a.parts1 = p.parts1;
  int own = 1;
  if (!p.few) {
    own = own_parts(p, s.lk);
  } else if (p.split) {
    const int r = (tok - s.q0) * p.group + h % p.group, blocks = (s.lq * p.group + F_ROWS - 1) / F_ROWS;
    const long length = few_length(s.lk), share = p.place[0];
    const long start = p.place[1 + seq] + ((long)(h / p.group) * blocks + r / F_ROWS) * length;
    const long c0 = start / share, c1 = (start + length - 1) / share;
    if (c1 > c0) {
      own = (int)(c1 - c0) + 1;
      a.piece = c0 * 2 * F_ROWS + r % F_ROWS;
    }
  }
  a.n = p.parts1 == 0 && own <= 1 ? 0 : p.parts1 + own;
  return a;
}
}  // namespace

// Joins the parts of a row and head: their weights first, then DH / 4 lanes a part, in a fixed order.  For few rows
// with many parts.  Bound: latency (28 heads of one token in 76 pieces: 4 to 5 us behind the kernel before).
template <bool F16, int DH>
__global__ void __launch_bounds__(JN_TH) attn_join_kernel(const PackedParams p) {
  constexpr int L = DH / 4, GROUPS = JN_TH / L;
  __shared__ float4 so[GROUPS][L];
  __shared__ float dens[GROUPS], red[JN_TH / 32];
  __shared__ float2 weight[JN_TH];
  __shared__ const float* from[JN_TH];
  grid_dep_sync();
  const int tok = (int)(blockIdx.x / p.heads), h = (int)(blockIdx.x % p.heads);
  Span s;
  const int seq = sequence_of(p, tok, &s);
  if (tok < s.q0 || tok >= s.q0 + s.lq) return;
  const Parts a = parts_of(p, seq, s, tok, h);
  if (a.n == 0) return;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = threadIdx.x / L, x = threadIdx.x % L;
  float top = -INFINITY;
  for (int i = threadIdx.x; i < a.n; i += JN_TH) {
    bool whole;
    const long at = a.at(i, &whole);
    top = fmaxf(top, (whole ? p.part_ml : p.piece_ml)[at].x);
  }
#pragma unroll
  for (int o = 16; o > 0; o /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (lane == 0) red[warp] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < JN_TH / 32; ++i) top = fmaxf(top, red[i]);
  float den = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i0 = 0; i0 < a.n; i0 += JN_TH) {
    if (i0) __syncthreads();
    if (i0 + (int)threadIdx.x < a.n) {  // weights of the next parts (0: no key of the part is seen)
      bool whole;
      const long at = a.at(i0 + threadIdx.x, &whole);
      const float2 f = (whole ? p.part_ml : p.piece_ml)[at];
      from[threadIdx.x] = (whole ? p.part_o : p.piece_o) + at * DH;
      weight[threadIdx.x] = make_float2(part_weight(f, top), f.y);
    }
    __syncthreads();
    const int n = min(JN_TH, a.n - i0);
#pragma unroll 8
    for (int i = g; i < n; i += GROUPS) {
      const float2 f = weight[i];
      const float4 v = *reinterpret_cast<const float4*>(from[i] + 4 * x);
      const bool none = f.y == 0.f;  // then v may be the product of no weight and NaN
      den += f.x * f.y;
      acc.x += none ? 0.f : f.x * v.x;
      acc.y += none ? 0.f : f.x * v.y;
      acc.z += none ? 0.f : f.x * v.z;
      acc.w += none ? 0.f : f.x * v.w;
    }
  }
  so[g][x] = acc;
  if (x == 0) dens[g] = den;
  __syncthreads();
  if (threadIdx.x >= L) return;
  acc = so[0][x];
  den = dens[0];
#pragma unroll
  for (int i = 1; i < GROUPS; ++i) {
    const float4 v = so[i][x];
    den += dens[i];
    acc.x += v.x;
    acc.y += v.y;
    acc.z += v.z;
    acc.w += v.w;
  }
  const float inv = inverse_sum(top, den);
  uint2 u;
  u.x = pack16<F16>(acc.x * inv, acc.y * inv);
  u.y = pack16<F16>(acc.z * inv, acc.w * inv);
  *reinterpret_cast<uint2*>(p.o + tok * p.ldo + (long)h * DH + 4 * x) = u;
  if (p.lse && x == 0) p.lse[(long)tok * p.heads + h] = (top + log2f(den)) * 0.6931471805599453f;
}

// The same for many rows with few parts: a CTA a row and some of its heads, a warp a head at a time, DH / 32 columns
// a lane.  Bound: HBM or L2, which the loads of a CTA's heads reach together (a CTA for each head took 80 us
// of the 130 for 2048 rows x 32 heads in two parts).
template <bool F16, int DH>
__global__ void __launch_bounds__(JR_TH) attn_join_rows_kernel(const PackedParams p) {
  constexpr int C = DH / 32;
  grid_dep_sync();
  const int tok = blockIdx.x, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  Span s;
  const int seq = sequence_of(p, tok, &s);
  if (tok < s.q0 || tok >= s.q0 + s.lq) return;
#pragma unroll 2
  for (int h = blockIdx.y * (JR_TH / 32) + warp; h < p.heads; h += gridDim.y * (JR_TH / 32)) {
    const Parts a = parts_of(p, seq, s, tok, h);
    if (a.n == 0) continue;
    float top = -INFINITY, den = 0.f, acc[C];
#pragma unroll
    for (int i = 0; i < C; ++i) acc[i] = 0.f;
    for (int i0 = 0; i0 < a.n; i0 += 32) {
      const int n = min(32, a.n - i0);
      bool whole = true;
      const long at = a.at(i0 + min(lane, n - 1), &whole);
      const float2 f = (whole ? p.part_ml : p.piece_ml)[at];
      const float* from = (whole ? p.part_o : p.piece_o) + at * DH;
      // four parts' columns at a time, the first ones on their way beside the weights
      float x[4][C];
      auto load = [&](int i) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float* v = reinterpret_cast<const float*>(
                               __shfl_sync(0xffffffffu, reinterpret_cast<uintptr_t>(from), min(i + k, n - 1))) + lane * C;
          if constexpr (C == 4)
            *reinterpret_cast<float4*>(x[k]) = *reinterpret_cast<const float4*>(v);
          else
            *reinterpret_cast<float2*>(x[k]) = *reinterpret_cast<const float2*>(v);
        }
      };
      load(0);
      float m = f.x;  // of 32 parts, then of those before too
#pragma unroll
      for (int o = 16; o > 0; o /= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
      m = fmaxf(m, top);
      const float before = part_weight(make_float2(top, den), m), w = part_weight(f, m);
      top = m;
      den *= before;
#pragma unroll
      for (int i = 0; i < C; ++i) acc[i] *= before;
      for (int i = 0; i < n; i += 4) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float wi = __shfl_sync(0xffffffffu, w, min(i + k, n - 1)), li = __shfl_sync(0xffffffffu, f.y, min(i + k, n - 1));
          if (i + k < n) {
            den += wi * li;
#pragma unroll
            for (int e = 0; e < C; ++e) acc[e] += li == 0.f ? 0.f : wi * x[k][e];  // no weight: x may be NaN
          }
        }
        if (i + 4 < n) load(i + 4);
      }
    }
    const float inv = inverse_sum(top, den);
    uint16_t* o = p.o + tok * p.ldo + (long)h * DH + lane * C;
    if constexpr (C == 4)
      *reinterpret_cast<uint2*>(o) = make_uint2(pack16<F16>(acc[0] * inv, acc[1] * inv), pack16<F16>(acc[2] * inv, acc[3] * inv));
    else
      *reinterpret_cast<uint32_t*>(o) = pack16<F16>(acc[0] * inv, acc[1] * inv);
    if (p.lse && lane == 0) p.lse[(long)tok * p.heads + h] = (top + log2f(den)) * 0.6931471805599453f;
  }
}

namespace {
// The form of a call: own keys by attn_few_kernel or the tensor cores, the prefix with all rows together (parts1)
// or before each sequence's own keys (fused key tiles).
struct Plan {
  int parts1, parts2, chunk1, chunk2;
  int few, split, ctas;       // ctas: of the few-row kernel
  int fused, rows, together;  // rows: of a unit of the tensor-core kernel
};

long cdiv(long a, long b) { return (a + b - 1) / b; }
size_t part_bytes(const PackedArgs& a) { return (size_t)a.nq * (size_t)a.heads * ((size_t)a.dh * 4 + 8); }
size_t piece_bytes(const PackedArgs& a, const Plan& t) {
  return t.split ? (size_t)t.ctas * 2 * F_ROWS * ((size_t)a.dh * 4 + 8) + ((size_t)a.seqs + 1) * 8 : 0;
}
// parts that are kept (with one in all it is the output)
long parts_of(const Plan& t) { return t.parts1 + t.parts2 > 1 ? t.parts1 + t.parts2 : 0; }

// How the rows and keys are cut, with a workspace of at most `bytes`.
Plan plan_of(const PackedArgs& a, size_t bytes) {
  Plan t{};
  const long G = a.heads / a.kv_heads, sms = sm_count();
  const long max_k = std::max(a.max_k, 1L);
  const long max_q = std::max(1L, std::min(a.max_q, a.nq)), rows = a.nq * G;
  const long most = (long)std::min<size_t>(bytes / part_bytes(a), 1u << 30);  // parts
  t.few = max_q * G <= F_ROWS;  // 64 tokens over 8192 keys, 16 heads on one key head 55 us, 32 on one (tensor cores) 67, floor 40
  // heads of a group that share a tile: as many as leave few of its rows empty, or whose rows of a
  // sequence fit one.  More units of a key head read its keys again, and a sequence's last tile is less full: with
  // one of seven heads, 24 prompts behind a prefix take 74 us, with all seven (126 of 128 rows) 46.
  t.together = 1;
  for (int g = 2; g <= G && g <= PT; ++g)
    if (G % g == 0 && (PT / g * g >= PT - PT / 10 || max_q * g <= PT)) t.together = g;
  // The prefix with the rows of all sequences together, or ahead of each one's own keys, by the expected time (ns; a
  // tile of rows against a tile of keys takes 5.4, or 7.8 where a sequence fills one tile only; a unit 25; sums of
  // parts are written and read at 5 TB/s).  64 sequences behind 2048 tokens, 32 / 8 heads: 5, 8, 16, 24 and 32
  // queries each 37, 43, 59, 86 and 102 us together, 71 to 74 apart; 16 of 32 behind 16,384: 112 and 165;
  // 24 of 16 to 300 behind 1003, 28 / 4 heads: 63 and 39.
  bool all_rows = a.n_prefix > 0 && most >= 2;
  const long all_parts = std::max(1L, std::min(cdiv(a.n_prefix, 512), sms / std::max(1L, cdiv(rows, 2 * PT) * a.kv_heads)));
  if (all_rows && !t.few) {
    const double each = (double)cdiv(cdiv(rows, a.seqs), PT), own = (double)a.kv_heads * a.seqs * each;
    const double pre = (double)cdiv(a.n_prefix, PT), keys = (double)cdiv(max_k, PT);
    const double apart = own * (pre + keys) * (each > 1 ? 5.4 : 7.8);
    const double together = (double)a.kv_heads * cdiv(rows, PT) * pre * 5.4 + own * (25.0 + keys * 7.8) +
                            (double)a.nq * a.heads * (8.0 * a.dh + 16.0) * (all_parts + 1) / 5000.0 + 8000.0;
    all_rows = together < apart;
  }
  // units of 256 rows where there are enough of them, or enough keys, and sequences (or the rows of all) fill
  // them: 16 x 512 tokens, 32 / 8 heads 62 us (72 with 128), 512 tokens over 33,000 keys 233 (244); but one prompt
  // of 77 tokens 6.9 (8.3), 512 x 28 / 4 heads 11.7 (12.9), 32 x 8 tokens over up to 8192 keys 49 (65).  Sequences of
  // very different lengths, with 256 and with 128: 32 prompts of 8 to 512 tokens 29 and 31 us, 24 behind a prefix 40
  // and 47, 8 texts in parts 90 and 117, 128 tokens behind 16,384 shared keys 58 and 87
  auto units = [&](long n) { return (rows / n + (a.seqs + 1) / 2) * a.kv_heads; };
  t.rows = (all_rows || max_q * G > PT) &&
                   (units(256) * 2 > sms || units(256) * cdiv(max_k + a.n_prefix, PT) >= 8 * sms) ? 256 : 128;
  if (a.n_prefix && !all_rows) t.few = 0;
  auto chunk = [](long keys, long parts) { return (int)std::min(cdiv(cdiv(keys, parts), PT) * PT, 0x7fffff80L); };
  long p1 = 0, p2 = 1;
  if (all_rows) p1 = t.rows == 2 * PT ? all_parts : std::max(1L, std::min(cdiv(a.n_prefix, 512), sms / std::max(1L, cdiv(rows, PT) * a.kv_heads)));
  t.fused = all_rows ? 0 : (int)cdiv(a.n_prefix, PT);
  const long keys = max_k + (long)t.fused * PT;
  // keys in parts where units are few, four for each SM: 8 texts with 16 to 512 new tokens of up to 16,896 162 -> 106 us
  // (2, 3, 4, 6 and 8 for each SM: 126, 105, 108, 122 and 120), at least 12 key tiles each (2048 tokens in two parts
  // of 8 took 78 us, whole 46: the sums of many rows)
  const long tiles = cdiv(keys, PT);
  if (!t.few && units(t.rows) < 2 * sms)
    p2 = std::max(1L, tiles / std::max(12L, tiles * units(t.rows) / (4 * sms)));
  if (p1 + p2 > most) {
    if (p1) p1 = std::max(1L, std::min(p1, most - 1));
    p2 = std::max(1L, most - p1);
  }
  t.chunk1 = p1 ? chunk(a.n_prefix, p1) : PT;
  t.parts1 = p1 ? (int)cdiv(a.n_prefix, t.chunk1) : 0;
  t.chunk2 = chunk(keys, p2);
  t.parts2 = (int)p2;
  if (t.few) {
    const long units16 = a.seqs * a.kv_heads * cdiv(max_q * G, F_ROWS), slots = sms * (a.dh == 64 ? few_ctas<64>() : few_ctas<128>());
    // equal shares, but for keys too few to be worth a join (2 to 3 us).  Of 32 / 8 heads, in whole units and in equal
    // shares: 64 tokens over 200 keys each 14 and 17 us, 128 over 6 to 200 20 and 17, over 6 to 400 33 and 18
    t.split = max_k > 256;
    t.ctas = (int)std::max(1L, std::min(slots, t.split ? units16 * std::min(cdiv(max_k, 2 * F_TILE), slots) : units16));
    if (t.split && bytes < parts_of(t) * part_bytes(a) + piece_bytes(a, t)) {
      t.split = 0;
      t.ctas = (int)std::min(slots, units16);
    }
  }
  return t;
}
}  // namespace

// A bound of what any call wants whose sizes are at most these (what one call wants is not monotone in them: few
// rows want many parts, many want none), for its parts as plan_of counts them before it rounds.
size_t attention_packed_work(const PackedArgs& a) {
  const long G = a.heads / a.kv_heads, sms = sm_count(), all = a.nq * a.heads;  // rows and heads
  const long max_q = std::max(1L, std::min(a.max_q, a.nq)), max_k = std::max(a.max_k, 1L);
  const long tiles = cdiv(max_k, PT), pre = cdiv(a.n_prefix, PT);
  const bool many = max_q * G > F_ROWS;  // beside calls for the few-row kernel others too
  // Own keys of units of n rows on the tensor cores: p2 <= tiles / 12, and with x = tiles * units / (4 sms), tiles / max(12,
  // floor(x)) < 13 / 12 * 4 sms / units, where n * units >= rows of all key heads.
  auto up_to = [](long times, long rows, long cap) { return rows >= cap ? cap : std::min(times * rows, cap); };  // times >= 1
  auto own = [&](long tiles, long rows, long n) { return many && tiles >= 24 ? up_to(tiles / 12, rows, 13 * sms * n / 3) : 0L; };
  long kept = own(tiles + pre, all, a.n_prefix == 0 && max_q * G <= PT ? PT : 2 * PT);
  if (a.n_prefix) {
    // The prefix with all rows together: few of each sequence, or so many as make that the faster way (writing and reading
    // two parts at least takes less time than the key tiles that it saves, at most one tile of rows a sequence).
    const long some = many ? std::min((double)all, (double)a.kv_heads * a.seqs * std::max((double)F_ROWS, pre * 7.8 * 2500.0 / (8.0 * a.dh + 16.0)))
                           : all;
    const long p1 = std::max(some, up_to(cdiv(a.n_prefix, 512), some, 2 * PT * sms));
    kept = std::max(kept, p1 + std::max(some, own(tiles, some, 2 * PT)));
  }
  size_t bytes = (size_t)kept * ((size_t)a.dh * 4 + 8);
  if (G <= F_ROWS && max_k > 256) {  // equal shares of single tokens' keys
    const long slots = sms * (a.dh == 64 ? few_ctas<64>() : few_ctas<128>());
    Plan t{};
    t.split = 1;
    t.ctas = (int)std::min(slots, a.seqs * a.kv_heads * std::min(cdiv(max_k, 2 * F_TILE), slots));
    bytes += piece_bytes(a, t);
  }
  return bytes;
}

cudaError_t attention_packed(const PackedArgs& a, cudaStream_t s) {
  if (a.nq <= 0 || a.seqs <= 0) return cudaSuccess;
  const Plan t = plan_of(a, a.work_bytes);
  PackedParams p{};
  auto u16 = [](const void* x) { return reinterpret_cast<const uint16_t*>(x); };
  p.q = u16(a.q), p.k = u16(a.k), p.v = u16(a.v), p.pk = u16(a.pk), p.pv = u16(a.pv);
  p.o = reinterpret_cast<uint16_t*>(a.o);
  p.ldq = a.ldq, p.ldk = a.ldk, p.ldv = a.ldv, p.ldpk = a.ldpk, p.ldpv = a.ldpv, p.ldo = a.ldo;
  p.lse = a.lse;
  p.q_start = a.q_start, p.k_start = a.k_start, p.k_len = a.k_len;
  p.nq = (int)a.nq, p.k_rows = (int)a.k_rows, p.n_prefix = (int)a.n_prefix, p.seqs = (int)a.seqs;
  p.heads = a.heads, p.kv_heads = a.kv_heads, p.group = a.heads / a.kv_heads, p.causal = a.causal;
  p.scale_log2 = a.scale_log2;
  p.parts1 = t.parts1, p.parts2 = t.parts2, p.chunk1 = t.chunk1, p.chunk2 = t.chunk2, p.fused = t.fused;
  // the workspace: sums of parts, of pieces, then what is 8 bytes wide
  const size_t kept = (size_t)parts_of(t) * a.nq * a.heads, pieces = t.split ? (size_t)t.ctas * 2 * F_ROWS : 0;
  p.part_o = reinterpret_cast<float*>(a.work);
  p.piece_o = p.part_o + kept * a.dh;
  p.part_ml = reinterpret_cast<float2*>(p.piece_o + pieces * a.dh);
  p.piece_ml = p.part_ml + kept;
  p.place = reinterpret_cast<long*>(p.piece_ml + pieces);
  p.few = t.few, p.split = t.split;
  p.together = t.together, p.tokens = PT / t.together;
  const long per = p.tokens * (t.rows / PT), groups = a.heads / t.together;
  const long slots1 = t.parts1 ? cdiv(a.nq, per) : 0, slots2 = t.few ? 0 : a.nq / per + a.seqs;
  p.err = a.err;
  const long tiles = (slots1 * t.parts1 + slots2 * t.parts2) * groups;
  const long few = t.few ? t.ctas : 0, joins = a.nq * a.heads;
  p.beside = few && tiles;
  if (tiles > 0x7fffffffL || joins > 0x7fffffffL || slots1 > 0x7fffffffL || slots2 > 0x7fffffffL)
    return cudaErrorInvalidConfiguration;
  p.slots1 = (int)slots1, p.slots2 = (int)slots2;
  // all heads of a slot together while the keys of a sequence fit L2: 4608 tokens x 24 heads 123 -> 103 us, 8192 x 24
  // 318 -> 282; not beyond: 16,384 x 24 1099 -> 1140, 32,760 x 40 6390 -> 6530
  p.by_head = (std::min(a.max_k, a.k_rows) + a.n_prefix) * a.kv_heads * a.dh * 4 > (128L << 20);
  CUtensorMap tq, tk, tv, tpk, tpv;
  if (tiles) {
    if (encode_tmap_3d_16(&tq, a.q, (uint64_t)a.dh, (uint64_t)a.heads, (uint64_t)a.nq, (uint64_t)a.dh * 2, (uint64_t)a.ldq * 2,
                          (uint32_t)t.together, (uint32_t)p.tokens))
      return cudaErrorInvalidValue;
    const uint64_t width = (uint64_t)a.kv_heads * a.dh;
    // a tensor without rows is never read: another one stands for its map
    auto map = [&](CUtensorMap* m, const void* x, long ld, long n) {
      return encode_tmap_2d_bf16(m, x, width, (uint64_t)n, (uint64_t)ld * 2, 64, PT) != 0;
    };
    if (a.k_rows && slots2 && (map(&tk, a.k, a.ldk, a.k_rows) || map(&tv, a.v, a.ldv, a.k_rows))) return cudaErrorInvalidValue;
    if (a.n_prefix) {
      if (map(&tpk, a.pk, a.ldpk, a.n_prefix) || map(&tpv, a.pv, a.ldpv, a.n_prefix)) return cudaErrorInvalidValue;
      if (!a.k_rows || !slots2) tk = tpk, tv = tpv;
    } else {
      if (!a.k_rows && (map(&tk, a.q, a.ldq, a.nq) || map(&tv, a.q, a.ldq, a.nq))) return cudaErrorInvalidValue;
      tpk = tk, tpv = tv;
    }
  }
  auto launch = [&](auto f16, auto width) {
    constexpr bool F16 = decltype(f16)::value;
    constexpr int DH = decltype(width)::value;
    cudaError_t e = cudaSuccess;
    if (few) e = launch_kernel(attn_few_kernel<F16, DH>, (unsigned)few, F_TH, few_smem<DH>(), s, p);
    if (tiles && e == cudaSuccess)
      e = t.rows == 256 ? launch_kernel(attn_packed_kernel<F16, DH, 2>, (unsigned)tiles, Pt<DH, 2>::THREADS,
                                        Pt<DH, 2>::BYTES, s, tq, tk, tv, tpk, tpv, p)
                        : launch_kernel(attn_packed_kernel<F16, DH, 1>, (unsigned)tiles, Pt<DH, 1>::THREADS,
                                        Pt<DH, 1>::BYTES, s, tq, tk, tv, tpk, tpv, p);
    if (e == cudaSuccess && (parts_of(t) || t.split))
      e = joins >= 4L * sm_count()
              ? launch_kernel(attn_join_rows_kernel<F16, DH>,
                              dim3((unsigned)a.nq, (unsigned)std::max(1L, std::min(cdiv(a.heads, 8), 8L * sm_count() / a.nq))),
                              JR_TH, 0, s, p)
              : launch_kernel(attn_join_kernel<F16, DH>, (unsigned)joins, JN_TH, 0, s, p);
    return e;
  };
  using Wide = std::integral_constant<int, 128>;
  using Narrow = std::integral_constant<int, 64>;
  if (a.dh == 128) return a.f16 ? launch(std::true_type{}, Wide{}) : launch(std::false_type{}, Wide{});
  return a.f16 ? launch(std::true_type{}, Narrow{}) : launch(std::false_type{}, Narrow{});
}

cudaError_t attention_packed_init() {
  cudaError_t r = cudaSuccess;
  auto smem = [&](auto kernel, int bytes) {
    if (r == cudaSuccess) r = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  };
  smem(attn_few_kernel<true, 128>, few_smem<128>());
  smem(attn_few_kernel<false, 128>, few_smem<128>());
  smem(attn_few_kernel<true, 64>, few_smem<64>());
  smem(attn_few_kernel<false, 64>, few_smem<64>());
  smem(attn_packed_kernel<true, 128, 1>, Pt<128, 1>::BYTES);
  smem(attn_packed_kernel<false, 128, 1>, Pt<128, 1>::BYTES);
  smem(attn_packed_kernel<true, 64, 1>, Pt<64, 1>::BYTES);
  smem(attn_packed_kernel<false, 64, 1>, Pt<64, 1>::BYTES);
  smem(attn_packed_kernel<true, 128, 2>, Pt<128, 2>::BYTES);
  smem(attn_packed_kernel<false, 128, 2>, Pt<128, 2>::BYTES);
  smem(attn_packed_kernel<true, 64, 2>, Pt<64, 2>::BYTES);
  smem(attn_packed_kernel<false, 64, 2>, Pt<64, 2>::BYTES);
  return r;
}

}  // namespace bag
