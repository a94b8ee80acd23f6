// Attention of packed sequences over their own rows of a key-value cache, behind a prefix that all of
// them share (heads of 64 or 128, 16-bit operands, grouped heads).
//
//   o_t = sum_j w_tj v_j / sum_j w_tj,  w_tj = exp(c q_t . k_j),
//
// over the prefix's keys and the own keys j <= t + lk - lq.  Sums over parts of the keys are kept as
// (m, l, O) with l = sum 2^(s - m), O = sum 2^(s - m) v, s in log2 units; parts are joined by
// m = max m_i, l = sum 2^(m_i - m) l_i, O likewise.
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
  // parts of the keys: parts1 of the prefix, chunk1 keys each, then own_parts() of a sequence, chunk2 keys each.
  // Part i of row t and head h: part_o[((i * nq + t) * heads + h) * dh ...], part_ml likewise.
  int parts1, parts2, chunk1, chunk2;
  float* part_o;
  float2* part_ml;
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
  return (int)min(((long)lk + p.chunk2 - 1) / p.chunk2, (long)p.parts2);
}

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

constexpr int F_WARPS = 8, F_TH = 32 * F_WARPS;
constexpr int F_KEYS = 16;  // of a warp's step
template <int DH>
constexpr int few_smem() {
  return F_WARPS * 16 * (DH + 4) * 4 + F_WARPS * 16 * 8;
}
}  // namespace

// Up to 16 rows (query token, head of the group) at a time against keys in registers: a warp takes 16
// keys a step.  A key's 16-byte pieces go from global memory straight into the B operands of
// mma.m16n8k16: the order of a contraction is free, so lane (n, c) holds head columns 32 j + 8 c .. + 7 of
// key n for Q K^T (the rows of Q are loaded in the same order), and columns 64 u + 8 n .. + 7 of keys 2 c,
// 2 c + 1, 2 c + 8 and 2 c + 9 for P V, whose pairs of keys a byte permutation makes; its column n of
// product t is then head column 64 u + 8 n + t, and a lane ends with runs of 8 columns of the output.
// Keys past the last are loaded as zeros (whatever lies there, NaN included).
template <bool F16, int DH>
__global__ void __launch_bounds__(F_TH, 1) attn_few_kernel(const PackedParams p) {
  extern __shared__ __align__(16) uint8_t smem[];
  constexpr int LD = DH + 4, U = DH / 64, J = DH / 32;
  float* so = reinterpret_cast<float*>(smem);                                      // [F_WARPS][16][LD]
  float2* sml = reinterpret_cast<float2*>(smem + F_WARPS * 16 * LD * 4);           // [F_WARPS][16]
  grid_dep_sync();
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, n = lane >> 2, c = lane & 3;
  const int G = p.group;
  long unit = blockIdx.x;
  const int head = (int)(unit % p.kv_heads);
  unit /= p.kv_heads;
  const bool prefix = unit < p.parts1;
  int part;       // index of the part
  int k_lo, k_hi; // its keys
  bool direct = false;
  Span s;
  const uint16_t *kb, *vb;
  long ldk, ldv;
  if (prefix) {
    s = span_all(p);
    part = (int)unit;
    k_lo = min((long)part * p.chunk1, (long)s.lk);
    k_hi = min((long)k_lo + p.chunk1, (long)s.lk);
    kb = p.pk, vb = p.pv, ldk = p.ldpk, ldv = p.ldpv;
  } else {
    unit -= p.parts1;
    s = span_of(p, (int)(unit / p.parts2));
    const int own = (int)(unit % p.parts2), parts = own_parts(p, s.lk);
    if (own >= (p.parts1 ? parts : max(parts, 1))) return;
    direct = p.parts1 == 0 && parts <= 1;
    part = p.parts1 + own;
    k_lo = (int)min((long)own * p.chunk2, (long)s.lk);
    k_hi = own == p.parts2 - 1 ? s.lk : (int)min((long)k_lo + p.chunk2, (long)s.lk);
    kb = p.k + s.k0 * p.ldk, vb = p.v + s.k0 * p.ldv, ldk = p.ldk, ldv = p.ldv;
  }
  kb += head * DH;
  vb += head * DH;
  const long R = (long)s.lq * G;
  // keys that row r of this part sees end before
  auto limit = [&](long r) {
    if (r >= R) return k_lo;
    if (prefix || !p.causal) return k_hi;
    return (int)min(max(r / G + 1 + s.lk - s.lq, (long)k_lo), (long)k_hi);
  };
  for (long r0 = 0; r0 < R; r0 += 16) {
    uint4 qa[2][J];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const long r = r0 + n + 8 * i;
      const uint16_t* at = p.q + (s.q0 + r / G) * p.ldq + (head * G + r % G) * DH;
#pragma unroll
      for (int j = 0; j < J; ++j) qa[i][j] = r < R ? __ldg(reinterpret_cast<const uint4*>(at + 32 * j + 8 * c)) : make_uint4(0, 0, 0, 0);
    }
    const int lim[2] = {limit(r0 + n), limit(r0 + n + 8)};
    const int end = limit(min(r0 + 15, R - 1));  // the last row sees most
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, o[U * 8][4];
#pragma unroll
    for (int i = 0; i < U * 8; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[i][e] = 0.f;
    uint4 kf[2][J], vf[4][U];
    auto load_k = [&](int k0) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int key = k0 + 8 * t + n;
#pragma unroll
        for (int j = 0; j < J; ++j)
          kf[t][j] = key < end ? ld_stream(kb + key * ldk + 32 * j + 8 * c) : make_uint4(0, 0, 0, 0);
      }
    };
    auto load_v = [&](int k0) {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int key = k0 + 2 * c + (t & 1) + 8 * (t >> 1);
#pragma unroll
        for (int u = 0; u < U; ++u)
          vf[t][u] = key < end ? ld_stream(vb + key * ldv + 64 * u + 8 * n) : make_uint4(0, 0, 0, 0);
      }
    };
    constexpr int STEP = F_WARPS * F_KEYS;
    int k0 = k_lo + warp * F_KEYS;
    if (k0 < end) {
      load_k(k0);
      load_v(k0);
    }
    for (; k0 < end; k0 += STEP) {
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
      if (k0 + STEP < end) load_k(k0 + STEP);
      bool moved = false;
      float alpha[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            if (k0 + 8 * t + 2 * c + e >= lim[i]) sc[t][2 * i + e] = -INFINITY;
        float mx = fmaxf(fmaxf(sc[0][2 * i], sc[0][2 * i + 1]), fmaxf(sc[1][2 * i], sc[1][2 * i + 1]));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2)) * p.scale_log2;
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
            const float w = ex2(fmaf(sc[t][2 * i + e], p.scale_log2, neg));
            l[i] += w;
            sc[t][2 * i + e] = w;
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
      const uint32_t a0 = pack16<F16>(sc[0][0], sc[0][1]), a1 = pack16<F16>(sc[0][2], sc[0][3]),
                     a2 = pack16<F16>(sc[1][0], sc[1][1]), a3 = pack16<F16>(sc[1][2], sc[1][3]);
#pragma unroll
      for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int t = 0; t < 8; ++t) {
          auto word = [&](const uint4& v) { return t < 2 ? v.x : (t < 4 ? v.y : (t < 6 ? v.z : v.w)); };
          const uint32_t sel = t & 1 ? 0x7632u : 0x5410u;
          mma16816<F16>(o[u * 8 + t], a0, a1, a2, a3, __byte_perm(word(vf[0][u]), word(vf[1][u]), sel),
                        __byte_perm(word(vf[2][u]), word(vf[3][u]), sel));
        }
      }
      if (k0 + STEP < end) load_v(k0 + STEP);
    }
    // the warps' parts
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
      l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
      if (c == 0) sml[warp * 16 + n + 8 * i] = make_float2(m[i], l[i]);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < F_WARPS; ++w) top = fmaxf(top, sml[w * 16 + n + 8 * i].x);
      const float f = m[i] == -INFINITY ? 0.f : ex2(m[i] - top);
      float* row = so + (warp * 16 + n + 8 * i) * LD;
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
    for (int it = threadIdx.x; it < 16 * (DH / 8); it += F_TH) {
      const int lr = it / (DH / 8), col = it % (DH / 8) * 8;
      const long r = r0 + lr;
      if (r >= R) continue;
      float top = -INFINITY, den = 0.f, v[8];
#pragma unroll
      for (int w = 0; w < F_WARPS; ++w) top = fmaxf(top, sml[w * 16 + lr].x);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = 0.f;
#pragma unroll
      for (int w = 0; w < F_WARPS; ++w) {
        const float2 f = sml[w * 16 + lr];
        den += f.x == -INFINITY ? 0.f : ex2(f.x - top) * f.y;
        const float* row = so + (w * 16 + lr) * LD + col;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += row[e];
      }
      const long tok = s.q0 + r / G;
      const int h = head * G + (int)(r % G);
      if (direct) {
        const float inv = top == -INFINITY ? 0.f : 1.f / den;
        uint4 w;
        w.x = pack16<F16>(v[0] * inv, v[1] * inv);
        w.y = pack16<F16>(v[2] * inv, v[3] * inv);
        w.z = pack16<F16>(v[4] * inv, v[5] * inv);
        w.w = pack16<F16>(v[6] * inv, v[7] * inv);
        *reinterpret_cast<uint4*>(p.o + tok * p.ldo + (long)h * DH + col) = w;
        if (p.lse && col == 0) p.lse[tok * p.heads + h] = (top + log2f(den)) * 0.6931471805599453f;
      } else {
        const long at = ((long)part * p.nq + tok) * p.heads + h;
        float4* d = reinterpret_cast<float4*>(p.part_o + at * DH + col);
        d[0] = make_float4(v[0], v[1], v[2], v[3]);
        d[1] = make_float4(v[4], v[5], v[6], v[7]);
        if (col == 0) p.part_ml[at] = make_float2(top, den);
      }
    }
    __syncthreads();
  }
}

namespace {
constexpr int JN_TH = 128;

// The sequence of query row t: the last one that starts at or before it.  Called by a whole warp.
BAG_DEV int sequence_of(const PackedParams& p, int t) {
  const int lane = threadIdx.x % 32;
  int lo = 0, n = p.seqs;
  while (n > 1) {
    const int step = (n + 31) / 32, i = lane * step;
    const uint32_t at = __ballot_sync(0xffffffffu, i < n && __ldg(p.q_start + lo + i) <= t);
    const int skip = max(__popc(at) - 1, 0) * step;
    lo += skip;
    n = min(step, n - skip);
  }
  return lo;
}
}  // namespace

// Joins the parts of a row and head: DH / 4 lanes a part, in turn over the parts, in a fixed order.
template <bool F16, int DH>
__global__ void __launch_bounds__(JN_TH) attn_join_kernel(const PackedParams p) {
  constexpr int L = DH / 4, GROUPS = JN_TH / L;
  __shared__ float4 so[GROUPS][L];
  __shared__ float2 sml[GROUPS];
  grid_dep_sync();
  const int tok = (int)(blockIdx.x / p.heads), h = (int)(blockIdx.x % p.heads);
  const Span s = span_of(p, sequence_of(p, tok));
  if (tok < s.q0 || tok >= s.q0 + s.lq) return;
  const int own = own_parts(p, s.lk), parts = p.parts1 + own;
  if (p.parts1 == 0 && own <= 1) return;  // written by its only part
  const int g = threadIdx.x / L, x = threadIdx.x % L;
  float m = -INFINITY, l = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i = g; i < parts; i += GROUPS) {
    const long at = ((long)i * p.nq + tok) * p.heads + h;
    const float2 f = p.part_ml[at];
    const float4 v = *reinterpret_cast<const float4*>(p.part_o + at * DH + 4 * x);
    if (f.x == -INFINITY) continue;
    const float top = fmaxf(m, f.x), a = m == -INFINITY ? 0.f : ex2(m - top), b = ex2(f.x - top);
    m = top;
    l = l * a + f.y * b;
    acc.x = acc.x * a + v.x * b;
    acc.y = acc.y * a + v.y * b;
    acc.z = acc.z * a + v.z * b;
    acc.w = acc.w * a + v.w * b;
  }
  so[g][x] = acc;
  if (x == 0) sml[g] = make_float2(m, l);
  __syncthreads();
  if (threadIdx.x >= L) return;
  float top = -INFINITY, den = 0.f;
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) top = fmaxf(top, sml[i].x);
  acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int i = 0; i < GROUPS; ++i) {
    const float w = sml[i].x == -INFINITY ? 0.f : ex2(sml[i].x - top);
    const float4 v = so[i][x];
    den += w * sml[i].y;
    acc.x += w * v.x;
    acc.y += w * v.y;
    acc.z += w * v.z;
    acc.w += w * v.w;
  }
  const float inv = top == -INFINITY ? 0.f : 1.f / den;
  uint2 u;
  u.x = pack16<F16>(acc.x * inv, acc.y * inv);
  u.y = pack16<F16>(acc.z * inv, acc.w * inv);
  *reinterpret_cast<uint2*>(p.o + tok * p.ldo + (long)h * DH + 4 * x) = u;
  if (p.lse && x == 0) p.lse[(long)tok * p.heads + h] = (top + log2f(den)) * 0.6931471805599453f;
}

namespace {
struct Plan {
  int parts1, parts2, chunk1, chunk2;
};

size_t part_bytes(const PackedArgs& a) { return (size_t)a.nq * (size_t)a.heads * ((size_t)a.dh * 4 + 8); }

// How the keys are cut, with at most `most` parts in all.
Plan plan_of(const PackedArgs& a, long most) {
  Plan t{};
  auto chunk = [](long keys, long parts) { return (int)((keys + parts * F_KEYS - 1) / (parts * F_KEYS) * F_KEYS); };
  const long max_k = std::min(std::max(a.max_k, 1L), std::max(a.k_rows, 1L));
  auto want = [&](long keys, long units) {
    return std::max(1L, std::min((keys + 255) / 256, 4L * sm_count() / std::max(1L, units)));
  };
  long p1 = a.n_prefix ? want(a.n_prefix, a.kv_heads) : 0;
  long p2 = want(max_k, a.seqs * a.kv_heads);
  if (p1 + p2 > most) {
    if (p1) p1 = std::max(1L, std::min(p1, most - 1));
    p2 = std::max(1L, most - p1);
  }
  t.chunk1 = p1 ? chunk(a.n_prefix, p1) : F_KEYS;
  t.parts1 = p1 ? (int)((a.n_prefix + t.chunk1 - 1) / t.chunk1) : 0;
  t.chunk2 = chunk(max_k, p2);
  t.parts2 = (int)p2;
  return t;
}
}  // namespace

size_t attention_packed_work(const PackedArgs& a, size_t* least) {
  const Plan t = plan_of(a, 1L << 30);
  const size_t one = part_bytes(a);
  *least = t.parts1 ? 2 * one : 0;
  return t.parts1 + t.parts2 > 1 ? (size_t)(t.parts1 + t.parts2) * one : 0;
}

cudaError_t attention_packed(const PackedArgs& a, cudaStream_t s) {
  if (a.nq <= 0 || a.seqs <= 0) return cudaSuccess;
  const size_t one = part_bytes(a);
  const long most = (long)std::min<size_t>(a.work_bytes / one, 1u << 30);
  const Plan t = plan_of(a, most);
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
  p.parts1 = t.parts1, p.parts2 = t.parts2, p.chunk1 = t.chunk1, p.chunk2 = t.chunk2;
  p.part_o = reinterpret_cast<float*>(a.work);
  p.part_ml = reinterpret_cast<float2*>(p.part_o + (size_t)(t.parts1 + t.parts2) * a.nq * a.heads * a.dh);
  const long units = (t.parts1 + a.seqs * t.parts2) * a.kv_heads, joins = a.nq * a.heads;
  if (units > 0x7fffffffL || joins > 0x7fffffffL) return cudaErrorInvalidConfiguration;
  auto launch = [&](auto few, auto join, int smem) {
    cudaError_t e = launch_kernel(few, (unsigned)units, F_TH, smem, s, p);
    if (e == cudaSuccess && t.parts1 + t.parts2 > 1) e = launch_kernel(join, (unsigned)joins, JN_TH, 0, s, p);
    return e;
  };
  if (a.dh == 128)
    return a.f16 ? launch(attn_few_kernel<true, 128>, attn_join_kernel<true, 128>, few_smem<128>())
                 : launch(attn_few_kernel<false, 128>, attn_join_kernel<false, 128>, few_smem<128>());
  return a.f16 ? launch(attn_few_kernel<true, 64>, attn_join_kernel<true, 64>, few_smem<64>())
               : launch(attn_few_kernel<false, 64>, attn_join_kernel<false, 64>, few_smem<64>());
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
  return r;
}

}  // namespace bag
