// Rotary positions of queries and keys on their way into attention and a key-value cache.
//
// Pair i of a head turns by the angle position * f_i.  The host hands f_i over as turns a position, a
// 64-bit fraction F_i of a turn: the low 64 bits of position * F_i are the angle modulo a turn, exactly
// but for F_i's own rounding (2^-65 turns a position, 2^-34 at position 2^31), so far positions lose
// nothing and nothing is computed in fp64.  Its nearest quarter turn is taken off in integers; what is left, at
// most an eighth of a turn, becomes fp32 with 24 bits of its own whatever its size (slow pairs at near
// positions turn by very little), and sine and cosine (sincospif) are swapped and signed by the quarter.
// A CTA computes a row's table once, in shared memory, for all heads; then a
// thread keeps the entries of its V pairs in registers and walks the heads.
// Bound: HBM (each element read and written once): 32,760 rows of 40 + 40 heads of 128, bf16, 196.6 us (100 % of the
// copy rate), 6111 rows of 32 + 8 + 8 heads, half of each rotated, into slots 25.7 (floor 22).  With loads only as
// the stores before them allowed 237 and 39 us.
#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "kernels.h"

namespace bag {

namespace {
constexpr int R_TH = 256, R_HEADS = 2;

template <typename T>
BAG_DEV float r_in(T x);
template <>
BAG_DEV float r_in(float x) { return x; }
template <>
BAG_DEV float r_in(__half x) { return __half2float(x); }
template <>
BAG_DEV float r_in(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T>
BAG_DEV T r_out(float x);
template <>
BAG_DEV float r_out(float x) { return x; }
template <>
BAG_DEV __half r_out(float x) { return __float2half_rn(x); }
template <>
BAG_DEV __nv_bfloat16 r_out(float x) { return __float2bfloat16_rn(x); }

// V elements that are loaded and stored at once: 16 bytes, kept as words, or one.
template <typename T, int V>
struct Elems {
  uint4 w;
  BAG_DEV void load(const T* p) { w = *reinterpret_cast<const uint4*>(p); }
  BAG_DEV void store(T* p) const { *reinterpret_cast<uint4*>(p) = w; }
  BAG_DEV void get(float* e) const {
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) {
        e[i] = __uint_as_float(v[i]);
      } else if constexpr (std::is_same_v<T, __half>) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&v[i]));
        e[2 * i] = f.x;
        e[2 * i + 1] = f.y;
      } else {  // bf16: the upper half of an fp32 word
        e[2 * i] = __uint_as_float(v[i] << 16);
        e[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
      }
    }
  }
  BAG_DEV void set(const float* e) {
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4)
        v[i] = __float_as_uint(e[i]);
      else if constexpr (std::is_same_v<T, __half>)
        v[i] = pack_f16x2(e[2 * i], e[2 * i + 1]);
      else
        v[i] = pack_bf16x2(e[2 * i], e[2 * i + 1]);
    }
    w = make_uint4(v[0], v[1], v[2], v[3]);
  }
};
template <typename T>
struct Elems<T, 1> {
  T w;
  BAG_DEV void load(const T* p) { w = *p; }
  BAG_DEV void store(T* p) const { *p = w; }
  BAG_DEV void get(float* e) const { e[0] = r_in(w); }
  BAG_DEV void set(const float* e) { w = r_out<T>(e[0]); }
};
}  // namespace

// A head is taken in chunks of 2 V elements, V pairs (their first and second elements, or the elements in turn)
// or V and V columns past the rotated ones; a thread has one chunk of a row, and some of its heads.  rows_cta
// rows a CTA, each by R_TH / rows_cta threads.  The first heads are on their way while the table is made.
// Output elements may be the input's own (in place), so the loads of R_HEADS heads go ahead of their stores by hand.
template <typename T, int V, bool HALF>
__global__ void __launch_bounds__(R_TH, 4) rope_kernel(const __grid_constant__ RopeArgs a) {
  __shared__ __align__(16) float2 table[R_TH];  // [rows_cta][pairs]
  grid_dep_sync();
  using E = Elems<T, V>;
  const long row0 = (long)blockIdx.x * a.rows_cta;
  const int per_row = R_TH / a.rows_cta, chunks = a.dh / (2 * V), lanes = per_row / chunks;
  const int lr = threadIdx.x / per_row, at = threadIdx.x - lr * per_row;
  const int hl = at / chunks, chunk = at - hl * chunks;
  const long row = row0 + lr;
  const bool works = row < a.rows && hl < lanes, turns = chunk * V < a.pairs;
  // heads in turn: those of q, of k, of v
  const int nq = a.q ? a.heads : 0, nk = a.k ? a.kv_heads : 0, nh = nq + nk + (a.v ? a.kv_heads : 0);
  // a thread's two vectors of a head
  const int o0 = turns ? (HALF ? chunk * V : 2 * chunk * V) : 2 * chunk * V;
  const int o1 = turns && HALF ? a.pairs + chunk * V : (2 * chunk + 1) * V;
  auto source = [&](int h) {
    if (h < nq) return reinterpret_cast<const T*>(a.q) + row * a.ldq + (long)h * a.dh;
    if (h < nq + nk) return reinterpret_cast<const T*>(a.k) + row * a.ldk + (long)(h - nq) * a.dh;
    return reinterpret_cast<const T*>(a.v) + row * a.ldv + (long)(h - nq - nk) * a.dh;
  };
  E u[R_HEADS], w[R_HEADS];
  auto load = [&](int h0) {
#pragma unroll
    for (int i = 0; i < R_HEADS; ++i) {
      const int h = h0 + i * lanes;
      if (h < nh) {
        const T* x = source(h);
        u[i].load(x + o0);
        w[i].load(x + o1);
      }
    }
  };
  if (works) load(hl);
  long kv_row = row;
  if (works && a.slots) kv_row = __ldg(a.slots + row);
  for (int i = threadIdx.x; i < a.rows_cta * a.pairs; i += R_TH) {
    const int r = i / a.pairs, pair = i - r * a.pairs;
    if (row0 + r < a.rows) {
      const uint64_t pos = (uint64_t)(a.pos ? (long)__ldg(a.pos + row0 + r) : a.pos0 + row0 + r);
      const uint64_t angle = pos * a.turns[pair];
      const uint64_t quarter = (angle + (1ull << 61)) >> 62;  // the nearest, 0 to 3
      const float half_turns = (float)(int64_t)(angle - (quarter << 62)) * 0x1p-63f;  // [-1/4, 1/4]
      float s, c;
      sincospif(half_turns, &s, &c);
      const float cos = quarter & 1 ? s : c, sin = quarter & 1 ? c : s;
      table[i] = make_float2((quarter == 1 || quarter == 2 ? -cos : cos) * a.scale,
                             ((quarter >= 2) != (a.inverse != 0) ? -sin : sin) * a.scale);
    }
  }
  __syncthreads();
  if (!works) return;
  const bool kept = kv_row >= 0 && kv_row < a.capacity;  // the row has a place in the cache
  float c[V], s[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float2 t = turns ? table[lr * a.pairs + chunk * V + i] : make_float2(1.f, 0.f);
    c[i] = t.x;
    s[i] = t.y;
  }
  for (int h0 = hl; h0 < nh; h0 += R_HEADS * lanes) {
#pragma unroll
    for (int i = 0; i < R_HEADS; ++i) {
      const int h = h0 + i * lanes;
      if (h >= nh) continue;
      T* y;
      if (h < nq)
        y = reinterpret_cast<T*>(a.q_out) + row * a.ldqo + (long)h * a.dh;
      else if (!kept)
        continue;
      else if (h < nq + nk)
        y = reinterpret_cast<T*>(a.k_out) + kv_row * a.ldko + (long)(h - nq) * a.dh;
      else
        y = reinterpret_cast<T*>(a.v_out) + kv_row * a.ldvo + (long)(h - nq - nk) * a.dh;
      if (turns && h < nq + nk) {
        float e[2 * V];
        u[i].get(e);
        w[i].get(e + V);
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const int i0 = HALF ? k : 2 * k, i1 = HALF ? V + k : 2 * k + 1;
          const float p = e[i0], q = e[i1];
          e[i0] = p * c[k] - q * s[k];
          e[i1] = p * s[k] + q * c[k];
        }
        u[i].set(e);
        w[i].set(e + V);
      }
      u[i].store(y + o0);
      w[i].store(y + o1);
    }
    if (h0 + R_HEADS * lanes < nh) load(h0 + R_HEADS * lanes);
  }
}

cudaError_t rope(RopeArgs a, int size, int f16, cudaStream_t s) {
  if (a.rows <= 0) return cudaSuccess;
  const int v = 16 / size;
  auto fits = [&](const void* p, long ld) {
    return !p || ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * size)) & 15) == 0;
  };
  const bool vec = a.pairs % v == 0 && a.dh % (2 * v) == 0 && fits(a.q, a.ldq) && fits(a.q_out, a.ldqo) && fits(a.k, a.ldk) &&
                   fits(a.k_out, a.ldko) && fits(a.v, a.ldv) && fits(a.v_out, a.ldvo);
  // few rows: one a CTA, so that they spread over the SMs
  a.rows_cta = 1;
  const int chunks = vec ? a.dh / (2 * v) : (a.dh + 1) / 2;
  if (a.rows >= 4L * sm_count())
    while (a.rows_cta < 4 && 2 * a.rows_cta * std::max(a.pairs, chunks) <= R_TH) a.rows_cta *= 2;
  const long ctas = (a.rows + a.rows_cta - 1) / a.rows_cta;
  if (ctas > 0x7fffffffL) return cudaErrorInvalidConfiguration;
  auto launch = [&](auto kernel) { return launch_kernel(kernel, (unsigned)ctas, R_TH, 0, s, a); };
  auto pick = [&](auto type, auto wide) {
    using T = decltype(type);
    constexpr int V = decltype(wide)::value;
    return a.half ? launch(rope_kernel<T, V, true>) : launch(rope_kernel<T, V, false>);
  };
  using One = std::integral_constant<int, 1>;
  if (size == 4) return vec ? pick(float{}, std::integral_constant<int, 4>{}) : pick(float{}, One{});
  if (f16) return vec ? pick(__half{}, std::integral_constant<int, 8>{}) : pick(__half{}, One{});
  return vec ? pick(__nv_bfloat16{}, std::integral_constant<int, 8>{}) : pick(__nv_bfloat16{}, One{});
}

}  // namespace bag
