// Rotary positions of queries and keys on their way into attention and a key-value cache.
//
// Pair i of a head turns by the angle position * f_i.  The host hands f_i over as turns a position, a
// 64-bit fraction F_i of a turn: the low 64 bits of position * F_i are the angle modulo a turn, exactly
// but for F_i's own rounding (2^-65 turns a position, 2^-34 at position 2^31), so far positions lose
// nothing and nothing is computed in fp64.  Its upper 32 bits, as a signed fraction of a turn, give sine
// and cosine (sincospif).  A CTA computes a row's table once, in shared memory, for all heads; then a
// thread keeps the entries of its V pairs in registers and walks the heads.
// Bound: HBM (each element read and written once).
#include "common.cuh"
#include "kernels.h"

namespace bag {

namespace {
constexpr int R_TH = 256;

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

// V elements that are loaded and stored at once
template <typename T, int V>
struct alignas(sizeof(T) * V) Elems {
  T e[V];
};
}  // namespace

// V: pairs of a thread's chunk (16 bytes of elements, or 1).  rows_cta rows a CTA, each by R_TH / rows_cta
// threads.
template <typename T, int V, bool HALF>
__global__ void __launch_bounds__(R_TH) rope_kernel(const __grid_constant__ RopeArgs a) {
  __shared__ __align__(16) float2 table[R_TH];  // [rows_cta][pairs]
  grid_dep_sync();
  const long row0 = (long)blockIdx.x * a.rows_cta;
  for (int i = threadIdx.x; i < a.rows_cta * a.pairs; i += R_TH) {
    const int lr = i / a.pairs, pair = i - lr * a.pairs;
    const long row = row0 + lr;
    if (row < a.rows) {
      const uint64_t pos = (uint64_t)(a.pos ? (long)__ldg(a.pos + row) : a.pos0 + row);
      const uint64_t angle = pos * a.turns[pair];
      const float u = (float)(int)((angle + 0x80000000ull) >> 32) * 0x1p-31f;  // half turns, [-1, 1]
      float s, c;
      sincospif(u, &s, &c);
      table[i] = make_float2(c * a.scale, (a.inverse ? -s : s) * a.scale);
    }
  }
  __syncthreads();
  const int per_row = R_TH / a.rows_cta, chunks = a.pairs / V, lanes = per_row / chunks;
  const int lr = threadIdx.x / per_row, at = threadIdx.x - lr * per_row;
  const long row = row0 + lr;
  if (row >= a.rows) return;
  long kv_row = row;
  bool kept = true;  // the row has a place in the cache
  if (a.slots) {
    kv_row = __ldg(a.slots + row);
    kept = kv_row >= 0 && kv_row < a.capacity;
  }
  // heads in turn: those of q, of k, of v
  const int nq = a.q ? a.heads : 0, nk = a.k && kept ? a.kv_heads : 0, nv = a.v && kept ? a.kv_heads : 0;
  auto place = [&](int h, const T*& x, T*& y) {
    if (h < nq) {
      x = reinterpret_cast<const T*>(a.q) + row * a.ldq + (long)h * a.dh;
      y = reinterpret_cast<T*>(a.q_out) + row * a.ldqo + (long)h * a.dh;
    } else if (h < nq + nk) {
      x = reinterpret_cast<const T*>(a.k) + row * a.ldk + (long)(h - nq) * a.dh;
      y = reinterpret_cast<T*>(a.k_out) + kv_row * a.ldko + (long)(h - nq) * a.dh;
    } else {
      x = reinterpret_cast<const T*>(a.v) + row * a.ldv + (long)(h - nq - nk) * a.dh;
      y = reinterpret_cast<T*>(a.v_out) + kv_row * a.ldvo + (long)(h - nq - nk) * a.dh;
    }
  };
  using E = Elems<T, V>;
  const int hl = at / chunks, chunk = at - hl * chunks;
  if (hl < lanes) {
    float c[V], s[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float2 t = table[lr * a.pairs + chunk * V + i];
      c[i] = t.x;
      s[i] = t.y;
    }
    // a thread's two vectors of a head: the pairs' first and second elements, or their elements in turn
    const int o0 = HALF ? chunk * V : 2 * chunk * V, o1 = HALF ? a.pairs + chunk * V : (2 * chunk + 1) * V;
#pragma unroll 4
    for (int h = hl; h < nq + nk + nv; h += lanes) {
      const T* x;
      T* y;
      place(h, x, y);
      E u = *reinterpret_cast<const E*>(x + o0), w = *reinterpret_cast<const E*>(x + o1);
      if (h < nq + nk) {
        float e[2 * V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          e[i] = r_in(u.e[i]);
          e[V + i] = r_in(w.e[i]);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const int i0 = HALF ? i : 2 * i, i1 = HALF ? V + i : 2 * i + 1;
          const float p = e[i0], q = e[i1];
          e[i0] = p * c[i] - q * s[i];
          e[i1] = p * s[i] + q * c[i];
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
          u.e[i] = r_out<T>(e[i]);
          w.e[i] = r_out<T>(e[V + i]);
        }
      }
      *reinterpret_cast<E*>(y + o0) = u;
      *reinterpret_cast<E*>(y + o1) = w;
    }
  }
  // columns past the rotated ones
  const int rest = (a.dh - 2 * a.pairs) / V;
  for (int i = at; i < rest * (nq + nk + nv); i += per_row) {
    const int h = i / rest, col = 2 * a.pairs + (i - h * rest) * V;
    const T* x;
    T* y;
    place(h, x, y);
    if (x != y) *reinterpret_cast<E*>(y + col) = *reinterpret_cast<const E*>(x + col);
  }
}

cudaError_t rope(RopeArgs a, int size, int f16, cudaStream_t s) {
  if (a.rows <= 0) return cudaSuccess;
  const int v = 16 / size;
  auto fits = [&](const void* p, long ld) {
    return !p || ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * size)) & 15) == 0;
  };
  const bool vec = a.pairs % v == 0 && a.dh % v == 0 && fits(a.q, a.ldq) && fits(a.q_out, a.ldqo) && fits(a.k, a.ldk) &&
                   fits(a.k_out, a.ldko) && fits(a.v, a.ldv) && fits(a.v_out, a.ldvo);
  // few rows: one a CTA, so that they spread over the SMs
  a.rows_cta = 1;
  if (a.rows >= 4L * sm_count())
    while (a.rows_cta < 4 && 2 * a.rows_cta * a.pairs <= R_TH) a.rows_cta *= 2;
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
