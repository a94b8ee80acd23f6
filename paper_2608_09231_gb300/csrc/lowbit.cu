// Memory-bound low-precision passes: rows to 8-bit codes with block scales (alone or behind
// LayerNorm + modulation), the quantised cache's write and read, and the pooled vectors and
// selection of block-sparse attention.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "lowbit.cuh"
#include "kernels.h"

namespace bag {

namespace {

template <typename T>
BAG_DEV float to_f32(T x) { return (float)x; }

// ---------------------------------------------------------------------------
// rows -> codes + scales
// ---------------------------------------------------------------------------
// 16 bytes of a row, as loaded: N elements.
template <typename T>
struct Piece {
  static constexpr int N = 16 / sizeof(T);
  uint4 u;
  BAG_DEV void load(const T* p, int valid, bool vec) {
    u = make_uint4(0u, 0u, 0u, 0u);
    if (vec && valid >= N) {
      u = __ldg(reinterpret_cast<const uint4*>(p));
    } else {
      T* t = reinterpret_cast<T*>(&u);
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (i < valid) t[i] = p[i];
    }
  }
  // Largest magnitude of the block that LANES neighbouring lanes hold, as fp32 bits.  Of bf16 pairs
  // both halves are compared at once, as integers.
  template <int LANES>
  BAG_DEV uint32_t block_max() const {
    if constexpr (sizeof(T) == 4) {
      return group_max<LANES>(max(max(u.x & 0x7fffffffu, u.y & 0x7fffffffu), max(u.z & 0x7fffffffu, u.w & 0x7fffffffu)));
    } else {
      uint32_t m = __vmaxu2(__vmaxu2(u.x & 0x7fff7fffu, u.y & 0x7fff7fffu), __vmaxu2(u.z & 0x7fff7fffu, u.w & 0x7fff7fffu));
#pragma unroll
      for (int o = LANES / 2; o > 0; o >>= 1) m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, o));
      return max(m & 0xffff0000u, m << 16);
    }
  }
  // element pair i
  BAG_DEV float2 pair(int i) const {
    const uint32_t* w = reinterpret_cast<const uint32_t*>(&u);
    if constexpr (sizeof(T) == 4)
      return make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
    else
      return make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
  }
};

// A warp takes QS steps of a row, each 32 lanes x 16 bytes (128 fp32 or 256 bf16 columns); a
// block's largest magnitude passes between its 32 or 16 lanes.  Bound: HBM.  The steps' loads are
// all in flight before the first reduction, and stay as loaded until then: 32,760 x 5120 bf16 took
// 148 us with elements converted on arrival (40 % of HBM's rate), 80 so (6.3 TB/s; floor 74), 85 with
// five steps, 101 with eight; 4608 x 3072 fp32 12.9 (floor 10.4).
constexpr int QS = 4, Q_WARPS = 8;

template <typename T, bool VEC>
__global__ void __launch_bounds__(Q_WARPS * 32) quant_kernel(const T* __restrict__ x, long ldx, long rows, long cols,
                                                             uint8_t* __restrict__ codes, long ldc,
                                                             uint8_t* __restrict__ scales, long lds, int segs) {
  grid_dep_sync();
  constexpr int N = Piece<T>::N, STEP = 32 * N, LANES = kScaleBlock / N;
  const long item = (long)blockIdx.x * Q_WARPS + threadIdx.x / 32;
  const int lane = threadIdx.x % 32;
  const long row = item / segs;
  if (row >= rows) return;
  const long c0 = (item - row * segs) * (QS * STEP) + lane * N;
  const T* xr = x + row * ldx;
  Piece<T> v[QS];
#pragma unroll
  for (int s = 0; s < QS; ++s) {
    const long c = c0 + s * STEP;
    v[s].load(xr + c, (int)min((long)N, max(0L, cols - c)), VEC);
  }
#pragma unroll
  for (int s = 0; s < QS; ++s) {
    const long c = c0 + s * STEP;
    const uint32_t b = e8m0_of(v[s].template block_max<LANES>());
    const float inv = e8m0_inverse(b);
    if (c >= cols) continue;
    if (lane % LANES == 0) scales[row * lds + c / kScaleBlock] = (uint8_t)b;
    const int n = (int)min((long)N, cols - c);
    uint8_t* o = codes + row * ldc + c;
    uint32_t w[N / 4];
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const float2 lo = mul2(v[s].pair(2 * i), make_float2(inv, inv));
      const float2 hi = mul2(v[s].pair(2 * i + 1), make_float2(inv, inv));
      w[i] = pack_e4m3x4(lo.x, lo.y, hi.x, hi.y);
    }
    if (N == 8 && n == 8) {
      *reinterpret_cast<uint2*>(o) = make_uint2(w[0], w[N / 4 - 1]);
    } else {
#pragma unroll
      for (int i = 0; i < N / 4; ++i) store_bytes(o + 4 * i, w[i], n - 4 * i);
    }
  }
}

// ---------------------------------------------------------------------------
// LayerNorm + modulation -> codes + scales
// ---------------------------------------------------------------------------
template <int TH>
BAG_DEV float block_sum(float v, float* red) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
  if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < TH / 32; ++w) s += red[w];
  return s;
}

// A CTA a row; the row stays in registers (VPT float4 a thread, statistics in two passes over it), so
// that x is read once.  A warp's 32 float4 are 128 consecutive columns, which is one scale block.
// Bound: HBM behind the row's phases (load, two reductions, encode), which CTAS rows on an SM hide
// from each other, and the issue of the encoding: packed arithmetic, one maximum of three and (at
// 5120) CTAS held to 42 registers took 32,760 x 5120 from 155 to 132 us (floor 124: 6.4 TB/s), 4608 x
// 3072 from 16.3 to 14.8 (10.4; its 4608 CTAs are 3.03 waves, whose last is 48 rows).  Two rows a CTA took 17.4 against
// those 16.3, four 23.6; a row of 3072 on 192 threads 14.5 (7145 rows 20.8 against 20.5), on 96 16.2.
template <int TH, int VPT, int CTAS>
__global__ void __launch_bounds__(TH, CTAS) ln_fp8_kernel(const float* __restrict__ x, long ldx,
                                                    const float* __restrict__ shift, const float* __restrict__ scale,
                                                    int cols, uint8_t* __restrict__ codes, long ldc,
                                                    uint8_t* __restrict__ scales, long lds) {
  grid_dep_sync();
  __shared__ float red_mean[TH / 32], red_var[TH / 32];
  const long row = blockIdx.x;
  const float4* xr = reinterpret_cast<const float4*>(x + row * ldx);
  const int nv = cols / 4;
  float2 v[2 * VPT];
  float2 s = make_float2(0.f, 0.f);
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int c = threadIdx.x + i * TH;
    const float4 f = c < nv ? __ldcs(xr + c) : make_float4(0.f, 0.f, 0.f, 0.f);
    v[2 * i] = make_float2(f.x, f.y);
    v[2 * i + 1] = make_float2(f.z, f.w);
  }
#pragma unroll
  for (int i = 0; i < 2 * VPT; ++i) s = sum2(s, v[i]);
  const float mean = block_sum<TH>(s.x + s.y, red_mean) / (float)cols;
  float2 q = make_float2(0.f, 0.f);
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    if (threadIdx.x + i * TH < nv) {
#pragma unroll
      for (int j = 2 * i; j < 2 * i + 2; ++j) {
        v[j] = sum2(v[j], make_float2(-mean, -mean));
        q = muladd2(v[j], v[j], q);
      }
    }
  }
  const float rstd = rsqrtf(block_sum<TH>(q.x + q.y, red_var) / (float)cols + 1e-6f);
  uint8_t* const to = codes + row * ldc;
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const int c = threadIdx.x + i * TH;
    const int c0 = c - (int)(threadIdx.x % 32);  // the warp's first float4: warp-uniform
    if (c0 >= nv) break;
    float2 y0 = mul2(v[2 * i], make_float2(rstd, rstd)), y1 = mul2(v[2 * i + 1], make_float2(rstd, rstd));
    if (c < nv) {
      if (scale) {
        const float4 g = __ldg(reinterpret_cast<const float4*>(scale) + c);
        y0 = mul2(y0, sum2(make_float2(g.x, g.y), make_float2(1.f, 1.f)));
        y1 = mul2(y1, sum2(make_float2(g.z, g.w), make_float2(1.f, 1.f)));
      }
      if (shift) {
        const float4 g = __ldg(reinterpret_cast<const float4*>(shift) + c);
        y0 = sum2(y0, make_float2(g.x, g.y));
        y1 = sum2(y1, make_float2(g.z, g.w));
      }
    }
    const uint32_t b = e8m0_of(group_max<32>(abs_bits(max3_abs(max3_abs(y0.x, y0.y, y1.x), y1.y, 0.f))));
    const float inv = e8m0_inverse(b);
    if (c == c0) scales[row * lds + c / 32] = (uint8_t)b;
    if (c < nv) {
      y0 = mul2(y0, make_float2(inv, inv));
      y1 = mul2(y1, make_float2(inv, inv));
      *reinterpret_cast<uint32_t*>(to + 4 * c) = pack_e4m3x4(y0.x, y0.y, y1.x, y1.y);
    }
  }
}

// ---------------------------------------------------------------------------
// quantised cache
// ---------------------------------------------------------------------------
template <int BITS>
struct CacheFmt {
  static constexpr int GROUP = BITS == 8 ? 128 : 32;
  static constexpr int TOP = BITS == 8 ? 127 : 7;
  static constexpr int LANES = GROUP / 4;  // lanes of one group, four columns a lane
};
// A warp takes CS steps of 128 columns of a row, all loads first; 8-bit groups are its 32 lanes, 4-bit
// ones eight lanes.  Bound: HBM, at the rate of a plain copy: 32,760 x 5120 written in 218 us and read in
// 213 (8 bits, 9 bytes an element: 6.9 TB/s), 206 and 204 (4 bits); 6889 x 3072, 8 bits, one after the other 61.7.
constexpr int CS = 4, C_WARPS = 8, C_SEG = CS * 128;  // steps of a warp, warps of a CTA, columns of a warp

BAG_DEV float4 load_cols(const float* p, int valid, bool vec) {
  if (vec && valid >= 4) return *reinterpret_cast<const float4*>(p);
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  if (valid > 0) v.x = p[0];
  if (valid > 1) v.y = p[1];
  if (valid > 2) v.z = p[2];
  if (valid > 3) v.w = p[3];
  return v;
}

template <int BITS>
__global__ void __launch_bounds__(C_WARPS * 32) cache_write_kernel(const CacheArgs a) {
  grid_dep_sync();
  using F = CacheFmt<BITS>;
  const long item = (long)blockIdx.x * C_WARPS + threadIdx.x / 32;
  const int lane = threadIdx.x % 32;
  const long row = item / a.segs;
  if (row >= a.rows) return;
  const long slot = a.slots ? (long)__ldg(a.slots + row) : row;
  if (slot < 0 || slot >= a.capacity) return;
  const long c0 = (item - row * a.segs) * C_SEG + lane * 4;
  float4 x[CS], h[CS];
#pragma unroll
  for (int s = 0; s < CS; ++s) {
    const long c = c0 + s * 128;
    const int valid = (int)min(4L, a.cols - c);
    x[s] = load_cols(a.x + row * a.ldx + c, valid, a.vec);
    h[s] = a.base ? load_cols(a.base + row * a.ldb + c, valid, a.vec) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
#pragma unroll
  for (int s = 0; s < CS; ++s) {
    const long c = c0 + s * 128;
    const float v[4] = {x[s].x - h[s].x, x[s].y - h[s].y, x[s].z - h[s].z, x[s].w - h[s].w};
    const uint32_t m = max(max(abs_bits(v[0]), abs_bits(v[1])), max(abs_bits(v[2]), abs_bits(v[3])));
    const uint32_t amax = group_max<F::LANES>(m);
    const __nv_bfloat16 sb = __float2bfloat16_rn(__uint_as_float(amax) * (1.0f / F::TOP));
    float sc = __bfloat162float(sb);
    uint16_t bits = __bfloat16_as_ushort(sb);
    if (amax >= kInfBits) {  // reads as NaN
      sc = 0.f;
      bits = 0x7fffu;
    } else if (sc < 1.17549435e-38f) {  // 1 / scale could overflow
      sc = 0.f;
      bits = 0;
    }
    const float inv = sc > 0.f ? 1.0f / sc : 0.f;
    if (c >= a.cols) continue;
    if (lane % F::LANES == 0) reinterpret_cast<uint16_t*>(a.scales)[slot * a.lds + c / F::GROUP] = bits;
    int q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      q[i] = sc > 0.f ? max(-F::TOP, min(F::TOP, __float2int_rn(v[i] * inv))) : 0;
    const int n = (int)min(4L, a.cols - c);
    if constexpr (BITS == 8) {
      const uint32_t u = (uint32_t)(q[0] & 255) | (uint32_t)(q[1] & 255) << 8 | (uint32_t)(q[2] & 255) << 16 |
                         (uint32_t)q[3] << 24;
      store_bytes(a.codes + slot * a.ldc + c, u, n);
    } else {
      const uint32_t u = (uint32_t)(q[0] & 15) | (uint32_t)(q[1] & 15) << 4 | (uint32_t)(q[2] & 15) << 8 |
                         (uint32_t)(q[3] & 15) << 12;
      uint8_t* o = a.codes + slot * a.ldc + c / 2;
      if (n > 2)
        *reinterpret_cast<uint16_t*>(o) = (uint16_t)u;
      else
        *o = (uint8_t)u;
    }
  }
}

template <int BITS>
__global__ void __launch_bounds__(C_WARPS * 32) cache_read_kernel(const CacheArgs a) {
  grid_dep_sync();
  using F = CacheFmt<BITS>;
  const long item = (long)blockIdx.x * C_WARPS + threadIdx.x / 32;
  const int lane = threadIdx.x % 32;
  const long row = item / a.segs;
  if (row >= a.rows) return;
  const long slot = a.slots ? (long)__ldg(a.slots + row) : row;
  const bool held = slot >= 0 && slot < a.capacity;
  const long c0 = (item - row * a.segs) * C_SEG + lane * 4;
  uint32_t u[CS];
  float sc[CS];
  float4 h[CS];
#pragma unroll
  for (int s = 0; s < CS; ++s) {
    const long c = c0 + s * 128;
    u[s] = 0;
    sc[s] = 0.f;
    h[s] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c >= a.cols) continue;
    const int valid = (int)min(4L, a.cols - c);
    if (held) {
      // code rows are multiples of 16 bytes, so a whole word may be loaded past the last column
      if constexpr (BITS == 8)
        u[s] = __ldg(reinterpret_cast<const uint32_t*>(a.codes + slot * a.ldc + c));
      else
        u[s] = __ldg(reinterpret_cast<const uint16_t*>(a.codes + slot * a.ldc + c / 2));
      sc[s] = __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(a.scales)[slot * a.lds + c / F::GROUP]);
    }
    if (a.base) h[s] = load_cols(a.base + row * a.ldb + c, valid, a.vec);
  }
#pragma unroll
  for (int s = 0; s < CS; ++s) {
    const long c = c0 + s * 128;
    if (c >= a.cols) break;
    float q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)  // the code's bits to the top, then an arithmetic shift down
      q[i] = (float)((int)(u[s] << (32 - BITS * (i + 1))) >> (32 - BITS));
    const float4 o = make_float4(h[s].x + q[0] * sc[s], h[s].y + q[1] * sc[s], h[s].z + q[2] * sc[s],
                                 h[s].w + q[3] * sc[s]);
    float* p = a.out + row * a.ldo + c;
    const long n = a.cols - c;
    if (a.vec && n >= 4) {
      *reinterpret_cast<float4*>(p) = o;
    } else {
      p[0] = o.x;
      if (n > 1) p[1] = o.y;
      if (n > 2) p[2] = o.z;
      if (n > 3) p[3] = o.w;
    }
  }
}

// ---------------------------------------------------------------------------
// pooled vectors and selection of attention blocks
// ---------------------------------------------------------------------------
// Bound: HBM, which 128 rows' bytes of a head (32 KB a CTA) reach in one round of loads: 32,760 rows x 40
// heads 54 us (floor 49; 125 with rows converted as they came).
constexpr int P_TH = 256;

// Eight elements of a row as 16 bytes, zeros where there is no row.
template <typename T>
BAG_DEV uint4 raw8(const T* p, bool row, bool vec) {
  uint4 u = make_uint4(0u, 0u, 0u, 0u);
  if (!row) return u;
  if (vec) return __ldg(reinterpret_cast<const uint4*>(p));
  const unsigned short* q = reinterpret_cast<const unsigned short*>(p);
  uint32_t w[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) w[j] = __ldg(q + j);
  return make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
}

// Mean of up to 128 rows of 128 columns by all P_TH threads, as 8-bit codes of threads 0 .. 127
// (thread = column); returns the vector's scale to every thread.  Thread (rg, cg) holds rows rg
// + 16 i of eight columns, so the first three halvings (64, 32 and 16 rows apart) are its own;
// the other four pass through shared memory.  All eight rows are loaded before the first is
// converted, and kept as 16 bits until then (eight rows in fp32 would halve the CTAs on an SM).
template <typename T>
BAG_DEV float pool_block(const T* __restrict__ x, long ld, int rows, bool vec, float (*sums)[128], uint32_t* red,
                         int* code) {
  const int rg = threadIdx.x / 16, c = (threadIdx.x % 16) * 8;
  uint4 u[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) u[i] = raw8<T>(x + (long)(rg + 16 * i) * ld + c, rg + 16 * i < rows, vec);
  float v[4][8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const T *a = reinterpret_cast<const T*>(&u[i]), *b = reinterpret_cast<const T*>(&u[i + 4]);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] = to_f32(a[j]) + to_f32(b[j]);
  }
#pragma unroll
  for (int h = 2; h > 0; h /= 2)
#pragma unroll
    for (int i = 0; i < h; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] += v[i + h][j];
  *reinterpret_cast<float4*>(&sums[rg][c]) = make_float4(v[0][0], v[0][1], v[0][2], v[0][3]);
  *reinterpret_cast<float4*>(&sums[rg][c + 4]) = make_float4(v[0][4], v[0][5], v[0][6], v[0][7]);
  __syncthreads();
  float mean = 0.f;
  if (threadIdx.x < 128) {
    float s[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = sums[i][threadIdx.x];
#pragma unroll
    for (int h = 8; h > 0; h /= 2)
#pragma unroll
      for (int i = 0; i < h; ++i) s[i] += s[i + h];
    mean = s[0] * (1.0f / (float)rows);
    const uint32_t m = group_max<32>(abs_bits(mean));
    if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = m;
  }
  __syncthreads();
  const uint32_t amax = max(max(red[0], red[1]), max(red[2], red[3]));
  float sc = amax >= kInfBits ? 0.f : __uint_as_float(amax) * (1.0f / 127.0f);
  if (sc < 1.17549435e-38f) sc = 0.f;  // 1 / scale could overflow
  *code = sc > 0.f ? max(-127, min(127, __float2int_rn(mean * (1.0f / sc)))) : 0;
  return sc;
}

template <typename T>
__global__ void __launch_bounds__(P_TH, 4) block_pool_kernel(const T* __restrict__ x, long ld, long rows, int vec,
                                                          int8_t* __restrict__ codes, float* __restrict__ scales,
                                                          long ldb) {
  grid_dep_sync();
  __shared__ __align__(16) float sums[16][128];
  __shared__ uint32_t red[4];
  const long b = blockIdx.x, h = blockIdx.y;
  int code;
  const float sc = pool_block<T>(x + b * 128 * ld + h * 128, ld, (int)min(128L, rows - b * 128), vec, sums, red, &code);
  const long at = h * ldb + b;
  if (threadIdx.x < 128) codes[at * 128 + threadIdx.x] = (int8_t)code;
  if (threadIdx.x == 0) scales[at] = sc;
}

// One CTA pools its block of queries, scores every key block (eight lanes a block, 16 codes a
// lane, sums of four products in integers) and keeps the `keep` largest scores.  Scores become
// unsigned keys of the same order; passes over 8-bit digits find the keep-th largest, as many as it
// takes until all keys with the digits found so far are kept (two, mostly).  Bound: latency (the query
// block's rows, the pooled keys, then some ten barriers), which the CTAs of an SM hide from each other:
// five (48 registers) with four key steps in flight take 96 us for 32,760 queries, 40 heads and 256 key
// blocks (reading q 49), 12.5 for 4 heads, 4.2 for one query and 40 heads.  Four CTAs with eight steps in
// flight took 107, 13.4 and 4.2, and 32 us instead of 36 for one query and 7813 key blocks; key codes
// brought to shared memory while the queries are pooled 113, 15.0 and 4.6; always four passes 119 and 14.4.
template <typename T>
__global__ void __launch_bounds__(P_TH, 5)
    block_select_kernel(const T* __restrict__ q, long ldq, long nq, int vec, const int8_t* __restrict__ codes,
                        const float* __restrict__ scales, long ldb, int nkb, int group, int keep,
                        int* __restrict__ blocks) {
  grid_dep_sync();
  extern __shared__ uint32_t key[];
  __shared__ __align__(16) float sums[16][128];
  __shared__ uint32_t red[4];
  __shared__ __align__(16) int8_t qc[128];
  __shared__ int hist[2][256], warp_sum[P_TH / 32];
  __shared__ uint32_t found[3];  // the digit, how many keys are above it and how many have it
  const long b = blockIdx.x, h = blockIdx.y, kh = h / group;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  hist[0][threadIdx.x] = 0;
  int code;
  pool_block<T>(q + b * 128 * ldq + h * 128, ldq, (int)min(128L, nq - b * 128), vec, sums, red, &code);
  if (threadIdx.x < 128) qc[threadIdx.x] = (int8_t)code;
  __syncthreads();
  const int4 a = reinterpret_cast<const int4*>(qc)[lane % 8];
  const int4* kc = reinterpret_cast<const int4*>(codes + kh * ldb * 128) + lane % 8;
  constexpr int KU = 4;  // steps whose loads are in flight together
  for (int j0 = warp * 4 + lane / 8; j0 - lane / 8 < nkb; j0 += KU * P_TH / 8) {
    int4 k[KU];
    float sc[KU];
#pragma unroll
    for (int i = 0; i < KU; ++i) {
      const int j = min(j0 + i * (P_TH / 8), nkb - 1);
      k[i] = __ldg(kc + (long)j * 8);
      sc[i] = __ldg(scales + kh * ldb + j);
    }
#pragma unroll
    for (int i = 0; i < KU; ++i) {
      const int j = j0 + i * (P_TH / 8);
      int dot = __dp4a(a.x, k[i].x, __dp4a(a.y, k[i].y, __dp4a(a.z, k[i].z, __dp4a(a.w, k[i].w, 0))));
#pragma unroll
      for (int o = 4; o > 0; o /= 2) dot += __shfl_xor_sync(0xffffffffu, dot, o);
      if (j < nkb && lane % 8 == 0) {
        const uint32_t u = __float_as_uint((float)dot * sc[i] + 0.f);  // no -0
        key[j] = u & 0x80000000u ? ~u : u | 0x80000000u;
      }
    }
  }
  __syncthreads();
  uint32_t top = 0, mask = 0;  // the digits found so far, and where they are
  int need = keep, same_all = nkb;  // of the keys that have them: how many are kept, and how many there are
  for (int shift = 24; shift >= 0 && need < same_all; shift -= 8) {
    int* bins = hist[shift >> 3 & 1 ^ 1];
    for (int j = threadIdx.x; j < nkb; j += P_TH)
      if ((key[j] & mask) == top) atomicAdd(bins + (key[j] >> shift & 255u), 1);
    hist[shift >> 3 & 1][threadIdx.x] = 0;  // the next pass's
    __syncthreads();
    if (warp == 0) {  // lane l: digits 255 - 8 l .. 248 - 8 l
      int n[8], mine = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) mine += n[i] = bins[255 - 8 * lane - i];
      int before = mine;
#pragma unroll
      for (int o = 1; o < 32; o *= 2) {
        const int y = __shfl_up_sync(0xffffffffu, before, o);
        if (lane >= o) before += y;
      }
      before -= mine;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (before < need && before + n[i] >= need) {
          found[0] = (uint32_t)(255 - 8 * lane - i);
          found[1] = (uint32_t)before;
          found[2] = (uint32_t)n[i];
        }
        before += n[i];
      }
    }
    __syncthreads();
    top |= found[0] << shift;
    mask |= 255u << shift;
    need -= (int)found[1];
    same_all = (int)found[2];
  }
  // every key whose digits are above `top`, and the first `need` that have them, in order
  int* out = blocks + (h * gridDim.x + b) * keep;
  int kept = 0, equal = 0;  // of the keys before this round's
  for (int j0 = 0; j0 < nkb; j0 += P_TH) {
    const int j = j0 + (int)threadIdx.x;
    const uint32_t k = j < nkb ? key[j] & mask : 0u;
    const bool above = j < nkb && k > top, same = j < nkb && k == top;
    const uint32_t wa = __ballot_sync(0xffffffffu, above), ws = __ballot_sync(0xffffffffu, same);
    if (lane == 0) warp_sum[warp] = __popc(wa) << 16 | __popc(ws);
    __syncthreads();
    int na = 0, ns = 0, ta = 0, ts = 0;
#pragma unroll
    for (int w = 0; w < P_TH / 32; ++w) {
      const int n = warp_sum[w];
      if (w < warp) na += n >> 16, ns += n & 0xffff;
      ta += n >> 16;
      ts += n & 0xffff;
    }
    const uint32_t below = (1u << lane) - 1u;
    na += __popc(wa & below);
    ns += equal + __popc(ws & below);
    const int taken = min(ns, need) - min(equal, need);  // equal keys of this round kept before this one
    if (above || (same && ns < need)) out[kept + na + taken] = j;
    kept += ta + min(equal + ts, need) - min(equal, need);
    equal += ts;
    __syncthreads();
  }
}

bool rows16(const void* p, long ld, int size) { return ((reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * size)) & 15) == 0; }

// CTAs of `per` items for rows of segs items each (refused before the product could overflow).
cudaError_t grid_of(long rows, long segs, int per, unsigned* grid) {
  if (segs > 0x7fffffffL || rows > 0x7fffffffL * per / segs) return cudaErrorInvalidConfiguration;
  *grid = (unsigned)((rows * segs + per - 1) / per);
  return cudaSuccess;
}

}  // namespace

cudaError_t quant_fp8(const void* x, int bf16, long ldx, long rows, long cols, void* codes, long ldc, void* scales,
                      long lds, cudaStream_t s) {
  if (rows <= 0 || cols <= 0) return cudaSuccess;
  const int seg = QS * 32 * (bf16 ? 8 : 4);
  const long segs = (cols + seg - 1) / seg;
  unsigned grid;
  if (cudaError_t e = grid_of(rows, segs, Q_WARPS, &grid)) return e;
  auto launch = [&](auto kernel, auto type) {
    using T = decltype(type);
    return launch_kernel(kernel, grid, Q_WARPS * 32, 0, s, reinterpret_cast<const T*>(x), ldx, rows, cols,
                         reinterpret_cast<uint8_t*>(codes), ldc, reinterpret_cast<uint8_t*>(scales), lds, (int)segs);
  };
  if (bf16)
    return rows16(x, ldx, 2) ? launch(quant_kernel<__nv_bfloat16, true>, __nv_bfloat16{})
                             : launch(quant_kernel<__nv_bfloat16, false>, __nv_bfloat16{});
  return rows16(x, ldx, 4) ? launch(quant_kernel<float, true>, 0.f) : launch(quant_kernel<float, false>, 0.f);
}

cudaError_t ln_mod_fp8(const float* x, long ldx, const float* shift, const float* scale, long rows, int cols,
                       void* codes, long ldc, void* scales, long lds, cudaStream_t s) {
  if (rows <= 0) return cudaSuccess;
  if (rows > 0x7fffffffL) return cudaErrorInvalidConfiguration;
  auto launch = [&](auto kernel, int threads) {
    return launch_kernel(kernel, (unsigned)rows, threads, 0, s, x, ldx, shift, scale, cols,
                         reinterpret_cast<uint8_t*>(codes), ldc, reinterpret_cast<uint8_t*>(scales), lds);
  };
  if (cols > 5120) return launch(ln_fp8_kernel<256, 6, 5>, 256);
  if (cols > 3072) return launch(ln_fp8_kernel<256, 5, 6>, 256);
  if (cols > 1536) return launch(ln_fp8_kernel<128, 6, 10>, 128);
  return launch(ln_fp8_kernel<128, 3, 14>, 128);  // 4608 x 1536: 9.3 us with the 6, 8.6 so
}

static cudaError_t cache_grid(CacheArgs* a, unsigned* grid) {
  const long segs = (a->cols + C_SEG - 1) / C_SEG;
  a->segs = (int)segs;
  return grid_of(a->rows, segs, C_WARPS, grid);
}

cudaError_t cache_write(CacheArgs a, int bits, cudaStream_t s) {
  if (a.rows <= 0 || a.cols <= 0) return cudaSuccess;
  unsigned grid;
  if (cudaError_t e = cache_grid(&a, &grid)) return e;
  a.vec = rows16(a.x, a.ldx, 4) && (!a.base || rows16(a.base, a.ldb, 4));
  return launch_kernel(bits == 8 ? cache_write_kernel<8> : cache_write_kernel<4>, grid, C_WARPS * 32, 0, s, a);
}

cudaError_t cache_read(CacheArgs a, int bits, cudaStream_t s) {
  if (a.rows <= 0 || a.cols <= 0) return cudaSuccess;
  unsigned grid;
  if (cudaError_t e = cache_grid(&a, &grid)) return e;
  a.vec = rows16(a.out, a.ldo, 4) && (!a.base || rows16(a.base, a.ldb, 4));
  return launch_kernel(bits == 8 ? cache_read_kernel<8> : cache_read_kernel<4>, grid, C_WARPS * 32, 0, s, a);
}

cudaError_t block_pool(const void* x, int f16, long ld, long rows, int heads, void* codes, float* scales, long ldb,
                       cudaStream_t s) {
  if (rows <= 0) return cudaSuccess;
  const dim3 grid((unsigned)((rows + 127) / 128), (unsigned)heads);
  const int vec = rows16(x, ld, 2);
  if (f16)
    return launch_kernel(block_pool_kernel<__half>, grid, P_TH, 0, s, reinterpret_cast<const __half*>(x), ld, rows, vec,
                         reinterpret_cast<int8_t*>(codes), scales, ldb);
  return launch_kernel(block_pool_kernel<__nv_bfloat16>, grid, P_TH, 0, s, reinterpret_cast<const __nv_bfloat16*>(x),
                       ld, rows, vec, reinterpret_cast<int8_t*>(codes), scales, ldb);
}

cudaError_t block_select(const void* q, int f16, long ldq, long nq, int heads, const void* codes, const float* scales,
                         long ldb, int nkb, int kv_heads, int keep, int* blocks, cudaStream_t s) {
  if (nq <= 0) return cudaSuccess;
  const dim3 grid((unsigned)((nq + 127) / 128), (unsigned)heads);
  const int vec = rows16(q, ldq, 2), smem = nkb * 4, group = heads / kv_heads;
  if (f16)
    return launch_kernel(block_select_kernel<__half>, grid, P_TH, smem, s, reinterpret_cast<const __half*>(q), ldq, nq,
                         vec, reinterpret_cast<const int8_t*>(codes), scales, ldb, nkb, group, keep, blocks);
  return launch_kernel(block_select_kernel<__nv_bfloat16>, grid, P_TH, smem, s,
                       reinterpret_cast<const __nv_bfloat16*>(q), ldq, nq, vec,
                       reinterpret_cast<const int8_t*>(codes), scales, ldb, nkb, group, keep, blocks);
}

}  // namespace bag
