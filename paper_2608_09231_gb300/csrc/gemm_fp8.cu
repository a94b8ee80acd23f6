// Products of 8-bit operands with block scales: y[m, n] = sum over K blocks of 128 of
// 2^(sa + sw) * sum a[m, k] w[n, k], on the tensor cores' block-scaled MMA (kind::mxf8f6f4).
//
// The tensor core takes one scale byte for a row and 32 columns of K from tensor memory.  A block
// here is 128 columns, four MMAs, so one byte serves them all: a 32-bit word holds four
// consecutive blocks' bytes, tcgen05.cp brings the words of 128 rows in one copy (32 lanes x 16
// bytes: lane i, word c = row 32 c + i, repeated for the four lane quarters), and the
// instruction descriptor picks the block's byte.  Scales are then applied inside the MMA at its
// full rate, and the accumulator is the plain fp32 sum over K.
#include <algorithm>

#include "lowbit.cuh"
#include "bag.h"
#include "kernels.h"
#include "peer.cuh"

namespace bag {

namespace {

constexpr int F8_BK = kScaleBlock;      // K columns (bytes) of a pipeline stage
constexpr int F8_TILE = 128 * F8_BK;    // bytes of 128 rows
constexpr int F8_GROUP = 4;             // K blocks whose scale bytes share a word
constexpr int F8_ATOM = 512;            // bytes of 128 rows' scale words

// Shared-memory descriptor of a scale atom: 16-byte rows, groups of eight 128 bytes apart.
BAG_DEV uint64_t scale_desc(uint32_t saddr) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
}

// Instruction descriptor: D f32, A and B e4m3, K-major, E8M0 scales.  The byte of the scale
// words is added by scale_byte.
__host__ __device__ constexpr uint32_t idesc_mxf8(int M, int N) {
  return (uint32_t)(N >> 3) << 17 | 1u << 23 | (uint32_t)(M >> 4) << 24;
}
__host__ __device__ constexpr uint32_t scale_byte(uint32_t b) { return b << 4 | b << 29; }

BAG_DEV void copy_scales(uint32_t taddr, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}

BAG_DEV void mma_mxf8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(acc)
      : "memory");
}

// 16 consecutive TMEM columns of this thread's lane
BAG_DEV void tmem_ld16(uint32_t taddr, float* v) {
  uint32_t r[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}

// The scale words of K blocks 4 g .. 4 g + 3 for rows row0 + 32 c + lane (c = 0 .. 3); rows past
// the end have scale 1 (their codes are zeros).
BAG_DEV uint4 scale_words(const uint8_t* __restrict__ s, long lds, int row0, int rows, int g) {
  const int r = row0 + (int)(threadIdx.x & 31);
  auto at = [&](int row) {
    return row < rows ? __ldg(reinterpret_cast<const uint32_t*>(s + (long)row * lds) + g) : 0x7f7f7f7fu;
  };
  return make_uint4(at(r), at(r + 32), at(r + 64), at(r + 96));
}

}  // namespace

// ---------------------------------------------------------------------------
// Few rows: W is the M operand
// ---------------------------------------------------------------------------
// A CTA computes the transposed tile of 128 columns n and BN rows m: W's rows are the MMA's 128
// rows, A's the N operand, which may be as narrow as 16.  Clusters of S CTAs split K and add
// their parts through distributed shared memory in rank order (rank r finishes rows m = r, r + S,
// ... of the tile).
// warp 0: TMA producer; 1: MMA; 2: scale words; 4 .. 7: epilogue, thread = column n.
template <int BN>
struct FewCfg {
  static constexpr int STAGE = F8_TILE + BN * F8_BK;
  static constexpr int STAGES = BN == 16 ? 6 : (BN == 32 ? 5 : (BN == 64 ? 4 : 3));
  static constexpr int OFF_SF = STAGES * STAGE;              // two stages of W's and A's scale words
  static constexpr int OFF_RED = OFF_SF + 2 * 2 * F8_ATOM;   // [BN][4] block maxima of warps
  static constexpr int OFF_BAR = OFF_RED + BN * 16;
  static constexpr int SMEM = OFF_BAR + 256 + 1024;
  static constexpr int SF_COL = BN;                          // 8 TMEM columns a scale stage
  static constexpr int TMEM_COLS = 2 * BN;
  static_assert(BN + 16 <= TMEM_COLS, "accumulator and two scale stages");
  static_assert(128 * BN * 4 <= OFF_SF, "the exchange fits the ring");
};

template <int BN>
__global__ void __launch_bounds__(256)
    gemm_fp8_few_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmA,
                        const __grid_constant__ Fp8Gemm g, int S) {
  using C = FewCfg<BN>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + C::OFF_BAR);
  uint64_t* empty = full + C::STAGES;
  uint64_t* sf_full = empty + C::STAGES;
  uint64_t* sf_empty = sf_full + 2;
  uint64_t* tfull = sf_empty + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(tfull + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int rank = S > 1 ? (int)cluster_ctarank() : 0;
  const int mt = (g.M + BN - 1) / BN, unit = blockIdx.x / S;
  const int m0 = unit % mt * BN, n0 = unit / mt * 128;
  const int nkb = (g.K + F8_BK - 1) / F8_BK;
  const int kb0 = (int)((long)rank * nkb / S), kb1 = (int)((long)(rank + 1) * nkb / S);

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::STAGES; ++s) {
      mbar_init(full + s, 1);
      mbar_init(empty + s, 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(sf_full + s, 1);
      mbar_init(sf_empty + s, 1);
    }
    mbar_init(tfull, 1);
    *abort_flag = 0;
    fence_mbar_init();
    tma_prefetch_desc(&tmW);
    tma_prefetch_desc(&tmA);
  }
  grid_dep_sync();
  __syncwarp();
  if (warp == 1) {
    tmem_alloc(tmem_slot, C::TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  if (warp == 0) {
    if (lane == 0) {
      // ---------------- TMA producer ----------------
      int s = 0;
      uint32_t ph = 0;
      int issued = 0;
      bool ok = true;
      for (int kb = kb0; kb < kb1; ++kb) {
        if (!mbar_wait(empty + s, ph ^ 1, abort_flag)) {
          ok = false;
          break;
        }
        mbar_arrive_expect_tx(full + s, C::STAGE);
        tma_load_2d(smem + s * C::STAGE, &tmW, kb * F8_BK, n0, full + s);
        tma_load_2d(smem + s * C::STAGE + F8_TILE, &tmA, kb * F8_BK, m0, full + s);
        ++issued;
        if (++s == C::STAGES) {
          s = 0;
          ph ^= 1;
        }
      }
      if (!ok) {
        // wait (bounded) for the copies this thread may still have in flight
        const uint64_t t0 = global_ns();
        for (int i = 0; i < C::STAGES && i < issued; ++i) {
          if (--s < 0) {
            s = C::STAGES - 1;
            ph ^= 1;
          }
          while (!mbar_try_wait(full + s, ph) && global_ns() - t0 < kWaitLimitNs) {
          }
        }
      }
    }
  } else if (warp == 1) {
    // ---------------- MMA issuer (converged warp, one elected lane issues) ----------------
    const uint32_t base = smem_u32(smem);
    int s = 0, ss = 0;
    uint32_t ph = 0, sph = 0;
    for (int kb = kb0; kb < kb1; ++kb) {
      const uint32_t sw = tmem + C::SF_COL + ss * 8;
      if (kb == kb0 || kb % F8_GROUP == 0) {
        if (!mbar_wait_warp(sf_full + ss, sph, abort_flag)) break;
        tc_fence_after();
        const uint64_t d = scale_desc(base + C::OFF_SF + ss * 2 * F8_ATOM);
        if (elect_one()) {
          copy_scales(sw, d);
          copy_scales(sw + 4, d + (F8_ATOM >> 4));
        }
        __syncwarp();
      }
      if (!mbar_wait_warp(full + s, ph, abort_flag)) break;
      tc_fence_after();
      const uint64_t wd = sw128_desc(base + s * C::STAGE);
      const uint64_t ad = sw128_desc(base + s * C::STAGE + F8_TILE);
      const uint32_t idesc = idesc_mxf8(128, BN) | scale_byte((uint32_t)(kb % F8_GROUP));
      const bool last = kb + 1 == kb1 || (kb + 1) % F8_GROUP == 0;
      if (elect_one()) {
#pragma unroll
        for (int k = 0; k < F8_BK / 32; ++k)  // 32 bytes along K: two 16-byte units
          mma_mxf8(tmem, wd + 2 * k, ad + 2 * k, idesc, sw, sw + 4, (kb > kb0 || k > 0) ? 1u : 0u);
        mma_commit(empty + s);
        if (last) mma_commit(sf_empty + ss);
      }
      __syncwarp();
      if (++s == C::STAGES) {
        s = 0;
        ph ^= 1;
      }
      if (last && (ss ^= 1) == 0) sph ^= 1;
    }
    // all MMAs issued so far (whatever happened above) finish before tfull completes, and
    // the bounded wait keeps tensor memory until then
    if (elect_one()) {
      mma_commit(tfull);
      const uint64_t t0 = global_ns();
      while (!mbar_try_wait(tfull, 0) && global_ns() - t0 < kWaitLimitNs) {
      }
    }
    __syncwarp();
  } else if (warp == 2) {
    // ---------------- scale words, a group of four K blocks at a time ----------------
    const int g0 = kb0 / F8_GROUP, g1 = (kb1 + F8_GROUP - 1) / F8_GROUP;
    uint4 w = make_uint4(0u, 0u, 0u, 0u), a = w;
    auto fetch = [&](int gi) {
      if (gi < g1) {
        w = scale_words(g.w_s, g.ldws, n0, g.N, gi);
        a = scale_words(g.a_s, g.ldas, m0, min(g.M, m0 + BN), gi);
      }
    };
    fetch(g0);
    int ss = 0;
    uint32_t sph = 0;
    for (int gi = g0; gi < g1 && kb0 < kb1; ++gi) {
      if (!mbar_wait_warp(sf_empty + ss, sph ^ 1, abort_flag)) break;
      uint4* d = reinterpret_cast<uint4*>(smem + C::OFF_SF + ss * 2 * F8_ATOM);
      d[lane] = w;
      d[32 + lane] = a;
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(sf_full + ss);
      fetch(gi + 1);
      if ((ss ^= 1) == 0) sph ^= 1;
    }
  }
  // ---------------- epilogue ----------------
  const bool epi = warp >= 4;
  const int row = (int)threadIdx.x - 128, n = n0 + row;  // of an epilogue thread
  const int cols = min(BN, g.M - m0);
  const int per = BN / S;                                // rows m of the tile a rank finishes
  float* part = reinterpret_cast<float*>(smem);          // [S][per][128]
  if (epi) mbar_wait(tfull, 0, abort_flag);
  __syncwarp();
  tc_fence_before();
  // every product is done, here and in the cluster: the rings are free.  No role waits after
  // this, so all threads see the same abort flag.
  if (S > 1)
    cluster_sync_all();
  else
    __syncthreads();
  tc_fence_after();
  const bool ok = !*abort_flag;
  if (epi && ok) {
    const uint32_t tb = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t here = smem_u32(part) + (uint32_t)(rank * per * 128 + row) * 4u;
#pragma unroll 1
    for (int c = 0; c < cols; c += 16) {
      float v[16];
      tmem_ld16(tb + (uint32_t)c, v);
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (c + j < cols) {
          const uint32_t at = here + (uint32_t)((c + j) / S * 128) * 4u;
          peer_store1(S > 1 ? mapa_shared(at, (uint32_t)((c + j) % S)) : at, v[j]);
        }
    }
  }
  tc_fence_before();
  __syncwarp();
  if (S > 1) cluster_sync_all();  // every part has arrived; no access to another CTA follows
  if (epi && ok) {
    const bool in = n < g.N;
    const float bias = in && g.bias ? __ldg(g.bias + n) : 0.f;
    const float gate = in && g.gate ? __ldg(g.gate + n) : 1.f;
    const int mine = (cols - rank + S - 1) / S;
    uint32_t* red = reinterpret_cast<uint32_t*>(smem + C::OFF_RED);
#pragma unroll 1
    for (int j = 0; j < mine; ++j) {
      float y = part[j * 128 + row];
      for (int p = 1; p < S; ++p) y += part[(p * per + j) * 128 + row];
      y += bias;
      if (g.act) y = gelu_sigmoid(y);
      const long at = (long)(m0 + j * S + rank) * g.ldo + n;
      if (g.kind == BAG_FP8_CODES) {
        y = in ? y : 0.f;
        part[j * 128 + row] = y;  // this thread's own word
        const uint32_t m = group_max<32>(abs_bits(y));
        if (lane == 0) red[j * 4 + (warp & 3)] = m;
      } else if (in) {
        if (g.kind == BAG_FP8_F32)
          reinterpret_cast<float*>(g.out)[at] = y;
        else if (g.kind == BAG_FP8_BF16)
          reinterpret_cast<__nv_bfloat16*>(g.out)[at] = __float2bfloat16_rn(y);
        else
          reinterpret_cast<float*>(g.out)[at] += gate * y;
      }
    }
    if (g.kind == BAG_FP8_CODES) {
      asm volatile("bar.sync 1, 128;" ::: "memory");
#pragma unroll 1
      for (int j = 0; j < mine; ++j) {
        const uint4 r = *reinterpret_cast<const uint4*>(red + j * 4);
        const uint32_t b = e8m0_of(max(max(r.x, r.y), max(r.z, r.w)));
        const float y = part[j * 128 + row] * e8m0_inverse(b);
        const long m = m0 + j * S + rank;
        if (in)
          reinterpret_cast<uint8_t*>(g.out)[m * g.ldo + n] = __nv_cvt_float_to_fp8(y, __NV_SATFINITE, __NV_E4M3);
        if (row == 0) g.out_s[m * g.ldos + n0 / kScaleBlock] = (uint8_t)b;
      }
    }
  }
  __syncthreads();
  if (threadIdx.x == 0 && !ok && g.err) atomicOr(g.err, 1);
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, C::TMEM_COLS);
  }
}

template <int BN>
static cudaError_t launch_few(const Fp8Gemm& g, int S, cudaStream_t s) {
  CUtensorMap tw, ta;
  if (encode_tmap_2d_u8(&tw, g.w, (uint64_t)g.K, (uint64_t)g.N, (uint64_t)g.ldw, F8_BK, 128) ||
      encode_tmap_2d_u8(&ta, g.a, (uint64_t)g.K, (uint64_t)g.M, (uint64_t)g.lda, F8_BK, BN))
    return cudaErrorInvalidValue;
  const long units = (long)((g.M + BN - 1) / BN) * ((g.N + 127) / 128);
  if (units * S > 0x7fffffffL) return cudaErrorInvalidConfiguration;
  return launch_cluster(gemm_fp8_few_kernel<BN>, S > 1 ? (unsigned)S : 0u, (unsigned)(units * S), 256,
                        FewCfg<BN>::SMEM, s, tw, ta, g, S);
}

cudaError_t gemm_fp8_init() {
  cudaError_t r = cudaSuccess;
  auto smem = [&](auto kernel, int bytes) {
    if (r == cudaSuccess) r = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  };
  smem(gemm_fp8_few_kernel<16>, FewCfg<16>::SMEM);
  smem(gemm_fp8_few_kernel<32>, FewCfg<32>::SMEM);
  smem(gemm_fp8_few_kernel<64>, FewCfg<64>::SMEM);
  smem(gemm_fp8_few_kernel<128>, FewCfg<128>::SMEM);
  return r;
}

cudaError_t gemm_fp8(Fp8Gemm g, cudaStream_t s) {
  if (g.M <= 0 || g.N <= 0) return cudaSuccess;
  const int BN = g.M <= 16 ? 16 : (g.M <= 32 ? 32 : (g.M <= 64 ? 64 : 128));
  const long units = (long)((g.M + BN - 1) / BN) * ((g.N + 127) / 128);
  const int nkb = (g.K + F8_BK - 1) / F8_BK;
  int S = 1;
  while (S < 8 && units * S * 2 <= sm_count() && nkb >= S * 2 * 4) S *= 2;
  if (BN == 16) return launch_few<16>(g, S, s);
  if (BN == 32) return launch_few<32>(g, S, s);
  if (BN == 64) return launch_few<64>(g, S, s);
  return launch_few<128>(g, S, s);
}

}  // namespace bag
