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
#include <cmath>

#include "attn_common.cuh"
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
constexpr int F8_RUN = 4;               // groups that are fetched and handed over together (16 bytes a row)

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

// The scale words of one run of groups (run r: K blocks 16 r .. 16 r + 15) for the 128 rows from
// row0 on: rows row0 + 32 c + lane, c = 0 .. 3.  Rows past the end have scale 1 (their codes are
// zeros), and so have K blocks in words past the last of the nkb.  16-byte loads where the rows
// allow them: a row's words of a run lie in one sector, and with word loads every group would fetch
// it again (the ring leaves L1 too small to keep it).  Each load holds a byte of the row, so none
// leaves the operand, also where the row is a part of a longer one (columns of a wider buffer).
struct ScaleRun {
  uint4 w[4];
  BAG_DEV void fetch(const uint8_t* __restrict__ s, long lds, bool wide, int row0, int rows, int run, int nkb) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int row = row0 + 32 * c + (int)(threadIdx.x & 31);
      w[c] = make_uint4(0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu, 0x7f7f7f7fu);
      if (row >= rows) continue;
      const uint8_t* p = s + (long)row * lds + run * 16;
      if (wide) {
        w[c] = __ldg(reinterpret_cast<const uint4*>(p));
      } else {
        const uint32_t* q = reinterpret_cast<const uint32_t*>(p);
        const int left = (nkb + 3) / 4 - run * 4;  // words of the row from here on
        if (left > 0) w[c].x = __ldg(q);
        if (left > 1) w[c].y = __ldg(q + 1);
        if (left > 2) w[c].z = __ldg(q + 2);
        if (left > 3) w[c].w = __ldg(q + 3);
      }
    }
  }
  // to shared memory, group after group `step` bytes apart: lane i's 16 bytes are the words of rows
  // i, 32 + i, 64 + i and 96 + i
  BAG_DEV void put(uint8_t* dst, int step) const {
    const int lane = threadIdx.x & 31;
    auto at = [&](int j) -> uint4& { return reinterpret_cast<uint4*>(dst + j * step)[lane]; };
    at(0) = make_uint4(w[0].x, w[1].x, w[2].x, w[3].x);
    at(1) = make_uint4(w[0].y, w[1].y, w[2].y, w[3].y);
    at(2) = make_uint4(w[0].z, w[1].z, w[2].z, w[3].z);
    at(3) = make_uint4(w[0].w, w[1].w, w[2].w, w[3].w);
  }
};

// Whether rows of scale bytes are whole 16-byte units.
__host__ __device__ __forceinline__ bool wide_scales(const uint8_t* s, long lds) {
  return ((reinterpret_cast<uintptr_t>(s) | (uintptr_t)lds) & 15) == 0;
}

}  // namespace

// The tensor core cuts what an addend has below the accumulator's last bits, towards zero, so the
// error of a sum grows with K (1.4e-7 of the result at K = 3072, 9.3e-7 at 13824).  A sum of more K
// blocks than pass_blocks (the kernels' LONG forms) is therefore computed in passes of at most that
// many, which the epilogue adds in registers (rounded to nearest).
// Most K blocks of a pass.  fp32 outputs: 32, which takes the error of a sum (2-norm, against 64
// bits) from 1.2e-6 to 2.4e-7 at K = 13824 for 4 % of the time, and leaves K <= 4096 in one pass
// (2.1e-7 at 3072; 40 blocks in two passes cost 6 %).  bf16 rounds to 4e-3: 64.  Codes: 20, since a
// sum near the middle of two codes goes to the other one with its whole step: of the 12.6 million
// codes of 1024 x 12288 x 3072 81 differ from 64 bits in one pass, 51 in two, for 3 % more time.
__host__ __device__ constexpr int pass_blocks(int kind) {
  return kind == BAG_FP8_CODES ? 20 : (kind == BAG_FP8_BF16 ? 64 : 32);
}
// Blocks of one of the passes that n K blocks take: about as many in each, whole groups of scale words.
__host__ __device__ constexpr int pass_length(int n, int most) {
  const int passes = (n + most - 1) / most;  // but for the rounding up to groups
  return ((n + passes - 1) / passes + F8_GROUP - 1) / F8_GROUP * F8_GROUP;
}
static_assert(pass_blocks(BAG_FP8_F32) % F8_GROUP == 0 && pass_blocks(BAG_FP8_BF16) % F8_GROUP == 0 &&
                  pass_blocks(BAG_FP8_CODES) % F8_GROUP == 0 && pass_blocks(BAG_FP8_RESID) % F8_GROUP == 0,
              "passes of whole groups");

// ---------------------------------------------------------------------------
// Few rows: W is the M operand
// ---------------------------------------------------------------------------
// A CTA computes the transposed tile of 128 columns n and BN rows m: W's rows are the MMA's 128
// rows, A's the N operand, which may be as narrow as 16.  Clusters of S CTAs split K and add
// their parts through distributed shared memory in rank order (rank r finishes rows m = r, r + S,
// ... of the tile).  A CTA's part of K that is longer than a pass (LONG) is summed in passes, like the
// pair kernel's units; the sums go back to tensor memory, from where the epilogue takes them either way
// (16 x 512 x 65536 to fp32: 22.2 us, 20.6 with parts of 64 K blocks in one sum each).
// warp 0: TMA producer; 1: MMA; 2: scale words to shared memory; 3: and to tensor memory; 4 .. 7:
// epilogue, thread = column n.
// The ring is as deep as the CTAs that share an SM leave room for (`stages`, at most F8F_MAX).
// Bound: W's way from HBM where it is large, the launch's start and end where not.  1 x 13824 x 5120
// (BN 16, four CTAs a tile, 432 of them) takes 12 us in a chain of launches (6 TB/s of W; floor 10.5), 77 x
// 2048 x 512 about 5.
constexpr int F8F_MAX = 10;
template <int BN>
struct FewCfg {
  static constexpr int STAGE = F8_TILE + BN * F8_BK;
  static constexpr int SF_GROUP = 2 * F8_ATOM, SF_STAGE = F8_RUN * SF_GROUP;
  // after the ring: two runs of W's and A's scale words, [BN][4] block maxima of warps, barriers
  static constexpr int OFF_RED = 2 * SF_STAGE;
  static constexpr int OFF_BAR = OFF_RED + BN * 16;
  static constexpr int REST = OFF_BAR + 256 + 1024;
  static constexpr int MIN_STAGES = 3;
  static constexpr int SF_COL = BN;                          // 8 TMEM columns a scale stage
  static constexpr int TMEM_COLS = 2 * BN;
  static_assert(BN + 16 <= TMEM_COLS, "accumulator and two scale stages");
  static_assert(128 * BN * 4 <= MIN_STAGES * STAGE, "the exchange fits the ring");
  // ring depth where `ctas` share an SM (each takes 1 KB of it besides its own)
  static int stages(int ctas) {
    return std::max(MIN_STAGES, std::min(F8F_MAX, (228 * 1024 / ctas - 1024 - REST) / STAGE));
  }
};

// First K block of a rank's part (rank S: one past the last): an even one, since blocks are issued in
// pairs.
__host__ __device__ constexpr int few_cut(int r, int S, int nkb) {
  return r == S ? nkb : (int)((long)r * nkb / S) & ~1;
}

template <int BN, bool LONG>
__global__ void __launch_bounds__(256)
    gemm_fp8_few_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmA,
                        const __grid_constant__ Fp8Gemm g, int logS, int stages) {
  using C = FewCfg<BN>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  uint8_t* rest = smem + stages * C::STAGE;
  uint64_t* full = reinterpret_cast<uint64_t*>(rest + C::OFF_BAR);
  uint64_t* empty = full + F8F_MAX;
  uint64_t* sf_full = empty + F8F_MAX;
  uint64_t* sf_empty = sf_full + 2;
  uint64_t* sf_ready = sf_empty + 2;  // [2]: a group's scales are in tensor memory
  uint64_t* sf_used = sf_ready + 2;   // [2]: a group's products are done, its TMEM columns free
  uint64_t* tfull = sf_used + 2;
  uint64_t* tempty = tfull + 1;       // LONG: a pass's sums are read
  uint64_t* sf_drain = tempty + 1;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sf_drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  static_assert((2 * F8F_MAX + 11) * 8 + 8 <= 256, "the barriers, the address of tensor memory and the flag");

  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int S = 1 << logS, rank = logS > 0 ? (int)cluster_ctarank() : 0;
  const int mt = (g.M + BN - 1) / BN, unit = (int)(blockIdx.x >> logS);
  const int m0 = unit % mt * BN, n0 = unit / mt * 128;
  const int nkb = (g.K + F8_BK - 1) / F8_BK;
  const int kb0 = few_cut(rank, S, nkb), kb1 = few_cut(rank + 1, S, nkb);  // this rank's K blocks
  const int kg0 = kb0 & ~(F8_GROUP - 1);                                   // and their first group
  const int pass_kb = LONG ? pass_length(kb1 - kg0, pass_blocks(g.kind)) : 0;

  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
      mbar_init(full + s, 1);
      mbar_init(empty + s, 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(sf_full + s, 1);
      mbar_init(sf_empty + s, 1);
      mbar_init(sf_ready + s, 1);
      mbar_init(sf_used + s, 1);
    }
    mbar_init(tfull, 1);
    mbar_init(tempty, 4);  // the epilogue's warps
    mbar_init(sf_drain, 1);
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
        if (++s == stages) {
          s = 0;
          ph ^= 1;
        }
      }
      if (!ok) {
        // wait (bounded) for the copies this thread may still have in flight
        const uint64_t t0 = global_ns();
        for (int i = 0; i < stages && i < issued; ++i) {
          if (--s < 0) {
            s = stages - 1;
            ph ^= 1;
          }
          while (!mbar_try_wait(full + s, ph) && global_ns() - t0 < kWaitLimitNs) {
          }
        }
      }
    }
  } else if (warp == 1) {
    // ---------------- MMA issuer (converged warp, one elected lane issues) ----------------
    const uint32_t base = smem_u32(smem), tm = uniform(tmem);
    int s = 0, grp = 0;        // ring stage; groups handled so far
    uint32_t ph = 0, add = 0;  // the first product overwrites the accumulator
    auto next = [&](int& st, uint32_t& parity) {
      if (++st == stages) {
        st = 0;
        parity ^= 1;
      }
    };
    bool good = true;
    uint32_t passes = 0;  // handed to the epilogue so far
    for (int kg = kg0; kg < kb1 && good; kg += F8_GROUP, ++grp) {  // groups, maybe cut
      const uint32_t sw = tm + C::SF_COL + (grp & 1) * 8;
      if constexpr (LONG) {
        if (kg > kg0 && (kg - kg0) % pass_kb == 0) {
          if (elect_one()) mma_commit(tfull);
          __syncwarp();
          if (!(good = mbar_wait_warp(tempty, passes++ & 1u, abort_flag))) break;
          add = 0;
        }
      }
      if (!(good = mbar_wait_warp(sf_ready + (grp & 1), (uint32_t)(grp >> 1) & 1u, abort_flag))) break;
#pragma unroll
      for (int b = 0; b < F8_GROUP; b += 2) {
        if (kg + b < kb0 || kg + b >= kb1) continue;
        const bool two = kg + b + 1 < kb1;
        int s1 = s;
        uint32_t ph1 = ph;
        next(s1, ph1);
        if (!(good = good && mbar_wait_warp(full + s, ph, abort_flag))) break;
        if (two && !(good = mbar_wait_warp(full + s1, ph1, abort_flag))) break;
        tc_fence_after();
        const uint64_t w0 = sw128_desc(base + s * C::STAGE), w1 = sw128_desc(base + s1 * C::STAGE);
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < F8_BK / 32; ++k)  // 32 bytes along K: two 16-byte units
            mma_mxf8(tm, w0 + 2 * k, w0 + (F8_TILE >> 4) + 2 * k, idesc_mxf8(128, BN) | scale_byte(b), sw, sw + 4,
                     k > 0 ? 1u : add);
          mma_commit(empty + s);
          if (two) {
#pragma unroll
            for (int k = 0; k < F8_BK / 32; ++k)
              mma_mxf8(tm, w1 + 2 * k, w1 + (F8_TILE >> 4) + 2 * k, idesc_mxf8(128, BN) | scale_byte(b + 1), sw,
                       sw + 4, 1u);
            mma_commit(empty + s1);
          }
          if (b + 2 == F8_GROUP || kg + b + 2 >= kb1) mma_commit(sf_used + (grp & 1));
        }
        __syncwarp();
        add = 1;
        s = s1;
        ph = ph1;
        if (two) next(s, ph);
      }
    }
    // all MMAs issued so far (whatever happened above) finish before tfull completes, and
    // the bounded wait keeps tensor memory until then
    if (elect_one()) {
      const uint64_t t0 = global_ns();
      while (passes > 0 && !mbar_try_wait(tfull, (passes - 1) & 1u) && global_ns() - t0 < kWaitLimitNs) {
      }
      mma_commit(tfull);
      while (!mbar_try_wait(tfull, passes & 1u) && global_ns() - t0 < kWaitLimitNs) {
      }
    }
    __syncwarp();
  } else if (warp == 3) {
    // ---------------- scales to tensor memory, a group ahead of the products ----------------
    const uint32_t sf = smem_u32(rest);
    int run = 0, grp = 0;
    for (int kg = kg0; kg < kb1; kg += F8_GROUP, ++grp) {
      if (run == 0 || kg % (F8_GROUP * F8_RUN) == 0) {
        if (!mbar_wait_warp(sf_full + (run & 1), (uint32_t)(run >> 1) & 1u, abort_flag)) break;
        ++run;
      }
      if (!mbar_wait_warp(sf_used + (grp & 1), ((uint32_t)(grp >> 1) & 1u) ^ 1u, abort_flag)) break;
      tc_fence_after();
      const uint32_t sw = tmem + C::SF_COL + (grp & 1) * 8;
      const uint64_t d = scale_desc(sf + ((run - 1) & 1) * C::SF_STAGE + kg / F8_GROUP % F8_RUN * C::SF_GROUP);
      if (elect_one()) {
        copy_scales(sw, d);
        copy_scales(sw + 4, d + (F8_ATOM >> 4));
        mma_commit(sf_ready + (grp & 1));
        if (kg + F8_GROUP >= kb1 || (kg / F8_GROUP + 1) % F8_RUN == 0) mma_commit(sf_empty + ((run - 1) & 1));
      }
      __syncwarp();
    }
    // every copy has ended before tensor memory is released
    if (elect_one()) {
      mma_commit(sf_drain);
      const uint64_t t0 = global_ns();
      while (!mbar_try_wait(sf_drain, 0) && global_ns() - t0 < kWaitLimitNs) {
      }
    }
    __syncwarp();
  } else if (warp == 2) {
    // ---------------- scale words, a run of groups at a time ----------------
    const int r0 = kb0 / (F8_GROUP * F8_RUN), r1 = (kb1 + F8_GROUP * F8_RUN - 1) / (F8_GROUP * F8_RUN);
    const bool wide_w = wide_scales(g.w_s, g.ldws), wide_a = wide_scales(g.a_s, g.ldas);
    ScaleRun w, a;
    auto fetch = [&](int r) {
      if (r < r1) {
        w.fetch(g.w_s, g.ldws, wide_w, n0, g.N, r, nkb);
        a.fetch(g.a_s, g.ldas, wide_a, m0, min(g.M, m0 + BN), r, nkb);
      }
    };
    fetch(r0);
    for (int r = r0; r < r1; ++r) {
      const int i = r - r0, st = i & 1;
      if (!mbar_wait_warp(sf_empty + st, ((uint32_t)(i >> 1) & 1u) ^ 1u, abort_flag)) break;
      uint8_t* d = rest + st * C::SF_STAGE;
      w.put(d, C::SF_GROUP);
      a.put(d + F8_ATOM, C::SF_GROUP);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(sf_full + st);
      fetch(r + 1);
    }
  }
  // ---------------- epilogue ----------------
  const bool epi = warp >= 4;
  const int row = (int)threadIdx.x - 128, n = n0 + row;  // of an epilogue thread
  const int cols = min(BN, g.M - m0);
  const int per = BN >> logS;                            // rows m of the tile a rank finishes
  float* part = reinterpret_cast<float*>(smem);          // [S][per][128]
  const uint32_t tb = tmem + ((uint32_t)((warp & 3) * 32) << 16);
  if constexpr (LONG) {
    if (epi) {
      float sum[BN];
#pragma unroll
      for (int c = 0; c < BN; ++c) sum[c] = 0.f;
      bool good = true;
      uint32_t pass = 0;
#pragma unroll 1
      for (int kg = kg0; kg < kb1; kg += pass_kb, ++pass) {
        if (!(good = __all_sync(0xffffffffu, mbar_wait(tfull, pass & 1u, abort_flag)))) break;
        tc_fence_after();
#pragma unroll
        for (int c = 0; c < BN; c += 16) {
          float t[16];
          tmem_ld16(tb + (uint32_t)c, t);
#pragma unroll
          for (int j = 0; j < 16; ++j) sum[c + j] += t[j];
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(tempty);
      }
      if (good) {  // no product writes the accumulator any more
#pragma unroll
        for (int c = 0; c < BN; c += 16) tmem_st16(tb + (uint32_t)c, reinterpret_cast<const uint32_t*>(sum + c));
        tmem_st_wait();
      }
    }
  } else {
    if (epi) mbar_wait(tfull, 0, abort_flag);
  }
  __syncwarp();
  tc_fence_before();
  // every product is done, here and in the cluster: the rings are free.  No role waits after
  // this, so all threads see the same abort flag.
  if (logS > 0)
    cluster_sync_all();
  else
    __syncthreads();
  tc_fence_after();
  const bool ok = !*abort_flag;
  if (logS > 0) {
    if (epi && ok) {
      const uint32_t here = smem_u32(part) + (uint32_t)((rank * per * 128 + row) * 4);
#pragma unroll 1
      for (int c = 0; c < cols; c += 16) {
        float v[16];
        tmem_ld16(tb + (uint32_t)c, v);
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (c + j < cols)
            peer_store1(mapa_shared(here + (uint32_t)((c + j) >> logS) * 512u, (uint32_t)((c + j) & (S - 1))), v[j]);
      }
    }
    __syncwarp();
    cluster_sync_all();  // every part has arrived; no access to another CTA follows
  }
  if (epi && ok) {
    const bool in = n < g.N;
    const float bias = in && g.bias ? __ldg(g.bias + n) : 0.f;
    const float gate = in && g.gate ? __ldg(g.gate + n) : 1.f;
    const int mine = (cols - rank + S - 1) >> logS;
    uint4* red = reinterpret_cast<uint4*>(rest + C::OFF_RED);  // [row m of the tile]: the warps' maxima
#pragma unroll 1
    for (int j0 = 0; j0 < mine; j0 += 16) {
      float y[16];
      if (logS == 0) {
        tmem_ld16(tb + (uint32_t)j0, y);
      } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) y[j] = j0 + j < mine ? part[(j0 + j) * 128 + row] : 0.f;
        for (int p = 1; p < S; ++p)
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (j0 + j < mine) y[j] += part[(p * per + j0 + j) * 128 + row];
      }
#pragma unroll
      for (int j = 0; j < 16; ++j) y[j] += bias;
      if (g.act) {
#pragma unroll
        for (int j = 0; j < 16; j += 2) {
          const float2 t = gelu2(make_float2(y[j], y[j + 1]));
          y[j] = t.x;
          y[j + 1] = t.y;
        }
      }
      const long m = m0 + rank + ((long)j0 << logS);  // of y[0]; the others S rows apart
      const long at = m * g.ldo + n, step = g.ldo << logS;
      if (g.kind == BAG_FP8_CODES) {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const uint32_t top = group_max<32>(in ? abs_bits(y[j]) : 0u);
          if (lane == 0) reinterpret_cast<uint32_t*>(red + j0 + j)[warp & 3] = top;
        }
        asm volatile("bar.sync 1, 128;" ::: "memory");  // the four epilogue warps
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          if (j0 + j >= mine) break;
          const uint4 r = red[j0 + j];
          const uint32_t b = e8m0_of(max(max(r.x, r.y), max(r.z, r.w)));
          if (in)
            reinterpret_cast<uint8_t*>(g.out)[at + j * step] =
                __nv_cvt_float_to_fp8(y[j] * e8m0_inverse(b), __NV_SATFINITE, __NV_E4M3);
          if (row == 0) g.out_s[(m + ((long)j << logS)) * g.ldos + n0 / kScaleBlock] = (uint8_t)b;
        }
      } else if (in) {
        if (g.kind == BAG_FP8_BF16) {
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (j0 + j < mine) reinterpret_cast<__nv_bfloat16*>(g.out)[at + j * step] = __float2bfloat16_rn(y[j]);
        } else {
          float* o = reinterpret_cast<float*>(g.out) + at;
          if (g.kind == BAG_FP8_RESID) {
            float h[16];
#pragma unroll
            for (int j = 0; j < 16; ++j) h[j] = j0 + j < mine ? o[j * step] : 0.f;
#pragma unroll
            for (int j = 0; j < 16; ++j) y[j] = h[j] + gate * y[j];
          }
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (j0 + j < mine) o[j * step] = y[j];
        }
      }
      __syncwarp();
    }
  }
  __syncthreads();
  if (threadIdx.x == 0 && !ok && g.err) atomicOr(g.err, 1);
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, C::TMEM_COLS);
  }
}

// SMs that clusters of S CTAs reach (a cluster stays inside one group of SMs).
static long cluster_sms(int logS) {
  const long sms = sm_count();
  return logS < 2 ? sms : (logS == 2 ? sms - sms / 19 : sms - sms / 19 * 4);  // 152, 152, 144, 120 of 152
}

// K blocks of the longest of S parts.
static int few_longest(int S, int nkb) {
  int most = 0;
  for (int r = 0; r < S; ++r) most = std::max(most, few_cut(r + 1, S, nkb) - few_cut(r, S, nkb));
  return most;
}

template <int BN>
static cudaError_t launch_few(const Fp8Gemm& g, int logS, cudaStream_t s) {
  CUtensorMap tw, ta;
  if (encode_tmap_2d_bytes(&tw, 1, g.w, (uint64_t)g.K, (uint64_t)g.N, (uint64_t)g.ldw, F8_BK, 128) ||
      encode_tmap_2d_bytes(&ta, 1, g.a, (uint64_t)g.K, (uint64_t)g.M, (uint64_t)g.lda, F8_BK, BN))
    return cudaErrorInvalidValue;
  const long units = (long)((g.M + BN - 1) / BN) * ((g.N + 127) / 128);
  if (units << logS > 0x7fffffffL) return cudaErrorInvalidConfiguration;
  const long sms = cluster_sms(logS), ctas = units << logS;
  const int stages = FewCfg<BN>::stages(ctas <= sms ? 1 : (ctas <= 2 * sms ? 2 : 3));
  auto launch = [&](auto kernel) {
    return launch_cluster(kernel, logS > 0 ? 1u << logS : 0u, (unsigned)ctas, 256,
                          stages * FewCfg<BN>::STAGE + FewCfg<BN>::REST, s, tw, ta, g, logS, stages);
  };
  const int part = few_longest(1 << logS, (g.K + F8_BK - 1) / F8_BK);
  return part > pass_blocks(g.kind) ? launch(gemm_fp8_few_kernel<BN, true>) : launch(gemm_fp8_few_kernel<BN, false>);
}

// ---------------------------------------------------------------------------
// Many rows: CTA pairs
// ---------------------------------------------------------------------------
// Clusters of two CTAs compute 256 x 256 tiles (M = 256, N = 256, K = 32 an instruction), each CTA
// staging its 128 rows of A and of W and receiving its 128 rows of the accumulator; both hold the
// scales of all 256 columns.  Persistent, in an order that shares A's rows in L2.
// Two accumulators of 256 columns fill tensor memory, which the scales need a little of: the second
// one starts 32 columns inside the first (columns 224 .. 479), and the tile after this one waits
// only for this one's drain of the shared 32 columns, which the epilogue reads first.
// Tiles of a last wave that would leave half of the pairs idle are worked on as two halves of 128
// columns (M = 256, N = 128).
// Bound: tensor cores and power.  A K block takes about 650 cycles of 512 ideal ones (a stage of the ring comes
// round in 3300); 8192^3 to fp32 287 to 300 us, 4608 x 12288 x 3072 with GELU to codes 109 (3190 TFLOP/s;
// floor 92), 4608 x 3072 x 12288 into the residual stream 107.
// warp 0: TMA producer; 1: MMA (even CTA); 2: scale words to shared memory; 3 (even CTA): and to
// tensor memory; 4 .. 11: epilogue, two warps to each lane quarter, 128 columns (one output block) each.
// The epilogue is the longer part of a tile with few K blocks (24 are 12,300 cycles), so it keeps a
// row a thread, with bias and gate broadcast from shared memory, and its output leaves by TMA:
// stores, or for the residual stream an add that L2 carries out, so that the stream is not read.
constexpr int F8P_STAGES = 5, F8P_STAGE = 2 * F8_TILE;
constexpr int F8P_SHARED = 32, F8P_ACC1 = 256 - F8P_SHARED;  // TMEM columns
constexpr int F8P_SF_COL = F8P_ACC1 + 256, F8P_SF_COLS = 12;  // A's 4 columns, W's 8
constexpr int F8P_SF_GROUP = 3 * F8_ATOM, F8P_SF_STAGE = F8_RUN * F8P_SF_GROUP;
constexpr int F8P_BUF = 32 * 128;    // bytes of an epilogue warp's staged output: 32 rows of 128 bytes
constexpr int F8P_OFF_BUF = F8P_STAGES * F8P_STAGE;
constexpr int F8P_OFF_SF = F8P_OFF_BUF + 8 * F8P_BUF;
constexpr int F8P_OFF_VEC = F8P_OFF_SF + 2 * F8P_SF_STAGE;  // bias and gate of each warp's 128 columns
constexpr int F8P_OFF_BAR = F8P_OFF_VEC + 8 * 2 * 512;
constexpr int F8P_SMEM = F8P_OFF_BAR + 256 + 1024;
constexpr int F8P_THREADS = 384;
// registers a thread: 168 at launch; 128 * 88 + 256 * 208 = 384 * 168
constexpr int F8P_REGS_ISSUE = 88, F8P_REGS_EPI = 208;
static_assert(F8P_SF_COL + 2 * F8P_SF_COLS <= 512, "tensor memory");
static_assert(F8P_SMEM <= 232448, "shared memory");

namespace {

BAG_DEV void copy_scales_pair(uint32_t taddr, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}

BAG_DEV void pair_mma_mxf8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb,
                           uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(acc)
      : "memory");
}

// A tile in shared memory to (or added to) the tensor of `map` at column x, row y; rows past its
// last are left out.
BAG_DEV void tma_store_2d(const CUtensorMap* map, const void* smem, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(
                   reinterpret_cast<uint64_t>(map)),
               "r"(x), "r"(y), "r"(smem_u32(smem))
               : "memory");
}
BAG_DEV void tma_add_2d(const CUtensorMap* map, const void* smem, int x, int y) {
  asm volatile("cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(
                   reinterpret_cast<uint64_t>(map)),
               "r"(x), "r"(y), "r"(smem_u32(smem))
               : "memory");
}
BAG_DEV void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
BAG_DEV void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
BAG_DEV void bulk_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

// f(v[j], s[j]) of 32 columns, two at a time (16-byte broadcasts from shared memory).
template <typename F>
BAG_DEV void with_vector(const float* s, float* v, F f) {
#pragma unroll
  for (int j = 0; j < 32; j += 4) {
    const float4 b = *reinterpret_cast<const float4*>(s + j);
    const float2 x = f(make_float2(v[j], v[j + 1]), make_float2(b.x, b.y));
    const float2 y = f(make_float2(v[j + 2], v[j + 3]), make_float2(b.z, b.w));
    v[j] = x.x;
    v[j + 1] = x.y;
    v[j + 2] = y.x;
    v[j + 3] = y.y;
  }
}

// 16-byte unit u of this lane's 128-byte row in a staged tile (the 128-byte swizzle of TMA).
BAG_DEV uint4& staged(uint8_t* buf, int u) {
  const int lane = threadIdx.x & 31;
  return *reinterpret_cast<uint4*>(buf + lane * 128 + ((u ^ (lane & 7)) << 4));
}

// A staged tile (32 rows of 128 bytes: W columns of T) to rows that TMA cannot address or past whose
// end it would write, a row at a time, lane after lane along it.
template <typename T, bool ADD>
BAG_DEV void store_rows(const Fp8Gemm& g, const uint8_t* buf, int row0, int col0) {
  constexpr int W = 128 / (int)sizeof(T);
  const int lane = threadIdx.x & 31;
  T* o = reinterpret_cast<T*>(g.out) + (long)row0 * g.ldo + col0;
  const int rows = min(32, g.M - row0);
#pragma unroll 4
  for (int r = 0; r < rows; ++r) {
#pragma unroll
    for (int c = lane; c < W; c += 32) {
      const int byte = c * (int)sizeof(T);
      const T v = *reinterpret_cast<const T*>(buf + r * 128 + ((((byte >> 4) ^ (r & 7)) << 4) | (byte & 15)));
      if (col0 + c < g.N) {
        T* p = o + (long)r * g.ldo + c;
        if constexpr (ADD)
          *p += v;
        else
          *p = v;
      }
    }
  }
}

}  // namespace

template <int KIND, bool LONG>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(F8P_THREADS, 1)
    gemm_fp8_pair_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmW,
                         const __grid_constant__ CUtensorMap tmHalf, const __grid_constant__ CUtensorMap tmOut,
                         const __grid_constant__ Fp8Gemm g, int group_rows, long whole) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + F8P_OFF_BAR);
  uint64_t* empty = full + F8P_STAGES;
  uint64_t* sf_full = empty + F8P_STAGES;
  uint64_t* sf_empty = sf_full + 2;
  uint64_t* sf_ready = sf_empty + 2;   // [2], even CTA: a group's scales are in tensor memory
  uint64_t* sf_used = sf_ready + 2;    // [2], even CTA: a group's products are done, its TMEM columns free
  uint64_t* tfull = sf_used + 2;
  uint64_t* tempty = tfull + 2;
  uint64_t* shared_free = tempty + 2;  // [2]: accumulator b's columns that the other one shares are drained
  uint64_t* drain = shared_free + 2;
  uint64_t* sf_drain = drain + 1;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sf_drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1, npairs = gridDim.x >> 1;
  const int num_m = (g.M + 255) / 256, num_n = (g.N + 255) / 256;
  const int nkb = (g.K + F8_BK - 1) / F8_BK, nruns = (nkb + F8_GROUP * F8_RUN - 1) / (F8_GROUP * F8_RUN);
  const int pass_kb = LONG ? pass_length(nkb, pass_blocks(KIND)) : nkb;
  const int passes = LONG ? (nkb + pass_kb - 1) / pass_kb : 1;
  // units of work: `whole` tiles of 256 x 256, then every later tile as two of 256 x 128
  const long units = 2 * (long)num_m * num_n - whole;
  // first row and column of a unit, and whether it is half a tile; groups of group_rows row tiles
  // visit every column tile, the row tile varying fastest
  auto decode = [&](long unit, int& m0, int& n0) {
    const bool half = unit >= whole;
    const long tile = half ? whole + ((unit - whole) >> 1) : unit;
    const long per = (long)group_rows * num_n;
    const int gr = (int)(tile / per);
    const int i = (int)(tile - gr * per), rows = min(group_rows, num_m - gr * group_rows);
    m0 = (gr * group_rows + i % rows) * 256;
    n0 = i / rows * 256 + (half && ((unit - whole) & 1) ? 128 : 0);
    return half;
  };

  if (threadIdx.x == 0) {
    for (int s = 0; s < F8P_STAGES; ++s) {
      mbar_init(full + s, 1);   // even CTA: its producer's expect_tx; both CTAs' bytes
      mbar_init(empty + s, 1);  // both CTAs: one multicast commit per consumed stage
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(sf_full + s, 2);       // even CTA: both CTAs' scale warps
      mbar_init(sf_empty + s, 1);      // both CTAs: multicast commit
      mbar_init(sf_ready + s, 1);
      mbar_init(sf_used + s, 1);
      mbar_init(tfull + s, 1);         // both CTAs: multicast commit
      mbar_init(tempty + s, 16);       // even CTA: every epilogue warp of both CTAs
      mbar_init(shared_free + s, 8);   // even CTA: the warps that hold the shared columns
    }
    mbar_init(drain, 1);
    mbar_init(sf_drain, 1);
    *abort_flag = 0;
    fence_mbar_init();
    tma_prefetch_desc(&tmA);
    tma_prefetch_desc(whole > 0 ? &tmW : &tmHalf);
  }
  grid_dep_sync();
  __syncwarp();
  if (warp == 1) {
    tmem_alloc_pair(tmem_slot, 512);
    tmem_relinquish_pair();
  }
  tc_fence_before();
  __syncwarp();
  cluster_sync_all();  // barriers of both CTAs initialised, tensor memory allocated
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(F8P_REGS_ISSUE));
    if (warp == 0) {
      if (lane == 0) {
        // ---------------- TMA producer (both CTAs: their own halves) ----------------
        int s = 0;
        uint32_t ph = 0;
        long issued = 0;
        bool ok = true;
        for (long unit = pair; unit < units && ok; unit += npairs) {
          int m0, n0;
          const bool half = decode(unit, m0, n0);
          const CUtensorMap* mapW = half ? &tmHalf : &tmW;
          const int am = m0 + (int)rank * 128, wn = n0 + (int)rank * (half ? 64 : 128);
          const uint32_t bytes = half ? 2 * F8P_STAGE - F8_TILE : 2 * F8P_STAGE;  // of both CTAs
          for (int kb = 0; kb < nkb; ++kb) {
            if (!mbar_wait(empty + s, ph ^ 1, abort_flag)) {
              ok = false;
              break;
            }
            if (rank == 0) mbar_arrive_expect_tx(full + s, bytes);
            const uint32_t fb = mapa_shared(smem_u32(full + s), 0);
            pair_load_2d(smem + s * F8P_STAGE, &tmA, kb * F8_BK, am, fb);
            pair_load_2d(smem + s * F8P_STAGE + F8_TILE, mapW, kb * F8_BK, wn, fb);
            ++issued;
            if (++s == F8P_STAGES) {
              s = 0;
              ph ^= 1;
            }
          }
        }
        if (!ok && rank == 0) {
          // wait (bounded): both CTAs' copies in flight complete on this CTA's barriers
          const uint64_t t0 = global_ns();
          for (int i = 0; i < F8P_STAGES && i < issued; ++i) {
            if (--s < 0) {
              s = F8P_STAGES - 1;
              ph ^= 1;
            }
            while (!mbar_try_wait(full + s, ph) && global_ns() - t0 < kWaitLimitNs) {
            }
          }
        }
      }
    } else if (warp == 1) {
      if (rank == 0) {
        // -------- MMA issuer (even CTA; converged warp, one elected lane issues) --------
        const uint32_t base = smem_u32(smem), tm = uniform(tmem);
        int s = 0;
        uint32_t ph = 0;
        uint32_t grp = 0;  // groups of scales handled so far
        auto next = [&](int& st, uint32_t& parity) {
          if (++st == F8P_STAGES) {
            st = 0;
            parity ^= 1;
          }
        };
        long i = 0;            // accumulators of this pair so far
        int k0 = 0, k1 = 0;    // the pass's K blocks
        bool ok = true;
        for (long unit = pair; unit < units && ok; unit += k1 == nkb ? npairs : 0, ++i) {
          k0 = k1 == nkb ? 0 : k1;
          k1 = min(nkb, k0 + pass_kb);
          const int acc = (int)(i & 1);
          const uint32_t shape = unit >= whole ? idesc_mxf8(256, 128) : idesc_mxf8(256, 256);
          const uint32_t dt = tm + (acc ? F8P_ACC1 : 0);
          // the accumulator is drained, and the other one's shared columns
          if (!mbar_wait_warp(tempty + acc, (uint32_t)((i >> 1) & 1) ^ 1u, abort_flag)) break;
          if (i > 0 && !mbar_wait_warp(shared_free + (acc ^ 1), (uint32_t)(((i - 1) >> 1) & 1), abort_flag)) break;
          tc_fence_after();
          uint32_t add = 0;  // the first product overwrites the accumulator
          for (int kg = k0; kg < k1 && ok; kg += F8_GROUP, ++grp) {
            const uint32_t sa = tm + F8P_SF_COL + (grp & 1) * F8P_SF_COLS;
            if (!(ok = mbar_wait_warp(sf_ready + (grp & 1), (grp >> 1) & 1u, abort_flag))) break;
            // a K block at a time: to wait for two holds the first one's stage longer, and the ring is what
            // limits the rate (8192^3, operands of zeros: 297 us in pairs, 287 so; 348 with four stages)
#pragma unroll
            for (int b = 0; b < F8_GROUP; ++b) {
              if (kg + b >= k1) break;
              if (!(ok = mbar_wait_warp(full + s, ph, abort_flag))) break;
              tc_fence_after();
              const uint64_t a0 = sw128_desc(base + s * F8P_STAGE);
              if (elect_one()) {
#pragma unroll
                for (int k = 0; k < F8_BK / 32; ++k)  // 32 bytes along K: two 16-byte units
                  pair_mma_mxf8(dt, a0 + 2 * k, a0 + (F8_TILE >> 4) + 2 * k, shape | scale_byte(b), sa, sa + 4,
                                k > 0 ? 1u : add);
                pair_commit(empty + s, 3);
                if (b + 1 == F8_GROUP || kg + b + 1 >= k1) pair_commit(sf_used + (grp & 1), 1);
              }
              __syncwarp();
              add = 1;
              next(s, ph);
            }
          }
          if (!ok) break;
          if (elect_one()) pair_commit(tfull + acc, 3);
          __syncwarp();
        }
        // every issued MMA has finished before tensor memory is released
        if (elect_one()) {
          pair_commit(drain, 1);
          const uint64_t t0 = global_ns();
          while (!mbar_try_wait(drain, 0) && global_ns() - t0 < kWaitLimitNs) {
          }
        }
        __syncwarp();
      }
    } else if (warp == 3) {
      if (rank == 0) {
        // -------- scales to both CTAs' tensor memory, a group ahead of the products --------
        const uint32_t sf = smem_u32(smem + F8P_OFF_SF);
        uint32_t run = 0, grp = 0;  // runs and groups handled so far
        bool ok = true;
        for (long unit = pair; unit < units && ok; unit += npairs) {
          for (int kg = 0; kg < nkb; kg += F8_GROUP, ++grp) {
            if (kg % (F8_GROUP * F8_RUN) == 0) {
              if (!(ok = wait_warp_cluster(sf_full + (run & 1), (run >> 1) & 1u, abort_flag))) break;
              ++run;
            }
            if (!(ok = mbar_wait_warp(sf_used + (grp & 1), ((grp >> 1) & 1u) ^ 1u, abort_flag))) break;
            tc_fence_after();
            const uint32_t sa = tmem + F8P_SF_COL + (grp & 1) * F8P_SF_COLS;
            const uint64_t d = scale_desc(sf + ((run - 1) & 1) * F8P_SF_STAGE + kg / F8_GROUP % F8_RUN * F8P_SF_GROUP);
            if (elect_one()) {
#pragma unroll
              for (int a = 0; a < 3; ++a)
                if (a < 2 || unit < whole) copy_scales_pair(sa + 4 * a, d + a * (F8_ATOM >> 4));
              pair_commit(sf_ready + (grp & 1), 1);
              if (kg + F8_GROUP >= nkb || (kg / F8_GROUP + 1) % F8_RUN == 0) pair_commit(sf_empty + ((run - 1) & 1), 3);
            }
            __syncwarp();
          }
        }
        // every copy has ended before tensor memory is released
        if (elect_one()) {
          pair_commit(sf_drain, 1);
          const uint64_t t0 = global_ns();
          while (!mbar_try_wait(sf_drain, 0) && global_ns() - t0 < kWaitLimitNs) {
          }
        }
        __syncwarp();
      }
    } else if (warp == 2) {
      // ---------------- scale words (both CTAs: A's own rows, all 256 of W) ----------------
      int m0 = 0, n0 = 0, r = 0;
      bool half = false;
      const uint32_t full_even = mapa_shared(smem_u32(sf_full), 0);
      const bool wide_a = wide_scales(g.a_s, g.ldas), wide_w = wide_scales(g.w_s, g.ldws);
      ScaleRun w[3];
      auto fetch = [&]() {
        w[0].fetch(g.a_s, g.ldas, wide_a, m0 + (int)rank * 128, g.M, r, nkb);
        w[1].fetch(g.w_s, g.ldws, wide_w, n0, g.N, r, nkb);
        if (!half) w[2].fetch(g.w_s, g.ldws, wide_w, n0 + 128, g.N, r, nkb);
      };
      long unit = pair;
      if (unit < units) {
        half = decode(unit, m0, n0);
        fetch();
      }
      for (uint32_t i = 0; unit < units; ++i) {
        if (!mbar_wait_warp(sf_empty + (i & 1), ((i >> 1) & 1u) ^ 1u, abort_flag)) break;
        uint8_t* d = smem + F8P_OFF_SF + (i & 1) * F8P_SF_STAGE;
#pragma unroll
        for (int a = 0; a < 3; ++a)
          if (a < 2 || !half) w[a].put(d + a * F8_ATOM, F8P_SF_GROUP);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) peer_arrive(full_even + (uint32_t)((i & 1) * sizeof(uint64_t)));
        if (++r == nruns) {
          r = 0;
          unit += npairs;
          if (unit < units) half = decode(unit, m0, n0);
        }
        if (unit < units) fetch();
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(F8P_REGS_EPI));
    // ---------------- epilogue (both CTAs: their 128 rows of each tile) ----------------
    const int q = warp & 3, side = (warp - 4) >> 2;  // columns 0 .. 127 of a tile, 128 .. 255
    uint8_t* buf = smem + F8P_OFF_BUF + (warp - 4) * F8P_BUF;
    float* sbias = reinterpret_cast<float*>(smem + F8P_OFF_VEC) + (warp - 4) * 256;
    float* sgate = sbias + 128;
    const uint32_t tempty_even = mapa_shared(smem_u32(tempty), 0), free_even = mapa_shared(smem_u32(shared_free), 0);
    constexpr int CW = KIND == BAG_FP8_BF16 ? 64 : (KIND == BAG_FP8_CODES ? 128 : 32);  // columns of a staged row
    constexpr int NC = 128 / CW;
    long i = 0;  // accumulators so far
    for (long unit = pair; unit < units; unit += npairs) {
      int m0, n0;
      const bool half = decode(unit, m0, n0);
      const int row0 = m0 + (int)rank * 128 + q * 32, col0 = n0 + side * 128;
      {
        float b[4], t[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int c = col0 + lane * 4 + j;
          b[j] = g.bias && c < g.N ? __ldg(g.bias + c) : 0.f;
          t[j] = KIND == BAG_FP8_RESID && g.gate && c < g.N ? __ldg(g.gate + c) : 1.f;
        }
        reinterpret_cast<float4*>(sbias)[lane] = make_float4(b[0], b[1], b[2], b[3]);
        if (KIND == BAG_FP8_RESID) reinterpret_cast<float4*>(sgate)[lane] = make_float4(t[0], t[1], t[2], t[3]);
        __syncwarp();
      }
      uint32_t tb = 0;
      int acc = 0;
      bool shares = false;  // whether this warp's columns are shared: the last 32 of accumulator 0, the first 32 of 1
      auto begin = [&]() {
        acc = (int)(i & 1);
        const bool ok = mbar_wait(tfull + acc, (uint32_t)((i >> 1) & 1), abort_flag);
        ++i;
        if (!__all_sync(0xffffffffu, ok)) return false;
        tc_fence_after();
        tb = tmem + (uint32_t)((acc ? F8P_ACC1 : 0) + side * 128) + ((uint32_t)(q * 32) << 16);
        shares = side == (acc ^ 1);
        return true;
      };
      auto release = [&](uint32_t bar) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) peer_signal(bar + (uint32_t)(acc * sizeof(uint64_t)));
      };
      // CW finished sums from column c of this warp's 128 on, to where they go
      auto finish = [&](float* v, int c) {
      if (g.bias) {
#pragma unroll
        for (int j = 0; j < CW; j += 32) with_vector(sbias + c + j, v + j, sum2);
      }
      if (g.act) {
#pragma unroll
        for (int j = 0; j < CW; j += 2) {
          const float2 t = gelu2(make_float2(v[j], v[j + 1]));
          v[j] = t.x;
          v[j + 1] = t.y;
        }
      }
      if (KIND == BAG_FP8_RESID) with_vector(sgate + c, v, mul2);
      // the staged tile's last store has read it
      if (lane == 0) bulk_wait_read();
      __syncwarp();
      if constexpr (KIND == BAG_FP8_CODES) {
        const int valid = g.N - col0;
        float m[4] = {0.f, 0.f, 0.f, 0.f};
        if (valid < 128) {  // columns past the end count as zeros
#pragma unroll
          for (int j = 0; j < 128; ++j) v[j] = j < valid ? v[j] : 0.f;
        }
#pragma unroll
        for (int j = 0; j < 128; j += 2) m[(j >> 1) & 3] = max3_abs(m[(j >> 1) & 3], v[j], v[j + 1]);
        const uint32_t b = e8m0_of(abs_bits(max3_abs(max3_abs(m[0], m[1], m[2]), m[3], 0.f)));
        const float inv = e8m0_inverse(b);
        if (valid > 0 && row0 + lane < g.M) g.out_s[(long)(row0 + lane) * g.ldos + col0 / kScaleBlock] = (uint8_t)b;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          uint32_t w[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float* x = v + 16 * u + 4 * e;
            const float2 lo = mul2(make_float2(x[0], x[1]), make_float2(inv, inv));
            const float2 hi = mul2(make_float2(x[2], x[3]), make_float2(inv, inv));
            w[e] = pack_e4m3x4(lo.x, lo.y, hi.x, hi.y);
          }
          staged(buf, u) = make_uint4(w[0], w[1], w[2], w[3]);
        }
      } else if constexpr (KIND == BAG_FP8_BF16) {
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const float* x = v + 8 * u;
          staged(buf, u) = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                                      pack_bf16x2(x[6], x[7]));
        }
      } else {
#pragma unroll
        for (int u = 0; u < 8; ++u)
          staged(buf, u) = make_uint4(__float_as_uint(v[4 * u]), __float_as_uint(v[4 * u + 1]),
                                      __float_as_uint(v[4 * u + 2]), __float_as_uint(v[4 * u + 3]));
      }
      // TMA writes whole 16-byte units, also where the tensor ends inside one: the last columns
      // go the other way
      if (g.vec && col0 + c + CW <= g.N) {
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0 && row0 < g.M) {
          if (KIND == BAG_FP8_RESID)
            tma_add_2d(&tmOut, buf, col0 + c, row0);
          else
            tma_store_2d(&tmOut, buf, col0 + c, row0);
          bulk_commit();
        }
      } else {
        __syncwarp();
        if constexpr (KIND == BAG_FP8_CODES)
          store_rows<uint8_t, false>(g, buf, row0, col0 + c);
        else if constexpr (KIND == BAG_FP8_BF16)
          store_rows<__nv_bfloat16, false>(g, buf, row0, col0 + c);
        else
          store_rows<float, KIND == BAG_FP8_RESID>(g, buf, row0, col0 + c);
        __syncwarp();
      }
        __syncwarp();
      };
      bool ok = true;
      if (half && side) {  // half a tile has no columns for these warps
        for (int pass = 0; pass < passes && (ok = begin()); ++pass) {
          if (shares) release(free_even);
          release(tempty_even);
        }
      } else if constexpr (LONG) {
        // the first pass's loads are in flight together (a wait for each 16 columns, added to zeros:
        // 4608 x 12288 x 3072 codes 114 us against 110)
        float v[128];
        if (!(ok = begin())) break;
        auto load = [&](int c) { tmem_ld32_nowait(tb + (uint32_t)c, reinterpret_cast<uint32_t*>(v) + c); };
        if (acc) {  // the shared columns first
          load(0);
          tmem_ld_wait();
          if (shares) release(free_even);
          load(96);
        } else {
          load(96);
          tmem_ld_wait();
          if (shares) release(free_even);
          load(0);
        }
        load(32);
        load(64);
        tmem_ld_wait();
        release(tempty_even);
#pragma unroll 1
        for (int pass = 1; pass < passes && (ok = begin()); ++pass) {
          auto add = [&](int c) {
            float t[32];
            tmem_ld32(tb + (uint32_t)c, t);
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
              const float2 w = sum2(make_float2(v[c + j], v[c + j + 1]), make_float2(t[j], t[j + 1]));
              v[c + j] = w.x;
              v[c + j + 1] = w.y;
            }
          };
          if (acc) {
            add(0);
            if (shares) release(free_even);
            add(96);
          } else {
            add(96);
            if (shares) release(free_even);
            add(0);
          }
          add(32);
          add(64);
          release(tempty_even);
        }
        if (!ok) break;
#pragma unroll
        for (int c = 0; c < 128; c += CW) finish(v + c, c);
      } else {
        if (!(ok = begin())) break;
#pragma unroll 1
        for (int k = 0; k < NC; ++k) {
          const int c = (acc ? k : NC - 1 - k) * CW;  // the shared columns' part first
          float v[CW];
          // whole 32-column loads, the shared columns' first
          if (!acc) tmem_ld32(tb + (uint32_t)(c + CW - 32), v + CW - 32);
          if (acc) tmem_ld32(tb + (uint32_t)c, v);
          if (k == 0 && shares) release(free_even);
#pragma unroll
          for (int j = 0; j < CW; j += 32) {
            if (j > 0 && j < CW - 32) tmem_ld32(tb + (uint32_t)(c + j), v + j);
          }
          if (CW > 32) {
            if (acc)
              tmem_ld32(tb + (uint32_t)(c + CW - 32), v + CW - 32);
            else
              tmem_ld32(tb + (uint32_t)c, v);
          }
          if (k == NC - 1) release(tempty_even);
          finish(v, c);
        }
      }
      if (!ok) break;
    }
    if (lane == 0) bulk_wait_all();
    __syncwarp();
  }
  tc_fence_before();
  __syncwarp();
  cluster_sync_all();  // no CTA of the pair still uses the pair's tensor memory
  if (threadIdx.x == 0 && *abort_flag && g.err) atomicOr(g.err, 1);
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem, 512);
  }
}

// Tiles that keep their size: those of the last wave are halved where that gives each pair at most
// one half.
static long whole_tiles(long tiles, long pairs) {
  const long rest = tiles % pairs;
  return 2 * rest <= pairs ? tiles - rest : tiles;
}

static cudaError_t launch_pair(Fp8Gemm g, cudaStream_t s) {
  CUtensorMap ta, tw, th;
  if (encode_tmap_2d_bytes(&ta, 1, g.a, (uint64_t)g.K, (uint64_t)g.M, (uint64_t)g.lda, F8_BK, 128) ||
      encode_tmap_2d_bytes(&tw, 1, g.w, (uint64_t)g.K, (uint64_t)g.N, (uint64_t)g.ldw, F8_BK, 128) ||
      encode_tmap_2d_bytes(&th, 1, g.w, (uint64_t)g.K, (uint64_t)g.N, (uint64_t)g.ldw, F8_BK, 64))
    return cudaErrorInvalidValue;
  // the output map: boxes of 32 rows of 128 bytes; rows that TMA cannot address are stored otherwise
  CUtensorMap to = ta;
  const int size = g.kind == BAG_FP8_CODES ? 1 : (g.kind == BAG_FP8_BF16 ? 2 : 4);
  g.vec = ((reinterpret_cast<uintptr_t>(g.out) | (uintptr_t)(g.ldo * size)) & 15) == 0;
  if (g.vec && encode_tmap_2d_bytes(&to, size, g.out, (uint64_t)g.N, (uint64_t)g.M, (uint64_t)(g.ldo * size),
                                    128u / (unsigned)size, 32))
    return cudaErrorInvalidValue;
  const int num_m = (g.M + 255) / 256, num_n = (g.N + 255) / 256;
  const long tiles = (long)num_m * num_n, most = std::max(1, sm_count() / 2), whole = whole_tiles(tiles, most);
  const int pairs = (int)std::min(2 * tiles - whole, most);
  const int rows = (int)std::max(1.0, std::min((double)num_m, 40.0 * 1048576.0 / (256.0 * g.K)));
  auto launch = [&](auto kernel) {
    return launch_kernel(kernel, 2 * pairs, F8P_THREADS, F8P_SMEM, s, ta, tw, th, to, g, rows, whole);
  };
  const bool l = g.K > pass_blocks(g.kind) * F8_BK;
  switch (g.kind) {
    case BAG_FP8_F32: return l ? launch(gemm_fp8_pair_kernel<BAG_FP8_F32, true>) : launch(gemm_fp8_pair_kernel<BAG_FP8_F32, false>);
    case BAG_FP8_BF16: return l ? launch(gemm_fp8_pair_kernel<BAG_FP8_BF16, true>) : launch(gemm_fp8_pair_kernel<BAG_FP8_BF16, false>);
    case BAG_FP8_CODES: return l ? launch(gemm_fp8_pair_kernel<BAG_FP8_CODES, true>) : launch(gemm_fp8_pair_kernel<BAG_FP8_CODES, false>);
    default: return l ? launch(gemm_fp8_pair_kernel<BAG_FP8_RESID, true>) : launch(gemm_fp8_pair_kernel<BAG_FP8_RESID, false>);
  }
}

cudaError_t gemm_fp8_init() {
  cudaError_t r = cudaSuccess;
  auto smem = [&](auto kernel, int bytes) {
    if (r == cudaSuccess) r = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  };
  smem(gemm_fp8_few_kernel<16, false>, FewCfg<16>::stages(1) * FewCfg<16>::STAGE + FewCfg<16>::REST);
  smem(gemm_fp8_few_kernel<16, true>, FewCfg<16>::stages(1) * FewCfg<16>::STAGE + FewCfg<16>::REST);
  smem(gemm_fp8_few_kernel<32, false>, FewCfg<32>::stages(1) * FewCfg<32>::STAGE + FewCfg<32>::REST);
  smem(gemm_fp8_few_kernel<32, true>, FewCfg<32>::stages(1) * FewCfg<32>::STAGE + FewCfg<32>::REST);
  smem(gemm_fp8_few_kernel<64, false>, FewCfg<64>::stages(1) * FewCfg<64>::STAGE + FewCfg<64>::REST);
  smem(gemm_fp8_few_kernel<64, true>, FewCfg<64>::stages(1) * FewCfg<64>::STAGE + FewCfg<64>::REST);
  smem(gemm_fp8_few_kernel<128, false>, FewCfg<128>::stages(1) * FewCfg<128>::STAGE + FewCfg<128>::REST);
  smem(gemm_fp8_few_kernel<128, true>, FewCfg<128>::stages(1) * FewCfg<128>::STAGE + FewCfg<128>::REST);
  smem(gemm_fp8_pair_kernel<BAG_FP8_F32, false>, F8P_SMEM);
  smem(gemm_fp8_pair_kernel<BAG_FP8_F32, true>, F8P_SMEM);
  smem(gemm_fp8_pair_kernel<BAG_FP8_BF16, false>, F8P_SMEM);
  smem(gemm_fp8_pair_kernel<BAG_FP8_BF16, true>, F8P_SMEM);
  smem(gemm_fp8_pair_kernel<BAG_FP8_CODES, false>, F8P_SMEM);
  smem(gemm_fp8_pair_kernel<BAG_FP8_CODES, true>, F8P_SMEM);
  smem(gemm_fp8_pair_kernel<BAG_FP8_RESID, false>, F8P_SMEM);
  smem(gemm_fp8_pair_kernel<BAG_FP8_RESID, true>, F8P_SMEM);
  return r;
}

// Which kernel, tile and split: the least expected time.  The constants (us) fit 247 shapes of 1 to
// 2048 rows, 512 to 13824 columns and K, each timed under every choice (3000 timings, chained
// launches); the choice is within 1.1 % of the best one on average, 24 % at most (50 rows through
// 5120 x 13824).  A CTA of either kernel takes about 0.2 us a K block whatever its tile (the issue
// of its four MMAs and their waits), so few tiles want K split, and many the largest tile.
struct Fp8Plan {
  int BN;    // 0: CTA pairs
  int logS;
};
static Fp8Plan plan_fp8(long M, long N, long K, int kind) {
  auto cd = [](long a, long b) { return (a + b - 1) / b; };
  const double nkb = (double)cd(K, F8_BK);
  // the operands' way from HBM beside the time of the CTAs: a smooth maximum of the two, so that of
  // splits that HBM bounds alike the one with more loads in flight is taken
  const double dram = (double)(M + N) * (double)K / 6.5e6 + 3.8;
  auto pow8 = [](double x) {
    x *= x;
    x *= x;
    return x * x;
  };
  const double dram8 = pow8(dram);
  auto together = [&](double us) { return std::sqrt(std::sqrt(std::sqrt(pow8(us) + dram8))); };
  const long full = cd(M, 256) * cd(N, 256), pairs = std::max(1, sm_count() / 2), whole = whole_tiles(full, pairs);
  double us = 4.6 + (double)cd(whole, pairs) * (3.6 + 0.27 * nkb);
  if (whole < full) us += 1.6 + 0.19 * nkb;  // a wave of halves
  double best = together(us);
  Fp8Plan p{0, 0};
  const struct {
    int BN;
    double start, wave, share;  // of a launch, of a further wave, of its K blocks (SMs shared)
  } tiles[] = {{16, 2.6, 1.3, 0.01}, {32, 2.5, 2.0, 0.01}, {64, 5.8, 3.4, 0.28}, {128, 6.2, 5.7, 0.28}};
  for (const auto& t : tiles) {
    if (t.BN < 64 && M > t.BN) continue;  // narrow tiles read W again for every tile of rows
    for (int logS = 0; logS <= 3 && nkb >= (double)(2 << logS); ++logS) {
      const double kb = (double)cd(cd(K, F8_BK), 1L << logS);
      if (kb > pass_blocks(kind) && logS < 3) continue;  // passes (LONG) only where eight parts are too long still
      const double more = (double)(cd(cd(M, t.BN) * cd(N, 128) << logS, cluster_sms(logS)) - 1);
      us = together(t.start + 0.2 * kb + more * (t.wave + t.share * kb) + (logS ? 0.84 : 0.0) + 0.15 * (1 << logS));
      if (us < best) {
        best = us;
        p = Fp8Plan{t.BN, logS};
      }
    }
  }
  return p;
}

cudaError_t gemm_fp8(Fp8Gemm g, cudaStream_t s) {
  if (g.M <= 0 || g.N <= 0) return cudaSuccess;
  const Fp8Plan p = plan_fp8(g.M, g.N, g.K, g.kind);
  switch (p.BN) {
    case 16: return launch_few<16>(g, p.logS, s);
    case 32: return launch_few<32>(g, p.logS, s);
    case 64: return launch_few<64>(g, p.logS, s);
    case 128: return launch_few<128>(g, p.logS, s);
    default: return launch_pair(g, s);
  }
}

}  // namespace bag
