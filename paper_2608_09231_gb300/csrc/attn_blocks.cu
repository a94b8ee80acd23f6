// Attention over selected blocks of keys, on the 5th-generation tensor cores (heads of 128, 16-bit
// operands): softmax(q k^T / sqrt(128)) v for each block of 128 queries over the key blocks of its
// own list.
//
// One CTA works on two slots, each a block of queries with a list of key blocks:
//   warp 0       TMA producer: the queries, then K and V^T blocks of both slots through one ring,
//                in the order in which the MMAs consume them
//   warp 1       MMA issuer, in turn between the slots:
//                  S_A,0  S_B,0 | PV_A,j  S_A,j+1 | PV_B,j  S_B,j+1 | ...
//                so that one slot's products run beside the other's softmax
//   warps 4..7   softmax of slot A, 8..11 of slot B: thread = query row; the row's scores are read
//                from TMEM at once, P = exp2(s - m) goes back over them in 16 bits and enters the
//                PV product from TMEM; O stays in TMEM and is rescaled only when the running
//                maximum has grown by more than 8 (in log2 units)
// P has 16 bits because both operands of an MMA are of one type and V's are given; the sum l is of the
// unrounded P, in fp32.  Against 64 bits (2-norm) fp16 is off by 1.67e-3, the output's own rounding to
// bf16 (1.66e-3); bf16 by 2.2e-3, its P adding eight-bit roundings of about the output's size.  Two
// products of a P in two bf16 parts would take that away for half as much tensor work again; the dense
// kernel makes the same choice, and a caller who wants the bits has fp16.
// The slots are two (head, query block) units, or one unit is shared: its list is cut into 2 C
// parts for a cluster of C CTAs, and rank r merges 128 / C rows of the 2 C partial outputs through
// distributed shared memory.  A launch in pairs shares (C = 1) the units of its last wave where
// they would leave half of the slots idle.
//
// Bound: shared memory.  Lists differ from slot to slot, so each slot loads its own K and V^T, and a step of
// both moves 320 KB through it (2560 cycles at 128 bytes; the products are 2048 and dense attention,
// whose slots share the tiles, takes 2800): 3400 cycles taken.  32,760 queries x 4 heads, 64 of 256
// blocks: 392 us (1402 TFLOP/s; floor 290), 40 heads 4.1 ms.
#include <algorithm>
#include <cmath>

#include "attn_common.cuh"
#include "epilogue.cuh"
#include "kernels.h"
#include "peer.cuh"

namespace bag {

namespace {
constexpr int BT = 128;                    // queries, keys and columns of a tile
constexpr int BT_CHUNK = BT * 64 * 2;      // 128 rows x 64 columns: one 128-byte swizzle column
constexpr int BT_TILE = 2 * BT_CHUNK;
constexpr int BT_STAGES = 5;               // of the ring (a K or V^T tile each)
constexpr int BT_OFF_RING = 2 * BT_TILE;   // after the slots' queries
constexpr int BT_OFF_BAR = BT_OFF_RING + BT_STAGES * BT_TILE;
constexpr int BT_SMEM = BT_OFF_BAR + 256 + 1024;
constexpr int BT_TMEM_COLS = 512;          // S_A [0,128) S_B [128,256) O_A [256,384) O_B [384,512)
constexpr int BT_THREADS = 384;
// registers a thread: 168 at launch; 128 * 72 + 256 * 216 = 384 * 168
constexpr int BT_REGS_ISSUE = 72, BT_REGS_SOFTMAX = 216;
constexpr int BT_OLD = 36;                 // floats a row in the output transpose
// exchange of partial outputs over the tiles: 256 rows of 128 floats (4 more a row against
// bank conflicts), then (maximum, sum) of each
constexpr int BT_XLD = BT + 4;
constexpr int BT_OFF_ML = 2 * BT * BT_XLD * 4;
static_assert(BT_OFF_ML + 2 * BT * 8 <= BT_OFF_BAR, "the exchange fits the operand tiles");

struct BlockAttnParams {
  int nq, nk, nqb, nkb, keep, group;  // group: query heads of a key head
  long units;                         // heads * nqb
  const int* blocks;
  __nv_bfloat16* o;
  long ldo;
  float scale_log2;
  int c;                              // CTAs of a shared unit (PAIR: 1)
  int pairs;                          // PAIR: CTAs that work on two units; later ones share one each
  int* err;
};
}  // namespace

template <bool F16, bool PAIR>
__global__ void __launch_bounds__(BT_THREADS, 1)
    attn_blocks_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                       const __grid_constant__ CUtensorMap tmV, const BlockAttnParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  uint8_t* ring = smem + BT_OFF_RING;
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + BT_OFF_BAR);
  uint64_t* q_full = bars;
  uint64_t* full = bars + 1;               // [BT_STAGES]
  uint64_t* empty = full + BT_STAGES;      // [BT_STAGES]
  uint64_t* s_full = empty + BT_STAGES;    // [2] per slot
  uint64_t* p_full = s_full + 2;           // [2]
  uint64_t* o_done = p_full + 2;           // [2]
  uint64_t* drain = o_done + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* length = reinterpret_cast<int*>(tmem_slot + 2);  // [2] of the slots' lists

  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const bool pair = PAIR && (int)blockIdx.x < p.pairs;  // two units
  const int C = PAIR ? 1 : p.c;
  const int rank = !PAIR && C > 1 ? (int)cluster_ctarank() : 0;
  const long u0 = PAIR ? (pair ? 2L * blockIdx.x : (long)blockIdx.x + p.pairs) : (long)blockIdx.x / C;
  auto unit_of = [&](int x) { return pair ? u0 + x : u0; };
  auto list_of = [&](int x) { return p.blocks + unit_of(x) * p.keep; };

  if (threadIdx.x == 0) {
    mbar_init(q_full, 1);
    for (int i = 0; i < BT_STAGES; ++i) {
      mbar_init(full + i, 1);
      mbar_init(empty + i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_full + i, 1);
      mbar_init(p_full + i, 4);  // one arrival per softmax warp of the slot
      mbar_init(o_done + i, 1);
    }
    mbar_init(drain, 1);
    *abort_flag = 0;
    length[0] = unit_of(0) < p.units ? p.keep : 0;
    length[1] = unit_of(1) < p.units ? p.keep : 0;
    fence_mbar_init();
    tma_prefetch_desc(&tmQ);
    tma_prefetch_desc(&tmK);
    tma_prefetch_desc(&tmV);
  }
  grid_dep_sync();
  __syncthreads();
  // a list ends at its first entry that names no block
  for (int x = 0; x < (pair ? 2 : 1); ++x) {
    if (unit_of(x) >= p.units) continue;
    const int* list = list_of(x);
    for (int i = threadIdx.x; i < p.keep; i += BT_THREADS)
      if ((unsigned)__ldg(list + i) >= (unsigned)p.nkb) atomicMin(length + x, i);
  }
  __syncwarp();
  if (warp == 1) {
    tmem_alloc(tmem_slot, BT_TMEM_COLS);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  // slot x works on entries [first[x], first[x] + n[x]) of its list
  int first[2], n[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    if (pair) {
      first[x] = 0;
      n[x] = length[x];
    } else {
      const long part = 2 * rank + x, all = length[0];
      first[x] = (int)(part * all / (2 * C));
      n[x] = (int)((part + 1) * all / (2 * C)) - first[x];
    }
  }
  const int most = max(n[0], n[1]);

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(BT_REGS_ISSUE));
    if (warp == 0 && lane == 0 && most > 0) {
      // ---------------- TMA producer ----------------
      int kvx[2], qx[2], qy[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const long u = min(unit_of(x), p.units - 1);
        const int head = (int)(u / p.nqb);
        kvx[x] = head / p.group * BT;
        qx[x] = head * BT;
        qy[x] = (int)(u % p.nqb) * BT;
      }
      const int qt = pair ? 2 : 1;
      mbar_arrive_expect_tx(q_full, qt * BT_TILE);
      for (int x = 0; x < qt; ++x) {
        tma_load_2d(smem + x * BT_TILE, &tmQ, qx[x], qy[x], q_full);
        tma_load_2d(smem + x * BT_TILE + BT_CHUNK, &tmQ, qx[x] + 64, qy[x], q_full);
      }
      int s = 0, issued = 0;
      uint32_t ph = 1;
      bool ok = true;
      auto stage = [&]() {
        if (!(ok = ok && mbar_wait(empty + s, ph, abort_flag))) return false;
        mbar_arrive_expect_tx(full + s, BT_TILE);
        return true;
      };
      auto next = [&]() {
        ++issued;
        if (++s == BT_STAGES) {
          s = 0;
          ph ^= 1;
        }
      };
      auto load_k = [&](int x, int b) {
        if (!stage()) return;
        uint8_t* t = ring + s * BT_TILE;
        tma_load_2d(t, &tmK, kvx[x], b * BT, full + s);
        tma_load_2d(t + BT_CHUNK, &tmK, kvx[x] + 64, b * BT, full + s);
        next();
      };
      auto load_v = [&](int x, int b) {
        if (!stage()) return;
        uint8_t* t = ring + s * BT_TILE;
        tma_load_2d(t, &tmV, b * BT, kvx[x], full + s);
        tma_load_2d(t + BT_CHUNK, &tmV, b * BT + 64, kvx[x], full + s);
        next();
      };
      int now[2] = {0, 0};  // the block whose K was loaded last
#pragma unroll
      for (int x = 0; x < 2; ++x)
        if (n[x] > 0) {
          now[x] = __ldg(list_of(x) + first[x]);
          load_k(x, now[x]);
        }
      for (int j = 0; j < most && ok; ++j) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          if (j >= n[x]) continue;
          const int b = j + 1 < n[x] ? __ldg(list_of(x) + first[x] + j + 1) : 0;
          load_v(x, now[x]);
          if (j + 1 < n[x]) load_k(x, now[x] = b);
        }
      }
      if (!ok) {
        // wait (bounded) for copies still in flight before the CTA may exit
        const uint64_t t0 = global_ns();
        auto landed = [&](uint64_t* bar, uint32_t parity) {
          while (!mbar_try_wait(bar, parity) && global_ns() - t0 < kWaitLimitNs) {
          }
        };
        landed(q_full, 0);
        for (int i = max(0, issued - BT_STAGES); i < issued; ++i) landed(full + i % BT_STAGES, (i / BT_STAGES) & 1);
      }
    } else if (warp == 1 && most > 0) {
      // ---------------- MMA issuer (converged warp, one elected lane issues) ----------------
      constexpr uint32_t idesc = F16 ? idesc_f16_f32(BT, BT) : idesc_bf16_f32(BT, BT);
      const uint32_t q_addr = smem_u32(smem), r_addr = smem_u32(ring), tm = uniform(tmem);
      const int len[2] = {(int)uniform((uint32_t)n[0]), (int)uniform((uint32_t)n[1])};
      const int longest = max(len[0], len[1]);
      // K step kk of a tile: 64-column chunk kk / 4, 32 bytes per step inside it (16-byte units)
      auto koff = [](int kk) { return (uint64_t)(((kk >> 2) * BT_CHUNK + (kk & 3) * 32) >> 4); };
      int s = 0;
      uint32_t ph = 0;
      auto wait = [&](uint64_t* bar, uint32_t parity) {
        const bool w = mbar_wait_warp(bar, parity, abort_flag);
        tc_fence_after();
        return w;
      };
      auto next = [&]() {
        if (++s == BT_STAGES) {
          s = 0;
          ph ^= 1;
        }
      };
      auto issue_s = [&](int x) {  // scores of the ring's next tile
        if (!wait(full + s, ph)) return false;
        const uint64_t qd = sw128_desc(q_addr + (pair ? x * BT_TILE : 0));
        const uint64_t kd = sw128_desc(r_addr + s * BT_TILE);
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < BT / 16; ++kk)
            mma_bf16(tm + x * 128, qd + koff(kk), kd + koff(kk), idesc, kk > 0 ? 1u : 0u);
          mma_commit(s_full + x);
          mma_commit(empty + s);
        }
        __syncwarp();
        next();
        return true;
      };
      auto issue_pv = [&](int x, int j) {
        if (!wait(full + s, ph)) return false;
        const uint64_t vd = sw128_desc(r_addr + s * BT_TILE);
        if (elect_one()) {
#pragma unroll
          for (int kk = 0; kk < BT / 16; ++kk)
            mma_bf16_ts(tm + 256 + x * 128, tm + x * 128 + kk * 8, vd + koff(kk), idesc,
                        (j > 0 || kk > 0) ? 1u : 0u);
          mma_commit(empty + s);
          if (j + 1 == len[x]) mma_commit(o_done + x);
        }
        __syncwarp();
        next();
        return true;
      };
      bool ok = wait(q_full, 0);
#pragma unroll
      for (int x = 0; x < 2; ++x)
        if (len[x] > 0) ok = ok && issue_s(x);
      for (int j = 0; j < longest && ok; ++j) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          if (j >= len[x] || !ok) continue;
          ok = wait(p_full + x, j & 1) && issue_pv(x, j);
          if (ok && j + 1 < len[x]) ok = issue_s(x);
        }
      }
      if (elect_one()) {
        mma_commit(drain);
        const uint64_t t0 = global_ns();
        while (!mbar_try_wait(drain, 0) && global_ns() - t0 < kWaitLimitNs) {
        }
      }
    }
    __syncwarp();
    if (!pair) {  // the two barriers of the exchange
      if (!PAIR && C > 1) {
        cluster_sync_all();
        cluster_sync_all();
      } else {
        __syncthreads();
        __syncthreads();
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(BT_REGS_SOFTMAX));
    // ---------------- softmax warpgroups ----------------
    const int x = (warp - 4) >> 2;
    const int quad = warp & 3;
    const int mine = x ? n[1] : n[0];
    const int* list = list_of(x) + (x ? first[1] : first[0]);
    const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
    const uint32_t s_addr = tmem + lane_base + x * 128;
    const uint32_t o_addr = tmem + lane_base + 256 + x * 128;
    float m_use = -INFINITY, l = 0.f;
    bool ok = true;
    for (int j = 0; j < mine; ++j) {
      const int kvalid = p.nk - __ldg(list + j) * BT;  // keys of this block (< 128 only at the end)
      const bool w = mbar_wait(s_full + x, j & 1, abort_flag);
      if (!__all_sync(0xffffffffu, w)) {
        ok = false;
        break;
      }
      tc_fence_after();
      uint32_t r[BT];
#pragma unroll
      for (int c = 0; c < BT / 32; ++c) tmem_ld32_nowait(s_addr + c * 32, r + c * 32);
      tmem_ld_wait();
      if (kvalid < BT) {
#pragma unroll
        for (int i = 0; i < BT; ++i)
          if (i >= kvalid) r[i] = __float_as_uint(-INFINITY);
      }
      // row maximum: four independent chains of three-input maxima
      float mq[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) mq[u] = fmaxf(__uint_as_float(r[2 * u]), __uint_as_float(r[2 * u + 1]));
#pragma unroll
      for (int i = 8; i < BT; i += 8)
#pragma unroll
        for (int u = 0; u < 4; ++u)
          mq[u] = max3(mq[u], __uint_as_float(r[i + 2 * u]), __uint_as_float(r[i + 2 * u + 1]));
      const float mx2 = fmaxf(fmaxf(mq[0], mq[1]), fmaxf(mq[2], mq[3])) * p.scale_log2;
      float alpha = 1.f;
      if (mx2 > m_use + 8.f) {
        alpha = ex2(m_use - mx2);
        m_use = mx2;
        l *= alpha;
      }
      // a tile of nothing but -inf scores before any other weighs nothing
      const float neg_m = m_use == -INFINITY ? 0.f : -m_use;
      float ls0 = 0.f, ls1 = 0.f;
#pragma unroll
      for (int c = 0; c < BT / 32; ++c) {
        uint32_t pk[16];
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
          float x0, x1;
          fma2(x0, x1, __uint_as_float(r[c * 32 + i]), __uint_as_float(r[c * 32 + i + 1]), p.scale_log2, neg_m);
          const float a0 = ex2(x0), a1 = ex2(x1);
          add2(ls0, ls1, a0, a1);
          pk[i / 2] = F16 ? pack_f16x2(a0, a1) : pack_bf16x2(a0, a1);
        }
        tmem_st16(s_addr + c * 16, pk);
      }
      l += ls0 + ls1;
      // O holds PV of every earlier tile; rescale it before this tile's PV is issued
      if (j > 0 && __any_sync(0xffffffffu, alpha != 1.f)) {
#pragma unroll 1
        for (int c = 0; c < BT / 32; ++c) {
          float o[32];
          tmem_ld32(o_addr + c * 32, o);
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] *= alpha;
          tmem_st32(o_addr + c * 32, o);
        }
      }
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(p_full + x);
    }
    if (mine > 0 && ok) ok = __all_sync(0xffffffffu, mbar_wait(o_done + x, 0, abort_flag));
    tc_fence_after();
    if (pair) {
      const long u = unit_of(x);
      if (ok && u < p.units) {
        const int head = (int)(u / p.nqb), q0 = (int)(u % p.nqb) * BT;
        const float inv = 1.f / l;
        // through shared memory (this slot's queries, which no product reads any more): four
        // lanes hold 32 consecutive columns of a row, so a store covers eight rows' 64-byte runs.
        // An empty list's zeros stay out of it: its queries may still be landing there.
        float* buf = reinterpret_cast<float*>(smem + x * BT_TILE) + quad * 32 * BT_OLD;
        const int r = lane >> 2, c8 = (lane & 3) * 8;
        const int qw = q0 + quad * 32 + r;
#pragma unroll 1
        for (int c = 0; c < BT; c += 32) {
          float o[32];
          if (mine > 0) {
            tmem_ld32(o_addr + c, o);
#pragma unroll
            for (int i = 0; i < 32; i += 4)
              *reinterpret_cast<float4*>(buf + lane * BT_OLD + i) =
                  make_float4(o[i] * inv, o[i + 1] * inv, o[i + 2] * inv, o[i + 3] * inv);
          }
          __syncwarp();
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int q = qw + 8 * i;
            float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (mine > 0) ld_chunk<8>(buf + (8 * i + r) * BT_OLD + c8, v);
            if (q < p.nq) store_vals<8>(p.o, (long)q * p.ldo + head * BT + c + c8, v, kStoreBF16);
          }
          __syncwarp();
        }
      }
    } else {
      const int rpo = BT / C;  // rows a rank merges
      __syncwarp();
      if (!PAIR && C > 1)
        cluster_sync_all();  // every CTA's products are done: the operand tiles are free
      else
        __syncthreads();
      if (ok) {
        const int R = quad * 32 + lane;
        const int at = (2 * rank + x) * rpo + R % rpo;
        const uint32_t here = smem_u32(smem);
        const uint32_t dst = !PAIR && C > 1 ? mapa_shared(here, (uint32_t)(R / rpo)) : here;
#pragma unroll 1
        for (int c = 0; c < BT; c += 32) {
          float o[32];
          if (mine > 0) tmem_ld32(o_addr + c, o);
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] = mine > 0 ? o[i] : 0.f;
#pragma unroll
          for (int i = 0; i < 32; i += 4)
            peer_store4(dst + (uint32_t)(at * BT_XLD + c + i) * 4, o[i], o[i + 1], o[i + 2], o[i + 3]);
        }
        peer_store2(dst + BT_OFF_ML + (uint32_t)at * 8, m_use, l);
      }
      __syncwarp();
      if (!PAIR && C > 1)
        cluster_sync_all();  // every part has arrived; no access to another CTA follows
      else
        __syncthreads();
      const float* part = reinterpret_cast<const float*>(smem);
      const float2* ml = reinterpret_cast<const float2*>(smem + BT_OFF_ML);
      const int head = (int)(u0 / p.nqb), q0 = (int)(u0 % p.nqb) * BT;
      for (int lr = warp - 4; lr < rpo; lr += 8) {  // a warp a row, four columns a lane
        const int q = q0 + rank * rpo + lr;
        if (q >= p.nq) break;
        float m = -INFINITY, den = 0.f;
        for (int s = 0; s < 2 * C; ++s) m = fmaxf(m, ml[s * rpo + lr].x);
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int s = 0; s < 2 * C; ++s) {
          const float2 f = ml[s * rpo + lr];
          const float w = f.x == -INFINITY ? 0.f : ex2(f.x - m);
          const float4 o = *reinterpret_cast<const float4*>(part + (s * rpo + lr) * BT_XLD + lane * 4);
          den += w * f.y;
          acc.x += w * o.x;
          acc.y += w * o.y;
          acc.z += w * o.z;
          acc.w += w * o.w;
        }
        const float inv = length[0] > 0 ? 1.f / den : 0.f;
        uint2 u;
        u.x = pack_bf16x2(acc.x * inv, acc.y * inv);
        u.y = pack_bf16x2(acc.z * inv, acc.w * inv);
        *reinterpret_cast<uint2*>(p.o + (long)q * p.ldo + head * BT + lane * 4) = u;
      }
    }
  }
  __syncthreads();
  if (threadIdx.x == 0 && *abort_flag && p.err) atomicOr(p.err, 1);
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, BT_TMEM_COLS);
  }
}

// ---------------------------------------------------------------------------
// One query
// ---------------------------------------------------------------------------
// The scores of one query row are no matrix product: its keys and values are read once and used
// once, 64 KB a block, so the row is bound by HBM and by how many of those bytes are in flight.  A
// cluster of C CTAs shares a head's list; a CTA walks its part block by block on CUDA cores, with
// fp32 products, sums and probabilities.  Sixteen lanes hold a row of K (16 bytes each), or of V^T;
// eight rows a lane, so a warp takes 16 keys, then 16 columns of the output.  The values of a block
// are in flight while its scores are taken, the next block's keys while the values are summed.
// Rank 0 merges the ranks' sums in order.  40 heads x 32 blocks of 256: 15.4 us (5.5 TB/s; floor 12.4); 24
// heads x 8 blocks 4.5.
constexpr int TK_TH = 256, TK_MAX_C = 8;

// Element pairs of 16 bytes.
template <bool F16>
BAG_DEV float2 pair_of(uint32_t u) {
  if constexpr (F16)
    return __half22float2(*reinterpret_cast<const __half2*>(&u));
  else
    return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
}
template <bool F16>
BAG_DEV float dot8(uint4 u, const float* w) {
  const float2 a = pair_of<F16>(u.x), b = pair_of<F16>(u.y), c = pair_of<F16>(u.z), d = pair_of<F16>(u.w);
  float s = a.x * w[0];
  s = fmaf(a.y, w[1], s);
  s = fmaf(b.x, w[2], s);
  s = fmaf(b.y, w[3], s);
  s = fmaf(c.x, w[4], s);
  s = fmaf(c.y, w[5], s);
  s = fmaf(d.x, w[6], s);
  return fmaf(d.y, w[7], s);
}

// Sums of eight values over sixteen lanes, half of the values handed over in each step: the lane's
// result is value (its index within the sixteen) / 2.
BAG_DEV float sum_16lanes(float* v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int n = 4; n > 0; n /= 2) {  // lanes 2 n apart
    const bool up = lane & (2 * n);
#pragma unroll
    for (int j = 0; j < n; ++j) {
      const float give = up ? v[j] : v[j + n], keep = up ? v[j + n] : v[j];
      v[j] = keep + __shfl_xor_sync(0xffffffffu, give, 2 * n);
    }
  }
  return v[0] + __shfl_xor_sync(0xffffffffu, v[0], 1);
}

template <bool F16>
__global__ void __launch_bounds__(TK_TH, 2)
    attn_token_kernel(const uint16_t* __restrict__ q, const uint16_t* __restrict__ k, long ldk,
                      const uint16_t* __restrict__ v, long vpad, const BlockAttnParams p) {
  __shared__ __align__(16) float sc[2][BT];
  __shared__ float part[TK_MAX_C][BT];
  __shared__ float2 ml[TK_MAX_C];
  __shared__ int length;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, li = lane % 16, hl = lane / 16;
  const int C = p.c, rank = C > 1 ? (int)cluster_ctarank() : 0;
  const int head = (int)(blockIdx.x / C), kh = head / p.group;
  const int* list = p.blocks + (long)head * p.keep;
  if (threadIdx.x == 0) length = p.keep;
  if (C > 1)
    cluster_sync_all();  // every CTA has started
  else
    __syncthreads();
  grid_dep_sync();
  // a list ends at its first entry that names no block
  for (int i = threadIdx.x; i < p.keep; i += TK_TH)
    if ((unsigned)__ldg(list + i) >= (unsigned)p.nkb) atomicMin(&length, i);
  float qv[8];
  {
    const uint4 u = __ldg(reinterpret_cast<const uint4*>(q + head * BT) + li);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 t = pair_of<F16>(w[i]);
      qv[2 * i] = t.x * p.scale_log2;
      qv[2 * i + 1] = t.y * p.scale_log2;
    }
  }
  __syncthreads();
  const int first = (int)((long)rank * length / C), last = (int)((long)(rank + 1) * length / C);
  uint4 kr[8], vr[8];
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  auto load_k = [&](int b) {  // rows 2 i + hl of the warp's 16 keys
    const int key = b * BT + warp * 16 + hl;
    const uint16_t* r = k + (long)key * ldk + kh * BT + li * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      kr[i] = key + 2 * i < p.nk ? __ldg(reinterpret_cast<const uint4*>(r + (long)(2 * i) * ldk)) : zero;
  };
  auto load_v = [&](int b) {  // columns 2 i + hl of the warp's 16
    const int key = b * BT + li * 8;
    const uint16_t* r = v + ((long)kh * BT + warp * 16 + hl) * vpad + key;
#pragma unroll
    for (int i = 0; i < 8; ++i) vr[i] = key < p.nk ? __ldg(reinterpret_cast<const uint4*>(r + (long)(2 * i) * vpad)) : zero;
    const int left = p.nk - key;
    if (left > 0 && left < 8) {  // what lies past the last key may be anything
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        uint16_t* t = reinterpret_cast<uint16_t*>(&vr[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = j < left ? t[j] : (uint16_t)0;
      }
    }
  };
  float m = -INFINITY, l = 0.f, acc[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) acc[i] = 0.f;
  int b = first < last ? __ldg(list + first) : 0;
  if (first < last) load_k(b);
  for (int j = first; j < last; ++j) {
    float* s = sc[j & 1];
    load_v(b);
    float t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = dot8<F16>(kr[i], qv);
    const float mine = sum_16lanes(t);
    const int key = warp * 16 + (li >> 1) * 2 + hl;
    if ((li & 1) == 0) s[key] = b * BT + key < p.nk ? mine : -INFINITY;
    if (j + 1 < last) {
      b = __ldg(list + j + 1);
      load_k(b);
    }
    __syncthreads();  // (the other buffer was read before this barrier's predecessor)
    float w[8];
    ld_chunk<8>(s + li * 8, w);
    float mx = fmaxf(fmaxf(fmaxf(w[0], w[1]), fmaxf(w[2], w[3])), fmaxf(fmaxf(w[4], w[5]), fmaxf(w[6], w[7])));
#pragma unroll
    for (int o = 8; o > 0; o /= 2) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    const float m1 = fmaxf(m, mx);
    const float ref = m1 == -INFINITY ? 0.f : m1;  // nothing but -inf so far weighs nothing
    const float alpha = ex2(m - ref);
    m = m1;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      w[i] = ex2(w[i] - ref);
      sum += w[i];
    }
#pragma unroll
    for (int o = 8; o > 0; o /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    l = l * alpha + sum;
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = fmaf(acc[i], alpha, dot8<F16>(vr[i], w));
  }
  const float o = sum_16lanes(acc);
  const int col = warp * 16 + (li >> 1) * 2 + hl;
  if (C > 1) {
    if ((li & 1) == 0) peer_store1(mapa_shared(smem_u32(&part[rank][col]), 0), o);
    if (threadIdx.x == 0) peer_store2(mapa_shared(smem_u32(&ml[rank]), 0), m, l);
    __syncwarp();
    cluster_sync_all();  // every part has arrived; no access to another CTA follows
    if (rank == 0 && threadIdx.x < BT) {
      float top = -INFINITY, den = 0.f, num = 0.f;
      for (int r = 0; r < C; ++r) top = fmaxf(top, ml[r].x);
      for (int r = 0; r < C; ++r) {
        const float w = ml[r].x == -INFINITY ? 0.f : ex2(ml[r].x - top);
        den += w * ml[r].y;
        num += w * part[r][threadIdx.x];
      }
      p.o[head * BT + threadIdx.x] = __float2bfloat16_rn(length > 0 ? num / den : 0.f);
    }
  } else if ((li & 1) == 0) {
    p.o[head * BT + col] = __float2bfloat16_rn(length > 0 ? o / l : 0.f);
  }
}

static int g_token_clusters[TK_MAX_C + 1];  // clusters of 1 .. TK_MAX_C CTAs that run at once

// CTAs that share a head, by the expected time (us; 12 shapes of 8 to 192 heads and 8 to 200 blocks
// under every split): a CTA takes 1.5 a block, 2.1 where an SM holds two of them, and 2.5 go to the
// start and the merge.  40 heads x 32 blocks: 49.1, 26.9, 19.8, 18.8, 17.3, 15.3, 22.8 and 20.4
// shared by 1 .. 8.
static int token_split(int heads, int keep) {
  int best = 1;
  double least = 1e30;
  for (int c = 1; c <= TK_MAX_C && c <= keep; ++c) {
    const int at_once = std::max(1, g_token_clusters[c]);
    const long waves = ((long)heads + at_once - 1) / at_once;
    const double block = (long)std::min(heads, at_once) * c <= sm_count() ? 1.5 : 2.1;
    const double us = (double)waves * ((keep + c - 1) / c) * block + 2.5;
    if (us < least) {
      least = us;
      best = c;
    }
  }
  return best;
}

static cudaError_t attention_token(const BlockAttnArgs& a, BlockAttnParams p, cudaStream_t s) {
  p.c = token_split(a.heads, a.keep);
  auto launch = [&](auto kernel) {
    return launch_cluster(kernel, p.c > 1 ? (unsigned)p.c : 0u, (unsigned)(a.heads * p.c), TK_TH, 0, s,
                          reinterpret_cast<const uint16_t*>(a.q), reinterpret_cast<const uint16_t*>(a.k), a.ldk,
                          reinterpret_cast<const uint16_t*>(a.v), a.vpad, p);
  };
  return a.f16 ? launch(attn_token_kernel<true>) : launch(attn_token_kernel<false>);
}

cudaError_t attention_blocks_init() {
  const void* kernels[] = {(const void*)attn_blocks_kernel<false, false>, (const void*)attn_blocks_kernel<false, true>,
                           (const void*)attn_blocks_kernel<true, false>, (const void*)attn_blocks_kernel<true, true>};
  cudaError_t r = cudaSuccess;
  for (const void* k : kernels)
    if (r == cudaSuccess) r = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, BT_SMEM);
  for (int c = 1; c <= TK_MAX_C && r == cudaSuccess; ++c) {
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = (unsigned)c;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = (unsigned)(c * 1024);
    cfg.blockDim = TK_TH;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    r = cudaOccupancyMaxActiveClusters(&g_token_clusters[c], attn_token_kernel<true>, &cfg);
  }
  return r;
}

// CTAs that share a unit (0: a CTA takes two units, and *pairs CTAs do; units of the last wave
// follow alone), by the time each way would take (us; 15 shapes of 1 to 32,760 queries and 2 to
// 2560 units, each timed in every way): a wave of CTAs that walk k blocks on each slot takes 1.7 k,
// and 5 more where the slots are units of their own, 9 to 13 with the exchange.  32,760 queries x 4
// heads x 64 of 256 blocks: 449 us in pairs, 452, 541, 748 and 1371 shared by 1, 2, 4 and 8; one
// query x 40 heads x 32 blocks: 59 in pairs, 33, 24, 37 and 49.
static int blocks_split(long units, int keep, long* pairs) {
  const long sms = sm_count();
  auto cd = [](long a, long b) { return (a + b - 1) / b; };
  auto shared = [&](long n, int log) {
    const long reach = log < 2 ? sms : (log == 2 ? sms - sms / 19 : sms - sms / 19 * 4);  // by clusters of 2^log
    return (double)cd(n << log, reach) * (1.7 * (double)cd(keep, 2L << log) + 9.0 + 1.3 * log);
  };
  const double wave = 1.7 * keep + 5.0;
  *pairs = cd(units, 2);
  double best = (double)cd(*pairs, sms) * wave;
  const long full = units / (2 * sms), rest = units - full * 2 * sms;
  if (full > 0 && rest > 0 && shared(rest, 0) < wave) {
    *pairs = full * sms;
    best = (double)full * wave + shared(rest, 0);
  }
  int c = 0;
  for (int log = 0; log <= 3 && (log == 0 || 2 << log <= keep); ++log) {
    if (shared(units, log) < best) {
      best = shared(units, log);
      c = 1 << log;
    }
  }
  if (c == 1) {  // the same kernel as pairs, with none
    c = 0;
    *pairs = 0;
  }
  return c;
}

cudaError_t attention_blocks(const BlockAttnArgs& a, cudaStream_t s) {
  if (a.nq <= 0) return cudaSuccess;
  CUtensorMap tq, tk, tv;
  const uint64_t kw = (uint64_t)a.kv_heads * BT;
  BlockAttnParams p;
  p.nq = a.nq;
  p.nk = a.nk;
  p.nqb = (a.nq + BT - 1) / BT;
  p.nkb = (a.nk + BT - 1) / BT;
  p.keep = a.keep;
  p.group = a.heads / a.kv_heads;
  p.units = (long)a.heads * p.nqb;
  p.blocks = a.blocks;
  p.o = reinterpret_cast<__nv_bfloat16*>(a.o);
  p.ldo = a.ldo;
  p.scale_log2 = (float)(1.4426950408889634 / std::sqrt((double)BT));
  p.c = 1;
  p.pairs = 0;
  p.err = a.err;
  if (a.nq == 1) return attention_token(a, p, s);
  if (encode_tmap_2d_bf16(&tq, a.q, (uint64_t)a.heads * BT, (uint64_t)a.nq, (uint64_t)a.ldq * 2, 64, BT) ||
      encode_tmap_2d_bf16(&tk, a.k, kw, (uint64_t)a.nk, (uint64_t)a.ldk * 2, 64, BT) ||
      encode_tmap_2d_bf16(&tv, a.v, (uint64_t)a.nk, kw, (uint64_t)a.vpad * 2, 64, BT))
    return cudaErrorInvalidValue;
  long pairs;
  const int c = blocks_split(p.units, a.keep, &pairs);
  p.c = std::max(1, c);
  const long ctas = c ? p.units * c : pairs + std::max(0L, p.units - 2 * pairs);
  p.pairs = (int)std::min(pairs, 0x7fffffffL);
  if (ctas > 0x7fffffffL) return cudaErrorInvalidConfiguration;
  auto launch = [&](auto kernel) {
    return launch_cluster(kernel, c > 1 ? (unsigned)c : 0u, (unsigned)ctas, BT_THREADS, BT_SMEM, s, tq, tk, tv, p);
  };
  if (a.f16) return c ? launch(attn_blocks_kernel<true, false>) : launch(attn_blocks_kernel<true, true>);
  return c ? launch(attn_blocks_kernel<false, false>) : launch(attn_blocks_kernel<false, true>);
}

}  // namespace bag
