// C[m, n] = sum over blocks kb of 128 of  2^(ea[m, kb] + eb[n, kb]) * sum_{k in kb} A[m, k] B[n, k],  A and B in e4m3 (vsa2_fp8_quantize), C in bf16 or fp32.
//
// On the tensor cores: tcgen05.mma kind::mxf8f6f4 multiplies by a power-of-two scale for every 32 values of a row itself; the four groups of a block
// of 128 get the same one.  The scales' words (four blocks of a row, the layout of the quantiser) go to tensor memory as they are, and the
// instruction's scale selector picks the block's byte: one copy serves 512 values of K.
//
// B's rows (n, the weights of a projection) are the 128 rows of a tile, A's rows (m, the tokens) its NT columns.  A warp of the epilogue then holds 32
// neighbouring elements of a row of C, whatever C's row length or alignment, and few tokens take a narrow tile (NT = 16 .. 224) under
// weights that stream through at the same rate.
// Persistent CTAs, one per SM: a producer warp (TMA), an issuer, a warp for the scales, four for the epilogue; two accumulators in tensor memory, so that
// a tile's epilogue runs behind the next tile's products.
//
// Whole tiles are dealt out in rounds; what is left of the last rounds (all, where there are fewer tiles than CTAs) is cut along K so that every CTA gets the
// same share: a tile's parts go to the workspace in fp32 and the CTA that delivers the last part adds them in their order (results do not depend on which that is).
#include <cuda.h>

#include "common.cuh"
#include "heads.cuh"
#include "tc05.cuh"
#include "tc_attn.cuh"
#include "tmap.cuh"

namespace vsa2 {

namespace {

constexpr int kMmCtas = 148;            // most CTAs (the workspace is laid out for them)
constexpr int kMmThreads = 384;
constexpr int kMmStagesMost = 12;
constexpr int kMmCounters = 2 * kMmCtas;
constexpr int kMmChunk = 64;            // blocks of K that an accumulator sums for an fp32 result
constexpr uint32_t kMmPBytes = 128 * 128;
constexpr uint32_t kMmTileBytes = 32 * 128 * 2;      // 32 rows of C x 128 elements of bf16

// NT columns an accumulator; PAIR: CTAs that share a tile (2: a pair of SMs, 256 rows of B, each CTA fetches its rows of B and half the rows
// of A); HALVES: accumulators side by side (2: a tile of 2 NT columns takes both)
template <int NT, int PAIR, int HALVES, typename TO>
struct MmTile {
  static constexpr int COLS = NT * HALVES;
  static constexpr uint32_t QBYTES = NT / PAIR * 128;                       // rows of A for one accumulator
  static constexpr uint32_t STAGE = kMmPBytes + HALVES * QBYTES;
  static constexpr int SFQ = (NT + 127) / 128;                              // 512-byte pieces of A's scales for one accumulator
  static constexpr uint32_t SCALES = 512 + HALVES * SFQ * 512;              // words of 128 rows of B, of the rows of A
  static constexpr int SLOTS = HALVES == 2 ? 2 : 4;
  static constexpr uint32_t STAGING = sizeof(TO) == 2 ? 4 * kMmTileBytes : 0;      // two tiles of results for each group of the epilogue
  static constexpr uint32_t ROOM = 227 * 1024 - 2048 - SLOTS * SCALES - STAGING;
  static constexpr int STAGES = ROOM / STAGE < kMmStagesMost ? ROOM / STAGE : kMmStagesMost;
  static constexpr size_t SMEM = 1024 + (size_t)STAGES * STAGE + STAGING + SLOTS * SCALES;
  // HALVES = 2: blocks whose products with one half are issued together at a tile's two ends
  static constexpr int BUNCH = STAGES > 4 ? 3 : 2;
  // columns of tensor memory: accumulators at 0 and 256 (of 224 at most), scales of even and odd groups of four blocks behind them
  __host__ __device__ static constexpr uint32_t scales_at(uint32_t group) { return 224 + (group & 1) * 256; }
};

// P: the operand whose rows are the accumulators' lanes, Q: the one whose rows are its columns
struct MmArgs {
  int p_rows, q_rows, kb;            // kb: blocks of K
  int pt, qt, gq;                    // tiles along P, along Q; tiles along Q that are taken together
  int tensor_stores;                 // C lies as tensor copies need it
  int chunk;                         // most blocks of K in one accumulator
  int whole, rest, splits;           // tiles that are dealt out whole; the others, each cut into `splits` ranges of K
  const uint32_t* p_scales;
  const uint32_t* q_scales;
  void* c;
  long long ldc;
  StatusBlock* status;
  int* counters;
  float* partial;
};

struct MmMisc {
  uint64_t full[kMmStagesMost], empty[kMmStagesMost], sc_full[4], sc_empty[4], d_full[2], d_empty[2], group[2], written[2];
  uint32_t tmem_base;
  int abort_flag;
  int last[2];
};

// The items of a CTA (or pair): every `all`-th, the whole tiles first, then the first ranges of the others, their second ranges, ..: CTAs that run at the
// same time read the same part of K, so that rows they share come from memory once (shares of equal size, begun anywhere: 2304 x 1536, K = 32760
// 192 us).  Each item in pieces of at most `chunk` blocks.
struct MmWalk {
  int tile, kb0, kb1;                // current piece
  int r0, r1, part;                  // the item's blocks; its place among the parts, -1: a whole tile
  int item, all;
  __device__ __forceinline__ void init(int me, int of) {
    item = me;
    all = of;
    kb1 = r1 = 0;
  }
  __device__ __forceinline__ bool advance(const MmArgs& a) {
    if (kb1 < r1) {
      kb0 = kb1;
    } else {
      if (item >= a.whole + a.rest * a.splits) return false;
      part = -1;
      tile = item; r0 = 0; r1 = a.kb;
      if (item >= a.whole && a.splits > 1) {
        part = item - a.whole;
        const int split = part / a.rest;
        tile = a.whole + part - split * a.rest;
        r0 = (int)((long long)a.kb * split / a.splits);
        r1 = (int)((long long)a.kb * (split + 1) / a.splits);
      }
      item += all;
      kb0 = r0;
    }
    kb1 = min(r1, kb0 + a.chunk);
    return true;
  }
};
__device__ __forceinline__ void mm_place(const MmArgs& a, int tile, int& p, int& q) {
  const int per = a.gq * a.pt, g = tile / per, r = tile - g * per, w = min(a.gq, a.qt - g * a.gq);
  p = r / w;
  q = g * a.gq + r - p * w;
}

// ---- a CTA alone, or a pair whose first CTA issues the products and holds the barriers that both sides arrive at
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t leaders(uint64_t* bar) {      // address of the first CTA's barrier
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(tc::smem_u32(bar)));
  return r;
}
__device__ __forceinline__ void arrive_leader(uint64_t* bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(leaders(bar)) : "memory");
}
// tc::mbar_wait on a barrier that the other CTA of a pair arrives at too
template <int PAIR>
__device__ __forceinline__ bool wait_pair(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
  if constexpr (PAIR == 1) {
    return tc::mbar_wait(bar, parity, abort_flag);
  } else {
    const uint32_t t0 = tc::timer_lo_ns();
    for (;;) {
      uint32_t ok;
      asm volatile(
          "{\n\t.reg .pred p;\n\t"
          "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
          "selp.u32 %0, 1, 0, p;\n\t}"
          : "=r"(ok)
          : "r"(tc::smem_u32(bar)), "r"(parity)
          : "memory");
      if (ok != 0) return true;
      if (*abort_flag || tc::timer_lo_ns() - t0 > tc::kWaitLimitNs) {
        *abort_flag = 1;
        return false;
      }
    }
  }
}
#define VSA2_WAIT_PAIR(bar, parity)                                            \
  do {                                                                         \
    if (!wait_pair<PAIR>((bar), (parity), &misc->abort_flag)) goto done;       \
  } while (0)
template <int PAIR>
__device__ __forceinline__ void tma_load_rows(void* dst, const CUtensorMap* m, uint64_t* bar, int c0, int c1) {
  if constexpr (PAIR == 1)
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(tc::smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(m)), "r"(tc::smem_u32(bar)), "r"(c0), "r"(c1)
                 : "memory");
  else
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(tc::smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(m)), "r"(leaders(bar)), "r"(c0), "r"(c1)
                 : "memory");
}
// 32 x 16 bytes of shared memory to four columns of tensor memory, the same in each group of 32 lanes: words (r, j) of row j * 32 + r
// (a pair: each CTA's own)
template <int PAIR>
__device__ __forceinline__ void copy_scales(uint32_t taddr, uint64_t desc) {
  if constexpr (PAIR == 1) asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
  else asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
template <int PAIR>
__device__ __forceinline__ void mma_scaled(uint32_t d, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t sfa, uint32_t sfb, bool accumulate) {
  if constexpr (PAIR == 1)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sfa), "r"(sfb), "r"((uint32_t)accumulate)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sfa), "r"(sfb), "r"((uint32_t)accumulate)
        : "memory");
}
// arrives at the barrier of this CTA, or of both of the pair, once the products and copies issued so far are done
template <int PAIR>
__device__ __forceinline__ void commit_all(uint64_t* bar) {
  if constexpr (PAIR == 1) tc::mma_commit(bar);
  else
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(tc::smem_u32(bar)), "h"((uint16_t)3)
                 : "memory");
}
template <int PAIR>
__device__ __forceinline__ void mm_alloc(uint32_t* to) {
  if constexpr (PAIR == 1) {
    tc::tmem_alloc(to, 512);
    tc::tmem_relinquish();
  } else {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(tc::smem_u32(to)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
}
template <int PAIR>
__device__ __forceinline__ void mm_dealloc(uint32_t base) {
  if constexpr (PAIR == 1) tc::tmem_dealloc(base, 512);
  else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(base) : "memory");
}
// 32 lanes x STEP columns of an accumulator
template <int STEP>
__device__ __forceinline__ void load_columns(uint32_t taddr, float (&v)[STEP]) {
  uint32_t r[STEP];
  tc::tmem_ld32(taddr, r);
  tc::tmem_ld_wait();
#pragma unroll
  for (int c = 0; c < STEP; ++c) v[c] = __uint_as_float(r[c]);
}
// e4m3 x e4m3, ue8m0 scales, both operands K-major, 128 rows a CTA; `sf`: which byte of the scales' words
template <int NT, int PAIR>
__device__ __forceinline__ constexpr uint32_t idesc_scaled(uint32_t sf) {
  return (sf << 4) | ((uint32_t)(NT >> 3) << 17) | (1u << 23) | ((uint32_t)PAIR << 27) | (sf << 29);
}

// 32 columns of an accumulator's row, straight code where all of them exist: with a test for each element the loads and stores came one at a time, and
// the epilogue took longer than the products of 40 blocks.
__device__ __forceinline__ void put(float* to, float v) { *to = v; }
__device__ __forceinline__ void put(bf16* to, float v) { *to = __float2bfloat16_rn(v); }
// elements `stride` apart (a warp's 32 rows lie next to one another in C)
template <typename TO>
__device__ __forceinline__ void put_column(TO* to, long long stride, int count, const float (&v)[32]) {
  if (count >= 32) {
#pragma unroll
    for (int c = 0; c < 32; ++c, to += stride) put(to, v[c]);
  } else {
#pragma unroll
    for (int c = 0; c < 32; ++c, to += stride)
      if (c < count) put(to, v[c]);
  }
}
__device__ __forceinline__ void add_column(const float* from, long long stride, int count, float (&v)[32]) {
  float old[32];
#pragma unroll
  for (int c = 0; c < 32; ++c) {
    old[c] = __ldcg(from);
    if (c + 1 < count) from += stride;
  }
#pragma unroll
  for (int c = 0; c < 32; ++c) v[c] += old[c];
}

// bf16: 32 rows x 32 columns of an accumulator (lanes and columns of `taddr`) as the fragments that stmatrix turns: four 8 x 8 blocks for each 8 columns
__device__ __forceinline__ void take_tile(uint32_t taddr, uint32_t (&u)[16]) {
  uint32_t r[2][16];
  tc::tmem_ld_16x256b_x4(taddr, r[0]);
  tc::tmem_ld_16x256b_x4(taddr + (16u << 16), r[1]);
  tc::tmem_ld_wait();
#pragma unroll
  for (int g = 0; g < 4; ++g)
#pragma unroll
    for (int b = 0; b < 4; ++b)
      u[4 * g + b] = pack_bf16x2(__uint_as_float(r[b >> 1][4 * g + 2 * (b & 1)]), __uint_as_float(r[b >> 1][4 * g + 2 * (b & 1) + 1]));
}
// .. to 32 rows of C of 32 elements, in a tile of 32 rows x 128 elements that lies as the tensor copy takes it: two boxes of 64 elements, rows of 128 bytes, 16-byte places
// exchanged by the row
__device__ __forceinline__ void stage_tile(unsigned char* tile, const uint32_t (&u)[16], int quad, int lane) {
  const int row = lane & 7, block = (quad & 1) * 4 + (lane >> 3);      // of C; of 8 elements in the box
  const uint32_t to = tc::smem_u32(tile) + (quad >> 1) * 4096 + row * 128 + ((block ^ row) << 4);
#pragma unroll
  for (int g = 0; g < 4; ++g)
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};"
                 ::"r"(to + g * 1024), "r"(u[4 * g]), "r"(u[4 * g + 1]), "r"(u[4 * g + 2]), "r"(u[4 * g + 3])
                 : "memory");
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* m, const void* from, int c0, int c1) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];"
               ::"l"(reinterpret_cast<uint64_t>(m)), "r"(tc::smem_u32(from)), "r"(c0), "r"(c1)
               : "memory");
}

template <int NT, int PAIR, int HALVES, typename TO>
__global__ void __cluster_dims__(PAIR, 1, 1) __launch_bounds__(kMmThreads, 1)
fp8_matmul_kernel(const __grid_constant__ CUtensorMap tm_p, const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_c,
                  const __grid_constant__ MmArgs a) {
  using T = MmTile<NT, PAIR, HALVES, TO>;
  extern __shared__ unsigned char mm_smem[];
  __shared__ MmMisc misc_store;
  MmMisc* misc = &misc_store;
  unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(mm_smem) + 1023) & ~(uintptr_t)1023);
  unsigned char* staging = ring + T::STAGES * T::STAGE;
  unsigned char* scales = staging + T::STAGING;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = PAIR == 1 ? 0 : (int)cluster_rank();
  if (tid == 0) {
    misc->abort_flag = 0;
    for (int s = 0; s < T::STAGES; ++s) {
      tc::mbar_init(&misc->full[s], 1);
      tc::mbar_init(&misc->empty[s], 1);
    }
    for (int s = 0; s < T::SLOTS; ++s) {
      tc::mbar_init(&misc->sc_full[s], rank == 0 ? PAIR : 1);
      tc::mbar_init(&misc->sc_empty[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      tc::mbar_init(&misc->d_full[s], 1);
      tc::mbar_init(&misc->d_empty[s], rank == 0 ? 3 + PAIR : 4);
      tc::mbar_init(&misc->group[s], 128);
      tc::mbar_init(&misc->written[s], 128);
    }
    tc::fence_barrier_init();
    tc::prefetch_tmap(&tm_p);
    tc::prefetch_tmap(&tm_q);
  }
  if (warp == 3) mm_alloc<PAIR>(&misc->tmem_base);
  tc::tc_fence_before();
  __syncthreads();
  if constexpr (PAIR == 2) cluster_sync_all();
  tc::tc_fence_after();
  const uint32_t tmem_base = misc->tmem_base;
  grid_enter(false);
  {
    MmWalk w;
    w.init(blockIdx.x / PAIR, gridDim.x / PAIR);
    if (warp == 0) {
      // ---------------------------------------------------------------- operands: a lane for B's rows, one for A's rows of each accumulator
      // (in one warp or two, in copies of 128 rows or of 32: no difference)
      uint32_t s = 0, parity = 1;
      const CUtensorMap* tm = lane == 0 ? &tm_p : &tm_q;
      const uint32_t offset = lane == 0 ? 0 : kMmPBytes + (lane - 1) * T::QBYTES;
      while (w.advance(a)) {
        int p, q;
        mm_place(a, w.tile, p, q);
        const int row = lane == 0 ? (p * PAIR + rank) * 128 : q * T::COLS + (lane - 1) * NT + rank * (NT / PAIR);
        for (int kb = w.kb0; kb < w.kb1; ++kb) {
          VSA2_WAIT(&misc->empty[s], parity);
          if (rank == 0 && lane == 0) tc::mbar_expect_tx(&misc->full[s], PAIR * T::STAGE);
          if (lane <= HALVES) tma_load_rows<PAIR>(ring + s * T::STAGE + offset, tm, &misc->full[s], kb * 128, row);
          __syncwarp();
          if (++s == T::STAGES) {
            s = 0;
            parity ^= 1;
          }
        }
      }
    } else if (warp == 1 && rank == 0) {
      // ---------------------------------------------------------------- products (converged warp, one lane issues)
      const uint64_t ring_desc = tc::smem_desc_sw128(tc::smem_u32(ring), 16, 1024);
      const uint64_t scale_desc = tc::smem_desc_plain(tc::smem_u32(scales), 16, 128);
      uint32_t stage = 0, parity = 0, sc = 0, seg = 0;
      // products of block kb in stage s with half h of the columns, scales of group number `group`
      auto products = [&](int kb, uint32_t s, uint32_t group, uint32_t buf, int h, bool first) {
        const uint64_t dp = ring_desc + (uint64_t)(s * T::STAGE >> 4), dq = dp + (uint64_t)((kMmPBytes + h * T::QBYTES) >> 4);
        const uint32_t idesc = idesc_scaled<NT, PAIR>(kb & 3), tm_sc = tmem_base + T::scales_at(group);
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
          mma_scaled<PAIR>(tmem_base + buf * 256, dp + 2 * ks, dq + 2 * ks, idesc, tm_sc, tm_sc + 4 + h * 4 * T::SFQ, ks > 0 || !first);
      };
      for (; w.advance(a); ++seg) {
        if constexpr (HALVES == 1) VSA2_WAIT_PAIR(&misc->d_empty[seg & 1], ((seg >> 1) & 1) ^ 1);
        else VSA2_WAIT_PAIR(&misc->d_empty[0], (seg & 1) ^ 1);
        // HALVES = 2: both accumulators are in use all the time.  Of the last blocks of a tile those with the first half come first, so that its epilogue
        // runs behind those with the second half; of the first blocks likewise, so that the second half's epilogue runs behind those with the first
        int kb = w.kb0;
        while (kb < w.kb1) {
          const int bunch = HALVES == 1 ? 1 : kb == w.kb0 || kb == w.kb1 - T::BUNCH ? min(T::BUNCH, w.kb1 - kb) : 1;
          uint32_t first_group = sc, s = stage, s_parity = parity;
          for (int i = 0; i < bunch; ++i) {
            const bool fresh = kb + i == w.kb0 || ((kb + i) & 3) == 0;
            if (fresh) {
              VSA2_WAIT_PAIR(&misc->sc_full[sc % T::SLOTS], (sc / T::SLOTS) & 1);
              ++sc;
            }
            if (i == 0) first_group = sc - 1;
            VSA2_WAIT(&misc->full[s], s_parity);
            tc::tc_fence_after();
            if (tc::elect_one()) {
              if (fresh) {
                const uint32_t slot = (sc - 1) % T::SLOTS, tm_sc = tmem_base + T::scales_at(sc - 1);
                const uint64_t d = scale_desc + (uint64_t)(slot * T::SCALES >> 4);
#pragma unroll
                for (int j = 0; j < 1 + HALVES * T::SFQ; ++j) copy_scales<PAIR>(tm_sc + 4 * j, d + (uint64_t)(512 * j >> 4));
                commit_all<PAIR>(&misc->sc_empty[slot]);
              }
              products(kb + i, s, sc - 1, HALVES == 1 ? seg & 1 : 0, 0, kb + i == w.kb0);
              if (HALVES == 1) commit_all<PAIR>(&misc->empty[s]);
              if (kb + i == w.kb1 - 1) commit_all<PAIR>(&misc->d_full[HALVES == 1 ? seg & 1 : 0]);
            }
            __syncwarp();
            if (++s == T::STAGES) {
              s = 0;
              s_parity ^= 1;
            }
          }
          if constexpr (HALVES == 2) {
            if (kb == w.kb0) {
              VSA2_WAIT_PAIR(&misc->d_empty[1], (seg & 1) ^ 1);
              tc::tc_fence_after();
            }
            uint32_t group = first_group;
            for (int i = 0; i < bunch; ++i) {
              if (i > 0 && ((kb + i) & 3) == 0) ++group;
              if (tc::elect_one()) {
                products(kb + i, stage, group, 1, 1, kb + i == w.kb0);
                commit_all<PAIR>(&misc->empty[stage]);
                if (kb + i == w.kb1 - 1) commit_all<PAIR>(&misc->d_full[1]);
              }
              __syncwarp();
              if (++stage == T::STAGES) stage = 0;
            }
          }
          stage = s;
          parity = s_parity;
          kb += bunch;
        }
      }
    } else if ((warp == 1 || warp == 3) && rank == 1) {
      // ---------------------------------------------------------------- tells the first CTA what this one has ready: scales (warp 1), accumulators that have
      // been read (warp 3).  An arrival at the other CTA waits for all that its warp has under way: by the scales' own warp (loads) or the epilogue's (stores)
      // it came a memory latency late, 1500 cycles for each four blocks
      uint32_t sc = 0;
      for (uint32_t seg = 0; w.advance(a); ++seg) {
        if (warp == 1) {
          for (int g = w.kb0 >> 2; g <= (w.kb1 - 1) >> 2; ++g, ++sc) {
            VSA2_WAIT(&misc->sc_full[sc % T::SLOTS], (sc / T::SLOTS) & 1);
            if (lane == 0) arrive_leader(&misc->sc_full[sc % T::SLOTS]);
            __syncwarp();
          }
        } else {
#pragma unroll
          for (int h = 0; h < HALVES; ++h) {
            const uint32_t buf = HALVES == 2 ? h : seg & 1;
            VSA2_WAIT(&misc->d_empty[buf], (HALVES == 2 ? seg : seg >> 1) & 1);
            if (lane == 0) arrive_leader(&misc->d_empty[buf]);
            __syncwarp();
          }
        }
      }
    } else if (warp == 2) {
      // ---------------------------------------------------------------- scales: words of rows lane, lane + 32, .. as 16 bytes a lane
      // AHEAD groups of four blocks are on their way from memory at a time: with one, a group's latency bound short rows (one row of A against 15,360 x
      // 5,120: 26 us)
      constexpr int NV = 4 + 4 * HALVES * T::SFQ, AHEAD = NV <= 8 ? 6 : NV <= 12 ? 4 : 2;
      uint32_t v[AHEAD][NV];
      bool there[AHEAD];
      int g = 0, g_end = 0, row_p = 0, row_q = 0;
      auto next = [&](uint32_t (&to)[NV]) {
        if (g >= g_end) {
          if (!w.advance(a)) return false;
          int p, q;
          mm_place(a, w.tile, p, q);
          row_p = (p * PAIR + rank) * 128 + lane;
          row_q = q * T::COLS + lane;
          g = w.kb0 >> 2;
          g_end = ((w.kb1 - 1) >> 2) + 1;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) to[j] = row_p + j * 32 < a.p_rows ? a.p_scales[(size_t)g * a.p_rows + row_p + j * 32] : 0u;
#pragma unroll
        for (int j = 0; j < NV - 4; ++j) {
          const int h = j / (4 * T::SFQ), i = (j - h * 4 * T::SFQ) * 32, r = row_q + h * NT + i;
          to[4 + j] = i < NT && r < a.q_rows ? a.q_scales[(size_t)g * a.q_rows + r] : 0u;
        }
        ++g;
        return true;
      };
#pragma unroll
      for (int d = 0; d < AHEAD; ++d) there[d] = (d == 0 || there[d > 0 ? d - 1 : 0]) && next(v[d]);
      for (uint32_t sc = 0; there[0];) {
#pragma unroll
        for (int d = 0; d < AHEAD; ++d) {
          if (!there[d]) continue;      // (then none of those behind it is there either)
          const uint32_t slot = sc % T::SLOTS;
          VSA2_WAIT_PARKED(&misc->sc_empty[slot], ((sc / T::SLOTS) & 1) ^ 1);
          unsigned char* to = scales + slot * T::SCALES + lane * 16;
#pragma unroll
          for (int j = 0; j < NV / 4; ++j)
            *reinterpret_cast<uint4*>(to + j * 512) = make_uint4(v[d][4 * j], v[d][4 * j + 1], v[d][4 * j + 2], v[d][4 * j + 3]);
          tc::fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(&misc->sc_full[slot]);
          ++sc;
          there[d] = next(v[d]);
        }
      }
    } else if (warp >= 4) {
      // ---------------------------------------------------------------- epilogue: four warps for each accumulator
      const int quad = warp & 3, buf = (warp >> 2) - 1;
      uint32_t syncs = 0, turn = 0, tiles = 0;
      for (uint32_t seg = 0; w.advance(a); ++seg) {
        if (HALVES == 1 && (int)(seg & 1) != buf) continue;
        int p, q;
        mm_place(a, w.tile, p, q);
        const int row = (p * PAIR + rank) * 128 + quad * 32 + lane, col = q * T::COLS + (HALVES == 2 ? buf * NT : 0);
        const int cols = min(NT, a.q_rows - col);      // (0 or less: the second half of a tile that ends in the first)
        const bool in = row < a.p_rows;
        VSA2_WAIT_PARKED(&misc->d_full[buf], turn & 1);
        ++turn;
        tc::tc_fence_after();
        const bool adds = w.kb0 > w.r0;
        // Pieces of one item come to the two groups of warps in turn (HALVES = 1), each adding to what the other has written: one after the other
        const bool in_turn = HALVES == 1 && a.chunk < a.kb;
        if (in_turn && seg > 0) VSA2_WAIT_PARKED(&misc->written[buf ^ 1], ((seg - 1) >> 1) & 1);
        constexpr int WIDE = HALVES == 2 ? 2 : 1;
        // [part][half][rank][column][row]
        const size_t of_part = (size_t)WIDE * PAIR * 128 * NT;
        float* const parts = a.partial + (size_t)((HALVES == 2 ? buf : 0) * PAIR + rank) * (128 * NT) + quad * 32 + lane;
        TO* const out = reinterpret_cast<TO*>(a.c) + (long long)col * a.ldc + row;      // (this thread's elements of C lie ldc apart)
        const uint32_t tmem = tmem_base + buf * 256 + ((uint32_t)(quad * 32) << 16);
        auto release = [&] {
          tc::tc_fence_before();
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(&misc->d_empty[buf]);
        };
        if (sizeof(TO) == 2 && w.part < 0 && a.tensor_stores) {
          // bf16: all columns to registers first (the CTAs' stores come at the same time and take 5000 cycles; with both accumulators in one tile the products would
          // wait for them), then turned in shared memory, 32 rows of C at a time, and stored by tensor copies that drop what lies outside C.  (Stored by the
          // warps as they hold it, 64 bytes at a time, an accumulator took 13,000 cycles; with the operands' parts exchanged, sectors of 32 rows at a time, 4000.)
          uint32_t u[NT / 32][16];
#pragma unroll
          for (int i = 0; i < NT / 32; ++i) take_tile(tmem + 32 * i, u[i]);
          release();
#pragma unroll
          for (int i = 0; i < NT / 32; ++i) {
            if (32 * i >= cols) break;
            unsigned char* tile = staging + (buf * 2 + (tiles & 1)) * kMmTileBytes;
            stage_tile(tile, u[i], quad, lane);
            tc::fence_proxy_async_smem();
            if (quad == 0 && lane == 0) tc::bulk_store_wait_read();      // the tile before has been read: behind the barrier its place is free
            VSA2_GROUP_SYNC(&misc->group[buf], syncs);
            if (quad == 0 && lane == 0) {
              const int first = (p * PAIR + rank) * 128;
#pragma unroll
              for (int b = 0; b < 2; ++b)
                if (first + 64 * b < a.p_rows) tma_store_2d(&tm_c, tile + b * 4096, first + 64 * b, col + 32 * i);
              tc::bulk_store_commit();
            }
            ++tiles;
          }
        } else {
#pragma unroll 1
          for (int c0 = 0; c0 < cols; c0 += 32) {
            float v[32];
            load_columns<32>(tmem + c0, v);
            if (w.part >= 0) {
              float* to = parts + w.part * of_part + (size_t)c0 * 128;
              if (adds) add_column(to, 128, 32, v);
              put_column(to, 128, 32, v);
            } else if (in) {
              TO* to = out + (long long)c0 * a.ldc;
              if constexpr (sizeof(TO) == 4)      // (fp32 results: what has been written there for the blocks before)
                if (adds) add_column(to, a.ldc, cols - c0, v);
              put_column(to, a.ldc, cols - c0, v);
            }
          }
          release();
        }
        if (in_turn) {
          __threadfence();
          tc::mbar_arrive(&misc->written[buf]);
        }
        if (w.part >= 0 && w.kb1 == w.r1) {
          __threadfence();
          VSA2_GROUP_SYNC(&misc->group[buf], syncs);
          if (quad == 0 && lane == 0) {
            int* counter = a.counters + ((w.tile - a.whole) * WIDE + (HALVES == 2 ? buf : 0)) * PAIR + rank;
            const bool last = atomicAdd(counter, 1) == a.splits - 1;
            if (last) *counter = 0;
            misc->last[buf] = last;
            __threadfence();
          }
          VSA2_GROUP_SYNC(&misc->group[buf], syncs);
          if (misc->last[buf]) {
            __threadfence();
            const float* const mine = parts + (size_t)(w.tile - a.whole) * of_part;
#pragma unroll 1
            for (int c0 = 0; c0 < cols; c0 += 32) {
              float sum[32];
#pragma unroll
              for (int c = 0; c < 32; ++c) sum[c] = 0.f;
#pragma unroll 1
              for (int o = 0; o < a.splits; ++o) add_column(mine + (size_t)o * a.rest * of_part + (size_t)c0 * 128, 128, 32, sum);
              if (in) put_column(out + (long long)c0 * a.ldc, a.ldc, cols - c0, sum);
            }
          }
          VSA2_GROUP_SYNC(&misc->group[buf], syncs);       // (misc->last is read before it is written again)
        }
      }
      if (sizeof(TO) == 2 && quad == 0 && lane == 0) tc::bulk_store_wait();
    }
  }

done:
  tc::tc_fence_before();
  __syncthreads();
  if (misc->abort_flag) {
    if (tid == 0) atomicExch(&a.status->status, VSA2_ERR_DEVICE_TIMEOUT);
    if (tid == 0) {
      // copies and products in flight end within this time; the tensor memory is given back behind them
      const unsigned long long t0 = tc::global_timer_ns();
      while (tc::global_timer_ns() - t0 < 200000ull) {
      }
    }
    __syncthreads();
  }
  if constexpr (PAIR == 2) cluster_sync_all();        // (neither leaves while the other may still arrive at its barriers or read its operands)
  if (warp == 3) mm_dealloc<PAIR>(tmem_base);
}

bool make_row_tmap(CUtensorMap* out, const void* base, int rows, int cols, long long ld, int box_rows) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (fn == nullptr) return false;
  cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)ld};
  cuuint32_t box[2] = {128, (cuuint32_t)box_rows};
  cuuint32_t estr[2] = {1, 1};
  return fn(out, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// C as boxes of 32 rows x 64 elements of bf16
bool make_result_tmap(CUtensorMap* out, void* base, int rows, int cols, long long ld) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (fn == nullptr) return false;
  cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)ld * 2};
  cuuint32_t box[2] = {64, 32};
  cuuint32_t estr[2] = {1, 1};
  return fn(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// How a product is cut: tiles, and ranges of K for those that do not fill a round of all CTAs (or pairs).  `cycles`: estimate that the choice is made by.
struct MmPlan {
  int pt, qt, whole, rest, splits;
  double cycles;
};
struct MmShape {
  int rows, cols, stage, of, sms_each, halves;
  double epilogue;
};
// A block takes the tensor cores 2 cycles a column (128 rows of an SM); the SMs are fed 52 bytes a cycle when all of them are, up to 64 when few are.  An epilogue
// hides behind the next tile's products; with both accumulators in one tile behind 1300 cycles of them.  Cutting what is left of the last rounds into
// ranges of K takes the parts through memory.
MmPlan mm_plan(int p_rows, int q_rows, int kb, const MmShape& t) {
  MmPlan best = {};
  best.pt = (p_rows + t.rows - 1) / t.rows;
  best.qt = (q_rows + t.cols - 1) / t.cols;
  const long long tiles = (long long)best.pt * best.qt;
  const double epilogue = t.epilogue;
  auto item = [&](long long active, int blocks, double last) {
    const double feed = 52.0 * 148 / ((active < t.of ? active : t.of) * t.sms_each);
    const double fed = t.stage / (feed < 64.0 ? feed : 64.0), mma = 2.0 * t.cols, products = blocks * (fed > mma ? fed : mma);
    return t.halves == 2 ? products + (last > 1300 ? last - 1300 : 0) : products > last ? products : last;
  };
  best.whole = (int)(tiles / t.of * t.of);
  best.rest = (int)(tiles - best.whole);
  best.splits = 1;
  const double rounds = (double)(tiles / t.of) * item(t.of, kb, epilogue);
  best.cycles = rounds + (best.rest > 0 ? item(best.rest, kb, epilogue) : 0) + epilogue;
  for (int s = 2; s <= 8 && s <= kb && best.rest > 0 && s * best.rest <= 2 * t.of / t.halves; ++s) {
    const long long items = (long long)s * best.rest;
    const double parts = 3000 + t.cols * (6.0 + 4.0 * s);
    const double cut = (double)((items + t.of - 1) / t.of) * item(items, (kb + s - 1) / s, 1500) + parts + epilogue;
    if (rounds + cut < best.cycles) {
      best.cycles = rounds + cut;
      best.splits = s;
    }
  }
  return best;
}

struct MmCall {
  int m, n, k, ctas;
  Fp8Arg fa, fb;
  cudaStream_t st;
  MmArgs a;
};
template <int NT, int PAIR, int HALVES, typename TO>
MmPlan plan_mm(const MmCall& c) {
  using T = MmTile<NT, PAIR, HALVES, TO>;
  const double epilogue = (sizeof(TO) == 2 && c.a.tensor_stores ? HALVES == 2 ? 3.0 : 25.0 : 55.0) * NT;      // until an accumulator can be used again
  return mm_plan(c.n, c.m, c.a.kb, MmShape{128 * PAIR, T::COLS, (int)T::STAGE, c.ctas / PAIR, PAIR, HALVES, epilogue});
}
template <int NT, int PAIR, int HALVES, typename TO>
cudaError_t launch_mm_of(const MmCall& c, const MmPlan& plan) {
  using T = MmTile<NT, PAIR, HALVES, TO>;
  MmArgs a = c.a;
  const Fp8Arg &p = c.fb, &q = c.fa;
  a.p_rows = c.n;
  a.q_rows = c.m;
  a.p_scales = reinterpret_cast<const uint32_t*>(p.scales);
  a.q_scales = reinterpret_cast<const uint32_t*>(q.scales);
  CUtensorMap tp, tq;
  if (!make_row_tmap(&tp, p.values, a.p_rows, c.k, p.ld, 128) || !make_row_tmap(&tq, q.values, a.q_rows, c.k, q.ld, NT / PAIR))
    return cudaErrorInvalidValue;
  CUtensorMap tm_c = tq;      // (no map of C: never used)
  if (sizeof(TO) == 2 && a.tensor_stores && !make_result_tmap(&tm_c, a.c, c.m, c.n, a.ldc)) return cudaErrorInvalidValue;
  a.pt = plan.pt; a.qt = plan.qt; a.whole = plan.whole; a.rest = plan.rest; a.splits = plan.splits;
  // tiles along Q that share P's rows while they pass through L2
  a.gq = a.qt < 12 / HALVES ? a.qt : 12 / HALVES;
  const long long items = a.whole + (long long)a.rest * a.splits;
  int of = c.ctas / PAIR;
  if (items < of) of = (int)items;
  static KernelAttr attr;
  cudaError_t e;
  if ((e = prepare_kernel((const void*)fp8_matmul_kernel<NT, PAIR, HALVES, TO>, attr, T::SMEM))) return e;
  return launch_kernel(fp8_matmul_kernel<NT, PAIR, HALVES, TO>, of * PAIR, kMmThreads, T::SMEM, c.st, tp, tq, tm_c, a);
}
template <int NT, int PAIR, int HALVES, typename TO>
cudaError_t launch_mm(const MmCall& c) { return launch_mm_of<NT, PAIR, HALVES, TO>(c, plan_mm<NT, PAIR, HALVES, TO>(c)); }

// B's rows are the accumulators' lanes, A's their columns: few rows of A take the narrowest tile that holds them, many by the estimate tiles of 256 x 224 or
// 256 x 448.
template <typename TO>
cudaError_t launch_product(const MmCall& c, bool pair) {
  if (c.m <= 32) return launch_mm<32, 1, 1, TO>(c);
  if (!pair) return launch_mm<128, 1, 1, TO>(c);
  if (c.m <= 128) return launch_mm<128, 2, 1, TO>(c);
  const MmPlan one = plan_mm<224, 2, 1, TO>(c), two = plan_mm<224, 2, 2, TO>(c);
  return one.cycles <= two.cycles ? launch_mm_of<224, 2, 1, TO>(c, one) : launch_mm_of<224, 2, 2, TO>(c, two);
}

}  // namespace

// [status][counters of the tiles that are cut][two parts a CTA]
size_t fp8_matmul_workspace_bytes(int m, int n, int k) {
  (void)n;
  (void)k;
  const int columns = m <= 32 ? 32 : m <= 128 ? 128 : 224;      // (the widest accumulator that a product of m rows may take)
  return align_up(sizeof(StatusBlock) + kMmCounters * sizeof(int), 256) + (size_t)2 * kMmCtas * 128 * columns * sizeof(float);
}

cudaError_t launch_fp8_matmul(int m, int n, int k, const Fp8Arg& fa, const Fp8Arg& fb, void* c, int c_f32, long long ldc,
                              void* workspace, cudaStream_t st) {
  int sms = 0;
  cudaError_t e;
  if ((e = sm_count(&sms)) != cudaSuccess) return e;
  const int ctas = sms < kMmCtas ? sms : kMmCtas;
  // Pairs wherever B has rows for both (a pair fetches half a tile's columns for each SM) and the context has room for one
  bool pair = n > 128 && ctas >= 2;
  if (pair) {
    static ClusterRoom room;
    if ((e = cluster_room((const void*)fp8_matmul_kernel<224, 2, 2, float>, room, 2, kMmThreads, MmTile<224, 2, 2, float>::SMEM, &pair))) return e;
  }
  MmCall call;
  call.m = m; call.n = n; call.k = k; call.ctas = ctas;
  call.fa = fa; call.fb = fb;
  call.st = st;
  MmArgs& a = call.a;
  a = MmArgs{};
  a.kb = (k + 127) / 128;
  a.chunk = c_f32 ? kMmChunk : a.kb;
  a.c = c; a.ldc = ldc;
  a.tensor_stores = !c_f32 && (reinterpret_cast<uintptr_t>(c) & 15u) == 0 && ldc % 8 == 0;
  unsigned char* ws = reinterpret_cast<unsigned char*>(workspace);
  a.status = reinterpret_cast<StatusBlock*>(ws);
  a.counters = reinterpret_cast<int*>(ws + sizeof(StatusBlock));
  a.partial = reinterpret_cast<float*>(ws + align_up(sizeof(StatusBlock) + kMmCounters * sizeof(int), 256));
  return c_f32 ? launch_product<float>(call, pair) : launch_product<bf16>(call, pair);
}

}  // namespace vsa2
