// C[m, n] = sum over blocks kb of 128 of  2^(ea[m, kb] + eb[n, kb]) * sum_{k in kb} A[m, k] B[n, k],  A and B in e4m3 (vsa2_fp8_quantize), C in bf16 or fp32.
//
// On the tensor cores: tcgen05.mma kind::mxf8f6f4 multiplies by a power-of-two scale for every 32 values of a row itself; the four groups of a block
// of 128 get the same one.  The scales' words (four blocks of a row, the layout of the quantiser) go to tensor memory as they are, and the
// instruction's scale selector picks the block's byte: one copy serves 512 values of K.
//
// B's rows (n, the weights of a projection) are the 128 rows of a CTA's tile, A's rows (m, the tokens) its NT columns: few tokens take a narrow tile under weights that
// stream through.  Many take 224 columns on a pair of SMs (cta_group::2): 256 rows of B, each CTA fetches its half of B's rows and half of A's, 30 KB
// for 2 x 128 x 224 x 128 multiply-adds, where a CTA alone fetches 45.  Persistent CTAs, one per SM: a producer warp (TMA), an issuer, a warp for the scales, two
// groups of four, half the columns each, for the epilogue; two accumulators in tensor memory, so that a tile's epilogue runs behind the next tile's products.
//
// What bounds it: in long runs the power limit, at which values of normal numbers draw a quarter more than small whole ones (75600 x 15360 x 5120: 4.5 - 5.0 ms from box to box,
// 2.4 - 2.6 PFLOP/s, against 3.7 ms and 3.2 PFLOP/s, twice the library's bf16 product); else the intake from L2 (8192 x 4096 x 4096 90 us: 51 bytes a cycle and SM, 600
// cycles a block where the tensor cores need 448).  Tiles of 448 columns, both accumulators in one tile, need 27 % less intake and were as fast at large sizes (20000 x 15360 x
// 5120 1028 us both ways), slower where rounds are few (4096^3 60 us instead of 52).  One row of A: the weights' bytes (15360 x 5120 16 us, 4.9 TB/s with the
// launch); few tiles and short K: the launch, the first block's way from memory and the epilogue, 3 - 5 us.
#include <cuda.h>

#include "common.cuh"
#include "heads.cuh"
#include "tc05.cuh"
#include "tc_attn.cuh"
#include "tmap.cuh"

namespace vsa2 {

namespace {

constexpr int kMmCtas = 148;            // most CTAs
constexpr int kMmThreads = 384;
constexpr int kMmStagesMost = 12;
constexpr int kMmScaleSlots = 4;
constexpr int kMmSplits = 16;           // most ranges that K is cut into
// Blocks of K that an accumulator sums for an fp32 result; the epilogue adds the pieces.  (The tensor cores cut what does not fit an accumulator instead of rounding
// it: with 24,000 values of K in one the result was 1.7e-6 off.  2304 x 1536 x 32760, where fp32 torch is 3.0e-7 off: pieces of 16 blocks 1.3e-7 and 109.2 us, of 32 2.2e-7 and
// 108.5, of 40 2.7e-7 and 108.3, of 64 4.8e-7.)
constexpr int kMmChunk = 40;
constexpr uint32_t kMmPBytes = 128 * 128;
constexpr uint32_t kMmTileBytes = 32 * 128 * 2;      // 32 rows of C x 128 elements of bf16

// NT columns; PAIR: CTAs that share a tile; TO: type of the results
template <int NT, int PAIR, typename TO>
struct MmTile {
  static constexpr uint32_t STAGE = kMmPBytes + NT / PAIR * 128;
  static constexpr int SFQ = (NT + 127) / 128;                              // 512-byte pieces of the scales of the columns' rows
  static constexpr uint32_t SCALES = 512 + SFQ * 512;
  static constexpr uint32_t STAGING = sizeof(TO) == 2 ? (NT > 32 ? 4 : 2) * kMmTileBytes : 0;      // two tiles of results for each group of the epilogue
  static constexpr uint32_t ROOM = 227 * 1024 - 2048 - kMmScaleSlots * SCALES - STAGING;
  static constexpr int STAGES = ROOM / STAGE < kMmStagesMost ? ROOM / STAGE : kMmStagesMost;
  static constexpr size_t SMEM = 1024 + (size_t)STAGES * STAGE + STAGING + kMmScaleSlots * SCALES;
  // columns of tensor memory: accumulators at 0 and 256 (of 224 at most), scales of even and odd groups of four blocks behind them
  __host__ __device__ static constexpr uint32_t scales_at(uint32_t group) { return 224 + (group & 1) * 256; }
};

// P: the operand whose rows are the accumulators' lanes, Q: the one whose rows are its columns
struct MmArgs {
  int p_rows, q_rows, kb;            // kb: blocks of K
  int pt, qt, gq;                    // tiles along P, along Q; tiles along Q that are taken together
  int splits, chunk;                 // ranges that K is cut into; most blocks of K in one accumulator
  Divisor by_tiles, by_group, by_gq, by_rest, by_splits;      // pt qt; gq pt; gq, and what the last group has of tiles along Q
  int tensor_stores;                 // C lies as tensor copies need it, and ends where they end
  int in_pieces;                     // some range has more blocks than one accumulator sums
  const uint32_t* p_scales;
  const uint32_t* q_scales;
  void* c;
  long long ldc, split_stride;       // elements between the results of two ranges
  StatusBlock* status;
};

struct MmMisc {
  uint64_t full[kMmStagesMost], empty[kMmStagesMost], sc_full[kMmScaleSlots], sc_empty[kMmScaleSlots];
  uint64_t d_full[2], d_empty[2], group[2];
  uint32_t tmem_base;
  int abort_flag;
};

// The items of a CTA (or pair): every `all`-th of the tiles with the first range of K, then with the second, ..: CTAs that run at the same time read the same part
// of K, so that rows they share come from memory once.  Each item in pieces of at most `chunk` blocks.
struct MmWalk {
  int p, q, split;                   // tile, range
  int kb0, kb1, r0, r1;              // blocks of the current piece, of the item
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
      const int tiles = a.pt * a.qt;
      if (item >= tiles * a.splits) return false;
      split = divided(item, a.by_tiles);
      const int tile = item - split * tiles, g = divided(tile, a.by_group), r = tile - g * a.gq * a.pt, w = min(a.gq, a.qt - g * a.gq);
      p = w == a.gq ? divided(r, a.by_gq) : divided(r, a.by_rest);
      q = g * a.gq + r - p * w;
      r0 = divided(a.kb * split, a.by_splits);      // (at most 2^23 blocks and 16 ranges)
      r1 = divided(a.kb * (split + 1), a.by_splits);
      item += all;
      kb0 = r0;
    }
    kb1 = min(r1, kb0 + a.chunk);
    return true;
  }
};

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
// 32 lanes x 32 columns, or 16, of an accumulator
template <int N>
__device__ __forceinline__ void load_columns(uint32_t taddr, float (&v)[N]) {
  uint32_t r[N];
  if constexpr (N == 32) tc::tmem_ld32(taddr, r);
  else tc::tmem_ld16(taddr, r);
  tc::tmem_ld_wait();
#pragma unroll
  for (int c = 0; c < N; ++c) v[c] = __uint_as_float(r[c]);
}
// e4m3 x e4m3, ue8m0 scales, both operands K-major, 128 rows a CTA; `sf`: which byte of the scales' words
template <int NT, int PAIR>
__device__ __forceinline__ constexpr uint32_t idesc_scaled(uint32_t sf) {
  return (sf << 4) | ((uint32_t)(NT >> 3) << 17) | (1u << 23) | ((uint32_t)PAIR << 27) | (sf << 29);
}

// Columns of an accumulator's row, straight code where all of them exist: with a test for each element the loads and stores came one at a time, and
// the epilogue took longer than the products of 40 blocks.
__device__ __forceinline__ void put(float* to, float v) { *to = v; }
__device__ __forceinline__ void put(bf16* to, float v) { *to = __float2bfloat16_rn(v); }
// elements `stride` apart (a warp's 32 rows lie next to one another in C)
// (in the pieces' epilogue eight addresses at a time: all of them at once are more registers than there are)
template <typename TO, int N>
__device__ __forceinline__ void put_columns(TO* to, long long stride, int count, const float (&v)[N]) {
  constexpr int AT = N < 32 ? 8 : N;
#pragma unroll
  for (int c0 = 0; c0 < N; c0 += AT) {
    if (AT < N) asm volatile("" : "+l"(to));
    if (count >= N) {
#pragma unroll
      for (int c = 0; c < AT; ++c, to += stride) put(to, v[c0 + c]);
    } else {
#pragma unroll
      for (int c = 0; c < AT; ++c, to += stride)
        if (c0 + c < count) put(to, v[c0 + c]);
    }
  }
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
// .. to rows of C in a tile that lies as the tensor copy takes it, 16-byte places exchanged by the row.  SWAP: 32 rows of C of this warp's, 64 bytes each, in
// one box of 128 rows.  Else turned, 32 rows of C of 32 elements, in two boxes of 32 rows x 64 elements (128 bytes)
template <bool SWAP>
__device__ __forceinline__ void stage_tile(unsigned char* tile, const uint32_t (&u)[16], int quad, int lane) {
  if constexpr (SWAP) {
    const int row = quad * 32 + (lane >> 3) * 8 + (lane & 7);
    const uint32_t to = tc::smem_u32(tile) + row * 64;
#pragma unroll
    for (int g = 0; g < 4; ++g)
      asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1, %2, %3, %4};"
                   ::"r"(to + ((g ^ ((row >> 1) & 3)) << 4)), "r"(u[4 * g]), "r"(u[4 * g + 1]), "r"(u[4 * g + 2]), "r"(u[4 * g + 3])
                   : "memory");
    return;
  }
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

template <int NT, int PAIR, bool SWAP, typename TO>
__global__ void __cluster_dims__(PAIR, 1, 1) __launch_bounds__(kMmThreads, 1)
fp8_matmul_kernel(const __grid_constant__ CUtensorMap tm_p, const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_c,
                  const __grid_constant__ MmArgs a) {
  using T = MmTile<NT, PAIR, TO>;
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
    for (int s = 0; s < kMmScaleSlots; ++s) {
      tc::mbar_init(&misc->sc_full[s], rank == 0 ? PAIR : 1);
      tc::mbar_init(&misc->sc_empty[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      tc::mbar_init(&misc->d_full[s], 1);
      tc::mbar_init(&misc->d_empty[s], (NT > 32 ? 8 : 4) + (rank == 0 ? PAIR - 1 : 0));
      tc::mbar_init(&misc->group[s], 128);
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
  grid_enter(a.splits > 1);      // (the kernel that adds the ranges finds room beside this one)
  {
    MmWalk w;
    w.init(blockIdx.x / PAIR, gridDim.x / PAIR);
    if (warp == 0) {
      // ---------------------------------------------------------------- operands: a lane for P's rows, one for Q's
      // (in one warp or two, in copies of 128 rows or of 32: no difference)
      uint32_t s = 0, parity = 1;
      const CUtensorMap* tm = lane == 0 ? &tm_p : &tm_q;
      const uint32_t offset = lane == 0 ? 0 : kMmPBytes;
      while (w.advance(a)) {
        const int row = lane == 0 ? (w.p * PAIR + rank) * 128 : w.q * NT + rank * (NT / PAIR);
        for (int kb = w.kb0; kb < w.kb1; ++kb) {
          VSA2_WAIT(&misc->empty[s], parity);
          if (rank == 0 && lane == 0) tc::mbar_expect_tx(&misc->full[s], PAIR * T::STAGE);
          if (lane < 2) tma_load_rows<PAIR>(ring + s * T::STAGE + offset, tm, &misc->full[s], kb * 128, row);
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
      uint32_t s = 0, parity = 0, sc = 0, seg = 0;
      for (; w.advance(a); ++seg) {
        const uint32_t buf = seg & 1;
        VSA2_WAIT_PAIR(&misc->d_empty[buf], ((seg >> 1) & 1) ^ 1);
        for (int kb = w.kb0; kb < w.kb1; ++kb) {
          const bool fresh = kb == w.kb0 || (kb & 3) == 0;
          if (fresh) {
            VSA2_WAIT_PAIR(&misc->sc_full[sc % kMmScaleSlots], (sc / kMmScaleSlots) & 1);
            ++sc;
          }
          VSA2_WAIT(&misc->full[s], parity);
          tc::tc_fence_after();
          if (tc::elect_one()) {
            const uint32_t slot = (sc - 1) % kMmScaleSlots, tm_sc = tmem_base + T::scales_at(sc - 1);
            if (fresh) {
              const uint64_t d = scale_desc + (uint64_t)(slot * T::SCALES >> 4);
#pragma unroll
              for (int j = 0; j < 1 + T::SFQ; ++j) copy_scales<PAIR>(tm_sc + 4 * j, d + (uint64_t)(512 * j >> 4));
              commit_all<PAIR>(&misc->sc_empty[slot]);
            }
            const uint64_t dp = ring_desc + (uint64_t)(s * T::STAGE >> 4), dq = dp + (uint64_t)(kMmPBytes >> 4);
            const uint32_t idesc = idesc_scaled<NT, PAIR>(kb & 3);
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
              mma_scaled<PAIR>(tmem_base + buf * 256, dp + 2 * ks, dq + 2 * ks, idesc, tm_sc, tm_sc + 4, ks > 0 || kb > w.kb0);
            commit_all<PAIR>(&misc->empty[s]);
            if (kb == w.kb1 - 1) commit_all<PAIR>(&misc->d_full[buf]);
          }
          __syncwarp();
          if (++s == T::STAGES) {
            s = 0;
            parity ^= 1;
          }
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
            VSA2_WAIT(&misc->sc_full[sc % kMmScaleSlots], (sc / kMmScaleSlots) & 1);
            if (lane == 0) arrive_leader(&misc->sc_full[sc % kMmScaleSlots]);
            __syncwarp();
          }
        } else {
          VSA2_WAIT(&misc->d_empty[seg & 1], (seg >> 1) & 1);
          if (lane == 0) arrive_leader(&misc->d_empty[seg & 1]);
          __syncwarp();
        }
      }
    } else if (warp == 2) {
      // ---------------------------------------------------------------- scales: words of rows lane, lane + 32, .. as 16 bytes a lane
      // AHEAD groups of four blocks are on their way from memory at a time
      constexpr int NV = 4 + 4 * T::SFQ, AHEAD = NV <= 8 ? 6 : 4;
      uint32_t v[AHEAD][NV];
      bool there[AHEAD];
      int g = 0, g_end = 0, row_p = 0, row_q = 0;
      auto next = [&](uint32_t (&to)[NV]) {
        if (g >= g_end) {
          if (!w.advance(a)) return false;
          row_p = (w.p * PAIR + rank) * 128 + lane;
          row_q = w.q * NT + lane;
          g = w.kb0 >> 2;
          g_end = ((w.kb1 - 1) >> 2) + 1;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) to[j] = row_p + j * 32 < a.p_rows ? a.p_scales[(size_t)g * a.p_rows + row_p + j * 32] : 0u;
#pragma unroll
        for (int j = 0; j < NV - 4; ++j) to[4 + j] = j * 32 < NT && row_q + j * 32 < a.q_rows ? a.q_scales[(size_t)g * a.q_rows + row_q + j * 32] : 0u;
        ++g;
        return true;
      };
#pragma unroll
      for (int d = 0; d < AHEAD; ++d) there[d] = (d == 0 || there[d > 0 ? d - 1 : 0]) && next(v[d]);
      for (uint32_t sc = 0; there[0];) {
#pragma unroll
        for (int d = 0; d < AHEAD; ++d) {
          if (!there[d]) continue;      // (then none of those behind it is there either)
          const uint32_t slot = sc % kMmScaleSlots;
          VSA2_WAIT_PARKED(&misc->sc_empty[slot], ((sc / kMmScaleSlots) & 1) ^ 1);
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
    } else if (sizeof(TO) == 4 && warp >= 4 && a.in_pieces) {
      // ---------------------------------------------------------------- epilogue of fp32 results in pieces: two groups of four warps, each half of the columns.  A thread keeps the
      // sums of its row's columns over the pieces in registers.  (Added up in C, through L2, they took a share of the products' intake: 2304 x 1536 x 32760 119.4 us in pieces of 40
      // blocks, 108.3 so.  It is long code, which a product of a single piece would have to fetch: 300 x 500 x 4000 8.8 us instead of 8.5)
      const int quad = warp & 3, group = (warp >> 2) - 1;
      constexpr int MINE = NT > 32 ? NT / 2 : NT, STEP = MINE % 32 == 0 ? 32 : 16;      // columns at a time
      if (group * MINE >= NT) goto done;
      float sum[MINE];
#pragma unroll
      for (int c = 0; c < MINE; ++c) sum[c] = 0.f;
      for (uint32_t seg = 0; w.advance(a); ++seg) {
        const uint32_t buf = seg & 1;
        VSA2_WAIT_PARKED(&misc->d_full[buf], (seg >> 1) & 1);
        tc::tc_fence_after();
        const uint32_t tmem = tmem_base + buf * 256 + group * MINE + ((uint32_t)(quad * 32) << 16);
        const int row = (w.p * PAIR + rank) * 128 + quad * 32 + lane, col = w.q * NT + group * MINE;
        const bool last = w.kb1 == w.r1;
        const int cols = row < a.p_rows ? a.q_rows - col : 0;      // columns that exist (or more)
        float* to = reinterpret_cast<float*>(a.c) + w.split * a.split_stride + (long long)col * a.ldc + row;
#pragma unroll
        for (int c0 = 0; c0 < MINE; c0 += STEP) {
          float v[STEP];
          load_columns(tmem + c0, v);
#pragma unroll
          for (int c = 0; c < STEP; ++c) {
            v[c] += sum[c0 + c];
            sum[c0 + c] = last ? 0.f : v[c];
          }
          if (last) {
            put_columns(to, a.ldc, cols - c0, v);
            to += STEP * a.ldc;
            __syncwarp();
          }
        }
        tc::tc_fence_before();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&misc->d_empty[buf]);
      }
    } else if (warp >= 4) {
      // ---------------------------------------------------------------- epilogue: two groups of four warps, each half of the columns
      const int quad = warp & 3, group = (warp >> 2) - 1;
      constexpr int FIRST = (NT / 32 + 1) / 2, MOST = FIRST;      // pieces of 32 columns that are group 0's
      const int piece0 = group == 0 ? 0 : FIRST, pieces = group == 0 ? FIRST : NT / 32 - FIRST;
      uint32_t syncs = 0, tiles = 0;
      if (pieces == 0) goto done;
      for (uint32_t seg = 0; w.advance(a); ++seg) {
        const uint32_t buf = seg & 1;
        const int first = (w.p * PAIR + rank) * 128, row = first + quad * 32 + lane, col = w.q * NT + piece0 * 32;
        const int cols = min(pieces * 32, a.q_rows - col);      // (0 or less: the tile ends before)
        VSA2_WAIT_PARKED(&misc->d_full[buf], (seg >> 1) & 1);
        tc::tc_fence_after();
        const uint32_t tmem = tmem_base + buf * 256 + piece0 * 32 + ((uint32_t)(quad * 32) << 16);
        auto release = [&] {
          tc::tc_fence_before();
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(&misc->d_empty[buf]);
        };
        if (sizeof(TO) == 2 && a.tensor_stores) {
          // bf16: all columns to registers first (the CTAs' stores come at the same time and take 5000 cycles), then in shared memory, turned unless SWAP, and out
          // by tensor copies that drop what lies outside C.  (Stored by the warps as they hold it, 64 bytes at a time, an accumulator took 13,000 cycles.)
          uint32_t u[MOST][16];
#pragma unroll
          for (int i = 0; i < MOST; ++i)
            if (i < pieces) take_tile(tmem + 32 * i, u[i]);
          release();
#pragma unroll
          for (int i = 0; i < MOST; ++i) {
            if (32 * i >= cols) break;
            unsigned char* tile = staging + (group * 2 + (tiles & 1)) * kMmTileBytes;
            stage_tile<SWAP>(tile, u[i], quad, lane);
            tc::fence_proxy_async_smem();
            if (quad == 0 && lane == 0) tc::bulk_store_wait_read();      // the tile before has been read: behind the barrier its place is free
            VSA2_GROUP_SYNC(&misc->group[group], syncs);
            if (quad == 0 && lane == 0) {
              if (SWAP) {
                if (first < a.p_rows) tma_store_2d(&tm_c, tile, col + 32 * i, first);
              } else {
#pragma unroll
                for (int b = 0; b < 2; ++b)
                  if (first + 64 * b < a.p_rows) tma_store_2d(&tm_c, tile + b * 4096, first + 64 * b, col + 32 * i);
              }
              tc::bulk_store_commit();
            }
            ++tiles;
          }
        } else {
          // (not SWAP: a thread's elements of C lie ldc apart)
          TO* const out = reinterpret_cast<TO*>(a.c) + w.split * a.split_stride + (long long)col * a.ldc + row;
#pragma unroll 1
          for (int c0 = 0; c0 < cols; c0 += 32) {
            float v[32];
            load_columns(tmem + c0, v);
            if (row < a.p_rows) put_columns(out + (long long)c0 * a.ldc, a.ldc, cols - c0, v);
          }
          release();
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

// The ranges of K, each a matrix [m, ldp] in fp32, added in their order.  Four elements of a row a thread.
template <typename TO>
__global__ void __launch_bounds__(256) fp8_sum_kernel(const float* parts, int splits, int m, int n, long long ldp, Divisor by_row, TO* __restrict__ c, long long ldc) {
  grid_enter();
  const int i = blockIdx.x * 256 + threadIdx.x, row = divided(i, by_row);      // (the parts have 4.3 million elements at most)
  if (row >= m) return;
  const int col = (i - row * (int)(ldp / 4)) * 4;
  const float* from = parts + row * ldp + col;
  float4 v[kMmSplits];
#pragma unroll
  for (int s = 0; s < kMmSplits; ++s)
    if (s < splits) v[s] = *reinterpret_cast<const float4*>(from + s * (m * ldp));
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < kMmSplits; ++s) {
    if (s < splits) {
      sum[0] += v[s].x; sum[1] += v[s].y; sum[2] += v[s].z; sum[3] += v[s].w;
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (col + j < n) put(c + row * ldc + col + j, sum[j]);
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
// C as boxes of 32 rows x 64 elements of bf16, with `swap` of 128 rows x 32
bool make_result_tmap(CUtensorMap* out, void* base, int rows, int cols, long long ld, bool swap) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (fn == nullptr) return false;
  cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)ld * 2};
  cuuint32_t box[2] = {swap ? 32u : 64u, swap ? 128u : 32u};
  cuuint32_t estr[2] = {1, 1};
  return fn(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            swap ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// One call
struct MmCall {
  int m, n, k, kb, ctas;
  Fp8Arg fa, fb;
  void* c;
  long long ldc;
  bool f32, tensor_stores;
  StatusBlock* status;
  float* parts;
  cudaStream_t st;
};

// How a product is cut, and the cycles that it is estimated at.  A block of K takes the tensor cores 2 cycles a column (128 rows of an SM), an issue of at least 300, and
// an SM is fed 52 bytes a cycle when all of them are, up to 64 when few are.  Where half the CTAs (or pairs) and more would have no tile, K is cut into ranges, each a
// matrix of its own in the workspace, which a second kernel adds (about 5000 cycles, and the bytes).
struct MmPlan {
  int pt, qt, splits;
  double cycles;
};
template <int NT, int PAIR>
MmPlan plan_mm(const MmCall& c, bool swap) {
  MmPlan plan;
  plan.pt = ((swap ? c.m : c.n) + 128 * PAIR - 1) / (128 * PAIR);
  plan.qt = ((swap ? c.n : c.m) + NT - 1) / NT;
  plan.splits = 1;
  const int of = c.ctas / PAIR;
  const long long tiles = (long long)plan.pt * plan.qt;
  auto products = [&](long long items, int blocks) {
    const double feed = 52.0 * kMmCtas / ((items < of ? items : of) * PAIR);
    const double fed = (kMmPBytes + NT / PAIR * 128) / (feed < 64.0 ? feed : 64.0);
    const double block = fed > 2.0 * NT ? fed : 2.0 * NT;
    return (double)((items + of - 1) / of) * blocks * (block > 300.0 ? block : 300.0);
  };
  const double epilogue = 12.0 * NT;      // of the last tile
  plan.cycles = products(tiles, c.kb) + epilogue;
  if (swap) plan.cycles *= 1.06;      // (its results go out 64 bytes at a time: 8192 x 4096 x 4096 98 us instead of 91)
  for (int s = 2; !swap && s <= kMmSplits && s <= c.kb && tiles * s <= of; ++s) {
    const double cycles = products(tiles * s, (c.kb + s - 1) / s) + epilogue + 5000 + 8.0 * s * c.m * c.n / (30.0 * kMmCtas);
    if (cycles < plan.cycles) {
      plan.cycles = cycles;
      plan.splits = s;
    }
  }
  return plan;
}

// Tiles along Q that are taken together, under all of P's rows one after the other: half a round of pairs, as far as their rows lie in L2 (48 MB).
// 75600 x 15360 x 5120, us: 6 tiles 4910, 12 4630, 24 4640, 37 4540, 74 5370
int tiles_together(int columns, int kb, int qt) {
  const long long group = (48LL << 20) / ((long long)columns * kb * 128);
  const int together = (int)(group < 4 ? 4 : group > 37 ? 37 : group);
  return together < qt ? together : qt;
}

template <int NT, int PAIR, bool SWAP, typename TO>
cudaError_t launch_tiles(const MmCall& c, const MmPlan& plan, void* result, long long ldc, long long split_stride) {
  using T = MmTile<NT, PAIR, TO>;
  const Fp8Arg &p = SWAP ? c.fa : c.fb, &q = SWAP ? c.fb : c.fa;
  MmArgs a;
  a.p_rows = SWAP ? c.m : c.n;
  a.q_rows = SWAP ? c.n : c.m;
  a.kb = c.kb;
  a.pt = plan.pt; a.qt = plan.qt; a.splits = plan.splits;
  a.gq = tiles_together(NT, c.kb, a.qt);
  a.by_tiles = divisor((long long)a.pt * a.qt);
  a.by_group = divisor((long long)a.gq * a.pt);
  a.by_gq = divisor(a.gq);
  a.by_rest = divisor(a.qt % a.gq > 0 ? a.qt % a.gq : a.gq);
  a.by_splits = divisor(a.splits);
  a.chunk = c.f32 ? kMmChunk : c.kb;
  a.in_pieces = (a.kb + a.splits - 1) / a.splits > a.chunk;
  a.tensor_stores = sizeof(TO) == 2 && c.tensor_stores;
  a.p_scales = reinterpret_cast<const uint32_t*>(p.scales);
  a.q_scales = reinterpret_cast<const uint32_t*>(q.scales);
  a.c = result; a.ldc = ldc; a.split_stride = split_stride;
  a.status = c.status;
  CUtensorMap tp, tq;
  if (!make_row_tmap(&tp, p.values, a.p_rows, c.k, p.ld, 128) || !make_row_tmap(&tq, q.values, a.q_rows, c.k, q.ld, NT / PAIR))
    return cudaErrorInvalidValue;
  CUtensorMap tm_c = tq;      // (without tensor stores: never used)
  if (a.tensor_stores && !make_result_tmap(&tm_c, result, c.m, c.n, ldc, SWAP)) return cudaErrorInvalidValue;
  const long long items = (long long)plan.pt * plan.qt * plan.splits;
  const int of = items < c.ctas / PAIR ? (int)items : c.ctas / PAIR;
  static KernelAttr attr;
  cudaError_t e;
  if ((e = prepare_kernel((const void*)fp8_matmul_kernel<NT, PAIR, SWAP, TO>, attr, T::SMEM))) return e;
  return launch_kernel(fp8_matmul_kernel<NT, PAIR, SWAP, TO>, of * PAIR, kMmThreads, T::SMEM, c.st, tp, tq, tm_c, a);
}

template <int NT, int PAIR>
cudaError_t launch_mm(const MmCall& c, const MmPlan& plan) {
  if (plan.splits == 1)
    return c.f32 ? launch_tiles<NT, PAIR, false, float>(c, plan, c.c, c.ldc, 0) : launch_tiles<NT, PAIR, false, bf16>(c, plan, c.c, c.ldc, 0);
  const long long ldp = (c.n + 3) / 4 * 4;
  const cudaError_t e = launch_tiles<NT, PAIR, false, float>(c, plan, c.parts, ldp, c.m * ldp);
  if (e != cudaSuccess) return e;
  const unsigned grid = (unsigned)((c.m * ldp / 4 + 255) / 256);
  const Divisor by_row = divisor(ldp / 4);
  return c.f32 ? launch_kernel(fp8_sum_kernel<float>, grid, 256, 0, c.st, c.parts, plan.splits, c.m, c.n, ldp, by_row, reinterpret_cast<float*>(c.c), c.ldc)
               : launch_kernel(fp8_sum_kernel<bf16>, grid, 256, 0, c.st, c.parts, plan.splits, c.m, c.n, ldp, by_row, reinterpret_cast<bf16*>(c.c), c.ldc);
}

// Tensor copies write whole units of 16 bytes: with an n that is no multiple of 8 they put zeros behind C's last column (into what else lies in its rows).  Such results take plain stores.
bool whole_units(int n) { return n % 8 == 0; }

// The kernel of a call: columns of a tile, CTAs that share one, which operand's rows are its lanes.  `pairs`: takes_pairs, and the context has room for one
struct MmChoice {
  int columns, pair;
  bool swap;
  MmPlan plan;
};
bool takes_pairs(const MmCall& call) { return call.m > 32 && call.n > 128 && call.ctas >= 2; }      // (wherever B has rows for both)
MmChoice choose_mm(const MmCall& call, bool pairs) {
  if (call.m <= 32) return {32, 1, false, plan_mm<32, 1>(call, false)};
  if (!pairs) return {128, 1, false, plan_mm<128, 1>(call, false)};
  const MmPlan narrow = plan_mm<128, 2>(call, false);
  if (call.m <= 128) return {128, 2, false, narrow};
  // The columns that waste least (256 x 4608 x 1536: two tiles of 128 instead of two of 224, 8.2 us instead of 9.5), and A's rows as the lanes, B's as the columns where that
  // fills the rounds better (512 x 15360 x 5120: 138 tiles instead of 180 on 74 pairs, 33 us instead of 45)
  const MmPlan wide = plan_mm<224, 2>(call, false);
  if (call.tensor_stores) {
    const MmPlan swapped = plan_mm<224, 2>(call, true);
    if (swapped.cycles < wide.cycles && swapped.cycles < narrow.cycles) return {224, 2, true, swapped};
  }
  return narrow.cycles < wide.cycles ? MmChoice{128, 2, false, narrow} : MmChoice{224, 2, false, wide};
}

// Most elements of the ranges of a product of up to m, n and k: tiles x ranges are at most the CTAs (or pairs), ranges at most the blocks of K.  (Grows with each of the three,
// so that one workspace serves smaller products, which are cut where a large one is not.)
size_t parts_elements(int m, int n, int k) {
  const size_t all = (size_t)kMmCtas * 128 * (m <= 32 ? 32 : m <= 128 ? 128 : 224), one = (size_t)m * (((size_t)n + 3) / 4 * 4);
  const int kb = (int)(((long long)k + 127) / 128), most = kb < kMmSplits ? kb : kMmSplits;
  if (most < 2) return 0;
  return one < all / most ? one * most : all;
}

}  // namespace

// [status][ranges of K]
size_t fp8_matmul_workspace_bytes(int m, int n, int k) { return align_up(sizeof(StatusBlock), 256) + parts_elements(m, n, k) * sizeof(float); }

cudaError_t launch_fp8_matmul(int m, int n, int k, const Fp8Arg& fa, const Fp8Arg& fb, void* c, int c_f32, long long ldc,
                              void* workspace, cudaStream_t st) {
  int sms = 0;
  cudaError_t e;
  if ((e = sm_count(&sms)) != cudaSuccess) return e;
  MmCall call;
  call.m = m; call.n = n; call.k = k;
  call.kb = (k + 127) / 128;
  call.ctas = sms < kMmCtas ? sms : kMmCtas;
  call.fa = fa; call.fb = fb;
  call.c = c; call.ldc = ldc;
  call.f32 = c_f32 != 0;
  call.tensor_stores = !c_f32 && (reinterpret_cast<uintptr_t>(c) & 15u) == 0 && ldc % 8 == 0 && whole_units(n);
  unsigned char* ws = reinterpret_cast<unsigned char*>(workspace);
  call.status = reinterpret_cast<StatusBlock*>(ws);
  call.parts = reinterpret_cast<float*>(ws + align_up(sizeof(StatusBlock), 256));
  call.st = st;
  bool pairs = takes_pairs(call);
  if (pairs) {
    static ClusterRoom room;
    if ((e = cluster_room((const void*)fp8_matmul_kernel<224, 2, false, float>, room, 2, kMmThreads, MmTile<224, 2, float>::SMEM, &pairs))) return e;
  }
  const MmChoice choice = choose_mm(call, pairs);
  if (choice.swap) return launch_tiles<224, 2, true, bf16>(call, choice.plan, c, ldc, 0);
  if (choice.columns == 32) return launch_mm<32, 1>(call, choice.plan);
  if (choice.pair == 1) return launch_mm<128, 1>(call, choice.plan);
  return choice.columns == 128 ? launch_mm<128, 2>(call, choice.plan) : launch_mm<224, 2>(call, choice.plan);
}

void fp8_matmul_plan(int m, int n, int k, int c_f32, bool tensor_stores, int sms, bool pairs, int32_t* out) {
  MmCall call = {};
  call.m = m; call.n = n; call.k = k;
  call.kb = (k + 127) / 128;
  call.ctas = sms < kMmCtas ? sms : kMmCtas;
  call.f32 = c_f32 != 0;
  call.tensor_stores = !c_f32 && tensor_stores && whole_units(n);
  const MmChoice choice = choose_mm(call, pairs && takes_pairs(call));
  out[0] = choice.columns; out[1] = choice.pair; out[2] = choice.swap;
  out[3] = choice.plan.splits; out[4] = choice.plan.qt; out[5] = tiles_together(choice.columns, call.kb, choice.plan.qt);
}

}  // namespace vsa2
