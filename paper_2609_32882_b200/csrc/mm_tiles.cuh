// What the products of 8-bit matrices share (fp8_matmul.cu, int8_matmul.cu): persistent CTAs, alone or in pairs of SMs, that walk over tiles and ranges of K; the ring's tensor copies;
// results on their way through shared memory.
#pragma once
#include <cuda.h>

#include "common.cuh"
#include "heads.cuh"
#include "tc05.cuh"
#include "tc_attn.cuh"
#include "tmap.cuh"

namespace vsa2 {

constexpr int kMmCtas = 148;            // most CTAs
constexpr int kMmThreads = 384;
constexpr int kMmSplits = 16;           // most ranges that K is cut into
constexpr uint32_t kMmPBytes = 128 * 128;
constexpr uint32_t kMmTileBytes = 32 * 128 * 2;      // 32 rows of C x 128 elements of bf16

// P: the operand whose rows are the accumulators' lanes, Q: the one whose rows are its columns
struct MmCut {
  int p_rows, q_rows, kb;            // kb: blocks of K
  int pt, qt, gq;                    // tiles along P, along Q; tiles along Q that are taken together
  int splits, chunk;                 // ranges that K is cut into; most blocks of K in one accumulator
  Divisor by_tiles, by_group, by_gq, by_rest, by_splits;      // pt qt; gq pt; gq, and what the last group has of tiles along Q
};
inline void fill_cut(MmCut& a, int p_rows, int q_rows, int kb, int pt, int qt, int splits, int gq, int chunk) {
  a.p_rows = p_rows; a.q_rows = q_rows;
  a.kb = kb;
  a.pt = pt; a.qt = qt; a.splits = splits;
  a.gq = gq;
  a.by_tiles = divisor((long long)a.pt * a.qt);
  a.by_group = divisor((long long)a.gq * a.pt);
  a.by_gq = divisor(a.gq);
  a.by_rest = divisor(a.qt % a.gq > 0 ? a.qt % a.gq : a.gq);
  a.by_splits = divisor(a.splits);
  a.chunk = chunk;
}

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
  __device__ __forceinline__ bool advance(const MmCut& a) {
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
// Columns of an accumulator's row, straight code where all of them exist: with a test for each element the loads and stores came one at a time, and
// the epilogue took longer than the products of 40 blocks.
__device__ __forceinline__ void put(float* to, float v) { *to = v; }
__device__ __forceinline__ void put(int* to, int v) { *to = v; }
__device__ __forceinline__ void put(bf16* to, float v) { *to = __float2bfloat16_rn(v); }
// elements `stride` apart (a warp's 32 rows lie next to one another in C)
// (in the pieces' epilogue eight addresses at a time: all of them at once are more registers than there are)
template <typename TO, typename TV, int N>
__device__ __forceinline__ void put_columns(TO* to, long long stride, int count, const TV (&v)[N]) {
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

// A tile of 32 x 32 results of bf16 as the fragments that stmatrix turns (four 8 x 8 blocks for each 8 columns), to rows of C in a tile that lies as the tensor copy takes it,
// 16-byte places exchanged by the row.  SWAP: 32 rows of C of this warp's, 64 bytes each, in one box of 128 rows.  Else turned, 32 rows of C of 32 elements, in two boxes of
// 32 rows x 64 elements (128 bytes)
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

inline bool make_row_tmap(CUtensorMap* out, const void* base, int rows, int cols, long long ld, int box_rows) {
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
inline bool make_result_tmap(CUtensorMap* out, void* base, int rows, int cols, long long ld, bool swap) {
  EncodeTiledFn fn = encode_tiled_fn();
  if (fn == nullptr) return false;
  cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  cuuint64_t strides[1] = {(cuuint64_t)ld * 2};
  cuuint32_t box[2] = {swap ? 32u : 64u, swap ? 128u : 32u};
  cuuint32_t estr[2] = {1, 1};
  return fn(out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            swap ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Tiles along Q that are taken together, under all of P's rows one after the other: half a round of pairs, as far as their rows lie in L2 (48 MB).
// 75600 x 15360 x 5120, us: 6 tiles 4910, 12 4630, 24 4640, 37 4540, 74 5370
inline int tiles_together(int columns, int kb, int qt) {
  const long long group = (48LL << 20) / ((long long)columns * kb * 128);
  const int together = (int)(group < 4 ? 4 : group > 37 ? 37 : group);
  return together < qt ? together : qt;
}

// Tensor copies write whole units of 16 bytes: with an n that is no multiple of 8 they put zeros behind C's last column (into what else lies in its rows).  Such results take plain stores.
inline bool whole_units(int n) { return n % 8 == 0; }

}  // namespace vsa2
