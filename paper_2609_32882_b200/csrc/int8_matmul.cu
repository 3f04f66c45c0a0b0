// C[m, n] = sa[m] sb[n] sum_k A[m, k] B[n, k] (+ bias[n]),  A and B in int8 with a scale a row (vsa2_int8_quantize, vsa2_residual_norm_fwd), C in bf16 or fp32.
//
// On the tensor cores: tcgen05.mma kind::i8 adds products of whole numbers in 32 bits, exactly, so ranges of K are added in any order and a result is the same however the product is
// cut.  The scales and the bias come in the epilogue: one of the two vectors is a lane's own, the other one lies in shared memory.
//
// Up to eight rows of A take a kernel of their own (int8_few_kernel).  Otherwise tiles and roles are as in the product of e4m3 matrices (fp8_matmul.cu): B's rows are the 128 rows of a CTA's tile, A's rows its NT columns; pairs of SMs share a tile of 256 x 256
// where there are rows for it.  No scales go to tensor memory, so the two accumulators have all of it.
//
// What bounds it: in long runs the power limit (75600 x 15360 x 5120 4.15 - 4.29 ms, 2.8 PFLOP/s; 18900 rows of it alone 866 us, 3.4 PFLOP/s, tensor pipe busy 93 % of the time);
// else the intake from L2 (8192 x 4096 x 4096 87 us, 4096^3 48); few tiles and short K: the launch, the first block's way from memory and the last tile's way out (2048 x 4608 x 1536
// 13.9 - 14.7 us, of which the products need 7); short K: each tile's way out of bf16 (30428 x 9048 x 171 214 us, K = 640 196, as fp32 219, the e4m3 product 175; pairs of 256 columns keep 64
// packed results a thread, and 44 bytes aside).  Asking for the next tile's scales ahead of time, or staging all of a tile's results at once in the place of a stage: no faster, or slower.
#include "mm_tiles.cuh"
#include "rows.cuh"

namespace vsa2 {

namespace {

constexpr int kI8StagesMost = 12;

// NT columns; PAIR: CTAs that share a tile; TO: type of the results, int32 for the sums of a range of K
template <int NT, int PAIR, typename TO>
struct I8Tile {
  static constexpr uint32_t STAGE = kMmPBytes + NT / PAIR * 128;
  static constexpr uint32_t STAGING = sizeof(TO) == 2 ? (NT > 32 ? 4 : 2) * kMmTileBytes : 0;      // two tiles of results for each group of the epilogue
  static constexpr uint32_t ROOM = 227 * 1024 - 8192 - STAGING;
  static constexpr int STAGES = ROOM / STAGE < kI8StagesMost ? ROOM / STAGE : kI8StagesMost;
  static constexpr size_t SMEM = 1024 + (size_t)STAGES * STAGE + STAGING;
  static constexpr int MINE = NT > 32 ? NT / 2 : NT;                        // columns of a group of the epilogue
};

struct I8Args : MmCut {
  int tensor_stores;                 // C lies as tensor copies need it, and ends where they end
  const float* p_scales;
  const float* q_scales;
  const float* p_bias;               // null: none
  void* c;
  long long ldc, split_stride;       // elements between the results of two ranges
  StatusBlock* status;
};

struct I8Misc {
  uint64_t full[kI8StagesMost], empty[kI8StagesMost];
  uint64_t d_full[2], d_empty[2], group[2];
  uint32_t tmem_base;
  int abort_flag;
  __align__(16) float of_column[2][2][128];      // scales of the columns, of even and odd items, of each group (read two at a time)
};

template <int PAIR>
__device__ __forceinline__ void mma_int8(uint32_t d, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, bool accumulate) {
  if constexpr (PAIR == 1)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"((uint32_t)accumulate)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"((uint32_t)accumulate)
        : "memory");
}
// signed 8 bits x signed 8 bits, sums of 32 bits, both operands K-major, 128 rows a CTA
template <int NT, int PAIR>
__device__ __forceinline__ constexpr uint32_t idesc_int8() {
  return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(NT >> 3) << 17) | ((uint32_t)(PAIR * 128 >> 4) << 24);
}

// The same steps wherever a result is formed, each rounded once
__device__ __forceinline__ float finished(int sum, float a_scale, float b_scale, float bias) {
  return __fmaf_rn(__fmul_rn(__int2float_rn(sum), a_scale), b_scale, bias);
}

template <int NT, int PAIR, typename TO>
__global__ void __cluster_dims__(PAIR, 1, 1) __launch_bounds__(kMmThreads, 1)
int8_matmul_kernel(const __grid_constant__ CUtensorMap tm_p, const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_c,
                   const __grid_constant__ I8Args a) {
  using T = I8Tile<NT, PAIR, TO>;
  constexpr bool SUMS = sizeof(TO) == 4 && TO(0.5f) == TO(0);      // a range's whole numbers
  extern __shared__ unsigned char mm_smem[];
  __shared__ I8Misc misc_store;
  I8Misc* misc = &misc_store;
  unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(mm_smem) + 1023) & ~(uintptr_t)1023);
  unsigned char* staging = ring + T::STAGES * T::STAGE;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = PAIR == 1 ? 0 : (int)cluster_rank();
  if (tid == 0) {
    misc->abort_flag = 0;
    for (int s = 0; s < T::STAGES; ++s) {
      tc::mbar_init(&misc->full[s], 1);
      tc::mbar_init(&misc->empty[s], 1);
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
      uint32_t s = 0, parity = 0, seg = 0;
      for (; w.advance(a); ++seg) {
        const uint32_t buf = seg & 1;
        VSA2_WAIT_PAIR(&misc->d_empty[buf], ((seg >> 1) & 1) ^ 1);
        for (int kb = w.kb0; kb < w.kb1; ++kb) {
          VSA2_WAIT(&misc->full[s], parity);
          tc::tc_fence_after();
          if (tc::elect_one()) {
            const uint64_t dp = ring_desc + (uint64_t)(s * T::STAGE >> 4), dq = dp + (uint64_t)(kMmPBytes >> 4);
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) mma_int8<PAIR>(tmem_base + buf * 256, dp + 2 * ks, dq + 2 * ks, idesc_int8<NT, PAIR>(), ks > 0 || kb > w.kb0);
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
    } else if (warp == 3 && rank == 1) {
      // ---------------------------------------------------------------- tells the first CTA which accumulators of this one have been read (by a warp that has no stores under way:
      // an arrival at the other CTA waits for them)
      for (uint32_t seg = 0; w.advance(a); ++seg) {
        VSA2_WAIT(&misc->d_empty[seg & 1], (seg >> 1) & 1);
        if (lane == 0) arrive_leader(&misc->d_empty[seg & 1]);
        __syncwarp();
      }
    } else if (warp >= 4) {
      // ---------------------------------------------------------------- epilogue: two groups of four warps, each half of the columns
      const int quad = warp & 3, group = (warp >> 2) - 1;
      constexpr int PIECES = T::MINE / 32;
      uint32_t syncs = 0, tiles = 0;
      if (group * T::MINE >= NT) goto done;
      for (uint32_t seg = 0; w.advance(a); ++seg) {
        const uint32_t buf = seg & 1;
        const int first = (w.p * PAIR + rank) * 128, row = first + quad * 32 + lane, col = w.q * NT + group * T::MINE;
        const int cols = min(T::MINE, a.q_rows - col);      // (0 or less: the tile ends before)
        const uint32_t tmem = tmem_base + buf * 256 + group * T::MINE + ((uint32_t)(quad * 32) << 16);
        const float* const of_column = misc->of_column[group][buf];
        auto release = [&] {
          tc::tc_fence_before();
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(&misc->d_empty[buf]);
        };
        if constexpr (SUMS) {
          VSA2_WAIT_PARKED(&misc->d_full[buf], (seg >> 1) & 1);
          tc::tc_fence_after();
          int* const out = reinterpret_cast<int*>(a.c) + w.split * a.split_stride + (long long)col * a.ldc + row;
#pragma unroll 1
          for (int c0 = 0; c0 < cols; c0 += 32) {
            uint32_t r[32];
            tc::tmem_ld32(tmem + c0, r);
            tc::tmem_ld_wait();
            int v[32];
#pragma unroll
            for (int c = 0; c < 32; ++c) v[c] = (int)r[c];
            if (row < a.p_rows) put_columns(out + (long long)c0 * a.ldc, a.ldc, cols - c0, v);
          }
          release();
        } else {
          // the columns' scales, while the products run.  (The other item's place may still be read: a warp that writes here has seen all four arrive behind the item before that one.)
          const int mine = quad * 32 + lane;
          if (mine < T::MINE) misc->of_column[group][buf][mine] = mine < cols ? a.q_scales[col + mine] : 0.f;
          if (sizeof(TO) == 2 && a.tensor_stores) {
            // bf16: through registers and shared memory, turned, and out by tensor copies that drop what lies outside C.  A thread's fragments are of four rows
            float scale[4], bias[4];
#pragma unroll
            for (int b = 0; b < 4; ++b) {
              const int r = first + quad * 32 + 8 * b + (lane >> 2);
              scale[b] = r < a.p_rows ? a.p_scales[r] : 0.f;
              bias[b] = r < a.p_rows && a.p_bias != nullptr ? a.p_bias[r] : 0.f;
            }
            VSA2_GROUP_SYNC(&misc->group[group], syncs);
            VSA2_WAIT_PARKED(&misc->d_full[buf], (seg >> 1) & 1);
            tc::tc_fence_after();
            uint32_t u[PIECES][16];
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
              uint32_t r[2][16];
              tc::tmem_ld_16x256b_x4(tmem + 32 * i, r[0]);
              tc::tmem_ld_16x256b_x4(tmem + 32 * i + (16u << 16), r[1]);
              tc::tmem_ld_wait();
#pragma unroll
              for (int g = 0; g < 4; ++g) {
                const float2 of = *reinterpret_cast<const float2*>(of_column + 32 * i + 8 * g + 2 * (lane & 3));      // of two columns
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                  const int lo = (int)r[b >> 1][4 * g + 2 * (b & 1)], hi = (int)r[b >> 1][4 * g + 2 * (b & 1) + 1];
                  u[i][4 * g + b] = pack_bf16x2(finished(lo, of.x, scale[b], bias[b]), finished(hi, of.y, scale[b], bias[b]));
                }
              }
            }
            release();
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
              if (32 * i >= cols) break;
              unsigned char* tile = staging + (group * 2 + (tiles & 1)) * kMmTileBytes;
              stage_tile<false>(tile, u[i], quad, lane);
              tc::fence_proxy_async_smem();
              if (quad == 0 && lane == 0) tc::bulk_store_wait_read();      // the tile before has been read: behind the barrier its place is free
              VSA2_GROUP_SYNC(&misc->group[group], syncs);
              if (quad == 0 && lane == 0) {
#pragma unroll
                for (int b = 0; b < 2; ++b)
                  if (first + 64 * b < a.p_rows) tma_store_2d(&tm_c, tile + b * 4096, first + 64 * b, col + 32 * i);
                tc::bulk_store_commit();
              }
              ++tiles;
            }
          } else {
            // (a thread's elements of C lie ldc apart)
            const float scale = row < a.p_rows ? a.p_scales[row] : 0.f, bias = row < a.p_rows && a.p_bias != nullptr ? a.p_bias[row] : 0.f;
            VSA2_GROUP_SYNC(&misc->group[group], syncs);
            VSA2_WAIT_PARKED(&misc->d_full[buf], (seg >> 1) & 1);
            tc::tc_fence_after();
            TO* const out = reinterpret_cast<TO*>(a.c) + (long long)col * a.ldc + row;
#pragma unroll 1
            for (int c0 = 0; c0 < cols; c0 += 32) {
              uint32_t r[32];
              tc::tmem_ld32(tmem + c0, r);
              tc::tmem_ld_wait();
              float v[32];
#pragma unroll
              for (int c = 0; c < 32; ++c) v[c] = finished((int)r[c], of_column[c0 + c], scale, bias);
              if (row < a.p_rows) put_columns(out + (long long)c0 * a.ldc, a.ldc, cols - c0, v);
            }
            release();
          }
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

// The ranges of K, each a matrix [m, ldp] of whole numbers, added and scaled.  Four elements of a row a thread.
template <typename TO>
__global__ void __launch_bounds__(256) int8_sum_kernel(const int* parts, int splits, int m, int n, long long ldp, Divisor by_row, const float* a_scales,
                                                       const float* b_scales, const float* n_bias, TO* __restrict__ c, long long ldc) {
  grid_enter();
  const int i = blockIdx.x * 256 + threadIdx.x, row = divided(i, by_row);      // (the parts have 4.9 million elements at most)
  if (row >= m) return;
  const int col = (i - row * (int)(ldp / 4)) * 4;
  const int* from = parts + row * ldp + col;
  int4 v[kMmSplits];
#pragma unroll
  for (int s = 0; s < kMmSplits; ++s)
    if (s < splits) v[s] = *reinterpret_cast<const int4*>(from + s * (m * ldp));
  int sum[4] = {0, 0, 0, 0};
#pragma unroll
  for (int s = 0; s < kMmSplits; ++s) {
    if (s < splits) {
      sum[0] += v[s].x; sum[1] += v[s].y; sum[2] += v[s].z; sum[3] += v[s].w;
    }
  }
  const float scale = a_scales[row];
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (col + j < n) put(c + row * ldc + col + j, finished(sum[j], scale, b_scales[col + j], n_bias != nullptr ? n_bias[col + j] : 0.f));
}

// Rows of the bias, or of zeros: a sum over nothing
template <typename TO>
__global__ void __launch_bounds__(256) int8_bias_kernel(int m, int n, const float* n_bias, TO* __restrict__ c, long long ldc) {
  grid_enter();
  const int col = blockIdx.x * 256 + threadIdx.x;
  if (col >= n) return;
  const float v = n_bias != nullptr ? n_bias[col] : 0.f;
  for (int row = blockIdx.y; row < m; row += gridDim.y) put(c + row * ldc + col, v);
}

// Few rows of A: every byte of B is read once and meets little work, and what counts is how many bytes are on their way.  The eight warps of a CTA share 16 rows of B; each has five
// neighbouring pieces of 64 bytes of them under way (four: 15.2 us instead of 14.3 for 1 x 15360 x 5120; pieces of a warp 512 bytes apart: 18.4).  The products are those of the warp-wide
// instruction on 16 x 8 x 32 values: memory is the bound (5.5 TB/s with the launch), and tensor memory and its pipeline are set up longer than a small product takes (1 x 4608 x 1536
// 2.6 us, on tiles of 32 columns 5.9; 8 x 15360 x 5120 15.1, 16.1).  Sums of four bytes at once by the integer units (dp4a) cost 12 cycles each: 14.4 us for one row, 56 for eight.
// The order in which the values of K are taken is of no account as long as it is the same for both: a lane's 16 neighbouring bytes are four of each quarter of two such products.
constexpr int kI8Few = 8, kI8FewThreads = 256;
// bytes at .. k - 1 of a row, less than 16, and zeros (bytes behind a row are not read)
__device__ __forceinline__ uint4 bytes16(const signed char* row, int at, int k) {
  uint32_t v[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int j = 0; j < 16; ++j)
    if (at + j < k) v[j / 4] |= (uint32_t)(unsigned char)row[at + j] << 8 * (j & 3);
  return make_uint4(v[0], v[1], v[2], v[3]);
}
// sum += rows g and g + 8 (values lo and hi, 32 of K) times columns g
__device__ __forceinline__ void mma_16x8x32(int (&sum)[4], uint32_t lo0, uint32_t hi0, uint32_t lo1, uint32_t hi1, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+r"(sum[0]), "+r"(sum[1]), "+r"(sum[2]), "+r"(sum[3]) : "r"(lo0), "r"(hi0), "r"(lo1), "r"(hi1), "r"(b0), "r"(b1));
}
template <typename TO>
__global__ void __launch_bounds__(kI8FewThreads, 4) int8_few_kernel(int m, int n, int k, const __grid_constant__ Int8Arg a, const __grid_constant__ Int8Arg b, const float* n_bias,
                                                                 TO* __restrict__ c, long long ldc) {
  constexpr int AHEAD = 5, WARPS = kI8FewThreads / 32;      // pieces of 64 bytes of a row under way
  __shared__ __align__(16) int part[WARPS][128];
  grid_enter();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, row = blockIdx.x * 16 + g;
  const signed char* const lo = b.values + min(row, n - 1) * b.ld;
  const signed char* const hi = b.values + min(row + 8, n - 1) * b.ld;
  const signed char* const x = a.values + min(g, m - 1) * a.ld;      // (columns behind m: not stored)
  int sum[4] = {0, 0, 0, 0};
  auto add = [&](const uint4& u, const uint4& v, const uint4& y) {
    mma_16x8x32(sum, u.x, v.x, u.y, v.y, y.x, y.y);
    mma_16x8x32(sum, u.z, v.z, u.w, v.w, y.z, y.w);
  };
  // rounds of `per` pieces a warp, next to one another in a row
  const int pieces = (k + 63) / 64, per = min(AHEAD, (pieces + WARPS - 1) / WARPS), in = (lane & 3) * 16;
#pragma unroll 1
  for (int first = warp * per; first < pieces; first += WARPS * per) {
    uint4 u[AHEAD], v[AHEAD];
    const int at = first * 64 + in;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const bool there = i < per && at + i * 64 + 16 <= k;
      u[i] = v[i] = make_uint4(0u, 0u, 0u, 0u);
      if (there) {
        u[i] = *reinterpret_cast<const uint4*>(lo + at + i * 64);
        v[i] = *reinterpret_cast<const uint4*>(hi + at + i * 64);
      }
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      uint4 y = make_uint4(0u, 0u, 0u, 0u);
      if (i < per && at + i * 64 + 16 <= k) y = *reinterpret_cast<const uint4*>(x + at + i * 64);
      if (i < per) add(u[i], v[i], y);
    }
  }
  if (warp == WARPS - 1 && k % 16 != 0) {      // what is behind the last whole 16
    const int at = in == 0 ? k / 16 * 16 : k;
    add(bytes16(lo, at, k), bytes16(hi, at, k), bytes16(x, at, k));
  }
  // the warps' parts: row g (+ 8), columns 2 (lane % 4), + 1
  *reinterpret_cast<int2*>(&part[warp][g * 8 + (lane & 3) * 2]) = make_int2(sum[0], sum[1]);
  *reinterpret_cast<int2*>(&part[warp][(g + 8) * 8 + (lane & 3) * 2]) = make_int2(sum[2], sum[3]);
  __syncthreads();
  const int i = threadIdx.x >> 4, col = blockIdx.x * 16 + (threadIdx.x & 15);      // (16 neighbouring results of a row of C)
  if (i >= m || i >= kI8Few || col >= n) return;
  int total = 0;
#pragma unroll
  for (int w = 0; w < WARPS; ++w) total += part[w][(threadIdx.x & 15) * 8 + i];
  put(c + i * ldc + col, finished(total, a.scales[i], b.scales[col], n_bias != nullptr ? n_bias[col] : 0.f));
}

// One call
struct I8Call {
  int m, n, k, kb, ctas;
  Int8Arg a, b;
  const float* bias;
  void* c;
  long long ldc;
  bool f32, tensor_stores;
  StatusBlock* status;
  int* parts;
  cudaStream_t st;
};

// How a product is cut, and the cycles that it is estimated at: as for e4m3 (fp8_matmul.cu), whose products run at the same pace.  Ranges of K are matrices of whole numbers in the
// workspace, which a second kernel adds (about 2000 cycles, and the bytes).
struct I8Plan {
  int pt, qt, splits;
  double cycles;
};
template <int NT, int PAIR>
I8Plan plan_i8(const I8Call& c) {
  I8Plan plan;
  plan.pt = (c.n + 128 * PAIR - 1) / (128 * PAIR);
  plan.qt = (c.m + NT - 1) / NT;
  plan.splits = 1;
  const int of = c.ctas / PAIR;
  const long long tiles = (long long)plan.pt * plan.qt;
  auto products = [&](long long items, int blocks) {
    const double feed = 52.0 * kMmCtas / ((items < of ? items : of) * PAIR);
    const double fed = (kMmPBytes + NT / PAIR * 128) / (feed < 64.0 ? feed : 64.0);
    const double block = fed > 2.0 * NT ? fed : 2.0 * NT;
    return (double)((items + of - 1) / of) * blocks * (block > 400.0 ? block : 400.0);
  };
  const double epilogue = 12.0 * NT + (PAIR == 2 ? 1500.0 : 0.0);      // of the last tile; a pair's start and end (103 x 893 x 150: 5.3 us, on CTAs alone 4.3)
  plan.cycles = products(tiles, c.kb) + epilogue;
  for (int s = 2; s <= kMmSplits && s <= c.kb && tiles * s <= of; ++s) {
    const double cycles = products(tiles * s, (c.kb + s - 1) / s) + epilogue + 2000 + 8.0 * s * c.m * c.n / (30.0 * kMmCtas);
    if (cycles < plan.cycles) {
      plan.cycles = cycles;
      plan.splits = s;
    }
  }
  return plan;
}

template <int NT, int PAIR, typename TO>
cudaError_t launch_i8_tiles(const I8Call& c, const I8Plan& plan, void* result, long long ldc, long long split_stride) {
  using T = I8Tile<NT, PAIR, TO>;
  const Int8Arg &p = c.b, &q = c.a;
  I8Args a;
  fill_cut(a, c.n, c.m, c.kb, plan.pt, plan.qt, plan.splits, tiles_together(NT, c.kb, plan.qt), c.kb);
  a.tensor_stores = sizeof(TO) == 2 && c.tensor_stores;
  a.p_scales = p.scales; a.q_scales = q.scales;
  a.p_bias = c.bias;
  a.c = result; a.ldc = ldc; a.split_stride = split_stride;
  a.status = c.status;
  CUtensorMap tp, tq;
  if (!make_row_tmap(&tp, p.values, a.p_rows, c.k, p.ld, 128) || !make_row_tmap(&tq, q.values, a.q_rows, c.k, q.ld, NT / PAIR)) return cudaErrorInvalidValue;
  CUtensorMap tm_c = tq;      // (without tensor stores: never used)
  if (a.tensor_stores && !make_result_tmap(&tm_c, result, c.m, c.n, ldc, false)) return cudaErrorInvalidValue;
  const long long items = (long long)plan.pt * plan.qt * plan.splits;
  const int of = items < c.ctas / PAIR ? (int)items : c.ctas / PAIR;
  static KernelAttr attr;
  cudaError_t e;
  if ((e = prepare_kernel((const void*)int8_matmul_kernel<NT, PAIR, TO>, attr, T::SMEM))) return e;
  return launch_kernel(int8_matmul_kernel<NT, PAIR, TO>, of * PAIR, kMmThreads, T::SMEM, c.st, tp, tq, tm_c, a);
}

template <int NT, int PAIR>
cudaError_t launch_i8(const I8Call& c, const I8Plan& plan) {
  if (plan.splits == 1)
    return c.f32 ? launch_i8_tiles<NT, PAIR, float>(c, plan, c.c, c.ldc, 0) : launch_i8_tiles<NT, PAIR, bf16>(c, plan, c.c, c.ldc, 0);
  const long long ldp = (c.n + 3) / 4 * 4;
  const cudaError_t e = launch_i8_tiles<NT, PAIR, int>(c, plan, c.parts, ldp, c.m * ldp);
  if (e != cudaSuccess) return e;
  const unsigned grid = (unsigned)((c.m * ldp / 4 + 255) / 256);
  const Divisor by_row = divisor(ldp / 4);
  return c.f32 ? launch_kernel(int8_sum_kernel<float>, grid, 256, 0, c.st, c.parts, plan.splits, c.m, c.n, ldp, by_row, c.a.scales, c.b.scales, c.bias,
                               reinterpret_cast<float*>(c.c), c.ldc)
               : launch_kernel(int8_sum_kernel<bf16>, grid, 256, 0, c.st, c.parts, plan.splits, c.m, c.n, ldp, by_row, c.a.scales, c.b.scales, c.bias,
                               reinterpret_cast<bf16*>(c.c), c.ldc);
}

template <typename TO>
cudaError_t launch_few(const I8Call& c) {
  return launch_kernel(int8_few_kernel<TO>, (c.n + 15) / 16, kI8FewThreads, 0, c.st, c.m, c.n, c.k, c.a, c.b, c.bias, reinterpret_cast<TO*>(c.c), c.ldc);
}

// The kernel of a call: columns of a tile, CTAs that share one, by the estimated cycles: over 110 random products of 9 to 20000 rows 1 % above the fastest cut on the average (pairs
// wherever they fit, and 5000 cycles for ranges: 9 %; 64 x 4608 x 1536 6.7 us on a pair, 5.9 on tiles of 32 columns; 955 x 216 x 1744 9.2 us whole, 7.6 in 4 ranges).
// `pairs`: takes_pairs, and the context has room for one.  (A's rows as lanes and B's as columns, which fills the rounds of e4m3 products on tiles of 256 x 224 better, is the same
// on square ones.)
struct I8Choice {
  int columns, pair;
  I8Plan plan;
};
bool takes_pairs(const I8Call& call) { return call.m > 32 && call.n > 128 && call.ctas >= 2; }      // (wherever B has rows for both)
I8Choice choose_i8(const I8Call& call, bool pairs) {
  I8Choice best = {128, 1, plan_i8<128, 1>(call)};
  auto consider = [&](int columns, int pair, const I8Plan& plan) {
    if (plan.cycles < best.plan.cycles) best = I8Choice{columns, pair, plan};
  };
  if (call.m <= 64) consider(32, 1, plan_i8<32, 1>(call));      // (more rows: several tiles that read the same weights)
  if (pairs) {
    consider(128, 2, plan_i8<128, 2>(call));
    if (call.m > 128) consider(256, 2, plan_i8<256, 2>(call));
  }
  return best;
}

// Most elements of the ranges of a product of up to m, n and k: tiles x ranges are at most the CTAs (or pairs), ranges at most the blocks of K.  (Grows with each of the three,
// so that one workspace serves smaller products, which are cut where a large one is not.)
size_t parts_elements(int m, int n, int k) {
  const size_t all = (size_t)kMmCtas * 128 * (m <= 32 ? 32 : m <= 128 ? 128 : 256), one = (size_t)m * (((size_t)n + 3) / 4 * 4);
  const int kb = (int)(((long long)k + 127) / 128), most = kb < kMmSplits ? kb : kMmSplits;
  if (most < 2) return 0;
  return one < all / most ? one * most : all;
}

}  // namespace

// [status][ranges of K]
size_t int8_matmul_workspace_bytes(int m, int n, int k) { return align_up(sizeof(StatusBlock), 256) + parts_elements(m, n, k) * sizeof(int); }

cudaError_t launch_bias_rows(int m, int n, const float* bias, void* c, int c_f32, long long ldc, cudaStream_t st) {
  const dim3 grid((n + 255) / 256, m < 1024 ? m : 1024);
  return c_f32 ? launch_kernel(int8_bias_kernel<float>, grid, 256, 0, st, m, n, bias, reinterpret_cast<float*>(c), ldc)
               : launch_kernel(int8_bias_kernel<bf16>, grid, 256, 0, st, m, n, bias, reinterpret_cast<bf16*>(c), ldc);
}

cudaError_t launch_int8_matmul(int m, int n, int k, const Int8Arg& a, const Int8Arg& b, const float* bias, void* c, int c_f32, long long ldc, void* workspace,
                               cudaStream_t st) {
  int sms = 0;
  cudaError_t e;
  if ((e = sm_count(&sms)) != cudaSuccess) return e;
  I8Call call;
  call.m = m; call.n = n; call.k = k;
  call.kb = (k + 127) / 128;
  call.ctas = sms < kMmCtas ? sms : kMmCtas;
  call.a = a; call.b = b;
  call.bias = bias;
  call.c = c; call.ldc = ldc;
  call.f32 = c_f32 != 0;
  call.tensor_stores = !c_f32 && (reinterpret_cast<uintptr_t>(c) & 15u) == 0 && ldc % 8 == 0 && whole_units(n);
  unsigned char* ws = reinterpret_cast<unsigned char*>(workspace);
  call.status = reinterpret_cast<StatusBlock*>(ws);
  call.parts = reinterpret_cast<int*>(ws + align_up(sizeof(StatusBlock), 256));
  call.st = st;
  if (m <= kI8Few) return call.f32 ? launch_few<float>(call) : launch_few<bf16>(call);
  bool pairs = takes_pairs(call);
  if (pairs) {
    static ClusterRoom room;
    if ((e = cluster_room((const void*)int8_matmul_kernel<256, 2, float>, room, 2, kMmThreads, I8Tile<256, 2, float>::SMEM, &pairs))) return e;
  }
  const I8Choice choice = choose_i8(call, pairs);
  if (choice.columns == 32) return launch_i8<32, 1>(call, choice.plan);
  if (choice.pair == 1) return launch_i8<128, 1>(call, choice.plan);
  return choice.columns == 128 ? launch_i8<128, 2>(call, choice.plan) : launch_i8<256, 2>(call, choice.plan);
}

void int8_matmul_plan(int m, int n, int k, int sms, bool pairs, int32_t* out) {
  I8Call call = {};
  call.m = m; call.n = n; call.k = k;
  call.kb = (k + 127) / 128;
  call.ctas = sms < kMmCtas ? sms : kMmCtas;
  if (m <= kI8Few) {
    out[0] = kI8Few;
    out[1] = out[2] = out[3] = out[4] = 1;
    return;
  }
  const I8Choice choice = choose_i8(call, pairs && takes_pairs(call));
  out[0] = choice.columns; out[1] = choice.pair;
  out[2] = choice.plan.splits; out[3] = choice.plan.qt; out[4] = tiles_together(choice.columns, call.kb, choice.plan.qt);
}

}  // namespace vsa2
