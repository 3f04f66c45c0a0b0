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
constexpr int kMmThreads = 256;
constexpr int kMmScaleSlots = 4;
constexpr int kMmCounters = 2 * kMmCtas;
constexpr uint32_t kMmPBytes = 128 * 128;
constexpr uint32_t kMmScaleBytes = 512 + 1024;       // words of 128 rows of B, of up to 256 rows of A
constexpr uint32_t kMmTmScales = 480;                // columns of tensor memory: accumulators at 0 and 256, scales here (2 x 16)

template <int NT>
struct MmTile {
  static constexpr uint32_t STAGE = kMmPBytes + NT * 128;
  static constexpr uint32_t ROOM = 227 * 1024 - 2048 - kMmScaleSlots * kMmScaleBytes;
  static constexpr int STAGES = ROOM / STAGE < 12 ? ROOM / STAGE : 12;
  static constexpr size_t SMEM = 1024 + (size_t)STAGES * STAGE + kMmScaleSlots * kMmScaleBytes;
  static constexpr int SFQ = (NT + 127) / 128;        // 512-byte pieces of A's scales
};

struct MmArgs {
  int m, n, k, kb;                   // kb: blocks of K
  int pt, qt, gq;                    // tiles along n, along m; tiles along m that are taken together
  int whole;                         // tiles that are dealt out whole (a multiple of the CTAs)
  long long units;                   // blocks of K of the other tiles, all told
  const uint32_t* a_scales;
  const uint32_t* b_scales;
  void* c;
  long long ldc;
  int c_f32;
  StatusBlock* status;
  int* counters;
  float* partial;
};

struct MmMisc {
  uint64_t full[12], empty[12], sc_full[kMmScaleSlots], sc_empty[kMmScaleSlots], d_full[2], d_empty[2], group;
  uint32_t tmem_base;
  int abort_flag;
  int last;
};

// A CTA's share: whole tiles first, then its part of the units of the others.
struct MmWalk {
  int tile, kb0, kb1;                // current segment
  int next;                          // its number
  long long u, u1;
  __device__ __forceinline__ void init(const MmArgs& a) {
    next = 0;
    u = a.units * blockIdx.x / gridDim.x;
    u1 = a.units * (blockIdx.x + 1) / gridDim.x;
  }
  __device__ __forceinline__ bool advance(const MmArgs& a) {
    const long long t = (long long)next * gridDim.x + blockIdx.x;
    if (t < a.whole) {
      ++next;
      tile = (int)t; kb0 = 0; kb1 = a.kb;
      return true;
    }
    if (u >= u1) return false;
    ++next;
    const int r = (int)(u / a.kb);
    tile = a.whole + r;
    kb0 = (int)(u - (long long)r * a.kb);
    kb1 = (int)min((long long)a.kb, kb0 + (u1 - u));
    u += kb1 - kb0;
    return true;
  }
};
__device__ __forceinline__ void mm_place(const MmArgs& a, int tile, int& p, int& q) {
  const int per = a.gq * a.pt, g = tile / per, r = tile - g * per, w = min(a.gq, a.qt - g * a.gq);
  p = r / w;
  q = g * a.gq + r - p * w;
}

__device__ __forceinline__ void tma_load_2d(void* dst, const CUtensorMap* m, uint64_t* bar, int c0, int c1) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
               ::"r"(tc::smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(m)), "r"(tc::smem_u32(bar)), "r"(c0), "r"(c1)
               : "memory");
}
// 32 x 16 bytes of shared memory to four columns of tensor memory, the same in each group of 32 lanes: words (r, j) of row j * 32 + r
__device__ __forceinline__ void copy_scales(uint32_t taddr, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
__device__ __forceinline__ void mma_scaled(uint32_t d, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t sfa, uint32_t sfb, bool accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
      ::"r"(d), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sfa), "r"(sfb), "r"((uint32_t)accumulate)
      : "memory");
}
// e4m3 x e4m3, ue8m0 scales, both operands K-major; `sf`: which byte of the scales' words
__device__ __forceinline__ constexpr uint32_t idesc_scaled(int n, uint32_t sf) {
  return (sf << 4) | ((uint32_t)(n >> 3) << 17) | (1u << 23) | (1u << 27) | (sf << 29);
}

template <int NT>
__global__ void __launch_bounds__(kMmThreads, 1) fp8_matmul_kernel(const __grid_constant__ CUtensorMap tm_p, const __grid_constant__ CUtensorMap tm_q,
                                                                   const __grid_constant__ MmArgs a) {
  using T = MmTile<NT>;
  extern __shared__ unsigned char mm_smem[];
  __shared__ MmMisc misc_store;
  MmMisc* misc = &misc_store;
  unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(mm_smem) + 1023) & ~(uintptr_t)1023);
  unsigned char* scales = ring + T::STAGES * T::STAGE;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    misc->abort_flag = 0;
    for (int s = 0; s < T::STAGES; ++s) {
      tc::mbar_init(&misc->full[s], 1);
      tc::mbar_init(&misc->empty[s], 1);
    }
    for (int s = 0; s < kMmScaleSlots; ++s) {
      tc::mbar_init(&misc->sc_full[s], 32);
      tc::mbar_init(&misc->sc_empty[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      tc::mbar_init(&misc->d_full[s], 1);
      tc::mbar_init(&misc->d_empty[s], 128);
    }
    tc::mbar_init(&misc->group, 128);
    tc::fence_barrier_init();
    tc::prefetch_tmap(&tm_p);
    tc::prefetch_tmap(&tm_q);
  }
  if (warp == 3) {
    tc::tmem_alloc(&misc->tmem_base, 512);
    tc::tmem_relinquish();
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem_base = misc->tmem_base;
  grid_enter(false);
  {
    MmWalk w;
    w.init(a);
    if (warp == 0) {
      // ---------------------------------------------------------------- operands
      uint32_t it = 0;
      while (w.advance(a)) {
        int p, q;
        mm_place(a, w.tile, p, q);
        for (int kb = w.kb0; kb < w.kb1; ++kb, ++it) {
          const uint32_t s = it % T::STAGES;
          int ok = 1;
          if (lane == 0) {
            ok = tc::mbar_wait(&misc->empty[s], ((it / T::STAGES) & 1) ^ 1, &misc->abort_flag);
            if (ok) {
              tc::mbar_expect_tx(&misc->full[s], T::STAGE);
              tma_load_2d(ring + s * T::STAGE, &tm_p, &misc->full[s], kb * 128, p * 128);
              tma_load_2d(ring + s * T::STAGE + kMmPBytes, &tm_q, &misc->full[s], kb * 128, q * NT);
            }
          }
          if (!__shfl_sync(0xffffffffu, ok, 0)) goto done;
        }
      }
    } else if (warp == 1) {
      // ---------------------------------------------------------------- products (converged warp, one lane issues)
      const uint64_t ring_desc = tc::smem_desc_sw128(tc::smem_u32(ring), 16, 1024);
      const uint64_t scale_desc = tc::smem_desc_plain(tc::smem_u32(scales), 16, 128);
      uint32_t it = 0, sc = 0, seg = 0;
      for (; w.advance(a); ++seg) {
        const uint32_t buf = seg & 1;
        VSA2_WAIT(&misc->d_empty[buf], ((seg >> 1) & 1) ^ 1);
        for (int kb = w.kb0; kb < w.kb1; ++kb, ++it) {
          const uint32_t s = it % T::STAGES;
          const bool fresh = kb == w.kb0 || (kb & 3) == 0;
          if (fresh) {
            VSA2_WAIT(&misc->sc_full[sc % kMmScaleSlots], (sc / kMmScaleSlots) & 1);
            ++sc;
          }
          VSA2_WAIT(&misc->full[s], (it / T::STAGES) & 1);
          tc::tc_fence_after();
          if (tc::elect_one()) {
            const uint32_t slot = (sc - 1) % kMmScaleSlots, tm_sc = tmem_base + kMmTmScales + ((sc - 1) & 1) * 16;
            if (fresh) {
              const uint64_t d = scale_desc + (uint64_t)(slot * kMmScaleBytes >> 4);
              copy_scales(tm_sc, d);
#pragma unroll
              for (int i = 0; i < T::SFQ; ++i) copy_scales(tm_sc + 4 + 4 * i, d + (uint64_t)((512 + 512 * i) >> 4));
              tc::mma_commit(&misc->sc_empty[slot]);
            }
            const uint64_t dp = ring_desc + (uint64_t)(s * T::STAGE >> 4), dq = dp + (uint64_t)(kMmPBytes >> 4);
            const uint32_t idesc = idesc_scaled(NT, kb & 3);
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
              mma_scaled(tmem_base + buf * 256, dp + 2 * ks, dq + 2 * ks, idesc, tm_sc, tm_sc + 4, ks > 0 || kb > w.kb0);
            tc::mma_commit(&misc->empty[s]);
            if (kb == w.kb1 - 1) tc::mma_commit(&misc->d_full[buf]);
          }
          __syncwarp();
        }
      }
    } else if (warp == 2) {
      // ---------------------------------------------------------------- scales: words of rows lane, lane + 32, .. as 16 bytes a lane
      uint32_t sc = 0;
      while (w.advance(a)) {
        int p, q;
        mm_place(a, w.tile, p, q);
        for (int g = w.kb0 >> 2; g <= (w.kb1 - 1) >> 2; ++g, ++sc) {
          const uint32_t slot = sc % kMmScaleSlots;
          uint32_t v[4 + 4 * T::SFQ];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int r = p * 128 + j * 32 + lane;
            v[j] = r < a.n ? a.b_scales[(size_t)g * a.n + r] : 0u;
          }
#pragma unroll
          for (int j = 0; j < 4 * T::SFQ; ++j) {
            const int i = j * 32 + lane, r = q * NT + i;
            v[4 + j] = i < NT && r < a.m ? a.a_scales[(size_t)g * a.m + r] : 0u;
          }
          VSA2_WAIT_PARKED(&misc->sc_empty[slot], ((sc / kMmScaleSlots) & 1) ^ 1);
          unsigned char* to = scales + slot * kMmScaleBytes + lane * 16;
#pragma unroll
          for (int j = 0; j <= T::SFQ; ++j)
            *reinterpret_cast<uint4*>(to + j * 512) = make_uint4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
          tc::fence_proxy_async_smem();
          tc::mbar_arrive(&misc->sc_full[slot]);
        }
      }
    } else if (warp >= 4) {
      // ---------------------------------------------------------------- epilogue
      const int quad = warp & 3;
      constexpr int STEP = NT < 32 ? 16 : 32;
      uint32_t syncs = 0;
      for (uint32_t seg = 0; w.advance(a); ++seg) {
        const uint32_t buf = seg & 1;
        int p, q;
        mm_place(a, w.tile, p, q);
        const int n = p * 128 + quad * 32 + lane, cols = min(NT, a.m - q * NT);
        const bool in = n < a.n;
        VSA2_WAIT_PARKED(&misc->d_full[buf], (seg >> 1) & 1);
        tc::tc_fence_after();
        const bool all = w.kb0 == 0 && w.kb1 == a.kb;
        float* part = nullptr;
        if (!all) part = a.partial + ((size_t)blockIdx.x * 2 + (w.kb0 == 0 ? 1 : 0)) * (128 * NT) + quad * 32 + lane;
        const size_t at = (size_t)(q * (long long)NT * a.ldc) + n;
#pragma unroll 1
        for (int c0 = 0; c0 < cols; c0 += STEP) {
          uint32_t r[STEP];
          const uint32_t taddr = tmem_base + buf * 256 + c0 + ((uint32_t)(quad * 32) << 16);
          if constexpr (STEP == 32) tc::tmem_ld32(taddr, r);
          else tc::tmem_ld16(taddr, r);
          tc::tmem_ld_wait();
#pragma unroll
          for (int c = 0; c < STEP; ++c) {
            if (!all) __stcg(part + (size_t)(c0 + c) * 128, __uint_as_float(r[c]));
            else if (in && c0 + c < cols) store_out(a.c, at + (size_t)(c0 + c) * a.ldc, __uint_as_float(r[c]), a.c_f32);
          }
        }
        tc::tc_fence_before();
        tc::mbar_arrive(&misc->d_empty[buf]);
        if (!all) {
          // the tile's parts: those of the CTAs that its units fall to, in their order
          const long long first = (long long)(w.tile - a.whole) * a.kb;
          int lo = (int)(first * gridDim.x / a.units), hi = (int)((first + a.kb - 1) * gridDim.x / a.units);
          while (a.units * (lo + 1) / gridDim.x <= first) ++lo;
          while (a.units * lo / gridDim.x > first) --lo;
          while (a.units * (hi + 1) / gridDim.x <= first + a.kb - 1) ++hi;
          while (a.units * hi / gridDim.x > first + a.kb - 1) --hi;
          __threadfence();
          VSA2_GROUP_SYNC(&misc->group, syncs);
          if (quad == 0 && lane == 0) {
            int* counter = a.counters + (w.tile - a.whole);
            const bool last = atomicAdd(counter, 1) == hi - lo;
            if (last) *counter = 0;
            misc->last = last;
            __threadfence();
          }
          VSA2_GROUP_SYNC(&misc->group, syncs);
          if (misc->last) {
            __threadfence();
#pragma unroll 1
            for (int c = 0; c < cols; ++c) {
              float sum = 0.f;
              for (int cta = lo; cta <= hi; ++cta) {
                const bool begins = a.units * cta / gridDim.x <= first;       // its part begins with the tile
                sum += __ldcg(a.partial + ((size_t)cta * 2 + (begins ? 1 : 0)) * (128 * NT) + (size_t)c * 128 + quad * 32 + lane);
              }
              if (in) store_out(a.c, at + (size_t)c * a.ldc, sum, a.c_f32);
            }
          }
          VSA2_GROUP_SYNC(&misc->group, syncs);       // (misc->last is read before it is written again)
        }
      }
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
  if (warp == 3) tc::tmem_dealloc(tmem_base, 512);
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

int mm_width(int m) { return m <= 16 ? 16 : m <= 32 ? 32 : m <= 64 ? 64 : m <= 128 ? 128 : 224; }

template <int NT>
cudaError_t launch_mm(MmArgs a, const Fp8Arg& fa, const Fp8Arg& fb, int ctas, cudaStream_t st) {
  CUtensorMap tp, tq;
  if (!make_row_tmap(&tp, fb.values, a.n, a.k, fb.ld, 128) || !make_row_tmap(&tq, fa.values, a.m, a.k, fa.ld, NT)) return cudaErrorInvalidValue;
  static KernelAttr attr;
  cudaError_t e;
  if ((e = prepare_kernel((const void*)fp8_matmul_kernel<NT>, attr, MmTile<NT>::SMEM))) return e;
  return launch_kernel(fp8_matmul_kernel<NT>, ctas, kMmThreads, MmTile<NT>::SMEM, st, tp, tq, a);
}

}  // namespace

// [status][counters of the tiles that are cut][two parts a CTA]
size_t fp8_matmul_workspace_bytes(int m, int n, int k) {
  (void)n;
  (void)k;
  return align_up(sizeof(StatusBlock) + kMmCounters * sizeof(int), 256) + (size_t)2 * kMmCtas * 128 * mm_width(m) * sizeof(float);
}

cudaError_t launch_fp8_matmul(int m, int n, int k, const Fp8Arg& fa, const Fp8Arg& fb, void* c, int c_f32, long long ldc,
                              void* workspace, cudaStream_t st) {
  int sms = 0;
  cudaError_t e;
  if ((e = sm_count(&sms)) != cudaSuccess) return e;
  const int nt = mm_width(m);
  MmArgs a;
  a.m = m; a.n = n; a.k = k;
  a.kb = (k + 127) / 128;
  a.pt = (n + 127) / 128;
  a.qt = (m + nt - 1) / nt;
  a.gq = a.qt < 12 ? a.qt : 12;
  int ctas = sms < kMmCtas ? sms : kMmCtas;
  const long long tiles = (long long)a.pt * a.qt, all_units = tiles * a.kb;
  if (all_units < ctas) ctas = (int)all_units;
  // whole rounds, but for the last full one, which joins the remainder (parts of about one to two tiles a CTA instead of less than one)
  long long rounds = tiles / ctas;
  if (tiles % ctas != 0 && rounds > 0) --rounds;
  a.whole = (int)(rounds * ctas);
  a.units = (tiles - a.whole) * a.kb;
  a.a_scales = reinterpret_cast<const uint32_t*>(fa.scales);
  a.b_scales = reinterpret_cast<const uint32_t*>(fb.scales);
  a.c = c; a.c_f32 = c_f32; a.ldc = ldc;
  unsigned char* ws = reinterpret_cast<unsigned char*>(workspace);
  a.status = reinterpret_cast<StatusBlock*>(ws);
  a.counters = reinterpret_cast<int*>(ws + sizeof(StatusBlock));
  a.partial = reinterpret_cast<float*>(ws + align_up(sizeof(StatusBlock) + kMmCounters * sizeof(int), 256));
  switch (nt) {
    case 16: return launch_mm<16>(a, fa, fb, ctas, st);
    case 32: return launch_mm<32>(a, fa, fb, ctas, st);
    case 64: return launch_mm<64>(a, fa, fb, ctas, st);
    case 128: return launch_mm<128>(a, fa, fb, ctas, st);
    default: return launch_mm<224>(a, fa, fb, ctas, st);
  }
}

}  // namespace vsa2
