// The residual stream of a layer: h = residual + dropout(x) and y = h / sqrt(mean(h^2) + eps) * w, row by row, and back.
//   forward : y leaves in bf16 or fp32, in e4m3 with a power-of-two scale for each 128 values (the operand of vsa2_fp8_matmul), in int8 with a scale for the row (that of
//             vsa2_int8_matmul), or several of these; h is rounded to the stream's type first, and the norm is that of what is stored
//   backward: with r = 1 / sqrt(mean(h^2) + eps), g = w dy:  dh' = dh + r g - h r^3 mean(g h);  dx = dropout's part of dh';  dw = sum over the rows of dy h r
//   int8    : v = h w (for vsa2_int8_quantize a matrix' own values), s = max |v| / 127, value = v * (127 / max |v|) rounded to nearest, ties to even; the row's r is part of its
//             scale alone, so a value does not depend on how the sum of squares was rounded
// A CTA takes a row at a time, eight neighbouring elements in each of a thread's V pieces: the row is read once, stays in registers while its sums pass through one barrier, and
// leaves.  Bound by memory.  Rows of more than 8192 elements (MANY) are read twice, the second time from L2, in a loop over the pieces.
#include "fp8_values.cuh"
#include "rows.cuh"

namespace vsa2 {

namespace {

constexpr int kNormMost = 512;       // threads of a CTA at most
constexpr int kNormParts = 1184;     // most CTAs of the backward, each with its own partial sums of the weight's gradient (eight for each of 148 SMs)
constexpr float kInt8Least = 0x1p-100f;      // least max |v|: below it 127 / max |v| would leave fp32's range

// Rows whose mean square lies outside are taken again times a power of two: their squares could vanish or pass fp32's range
constexpr float kLeastSquare = 0x1p-40f, kMostSquare = 0x1p40f;
__device__ __forceinline__ bool in_range(float mean_square) { return mean_square >= kLeastSquare && mean_square <= kMostSquare; }
// The power of two that brings the larger of a row's largest magnitude (its bits) and sqrt(eps) to about one; one where that is zero or not finite
__device__ __forceinline__ float power_for(uint32_t top_bits, float eps) {
  const int e = max(top_bits, __float_as_uint(sqrtf(eps))) >> 23;
  return e == 0 || e == 255 ? (e == 0 && top_bits != 0 ? 0x1p126f : 1.f) : __int_as_float(max(254 - e, 1) << 23);
}

struct RowSums {      // double-buffered by the row's parity: one barrier a row
  float2 of[2][kNormMost / 32];
};
// Sum of `sum` and of `other` (MAX: the largest of its bits as an unsigned number) over the CTA, the same bits in every thread
template <bool MAX>
__device__ __forceinline__ float2 row_total(float sum, float other, RowSums& sh, uint32_t parity) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (!MAX) other += __shfl_xor_sync(0xffffffffu, other, o);
  }
  if (MAX) other = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(other)));
  if (warps == 1) return make_float2(sum, other);
  float2* of = sh.of[parity & 1];
  if (lane == 0) of[warp] = make_float2(sum, other);
  __syncthreads();
  const float2 v = lane < warps ? of[lane] : make_float2(0.f, 0.f);
  sum = v.x;
  other = v.y;
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) {      // (16 warps at most)
    sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (!MAX) other += __shfl_xor_sync(0xffffffffu, other, o);
  }
  sum = __shfl_sync(0xffffffffu, sum, 0);
  if (MAX) other = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(other)));
  else other = __shfl_sync(0xffffffffu, other, 0);
  return make_float2(sum, other);
}

__device__ __forceinline__ void load_weight(float (&w)[8], const float* from, int i, int cols) {
  // (weights may lie at any fp32's address)
#pragma unroll
  for (int j = 0; j < 8; ++j) w[j] = from == nullptr ? 1.f : i + j < cols ? from[i + j] : 0.f;
}
// (aligned, whole pieces)
__device__ __forceinline__ void load_weight(float (&w)[8], const float4* from) {
  const float4 a = from[0], b = from[1];
  w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
}
template <bool VEC>
__device__ __forceinline__ void weight_of(float (&w)[8], const float* from, int i, int cols) {
  if (VEC && from != nullptr && i + 8 <= cols) load_weight(w, reinterpret_cast<const float4*>(from + i));
  else load_weight(w, from, i, cols);
}

// ---- the forms that y leaves in
// e4m3: the 16 threads of a block of 128 find its scale together.  (By whole warps; pieces behind the row are zeros.)
__device__ __forceinline__ void put_fp8(const float (&v)[8], float r, const NormFwdArgs& a, int row, int oct) {
  float f[8];
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    f[j] = v[j] * r;
    top = max(top, __float_as_uint(f[j]) & 0x7fffffffu);
  }
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  const bool odd = __any_sync(0xffffffffu, top >= kInf);
  if (odd) {
    top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (finite_bits(f[j])) top = max(top, __float_as_uint(f[j]) & 0x7fffffffu);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  }
  if (oct >= a.octs) return;
  const uint32_t byte = scale_byte(top);
  const float inv = inverse_scale(byte);
#pragma unroll
  for (int j = 0; j < 8; ++j) f[j] = odd ? scaled<true>(f[j], inv) : f[j] * inv;
  put8(a.fp8.values + row * a.fp8.ld, oct * 8, a.cols, e4m3x4(f[0], f[1], f[2], f[3]), e4m3x4(f[4], f[5], f[6], f[7]));
  if ((oct & 15) == 0) put_scale(a.fp8.scales, a.rows, row, oct >> 4, (a.octs + 15) >> 4, byte);
}
// int8: the product is rounded once, then to a whole number by an addition whose last bit is one (1.5 * 2^23; |product| is 127 and a little at most)
__device__ __forceinline__ uint32_t int8x4(float a, float b, float c, float d, float inv) {
  const uint32_t i = __float_as_uint(__fadd_rn(__fmul_rn(a, inv), 12582912.f)), j = __float_as_uint(__fadd_rn(__fmul_rn(b, inv), 12582912.f)),
                 k = __float_as_uint(__fadd_rn(__fmul_rn(c, inv), 12582912.f)), l = __float_as_uint(__fadd_rn(__fmul_rn(d, inv), 12582912.f));
  return __byte_perm(__byte_perm(i, j, 0x0040), __byte_perm(k, l, 0x0040), 0x5410);
}
// top: bits of the row's max |v|.  A row that holds something that is not finite has no scale: zeros, and a scale that makes its products NaN
__device__ __forceinline__ void put_int8(const float (&v)[8], uint32_t top, const Int8Arg& out, int row, int oct, int cols) {
  const float inv = __fdiv_rn(127.f, fmaxf(__uint_as_float(top), kInt8Least));
  const bool fine = top < kInf;
  put8(reinterpret_cast<unsigned char*>(out.values) + row * out.ld, oct * 8, cols, fine ? int8x4(v[0], v[1], v[2], v[3], inv) : 0u,
       fine ? int8x4(v[4], v[5], v[6], v[7], inv) : 0u);
}
__device__ __forceinline__ float int8_scale(uint32_t top, float r) {
  return top < kInf ? __fdiv_rn(fmaxf(__uint_as_float(top), kInt8Least), 127.f) * r : __uint_as_float(0x7fffffffu);
}

// V: pieces of eight elements a thread (MANY: as many as it takes, in a loop); NORM: else the int8 form of x as it is
template <int V, bool MANY, typename X, typename S, bool NORM, bool VEC>
__global__ void __launch_bounds__(kNormMost) norm_fwd_kernel(const __grid_constant__ NormFwdArgs a) {
  __shared__ RowSums sh;
  grid_enter();
  const int t = threadIdx.x, T = blockDim.x;
  DropMask mask;
  mask.init(a.drop);
  const int rounds = MANY ? (a.octs + T * V - 1) / (T * V) : 1;
  const bool want_int8 = a.int8.values != nullptr;
  uint32_t turn = 0;
  for (int row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const X* const xp = reinterpret_cast<const X*>(a.x.p) + row * a.x.ld;
    const S* const rp = a.r.p != nullptr ? reinterpret_cast<const S*>(a.r.p) + row * a.r.ld : nullptr;
    Eight<S> h[V];
    auto fetch = [&](int first) {      // h of the pieces first + t, first + t + T, ..
      Eight<X> x[V];
#pragma unroll
      for (int v = 0; v < V; ++v) load_eight<VEC>(x[v], xp, (first + v * T + t) * 8, a.cols);
      if (rp != nullptr) {
#pragma unroll
        for (int v = 0; v < V; ++v) load_eight<VEC>(h[v], rp, (first + v * T + t) * 8, a.cols);
      }
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = x[v].get(j);
        mask.apply(f, row, first + v * T + t);
        if (rp != nullptr) {
#pragma unroll
          for (int j = 0; j < 8; ++j) f[j] = __fadd_rn(h[v].get(j), f[j]);
        }
        h[v].round(f);
      }
    };
    auto keep = [&](int first) {
      if (a.h.p == nullptr) return;
#pragma unroll
      for (int v = 0; v < V; ++v) store_eight<VEC>(h[v], reinterpret_cast<S*>(a.h.p) + row * a.h.ld, (first + v * T + t) * 8, a.cols);
    };
    // sum of squares and the largest |h w|, of h times s; `largest`: of |h|
    auto sums = [&](int first, float s, bool weighted, float& ss, uint32_t& top) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float w[8];
        if (NORM && weighted && want_int8) weight_of<VEC>(w, a.w, (first + v * T + t) * 8, a.cols);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float f = h[v].get(j) * s;
          if (NORM) ss += f * f;
          if (!weighted || want_int8) top = max(top, __float_as_uint(NORM && weighted ? __fmul_rn(f, w[j]) : f) & 0x7fffffffu);
        }
      }
    };
    auto total = [&](float s, bool weighted) {
      float ss = 0.f;
      uint32_t top = 0;
      for (int i = 0; i < rounds; ++i) {
        if (MANY) fetch(i * T * V);
        sums(i * T * V, s, weighted, ss, top);
      }
      return row_total<true>(ss, __uint_as_float(top), sh, turn++);
    };
    if (!MANY) {
      fetch(0);
      keep(0);
    }
    float2 of = total(1.f, true);
    float r = 1.f, s = 1.f;
    if (NORM) {
      float ms = of.x * a.inv_cols + a.eps;
      if (!in_range(ms)) {
        s = power_for(__float_as_uint(total(1.f, false).y), a.eps);
        of = total(s, true);
        ms = of.x * a.inv_cols + a.eps * s * s;
      }
      r = rsqrtf(ms);
    }
    const uint32_t top = __float_as_uint(of.y);
    for (int i = 0; i < rounds; ++i) {
      const int first = i * T * V;
      if (MANY) {
        fetch(first);
        keep(first);
      }
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int oct = first + v * T + t;
        float f[8], w[8];
        if (NORM) weight_of<VEC>(w, a.w, oct * 8, a.cols);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = NORM ? __fmul_rn(h[v].get(j) * s, w[j]) : h[v].get(j);
        if (NORM && a.fp8.values != nullptr) put_fp8(f, r, a, row, oct);
        if (want_int8 && oct < a.octs) put_int8(f, top, a.int8, row, oct, a.cols);
        if (NORM && a.y.p != nullptr) {
#pragma unroll
          for (int j = 0; j < 8; ++j) f[j] *= r;
          if (a.y_f32) store_floats<VEC>(f, reinterpret_cast<float*>(a.y.p) + row * a.y.ld, oct * 8, a.cols);
          else store_floats<VEC>(f, reinterpret_cast<bf16*>(a.y.p) + row * a.y.ld, oct * 8, a.cols);
        }
      }
    }
    if (want_int8 && t == 0) a.int8.scales[row] = int8_scale(top, r);
  }
}

// MANY: the sums of the weight's gradient are kept in the CTA's row of `parts`, where a thread finds its own again; else in registers
template <int V, bool MANY, typename S, typename G, bool VEC>
__global__ void __launch_bounds__(kNormMost) norm_bwd_kernel(const __grid_constant__ NormBwdArgs a) {
  __shared__ RowSums sh;
  grid_enter();
  const int t = threadIdx.x, T = blockDim.x;
  DropMask mask;
  mask.init(a.drop);
  const int rounds = MANY ? (a.octs + T * V - 1) / (T * V) : 1;
  float dw[V][8];
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int j = 0; j < 8; ++j) dw[v][j] = 0.f;
  float* const part = a.parts != nullptr ? a.parts + (size_t)blockIdx.x * a.octs * 8 : nullptr;
  uint32_t turn = 0;
  for (int row = blockIdx.x; row < a.rows; row += gridDim.x) {
    Eight<S> h[V], dh[V];
    Eight<G> dy[V];
    auto fetch = [&](int first, bool both) {
#pragma unroll
      for (int v = 0; v < V; ++v) load_eight<VEC>(h[v], reinterpret_cast<const S*>(a.h.p) + row * a.h.ld, (first + v * T + t) * 8, a.cols);
#pragma unroll
      for (int v = 0; v < V; ++v) load_eight<VEC>(dy[v], reinterpret_cast<const G*>(a.dy.p) + row * a.dy.ld, (first + v * T + t) * 8, a.cols);
      if (both && a.dh.p != nullptr) {
#pragma unroll
        for (int v = 0; v < V; ++v) load_eight<VEC>(dh[v], reinterpret_cast<const S*>(a.dh.p) + row * a.dh.ld, (first + v * T + t) * 8, a.cols);
      }
    };
    // of h times s: sum of squares, and of the weighted gradient along it
    auto total = [&](float s) {
      float ss = 0.f, dot = 0.f;
      for (int i = 0; i < rounds; ++i) {
        if (MANY) fetch(i * T * V, false);
#pragma unroll
        for (int v = 0; v < V; ++v) {
          float w[8];
          weight_of<VEC>(w, a.w, (i * T * V + v * T + t) * 8, a.cols);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float f = h[v].get(j) * s;
            ss += f * f;
            dot += dy[v].get(j) * w[j] * f;
          }
        }
      }
      return row_total<false>(ss, dot, sh, turn++);
    };
    if (!MANY) fetch(0, true);
    float2 of = total(1.f);
    float s = 1.f, ms = of.x * a.inv_cols + a.eps;
    if (!in_range(ms)) {
      uint32_t top = 0;
      for (int i = 0; i < rounds; ++i) {
        if (MANY) fetch(i * T * V, false);
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(h[v].get(j)) & 0x7fffffffu);
      }
      s = power_for(__float_as_uint(row_total<true>(0.f, __uint_as_float(top), sh, turn++).y), a.eps);
      of = total(s);
      ms = of.x * a.inv_cols + a.eps * s * s;
    }
    // (h times s) r is the normed row, and r s what its gradient is multiplied by
    const float r = rsqrtf(ms), out = r * s, along = of.y * r * a.inv_cols;
    for (int i = 0; i < rounds; ++i) {
      const int first = i * T * V;
      if (MANY) fetch(first, true);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int oct = first + v * T + t;
        float f[8], w[8];
        weight_of<VEC>(w, a.w, oct * 8, a.cols);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float hat = h[v].get(j) * s * r, g = dy[v].get(j);
          f[j] = out * (g * w[j] - hat * along);
          if (a.dh.p != nullptr) f[j] += dh[v].get(j);
          dw[v][j] += g * hat;
        }
        if (a.dr.p != nullptr) store_floats<VEC>(f, reinterpret_cast<S*>(a.dr.p) + row * a.dr.ld, oct * 8, a.cols);
        if (a.dx.p != nullptr) {
          mask.apply(f, row, oct);
          if (a.dx_f32) store_floats<VEC>(f, reinterpret_cast<float*>(a.dx.p) + row * a.dx.ld, oct * 8, a.cols);
          else store_floats<VEC>(f, reinterpret_cast<bf16*>(a.dx.p) + row * a.dx.ld, oct * 8, a.cols);
        }
        if (MANY) {
          if (part != nullptr && oct < a.octs) {
            Eight<float> sum;
            if (row == (int)blockIdx.x) sum.zero();
            else sum.load(part + oct * 8);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum.f[j] += dw[v][j];
            sum.store(part + oct * 8);
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) dw[v][j] = 0.f;
        }
      }
    }
  }
  if (!MANY && part != nullptr) {
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (v * T + t < a.octs) {
        Eight<float> sum;
        sum.round(dw[v]);
        sum.store(part + (v * T + t) * 8);
      }
  }
}

// The weight's gradient: the CTAs' parts, each of `width` columns, added in a fixed order.  32 columns a CTA, eight ranges of the parts.
__global__ void __launch_bounds__(256) norm_weight_kernel(const float* parts, int count, int cols, int width, float* __restrict__ dw) {
  __shared__ float sh[8][32];
  grid_enter();
  const int lane = threadIdx.x & 31, range = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
  float sum = 0.f;
  if (col < cols) {
    const float* from = parts + col;
#pragma unroll 8
    for (int i = range; i < count; i += 8) sum += from[(size_t)i * width];
  }
  sh[range][lane] = sum;
  __syncthreads();
  if (range == 0 && col < cols) {
#pragma unroll
    for (int i = 1; i < 8; ++i) sum += sh[i][lane];
    dw[col] = sum;
  }
}

// CTAs of a kernel that an SM holds, asked once for each number of warps, device and context
struct Residents {
  std::atomic<int> known[kMaxDevices][kNormMost / 32 + 1] = {};
};
cudaError_t resident_ctas(const void* kernel, Residents& r, int threads, int* ctas) {
  int dev = 0, sms = 0, n = 0;
  cudaError_t e;
  if ((e = cudaGetDevice(&dev)) != cudaSuccess || (e = sm_count(&sms)) != cudaSuccess) return e;
  if (dev < kMaxDevices) n = r.known[dev][threads / 32].load(std::memory_order_relaxed);
  if (n == 0) {
    if ((e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, 0)) != cudaSuccess) return e;
    if (n < 1) n = 1;
    if (dev < kMaxDevices) r.known[dev][threads / 32].store(n, std::memory_order_relaxed);
  }
  *ctas = n * sms;
  return cudaSuccess;
}

// Threads that take `octs` pieces, V each
int threads_for(int octs, int v) {
  const int t = (octs + v * 32 - 1) / (v * 32) * 32;
  return t < 32 ? 32 : t > kNormMost ? kNormMost : t;
}

template <int V, bool MANY, typename X, typename S, bool NORM, bool VEC>
cudaError_t go_fwd(const NormFwdArgs& a, cudaStream_t st) {
  static Residents residents;
  const int threads = threads_for(a.octs, V);
  int ctas = 0;
  const cudaError_t e = resident_ctas((const void*)norm_fwd_kernel<V, MANY, X, S, NORM, VEC>, residents, threads, &ctas);
  if (e != cudaSuccess) return e;
  return launch_kernel(norm_fwd_kernel<V, MANY, X, S, NORM, VEC>, a.rows < ctas ? a.rows : ctas, threads, 0, st, a);
}
template <typename X, typename S, bool NORM, bool VEC>
cudaError_t size_fwd(const NormFwdArgs& a, cudaStream_t st) {
  if (a.octs <= 128) return go_fwd<1, false, X, S, NORM, VEC>(a, st);
  if (a.octs <= 512) return go_fwd<2, false, X, S, NORM, VEC>(a, st);
  if (a.octs <= 4 * kNormMost) return go_fwd<4, false, X, S, NORM, VEC>(a, st);
  return go_fwd<2, true, X, S, NORM, VEC>(a, st);
}

template <int V, bool MANY, typename S, typename G, bool VEC>
cudaError_t go_bwd(const NormBwdArgs& a, float* dw, cudaStream_t st) {
  static Residents residents;
  const int threads = threads_for(a.octs, V);
  int ctas = 0;
  cudaError_t e = resident_ctas((const void*)norm_bwd_kernel<V, MANY, S, G, VEC>, residents, threads, &ctas);
  if (e != cudaSuccess) return e;
  if (ctas > kNormParts) ctas = kNormParts;
  if (ctas > a.rows) ctas = a.rows;
  if ((e = launch_kernel(norm_bwd_kernel<V, MANY, S, G, VEC>, ctas, threads, 0, st, a)) != cudaSuccess || dw == nullptr) return e;
  return launch_kernel(norm_weight_kernel, (a.cols + 31) / 32, 256, 0, st, a.parts, ctas, a.cols, a.octs * 8, dw);
}
template <typename S, typename G, bool VEC>
cudaError_t size_bwd(const NormBwdArgs& a, float* dw, cudaStream_t st) {
  if (a.octs <= 128) return go_bwd<1, false, S, G, VEC>(a, dw, st);
  if (a.octs <= 2 * kNormMost) return go_bwd<2, false, S, G, VEC>(a, dw, st);
  return go_bwd<1, true, S, G, VEC>(a, dw, st);
}

}  // namespace

cudaError_t launch_norm_fwd(NormFwdArgs a, bool x_f32, bool h_f32, cudaStream_t st) {
  a.octs = (a.cols + 7) / 8;
  a.inv_cols = 1.f / a.cols;
  const size_t size = h_f32 ? 4 : 2;
  const bool vec = rows_aligned(a.x, x_f32 ? 4 : 2) && rows_aligned(a.r, size) && rows_aligned(a.h, size) && rows_aligned(a.y, a.y_f32 ? 4 : 2) &&
                   (reinterpret_cast<uintptr_t>(a.w) & 15u) == 0;
  auto go = [&](auto aligned, auto any) { return vec ? aligned(a, st) : any(a, st); };
  if (x_f32) return h_f32 ? go(size_fwd<float, float, true, true>, size_fwd<float, float, true, false>) : go(size_fwd<float, bf16, true, true>, size_fwd<float, bf16, true, false>);
  return h_f32 ? go(size_fwd<bf16, float, true, true>, size_fwd<bf16, float, true, false>) : go(size_fwd<bf16, bf16, true, true>, size_fwd<bf16, bf16, true, false>);
}

cudaError_t launch_int8_quantize(const RowsArg& x, bool x_f32, int rows, int cols, const Int8Arg& out, cudaStream_t st) {
  NormFwdArgs a = {};
  a.x = x;
  a.int8 = out;
  a.rows = rows; a.cols = cols;
  a.octs = (cols + 7) / 8;
  const bool vec = rows_aligned(x, x_f32 ? 4 : 2);
  if (x_f32) return vec ? size_fwd<float, float, false, true>(a, st) : size_fwd<float, float, false, false>(a, st);
  return vec ? size_fwd<bf16, bf16, false, true>(a, st) : size_fwd<bf16, bf16, false, false>(a, st);
}

// a row of sums for each CTA
size_t norm_bwd_workspace_bytes(int rows, int cols) {
  return align_up((size_t)(rows < kNormParts ? rows : kNormParts) * (((size_t)cols + 7) / 8 * 8) * sizeof(float), 256);
}

cudaError_t launch_norm_bwd(NormBwdArgs a, bool h_f32, bool dy_f32, float* dw, float* parts, cudaStream_t st) {
  a.octs = (a.cols + 7) / 8;
  a.inv_cols = 1.f / a.cols;
  a.parts = dw != nullptr ? parts : nullptr;
  const size_t size = h_f32 ? 4 : 2;
  const bool vec = rows_aligned(a.h, size) && rows_aligned(a.dy, dy_f32 ? 4 : 2) && rows_aligned(a.dh, size) && rows_aligned(a.dr, size) &&
                   rows_aligned(a.dx, a.dx_f32 ? 4 : 2) && (reinterpret_cast<uintptr_t>(a.w) & 15u) == 0;
  auto go = [&](auto aligned, auto any) { return vec ? aligned(a, dw, st) : any(a, dw, st); };
  if (h_f32) return dy_f32 ? go(size_bwd<float, float, true>, size_bwd<float, float, false>) : go(size_bwd<float, bf16, true>, size_bwd<float, bf16, false>);
  return dy_f32 ? go(size_bwd<bf16, float, true>, size_bwd<bf16, float, false>) : go(size_bwd<bf16, bf16, true>, size_bwd<bf16, bf16, false>);
}

}  // namespace vsa2
