// The residual stream of a layer: h = residual + dropout(x) and y = h / sqrt(mean(h^2) + eps) * w, row by row, and back.
//   forward : y leaves in bf16 or fp32, in e4m3 with a power-of-two scale for each 128 values (the operand of vsa2_fp8_matmul), in int8 with a scale for the row (that of
//             vsa2_int8_matmul), or several of these; h is rounded to the stream's type first, and the norm is that of what is stored
//   backward: with r = 1 / sqrt(mean(h^2) + eps), g = w dy:  dh' = dh + r g - h r^3 mean(g h);  dx = dropout's part of dh';  dw = sum over the rows of dy h r
//   int8    : v = h w (for vsa2_int8_quantize a matrix' own values), s = max |v| / 127, value = v * (127 / max |v|) rounded to nearest, ties to even; the row's r is part of its
//             scale alone, so a value does not depend on how the sum of squares was rounded
// A CTA takes a row at a time, eight neighbouring elements in each of a thread's pieces.  Rows on 16-byte boundaries of up to 8192 elements (the ring kernels): each thread asks for its own
// pieces of the next rows ahead of time, in places of shared memory that are its own, so that memory is kept busy while a row's sums pass through the CTA's one barrier.
// Other rows come as they are needed: of up to 8192 elements they stay in registers, longer ones (MANY) are read twice, the second time from L2.  Bound by memory.
#include "fp8_values.cuh"
#include "rows.cuh"

namespace vsa2 {

namespace {

constexpr int kNormMost = 512;       // threads of a CTA at most
constexpr int kNormParts = 1184;     // most CTAs of the backward, each with its own partial sums of the weight's gradient (eight for each of 148 SMs)
constexpr int kAhead = 2;            // rows that a thread of the ring kernels has asked for beyond the one it works on
constexpr int kRingCols = 8192;      // their longest rows
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
// the larger magnitude; NaN where one is
__device__ __forceinline__ float larger(float top, float a, float b) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(top), "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float warp_largest(float v) {
  float r;
  asm volatile("redux.sync.max.abs.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
// Sum of `sum` and of `other` (MAX: the largest magnitude) over the CTA, the same bits in every thread
template <bool MAX>
__device__ __forceinline__ float2 row_total(float sum, float other, RowSums& sh, uint32_t parity) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (!MAX) other += __shfl_xor_sync(0xffffffffu, other, o);
  }
  if (MAX) other = warp_largest(other);
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
  if (MAX) other = warp_largest(other);
  else other = __shfl_sync(0xffffffffu, other, 0);
  return make_float2(sum, other);
}

// Weights of elements i .. i+7 (null: ones), zeros behind the row.  VEC: whole pieces on 16-byte boundaries
template <bool VEC>
__device__ __forceinline__ void weight_of(float2 (&w)[4], const float* from, int i, int cols) {
  if (VEC && from != nullptr && i < cols) {
    const float4 a = reinterpret_cast<const float4*>(from + i)[0], b = reinterpret_cast<const float4*>(from + i)[1];
    w[0] = make_float2(a.x, a.y); w[1] = make_float2(a.z, a.w);
    w[2] = make_float2(b.x, b.y); w[3] = make_float2(b.z, b.w);
  } else {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = from == nullptr ? 1.f : !VEC && i + j < cols ? from[i + j] : 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = make_float2(v[2 * j], v[2 * j + 1]);
  }
}
// times a power of two
template <typename S>
__device__ __forceinline__ void rescale(Eight<S>& e, float s) {
  float f[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) f[j] = e.get(j) * s;
  e.round(f);
}
template <typename S>
__device__ __forceinline__ float largest_of(const Eight<S>& e, float top) {
#pragma unroll
  for (int i = 0; i < 4; ++i) top = larger(top, e.pair(i).x, e.pair(i).y);
  return top;
}
// the row's sum of squares (two sums) and its largest |h w|
template <bool NORM, bool INT8, typename S>
__device__ __forceinline__ void add_sums(const Eight<S>& h, const float2 (&w)[4], float2& ss, float& top) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 p = h.pair(i);
    if (NORM) ss = __ffma2_rn(p, p, ss);
    if (INT8) {
      const float2 v = NORM ? __fmul2_rn(p, w[i]) : p;
      top = larger(top, v.x, v.y);
    }
  }
}

// ---- the forms that y leaves in
// e4m3: the 16 threads of a block of 128 find its scale together.  (By whole warps; pieces behind the row are zeros.)
__device__ __forceinline__ void put_fp8(const float2 (&y)[4], const NormFwdArgs& a, int row, int oct) {
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) top = larger(top, y[i].x, y[i].y);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) {
    const float other = __shfl_xor_sync(0xffffffffu, top, o);
    top = larger(top, other, other);
  }
  uint32_t bits = __float_as_uint(top);
  const bool odd = __any_sync(0xffffffffu, bits >= kInf);
  if (odd) {      // (rare) the largest of what is finite
    bits = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (finite_bits(y[i].x)) bits = max(bits, __float_as_uint(y[i].x) & 0x7fffffffu);
      if (finite_bits(y[i].y)) bits = max(bits, __float_as_uint(y[i].y) & 0x7fffffffu);
    }
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) bits = max(bits, __shfl_xor_sync(0xffffffffu, bits, o));
  }
  if (oct >= a.octs) return;
  const uint32_t byte = scale_byte(bits);
  const float inv = inverse_scale(byte);
  float f[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 v = __fmul2_rn(y[i], make_float2(inv, inv));
    f[2 * i] = !odd || finite_bits(y[i].x) ? v.x : __uint_as_float(0x7fffffffu);
    f[2 * i + 1] = !odd || finite_bits(y[i].y) ? v.y : __uint_as_float(0x7fffffffu);
  }
  put8(a.fp8.values + row * a.fp8.ld, oct * 8, a.cols, e4m3x4(f[0], f[1], f[2], f[3]), e4m3x4(f[4], f[5], f[6], f[7]));
  if ((oct & 15) == 0) put_scale(a.fp8.scales, a.rows, row, oct >> 4, (a.octs + 15) >> 4, byte);
}
// int8: the product is rounded once, then to a whole number by an addition whose last bit is one (1.5 * 2^23; |product| is 127 and a little at most).  (One at a time: the assembler makes
// one operation of a packed product and a packed sum behind it, also of mul.rn and add.rn, which rounds once, and numbers half way between two come out on the other side.)
__device__ __forceinline__ uint32_t int8_bits(float v, float factor) { return __float_as_uint(__fadd_rn(__fmul_rn(v, factor), 12582912.f)); }
__device__ __forceinline__ uint32_t int8x4(float2 a, float2 b, float factor) {
  return __byte_perm(__byte_perm(int8_bits(a.x, factor), int8_bits(a.y, factor), 0x0040), __byte_perm(int8_bits(b.x, factor), int8_bits(b.y, factor), 0x0040), 0x5410);
}
// What a row's max |v| stands for: what its values are multiplied by, and its scale.  A row that holds something that is not finite has no scale: zeros (times zero, plus a zero
// in place of the value), and a scale that makes its products NaN
__device__ __forceinline__ float int8_factor(float top) { return __fdiv_rn(127.f, fmaxf(top, kInt8Least)); }
__device__ __forceinline__ float int8_scale(float top, float r) {
  return __float_as_uint(top) < kInf ? __fdiv_rn(fmaxf(top, kInt8Least), 127.f) * r : __uint_as_float(0x7fffffffu);
}
// A piece of a row in every form that is wanted: h (or x), its weights, 1 / sqrt, the row's max |v| and what it is multiplied by
template <bool NORM, bool VEC, typename S>
__device__ __forceinline__ void put_piece(const Eight<S>& h, const float2 (&w)[4], float r, float top, float factor, bool int8, const NormFwdArgs& a, int row, int oct) {
  float2 v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = NORM ? __fmul2_rn(h.pair(i), w[i]) : h.pair(i);
  if (int8 && oct < a.octs) {
    const bool fine = __float_as_uint(top) < kInf;
    put8(reinterpret_cast<unsigned char*>(a.int8.values) + row * a.int8.ld, oct * 8, a.cols, fine ? int8x4(v[0], v[1], factor) : 0u, fine ? int8x4(v[2], v[3], factor) : 0u);
  }
  if (!NORM) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __fmul2_rn(v[i], make_float2(r, r));
  if (a.fp8.values != nullptr) put_fp8(v, a, row, oct);
  if (a.y.p != nullptr) {
    const float f[8] = {v[0].x, v[0].y, v[1].x, v[1].y, v[2].x, v[2].y, v[3].x, v[3].y};
    if (a.y_f32) store_floats<VEC>(f, reinterpret_cast<float*>(a.y.p) + row * a.y.ld, oct * 8, a.cols);
    else store_floats<VEC>(f, reinterpret_cast<bf16*>(a.y.p) + row * a.y.ld, oct * 8, a.cols);
  }
}
// h of a piece: x through the dropout, plus the residual, rounded to the stream's type
template <typename X, typename S>
__device__ __forceinline__ void combine(Eight<S>& h, const Eight<X>& x, const Eight<S>& r, bool residual, const DropMask& mask, int row, int oct) {
  float f[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) f[j] = x.get(j);
  mask.apply(f, row, oct);
  if (residual) add_eight(f, r);
  h.round(f);
}

// ---- rows on 16-byte boundaries: pieces on their way, each in 16-byte places `threads` apart that one thread writes and reads
__device__ __forceinline__ void ask(uint32_t to, const void* from, bool there) {      // (not there: zeros)
  asm volatile("cp.async.ca.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
}
template <typename T>
__device__ __forceinline__ void ask_eight(uint32_t to, uint32_t apart, const T* row, int oct, bool there) {
  const T* from = row + (there ? oct * 8 : 0);
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) ask(to + i * apart, reinterpret_cast<const char*>(from) + 16 * i, there);
}
__device__ __forceinline__ void asked() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void arrived() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }
__device__ __forceinline__ void take(Eight<bf16>& e, const unsigned char* from, uint32_t) {
  const uint4 v = *reinterpret_cast<const uint4*>(from);
  e.u[0] = v.x; e.u[1] = v.y; e.u[2] = v.z; e.u[3] = v.w;
}
__device__ __forceinline__ void take(Eight<float>& e, const unsigned char* from, uint32_t apart) {
  const float4 a = *reinterpret_cast<const float4*>(from), b = *reinterpret_cast<const float4*>(from + apart);
  e.f[0] = a.x; e.f[1] = a.y; e.f[2] = a.z; e.f[3] = a.w; e.f[4] = b.x; e.f[5] = b.y; e.f[6] = b.z; e.f[7] = b.w;
}

template <int V, typename X, typename S, bool NORM, bool INT8>
__global__ void __launch_bounds__(kNormMost, 2) norm_fwd_ring_kernel(const __grid_constant__ NormFwdArgs a) {
  extern __shared__ __align__(16) unsigned char ring[];
  __shared__ RowSums sh;
  constexpr int XP = sizeof(X) / 2, SP = sizeof(S) / 2;      // 16-byte places of a piece
  grid_enter();
  const int t = threadIdx.x, T = blockDim.x;
  const uint32_t apart = T * 16, slot = V * (XP + SP) * apart;
  unsigned char* const mine = ring + t * 16;
  const uint32_t to = (uint32_t)__cvta_generic_to_shared(mine);
  const bool residual = a.r.p != nullptr;
  auto ask_row = [&](int row, int s) {
    if (row < a.rows) {
      const X* xp = reinterpret_cast<const X*>(a.x.p) + row * a.x.ld;
      const S* rp = reinterpret_cast<const S*>(a.r.p) + row * a.r.ld;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int oct = v * T + t;
        ask_eight(to + s * slot + v * XP * apart, apart, xp, oct, oct < a.octs);
        if (residual) ask_eight(to + s * slot + (V * XP + v * SP) * apart, apart, rp, oct, oct < a.octs);
      }
    }
    asked();
  };
#pragma unroll
  for (int s = 0; s < kAhead; ++s) ask_row(blockIdx.x + s * gridDim.x, s);
  DropMask mask;
  mask.init(a.drop);
  float2 w[V][4];
  if (NORM) {
#pragma unroll
    for (int v = 0; v < V; ++v) weight_of<true>(w[v], a.w, (v * T + t) * 8, a.cols);
  }
  uint32_t turn = 0;
  int s = 0;
  for (int row = blockIdx.x; row < a.rows; row += gridDim.x) {
    // (the place behind the others is free: this thread has read it, and only it does)
    ask_row(row + kAhead * gridDim.x, s == 0 ? kAhead : s - 1);
    arrived<kAhead>();
    Eight<S> h[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const unsigned char* from = mine + s * slot;
      Eight<X> x;
      Eight<S> r;
      take(x, from + v * XP * apart, apart);
      if (residual) take(r, from + (V * XP + v * SP) * apart, apart);
      combine(h[v], x, r, residual, mask, row, v * T + t);
    }
    s = s == kAhead ? 0 : s + 1;
    if (NORM && a.h.p != nullptr) {
#pragma unroll
      for (int v = 0; v < V; ++v) store_eight<true>(h[v], reinterpret_cast<S*>(a.h.p) + row * a.h.ld, (v * T + t) * 8, a.cols);
    }
    float r = 1.f, top = 0.f, eps = a.eps;
#pragma unroll 1
    for (bool again = false;; again = true) {
      float2 ss = make_float2(0.f, 0.f);
      top = 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v) add_sums<NORM, INT8>(h[v], w[v], ss, top);
      const float2 of = row_total<true>(ss.x + ss.y, top, sh, turn++);
      top = of.y;
      if constexpr (NORM) {
        const float ms = of.x * a.inv_cols + eps;
        r = rsqrtf(ms);
        if (in_range(ms) || again) break;
        float size = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) size = largest_of(h[v], size);
        const float power = power_for(__float_as_uint(row_total<true>(0.f, size, sh, turn++).y), eps);
#pragma unroll
        for (int v = 0; v < V; ++v) rescale(h[v], power);
        eps = eps * power * power;
      } else {
        break;
      }
    }
    const float factor = INT8 ? int8_factor(top) : 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) put_piece<NORM, true>(h[v], w[v], r, top, factor, INT8, a, row, v * T + t);
    if (INT8 && t == 0) a.int8.scales[row] = int8_scale(top, r);
  }
  arrived<0>();
}

// Any rows.  V: pieces of eight elements a thread (MANY: as many as it takes, in a loop); NORM: else the int8 form of x as it is
template <int V, bool MANY, typename X, typename S, bool NORM, bool VEC>
__global__ void __launch_bounds__(kNormMost, 1) norm_fwd_kernel(const __grid_constant__ NormFwdArgs a) {
  __shared__ RowSums sh;
  grid_enter();
  const int t = threadIdx.x, T = blockDim.x;
  DropMask mask;
  mask.init(a.drop);
  const int rounds = MANY ? (a.octs + T * V - 1) / (T * V) : 1;
  const bool int8 = a.int8.values != nullptr;
  uint32_t turn = 0;
  for (int row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const X* const xp = reinterpret_cast<const X*>(a.x.p) + row * a.x.ld;
    const S* const rp = reinterpret_cast<const S*>(a.r.p) + row * a.r.ld;
    Eight<S> h[V];
    float power = 1.f;
    auto fetch = [&](int first) {      // h of the pieces first + t, first + t + T, ..
      Eight<X> x[V];
#pragma unroll
      for (int v = 0; v < V; ++v) load_eight<VEC>(x[v], xp, (first + v * T + t) * 8, a.cols);
      if (a.r.p != nullptr) {
#pragma unroll
        for (int v = 0; v < V; ++v) load_eight<VEC>(h[v], rp, (first + v * T + t) * 8, a.cols);
      }
#pragma unroll
      for (int v = 0; v < V; ++v) combine(h[v], x[v], h[v], a.r.p != nullptr, mask, row, first + v * T + t);
    };
    auto keep = [&](int first) {
      if (!NORM || a.h.p == nullptr) return;
#pragma unroll
      for (int v = 0; v < V; ++v) store_eight<VEC>(h[v], reinterpret_cast<S*>(a.h.p) + row * a.h.ld, (first + v * T + t) * 8, a.cols);
    };
    auto apply_power = [&] {
      if (power == 1.f) return;
#pragma unroll
      for (int v = 0; v < V; ++v) rescale(h[v], power);
    };
    if (!MANY) {
      fetch(0);
      keep(0);
    }
    float r = 1.f, top = 0.f, eps = a.eps;
#pragma unroll 1
    for (bool again = false;; again = true) {
      float2 ss = make_float2(0.f, 0.f);
      float size = 0.f;
      top = 0.f;
#pragma unroll 1
      for (int i = 0; i < rounds; ++i) {
        const int first = i * T * V;
        if (MANY) {
          fetch(first);
          apply_power();
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
          float2 w[4];
          if (NORM) weight_of<VEC>(w, a.w, (first + v * T + t) * 8, a.cols);
          if (int8) add_sums<NORM, true>(h[v], w, ss, top);
          else add_sums<NORM, false>(h[v], w, ss, top);
          if (NORM) size = largest_of(h[v], size);
        }
      }
      const float2 of = row_total<true>(ss.x + ss.y, top, sh, turn++);
      top = of.y;
      if constexpr (NORM) {
        const float ms = of.x * a.inv_cols + eps;
        r = rsqrtf(ms);
        if (in_range(ms) || again) break;
        power = power_for(__float_as_uint(row_total<true>(0.f, size, sh, turn++).y), eps);
        if (!MANY) apply_power();
        eps = eps * power * power;
      } else {
        break;
      }
    }
    const float factor = int8 ? int8_factor(top) : 0.f;
#pragma unroll 1
    for (int i = 0; i < rounds; ++i) {
      const int first = i * T * V;
      if (MANY) {
        fetch(first);
        keep(first);
        apply_power();
      }
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float2 w[4];
        if (NORM) weight_of<VEC>(w, a.w, (first + v * T + t) * 8, a.cols);
        put_piece<NORM, VEC>(h[v], w, r, top, factor, int8, a, row, first + v * T + t);
      }
    }
    if (int8 && t == 0) a.int8.scales[row] = int8_scale(top, r);
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
          float2 w[4];
          weight_of<VEC>(w, a.w, (i * T * V + v * T + t) * 8, a.cols);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float f = h[v].get(j) * s;
            ss += f * f;
            dot += dy[v].get(j) * (j & 1 ? w[j / 2].y : w[j / 2].x) * f;
          }
        }
      }
      return row_total<false>(ss, dot, sh, turn++);
    };
    if (!MANY) fetch(0, true);
    float2 of = total(1.f);
    float s = 1.f, ms = of.x * a.inv_cols + a.eps;
    if (!in_range(ms)) {
      float top = 0.f;
      for (int i = 0; i < rounds; ++i) {
        if (MANY) fetch(i * T * V, false);
#pragma unroll
        for (int v = 0; v < V; ++v) top = largest_of(h[v], top);
      }
      s = power_for(__float_as_uint(row_total<true>(0.f, top, sh, turn++).y), a.eps);
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
        float f[8];
        float2 w[4];
        weight_of<VEC>(w, a.w, oct * 8, a.cols);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float hat = h[v].get(j) * s * r, g = dy[v].get(j);
          f[j] = out * (g * (j & 1 ? w[j / 2].y : w[j / 2].x) - hat * along);
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

// CTAs of a kernel that the device holds, asked once for each number of warps and device (with the same shared memory each time); it is allowed its shared memory first
struct Residents {
  KernelAttr attr;
  std::atomic<int> known[kMaxDevices][kNormMost / 32 + 1] = {};
};
cudaError_t resident_ctas(const void* kernel, Residents& r, int threads, size_t smem, int* ctas) {
  int dev = 0, sms = 0, n = 0;
  cudaError_t e;
  if ((e = cudaGetDevice(&dev)) != cudaSuccess || (e = sm_count(&sms)) != cudaSuccess) return e;
  if (smem > 0 && (e = prepare_kernel(kernel, r.attr, smem)) != cudaSuccess) return e;
  if (dev < kMaxDevices) n = r.known[dev][threads / 32].load(std::memory_order_relaxed);
  if (n == 0) {
    if ((e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, smem)) != cudaSuccess) return e;
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

template <int V, typename X, typename S, bool NORM, bool INT8>
cudaError_t go_fwd_ring(const NormFwdArgs& a, cudaStream_t st) {
  static Residents residents;
  const int threads = threads_for(a.octs, V);
  const size_t smem = (size_t)(kAhead + 1) * V * threads * 8 * (sizeof(X) + sizeof(S));
  int ctas = 0;
  const cudaError_t e = resident_ctas((const void*)norm_fwd_ring_kernel<V, X, S, NORM, INT8>, residents, threads, smem, &ctas);
  if (e != cudaSuccess) return e;
  return launch_kernel(norm_fwd_ring_kernel<V, X, S, NORM, INT8>, a.rows < ctas ? a.rows : ctas, threads, smem, st, a);
}
template <int V, bool MANY, typename X, typename S, bool NORM, bool VEC>
cudaError_t go_fwd(const NormFwdArgs& a, cudaStream_t st) {
  static Residents residents;
  const int threads = threads_for(a.octs, V);
  int ctas = 0;
  const cudaError_t e = resident_ctas((const void*)norm_fwd_kernel<V, MANY, X, S, NORM, VEC>, residents, threads, 0, &ctas);
  if (e != cudaSuccess) return e;
  return launch_kernel(norm_fwd_kernel<V, MANY, X, S, NORM, VEC>, a.rows < ctas ? a.rows : ctas, threads, 0, st, a);
}
template <typename X, typename S, bool NORM>
cudaError_t size_fwd(const NormFwdArgs& a, bool vec, cudaStream_t st) {
  const bool many = a.cols > 2 * 8 * kNormMost;
  if (!vec) return many ? go_fwd<2, true, X, S, NORM, false>(a, st) : go_fwd<2, false, X, S, NORM, false>(a, st);
  if (a.cols > kRingCols) return go_fwd<2, true, X, S, NORM, true>(a, st);
  if (!NORM) return a.octs <= 128 ? go_fwd_ring<1, X, S, NORM, true>(a, st) : go_fwd_ring<2, X, S, NORM, true>(a, st);
  if (a.int8.values != nullptr) return a.octs <= 128 ? go_fwd_ring<1, X, S, true, true>(a, st) : go_fwd_ring<2, X, S, true, true>(a, st);
  return a.octs <= 128 ? go_fwd_ring<1, X, S, true, false>(a, st) : go_fwd_ring<2, X, S, true, false>(a, st);
}

template <int V, bool MANY, typename S, typename G, bool VEC>
cudaError_t go_bwd(const NormBwdArgs& a, float* dw, cudaStream_t st) {
  static Residents residents;
  const int threads = threads_for(a.octs, V);
  int ctas = 0;
  cudaError_t e = resident_ctas((const void*)norm_bwd_kernel<V, MANY, S, G, VEC>, residents, threads, 0, &ctas);
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
  const bool vec = a.cols % 8 == 0 && rows_aligned(a.x, x_f32 ? 4 : 2) && rows_aligned(a.r, size) && rows_aligned(a.h, size) &&
                   rows_aligned(a.y, a.y_f32 ? 4 : 2) && (reinterpret_cast<uintptr_t>(a.w) & 15u) == 0;
  if (x_f32) return h_f32 ? size_fwd<float, float, true>(a, vec, st) : size_fwd<float, bf16, true>(a, vec, st);
  return h_f32 ? size_fwd<bf16, float, true>(a, vec, st) : size_fwd<bf16, bf16, true>(a, vec, st);
}

cudaError_t launch_int8_quantize(const RowsArg& x, bool x_f32, int rows, int cols, const Int8Arg& out, cudaStream_t st) {
  NormFwdArgs a = {};
  a.x = x;
  a.int8 = out;
  a.rows = rows; a.cols = cols;
  a.octs = (cols + 7) / 8;
  const bool vec = cols % 8 == 0 && rows_aligned(x, x_f32 ? 4 : 2);
  return x_f32 ? size_fwd<float, float, false>(a, vec, st) : size_fwd<bf16, bf16, false>(a, vec, st);
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
  const bool vec = a.cols % 8 == 0 && rows_aligned(a.h, size) && rows_aligned(a.dy, dy_f32 ? 4 : 2) && rows_aligned(a.dh, size) && rows_aligned(a.dr, size) &&
                   rows_aligned(a.dx, a.dx_f32 ? 4 : 2) && (reinterpret_cast<uintptr_t>(a.w) & 15u) == 0;
  auto go = [&](auto aligned, auto any) { return vec ? aligned(a, dw, st) : any(a, dw, st); };
  if (h_f32) return dy_f32 ? go(size_bwd<float, float, true>, size_bwd<float, float, false>) : go(size_bwd<float, bf16, true>, size_bwd<float, bf16, false>);
  return dy_f32 ? go(size_bwd<bf16, float, true>, size_bwd<bf16, float, false>) : go(size_bwd<bf16, bf16, true>, size_bwd<bf16, bf16, false>);
}

}  // namespace vsa2
