// The residual stream of a layer: h = residual + dropout(x) and y = h / sqrt(mean(h^2) + eps) * w, row by row, and back.
//   forward : y leaves in bf16 or fp32, in e4m3 with a power-of-two scale for each 128 values (the operand of vsa2_fp8_matmul), in int8 with a scale for the row (that of
//             vsa2_int8_matmul), or several of these; h is rounded to the stream's type first, and the norm is that of what is stored
//   backward: with r = 1 / sqrt(mean(h^2) + eps), g = w dy:  dh' = dh + r g - h r^3 mean(g h);  dx = dropout's part of dh';  dw = sum over the rows of dy h r
//   int8    : v = h w (for vsa2_int8_quantize a matrix' own values), s = max |v| / 127, value = v * (127 / max |v|) rounded to nearest, ties to even; the row's r is part of its
//             scale alone, so a value does not depend on how the sum of squares was rounded
// A CTA takes a row at a time, eight neighbouring elements in each of a thread's pieces; the row is read once and stays in registers while its sums pass through the CTA's one barrier.
// (Rows of more than 16,384 elements forward, 8192 backward and where they lie anywhere, MANY, are read twice, the second time from L2.)  Bound by memory, and in runs of seconds by the power limit beside it:
// 75600 x 5120 with residual to e4m3 424 - 440 us (6.2 - 6.4 TB/s; 412 in short runs), 65972 x 1536 fp32 with dropout to bf16 and e4m3 207 - 213 us (6.2 - 6.4), its backward 255 - 275 us
// (5.9 - 6.4), int8 of 15360 x 5120 38 us (6.2).  With few rows it is the latency of one: a token to int8 3.5 us, 2048 x 1536 backward 11.8 - 12.8 us in two kernels.  Rows of few elements leave
// a warp to a CTA, of which an SM takes 32: 62500 x 64 bf16 25 us forward (5 of memory), 54 backward.
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

struct RowSums {      // double-buffered by the row's parity: one barrier a row.  Zeros behind the CTA's warps
  float sum[2][kNormMost / 32], other[2][kNormMost / 32];
  __device__ __forceinline__ void init() {
    if (threadIdx.x < 32) sum[threadIdx.x >> 4][threadIdx.x & 15] = other[threadIdx.x >> 4][threadIdx.x & 15] = 0.f;
    __syncthreads();
  }
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
// Over the CTA, the same bits in every thread: the sum of `sum`, where it is wanted (SUM), and of `other` the largest magnitude (MAX: 1), the sum (2) or nothing (0)
template <bool SUM, int MAX>
__device__ __forceinline__ float2 row_total(float sum, float other, RowSums& sh, uint32_t parity) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  parity &= 1;
  if constexpr (SUM && MAX == 2) {
    // (the lower half of the warp goes on with one sum, the upper half with the other)
    const bool upper = lane & 16;
    float mine = upper ? other : sum;
    mine += __shfl_xor_sync(0xffffffffu, upper ? sum : other, 16);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
    if (warps == 1) return make_float2(__shfl_sync(0xffffffffu, mine, 0), __shfl_sync(0xffffffffu, mine, 16));
    if ((lane & 15) == 0) (upper ? sh.other : sh.sum)[parity][warp] = mine;
  } else {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
      if (SUM) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (MAX == 1) other = warp_largest(other);
    if (warps == 1) return make_float2(sum, other);
    if (lane == 0) {
      if (SUM) sh.sum[parity][warp] = sum;
      if (MAX) sh.other[parity][warp] = other;
    }
  }
  __syncthreads();
  sum = other = 0.f;
#pragma unroll 1
  for (int i = 0; i < warps; i += 4) {
    if (SUM) {
      const float4 v = *reinterpret_cast<const float4*>(&sh.sum[parity][i]);
      sum += (v.x + v.y) + (v.z + v.w);
    }
    if (MAX) {
      const float4 v = *reinterpret_cast<const float4*>(&sh.other[parity][i]);
      if (MAX == 1) other = larger(larger(other, v.x, v.y), v.z, v.w);
      else other += (v.x + v.y) + (v.z + v.w);
    }
  }
  return make_float2(sum, other);
}

// Weights of elements i .. i+7 (null: ones); any behind the row, where all else is zero
__device__ __forceinline__ void weights_at(float2 (&w)[4], const float* p) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  w[0] = make_float2(a.x, a.y); w[1] = make_float2(a.z, a.w);
  w[2] = make_float2(b.x, b.y); w[3] = make_float2(b.z, b.w);
}
__device__ const __align__(16) float kOnes[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
template <int LIE>
__device__ __forceinline__ void weight_of(float2 (&w)[4], const float* from, int i, int cols) {
  if (LIE != ROWS_ANY) {
    weights_at(w, element(from != nullptr ? from : kOnes, from != nullptr && (LIE == ROWS_WHOLE || i < cols) ? i : 0));
  } else if (from == nullptr || i >= cols || (i + 8 <= cols && (reinterpret_cast<uintptr_t>(from) & 15u) == 0)) {
    weights_at(w, from == nullptr || i >= cols ? kOnes : element(from, i));
  } else {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = i + j < cols ? from[i + j] : 1.f;
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
// .. and, backward, the sum of the weighted gradient along h
template <typename S, typename G>
__device__ __forceinline__ void add_dots(const Eight<S>& h, const Eight<G>& dy, const float2 (&w)[4], float2& ss, float2& dot) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 p = h.pair(i);
    ss = __ffma2_rn(p, p, ss);
    dot = __ffma2_rn(__fmul2_rn(dy.pair(i), w[i]), p, dot);
  }
}
// A piece's gradient: out (w dy - hat along) (+ dh) with hat = h r, and out = r but for a row that was taken times a power of two; the weight's gets dy hat
template <typename S, typename G>
__device__ __forceinline__ void gradient_piece(float (&f)[8], const Eight<S>& h, const Eight<G>& dy, const Eight<S>& dh, bool stream, const float2 (&w)[4], float2 (&dw)[4], float r,
                                               float out, float along) {
  const float2 out2 = make_float2(out, out), by = make_float2(-along * r * out, -along * r * out);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 p = h.pair(i), g = dy.pair(i), t = __fmul2_rn(g, out2);
    const float2 v = __ffma2_rn(t, w[i], stream ? __ffma2_rn(p, by, dh.pair(i)) : __fmul2_rn(p, by));
    if (out == r) dw[i] = __ffma2_rn(t, p, dw[i]);
    else dw[i] = __ffma2_rn(g, __fmul2_rn(p, make_float2(r, r)), dw[i]);
    f[2 * i] = v.x;
    f[2 * i + 1] = v.y;
  }
}

// ---- the forms that y leaves in
// e4m3: the 16 threads of a block of 128 find its scale together (whole warps; pieces behind the row are zeros): of v times r, whose largest magnitude is the largest |v| times r, as
// rounding keeps the order, and whose product with a power of two is that of v with r times the power.
__device__ __forceinline__ uint2 fp8_piece(const float2 (&v)[4], float r, uint32_t& byte) {
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) top = larger(top, v[i].x, v[i].y);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) {
    const float other = __shfl_xor_sync(0xffffffffu, top, o);
    top = larger(top, other, other);
  }
  byte = scale_byte(__float_as_uint(top * r) & 0x7fffffffu);
  // (what is not finite, and scales whose product with r could leave fp32's range, zeros among them: rare)
  const bool odd = __any_sync(0xffffffffu, byte - 32u > 168u);
  float f[8];
  if (odd) {      // the largest of what is finite
    uint32_t bits = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (finite_bits(v[i].x * r)) bits = max(bits, __float_as_uint(v[i].x * r) & 0x7fffffffu);
      if (finite_bits(v[i].y * r)) bits = max(bits, __float_as_uint(v[i].y * r) & 0x7fffffffu);
    }
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) bits = max(bits, __shfl_xor_sync(0xffffffffu, bits, o));
    byte = scale_byte(bits);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = scaled<true>(v[i].x * r, inverse_scale(byte));
      f[2 * i + 1] = scaled<true>(v[i].y * r, inverse_scale(byte));
    }
  } else {
    const float by = inverse_scale(byte) * r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 p = __fmul2_rn(v[i], make_float2(by, by));
      f[2 * i] = p.x;
      f[2 * i + 1] = p.y;
    }
  }
  return make_uint2(e4m3x4(f[0], f[1], f[2], f[3]), e4m3x4(f[4], f[5], f[6], f[7]));
}
// int8: the product is rounded once, then to a whole number by an addition whose last bit is one (1.5 * 2^23; |product| is 127 and a little at most).  (One at a time: the assembler makes
// one operation of a packed product and a packed sum behind it, also of mul.rn and add.rn, which rounds once, and numbers half way between two come out on the other side.)
__device__ __forceinline__ uint32_t int8_bits(float v, float factor) { return __float_as_uint(__fadd_rn(__fmul_rn(v, factor), 12582912.f)); }
__device__ __forceinline__ uint32_t int8x4(float2 a, float2 b, float factor) {
  return __byte_perm(__byte_perm(int8_bits(a.x, factor), int8_bits(a.y, factor), 0x0040), __byte_perm(int8_bits(b.x, factor), int8_bits(b.y, factor), 0x0040), 0x5410);
}
// What a row's max |v| stands for: what its values are multiplied by, and its scale.  A row that holds something that is not finite has no scale: zeros, and a scale that makes its
// products NaN
__device__ __forceinline__ float int8_factor(float top) { return __fdiv_rn(127.f, fmaxf(top, kInt8Least)); }
__device__ __forceinline__ float int8_scale(float top, float r) {
  return __float_as_uint(top) < kInf ? __fdiv_rn(fmaxf(top, kInt8Least), 127.f) * r : __uint_as_float(0x7fffffffu);
}
__device__ __forceinline__ uint2 int8_piece(const float2 (&v)[4], float top, float factor) {
  const bool fine = __float_as_uint(top) < kInf;
  return make_uint2(fine ? int8x4(v[0], v[1], factor) : 0u, fine ? int8x4(v[2], v[3], factor) : 0u);
}
// eight bytes of a row of `cols`, at place i
template <int LIE>
__device__ __forceinline__ void put_bytes(uint2 q, unsigned char* row, int i, int cols) {
  if (LIE == ROWS_WHOLE) *reinterpret_cast<uint2*>(element(row, i)) = q;
  else if (i < cols) put8(row, i, cols, q.x, q.y);
}
// Pieces of fp32 numbers on their way to a row of another type, one after the other
template <typename T>
struct Outgoing {
  Eight<T> before;
  template <int LIE, int V>
  __device__ __forceinline__ void store(const float (&f)[8], int v, T* row, int i, int cols) {
    Eight<T> e;
    e.round(f);
    store_eight<LIE, V>(e, v > 0 ? before : e, v, row, i, cols);
    if (LIE == ROWS_ANY) before = e;
  }
};
// h of a piece: x through the dropout (`words`: the generator's, where there is one), plus the residual (in h), rounded to the stream's type
template <typename X, typename S>
__device__ __forceinline__ void combine(Eight<S>& h, const Eight<X>& x, bool residual, const DropMask& mask, const uint32_t (&words)[4]) {
  float f[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) f[j] = x.get(j);
  if (mask.limit != 0) mask.keep(f, words);
  if (residual) add_eight(f, h);
  h.round(f);
}
// A sum of two bf16 numbers rounded once is their fp32 sum rounded: where that is not exact the smaller one is less than 2^-16 of the other, far from half a step
__device__ __forceinline__ void combine_bf16(Eight<bf16>& h, const Eight<bf16>& x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 sum = __hadd2_rn(*reinterpret_cast<const __nv_bfloat162*>(&h.u[i]), *reinterpret_cast<const __nv_bfloat162*>(&x.u[i]));
    h.u[i] = *reinterpret_cast<const uint32_t*>(&sum);
  }
}

// V: pieces of eight elements a thread, two or four (MANY: as many as it takes, in a loop); NORM: else the int8 form of x as it is
template <int V, bool MANY, typename X, typename S, bool NORM, int LIE, bool DROP>
__global__ void __launch_bounds__(kNormMost, 2) norm_fwd_kernel(const __grid_constant__ NormFwdArgs a) {
  __shared__ __align__(16) RowSums sh;
  sh.init();
  grid_enter();
  const int t = threadIdx.x, T = blockDim.x, mine = (t >> 5) * (32 * V) + (t & 31);      // pieces mine, mine + 32, ..: a warp's lie next to one another
  DropMask mask;
  if (DROP) mask.init(a.drop);
  else mask.limit = 0;
  const int rounds = MANY ? (a.octs + T * V - 1) / (T * V) : 1;
  const bool int8 = a.int8.values != nullptr;
  uint32_t turn = 0;
  for (RowWalk walk{blockIdx.x, (uint32_t)a.rows, gridDim.x}; walk.here(); walk.next()) {
    const int row = (int)walk.row;
    const X* const xp = reinterpret_cast<const X*>(a.x.p) + row * a.x.ld;
    const S* const rp = reinterpret_cast<const S*>(a.r.p) + row * a.r.ld;
    Eight<S> h[V];
    float power = 1.f;
    auto fetch = [&](int first) {      // h of the pieces from `first` on
      Eight<X> x[V];
#pragma unroll
      for (int v = 0; v < V; ++v) load_eight<LIE>(x[v], xp, (first + mine + 32 * v) * 8, a.cols);
      if (a.r.p != nullptr) {
#pragma unroll
        for (int v = 0; v < V; ++v) load_eight<LIE>(h[v], rp, (first + mine + 32 * v) * 8, a.cols);
      }
      // (the generator's rounds of all pieces together, where the registers have room: 75600 x 5120 bf16 with dropout 541 us instead of 570, 65972 x 1536 fp32 215 instead of 209)
      constexpr bool TOGETHER = sizeof(X) + sizeof(S) == 4;
      uint32_t words[V][4];
      if (TOGETHER && DROP && mask.limit != 0) {
        uint32_t rows[V], octs[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
          rows[v] = row;
          octs[v] = first + mine + 32 * v;
        }
        mask.words(words, rows, octs);
      }
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if constexpr (sizeof(X) == 2 && sizeof(S) == 2) {
          if (DROP && mask.limit != 0) combine(h[v], x[v], a.r.p != nullptr, mask, words[v]);
          else if (a.r.p != nullptr) combine_bf16(h[v], x[v]);
          else h[v] = x[v];
        } else {
          uint32_t own[1][4];
          const uint32_t rows[1] = {(uint32_t)row}, octs[1] = {(uint32_t)(first + mine + 32 * v)};
          if (mask.limit != 0) mask.words(own, rows, octs);
          combine(h[v], x[v], a.r.p != nullptr, mask, own[0]);
        }
      }
    };
    auto keep = [&](int first) {
      if constexpr (NORM) {
        if (a.h.p == nullptr) return;
#pragma unroll
        for (int v = 0; v < V; ++v) store_eight<LIE, V>(h[v], h[v > 0 ? v - 1 : 0], v, reinterpret_cast<S*>(a.h.p) + row * a.h.ld, (first + mine + 32 * v) * 8, a.cols);
      }
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
    bool again = false;
#pragma unroll 1
    for (;;) {
      float2 ss = make_float2(0.f, 0.f);
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
          if (NORM) weight_of<LIE>(w, a.w, (first + mine + 32 * v) * 8, a.cols);
          if (int8) add_sums<NORM, true>(h[v], w, ss, top);
          else add_sums<NORM, false>(h[v], w, ss, top);
        }
      }
      const float2 of = row_total<NORM, 1>(ss.x + ss.y, top, sh, turn++);
      top = of.y;
      const float ms = NORM ? of.x * a.inv_cols + eps : 1.f;
      r = NORM ? rsqrtf(ms) : 1.f;
      if (in_range(ms) || again) break;
      if constexpr (NORM) {
        again = true;
        float size = 0.f;
#pragma unroll 1
        for (int i = 0; i < rounds; ++i) {
          if (MANY) fetch(i * T * V);
#pragma unroll
          for (int v = 0; v < V; ++v) size = largest_of(h[v], size);
        }
        power = power_for(__float_as_uint(row_total<false, 1>(0.f, size, sh, turn++).y), eps);
        if (!MANY) apply_power();
        eps = eps * power * power;
      }
    }
    const float factor = int8 ? int8_factor(top) : 0.f;
    uint32_t scales = 0u;
    Outgoing<float> y_wide;
    Outgoing<bf16> y_narrow;
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
        const int oct = first + mine + 32 * v;
        float2 w[4], f[4];
        if (NORM) weight_of<LIE>(w, a.w, oct * 8, a.cols);
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = NORM ? __fmul2_rn(h[v].pair(j), w[j]) : h[v].pair(j);
        if (int8) {
          put_bytes<LIE>(int8_piece(f, top, factor), reinterpret_cast<unsigned char*>(a.int8.values) + row * a.int8.ld, oct * 8, a.cols);
        }
        if (NORM && a.fp8.values != nullptr) {
          uint32_t byte;
          const uint2 q = fp8_piece(f, r, byte);
          put_bytes<LIE>(q, a.fp8.values + row * a.fp8.ld, oct * 8, a.cols);
          // four blocks, one word of scales, are in two pieces of a warp, two blocks each (zero for those behind the row)
          scales = v & 1 ? scales | byte << 16 : byte;
          if (v & 1) {
            const uint32_t others = __shfl_down_sync(0xffffffffu, scales, 16);
            if ((t & 31) == 0 && oct - 32 < a.octs) reinterpret_cast<uint32_t*>(a.fp8.scales)[(size_t)(oct >> 6) * a.rows + row] = scales | others << 8;
          }
        }
        if (NORM && a.y.p != nullptr) {
          float g[8];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            g[2 * j] = f[j].x * r;
            g[2 * j + 1] = f[j].y * r;
          }
          if (a.y_f32) y_wide.store<LIE, V>(g, v, reinterpret_cast<float*>(a.y.p) + row * a.y.ld, oct * 8, a.cols);
          else y_narrow.store<LIE, V>(g, v, reinterpret_cast<bf16*>(a.y.p) + row * a.y.ld, oct * 8, a.cols);
        }
      }
    }
    if (int8 && t == 0) a.int8.scales[row] = int8_scale(top, r);
  }
}

// Any rows.  MANY: the sums of the weight's gradient are kept in the CTA's row of `parts`, where a thread finds its own again; else in registers
// V: pieces of a thread, one up to 2048 elements of bf16 and 4096 of fp32, where it is faster or as fast: each has its sums of the weight's gradient in registers, which leave room for
// fewer warps (30000 x 1536 bf16 67.9 us, with two 72.2; in fp32 116.8, 126.5; 20000 x 4096 bf16 141.5, 135.7).  Two take 96 registers, with which an SM holds two CTAs of 320 threads
// (75600 x 5120 572 us, in 104 registers 889); up to 56 bytes a thread are put aside for it, up to 148 where rows lie anywhere.  One piece of bf16 takes 80, and has the next row under way (without it, in 64 registers: 30000 x 1536 77.6 us instead of 67.9, 60000 x 640 87.7
// instead of 69.5); in fp32 that has no room (65972 x 1536 281 us, without 255).
template <int V, bool MANY, typename S, typename G, int LIE>
__global__ void __maxnreg__(V == 2 ? 96 : sizeof(S) == 2 ? 80 : 64) norm_bwd_kernel(const __grid_constant__ NormBwdArgs a) {
  __shared__ __align__(16) RowSums sh;
  sh.init();
  grid_enter();
  const int t = threadIdx.x, T = blockDim.x, mine = (t >> 5) * (32 * V) + (t & 31);      // pieces mine, mine + 32, ..: a warp's lie next to one another
  DropMask mask;
  mask.init(a.drop);
  const int rounds = MANY ? (a.octs + T * V - 1) / (T * V) : 1;
  const bool stream = a.dh.p != nullptr;
  float2 dw[V][4];
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int i = 0; i < 4; ++i) dw[v][i] = make_float2(0.f, 0.f);
  float* const part = a.parts != nullptr ? a.parts + (size_t)blockIdx.x * a.octs * 8 : nullptr;
  auto sum_of = [&](int v) {
    Eight<float> e;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      e.f[2 * i] = dw[v][i].x;
      e.f[2 * i + 1] = dw[v][i].y;
    }
    return e;
  };
  constexpr bool AHEAD = V == 1 && !MANY && sizeof(S) == 2;      // the next row is asked for before this one is looked at
  Eight<S> h[V], dh[V];
  Eight<G> dy[V];
  auto fetch = [&](Eight<S> (&to_h)[V], Eight<G> (&to_dy)[V], Eight<S> (&to_dh)[V], int row, int first, bool both) {
#pragma unroll
    for (int v = 0; v < V; ++v) load_eight<LIE>(to_h[v], reinterpret_cast<const S*>(a.h.p) + row * a.h.ld, (first + mine + 32 * v) * 8, a.cols);
#pragma unroll
    for (int v = 0; v < V; ++v) load_eight<LIE>(to_dy[v], reinterpret_cast<const G*>(a.dy.p) + row * a.dy.ld, (first + mine + 32 * v) * 8, a.cols);
    if (both && stream) {
#pragma unroll
      for (int v = 0; v < V; ++v) load_eight<LIE>(to_dh[v], reinterpret_cast<const S*>(a.dh.p) + row * a.dh.ld, (first + mine + 32 * v) * 8, a.cols);
    }
  };
  Eight<S> next_h[V], next_dh[V];
  Eight<G> next_dy[V];
  if (AHEAD) fetch(next_h, next_dy, next_dh, blockIdx.x, 0, true);
  uint32_t turn = 0;
  for (int row = blockIdx.x; row < a.rows; row += gridDim.x) {
    float power = 1.f;
    auto apply_power = [&] {
      if (power == 1.f) return;
#pragma unroll
      for (int v = 0; v < V; ++v) rescale(h[v], power);
    };
    if (AHEAD) {
      h[0] = next_h[0];
      dy[0] = next_dy[0];
      dh[0] = next_dh[0];
      if (row + (int)gridDim.x < a.rows) fetch(next_h, next_dy, next_dh, row + gridDim.x, 0, true);
    } else if (!MANY) {
      fetch(h, dy, dh, row, 0, true);
    }
    float r, eps = a.eps, along;
    bool again = false;
#pragma unroll 1
    for (;;) {
      float2 ss = make_float2(0.f, 0.f), dot = ss;
#pragma unroll 1
      for (int i = 0; i < rounds; ++i) {
        const int first = i * T * V;
        if (MANY) {
          fetch(h, dy, dh, row, first, false);
          apply_power();
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
          float2 w[4];
          weight_of<LIE>(w, a.w, (first + mine + 32 * v) * 8, a.cols);
          add_dots(h[v], dy[v], w, ss, dot);
        }
      }
      const float2 of = row_total<true, 2>(ss.x + ss.y, dot.x + dot.y, sh, turn++);
      const float ms = of.x * a.inv_cols + eps;
      r = rsqrtf(ms);
      along = of.y * r * a.inv_cols;
      if (in_range(ms) || again) break;
      again = true;
      float size = 0.f;
#pragma unroll 1
      for (int i = 0; i < rounds; ++i) {
        if (MANY) fetch(h, dy, dh, row, i * T * V, false);
#pragma unroll
        for (int v = 0; v < V; ++v) size = largest_of(h[v], size);
      }
      power = power_for(__float_as_uint(row_total<false, 1>(0.f, size, sh, turn++).y), eps);
      eps = eps * power * power;
      if (!MANY) apply_power();
    }
    const float out = r * power;
    Outgoing<S> dr;
    Outgoing<float> dx_wide;
    Outgoing<bf16> dx_narrow;
#pragma unroll 1
    for (int i = 0; i < rounds; ++i) {
      const int first = i * T * V;
      if (MANY) {
        fetch(h, dy, dh, row, first, true);
        apply_power();
      }
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int oct = first + mine + 32 * v;
        float f[8];
        float2 w[4];
        weight_of<LIE>(w, a.w, oct * 8, a.cols);
        gradient_piece(f, h[v], dy[v], dh[v], stream, w, dw[v], r, out, along);
        if (a.dr.p != nullptr) dr.template store<LIE, V>(f, v, reinterpret_cast<S*>(a.dr.p) + row * a.dr.ld, oct * 8, a.cols);
        if (a.dx.p != nullptr) {
          mask.apply(f, row, oct);
          if (a.dx_f32) dx_wide.store<LIE, V>(f, v, reinterpret_cast<float*>(a.dx.p) + row * a.dx.ld, oct * 8, a.cols);
          else dx_narrow.store<LIE, V>(f, v, reinterpret_cast<bf16*>(a.dx.p) + row * a.dx.ld, oct * 8, a.cols);
        }
        if (MANY) {
          if (part != nullptr && oct < a.octs) {
            Eight<float> sum = sum_of(v);
            if (row != (int)blockIdx.x) {
              Eight<float> before;
              before.load(part + oct * 8);
#pragma unroll
              for (int j = 0; j < 8; ++j) sum.f[j] += before.f[j];
            }
            sum.store(part + oct * 8);
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) dw[v][j] = make_float2(0.f, 0.f);
        }
      }
    }
  }
  if (!MANY && part != nullptr) {
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (mine + 32 * v < a.octs) sum_of(v).store(part + (mine + 32 * v) * 8);
  }
}

// The weight's gradient: the CTAs' parts, each of `width` columns, added in a fixed order.  32 columns a CTA, 32 ranges of the parts, eight loads of a thread under way.
__global__ void __launch_bounds__(1024) norm_weight_kernel(const float* parts, int count, int cols, int width, float* __restrict__ dw) {
  __shared__ float sh[32][33];
  grid_enter();
  const int lane = threadIdx.x & 31, range = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
  float sum = 0.f;
  if (col < cols) {
    const float* from = parts + col;
#pragma unroll 8
    for (int i = range; i < count; i += 32) sum += from[(size_t)i * width];
  }
  sh[range][lane] = sum;
  __syncthreads();
  sum = sh[lane][range];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0 && blockIdx.x * 32 + range < cols) dw[blockIdx.x * 32 + range] = sum;
}

// CTAs of a kernel that the device holds at a time; asked for once for each number of warps and device
struct Residents {
  std::atomic<int> known[kMaxDevices][kNormMost / 32 + 1] = {};      // of an SM
};
cudaError_t resident_ctas(const void* kernel, Residents& r, int threads, int* ctas) {
  int dev = 0, sms = 0;
  cudaError_t e;
  if ((e = cudaGetDevice(&dev)) != cudaSuccess || (e = sm_count(&sms)) != cudaSuccess) return e;
  int n = dev < kMaxDevices ? r.known[dev][threads / 32].load(std::memory_order_relaxed) : 0;
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
// Pieces of a thread.  Forward: four share a row's fixed steps (its sums, the barrier, two divisions), two leave more warps whose latencies overlap.  Rows of bf16 of more than 4096
// elements take four (75600 x 5120 to e4m3 440 us, with two 500; 10000 x 8192 94, 110), shorter ones two (75600 x 1536 to e4m3 130 us, with four 185; 2048 x 1536 5.5, 7.6), and so
// do rows with fp32, of which four pieces do not fit the registers (65972 x 1536 219 us, with four 319).  Rows with fp32 of more than 8192 elements take four all the same, though up to
// 430 bytes a thread are put aside: 0, as many as it takes, reads them twice (10000 x 8200 fp32 to bf16 222 us, the loop 268; 12288 297, 333; 16384 387, 394; of int8 66, 101 .. 117, 145;
// only fp32 with a dropout is faster in the loop from 12,288 on: 405, 403; 16384 541, 457)
int pieces_fwd(int octs, bool narrow) { return octs <= (narrow ? kNormMost : 2 * kNormMost) ? 2 : octs <= 4 * kNormMost ? 4 : 0; }

template <int V, bool MANY, typename X, typename S, bool NORM, int LIE, bool DROP = NORM>
cudaError_t go_fwd(const NormFwdArgs& a, cudaStream_t st) {
  static Residents residents;
  const int threads = threads_for(a.octs, V);
  int ctas = 0;
  const cudaError_t e = resident_ctas((const void*)norm_fwd_kernel<V, MANY, X, S, NORM, LIE, DROP>, residents, threads, &ctas);
  if (e != cudaSuccess) return e;
  return launch_kernel(norm_fwd_kernel<V, MANY, X, S, NORM, LIE, DROP>, norm_fwd_ctas(a.rows, ctas), threads, 0, st, a);
}
template <int V, typename X, typename S, bool NORM, bool DROP>
cudaError_t lie_fwd(const NormFwdArgs& a, cudaStream_t st) {
  return a.octs % (V * 32) == 0 && threads_for(a.octs, V) * V == a.octs ? go_fwd<V, false, X, S, NORM, ROWS_WHOLE, DROP>(a, st)
                                                                        : go_fwd<V, false, X, S, NORM, ROWS_ALIGNED, DROP>(a, st);
}
template <int V, typename X, typename S, bool NORM>
cudaError_t drop_fwd(const NormFwdArgs& a, cudaStream_t st) {
  // (rows of bf16, whose kernels are the ones that are short of registers, have kernels without a dropout)
  if constexpr (NORM && sizeof(X) + sizeof(S) == 4) return a.drop.threshold ? lie_fwd<V, X, S, NORM, true>(a, st) : lie_fwd<V, X, S, NORM, false>(a, st);
  else return lie_fwd<V, X, S, NORM, NORM>(a, st);
}
template <typename X, typename S, bool NORM>
cudaError_t size_fwd(const NormFwdArgs& a, bool vec, cudaStream_t st) {
  if (!vec) return a.octs > 2 * kNormMost ? go_fwd<2, true, X, S, NORM, ROWS_ANY>(a, st) : go_fwd<2, false, X, S, NORM, ROWS_ANY>(a, st);
  switch (pieces_fwd(a.octs, sizeof(X) + sizeof(S) == 4)) {
    case 2: return drop_fwd<2, X, S, NORM>(a, st);
    case 4: return drop_fwd<4, X, S, NORM>(a, st);
    default: return go_fwd<2, true, X, S, NORM, ROWS_ALIGNED>(a, st);
  }
}

cudaError_t sum_parts(const NormBwdArgs& a, int ctas, float* dw, cudaStream_t st) {
  if (dw == nullptr) return cudaSuccess;
  return launch_kernel(norm_weight_kernel, (a.cols + 31) / 32, 1024, 0, st, a.parts, ctas, a.cols, a.octs * 8, dw);
}
template <int V, bool MANY, typename S, typename G, int LIE>
cudaError_t go_bwd(const NormBwdArgs& a, float* dw, cudaStream_t st) {
  static Residents residents;
  const int threads = threads_for(a.octs, V);
  int ctas = 0;
  cudaError_t e = resident_ctas((const void*)norm_bwd_kernel<V, MANY, S, G, LIE>, residents, threads, &ctas);
  if (e != cudaSuccess) return e;
  if (ctas > kNormParts) ctas = kNormParts;
  const int each = (a.rows + ctas - 1) / ctas;      // rows of a CTA: no more CTAs, and parts, than take the same time with as many each
  ctas = (a.rows + each - 1) / each;
  e = launch_kernel(norm_bwd_kernel<V, MANY, S, G, LIE>, ctas, threads, 0, st, a);
  return e != cudaSuccess ? e : sum_parts(a, ctas, dw, st);
}
template <int V, typename S, typename G>
cudaError_t lie_bwd(const NormBwdArgs& a, float* dw, cudaStream_t st) {
  return threads_for(a.octs, V) * V == a.octs ? go_bwd<V, false, S, G, ROWS_WHOLE>(a, dw, st) : go_bwd<V, false, S, G, ROWS_ALIGNED>(a, dw, st);
}
template <typename S, typename G>
cudaError_t size_bwd(const NormBwdArgs& a, bool vec, float* dw, cudaStream_t st) {
  if (!vec)
    return a.octs <= kNormMost ? go_bwd<1, false, S, G, ROWS_ANY>(a, dw, st) : a.octs <= 2 * kNormMost ? go_bwd<2, false, S, G, ROWS_ANY>(a, dw, st)
                                                                                                       : go_bwd<1, true, S, G, ROWS_ANY>(a, dw, st);
  if (a.octs <= (sizeof(S) == 2 ? kNormMost / 2 : kNormMost)) return lie_bwd<1, S, G>(a, dw, st);
  return a.octs <= 2 * kNormMost ? lie_bwd<2, S, G>(a, dw, st) : go_bwd<1, true, S, G, ROWS_ALIGNED>(a, dw, st);
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
  if (h_f32) return dy_f32 ? size_bwd<float, float>(a, vec, dw, st) : size_bwd<float, bf16>(a, vec, dw, st);
  return dy_f32 ? size_bwd<bf16, float>(a, vec, dw, st) : size_bwd<bf16, bf16>(a, vec, dw, st);
}

}  // namespace vsa2
