// Matrices whose rows are tokens, taken in pieces of eight neighbouring elements, and the dropout that falls on them: what the kernels of the
// residual stream (residual_norm.cu, dropout.cu) share, and their arguments.
#pragma once
#include "common.cuh"
#include "heads.cuh"

namespace vsa2 {

// [rows, cols] with contiguous rows `ld` elements apart; null: absent
struct RowsArg {
  void* p;
  long long ld;
};
// int8 values [rows, ld] and a scale a row
struct Int8Arg {
  signed char* values;
  float* scales;
  long long ld;
};
// rng: seed and offset, on the device; an element is kept where its 16 bits are at least `threshold` (0: no dropout)
struct DropArg {
  const unsigned long long* rng;
  uint32_t threshold;
  float scale;
};
struct NormFwdArgs {
  RowsArg x, r, h, y;
  Fp8Arg fp8;
  Int8Arg int8;
  const float* w;
  float eps, inv_cols;
  int rows, cols, octs, y_f32;
  DropArg drop;
};
struct NormBwdArgs {
  RowsArg h, dy, dh, dr, dx;
  const float* w;
  float* parts;      // null: the weight's gradient is not wanted
  float eps, inv_cols;
  int rows, cols, octs, dx_f32;
  DropArg drop;
};
struct DropoutArgs {
  RowsArg x, r, y;
  int rows, cols, octs;
  Divisor by_octs;
  unsigned long long per_octs;      // 2^64 / octs, rounded up
  DropArg drop;
};
// The rows of a CTA of the norm forward (and of the int8 quantisation): every ctas-th from its own number on.  Counted without a sign: what is formed behind its last row is less than
// rows + ctas, and with a CTA for each four rows that passes 2^31 from 1,717,986,917 rows on (2^31 + 2^29 at most)
struct RowWalk {
  uint32_t row, rows, ctas;
  __host__ __device__ __forceinline__ bool here() const { return row < rows; }
  __host__ __device__ __forceinline__ void next() { row += ctas; }
};
// CTAs for `rows` rows, where the device holds `resident` at a time.  Four rows a CTA, or as many as it takes: CTAs that end at different times keep memory busy (75600 x 5120 to e4m3
// 412 us, with CTAs that stay 429, of one row each 417; int8 of 15360 x 5120 42, 42, 47)
inline int norm_fwd_ctas(int rows, int resident) {
  const int fours = (rows + 3) / 4;
  return fours > resident ? fours : rows < resident ? rows : resident;
}
cudaError_t launch_norm_fwd(NormFwdArgs a, bool x_f32, bool h_f32, cudaStream_t st);
cudaError_t launch_int8_quantize(const RowsArg& x, bool x_f32, int rows, int cols, const Int8Arg& out, cudaStream_t st);
size_t norm_bwd_workspace_bytes(int rows, int cols);
cudaError_t launch_norm_bwd(NormBwdArgs a, bool h_f32, bool dy_f32, float* dw, float* parts, cudaStream_t st);
cudaError_t launch_dropout(DropoutArgs a, bool x_f32, bool y_f32, cudaStream_t st);
size_t int8_matmul_workspace_bytes(int m, int n, int k);
cudaError_t launch_int8_matmul(int m, int n, int k, const Int8Arg& a, const Int8Arg& b, const float* bias, void* c, int c_f32, long long ldc, void* workspace,
                               cudaStream_t st);
// vsa2_debug_int8_matmul_plan
void int8_matmul_plan(int m, int n, int k, int sms, bool pairs, int32_t* out);
// k = 0: the bias, or nothing
cudaError_t launch_bias_rows(int m, int n, const float* bias, void* c, int c_f32, long long ldc, cudaStream_t st);

// whether every row of a matrix of elements of `size` bytes begins on a 16-byte boundary
inline bool rows_aligned(const RowsArg& m, size_t size) {
  return m.p == nullptr || ((reinterpret_cast<uintptr_t>(m.p) & 15u) == 0 && m.ld * (long long)size % 16 == 0);
}

// Eight neighbouring elements as they lie in memory
template <typename T> struct Eight;
template <> struct Eight<bf16> {
  uint32_t u[4];
  __device__ __forceinline__ void zero() { u[0] = u[1] = u[2] = u[3] = 0u; }
  __device__ __forceinline__ void load(const bf16* p) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    u[0] = v.x; u[1] = v.y; u[2] = v.z; u[3] = v.w;
  }
  __device__ __forceinline__ void set(int j, const bf16* p) { u[j / 2] |= (uint32_t)*reinterpret_cast<const unsigned short*>(p) << 16 * (j & 1); }
  __device__ __forceinline__ float get(int j) const { return __uint_as_float(j & 1 ? u[j / 2] & 0xffff0000u : u[j / 2] << 16); }
  __device__ __forceinline__ float2 pair(int i) const { return make_float2(get(2 * i), get(2 * i + 1)); }
  __device__ __forceinline__ void round(const float (&f)[8]) {      // to the type
#pragma unroll
    for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(u[i]) : "f"(f[2 * i + 1]), "f"(f[2 * i]));
  }
  __device__ __forceinline__ void store(bf16* p) const { *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]); }
  __device__ __forceinline__ void store(bf16* p, int j) const { *reinterpret_cast<unsigned short*>(p) = (unsigned short)(u[j / 2] >> 16 * (j & 1)); }
};
template <> struct Eight<float> {
  float f[8];
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = 0.f;
  }
  __device__ __forceinline__ void load(const float* p) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
  __device__ __forceinline__ void set(int j, const float* p) { f[j] = *p; }
  __device__ __forceinline__ float get(int j) const { return f[j]; }
  __device__ __forceinline__ float2 pair(int i) const { return make_float2(f[2 * i], f[2 * i + 1]); }
  __device__ __forceinline__ void round(const float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = v[j];
  }
  __device__ __forceinline__ void store(float* p) const {
    reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
  }
  __device__ __forceinline__ void store(float* p, int j) const { *p = f[j]; }
};
// How the rows of a call lie: anywhere; on 16-byte boundaries and in whole pieces of eight elements; so, and as many pieces as the kernel's threads take
enum { ROWS_ANY = 0, ROWS_ALIGNED = 1, ROWS_WHOLE = 2 };
// element i of a row that is the same for all threads: a base of 64 bits and a thread's offset of 32 (2^22 elements at most), which a load adds by itself
template <typename T>
__device__ __forceinline__ T* element(T* row, int i) { return reinterpret_cast<T*>(reinterpret_cast<uintptr_t>(row) + (uint32_t)i * (uint32_t)sizeof(T)); }
// 16 bytes (bf16), or 32, that begin `shift` bytes (even, up to 16) into some words, of which those beyond the first 16 (32) matter only up to there
__device__ __forceinline__ void shifted(Eight<bf16>& e, const uint32_t (&w)[8], uint32_t shift) {
  uint32_t a[6], b[5];
#pragma unroll
  for (int k = 0; k < 6; ++k) a[k] = shift & 8 ? w[k + 2] : w[k];
#pragma unroll
  for (int k = 0; k < 5; ++k) b[k] = shift & 4 ? a[k + 1] : a[k];
#pragma unroll
  for (int k = 0; k < 4; ++k) e.u[k] = shift & 16 ? w[k + 4] : __funnelshift_r(b[k], b[k + 1], (shift & 2) * 8);
}
__device__ __forceinline__ void shifted(Eight<float>& e, const uint32_t (&w)[12], uint32_t shift) {      // (a multiple of four)
  uint32_t a[10];
#pragma unroll
  for (int k = 0; k < 10; ++k) a[k] = shift & 8 ? w[k + 2] : w[k];
#pragma unroll
  for (int k = 0; k < 8; ++k) e.f[k] = __uint_as_float(shift & 16 ? w[k + 4] : shift & 4 ? a[k + 1] : a[k]);
}
__device__ __forceinline__ uint32_t word_of(const Eight<bf16>& e, int k) { return e.u[k]; }
__device__ __forceinline__ uint32_t word_of(const Eight<float>& e, int k) { return __float_as_uint(e.f[k]); }

// Elements i .. i+7 of a row (zeros behind it, and for i beyond it).  Rows that lie anywhere: the aligned 16-byte places that the piece lies in, where the row has all of them, shifted into
// place; single elements at a row's two ends
template <int LIE, typename T>
__device__ __forceinline__ void load_eight(Eight<T>& e, const T* row, int i, int cols) {
  if (LIE == ROWS_WHOLE) {
    e.load(element(row, i));
  } else if (LIE == ROWS_ALIGNED) {
    if (i < cols) e.load(element(row, i));
    else e.zero();
  } else {
    constexpr int SIZE = sizeof(T), PLACES = SIZE / 2;      // of 16 bytes in a piece
    const T* const at = element(row, i);
    const int s = (int)(reinterpret_cast<uintptr_t>(at) & 15u), left = cols - i;
    if (i * SIZE >= s && left * SIZE + s >= 16 * (PLACES + 1)) {
      const uint4* from = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(at) - s);
      uint32_t w[4 * PLACES + 4];
#pragma unroll
      for (int k = 0; k <= PLACES; ++k) {
        const uint4 v = from[k];
        w[4 * k] = v.x; w[4 * k + 1] = v.y; w[4 * k + 2] = v.z; w[4 * k + 3] = v.w;
      }
      shifted(e, w, (uint32_t)s);      // (whole: more than eight elements are left)
    } else {
      e.zero();
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < left) e.set(j, at + j);
    }
  }
}
// .. back to a row.  By whole warps: a warp's pieces lie next to one another, 32 of number v and then those of number v + 1 (`before`: this thread's of number v - 1).  Rows that lie anywhere:
// a thread stores the aligned places that end in its piece, with what it is told of the piece before, where the row has all of them; single elements at the ends of a row and of a
// warp's pieces
template <int LIE, int V, typename T>
__device__ __forceinline__ void store_eight(const Eight<T>& e, const Eight<T>& before, int v, T* row, int i, int cols) {
  if (LIE != ROWS_ANY) {
    if (LIE == ROWS_WHOLE || i < cols) e.store(element(row, i));
  } else {
    constexpr int SIZE = sizeof(T), PLACES = SIZE / 2, WORDS = 4 * PLACES;
    const int lane = threadIdx.x & 31;
    T* const at = element(row, i);
    const int s = (int)(reinterpret_cast<uintptr_t>(at) & 15u);      // (the same for the whole row)
    uint32_t w[WORDS + 4];      // the 16 bytes in front of the piece, and it
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = __shfl_sync(0xffffffffu, lane == 31 && v > 0 ? word_of(before, WORDS - 4 + k) : word_of(e, WORDS - 4 + k), (lane + 31) & 31);
#pragma unroll
    for (int k = 0; k < WORDS; ++k) w[4 + k] = word_of(e, k);
    Eight<T> out;
    shifted(out, w, 16u - s);
    const int first = i - s / SIZE;      // element that it begins with
    const bool told = s == 0 || v > 0 || lane > 0;
    if (told && first >= 0 && first + 8 <= cols) {
      out.store(reinterpret_cast<T*>(reinterpret_cast<char*>(at) - s));
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (first + j >= 0 && first + j < cols && (told || j * SIZE >= s)) out.store(at - s / SIZE + j, j);
    }
    if (v == V - 1 && lane == 31) {      // what the places leave of the warp's last piece
#pragma unroll
      for (int j = 1; j < 8; ++j)
        if ((8 - j) * SIZE <= s && i + j < cols) e.store(at + j, j);
    }
  }
}

// f plus e, each sum rounded
template <typename T>
__device__ __forceinline__ void add_eight(float (&f)[8], const Eight<T>& e) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 v = __fadd2_rn(e.pair(i), make_float2(f[2 * i], f[2 * i + 1]));
    f[2 * i] = v.x;
    f[2 * i + 1] = v.y;
  }
}

// Which elements are kept.  The counter-based generator Philox 4x32 with ten rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011): its
// key is the seed, its counter (column / 8, row, offset), and its 128 bits are 16 for each of eight neighbours.  So the mask follows from seed, offset and an element's place alone: no
// shape of a launch, alignment or stride changes it, and a backward pass forms it again.  (32 bits an element would take twice the multiplications, and ten rounds for four
// elements run at the pace of memory.)
struct DropMask {
  uint32_t k0, k1, o0, o1, limit;
  float scale;
  __device__ __forceinline__ void init(const DropArg& d) {
    const unsigned long long seed = d.threshold ? d.rng[0] : 0, offset = d.threshold ? d.rng[1] : 0;
    k0 = (uint32_t)seed; k1 = (uint32_t)(seed >> 32);
    o0 = (uint32_t)offset; o1 = (uint32_t)(offset >> 32);
    limit = d.threshold << 16;
    scale = d.scale;
  }
  // The generator's four words for each of N pieces, round by round, so that a round's key is formed once
  template <int N>
  __device__ __forceinline__ void words(uint32_t (&w)[N][4], const uint32_t (&row)[N], const uint32_t (&oct)[N]) const {
    uint32_t p = k0, q = k1;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      w[n][0] = oct[n]; w[n][1] = row[n];
      w[n][2] = o0; w[n][3] = o1;
    }
#pragma unroll
    for (int i = 0; i < 10; ++i) {
#pragma unroll
      for (int n = 0; n < N; ++n) {
        unsigned long long u, v;
        asm("mul.wide.u32 %0, %1, %2;" : "=l"(u) : "r"(w[n][0]), "r"(0xD2511F53u));
        asm("mul.wide.u32 %0, %1, %2;" : "=l"(v) : "r"(w[n][2]), "r"(0xCD9E8D57u));
        w[n][0] = (uint32_t)(v >> 32) ^ w[n][1] ^ p;
        w[n][1] = (uint32_t)v;
        w[n][2] = (uint32_t)(u >> 32) ^ w[n][3] ^ q;
        w[n][3] = (uint32_t)u;
      }
      p += 0x9E3779B9u;
      q += 0xBB67AE85u;
    }
  }
  // Eight elements: zero, or times the scale.  (A product of its own, not part of a fused one: what the library computes does not depend on what is added behind it.)
  __device__ __forceinline__ void keep(float (&f)[8], const uint32_t (&w)[4]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 v = __fmul2_rn(make_float2(f[2 * i], f[2 * i + 1]), make_float2(scale, scale));
      f[2 * i] = w[i] << 16 >= limit ? v.x : 0.f;
      f[2 * i + 1] = w[i] >= limit ? v.y : 0.f;      // (the lower half decides nothing)
    }
  }
  __device__ __forceinline__ void apply(float (&f)[8], uint32_t row, uint32_t oct) const {
    if (limit == 0) return;
    uint32_t w[1][4];
    const uint32_t rows[1] = {row}, octs[1] = {oct};
    words(w, rows, octs);
    keep(f, w[0]);
  }
};

}  // namespace vsa2
