// 8-bit form of a matrix for vsa2_fp8_matmul: e4m3 values with a power-of-two scale for each block of 128 values along the rows, the same of
// the transpose (blocks along the columns), or both from one reading.
//   e = the least integer with max|x| <= 448 * 2^e over the block's finite values (448: the largest e4m3 value), at least -127
//   value = x * 2^-e rounded to e4m3 (to nearest, ties to even); what is not finite becomes NaN
// A power of two scales without rounding, so the 3 mantissa bits are all that is lost, and it is what the tensor cores multiply by themselves.
// x is read once, each form written once; bound by memory.  Rows: 75600 x 5120 184 us (6.3 TB/s), 20000 x 5120 47 us (6.5), of fp32 76 us (6.7).  Both forms in one reading: 20000 x 5120
// 69 us (6.0), of fp32 98 us (6.3), blocks of 128 x 128 of 15360 x 5120 53 us (5.9); 2025 x 4600, one wave of CTAs, 11.4 us.
#include "common.cuh"
#include "heads.cuh"

namespace vsa2 {

namespace {

constexpr int kQzThreads = 256;

// exponent + 127 from the bits of max|x|: 448 = 1.75 * 2^8, so a fraction above 0.75 carries (at most 254 - 8 + 1)
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) { return (uint32_t)max((int)((top + 0x1fffffu) >> 23) - 8, 0); }
__device__ __forceinline__ float inverse_scale(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }
__device__ __forceinline__ uint32_t scale_of(float inverse) { return 254u - (__float_as_uint(inverse) >> 23); }
__device__ __forceinline__ bool finite_bits(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
  uint32_t r;
  asm("{\n\t.reg .b16 lo, hi;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\t"
      "mov.b32 %0, {lo, hi};\n\t}"
      : "=r"(r) : "f"(a), "f"(b), "f"(c), "f"(d));
  return r;
}
// Blocks where something is not finite are rare: only they look at every value (CHECK).  (An infinity becomes NaN; the conversion alone would make it 448.)
template <bool CHECK>
__device__ __forceinline__ float scaled(float x, float inv) { return !CHECK || finite_bits(x) ? x * inv : __uint_as_float(0x7fffffffu); }

// Eight neighbouring elements of a row as they lie in memory; magnitudes as the bits of fp32 numbers, those of bf16 two in a word
template <bool F32> struct Oct;
template <> struct Oct<false> {
  uint32_t u[4];
  __device__ __forceinline__ void zero() { u[0] = u[1] = u[2] = u[3] = 0u; }
  __device__ __forceinline__ void load(const void* x, size_t at) {
    const uint4 v = *reinterpret_cast<const uint4*>(reinterpret_cast<const bf16*>(x) + at);
    u[0] = v.x; u[1] = v.y; u[2] = v.z; u[3] = v.w;
  }
  __device__ __forceinline__ void set(const void* x, size_t at, int j) {
    u[j / 2] |= (uint32_t)reinterpret_cast<const unsigned short*>(x)[at] << 16 * (j & 1);
  }
  __device__ __forceinline__ void keep(int n) {      // the first n of the eight
#pragma unroll
    for (int j = 0; j < 4; ++j) u[j] = 2 * j + 1 < n ? u[j] : 2 * j < n ? u[j] & 0xffffu : 0u;
  }
  __device__ __forceinline__ float get(int j) const { return __uint_as_float(j & 1 ? u[j / 2] & 0xffff0000u : u[j / 2] << 16); }
  __device__ __forceinline__ uint32_t top() const {
    const uint32_t t = __vmaxu2(__vmaxu2(u[0] & 0x7fff7fffu, u[1] & 0x7fff7fffu), __vmaxu2(u[2] & 0x7fff7fffu, u[3] & 0x7fff7fffu));
    return max(t & 0xffff0000u, t << 16);
  }
  struct Tops {                      // of the eight columns
    static constexpr int PER = 2;      // columns in a word
    uint32_t t[4] = {0u, 0u, 0u, 0u};
    __device__ __forceinline__ void set(int j, uint32_t top) { t[j / 2] |= j & 1 ? top : top >> 16; }
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return __vmaxu2(a, b); }
    static __device__ __forceinline__ uint32_t get(uint32_t word, int j) { return j & 1 ? word & 0xffff0000u : word << 16; }
  };
  // the row's, raising the columns'
  __device__ __forceinline__ uint32_t sweep(Tops& o) const {
    uint32_t m[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      m[i] = u[i] & 0x7fff7fffu;
      o.t[i] = __vmaxu2(o.t[i], m[i]);
    }
    const uint32_t t = __vmaxu2(__vmaxu2(m[0], m[1]), __vmaxu2(m[2], m[3]));
    return max(t & 0xffff0000u, t << 16);
  }
};
template <> struct Oct<true> {
  float f[8];
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = 0.f;
  }
  __device__ __forceinline__ void load(const void* x, size_t at) {
    const float4* p = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(x) + at);
    const float4 a = p[0], b = p[1];
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
  __device__ __forceinline__ void set(const void* x, size_t at, int j) { f[j] = reinterpret_cast<const float*>(x)[at]; }
  __device__ __forceinline__ void keep(int n) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j >= n) f[j] = 0.f;
  }
  __device__ __forceinline__ float get(int j) const { return f[j]; }
  __device__ __forceinline__ uint32_t top() const {
    uint32_t t = 0u;
#pragma unroll
    for (int j = 0; j < 8; ++j) t = max(t, __float_as_uint(f[j]) & 0x7fffffffu);
    return t;
  }
  struct Tops {
    static constexpr int PER = 1;
    uint32_t t[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
    __device__ __forceinline__ void set(int j, uint32_t top) { t[j] = top; }
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return max(a, b); }
    static __device__ __forceinline__ uint32_t get(uint32_t word, int) { return word; }
  };
  __device__ __forceinline__ uint32_t sweep(Tops& o) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) o.t[j] = max(o.t[j], __float_as_uint(f[j]) & 0x7fffffffu);
    return top();
  }
};
constexpr uint32_t kInf = 0x7f800000u;
// the largest finite magnitude of eight
template <bool F32>
__device__ __forceinline__ uint32_t finite_top(const Oct<F32>& o) {
  uint32_t t = 0u;
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (finite_bits(o.get(j))) t = max(t, __float_as_uint(o.get(j)) & 0x7fffffffu);
  return t;
}
// The matrix that is read
struct Source {
  const unsigned char* x;
  int rows, cols;
  long long ld;
};
// the oct that begins at byte `from` (0 .. 7) of some words
__device__ __forceinline__ void set_words(const uint32_t (&w)[6], uint32_t from, Oct<false>& o) {
  uint32_t a[5];
#pragma unroll
  for (int k = 0; k < 5; ++k) a[k] = from & 4 ? w[k + 1] : w[k];
#pragma unroll
  for (int k = 0; k < 4; ++k) o.u[k] = __funnelshift_r(a[k], a[k + 1], (from & 2) * 8);
}
__device__ __forceinline__ void set_words(const uint32_t (&w)[10], uint32_t from, Oct<true>& o) {
#pragma unroll
  for (int k = 0; k < 8; ++k) o.f[k] = __uint_as_float(from & 4 ? w[k + 1] : w[k]);
}
// Elements i .. i+7 of a row (zeros beyond it)
template <bool F32, bool VEC>
__device__ __forceinline__ void load8(const Source& m, size_t row_at, int i, Oct<F32>& o) {
  if (VEC && i + 8 <= m.cols) {
    o.load(m.x, row_at + i);
  } else {
    o.zero();
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (i + j < m.cols) o.set(m.x, row_at + i + j, j);
  }
}
// Rows that do not begin on 16-byte boundaries: N octs, `step` bytes and COLUMNS columns apart, of which `there` exist (zeros for the others).  The aligned pieces that an oct
// lies in, those of all N asked for before the first is shifted into place, where the matrix has all of these bytes; single elements at its two ends.
// 20001 x 5001: single elements everywhere, pieces of 16 bytes (two stages of selection instead of one), of 8: bf16 71, 68, 66 us, both forms 143, 119, 108; fp32 102, 83, 86,
// both forms 214, 158, 162 (with the reductions of then; now 63, 95, 84, 140, and 50, 80, 78, 104 on 16-byte boundaries).  With each oct's loads behind the one's before bf16 took 92.
template <bool F32, int N, int COLUMNS>
__device__ __forceinline__ void load_shifted(const Source& m, long long row, int col, int there, long long step, Oct<F32>* o) {
  constexpr int SIZE = F32 ? 4 : 2, PIECES = SIZE + 1;      // of 8 bytes
  const size_t at = (size_t)row * m.ld + col;
  const unsigned char* const a = m.x + at * SIZE;
  const long long before = at * SIZE, behind = ((long long)(m.rows - 1) * m.ld + m.cols) * SIZE - before;      // bytes of the matrix on either side
  uint32_t w[N][PIECES * 2];
  bool inside[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const uint32_t from = (uint32_t)reinterpret_cast<uintptr_t>(a + k * step) & 7u;
    inside[k] = k < there && col + COLUMNS * k < m.cols && before + k * step >= from && behind - k * step >= (int)(PIECES * 8 - from);
    const uint2* piece = reinterpret_cast<const uint2*>(a + k * step - from);
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      uint2 v = make_uint2(0u, 0u);
      if (inside[k]) v = piece[p];
      w[k][2 * p] = v.x; w[k][2 * p + 1] = v.y;
    }
  }
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int left = m.cols - col - COLUMNS * k;
    set_words(w[k], (uint32_t)reinterpret_cast<uintptr_t>(a + k * step) & 7u, o[k]);
    if (left < 8 || !inside[k]) {
      if (inside[k]) {
        o[k].keep(left);
      } else if (k < there && left > 0) {
        o[k].zero();
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (j < left) o[k].set(a + k * step, j, j);
      }
    }
  }
}
// bytes i .. i+7 of a row of `cols` values (its start 16-byte aligned, i a multiple of 8)
__device__ __forceinline__ void put8(unsigned char* row, int i, int cols, uint32_t lo, uint32_t hi) {
  if (i + 8 <= cols) {
    *reinterpret_cast<uint2*>(row + i) = make_uint2(lo, hi);
  } else {
    for (int j = 0; i + j < cols; ++j) row[i + j] = (unsigned char)((j < 4 ? lo >> 8 * j : hi >> 8 * (j - 4)) & 0xffu);
  }
}
template <bool CHECK, bool FULL, bool F32>
__device__ __forceinline__ void put_oct(unsigned char* row, int i, int cols, const Oct<F32>& o, float inv) {
  float f[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) f[j] = scaled<CHECK>(o.get(j), inv);
  put8(row, i, FULL ? i + 8 : cols, e4m3x4(f[0], f[1], f[2], f[3]), e4m3x4(f[4], f[5], f[6], f[7]));
}
// The largest of each of N values over a team's 16 threads, value l / (16 / N) in thread l: halves of the values change sides at each step, N shuffles in all and a few for
// what is left instead of 4 N (20000 x 5120: both forms 82 -> 69 us, of fp32 131 -> 98)
template <int N>
__device__ __forceinline__ uint32_t team_tops(uint32_t (&t)[N], int l) {
  int o = 8;
#pragma unroll
  for (int n = N / 2; n > 0; n >>= 1, o >>= 1) {
    const bool upper = l & o;
#pragma unroll
    for (int k = 0; k < n; ++k) {
      const uint32_t other = __shfl_xor_sync(0xffffffffu, upper ? t[k] : t[k + n], o);
      t[k] = max(upper ? t[k + n] : t[k], other);
    }
  }
#pragma unroll
  for (; o > 0; o >>= 1) t[0] = max(t[0], __shfl_xor_sync(0xffffffffu, t[0], o));
  return t[0];
}

// Rows alone: a team of 16 threads takes 512 columns of a row (four blocks, one word of scales).  grid (row tiles of 16, word groups)
template <bool F32, bool VEC>
__global__ void __launch_bounds__(kQzThreads, F32 ? 5 : 6) fp8_rows_kernel(const __grid_constant__ Source m, Fp8Arg out) {
  constexpr int G = F32 ? 2 : 4;      // blocks whose scales are found together: as many as the registers of five or six CTAs hold (fp32 in fours spilled, 85 us; in pairs 76)
  grid_enter();
  const int rows = m.rows, cols = m.cols;
  const int l = threadIdx.x & 15;
  const long long row = (long long)blockIdx.x * 16 + (threadIdx.x >> 4);
  const int c0 = blockIdx.y * 512;
  const long long r = row < rows ? row : rows - 1;
  Oct<F32> o[4];
  if constexpr (VEC) {
#pragma unroll
    for (int b = 0; b < 4; ++b) load8<F32, VEC>(m, (size_t)r * m.ld, c0 + b * 128 + l * 8, o[b]);
  } else {
    load_shifted<F32, 4, 128>(m, r, c0 + l * 8, 4, 128 * (F32 ? 4 : 2), o);
  }
  uint32_t word = 0;
#pragma unroll
  for (int b0 = 0; b0 < 4; b0 += G) {
    uint32_t tops[G];
#pragma unroll
    for (int b = 0; b < G; ++b) tops[b] = o[b0 + b].top();
    uint32_t byte = team_tops(tops, l);
    const bool odd = __any_sync(0xffffffffu, byte >= kInf);
    if (odd) {
#pragma unroll
      for (int b = 0; b < G; ++b) tops[b] = finite_top<F32>(o[b0 + b]);
      byte = team_tops(tops, l);
    }
    byte = scale_byte(byte);
#pragma unroll
    for (int b = 0; b < G; ++b) {
      const uint32_t s = __shfl_sync(0xffffffffu, byte, 16 / G * b, 16);
      const int col = c0 + (b0 + b) * 128;
      if (col >= cols) continue;
      word |= s << 8 * (b0 + b);
      if (row < rows) {
        unsigned char* to = out.values + row * out.ld;
        if (odd) put_oct<true, false, F32>(to, col + l * 8, cols, o[b0 + b], inverse_scale(s));
        else put_oct<false, false, F32>(to, col + l * 8, cols, o[b0 + b], inverse_scale(s));
      }
    }
  }
  if (l == 0 && row < rows) reinterpret_cast<uint32_t*>(out.scales)[(size_t)blockIdx.y * rows + row] = word;
}

// scale of block kb of row `row` (of a form with `rows` rows and `blocks` blocks a row); the last block clears what is left of its word
__device__ __forceinline__ void put_scale(unsigned char* scales, int rows, int row, int kb, int blocks, uint32_t byte) {
  unsigned char* word = scales + ((size_t)(kb >> 2) * rows + row) * 4;
  word[kb & 3] = (unsigned char)byte;
  if (kb == blocks - 1)
    for (int j = (kb & 3) + 1; j < 4; ++j) word[j] = 0;
}

struct TileShared {
  unsigned char turned[128 * 128];
  uint32_t col_top[16][128];
  float col_inv[128];
  uint32_t tops[kQzThreads / 32];
};

// A tile whose values are in the threads' registers: both forms, or either.  `tops`, `cols_top`: largest magnitudes of the thread's rows and columns (of no use with CHECK);
// FULL: the tile lies inside the matrix
template <bool CHECK, bool FULL, bool F32>
__device__ __forceinline__ void quantize_tile(const Oct<F32> (&o)[8], uint32_t (&tops)[8], const typename Oct<F32>::Tops& cols_top, TileShared& sh,
                                              int rows, int cols, int squares, const Fp8Arg& out, const Fp8Arg& out_t) {
  const int l = threadIdx.x & 15, team = threadIdx.x >> 4, tid = threadIdx.x;
  const int c0 = blockIdx.y * 128, r0 = blockIdx.x * 128;
  const int blocks = (cols + 127) / 128, blocks_t = (rows + 127) / 128;
  if (CHECK) {
#pragma unroll
    for (int i = 0; i < 8; ++i) tops[i] = finite_top<F32>(o[i]);
  }
  uint32_t top_all = 0;
  if (squares) {
#pragma unroll
    for (int i = 0; i < 8; ++i) top_all = max(top_all, tops[i]);
    top_all = __reduce_max_sync(0xffffffffu, top_all);
    if ((tid & 31) == 0) sh.tops[tid >> 5] = top_all;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kQzThreads / 32; ++i) top_all = max(top_all, sh.tops[i]);
  }
  if (out.values != nullptr) {
    unsigned char* to = out.values + (r0 + team * 8) * out.ld;
    const uint32_t mine = scale_byte(squares ? top_all : team_tops(tops, l));      // of row l / 2
    const int row = r0 + team * 8 + l / 2;
    if ((l & 1) == 0 && (FULL || row < rows)) put_scale(out.scales, rows, row, blockIdx.y, blocks, mine);
#pragma unroll
    for (int i = 0; i < 8; ++i, to += out.ld) {
      const uint32_t s = __shfl_sync(0xffffffffu, mine, 2 * i, 16);
      if (FULL || r0 + team * 8 + i < rows) put_oct<CHECK, FULL, F32>(to, c0 + l * 8, cols, o[i], inverse_scale(s));
    }
  }
  if (out_t.values == nullptr) return;
  using Tops = typename Oct<F32>::Tops;
  if (squares) {
    if (tid < 128) sh.col_inv[tid] = inverse_scale(scale_byte(top_all));
  } else {
    Tops mine = cols_top;
    if (CHECK) {
      mine = Tops();
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (finite_bits(o[i].get(j))) top = max(top, __float_as_uint(o[i].get(j)) & 0x7fffffffu);
        mine.set(j, top);
      }
    }
#pragma unroll
    for (int k = 0; k < 8 / Tops::PER; k += 4)
      *reinterpret_cast<uint4*>(&sh.col_top[team][l * (8 / Tops::PER) + k]) = make_uint4(mine.t[k], mine.t[k + 1], mine.t[k + 2], mine.t[k + 3]);
    __syncthreads();
    if (tid < 128 / Tops::PER) {
      uint32_t top = 0;
#pragma unroll
      for (int r = 0; r < 16; ++r) top = Tops::larger(top, sh.col_top[r][tid]);
#pragma unroll
      for (int j = 0; j < Tops::PER; ++j) sh.col_inv[tid * Tops::PER + j] = inverse_scale(scale_byte(Tops::get(top, j)));
    }
  }
  __syncthreads();
  const float4 inv0 = reinterpret_cast<const float4*>(sh.col_inv)[2 * l], inv1 = reinterpret_cast<const float4*>(sh.col_inv)[2 * l + 1];
  const float inv[8] = {inv0.x, inv0.y, inv0.z, inv0.w, inv1.x, inv1.y, inv1.z, inv1.w};
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = scaled<CHECK>(o[i].get(j), inv[j]);
    *reinterpret_cast<uint2*>(sh.turned + (l * 8 + j) * 128 + ((team ^ l) << 3)) =
        make_uint2(e4m3x4(f[0], f[1], f[2], f[3]), e4m3x4(f[4], f[5], f[6], f[7]));
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < 128 * 8 / kQzThreads; ++u) {
    const int e = u * kQzThreads + tid, c = e >> 3, part = (e & 7) * 2, g = c >> 3;      // places part, part + 1 of column c
    uint4 v = *reinterpret_cast<const uint4*>(sh.turned + c * 128 + (((part ^ g) & ~1) << 3));
    if (g & 1) v = make_uint4(v.z, v.w, v.x, v.y);
    if (FULL || c0 + c < cols) {
      unsigned char* row = out_t.values + (long long)(c0 + c) * out_t.ld;
      const int i = r0 + part * 8;
      if (FULL || i + 16 <= rows) {
        *reinterpret_cast<uint4*>(row + i) = v;
      } else {
        put8(row, i, rows, v.x, v.y);
        put8(row, i + 8, rows, v.z, v.w);
      }
    }
  }
  if (tid < 128 && c0 + tid < cols) put_scale(out_t.scales, cols, c0 + tid, blockIdx.x, blocks_t, scale_of(sh.col_inv[tid]));
}

// A tile of 128 x 128: both forms, or either.  A team of 16 threads holds 8 rows, 8 columns a thread.  The transpose passes through shared memory
// as bytes: a thread writes the 8 bytes that its rows give a column; the 8-byte places of a column are exchanged by column group
// so that neither side meets a bank twice.  grid (row tiles, column tiles)
template <bool F32, bool VEC>
__global__ void __launch_bounds__(kQzThreads, F32 ? 2 : 4) fp8_tile_kernel(const __grid_constant__ Source m, int squares, Fp8Arg out, Fp8Arg out_t) {
  grid_enter();
  __shared__ __align__(16) TileShared sh;
  const int rows = m.rows, cols = m.cols;
  const int l = threadIdx.x & 15, team = threadIdx.x >> 4;
  Oct<F32> o[8];
  uint32_t tops[8], top = 0;
  typename Oct<F32>::Tops cols_top;
  const bool full = (blockIdx.x + 1) * 128 <= rows && (blockIdx.y + 1) * 128 <= cols;
  if (VEC && full) {
    const size_t at = (size_t)(blockIdx.x * 128 + team * 8) * m.ld + blockIdx.y * 128 + l * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i].load(m.x, at + i * m.ld);
  } else {
    const int row = blockIdx.x * 128 + team * 8, col = blockIdx.y * 128 + l * 8;
    if constexpr (VEC) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (row + i < rows) load8<F32, VEC>(m, (size_t)(row + i) * m.ld, col, o[i]);
        else o[i].zero();
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; i += 4) load_shifted<F32, 4, 0>(m, row + i, col, rows - row - i, m.ld * (F32 ? 4 : 2), o + i);
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    tops[i] = o[i].sweep(cols_top);
    top = max(top, tops[i]);
  }
  if (__syncthreads_or(top >= kInf)) quantize_tile<true, false, F32>(o, tops, cols_top, sh, rows, cols, squares, out, out_t);
  else if (full) quantize_tile<false, true, F32>(o, tops, cols_top, sh, rows, cols, squares, out, out_t);
  else quantize_tile<false, false, F32>(o, tops, cols_top, sh, rows, cols, squares, out, out_t);
}

}  // namespace

cudaError_t launch_fp8_quantize(const void* x, int x_f32, int rows, int cols, long long ld, bool squares, const Fp8Arg& out,
                                const Fp8Arg& out_t, cudaStream_t st) {
  const size_t bytes = x_f32 ? 4 : 2;
  const Source m{reinterpret_cast<const unsigned char*>(x), rows, cols, ld};
  const bool vec = (reinterpret_cast<uintptr_t>(x) & 15u) == 0 && (size_t)ld * bytes % 16 == 0;
  auto go = [&](auto rows_kernel, auto tile_kernel) {
    if (!squares && out_t.values == nullptr)
      return launch_kernel(rows_kernel, dim3((rows + 15) / 16, (cols + 511) / 512), kQzThreads, 0, st, m, out);
    return launch_kernel(tile_kernel, dim3((rows + 127) / 128, (cols + 127) / 128), kQzThreads, 0, st, m, squares ? 1 : 0, out, out_t);
  };
  if (x_f32) return vec ? go(fp8_rows_kernel<true, true>, fp8_tile_kernel<true, true>) : go(fp8_rows_kernel<true, false>, fp8_tile_kernel<true, false>);
  return vec ? go(fp8_rows_kernel<false, true>, fp8_tile_kernel<false, true>) : go(fp8_rows_kernel<false, false>, fp8_tile_kernel<false, false>);
}

}  // namespace vsa2
