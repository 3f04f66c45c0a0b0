// y = (residual +) x / (1 - p) where an element is kept, zero (or the residual) elsewhere; its own backward.  The mask is formed from a counter
// (rows.cuh), never stored.  Bound by memory: x, the residual and y once each; 75600 x 5120 bf16 with residual 329 - 360 us (6.5 - 7.1 TB/s, passes that follow one another
// included), with ten rounds of the generator for eight elements in the issue slots beside it (52 %).
#include "rows.cuh"

namespace vsa2 {

namespace {

constexpr int kDropThreads = 256;
constexpr int kAnyOcts = 2;       // .. of rows that lie anywhere
// pieces of eight elements a thread, all asked for before the first is used: as many as 64 registers nearly hold (bf16 to bf16 puts 4 bytes a thread aside, 36 where
// rows are strided; four CTAs an SM: 75600 x 5120 with residual 361 us, three of 68 registers 382)
template <typename X, typename Y> constexpr int kDropOcts = sizeof(X) + sizeof(Y) == 4 ? 4 : 2;

// pieces of x through the dropout, plus r where there is one (y may be r)
template <int N, typename X, typename Y>
__device__ __forceinline__ void dropped(Eight<Y> (&y)[N], const Eight<X> (&x)[N], const Eight<Y> (&r)[N], bool residual, const DropMask& mask, const uint32_t (&row)[N],
                                        const uint32_t (&oct)[N]) {
  uint32_t w[N][4];
  if (mask.limit != 0) mask.words(w, row, oct);
#pragma unroll
  for (int u = 0; u < N; ++u) {
    float f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = x[u].get(j);
    if (mask.limit != 0) mask.keep(f, w[u]);
    if (residual) add_eight(f, r[u]);
    y[u].round(f);
  }
}

// Rows on 16-byte boundaries and in whole pieces: pieces in the order of the rows, whatever these are.  FLAT: the rows of all matrices lie right behind one another, and so do a thread's
// pieces, whatever row they are of.  (A CTA whose pieces all exist looks at none of them.)
template <typename X, typename Y, bool FLAT>
__global__ void __launch_bounds__(kDropThreads, 4) dropout_kernel(const __grid_constant__ DropoutArgs a) {
  grid_enter();
  constexpr int N = kDropOcts<X, Y>;
  DropMask mask;
  mask.init(a.drop);
  // the first of this CTA's pieces in 64 bits, the others from there (less than 2^40 pieces in all, 2^20 in a row: the product with 2^64 / octs is exact)
  constexpr int TILE = kDropThreads * N;
  const long long first = (long long)blockIdx.x * TILE, row0 = a.octs == 1 ? first : (long long)__umul64hi(first, a.per_octs);
  const long long total = (long long)a.rows * a.octs;
  const int skip = (int)(first - row0 * a.octs) + threadIdx.x;
  const bool whole = first + TILE <= total;
  Eight<X> x[N];
  Eight<Y> y[N];
  uint32_t row[N], oct[N];
  bool there[N];
#pragma unroll
  for (int u = 0; u < N; ++u) {
    const int at = skip + u * kDropThreads, down = divided(at, a.by_octs);
    row[u] = (uint32_t)(row0 + down);
    oct[u] = (uint32_t)(at - down * a.octs);
    there[u] = whole || first + threadIdx.x + u * kDropThreads < total;
  }
  auto place = [&](const RowsArg& m, auto* type, int u) {
    auto* p = reinterpret_cast<decltype(type)>(m.p);
    return FLAT ? p + (first + threadIdx.x) * 8 + u * (kDropThreads * 8) : p + row[u] * m.ld + oct[u] * 8;
  };
#pragma unroll
  for (int u = 0; u < N; ++u) {
    if (there[u]) x[u].load(place(a.x, (X*)nullptr, u));
    else x[u].zero();
  }
  if (a.r.p != nullptr) {
#pragma unroll
    for (int u = 0; u < N; ++u) {
      if (there[u]) y[u].load(place(a.r, (Y*)nullptr, u));
      else y[u].zero();
    }
  }
  dropped(y, x, y, a.r.p != nullptr, mask, row, oct);
#pragma unroll
  for (int u = 0; u < N; ++u)
    if (there[u]) y[u].store(place(a.y, (Y*)nullptr, u));
}
// Any rows: a warp takes up to 32 kAnyOcts neighbouring pieces of one
template <typename X, typename Y>
__global__ void __launch_bounds__(kDropThreads) dropout_any_kernel(const __grid_constant__ DropoutArgs a, int parts) {
  grid_enter();
  DropMask mask;
  mask.init(a.drop);
  const long long unit = (long long)blockIdx.x * (kDropThreads / 32) + (threadIdx.x >> 5), at = unit / parts;
  if (at >= a.rows) return;
  const int row = (int)at, first = (int)(unit - at * parts) * (32 * kAnyOcts) + (threadIdx.x & 31);
  Eight<X> x[kAnyOcts];
  Eight<Y> y[kAnyOcts];
  uint32_t rows[kAnyOcts], octs[kAnyOcts];
#pragma unroll
  for (int u = 0; u < kAnyOcts; ++u) {
    rows[u] = row;
    octs[u] = first + 32 * u;
    load_eight<ROWS_ANY>(x[u], reinterpret_cast<const X*>(a.x.p) + row * a.x.ld, (first + 32 * u) * 8, a.cols);
  }
  if (a.r.p != nullptr) {
#pragma unroll
    for (int u = 0; u < kAnyOcts; ++u) load_eight<ROWS_ANY>(y[u], reinterpret_cast<const Y*>(a.r.p) + row * a.r.ld, (first + 32 * u) * 8, a.cols);
  }
  dropped(y, x, y, a.r.p != nullptr, mask, rows, octs);
#pragma unroll
  for (int u = 0; u < kAnyOcts; ++u)
    store_eight<ROWS_ANY, kAnyOcts>(y[u], y[u > 0 ? u - 1 : 0], u, reinterpret_cast<Y*>(a.y.p) + row * a.y.ld, (first + 32 * u) * 8, a.cols);
}

}  // namespace

cudaError_t launch_dropout(DropoutArgs a, bool x_f32, bool y_f32, cudaStream_t st) {
  a.octs = (a.cols + 7) / 8;
  a.by_octs = divisor(a.octs);
  a.per_octs = ~0ULL / a.octs + 1;
  const size_t size = y_f32 ? 4 : 2;
  const bool vec = a.cols % 8 == 0 && rows_aligned(a.x, x_f32 ? 4 : 2) && rows_aligned(a.r, size) && rows_aligned(a.y, size);
  const int parts = (a.octs + 32 * kAnyOcts - 1) / (32 * kAnyOcts);
  const long long octs = (long long)a.rows * a.octs, units = (long long)a.rows * parts, warps = kDropThreads / 32;
  const bool flat = a.rows == 1 || (a.x.ld == a.cols && a.y.ld == a.cols && (a.r.p == nullptr || a.r.ld == a.cols));
  auto go = [&](auto x, auto y) {
    using X = decltype(x);
    using Y = decltype(y);
    const long long per = kDropThreads * kDropOcts<X, Y>;
    if (!vec) return launch_kernel(dropout_any_kernel<X, Y>, (unsigned)((units + warps - 1) / warps), kDropThreads, 0, st, a, parts);
    return launch_kernel(flat ? dropout_kernel<X, Y, true> : dropout_kernel<X, Y, false>, (unsigned)((octs + per - 1) / per), kDropThreads, 0, st, a);
  };
  if (x_f32) return y_f32 ? go(0.f, 0.f) : go(0.f, bf16());
  return y_f32 ? go(bf16(), 0.f) : go(bf16(), bf16());
}

}  // namespace vsa2
