// y = (residual +) x / (1 - p) where an element is kept, zero (or the residual) elsewhere; its own backward.  The mask is formed from a counter
// (rows.cuh), never stored.  Bound by memory: x, the residual and y once each; 75600 x 5120 bf16 with residual 329 - 400 us (5.8 - 7.1 TB/s, passes that follow one another
// included), with ten rounds of the generator for eight elements in the issue slots beside it (71 %).
#include "rows.cuh"

namespace vsa2 {

namespace {

constexpr int kDropThreads = 256;
constexpr int kAnyOcts = 2;       // .. of rows that lie anywhere
constexpr int kDropOcts = 4;      // pieces of eight elements a thread, all asked for before the first is used

// x through the dropout, plus r where there is one
template <typename X, typename Y>
__device__ __forceinline__ void dropped(Eight<Y>& y, const Eight<X>& x, const Eight<Y>& r, bool residual, const DropMask& mask, int row, int oct) {
  float f[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) f[j] = x.get(j);
  mask.apply(f, row, oct);
  if (residual) add_eight(f, r);
  y.round(f);
}

// Rows on 16-byte boundaries and in whole pieces: pieces in the order of the rows, whatever these are
template <typename X, typename Y>
__global__ void __launch_bounds__(kDropThreads) dropout_kernel(const __grid_constant__ DropoutArgs a) {
  grid_enter();
  DropMask mask;
  mask.init(a.drop);
  // the first of this CTA's pieces in 64 bits, the others from there (less than 2^40 pieces in all, 2^20 in a row: the product with 2^64 / octs is exact)
  const long long first = (long long)blockIdx.x * (kDropThreads * kDropOcts), row0 = a.octs == 1 ? first : (long long)__umul64hi(first, a.per_octs);
  const int skip = (int)(first - row0 * a.octs) + threadIdx.x;
  Eight<X> x[kDropOcts];
  Eight<Y> r[kDropOcts];
  int row[kDropOcts], oct[kDropOcts];
#pragma unroll
  for (int u = 0; u < kDropOcts; ++u) {
    const int at = skip + u * kDropThreads, down = divided(at, a.by_octs);
    row[u] = (int)min((long long)a.rows, row0 + down);
    oct[u] = at - down * a.octs;
    if (row[u] < a.rows) x[u].load(reinterpret_cast<const X*>(a.x.p) + row[u] * a.x.ld + oct[u] * 8);
    else x[u].zero();
  }
  if (a.r.p != nullptr) {
#pragma unroll
    for (int u = 0; u < kDropOcts; ++u) {
      if (row[u] < a.rows) r[u].load(reinterpret_cast<const Y*>(a.r.p) + row[u] * a.r.ld + oct[u] * 8);
      else r[u].zero();
    }
  }
#pragma unroll
  for (int u = 0; u < kDropOcts; ++u) {
    Eight<Y> y;
    dropped(y, x[u], r[u], a.r.p != nullptr, mask, row[u], oct[u]);
    if (row[u] < a.rows) y.store(reinterpret_cast<Y*>(a.y.p) + row[u] * a.y.ld + oct[u] * 8);
  }
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
#pragma unroll
  for (int u = 0; u < kAnyOcts; ++u) load_eight<ROWS_ANY>(x[u], reinterpret_cast<const X*>(a.x.p) + row * a.x.ld, (first + 32 * u) * 8, a.cols);
  if (a.r.p != nullptr) {
#pragma unroll
    for (int u = 0; u < kAnyOcts; ++u) load_eight<ROWS_ANY>(y[u], reinterpret_cast<const Y*>(a.r.p) + row * a.r.ld, (first + 32 * u) * 8, a.cols);
  }
#pragma unroll
  for (int u = 0; u < kAnyOcts; ++u) dropped(y[u], x[u], y[u], a.r.p != nullptr, mask, row, first + 32 * u);
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
  const long long octs = (long long)a.rows * a.octs, units = (long long)a.rows * parts, per = kDropThreads * kDropOcts, warps = kDropThreads / 32;
  auto go = [&](auto aligned, auto any) {
    return vec ? launch_kernel(aligned, (unsigned)((octs + per - 1) / per), kDropThreads, 0, st, a)
               : launch_kernel(any, (unsigned)((units + warps - 1) / warps), kDropThreads, 0, st, a, parts);
  };
  if (x_f32) return y_f32 ? go(dropout_kernel<float, float>, dropout_any_kernel<float, float>) : go(dropout_kernel<float, bf16>, dropout_any_kernel<float, bf16>);
  return y_f32 ? go(dropout_kernel<bf16, float>, dropout_any_kernel<bf16, float>) : go(dropout_kernel<bf16, bf16>, dropout_any_kernel<bf16, bf16>);
}

}  // namespace vsa2
