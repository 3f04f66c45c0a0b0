// y = (residual +) x / (1 - p) where an element is kept, zero (or the residual) elsewhere; its own backward.  The mask is formed from a counter
// (rows.cuh), never stored.  Bound by memory: x, the residual and y once each.
#include "rows.cuh"

namespace vsa2 {

namespace {

constexpr int kDropThreads = 256;
constexpr int kDropOcts = 4;      // pieces of eight elements a thread, all asked for before the first is used

template <typename X, typename Y, int LIE>
__global__ void __launch_bounds__(kDropThreads) dropout_kernel(const __grid_constant__ DropoutArgs a) {
  grid_enter();
  DropMask mask;
  mask.init(a.drop);
  // pieces in the order of the rows; the first of this CTA's in 64 bits, the others from there
  // (less than 2^40 pieces in all, 2^20 in a row: the product with 2^64 / octs is exact)
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
    if (row[u] < a.rows) load_eight<LIE>(x[u], reinterpret_cast<const X*>(a.x.p) + row[u] * a.x.ld, oct[u] * 8, a.cols);
    else x[u].zero();
  }
  if (a.r.p != nullptr) {
#pragma unroll
    for (int u = 0; u < kDropOcts; ++u) {
      if (row[u] < a.rows) load_eight<LIE>(r[u], reinterpret_cast<const Y*>(a.r.p) + row[u] * a.r.ld, oct[u] * 8, a.cols);
      else r[u].zero();
    }
  }
#pragma unroll
  for (int u = 0; u < kDropOcts; ++u) {
    float f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = x[u].get(j);
    mask.apply(f, row[u], oct[u]);
    if (a.r.p != nullptr) add_eight(f, r[u]);
    if (row[u] < a.rows) store_floats<LIE>(f, reinterpret_cast<Y*>(a.y.p) + row[u] * a.y.ld, oct[u] * 8, a.cols);
  }
}

}  // namespace

cudaError_t launch_dropout(DropoutArgs a, bool x_f32, bool y_f32, cudaStream_t st) {
  a.octs = (a.cols + 7) / 8;
  a.by_octs = divisor(a.octs);
  a.per_octs = ~0ULL / a.octs + 1;
  const long long octs = (long long)a.rows * a.octs, per = kDropThreads * kDropOcts;
  const unsigned grid = (unsigned)((octs + per - 1) / per);
  const size_t size = y_f32 ? 4 : 2;
  const bool vec = a.cols % 8 == 0 && rows_aligned(a.x, x_f32 ? 4 : 2) && rows_aligned(a.r, size) && rows_aligned(a.y, size);
  auto go = [&](auto aligned, auto any) { return launch_kernel(vec ? aligned : any, grid, kDropThreads, 0, st, a); };
  if (x_f32) return y_f32 ? go(dropout_kernel<float, float, ROWS_ALIGNED>, dropout_kernel<float, float, ROWS_ANY>) : go(dropout_kernel<float, bf16, ROWS_ALIGNED>, dropout_kernel<float, bf16, ROWS_ANY>);
  return y_f32 ? go(dropout_kernel<bf16, float, ROWS_ALIGNED>, dropout_kernel<bf16, float, ROWS_ANY>) : go(dropout_kernel<bf16, bf16, ROWS_ALIGNED>, dropout_kernel<bf16, bf16, ROWS_ANY>);
}

}  // namespace vsa2
