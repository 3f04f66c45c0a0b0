// Arguments of the kernels between a layer's projection and its attention (qkv.cu), and the launchers of the 8-bit products
// (fp8_quantize.cu, fp8_matmul.cu).
#pragma once
#include "common.cuh"

namespace vsa2 {

// [batch, heads, tokens, D] with any strides (in elements); the D channels of a row are contiguous
struct HeadsArg {
  void* p;
  long long sb, sh, st;
  int heads;
};
struct HeadsPair { HeadsArg v[2]; };

// n / d for 0 <= n < 2^31 and 0 < d < 2^31 by a product and a shift: with l = ceil(log2 d) and m = ceil(2^(31 + l) / d), which has 32 bits, m d is less than 2^l above
// 2^(31 + l), so n m / 2^(31 + l) lies less than 1 / d above n / d
struct Divisor {
  uint32_t m;
  int l;
};
inline Divisor divisor(long long d) {
  const int l = d > 1 ? 64 - __builtin_clzll((unsigned long long)d - 1) : 0;
  return Divisor{(uint32_t)(((1ULL << (31 + l)) + (unsigned long long)d - 1) / (unsigned long long)d), l};
}
__device__ __forceinline__ int divided(int n, const Divisor& by) { return (int)(__umulhi(2u * (uint32_t)n, by.m) >> by.l); }

struct TurnArgs {
  unsigned long long turn[64];      // 2^-64 turns per position of every pair
  int pairs, pairs_t, pairs_th;     // pairs that turn; those below pairs_t turn with t, below pairs_th with h, the others with w
  int H, W;                         // grid, L = T H W
  Divisor by_H, by_W;
  long long L;
  int first;                        // row of the views' first token
  float sign;                       // -1: the inverse
  const int* positions;             // null: from the grid
  long long positions_sb;
};
struct QkvArgs {
  HeadsArg x[3], y[3];              // q, k, v: what is read, what is written
  const float* w[2];                // norm weights of q and k, null: ones
  float eps;
  int norm, tokens;
  int tiles, jobs, per_cta;         // (set by the launcher, with their divisors) token tiles of a batch entry and of all, heads per CTA
  Divisor by_tiles, by_jobs;
  TurnArgs turn;
};
size_t qkv_bwd_workspace_bytes(int D);
cudaError_t launch_qkv_fwd(QkvArgs a, int D, int batch, int in_f32, int out_f32, bool halves, cudaStream_t st);
cudaError_t launch_qkv_bwd(QkvArgs a, const HeadsPair& fwd, int D, int batch, int x_f32, int g_f32, int out_f32, bool halves,
                           float* dwq, float* dwk, float* partial, cudaStream_t st);

// e4m3 values [rows, ld] and their scales (exponent + 127), [ceil(cols / 512)][rows][4]
struct Fp8Arg {
  unsigned char* values;
  unsigned char* scales;
  long long ld;
};
cudaError_t launch_fp8_quantize(const void* x, int x_f32, int rows, int cols, long long ld, bool squares, const Fp8Arg& out,
                                const Fp8Arg& out_t, cudaStream_t st);

size_t fp8_matmul_workspace_bytes(int m, int n, int k);
// vsa2_debug_fp8_matmul_plan
void fp8_matmul_plan(int m, int n, int k, int c_f32, bool tensor_stores, int sms, bool pairs, int32_t* out);
cudaError_t launch_fp8_matmul(int m, int n, int k, const Fp8Arg& a, const Fp8Arg& b, void* c, int c_f32, long long ldc,
                              void* workspace, cudaStream_t st);

}  // namespace vsa2
