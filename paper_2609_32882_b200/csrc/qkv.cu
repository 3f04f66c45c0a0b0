// From a layer's projection to its attention and back: the rows of q, k and v as a projection leaves them (token after token) become the
// heads that the attention reads ([batch, heads, tokens, D]), q and k normed and turned on the way.
//   forward : y = R(position) (x r w),  r = 1 / sqrt(mean(x^2) + eps) over the D channels of a head;  v is copied
//   backward: g = R(position)^-1 dy;  dw = sum g x r;  dx = r (w g) - x r^3 mean((w g) x)
// R turns pair p of a head's channels by (position on the pair's axis) * (its frequency); the inverse turns back, and is R's gradient too.
//
// Angles.  A frequency is held as a fraction of a turn in 64 bits (2^-64 turns per position).  The product with an integer position,
// modulo 2^64, is the angle modulo a turn without any rounding, however far the position; its upper half, 2^-32 turns, goes to sincospi.
// (In fp32, position * frequency alone is 2^-24 of the angle off: 4e-3 at position 65,536.)
//
// All of it is bound by memory: every element is read once and written once, the few operations hide behind that.  A team of D / 8
// threads holds one row of one head, 8 channels a thread; it keeps its token and walks through the heads, so that a token's sines and
// cosines (and the norm weights) are formed once, and the reads of a CTA's tokens are whole rows of the projection.
#include "common.cuh"
#include "heads.cuh"

namespace vsa2 {

namespace {

constexpr int kQkvThreads = 256;
constexpr int kQkvParts = 1024;      // most CTAs of the backward, each with its own partial sums of the weights' gradients

template <typename T> struct Raw8;      // eight channels as they lie in memory
template <> struct Raw8<bf16> {
  uint4 v;
  __device__ __forceinline__ void load(const bf16* p) { v = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(u[i] << 16);
      f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  }
};
template <> struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = reinterpret_cast<const float4*>(p)[0];
    b = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
    f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
  }
};
__device__ __forceinline__ void store8(bf16* p, const float (&f)[8]) {
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(u[i]) : "f"(f[2 * i + 1]), "f"(f[2 * i]));
  *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
}
__device__ __forceinline__ void store8(float* p, const float (&f)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}

// Sines and cosines of the pairs that a thread's channels 8l .. 8l+7 belong to, at one token.
// Neighbours as pairs: pairs 4l .. 4l+3, both channels in the thread.  Halves as pairs: the partner of channel c is c + P or c - P, in
// the same place of another thread of the team (P is a multiple of 8).
template <int D, bool HALVES>
struct Turn {
  static constexpr int N = HALVES ? 8 : 4;
  float c[N], s[N];
  int partner;      // lane of the warp (HALVES)

  __device__ __forceinline__ void init(const TurnArgs& t, int b, int tok, int l) {
    int pos[3] = {0, 0, 0};
    bool turns = t.pairs > 0;
    if (t.positions != nullptr) {
      const int* p = t.positions + b * t.positions_sb + (long long)tok * 3;
      pos[0] = p[0]; pos[1] = p[1]; pos[2] = p[2];
    } else {
      const long long r = (long long)t.first + tok;
      turns = turns && r < t.L;
      if (turns) {
        const int rr = (int)r, th = rr / t.W;
        pos[2] = rr - th * t.W;
        pos[0] = th / t.H;
        pos[1] = th - pos[0] * t.H;
      }
    }
    const int lane = threadIdx.x & 31;
    partner = lane;
    if (HALVES) {
      const int chunk = t.pairs >> 3;
      partner = l < chunk ? lane + chunk : l < 2 * chunk ? lane - chunk : lane;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      int p = HALVES ? l * 8 + i : l * 4 + i;
      float sign = t.sign;
      if (HALVES) {
        if (p < t.pairs) sign = -sign;      // (the first half: x cos - partner sin)
        else p -= t.pairs;
      }
      c[i] = 1.f;
      s[i] = 0.f;
      if (turns && p < t.pairs) {
        const int at = p < t.pairs_t ? pos[0] : p < t.pairs_th ? pos[1] : pos[2];
        const unsigned long long angle = t.turn[p] * (unsigned long long)(long long)at;
        float sn, cs;
        sincospif((float)(int)(angle >> 32) * 0x1p-31f, &sn, &cs);
        c[i] = cs;
        s[i] = sign * sn;
      }
    }
  }
  // (by all threads of a warp together)
  __device__ __forceinline__ void apply(float (&f)[8]) const {
    if (HALVES) {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = f[i] * c[i % N] + __shfl_sync(0xffffffffu, f[i], partner) * s[i % N];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = f[2 * i], y = f[2 * i + 1];
        f[2 * i] = x * c[i % N] - y * s[i % N];
        f[2 * i + 1] = x * s[i % N] + y * c[i % N];
      }
    }
  }
};

template <int TEAM>
__device__ __forceinline__ float team_sum(float v) {
#pragma unroll
  for (int o = TEAM / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// grid (token tiles of all batch entries, 1, groups of heads)
template <int D, typename TI, typename TO, bool HALVES>
__global__ void __launch_bounds__(kQkvThreads) qkv_fwd_kernel(const __grid_constant__ QkvArgs a) {
  constexpr int TEAM = D / 8, ROWS = kQkvThreads / TEAM, U = sizeof(TI) == 2 ? 4 : 2;
  grid_enter();
  const int l = threadIdx.x % TEAM;
  const int b = blockIdx.x / a.tiles, tile = blockIdx.x - b * a.tiles;
  const int row = tile * ROWS + threadIdx.x / TEAM;
  const bool valid = row < a.tokens;
  const int tok = min(row, a.tokens - 1);
  Turn<D, HALVES> turn;
  turn.init(a.turn, b, tok, l);
  const int h_lo = blockIdx.z * a.per_cta, h_hi = h_lo + a.per_cta;
  int base = 0;
#pragma unroll 1
  for (int seg = 0; seg < 3; ++seg) {
    const HeadsArg x = a.x[seg], y = a.y[seg];
    const int lo = max(h_lo - base, 0), hi = min(h_hi - base, x.heads);
    base += x.heads;
    if (lo >= hi) continue;
    const bool norm = a.norm && seg < 2, rotate = seg < 2;
    float w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = norm && a.w[seg & 1] != nullptr ? a.w[seg & 1][l * 8 + i] : 1.f;
    const TI* xp = reinterpret_cast<const TI*>(x.p) + b * x.sb + tok * x.st + l * 8;
    TO* yp = reinterpret_cast<TO*>(y.p) + b * y.sb + tok * y.st + l * 8;
    for (int h = lo; h < hi; h += U) {
      Raw8<TI> raw[U];
#pragma unroll
      for (int u = 0; u < U; ++u) raw[u].load(xp + min(h + u, hi - 1) * x.sh);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float f[8];
        raw[u].get(f);
        if (norm) {
          float ss = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) ss += f[i] * f[i];
          const float r = rsqrtf(team_sum<TEAM>(ss) * (1.f / D) + a.eps);
#pragma unroll
          for (int i = 0; i < 8; ++i) f[i] *= r * w[i];
        }
        if (rotate) turn.apply(f);
        if (valid && h + u < hi) store8(yp + (h + u) * y.sh, f);
      }
    }
  }
}

// grid (CTAs that walk through the token tiles, 1, groups of heads); x = the forward's rows of q and k, dy -> dx
template <int D, typename TI, typename TG, typename TO, bool HALVES>
__global__ void __launch_bounds__(kQkvThreads) qkv_bwd_kernel(const __grid_constant__ QkvArgs a, const __grid_constant__ HeadsPair fwd,
                                                              float* __restrict__ partial) {
  constexpr int TEAM = D / 8, ROWS = kQkvThreads / TEAM, U = 2;
  grid_enter();
  __shared__ float red[2][ROWS][D];
  const int l = threadIdx.x % TEAM, slot = threadIdx.x / TEAM;
  const int h_lo = blockIdx.z * a.per_cta, h_hi = h_lo + a.per_cta;
  float dw[2][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) dw[0][i] = dw[1][i] = 0.f;
  for (int job = blockIdx.x; job < a.jobs; job += gridDim.x) {
    const int b = job / a.tiles, tile = job - b * a.tiles;
    const int row = tile * ROWS + slot;
    const bool valid = row < a.tokens;
    const int tok = min(row, a.tokens - 1);
    Turn<D, HALVES> turn;
    turn.init(a.turn, b, tok, l);
    int base = 0;
#pragma unroll
    for (int seg = 0; seg < 3; ++seg) {
      const HeadsArg g = a.x[seg], y = a.y[seg];
      const int lo = max(h_lo - base, 0), hi = min(h_hi - base, g.heads);
      base += g.heads;
      if (lo >= hi) continue;
      const bool norm = a.norm && seg < 2;
      const TG* gp = reinterpret_cast<const TG*>(g.p) + b * g.sb + tok * g.st + l * 8;
      TO* yp = reinterpret_cast<TO*>(y.p) + b * y.sb + tok * y.st + l * 8;
      const HeadsArg x = fwd.v[seg & 1];
      const TI* xp = reinterpret_cast<const TI*>(x.p) + b * x.sb + tok * x.st + l * 8;
      float w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = norm && a.w[seg & 1] != nullptr ? a.w[seg & 1][l * 8 + i] : 1.f;
      Raw8<TG> g_next[U];
      Raw8<TI> x_next[U];
      auto fetch = [&](int h) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
          g_next[u].load(gp + min(h + u, hi - 1) * g.sh);
          if (norm) x_next[u].load(xp + min(h + u, hi - 1) * x.sh);
        }
      };
      fetch(lo);
      for (int h = lo; h < hi; h += U) {
        // (the next heads' rows are on their way while these are computed)
        Raw8<TG> gr[U];
        Raw8<TI> xr[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          gr[u] = g_next[u];
          xr[u] = x_next[u];
        }
        if (h + U < hi) fetch(h + U);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float f[8];
          gr[u].get(f);
          if (seg < 2) turn.apply(f);
          if (norm) {
            float xf[8], ss = 0.f, dot = 0.f;
            xr[u].get(xf);
            const bool counts = valid && h + u < hi;
            float g0[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              g0[i] = f[i];
              f[i] *= w[i];
              ss += xf[i] * xf[i];
              dot += f[i] * xf[i];
            }
            ss = team_sum<TEAM>(ss);
            dot = team_sum<TEAM>(dot);
            const float r = rsqrtf(ss * (1.f / D) + a.eps);
            const float m = dot * (1.f / D) * r * r * r;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              if (counts) dw[seg & 1][i] += g0[i] * (xf[i] * r);
              f[i] = r * f[i] - xf[i] * m;
            }
          }
          if (valid && h + u < hi) store8(yp + (h + u) * y.sh, f);
        }
      }
    }
  }
  if (!a.norm) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    red[0][slot][l * 8 + i] = dw[0][i];
    red[1][slot][l * 8 + i] = dw[1][i];
  }
  __syncthreads();
  const size_t cta = (size_t)blockIdx.z * gridDim.x + blockIdx.x;
  for (int i = threadIdx.x; i < 2 * D; i += kQkvThreads) {
    float sum = 0.f;
    for (int r = 0; r < ROWS; ++r) sum += red[i / D][r][i % D];
    partial[cta * (2 * D) + i] = sum;
  }
}

// Sums of the CTAs' partial sums in a fixed order: 32 columns a CTA, every 32nd part a warp row.
__global__ void __launch_bounds__(1024) qkv_bwd_reduce_kernel(const float* partial, int parts, int D, float* __restrict__ dwq,
                                                              float* __restrict__ dwk) {
  grid_enter();
  __shared__ float red[32][33];
  const int col = blockIdx.x * 32 + (threadIdx.x & 31), first = threadIdx.x >> 5;
  float sum = 0.f;
  for (int p = first; p < parts; p += 32) sum += partial[(size_t)p * (2 * D) + col];
  red[first][threadIdx.x & 31] = sum;
  __syncthreads();
  if (first == 0) {
    float total = 0.f;
    for (int r = 0; r < 32; ++r) total += red[r][threadIdx.x];
    float* out = col < D ? dwq : dwk;
    if (out != nullptr) out[col < D ? col : col - D] = total;
  }
}

template <typename F>
cudaError_t by_types(int in_f32, int out_f32, F f) {
  if (in_f32) return out_f32 ? f(float(), float()) : f(float(), bf16());
  return out_f32 ? f(bf16(), float()) : f(bf16(), bf16());
}

// groups of heads so that there are about four CTAs per SM where the tokens alone do not give them
int heads_per_cta(int tiles, int heads, int unit, int sms) {
  int groups = (4 * sms + tiles - 1) / tiles;
  const int most = (heads + unit - 1) / unit;
  groups = groups < 1 ? 1 : groups > most ? most : groups;
  return (heads + groups - 1) / groups;
}

}  // namespace

size_t qkv_bwd_workspace_bytes(int D) { return (size_t)kQkvParts * 2 * D * sizeof(float); }

cudaError_t launch_qkv_fwd(QkvArgs a, int D, int batch, int in_f32, int out_f32, bool halves, cudaStream_t st) {
  const int rows = kQkvThreads / (D / 8), heads = a.x[0].heads + a.x[1].heads + a.x[2].heads;
  int sms = 0;
  cudaError_t e;
  if ((e = sm_count(&sms)) != cudaSuccess) return e;
  a.tiles = (a.tokens + rows - 1) / rows;
  a.jobs = a.tiles * batch;
  a.per_cta = heads_per_cta(a.jobs, heads, in_f32 ? 2 : 4, sms);
  const dim3 grid(a.jobs, 1, (heads + a.per_cta - 1) / a.per_cta);
  return by_types(in_f32, out_f32, [&](auto ti, auto to) {
    using TI = decltype(ti);
    using TO = decltype(to);
    if (D == 128) return halves ? launch_kernel(qkv_fwd_kernel<128, TI, TO, true>, grid, kQkvThreads, 0, st, a)
                                : launch_kernel(qkv_fwd_kernel<128, TI, TO, false>, grid, kQkvThreads, 0, st, a);
    return halves ? launch_kernel(qkv_fwd_kernel<64, TI, TO, true>, grid, kQkvThreads, 0, st, a)
                  : launch_kernel(qkv_fwd_kernel<64, TI, TO, false>, grid, kQkvThreads, 0, st, a);
  });
}

cudaError_t launch_qkv_bwd(QkvArgs a, const HeadsPair& fwd, int D, int batch, int x_f32, int g_f32, int out_f32, bool halves,
                           float* dwq, float* dwk, float* partial, cudaStream_t st) {
  const int rows = kQkvThreads / (D / 8), heads = a.x[0].heads + a.x[1].heads + a.x[2].heads;
  int sms = 0;
  cudaError_t e;
  if ((e = sm_count(&sms)) != cudaSuccess) return e;
  a.tiles = (a.tokens + rows - 1) / rows;
  a.jobs = a.tiles * batch;
  a.per_cta = heads_per_cta(a.jobs, heads, 2, sms);
  const int groups = (heads + a.per_cta - 1) / a.per_cta;
  int ctas = a.jobs;
  if (ctas > kQkvParts / groups) ctas = kQkvParts / groups;
  const dim3 grid(ctas, 1, groups);
  auto go = [&](auto tx, auto tg, auto to) {
    using TX = decltype(tx);
    using TG = decltype(tg);
    using TO = decltype(to);
    if (D == 128) return halves ? launch_kernel(qkv_bwd_kernel<128, TX, TG, TO, true>, grid, kQkvThreads, 0, st, a, fwd, partial)
                                : launch_kernel(qkv_bwd_kernel<128, TX, TG, TO, false>, grid, kQkvThreads, 0, st, a, fwd, partial);
    return halves ? launch_kernel(qkv_bwd_kernel<64, TX, TG, TO, true>, grid, kQkvThreads, 0, st, a, fwd, partial)
                  : launch_kernel(qkv_bwd_kernel<64, TX, TG, TO, false>, grid, kQkvThreads, 0, st, a, fwd, partial);
  };
  e = by_types(g_f32, out_f32, [&](auto tg, auto to) { return x_f32 ? go(float(), tg, to) : go(bf16(), tg, to); });
  if (e != cudaSuccess || !a.norm) return e;
  return launch_kernel(qkv_bwd_reduce_kernel, 2 * D / 32, 1024, 0, st, partial, ctas * groups, D, dwq, dwk);
}

}  // namespace vsa2
