// From a layer's projection to its attention and back: the rows of q, k and v as a projection leaves them (token after token) become the
// heads that the attention reads ([batch, heads, tokens, D]), q and k normed and turned on the way.
//   forward : y = R(position) (x r w),  r = 1 / sqrt(mean(x^2) + eps) over the D channels of a head;  v is copied
//   backward: g = R(position)^-1 dy;  dw = sum g x r;  dx = r (w g) - x r^3 mean((w g) x)
// R turns pair p of a head's channels by (position on the pair's axis) * (its frequency); the inverse turns back, and is R's gradient too.
//
// Angles.  A frequency is held as a fraction of a turn in 64 bits (2^-64 turns per position).  The product with an integer position, modulo 2^64, is the angle modulo a turn: the
// product itself is exact however far the position, so what is off is the frequency's own rounding times the position (2^-33 turns at 2^31) and what goes to sincospi, the upper half
// (2^-32 turns) rounded to fp32's 24 bits: 2^-26 turns at most (9.4e-8 rad, near half a turn), as an fp32 angle of that size is.  (In fp32, position * frequency alone is 2^-24 of the
// angle off: 4e-3 at position 65,536.)
//
// All of it is bound by memory: every element is read once and written once, the few operations hide behind that.  A team of D / 8
// threads holds one row of one head, 8 channels a thread; it keeps its token and walks through the heads, so that a token's sines and
// cosines (and the norm weights) are formed once, and the reads of a CTA's tokens are whole rows of the projection.  At 75,600 tokens: rotation of 40
// heads 239 us (6.5 TB/s), norms, rotation and heads of 3 x 40 heads 736 us (6.3 TB/s), backward of 3 x 20 heads 485 - 494 us (6.3 TB/s); a copy reaches 6.45.
// With few tokens it is the latency of one row (2048 tokens, 3 x 12 heads: 8.7 us; 256 tokens, 3 x 2: 3.6 us).
#include "common.cuh"
#include "heads.cuh"

namespace vsa2 {

namespace {

constexpr int kQkvThreads = 256;
// Rows of `pieces` times 16 bytes that a thread of the backward has in its queue.  720p, 20 heads: two 558 us, three 487, four 536, six 513; with halves as pairs, whose
// registers leave room for three CTAs per SM instead of four, 480p, 24 heads: three 276, four 262
__host__ __device__ constexpr int bwd_ahead(int pieces, bool halves) { return pieces > 2 ? 2 : halves ? 4 : 3; }
constexpr int kQkvParts = 1024;      // most CTAs of the backward, each with its own partial sums of a weight's gradient

template <typename T> struct Raw8;      // eight channels as they lie in memory
template <> struct Raw8<bf16> {
  uint4 v;
  __device__ __forceinline__ void load(const bf16* p) { v = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void load(const uint4* p, int) { v = *p; }      // (pieces `apart` from one another)
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
  __device__ __forceinline__ void load(const uint4* p, int apart) {
    a = *reinterpret_cast<const float4*>(p);
    b = *reinterpret_cast<const float4*>(p + apart);
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
  int active;       // pairs of this thread that turn (HALVES: all 8 or none); the other channels stay as they are, infinities among them

  // `turns`: t.turn, in shared memory
  __device__ __forceinline__ void init(const TurnArgs& t, const unsigned long long* turns, int b, int tok, int l) {
    int pos[3] = {0, 0, 0};
    active = HALVES ? (l * 4 < t.pairs ? N : 0) : min(max(t.pairs - l * N, 0), N);
    if (t.positions != nullptr) {
      const int* p = t.positions + b * t.positions_sb + (long long)tok * 3;
      pos[0] = p[0]; pos[1] = p[1]; pos[2] = p[2];
    } else {
      const long long r = (long long)t.first + tok;
      if (r < t.L) {
        const int rr = (int)r, th = divided(rr, t.by_W);
        pos[2] = rr - th * t.W;
        pos[0] = divided(th, t.by_H);
        pos[1] = th - pos[0] * t.H;
      } else {
        active = 0;
      }
    }
    int p0 = l * N;                     // the thread's first pair
    float sign = t.sign;
    if (HALVES) {
      const int lane = threadIdx.x & 31, chunk = t.pairs >> 3;
      partner = l < chunk ? lane + chunk : l < 2 * chunk ? lane - chunk : lane;
      if (p0 < t.pairs) sign = -sign;   // (the first half: x cos - partner sin)
      else p0 -= t.pairs;
    }
    if (active > 0) {
#pragma unroll
      for (int i = 0; i < N; i += 2) {
        const ulonglong2 both = *reinterpret_cast<const ulonglong2*>(turns + p0 + i);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const unsigned long long turn = k == 0 ? both.x : both.y;
          const int p = p0 + i + k, at = p < t.pairs_t ? pos[0] : p < t.pairs_th ? pos[1] : pos[2];
          // upper half of turn * at modulo 2^64
          const uint32_t lo = (uint32_t)turn, angle = (uint32_t)(turn >> 32) * (uint32_t)at + __umulhi(lo, (uint32_t)at) - (at < 0 ? lo : 0u);
          float sn, cs;
          sincospif((float)(int)angle * 0x1p-31f, &sn, &cs);
          c[i + k] = cs;
          s[i + k] = sign * sn;
        }
      }
    }
  }
  // (by all threads of a warp together)
  __device__ __forceinline__ void apply(float (&f)[8]) const {
    if (HALVES) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float other = __shfl_sync(0xffffffffu, f[i], partner);
        if (active > 0) f[i] = f[i] * c[i % N] + other * s[i % N];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i >= active) continue;
        const float x = f[2 * i], y = f[2 * i + 1];
        f[2 * i] = x * c[i % N] - y * s[i % N];
        f[2 * i + 1] = x * s[i % N] + y * c[i % N];
      }
    }
  }
};

// t.turn for the CTA's threads.  (A warp that reads the kernel's arguments at 16 places waits for one after the other: 480p, 12 heads on 3, backward 160 us
// instead of 153, forward of 2048 tokens 10.0 instead of 9.1.  Quotients as products (Divisor) then gave 148.5 and 8.7.)
__device__ __forceinline__ void share_turns(const TurnArgs& t, unsigned long long* turns) {
  if (threadIdx.x < 64) turns[threadIdx.x] = t.turn[threadIdx.x];
  __syncthreads();
}

// Sums of each of N values over a team's threads, value l / (TEAM / N) in thread l: halves of the values change sides at each step
// (four rows of the forward: 480p, 24 heads, halves as pairs 209 -> 195 us; the backward's two sums: no faster, and one step more behind the other, clip 15.0 -> 15.8)
template <int TEAM, int N>
__device__ __forceinline__ float team_sums(float (&t)[N], int l) {
  int o = TEAM / 2;
#pragma unroll
  for (int n = N / 2; n > 0; n >>= 1, o >>= 1) {
    const bool upper = l & o;
#pragma unroll
    for (int k = 0; k < n; ++k) {
      const float other = __shfl_xor_sync(0xffffffffu, upper ? t[k] : t[k + n], o);
      t[k] = (upper ? t[k + n] : t[k]) + other;
    }
  }
#pragma unroll
  for (; o > 0; o >>= 1) t[0] += __shfl_xor_sync(0xffffffffu, t[0], o);
  return t[0];
}

// Rows whose mean square lies outside are normed with their channels scaled by a power of two: their squares, or the backward's r^3, could vanish or pass fp32's range (a channel of 2e19
// made a whole head zero).  Inside, nothing is near either end, whatever the gradients; with the usual eps no row is below.
constexpr float kPlainLeast = 0x1p-40f, kPlainMost = 0x1p40f;
// Positive numbers in the order of their bits, those below kPlainLeast and what is not a number behind all others
__device__ __forceinline__ uint32_t beyond_least(float mean_square) { return __float_as_uint(mean_square) - __float_as_uint(kPlainLeast); }
__device__ __forceinline__ bool plain_row(float mean_square) { return beyond_least(mean_square) <= beyond_least(kPlainMost); }
// 1 / sqrt of a plain row's: the instruction alone, without the steps for numbers below the normal ones
__device__ __forceinline__ float rsqrt_plain(float t) {
  float r;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(t));
  return r;
}
// The power of two that brings the larger of a row's largest magnitude and sqrt(eps) to about one; one where that is zero or not finite.  (By the threads of a team together)
template <int TEAM>
__device__ __forceinline__ float row_scale(const float (&f)[8], float eps) {
  float top = sqrtf(eps);
#pragma unroll
  for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(f[i]));
#pragma unroll
  for (int o = TEAM / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  const int e = __float_as_int(top) >> 23;
  return top == 0.f || e == 255 ? 1.f : __int_as_float(max(254 - e, 1) << 23);
}

// The rows of a warp that are not plain, once more on scaled channels.  Rare, and a function of its own: as a branch among the rows 480p, 24 heads, halves as pairs took 199.5 us, without
// the look at them 197.5, 197.7 so.
template <int D, typename TI, typename TO, bool HALVES>
__device__ __noinline__ void scaled_rows_fwd(const QkvArgs& a, const unsigned long long* turns) {
  constexpr int TEAM = D / 8, ROWS = kQkvThreads / TEAM;
  const int l = threadIdx.x % TEAM;
  const int b = divided(blockIdx.x, a.by_tiles), row = ((int)blockIdx.x - b * a.tiles) * ROWS + threadIdx.x / TEAM, tok = min(row, a.tokens - 1);
  Turn<D, HALVES> turn;
  turn.init(a.turn, turns, b, tok, l);
  const int h_lo = blockIdx.z * a.per_cta, h_hi = h_lo + a.per_cta;
  int base = 0;
#pragma unroll 1
  for (int seg = 0; seg < 2; ++seg) {
    const HeadsArg x = a.x[seg], y = a.y[seg];
    const int lo = max(h_lo - base, 0), hi = min(h_hi - base, x.heads);
    base += x.heads;
    const TI* xp = reinterpret_cast<const TI*>(x.p) + b * x.sb + tok * x.st + l * 8;
    TO* yp = reinterpret_cast<TO*>(y.p) + b * y.sb + tok * y.st + l * 8;
#pragma unroll 1
    for (int h = lo; h < hi; ++h) {
      Raw8<TI> raw;
      raw.load(xp + h * x.sh);
      float f[8];
      raw.get(f);
      float ss[1] = {0.f};
#pragma unroll
      for (int i = 0; i < 8; ++i) ss[0] += f[i] * f[i];
      const bool plain = plain_row(team_sums<TEAM>(ss, l) * (1.f / D) + a.eps);      // (one on the edge may come out either way: both ways are right there)
      const float s = row_scale<TEAM>(f, a.eps);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] *= s;
      float scaled[1] = {0.f};
#pragma unroll
      for (int i = 0; i < 8; ++i) scaled[0] += f[i] * f[i];
      const float r = rsqrtf(team_sums<TEAM>(scaled, l) * (1.f / D) + a.eps * s * s);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] *= r * (a.w[seg] != nullptr ? a.w[seg][l * 8 + i] : 1.f);
      turn.apply(f);
      if (row < a.tokens && !plain) store8(yp + h * y.sh, f);
    }
  }
}

// grid (token tiles of all batch entries, 1, groups of heads)
template <int D, typename TI, typename TO, bool HALVES>
__global__ void __launch_bounds__(kQkvThreads) qkv_fwd_kernel(const __grid_constant__ QkvArgs a) {
  constexpr int TEAM = D / 8, ROWS = kQkvThreads / TEAM, U = sizeof(TI) == 2 ? 4 : 2;
  __shared__ __align__(16) unsigned long long turns[64];
  share_turns(a.turn, turns);
  grid_enter();
  const int l = threadIdx.x % TEAM;
  const int b = divided(blockIdx.x, a.by_tiles), tile = blockIdx.x - b * a.tiles;
  const int row = tile * ROWS + threadIdx.x / TEAM;
  const bool valid = row < a.tokens;
  const int tok = min(row, a.tokens - 1);
  Turn<D, HALVES> turn;
  turn.init(a.turn, turns, b, tok, l);
  const int h_lo = blockIdx.z * a.per_cta, h_hi = h_lo + a.per_cta;
  uint32_t farthest = 0u;      // of the rows' mean squares
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
      float r = 1.f;      // of row l / (TEAM / U)
      if (norm) {
        float ss[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float f[8];
          raw[u].get(f);
          ss[u] = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) ss[u] += f[i] * f[i];
        }
        const float t = team_sums<TEAM>(ss, l) * (1.f / D) + a.eps;
        farthest = max(farthest, beyond_least(t));
        r = rsqrt_plain(t);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float f[8];
        raw[u].get(f);
        if (norm) {
          const float ru = __shfl_sync(0xffffffffu, r, TEAM / U * u, TEAM);
#pragma unroll
          for (int i = 0; i < 8; ++i) f[i] *= ru * w[i];
        }
        if (rotate) turn.apply(f);
        if (valid && h + u < hi) store8(yp + (h + u) * y.sh, f);
      }
    }
  }
  if (__any_sync(0xffffffffu, farthest > beyond_least(kPlainMost))) scaled_rows_fwd<D, TI, TO, HALVES>(a, turns);
}

// A thread's own queue in shared memory: 16-byte pieces that it asks for AHEAD rows before it uses them.  (Registers for that many in flight would cost the CTAs
// that hide the rest: with the next two heads' rows in registers 480p with text took 211 us.)
// (Through L1: the second half of an fp32 row's sectors comes from there.)
__device__ __forceinline__ void copy_async(void* to, const void* from) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}

// A row's sums over its team: x^2, and the weighted gradient along x.  (Two channels an instruction: 16 warps' issue slots are the next bound behind memory)
template <int TEAM>
__device__ __forceinline__ float2 row_sums(const float (&x)[8], const float (&g)[8], const float2 (&w)[4]) {
  float2 ss = make_float2(0.f, 0.f), dot = ss;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 x2 = make_float2(x[2 * i], x[2 * i + 1]), g2 = make_float2(g[2 * i], g[2 * i + 1]);
    ss = __ffma2_rn(x2, x2, ss);
    dot = __ffma2_rn(__fmul2_rn(g2, w[i]), x2, dot);
  }
  float2 sums = make_float2(ss.x + ss.y, dot.x + dot.y);
#pragma unroll
  for (int o = TEAM / 2; o > 0; o >>= 1)
    sums = __fadd2_rn(sums, make_float2(__shfl_xor_sync(0xffffffffu, sums.x, o), __shfl_xor_sync(0xffffffffu, sums.y, o)));
  return sums;
}
// g -> dx = r (w g) + m x; the weight's gradient gets g r x
__device__ __forceinline__ void dx_row(float (&g)[8], const float (&x)[8], const float2 (&w)[4], float2 (&dw)[4], float r, float m, bool counts) {
  const float2 r2 = make_float2(r, r), m2 = make_float2(m, m);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 x2 = make_float2(x[2 * i], x[2 * i + 1]), gr = __fmul2_rn(make_float2(g[2 * i], g[2 * i + 1]), r2);
    if (counts) dw[i] = __ffma2_rn(gr, x2, dw[i]);
    const float2 o = __ffma2_rn(x2, m2, __fmul2_rn(gr, w[i]));
    g[2 * i] = o.x;
    g[2 * i + 1] = o.y;
  }
}

struct BwdJobs { int ctas[2], jobs[2], per[2]; };      // of q, of k: CTAs, jobs, heads in a group
// The rows of a warp among which one is not plain, once more: such a row on scaled channels (x r does not change, dx is the scale's multiple), and the weight's gradient summed anew.
// Rare, and a function of its own so that the plain rows keep their registers: 480p with text 156.3 us without the look at the rows, 167 with a branch at each row, 160 with this in the
// kernel, 157.5 so.
template <int D, typename TI, typename TG, typename TO, bool HALVES>
__device__ __noinline__ void scaled_rows(const QkvArgs& a, const HeadsPair& fwd, const BwdJobs& list, const unsigned long long* turns, float2* anew) {
  constexpr int TEAM = D / 8, ROWS = kQkvThreads / TEAM;
  const int l = threadIdx.x % TEAM, slot = threadIdx.x / TEAM;
  const int side = (int)blockIdx.x < list.ctas[0] ? 0 : 1, first = (int)blockIdx.x - (side > 0 ? list.ctas[0] : 0);
  const HeadsArg g = a.x[side], y = a.y[side], x = fwd.v[side];
  float2 w[4], dw[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    dw[i] = make_float2(0.f, 0.f);
    w[i] = a.w[side] != nullptr ? make_float2(a.w[side][l * 8 + 2 * i], a.w[side][l * 8 + 2 * i + 1]) : make_float2(1.f, 1.f);
  }
#pragma unroll 1
  for (int job = first; job < list.jobs[side]; job += list.ctas[side]) {
    const int group = divided(job, a.by_jobs), lo = group * list.per[side], hi = min(lo + list.per[side], g.heads);
    const int at = job - group * a.jobs, b = divided(at, a.by_tiles), row = (at - b * a.tiles) * ROWS + slot, tok = min(row, a.tokens - 1);
    const bool valid = row < a.tokens;
    const TG* gp = reinterpret_cast<const TG*>(g.p) + b * g.sb + tok * g.st + l * 8;
    const TI* xp = reinterpret_cast<const TI*>(x.p) + b * x.sb + tok * x.st + l * 8;
    TO* yp = reinterpret_cast<TO*>(y.p) + b * y.sb + tok * y.st + l * 8;
    Turn<D, HALVES> turn;
    turn.init(a.turn, turns, b, tok, l);
#pragma unroll 1
    for (int h = lo; h < hi; ++h) {
      Raw8<TG> gr;
      Raw8<TI> xr;
      gr.load(gp + h * g.sh);
      xr.load(xp + h * x.sh);
      float f[8], xf[8];
      gr.get(f);
      xr.get(xf);
      turn.apply(f);
      float2 sums = row_sums<TEAM>(xf, f, w);
      float t = __fmaf_rn(sums.x, 1.f / D, a.eps);
      const bool plain = plain_row(t);
      const float scale = row_scale<TEAM>(xf, a.eps), s = plain ? 1.f : scale;
#pragma unroll
      for (int i = 0; i < 8; ++i) xf[i] *= s;
      const float2 scaled = row_sums<TEAM>(xf, f, w);
      if (!plain) {
        sums = scaled;
        t = sums.x * (1.f / D) + a.eps * s * s;
      }
      const float r = rsqrtf(t);
      dx_row(f, xf, w, dw, r, sums.y * (-1.f / D) * r * r * r, valid);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] *= s;
      if (valid && !plain) store8(yp + h * y.sh, f);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) anew[i] = dw[i];
}

// x = the forward's rows of q and k, dy -> dx.  A job is a tile of tokens and a group of heads.  The first CTAs take q's jobs, the others k's, so that a thread sums the
// gradient of one weight; then all take v's.
template <int D, typename TI, typename TG, typename TO, bool HALVES>
__global__ void __launch_bounds__(kQkvThreads, HALVES ? 3 : 4) qkv_bwd_kernel(const __grid_constant__ QkvArgs a, const __grid_constant__ HeadsPair fwd,
                                                                        const __grid_constant__ BwdJobs list, float* __restrict__ partial) {
  constexpr int TEAM = D / 8, ROWS = kQkvThreads / TEAM;
  constexpr int GV = sizeof(TG) / 2, XV = sizeof(TI) / 2, AHEAD = bwd_ahead(GV + XV, HALVES);      // 16-byte pieces of a row of dy, of x
  __shared__ __align__(16) unsigned long long turns[64];
  share_turns(a.turn, turns);
  grid_enter();
  extern __shared__ __align__(16) unsigned char qkv_smem[];
  uint4* const queue = reinterpret_cast<uint4*>(qkv_smem) + threadIdx.x;      // [AHEAD][GV + XV][thread]
  const int l = threadIdx.x % TEAM, slot = threadIdx.x / TEAM;
  // batch entry and token of a tile (a row behind the last one repeats it)
  struct Place { int b, tok; bool valid; };
  auto place = [&](int at) {
    const int b = divided(at, a.by_tiles), row = (at - b * a.tiles) * ROWS + slot;
    return Place{b, min(row, a.tokens - 1), row < a.tokens};
  };
  {
    const int side = (int)blockIdx.x < list.ctas[0] ? 0 : 1, first = (int)blockIdx.x - (side > 0 ? list.ctas[0] : 0);
    const int stride = list.ctas[side], per = list.per[side], jobs = list.jobs[side];
    const HeadsArg g = a.x[side], y = a.y[side], x = fwd.v[side];
    const bool norm = a.norm;
    float2 w[4], dw[4];
    uint32_t farthest = 0u;      // of the rows' mean squares
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      dw[i] = make_float2(0.f, 0.f);
      w[i] = norm && a.w[side] != nullptr ? make_float2(a.w[side][l * 8 + 2 * i], a.w[side][l * 8 + 2 * i + 1]) : make_float2(1.f, 1.f);
    }
    // the queue's end: job, head and place of the next row to ask for
    int ask_job = first, ask_h = 0, ask_hi = 0;
    const TG* ask_g = nullptr;
    const TI* ask_x = nullptr;
    auto ask = [&](int s) {
      if (ask_h == ask_hi && ask_job < jobs) {
        const int group = divided(ask_job, a.by_jobs), lo = group * per;
        const Place at = place(ask_job - group * a.jobs);
        ask_job += stride;
        ask_h = lo;
        ask_hi = min(lo + per, g.heads);
        ask_g = reinterpret_cast<const TG*>(g.p) + at.b * g.sb + at.tok * g.st + lo * g.sh + l * 8;
        if (norm) ask_x = reinterpret_cast<const TI*>(x.p) + at.b * x.sb + at.tok * x.st + lo * x.sh + l * 8;
      }
      if (ask_h < ask_hi) {
        uint4* to = queue + s * (GV + XV) * kQkvThreads;
#pragma unroll
        for (int v = 0; v < GV; ++v) copy_async(to + v * kQkvThreads, reinterpret_cast<const uint4*>(ask_g) + v);
        ask_g += g.sh;
        if (norm) {
#pragma unroll
          for (int v = 0; v < XV; ++v) copy_async(to + (GV + v) * kQkvThreads, reinterpret_cast<const uint4*>(ask_x) + v);
          ask_x += x.sh;
        }
        ++ask_h;
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int s = 0; s < AHEAD - 1; ++s) ask(s);
    int s = 0;
    for (int job = first; job < jobs; job += stride) {
      const int group = divided(job, a.by_jobs), lo = group * per, hi = min(lo + per, g.heads);
      const Place at = place(job - group * a.jobs);
      Turn<D, HALVES> turn;
      turn.init(a.turn, turns, at.b, at.tok, l);
      TO* yp = reinterpret_cast<TO*>(y.p) + at.b * y.sb + at.tok * y.st + lo * y.sh + l * 8;
      for (int h = lo; h < hi; ++h, yp += y.sh) {
        asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD - 2) : "memory");
        const uint4* from = queue + s * (GV + XV) * kQkvThreads;
        Raw8<TG> gr;
        gr.load(from, kQkvThreads);
        float f[8];
        gr.get(f);
        turn.apply(f);
        if (norm) {
          Raw8<TI> xr;
          xr.load(from + GV * kQkvThreads, kQkvThreads);
          float xf[8];
          xr.get(xf);
          const float2 sums = row_sums<TEAM>(xf, f, w);
          const float t = __fmaf_rn(sums.x, 1.f / D, a.eps);
          farthest = max(farthest, beyond_least(t));
          const float r = rsqrt_plain(t), m = sums.y * (-1.f / D) * r * r * r;
          dx_row(f, xf, w, dw, r, m, at.valid);
        }
        if (at.valid) store8(yp, f);
        ask(s == 0 ? AHEAD - 1 : s - 1);      // (the place that was read last time)
        if (++s == AHEAD) s = 0;
      }
    }
    if (norm) {
      asm volatile("cp.async.wait_all;" ::: "memory");
      if (__any_sync(0xffffffffu, farthest > beyond_least(kPlainMost))) {
        float2 anew[4];
        scaled_rows<D, TI, TG, TO, HALVES>(a, fwd, list, turns, anew);
#pragma unroll
        for (int i = 0; i < 4; ++i) dw[i] = anew[i];
      }
      __syncthreads();
      float2* red = reinterpret_cast<float2*>(qkv_smem);      // [ROWS][D / 2]
#pragma unroll
      for (int i = 0; i < 4; ++i) red[slot * (D / 2) + l * 4 + i] = dw[i];
      __syncthreads();
      for (int i = threadIdx.x; i < D; i += kQkvThreads) {
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) sum += reinterpret_cast<const float*>(red)[r * D + i];
        partial[(size_t)blockIdx.x * D + i] = sum;
      }
    }
  }
  const HeadsArg g = a.x[2], y = a.y[2];
  if (g.heads == 0) return;
  for (int job = blockIdx.x; job < a.jobs; job += gridDim.x) {
    const Place at = place(job);
    const TG* gp = reinterpret_cast<const TG*>(g.p) + at.b * g.sb + at.tok * g.st + l * 8;
    TO* yp = reinterpret_cast<TO*>(y.p) + at.b * y.sb + at.tok * y.st + l * 8;
    for (int h = 0; h < g.heads; h += 4) {
      Raw8<TG> gr[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) gr[u].load(gp + min(h + u, g.heads - 1) * g.sh);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        float f[8];
        gr[u].get(f);
        if (at.valid && h + u < g.heads) store8(yp + (h + u) * y.sh, f);
      }
    }
  }
}

// Sums of the CTAs' partial sums in a fixed order: 8 columns a CTA, 128 parts at a time, so that a thread's few loads are under way together.  grid (columns / 8, 2: q, k)
__global__ void __launch_bounds__(1024) qkv_bwd_reduce_kernel(const float* partial, int q_ctas, int qk_ctas, int D, float* __restrict__ dwq,
                                                              float* __restrict__ dwk) {
  constexpr int MOST = kQkvParts / 128;
  grid_enter();
  __shared__ float red[32][8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 8 + (lane & 7);
  const int lo = blockIdx.y == 0 ? 0 : q_ctas, hi = blockIdx.y == 0 ? q_ctas : qk_ctas, first = lo + warp * 4 + (lane >> 3);
  float v[MOST];
#pragma unroll
  for (int u = 0; u < MOST; ++u) v[u] = first + u * 128 < hi ? partial[(size_t)(first + u * 128) * D + col] : 0.f;
  float sum = 0.f;
#pragma unroll
  for (int u = 0; u < MOST; ++u) sum += v[u];
  sum += __shfl_xor_sync(0xffffffffu, sum, 8);
  sum += __shfl_xor_sync(0xffffffffu, sum, 16);
  if (lane < 8) red[warp][lane] = sum;
  __syncthreads();
  if (warp == 0) {
    float total = 0.f;
#pragma unroll
    for (int r = 0; r < 8; ++r) total += red[(lane >> 3) * 8 + r][lane & 7];
    total += __shfl_xor_sync(0xffffffffu, total, 8);
    total += __shfl_xor_sync(0xffffffffu, total, 16);
    float* out = blockIdx.y == 0 ? dwq : dwk;
    if (lane < 8 && out != nullptr) out[col] = total;
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

size_t qkv_bwd_workspace_bytes(int D) { return (size_t)kQkvParts * D * sizeof(float); }

cudaError_t launch_qkv_fwd(QkvArgs a, int D, int batch, int in_f32, int out_f32, bool halves, cudaStream_t st) {
  const int rows = kQkvThreads / (D / 8), heads = a.x[0].heads + a.x[1].heads + a.x[2].heads;
  int sms = 0;
  cudaError_t e;
  if ((e = sm_count(&sms)) != cudaSuccess) return e;
  a.tiles = (a.tokens + rows - 1) / rows;
  a.jobs = a.tiles * batch;
  a.by_tiles = divisor(a.tiles);
  a.by_jobs = divisor(a.jobs);
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
  const int rows = kQkvThreads / (D / 8);
  int sms = 0;
  cudaError_t e;
  if ((e = sm_count(&sms)) != cudaSuccess) return e;
  a.tiles = (a.tokens + rows - 1) / rows;
  a.jobs = a.tiles * batch;
  a.by_tiles = divisor(a.tiles);
  a.by_jobs = divisor(a.jobs);
  // CTAs for q and for k by what a tile of theirs costs: its heads and the sines and cosines of its tokens, about two heads' worth (40 q heads on one k head: one
  // head's worth 236 us, two 201, three 203; by the heads alone q waited for the k CTAs, more than twice that).  Heads go in groups where that makes the rounds of jobs even.
  BwdJobs list = {};
  const int at_once = (halves ? 3 : 4) * sms, ctas = at_once < kQkvParts ? at_once : kQkvParts;
  const int nq = a.x[0].heads, nk = a.x[1].heads;
  int share[2] = {nq == 0 ? 0 : ctas, nk == 0 ? 0 : ctas};
  if (nq > 0 && nk > 0) {
    share[0] = (int)((long long)ctas * (nq + 2) / (nq + nk + 4));
    share[0] = share[0] < 1 ? 1 : share[0] >= ctas ? ctas - 1 : share[0];
    share[1] = ctas - share[0];
  }
  for (int i = 0; i < 2; ++i) {
    const int n = a.x[i].heads;
    if (n == 0) continue;
    long long least = 0;
    int groups = 1;
    for (int g = 1; g <= 16 && g <= n; ++g) {
      const int per = (n + g - 1) / g, of = (n + per - 1) / per;
      const long long cost = ((long long)a.jobs * of + share[i] - 1) / share[i] * (2 + per);
      if (g == 1 || cost < least) {
        least = cost;
        list.per[i] = per;
        groups = of;
      }
    }
    const long long jobs = (long long)a.jobs * groups;
    if (jobs > 0x7fffffff - kQkvParts) return cudaErrorInvalidValue;
    list.jobs[i] = (int)jobs;
    list.ctas[i] = jobs < share[i] ? (int)jobs : share[i];
  }
  int grid = list.ctas[0] + list.ctas[1];
  if (grid == 0) {      // (v alone: CTAs whose list is empty)
    grid = a.jobs < ctas ? a.jobs : ctas;
    list.ctas[0] = grid;
  }
  const int pieces = (g_f32 ? 2 : 1) + (x_f32 ? 2 : 1);
  size_t smem = (size_t)bwd_ahead(pieces, halves) * pieces * kQkvThreads * 16;
  if (smem < kQkvThreads * 8 * sizeof(float)) smem = kQkvThreads * 8 * sizeof(float);      // (the CTA's sums)
  auto go = [&](auto tx, auto tg, auto to) {
    using TX = decltype(tx);
    using TG = decltype(tg);
    using TO = decltype(to);
    if (D == 128) return halves ? launch_kernel(qkv_bwd_kernel<128, TX, TG, TO, true>, grid, kQkvThreads, smem, st, a, fwd, list, partial)
                                : launch_kernel(qkv_bwd_kernel<128, TX, TG, TO, false>, grid, kQkvThreads, smem, st, a, fwd, list, partial);
    return halves ? launch_kernel(qkv_bwd_kernel<64, TX, TG, TO, true>, grid, kQkvThreads, smem, st, a, fwd, list, partial)
                  : launch_kernel(qkv_bwd_kernel<64, TX, TG, TO, false>, grid, kQkvThreads, smem, st, a, fwd, list, partial);
  };
  e = by_types(g_f32, out_f32, [&](auto tg, auto to) { return x_f32 ? go(float(), tg, to) : go(bf16(), tg, to); });
  if (e != cudaSuccess || !a.norm) return e;
  return launch_kernel(qkv_bwd_reduce_kernel, dim3(D / 8, 2), 1024, 0, st, partial, list.ctas[0], list.ctas[0] + list.ctas[1], D, dwq, dwk);
}

}  // namespace vsa2
