// Per-head RMS norm of queries and keys with the rotation of positions in the same pass, and its
// gradients, sm_103a.
//
// Mathematics, per row x of d features with weight w:  r = (mean x^2 + eps)^(-1/2),  u = w x r,
// and each pair (a, b) of the first d_rot features turns by its position's angle:
//     y_a = u_a c - u_b s,   y_b = u_b c + u_a s.
// Backward, g = dL/dy:  t = R^T g (the same turn by the opposite angle),
//     dw = sum over rows of t x r,    dx = r (w t - x r * mean(w t x r)).
// Everything is computed in fp32; outputs are rounded once, the weights' gradients stay fp32.
//
// What bounds it: memory, and in a launch of one round of CTAs its start and end.  Every element is read
// once and written once (backward: x and g read, dx written), with about ten operations for each, which
// fill 60 to 65 % of the issue slots.  Measured, bf16: forward 4 x (16 + 16) x 2048 x 64 13.4 us = 5.0
// TB/s; backward 2 x (32 + 8) x 8192 x 128 95.5 us = 5.3 TB/s; fp32 forward 3 x (10 + 2) x 1021 x 96,
// 5.1 us, backward 2 x (6 + 3) x 517 x 128, 6.9 us: a launch's own time.
//
// Layout of the work: a group of 8, 16 or 32 lanes owns one token and walks over a range of its
// heads, eight features a lane (one 16-byte load of bf16, two of fp32), in batches whose rows are all
// on their way before the first is used.  The token's cosines and sines are loaded once and serve all
// heads of the range; with halves, the other member of a lane's pairs comes by a shuffle of the row as
// it lies in memory.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdio>

#include "internal.h"
#include "ops_internal.h"

namespace moa {

__device__ unsigned int g_moa_norm_status = 0;

namespace {

constexpr int kThreads = 256;
constexpr int kV = 8;  // features of a lane
// Backward CTAs on an SM: three hold bf16 rows in 80 registers and 44 bytes of spills; fp32 rows, twice the
// registers, get two.
constexpr int bwd_ctas(bool f32) { return f32 ? 2 : 3; }
constexpr unsigned kErrIndex = 7u;  // MOA_ERR_DEVICE_INDEX

// Two floats in a register pair, and arithmetic on both at once (each rounded as by itself): half the
// instructions of a row, which are what the memory would otherwise wait for.
__device__ __forceinline__ uint64_t pair(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float low(uint64_t a) { return __uint_as_float(uint32_t(a)); }
__device__ __forceinline__ float high(uint64_t a) { return __uint_as_float(uint32_t(a >> 32)); }
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

__device__ __forceinline__ void load8(const __nv_bfloat16* p, float* x) {
  const uint4 v = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8(const float* p, float* x) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}
// A lane's features as they lie in memory, so that several rows can be on their way at once.
template <typename T>
struct Raw {
  uint4 w[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < int(sizeof(T) / 2); ++i) w[i] = reinterpret_cast<const uint4*>(p)[i];
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < int(sizeof(T) / 2); ++i) w[i] = make_uint4(0, 0, 0, 0);
  }
  // Those of lane `from` of the group.
  template <int LPR>
  __device__ __forceinline__ Raw of(int from) const {
    Raw r;
#pragma unroll
    for (int i = 0; i < int(sizeof(T) / 2); ++i)
      r.w[i] = make_uint4(__shfl_sync(0xffffffffu, w[i].x, from, LPR), __shfl_sync(0xffffffffu, w[i].y, from, LPR),
                          __shfl_sync(0xffffffffu, w[i].z, from, LPR), __shfl_sync(0xffffffffu, w[i].w, from, LPR));
    return r;
  }
  __device__ __forceinline__ void widen(uint64_t* x) const {   // kV / 2 pairs
    if constexpr (sizeof(T) == 2) {
      const uint32_t v[4] = {w[0].x, w[0].y, w[0].z, w[0].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = pair(__uint_as_float(v[i] << 16), __uint_as_float(v[i] & 0xffff0000u));
    } else {
#pragma unroll
      for (int i = 0; i < int(sizeof(T) / 2); ++i) {
        x[2 * i] = pair(__uint_as_float(w[i].x), __uint_as_float(w[i].y));
        x[2 * i + 1] = pair(__uint_as_float(w[i].z), __uint_as_float(w[i].w));
      }
    }
  }
};
__device__ __forceinline__ void store8(__nv_bfloat16* p, const uint64_t* x) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    __nv_bfloat162 v = __floats2bfloat162_rn(low(x[i]), high(x[i]));
    w[i] = *reinterpret_cast<uint32_t*>(&v);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(float* p, const uint64_t* x) {
  *reinterpret_cast<float4*>(p) = make_float4(low(x[0]), high(x[0]), low(x[1]), high(x[1]));
  *reinterpret_cast<float4*>(p + 4) = make_float4(low(x[2]), high(x[2]), low(x[3]), high(x[3]));
}
template <int LPR>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
  for (int o = LPR / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o, LPR);
  return v;
}

// One lane's share of a token's rotation: cosine and (signed) sine of its features' pairs.  With
// neighbouring pairs a lane holds four pairs; with halves its eight features meet the same eight
// of the lane half a rotation away.
struct Turn {
  float c[kV], s[kV];
};

// The other members of this lane's pairs.
template <typename T, int LPR, bool PAIRS>
__device__ __forceinline__ void others(const Raw<T>& raw, const uint64_t* x, int partner, uint64_t* o) {
  if constexpr (PAIRS) {
#pragma unroll
    for (int i = 0; i < kV / 2; ++i) o[i] = pair(high(x[i]), low(x[i]));
  } else {
    raw.template of<LPR>(partner).widen(o);
  }
}
// The sum of a lane's eight squares, or products.
__device__ __forceinline__ float dot8(const uint64_t* a, const uint64_t* b) {
  uint64_t s = mul2(a[0], b[0]);
#pragma unroll
  for (int i = 1; i < kV / 2; ++i) s = fma2(a[i], b[i], s);
  return low(s) + high(s);
}

struct Dims {
  int64_t tokens;    // B * N
  int64_t N, n_pos;
  int Hq, Hk, d, d_rot;
  int hp;            // heads of one range
  int nq;            // ranges of query heads (the ranges of key heads follow)
  float eps;
};

__device__ __forceinline__ int64_t sequence_of(int64_t token, const Dims& p) {
  return p.tokens <= 0x7fffffff ? uint32_t(token) / uint32_t(p.N) : token / p.N;
}

// The rotation of the token's position for this lane.  `dir` +1 forward, -1 backward.
template <bool PAIRS>
__device__ __forceinline__ void load_turn(Turn& t, const float* cosines, const float* sines,
                                          int64_t pos, const Dims& p, int f0, float dir) {
#pragma unroll
  for (int i = 0; i < kV; ++i) t.c[i] = 1.f, t.s[i] = 0.f;
  if (f0 >= p.d_rot) return;
  const int half = p.d_rot / 2;
  const float* c = cosines + pos * half;
  const float* s = sines + pos * half;
  if constexpr (PAIRS) {
    const float4 cc = *reinterpret_cast<const float4*>(c + f0 / 2);
    const float4 ss = *reinterpret_cast<const float4*>(s + f0 / 2);
    const float cv[4] = {cc.x, cc.y, cc.z, cc.w}, sv[4] = {ss.x, ss.y, ss.z, ss.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      t.c[2 * i] = t.c[2 * i + 1] = cv[i];
      t.s[2 * i] = -dir * sv[i];
      t.s[2 * i + 1] = dir * sv[i];
    }
  } else {
    const bool first = f0 < half;
    const int i0 = first ? f0 : f0 - half;
    const float sign = first ? -dir : dir;
    load8(c + i0, t.c);
    load8(s + i0, t.s);
#pragma unroll
    for (int i = 0; i < kV; ++i) t.s[i] *= sign;
  }
}

template <typename T, int LPR, bool PAIRS>
__global__ void __launch_bounds__(kThreads, 4)
norm_rope_kernel(View q, View k, View oq, View ok, const T* wq, const T* wk, const float* cosines,
                 const float* sines, const int32_t* pos, Dims p) {
  constexpr int kGroups = kThreads / LPR;
  constexpr int kBatch = 2;
  wait_for_previous();
  const int lane = threadIdx.x % LPR;
  const int64_t token = int64_t(blockIdx.x) * kGroups + threadIdx.x / LPR;
  const bool is_q = int(blockIdx.y) < p.nq;
  const int range = is_q ? int(blockIdx.y) : int(blockIdx.y) - p.nq;
  const View in = is_q ? q : k, out = is_q ? oq : ok;
  const int H = is_q ? p.Hq : p.Hk;
  const int h0 = range * p.hp, h1 = h0 + p.hp < H ? h0 + p.hp : H;
  const int f0 = lane * kV;
  const bool live = token < p.tokens;
  const bool mine = live && f0 < p.d;
  const int64_t b = live ? sequence_of(token, p) : 0, n = live ? token - b * p.N : 0;
  const T* src = static_cast<const T*>(in.p) + b * in.sb + n * in.sn + f0;
  T* dst = static_cast<T*>(out.p) + b * out.sb + n * out.sn + f0;
  Raw<T> raw[kBatch];
  auto fetch = [&](int hb) {
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (mine && hb + u < h1) raw[u].load(src + (hb + u) * in.sh);
      else raw[u].zero();
    }
  };
  fetch(h0);
  const int32_t at = live ? pos[token] : -1;
  const bool bad = live && at >= p.n_pos;
  if (bad && lane == 0) atomicExch(&g_moa_norm_status, kErrIndex);
  const int half_lanes = p.d_rot / 2 / kV;
  const int partner = f0 >= p.d_rot ? lane : (f0 < p.d_rot / 2 ? lane + half_lanes : lane - half_lanes);
  // y = (x c w + o s w_o) r: the weights of both members go into the angles
  Turn t;
  load_turn<PAIRS>(t, cosines, sines, at >= 0 && !bad ? at : 0, p, f0, 1.f);
  if (f0 < p.d) {
    float w[kV];
    const T* wp = is_q ? wq : wk;
    load8(wp + f0, w);
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      t.c[i] *= w[i];
      if (PAIRS) t.s[i] *= w[i ^ 1];
    }
    if (!PAIRS) {
      load8(wp + partner * kV, w);
#pragma unroll
      for (int i = 0; i < kV; ++i) t.s[i] *= w[i];
    }
  }
  uint64_t c2[kV / 2], s2[kV / 2];
#pragma unroll
  for (int i = 0; i < kV / 2; ++i) c2[i] = pair(t.c[2 * i], t.c[2 * i + 1]), s2[i] = pair(t.s[2 * i], t.s[2 * i + 1]);
  const float inv_d = 1.f / float(p.d);
  for (int hb = h0; hb < h1; hb += kBatch) {
    Raw<T> now[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) now[u] = raw[u];
    if (hb + kBatch < h1) fetch(hb + kBatch);
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int h = hb + u;
      if (h >= h1) break;
      uint64_t x[kV / 2], o[kV / 2];
      now[u].widen(x);
      others<T, LPR, PAIRS>(now[u], x, partner, o);
      const float r = rsqrtf(group_sum<LPR>(dot8(x, x)) * inv_d + p.eps);
      const uint64_t r2 = pair(r, r);
#pragma unroll
      for (int i = 0; i < kV / 2; ++i) x[i] = mul2(fma2(x[i], c2[i], mul2(o[i], s2[i])), r2);
      if (at < 0 || bad) {
        const float fill = bad ? __int_as_float(0x7fc00000) : 0.f;
#pragma unroll
        for (int i = 0; i < kV / 2; ++i) x[i] = pair(fill, fill);
      }
      if (mine) store8(dst + h * out.sh, x);
    }
  }
}

// The gradients: one launch for dx and, for each CTA, the sum of its rows' t x r; a second one
// adds the CTAs' sums in a fixed order.
template <typename T, int LPR, bool PAIRS>
__global__ void __launch_bounds__(kThreads, bwd_ctas(sizeof(T) == 4))
norm_rope_bwd_kernel(View q, View k, View gq, View gk, View oq, View ok, const T* wq, const T* wk,
                     const float* cosines, const float* sines, const int32_t* pos, float* partial,
                     Dims p) {
  constexpr int kGroups = kThreads / LPR;
  constexpr int kBatch = sizeof(T) == 2 ? 2 : 1;
  __shared__ float sums[kGroups][LPR * kV];
  wait_for_previous();
  const int lane = threadIdx.x % LPR, group = threadIdx.x / LPR;
  const bool is_q = int(blockIdx.y) < p.nq;
  const int range = is_q ? int(blockIdx.y) : int(blockIdx.y) - p.nq;
  const View in = is_q ? q : k, gin = is_q ? gq : gk, out = is_q ? oq : ok;
  const int H = is_q ? p.Hq : p.Hk;
  const int f0 = lane * kV;
  uint64_t acc[kV / 2];
  Raw<T> wraw;
  wraw.zero();
#pragma unroll
  for (int i = 0; i < kV / 2; ++i) acc[i] = 0;
  if (f0 < p.d) wraw.load((is_q ? wq : wk) + f0);
  const int half_lanes = p.d_rot / 2 / kV;
  const int partner = f0 >= p.d_rot ? lane : (f0 < p.d_rot / 2 ? lane + half_lanes : lane - half_lanes);
  const float inv_d = 1.f / float(p.d);
  // Rounds of gridDim.x groups of tokens.  In the last one `left` groups may be fewer than CTAs: then
  // several CTAs share a group's heads.
  const int64_t all = (p.tokens + kGroups - 1) / kGroups;
  auto token_of = [&](int64_t round) {
    const int64_t left = all - round;
    return (round + (left > 0 && left < gridDim.x ? blockIdx.x % uint32_t(left) : blockIdx.x)) * kGroups + group;
  };
  // a token's position is read while the token before it is worked on
  auto position = [&](int64_t token) { return token < p.tokens ? pos[token] : -1; };
  int32_t next_at = position(token_of(0));
  // every lane of a warp takes part in each turn of the loop (shuffles), whether its token exists
  for (int64_t round = 0; round < all; round += gridDim.x) {
    int h0 = range * p.hp, h1 = h0 + p.hp < H ? h0 + p.hp : H;
    const int64_t left = all - round;
    if (left < gridDim.x) {
      const uint32_t n = gridDim.x / uint32_t(left), mine = blockIdx.x / uint32_t(left);
      const int each = (h1 - h0 + int(n) - 1) / int(n);
      if (mine >= n || h0 + int(mine) * each >= h1) break;
      h0 += int(mine) * each;
      h1 = h0 + each < h1 ? h0 + each : h1;
    }
    const int64_t token = token_of(round);
    const bool live = token < p.tokens;
    const bool mine = live && f0 < p.d;
    const int64_t b = live ? sequence_of(token, p) : 0, n = live ? token - b * p.N : 0;
    const T* src = static_cast<const T*>(in.p) + b * in.sb + n * in.sn + f0;
    const T* gsrc = static_cast<const T*>(gin.p) + b * gin.sb + n * gin.sn + f0;
    T* dst = static_cast<T*>(out.p) + b * out.sb + n * out.sn + f0;
    Raw<T> xraw[kBatch], graw[kBatch];
    auto fetch = [&](int hb) {
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        if (mine && hb + u < h1) {
          xraw[u].load(src + (hb + u) * in.sh);
          graw[u].load(gsrc + (hb + u) * gin.sh);
        } else {
          xraw[u].zero();
          graw[u].zero();
        }
      }
    };
    fetch(h0);
    const int32_t at = next_at;
    const bool bad = at >= p.n_pos;
    if (bad && lane == 0) atomicExch(&g_moa_norm_status, kErrIndex);
    const bool counts = at >= 0 && !bad;
    Turn t;
    load_turn<PAIRS>(t, cosines, sines, counts ? at : 0, p, f0, -1.f);
    uint64_t c2[kV / 2], s2[kV / 2];
#pragma unroll
    for (int i = 0; i < kV / 2; ++i) c2[i] = pair(t.c[2 * i], t.c[2 * i + 1]), s2[i] = pair(t.s[2 * i], t.s[2 * i + 1]);
    next_at = position(token_of(round + gridDim.x));
    for (int hb = h0; hb < h1; hb += kBatch) {
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int h = hb + u;
        if (h >= h1) break;
        uint64_t x[kV / 2], g[kV / 2], o[kV / 2], w[kV / 2];
        xraw[u].widen(x);
        graw[u].widen(g);
        others<T, LPR, PAIRS>(graw[u], g, partner, o);
        // the row's registers are free: the same place of the next batch
        if (h + kBatch < h1 && mine) {
          xraw[u].load(src + (h + kBatch) * in.sh);
          graw[u].load(gsrc + (h + kBatch) * gin.sh);
        }
        const float r = rsqrtf(group_sum<LPR>(dot8(x, x)) * inv_d + p.eps);
        const uint64_t r2 = pair(r, r);
        wraw.widen(w);
#pragma unroll
        for (int i = 0; i < kV / 2; ++i) {
          const uint64_t turned = fma2(g[i], c2[i], mul2(o[i], s2[i]));
          x[i] = mul2(x[i], r2);
          o[i] = mul2(turned, x[i]);
          g[i] = mul2(w[i], turned);
        }
        const float mean = group_sum<LPR>(dot8(g, x)) * inv_d;
        const uint64_t m2 = pair(-mean, -mean);
#pragma unroll
        for (int i = 0; i < kV / 2; ++i) g[i] = mul2(r2, fma2(x[i], m2, g[i]));
        if (counts) {
#pragma unroll
          for (int i = 0; i < kV / 2; ++i) acc[i] = add2(acc[i], o[i]);
        } else {
          const float fill = bad ? __int_as_float(0x7fc00000) : 0.f;
#pragma unroll
          for (int i = 0; i < kV / 2; ++i) g[i] = pair(fill, fill);
        }
        if (mine) store8(dst + h * out.sh, g);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kV / 2; ++i) sums[group][f0 + 2 * i] = low(acc[i]), sums[group][f0 + 2 * i + 1] = high(acc[i]);
  __syncthreads();
  const int64_t row = int64_t(blockIdx.y) * gridDim.x + blockIdx.x;
  for (int f = threadIdx.x; f < p.d; f += kThreads) {
    float s = 0.f;
#pragma unroll 4
    for (int g = 0; g < kGroups; ++g) s += sums[g][f];
    partial[row * p.d + f] = s;
  }
}

// Sums of partial rows: block (column block, 0 = queries / 1 = keys); warp w adds rows w, w+32, ...
// of 32 columns, then the warps' sums are added in order, so that two runs give the same bits.  456 rows
// of 128: about 2 us behind the kernel before it, the latency of a chain of loads.
__global__ void __launch_bounds__(1024)
norm_rope_bwd_sum_kernel(const float* partial, float* dwq, float* dwk, int64_t rows_q, int64_t rows,
                         int d) {
  __shared__ float sums[32][33];
  wait_for_previous();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int f = blockIdx.x * 32 + lane;
  const int64_t r0 = blockIdx.y == 0 ? 0 : rows_q, r1 = blockIdx.y == 0 ? rows_q : rows;
  float s = 0.f;
  if (f < d) {
#pragma unroll 8
    for (int64_t r = r0 + warp; r < r1; r += 32) s += partial[r * d + f];
  }
  sums[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && f < d) {
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) s += sums[i][lane];
    (blockIdx.y == 0 ? dwq : dwk)[f] = s;
  }
}

int lanes_per_row(int64_t d) { return d <= 64 ? 8 : d <= 128 ? 16 : 32; }

struct Grid {
  int64_t x;
  int y, hp, nq;
};
// Ranges of heads.  A range costs its heads and about one and a half more (the token's place, angles
// and weights), a launch as many ranges as a CTA's place takes one after another: the number of heads with
// the smallest sum is taken, sixteen at most.  On 4 x (16 + 16) heads x 2048 x 64, 1024 CTAs of 8 heads make
// two rounds of the four that fit on an SM and 512 of 16 make one: 13.9 and 13.5 us.
// The backward's CTAs each leave one row of sums, so as many as are resident at once (`ctas` on an SM;
// 0 in the forward) walk over the tokens, and where the last round has fewer groups of tokens than
// CTAs, several share a group's heads (the same sizes: 25.0 us, without that 30.6).  Three CTAs an SM of
// fp32, where two fit, cost a second round: 8.4 instead of 6.9 us on 2 x (6 + 3) heads x 517 x 128.
Grid plan(int64_t tokens, int64_t Hq, int64_t Hk, int64_t d, int sms, int ctas) {
  const int64_t per = kThreads / lanes_per_row(d), groups = (tokens + per - 1) / per;
  const int64_t most = Hq > Hk ? Hq : Hk;
  Grid best{};
  double least = 0;
  for (int64_t hp = 1; hp <= 16 && hp <= most; ++hp) {
    Grid g;
    g.hp = int(hp);
    g.nq = int((Hq + hp - 1) / hp);
    g.y = g.nq + int((Hk + hp - 1) / hp);
    g.x = groups;
    double cost;
    if (ctas > 0) {
      const int64_t limit = int64_t(sms) * ctas / g.y;
      if (g.x > limit) g.x = limit < 1 ? 1 : limit;
      const int64_t left = groups % g.x;
      cost = double(groups / g.x) * (double(hp) + 1.5);
      if (left > 0) cost += double((hp + g.x / left - 1) / (g.x / left)) + 1.5;
    } else {
      cost = double((g.x * g.y + sms * 4 - 1) / (sms * 4)) * (double(hp) + 1.5);
    }
    if (best.hp == 0 || cost <= least) best = g, least = cost;
  }
  return best;
}

template <typename T, int LPR, bool PAIRS>
int run(const NormRopeArgs& a, const Grid& g, const Dims& p, bool bwd, char* msg, size_t msglen) {
  const T* wq = static_cast<const T*>(a.wq);
  const T* wk = static_cast<const T*>(a.wk);
  const dim3 grid{unsigned(g.x), unsigned(g.y), 1};
  cudaError_t e;
  if (!bwd) {
    e = launch_overlapped(norm_rope_kernel<T, LPR, PAIRS>, grid, dim3(kThreads), 0, a.stream, a.q, a.k, a.oq, a.ok, wq,
                          wk, a.cosines, a.sines, a.pos, p);
  } else {
    e = launch_overlapped(norm_rope_bwd_kernel<T, LPR, PAIRS>, grid, dim3(kThreads), 0, a.stream, a.q, a.k, a.gq, a.gk,
                          a.oq, a.ok, wq, wk, a.cosines, a.sines, a.pos, a.partial, p);
    if (e == cudaSuccess)
      e = launch_overlapped(norm_rope_bwd_sum_kernel, dim3(unsigned((a.d + 31) / 32), 2), dim3(1024), 0, a.stream,
                            a.partial, a.dwq, a.dwk, g.x * g.nq, g.x * g.y, a.d);
  }
  if (e != cudaSuccess) {
    snprintf(msg, msglen, "norm and rotation launch: %s", cudaGetErrorString(e));
    return 5;
  }
  return 0;
}

template <typename T, int LPR>
int run_style(const NormRopeArgs& a, const Grid& g, const Dims& p, bool bwd, char* msg, size_t n) {
  return a.pairs ? run<T, LPR, true>(a, g, p, bwd, msg, n) : run<T, LPR, false>(a, g, p, bwd, msg, n);
}

template <typename T>
int run_type(const NormRopeArgs& a, const Grid& g, const Dims& p, bool bwd, char* msg, size_t n) {
  switch (lanes_per_row(a.d)) {
    case 8: return run_style<T, 8>(a, g, p, bwd, msg, n);
    case 16: return run_style<T, 16>(a, g, p, bwd, msg, n);
    default: return run_style<T, 32>(a, g, p, bwd, msg, n);
  }
}

int launch(const NormRopeArgs& a, bool bwd, char* msg, size_t msglen) {
  int sms = 0;
  const cudaError_t e = device_sm_count(&sms);
  if (e != cudaSuccess) {
    snprintf(msg, msglen, "norm and rotation: SM count: %s", cudaGetErrorString(e));
    return 5;
  }
  const Grid g = plan(a.B * a.N, a.Hq, a.Hk, a.d, sms, bwd ? bwd_ctas(a.f32) : 0);
  if (g.x > 0x7fffffffLL || g.y > 65535) {
    snprintf(msg, msglen, "norm and rotation: too many tokens or heads for one launch");
    return 3;
  }
  const Dims p{a.B * a.N, a.N, a.n_pos, int(a.Hq), int(a.Hk), a.d, a.d_rot, g.hp, g.nq, a.eps};
  return a.f32 ? run_type<float>(a, g, p, bwd, msg, msglen)
               : run_type<__nv_bfloat16>(a, g, p, bwd, msg, msglen);
}

}  // namespace

int64_t norm_rope_partial_rows(int64_t B, int64_t Hq, int64_t Hk, int64_t N, int64_t d, int sms) {
  int64_t rows = 0;   // the larger of the two types'
  for (const bool f32 : {false, true}) {
    const Grid g = plan(B * N, Hq, Hk, d, sms, bwd_ctas(f32));
    rows = g.x * g.y > rows ? g.x * g.y : rows;
  }
  return rows;
}

int launch_norm_rope(const NormRopeArgs& a, char* msg, size_t msglen) {
  return launch(a, false, msg, msglen);
}
int launch_norm_rope_bwd(const NormRopeArgs& a, char* msg, size_t msglen) {
  return launch(a, true, msg, msglen);
}

cudaError_t norm_read_and_clear_status(unsigned* value) {
  cudaError_t e = cudaMemcpyFromSymbol(value, g_moa_norm_status, sizeof(unsigned));
  if (e != cudaSuccess || *value == 0) return e;
  const unsigned zero = 0;
  return cudaMemcpyToSymbol(g_moa_norm_status, &zero, sizeof(unsigned));
}

}  // namespace moa
