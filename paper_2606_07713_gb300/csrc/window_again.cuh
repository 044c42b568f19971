// Gradients of windowed attention on CUDA cores, a token's or a query's at a time, over the pairs that see one another and
// nothing else: for outputs that are not finite.  The sums of the tiles give hidden pairs the weight zero, and zero times what is not
// finite reaches every output of the tile.  Values that a pair does see stay as the formula has them.
//
// A warp four outputs, its pairs 32 at a time.  Rare: only where an output is not finite, and skipped there unless something that is not
// finite is hidden from a part of the tile (so that it may have come through the sums).  What bounds it then: the latency of one
// warp's loads, some 60 ns a pair of four outputs.
#pragma once
#include <cuda_bf16.h>
#include <cstdint>

#include "window.cuh"

namespace moa {
namespace win {

// 32-bit words of a row as numbers: one of float, two of bf16.
template <typename T>
constexpr int kPerWord = 4 / int(sizeof(T));
template <typename T>
__device__ __forceinline__ float number(uint32_t word, int which) {
  if (sizeof(T) == 4) return __uint_as_float(word);
  return __uint_as_float(which == 0 ? word << 16 : word & 0xffff0000u);
}
template <typename T>
__device__ __forceinline__ float dot16(const uint4& a, const uint4& b) {
  const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int e = 0; e < kPerWord<T>; ++e) s = fmaf(number<T>(x[i], e), number<T>(y[i], e), s);
  return s;
}
__device__ __forceinline__ bool is_finite(float x) { return fabsf(x) < INFINITY; }
__device__ __forceinline__ bool sees(const Mask& m, int pos, int j) { return j <= pos && (pos - j < m.window || j < m.sinks); }

template <typename T, int D>
__device__ __forceinline__ bool finite_row(const T* a) {
  constexpr int kWord = 16 / sizeof(T);
  float s = 0.f;   // NaN from the first member on that is not finite
#pragma unroll 4
  for (int c = 0; c < D; c += kWord) {
    const uint4 x = *reinterpret_cast<const uint4*>(a + c);
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < kPerWord<T>; ++e) s = fmaf(number<T>(w[i], e), 0.f, s);
  }
  return s == 0.f;
}
template <typename T>
__device__ __forceinline__ const T* from_lane(const T* p, int lane) {
  return reinterpret_cast<const T*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(p), lane));
}

constexpr int kOutputs = 4;   // of a warp at a time: their pairs' rows are loaded once

// The products of kOutputs rows with 32 others, whose 16-byte words lie with kLanes lanes a row.
template <typename T, int D>
class Dots {
  static constexpr int kWord = 16 / sizeof(T), kLanes = D / kWord, kRows = 32 / kLanes;   // rows a load
  uint4 own_[kOutputs];

 public:
  __device__ __forceinline__ void set(int t, const T* row) {   // (null: zeros)
    own_[t] = row == nullptr ? make_uint4(0, 0, 0, 0) : *reinterpret_cast<const uint4*>(row + (threadIdx.x & 31) % kLanes * kWord);
  }
  // with the lane's row (null: 0)
  __device__ __forceinline__ void operator()(const T* row, float (&out)[kOutputs]) const {
    constexpr int kBatch = kLanes < 8 ? kLanes : 8;   // loads on their way at a time
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int t = 0; t < kOutputs; ++t) out[t] = 0.f;
#pragma unroll 1
    for (int i0 = 0; i0 < kLanes; i0 += kBatch) {
      uint4 x[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const T* y = from_lane(row, (i0 + u) * kRows + lane / kLanes);
        x[u] = y == nullptr ? make_uint4(0, 0, 0, 0) : *reinterpret_cast<const uint4*>(y + lane % kLanes * kWord);
      }
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
#pragma unroll
        for (int t = 0; t < kOutputs; ++t) {
          float s = dot16<T>(own_[t], x[u]);
#pragma unroll
          for (int d = kLanes / 2; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
          s = __shfl_sync(0xffffffffu, s, lane % kRows * kLanes);
          if (lane / kRows == i0 + u) out[t] = s;
        }
      }
    }
  }
};

// acc[t] += w[t] y over the pairs (a lane each) that are pairs of output t, in their order; false once every feature of every
// output below `n_out` is NaN.
template <typename T, int NO>
__device__ __forceinline__ bool add_pairs(const bool (&pair)[kOutputs], const float (&w)[kOutputs], const T* y, int n_out,
                                          float (&acc)[kOutputs][NO]) {
  constexpr int kBatch = 8, kWords = NO / kPerWord<T>;   // 1, 2 or 4
  const int lane = threadIdx.x & 31;
  uint32_t of[kOutputs], any = 0;
#pragma unroll
  for (int t = 0; t < kOutputs; ++t) any |= of[t] = __ballot_sync(0xffffffffu, pair[t]);
  if (any != 0) {
#pragma unroll 1
    for (int b0 = 0; b0 < 32; b0 += kBatch) {
      uint32_t at[kBatch][kWords];
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const uint32_t* from = reinterpret_cast<const uint32_t*>(from_lane(y, b0 + u) + lane * NO);
#pragma unroll
        for (int i = 0; i < kWords; ++i) at[u][i] = any >> (b0 + u) & 1u ? from[i] : 0u;
      }
#pragma unroll
      for (int u = 0; u < kBatch; ++u)
#pragma unroll
        for (int t = 0; t < kOutputs; ++t) {
          const float wb = __shfl_sync(0xffffffffu, w[t], b0 + u);
          if (of[t] >> (b0 + u) & 1u) {
#pragma unroll
            for (int e = 0; e < NO; ++e) acc[t][e] = fmaf(wb, number<T>(at[u][e / kPerWord<T>], e % kPerWord<T>), acc[t][e]);
          }
        }
    }
  }
  bool left = false;
#pragma unroll
  for (int t = 0; t < kOutputs; ++t)
#pragma unroll
    for (int e = 0; e < NO; ++e) left |= t < n_out && acc[t][e] == acc[t][e];
  return __any_sync(0xffffffffu, left) != 0;
}

// A query row: its query and its output's gradient, -LSE log2 e, D, position.
template <typename T>
struct RowOf {
  const T* q;
  const T* go;
  float nl, d;
  int pos;
  bool real;
};
// A key head's keys and values: token j's at k + j * k_sn and v + j * v_sn.
template <typename T>
struct Tokens {
  const T* k;
  const T* v;
  int64_t k_sn, v_sn;
  __device__ __forceinline__ const T* key(int j) const { return k + j * k_sn; }
  __device__ __forceinline__ const T* value(int j) const { return v + j * v_sn; }
};

// dK (KEY) or dV of the tokens `bad` (bit b: token first + b) of a tile k0 .. k1, over the n rows row(x).  write(j, feature, sum of
// one lane's NO features) takes a token's result.  (What is given is held in registers: no reference to a kernel's parameters.)
template <typename T, int DK, int DV, bool KEY, typename Row, typename Write>
__device__ __forceinline__ void tokens_again(uint32_t bad, int first, int k0, int k1, int n, const Mask m, float c_log2, const Tokens<T> t,
                                             const Row row, const Write write) {
  constexpr int NO = (KEY ? DK : DV) / 32;
  const int lane = threadIdx.x & 31;
  __syncwarp();   // other lanes wrote what is written again
  bool found = false;   // a row with something that is not finite that a token of the tile does not see
  for (int x0 = 0; x0 < n && !found; x0 += 32) {
    bool odd = false;
    if (x0 + lane < n) {
      const RowOf<T> r = row(x0 + lane);
      if (r.real && !(r.pos >= k1 && (r.pos - k0 < m.window || k1 < m.sinks)))
        odd = !(r.nl < INFINITY) || !is_finite(r.d) || !finite_row<T, DK>(r.q) || !finite_row<T, DV>(r.go);
    }
    found = __any_sync(0xffffffffu, odd);
  }
  while (bad != 0) {
    int j[kOutputs], n_out = 0;
    Dots<T, DK> score;
    Dots<T, DV> change;
#pragma unroll
    for (int o = 0; o < kOutputs; ++o) {
      j[o] = 0x7fffffff;   // no row sees it
      while (bad != 0) {
        const int at = first + __ffs(bad) - 1;
        bad &= bad - 1;
        if (!found && finite_row<T, DK>(t.key(at)) && finite_row<T, DV>(t.value(at))) continue;
        // a row that sees the token and whose weights are none (for dK, whose D is): so is the sum
        bool done = false;
#pragma unroll 4
        for (int x = lane; x < n; x += 32) {
          const RowOf<T> r = row(x);
          done |= r.real && (!(r.nl < INFINITY) || (KEY && !is_finite(r.d))) && sees(m, r.pos, at);
        }
        if (__any_sync(0xffffffffu, done)) continue;
        j[o] = at;
        n_out = o + 1;
        break;
      }
      const bool some = j[o] != 0x7fffffff;
      score.set(o, some ? t.key(j[o]) : nullptr);
      change.set(o, some ? t.value(j[o]) : nullptr);
    }
    if (n_out == 0) return;
    float acc[kOutputs][NO] = {};
    bool open = true;
    for (int x0 = 0; x0 < n && open; x0 += 32) {
      RowOf<T> r{};
      bool pair[kOutputs] = {}, any = false;
      if (x0 + lane < n) {
        r = row(x0 + lane);
#pragma unroll
        for (int o = 0; o < kOutputs; ++o) any |= pair[o] = r.real && sees(m, r.pos, j[o]);
      }
      if (!__any_sync(0xffffffffu, any)) continue;
      float w[kOutputs];
      score(any ? r.q : nullptr, w);
#pragma unroll
      for (int o = 0; o < kOutputs; ++o) w[o] = exp2f(fmaf(w[o], c_log2, r.nl));
      if (KEY) {
        float dp[kOutputs];
        change(any ? r.go : nullptr, dp);
#pragma unroll
        for (int o = 0; o < kOutputs; ++o) w[o] *= dp[o] - r.d;
      }
      open = add_pairs(pair, w, KEY ? r.q : r.go, n_out, acc);
    }
#pragma unroll
    for (int o = 0; o < kOutputs; ++o)
      if (o < n_out) write(j[o], lane * NO, acc[o]);
  }
}

// dQ of the rows `bad` (bits; row(b) is bit b's) of positions p0 .. p1, over the n tokens token(x) (negative: none).
template <typename T, int DK, int DV, typename Row, typename Token, typename Write>
__device__ __forceinline__ void rows_again(uint32_t bad, int p0, int p1, int n, const Mask m, float c_log2, const Tokens<T> t, const Row row,
                                           const Token token, const Write write) {
  constexpr int NO = DK / 32;
  const int lane = threadIdx.x & 31;
  __syncwarp();   // other lanes wrote what is written again
  bool found = false;   // a token with something that is not finite that a row of the tile does not see
  for (int x0 = 0; x0 < n && !found; x0 += 32) {
    const int j = x0 + lane < n ? token(x0 + lane) : -1;
    bool odd = false;
    if (j >= 0 && !(j <= p0 && (p1 - j < m.window || j < m.sinks))) odd = !finite_row<T, DK>(t.key(j)) || !finite_row<T, DV>(t.value(j));
    found = __any_sync(0xffffffffu, odd);
  }
  while (bad != 0) {
    int which[kOutputs], pos[kOutputs], n_out = 0;
    float nl[kOutputs], d[kOutputs];
    Dots<T, DK> score;
    Dots<T, DV> change;
#pragma unroll
    for (int o = 0; o < kOutputs; ++o) {
      which[o] = 0, pos[o] = -1, nl[o] = d[o] = 0.f;   // sees nothing
      const T *q = nullptr, *go = nullptr;
      while (bad != 0) {
        const int b = __ffs(bad) - 1;
        bad &= bad - 1;
        const RowOf<T> r = row(b);
        // a row that sees something and is none itself: so are its gradients
        if (r.pos >= 0 && (!found || !(r.nl < INFINITY) || !is_finite(r.d))) continue;
        which[o] = b, pos[o] = r.pos, nl[o] = r.nl, d[o] = r.d, q = r.q, go = r.go;
        n_out = o + 1;
        break;
      }
      score.set(o, q);
      change.set(o, go);
    }
    if (n_out == 0) return;
    float acc[kOutputs][NO] = {};
    bool open = true;
    for (int x0 = 0; x0 < n && open; x0 += 32) {
      const int j = x0 + lane < n ? token(x0 + lane) : -1;
      bool pair[kOutputs], any = false;
#pragma unroll
      for (int o = 0; o < kOutputs; ++o) any |= pair[o] = j >= 0 && sees(m, pos[o], j);
      if (!__any_sync(0xffffffffu, any)) continue;
      const T* k = any ? t.key(j) : nullptr;
      float w[kOutputs], dp[kOutputs];
      score(k, w);
      change(any ? t.value(j) : nullptr, dp);
#pragma unroll
      for (int o = 0; o < kOutputs; ++o) w[o] = exp2f(fmaf(w[o], c_log2, nl[o])) * (dp[o] - d[o]);
      open = add_pairs(pair, w, k, n_out, acc);
    }
#pragma unroll
    for (int o = 0; o < kOutputs; ++o)
      if (o < n_out) write(which[o], lane * NO, acc[o]);
  }
}

}  // namespace win
}  // namespace moa
