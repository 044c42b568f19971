// Gradients of windowed attention on CUDA cores, a token's or a query's at a time, over the pairs that see one another and
// nothing else: for outputs that are not finite.  The sums of the tiles give hidden pairs the weight zero, and zero times what is not
// finite reaches every output of the tile.  Values that a pair does see stay as the formula has them.
//
// A warp an output: 32 pairs at a time, a pair a lane for the weights, then pair after pair, a few features a lane.  Rare: called only
// where an output is not finite, and skipped there unless something that is not finite is hidden from a part of the tile (so that
// it may have come through the sums).  About 0.4 us a pair, and few registers: more of them, for more loads on their way at a time, cost the
// tiles of which this is a branch 3 %.
#pragma once
#include <cuda_bf16.h>
#include <cstdint>

#include "window.cuh"

namespace moa {
namespace win {

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ bool is_finite(float x) { return fabsf(x) < INFINITY; }
__device__ __forceinline__ bool sees(const Mask& m, int pos, int j) { return j <= pos && (pos - j < m.window || j < m.sinks); }

// Rows lie on 16-byte boundaries.
template <typename T, int D>
__device__ __forceinline__ float dot(const T* a, const T* b) {
  constexpr int kWord = 16 / sizeof(T);
  float s = 0.f;
#pragma unroll 2
  for (int c = 0; c < D; c += kWord) {
    const uint4 x = *reinterpret_cast<const uint4*>(a + c), y = *reinterpret_cast<const uint4*>(b + c);
    const T *xs = reinterpret_cast<const T*>(&x), *ys = reinterpret_cast<const T*>(&y);
#pragma unroll
    for (int e = 0; e < kWord; ++e) s = fmaf(widen(xs[e]), widen(ys[e]), s);
  }
  return s;
}
template <typename T, int D>
__device__ __forceinline__ bool finite_row(const T* a) {
  constexpr int kWord = 16 / sizeof(T);
  float s = 0.f;   // x * 0 + s is NaN from the first x on that is not finite
#pragma unroll 2
  for (int c = 0; c < D; c += kWord) {
    const uint4 x = *reinterpret_cast<const uint4*>(a + c);
    const T* xs = reinterpret_cast<const T*>(&x);
#pragma unroll
    for (int e = 0; e < kWord; ++e) s = fmaf(widen(xs[e]), 0.f, s);
  }
  return s == 0.f;
}
// acc += w y over the pairs of `pairs` (a lane each), in their order; false once every feature is NaN.
template <typename T, int NO>
__device__ __forceinline__ bool add_pairs(uint32_t pairs, float w, const T* y, float (&acc)[NO]) {
  const int lane = threadIdx.x & 31;
  while (pairs != 0) {
    const int b = __ffs(pairs) - 1;
    pairs &= pairs - 1;
    const float wb = __shfl_sync(0xffffffffu, w, b);
    const T* at = reinterpret_cast<const T*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(y), b)) + lane * NO;
#pragma unroll
    for (int e = 0; e < NO; ++e) acc[e] = fmaf(wb, widen(at[e]), acc[e]);
  }
  bool left = false;
#pragma unroll
  for (int e = 0; e < NO; ++e) left |= acc[e] == acc[e];
  return __any_sync(0xffffffffu, left) != 0;
}

// A query row: its query and its output's gradient, -LSE log2 e, D, position.
template <typename T>
struct RowOf {
  const T* q;
  const T* go;
  float nl, d;
  int pos;
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
      if (!(r.pos >= k1 && (r.pos - k0 < m.window || k1 < m.sinks)))
        odd = !(r.nl < INFINITY) || !is_finite(r.d) || !finite_row<T, DK>(r.q) || !finite_row<T, DV>(r.go);
    }
    found = __any_sync(0xffffffffu, odd);
  }
  while (bad != 0) {
    const int j = first + __ffs(bad) - 1;
    bad &= bad - 1;
    const T *k = t.key(j), *v = t.value(j);
    if (!found && finite_row<T, DK>(k) && finite_row<T, DV>(v)) continue;
    float acc[NO] = {};
    bool open = true;
    for (int x0 = 0; x0 < n && open; x0 += 32) {
      RowOf<T> r{};
      bool pair = false;
      if (x0 + lane < n) {
        r = row(x0 + lane);
        pair = sees(m, r.pos, j);
      }
      float w = 0.f;
      if (pair) {
        w = exp2f(fmaf(dot<T, DK>(r.q, k), c_log2, r.nl));
        if (KEY) w *= dot<T, DV>(r.go, v) - r.d;
      }
      open = add_pairs(__ballot_sync(0xffffffffu, pair), w, KEY ? r.q : r.go, acc);
    }
    write(j, lane * NO, acc);
  }
}

// dQ of the rows `bad` (bits; row(b) is bit b's) of positions p0 .. p1, over the n tokens token(x).
template <typename T, int DK, int DV, typename Row, typename Token, typename Write>
__device__ __forceinline__ void rows_again(uint32_t bad, int p0, int p1, int n, const Mask m, float c_log2, const Tokens<T> t, const Row row,
                                           const Token token, const Write write) {
  constexpr int NO = DK / 32;
  const int lane = threadIdx.x & 31;
  __syncwarp();   // other lanes wrote what is written again
  bool found = false;   // a token with something that is not finite that a row of the tile does not see
  for (int x0 = 0; x0 < n && !found; x0 += 32) {
    bool odd = false;
    if (x0 + lane < n) {
      const int j = token(x0 + lane);
      if (!(j <= p0 && (p1 - j < m.window || j < m.sinks))) odd = !finite_row<T, DK>(t.key(j)) || !finite_row<T, DV>(t.value(j));
    }
    found = __any_sync(0xffffffffu, odd);
  }
  while (bad != 0) {
    const int b = __ffs(bad) - 1;
    bad &= bad - 1;
    const RowOf<T> r = row(b);
    // a row that sees something and is none itself: so are its gradients
    if (r.pos >= 0 && (!found || !(r.nl < INFINITY) || !is_finite(r.d))) continue;
    float acc[NO] = {};
    bool open = true;
    for (int x0 = 0; x0 < n && open; x0 += 32) {
      const int j = x0 + lane < n ? token(x0 + lane) : 0x7fffffff;
      const bool pair = sees(m, r.pos, j);
      float w = 0.f;
      const T* k = nullptr;
      if (pair) {
        k = t.key(j);
        w = exp2f(fmaf(dot<T, DK>(r.q, k), c_log2, r.nl)) * (dot<T, DV>(r.go, t.value(j)) - r.d);
      }
      open = add_pairs(__ballot_sync(0xffffffffu, pair), w, k, acc);
    }
    write(b, lane * NO, acc);
  }
}

}  // namespace win
}  // namespace moa
