// Which tokens a query row sees, shared by the kernels of windowed attention, its gradients and the
// attention over the 16- and 32-bit cache.
//
// Of a sequence's `len` tokens the N query rows' positions are the last N: row i stands at
// p = len - N + i and sees token j if (causal) j <= p, and j > p - window or j < sinks.
// So a row sees [0, min(sinks, low)) and [low, end), and the tiles of tokens that a block of rows
// has to visit are a few first ones and a run of later ones.
#pragma once
#include <cstdint>

namespace moa {
namespace win {

constexpr int kNoWindow = 0x7fffffff;
constexpr unsigned kErrIndex = 7u;   // MOA_ERR_DEVICE_INDEX

struct Mask {
  int window;   // kNoWindow: none
  int sinks;
  bool causal;
};

// The first position past what row i sees, and the first token of its window (0 <= low <= end).
__host__ __device__ __forceinline__ int row_end(const Mask& m, int len, int N, int i) {
  if (!m.causal) return len;
  const int n = len - N + i + 1;
  return n < 0 ? 0 : n;
}
__host__ __device__ __forceinline__ int row_low(const Mask& m, int len, int N, int i) {
  const int p = len - N + i;
  return p >= m.window ? p - m.window + 1 : 0;
}

// The tiles of `tile` tokens that rows with positions between those of rows i0 and i1 visit, in order:
// `first` tiles from the sequence's start, then those from `from` on; `n` in all (0: they see nothing).
struct Tiles {
  int first, from, n;
  __host__ __device__ __forceinline__ int at(int t) const { return t < first ? t : t - first + from; }
};
__host__ __device__ __forceinline__ Tiles tiles_of(const Mask& m, int len, int N, int i0, int i1, int tile) {
  const int end = row_end(m, len, N, i1), low = row_low(m, len, N, i0);
  const int stop = end / tile + (end % tile != 0);
  const int s = m.sinks < low ? m.sinks : low;
  Tiles t;
  t.first = s / tile + (s % tile != 0);
  t.from = low / tile;
  if (t.from < t.first) t.from = t.first;
  if (t.first > stop) t.first = stop;
  t.n = t.first + (stop > t.from ? stop - t.from : 0);
  return t;
}

// The same tokens as one sequence without the gap between them: token at(x) of the sequence is the x-th that
// rows i0 .. i1 visit, of n.
struct Run {
  int first, from, n;
  __host__ __device__ __forceinline__ int at(int x) const { return x < first ? x : x - first + from; }
};
__host__ __device__ __forceinline__ Run run_of(const Mask& m, int len, int N, int i0, int i1) {
  const int end = row_end(m, len, N, i1), low = row_low(m, len, N, i0);
  Run r;
  r.first = m.sinks < low ? m.sinks : low;
  r.from = low;
  if (r.first > end) r.first = end;
  r.n = r.first + (end > low ? end - low : 0);
  return r;
}

}  // namespace win
}  // namespace moa
