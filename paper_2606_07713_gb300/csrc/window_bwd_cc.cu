// Gradients of causal attention with a sliding window and first tokens that stay visible, on CUDA cores
// (sm_103a): for fp32, and for bf16 tensors whose strides no tensor map can describe.
//
// Mathematics, with P_ij = exp(scale <q_i, k_j> - LSE_i) for the tokens j that row i sees (window.cuh), 0 for
// the others, and D_i = <dO_i, O_i>:
//     dV_j = sum_i P_ij dO_i,   dS_ij = P_ij (<dO_i, v_j> - D_i),
//     dQ_i = scale sum_j dS_ij k_j,   dK_j = scale sum_i dS_ij q_i,
// the sums over i also over the query heads that share the key head.  The weights are rebuilt from the
// scores; nothing of N_q x N_k size is stored.
//
//   delta   D of every row and the row's -LSE log2 e (-infinity for rows that see nothing: their weights
//           are then zero), a warp a row;
//   tiles   one launch, two kinds of CTAs.  dK and dV: 64 tokens of a key head and a piece of the rows that see
//           them, 32 rows at a time.  A token's rows are those of its window; a sink's are all later ones: token
//           tiles with more rows than a piece are cut, a piece being a window's rows, or less where there are too
//           few CTAs for the machine.  dQ: 64 rows, 32 tokens at a time.  The next step's rows (tokens) are on their
//           way while a step is computed;
//   again   sums that are not finite, once more from the pairs that see one another (window_again.cuh), if there are any: 1.4 us of
//           a call that has none (its code as a branch of the tiles, called or inlined, cost their loops 2 to 18 %);
//   join    adds the pieces, in order.
// Rows of a key head are counted position by position (row r: position r / G, head r % G of the group).
// No atomics: results do not depend on the order in which CTAs run.
//
// What bounds it: shared memory's data path (47 %) and issue slots (40 %) about equally, with the barriers of a step as the largest
// wait; multiply-adds are at 23 % of their rate (2 x (6 / 3) heads x 517 x (128 / 64), window 100: 55.6 us, in four launches).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdio>

#include "internal.h"
#include "ops_internal.h"
#include "window.cuh"
#include "window_again.cuh"

namespace moa {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kKeysKv = 64, kRowsKv = 32;   // dkdv: tokens of a CTA, rows of a step
constexpr int kRowsQ = 64, kKeysQ = 32;     // dq: rows of a CTA, tokens of a step
constexpr int kThreads = 256;
constexpr int64_t kMostPieces = 1216;       // of cut token tiles: eight for each SM
constexpr int64_t kMostAgain = 304;         // CTAs that look for sums to compute once more: two for each SM

struct Params {
  View q, k, v, o, go, dq, dk, dv;
  const float* lse;
  float* nl;      // [B * Hk][N * G] -LSE log2 e, rows of a key head in their order
  float* delta;   // alike
  float* part;    // [piece item][64][DK + DV], null: no pieces
  float* part_q;  // [dQ tile][piece][64][DK], if dQ's tiles come in pieces
  uint32_t* odd;  // [CTA of the tiles][warp] which of its eight rows (tokens: dK, and dV in the second byte) have sums that are not finite
  int Hk, N, G, Nk;
  win::Mask mask;
  float c_log2, scale;
  int n_kt;       // tiles of tokens
  int cut;        // the first `cut` of them are cut into `pieces` pieces of `piece_rows` rows
  int pieces;
  int64_t piece_rows;
  int n_rt;       // tiles of rows
  int q_pieces;   // pieces of a dQ tile's tokens
};

template <typename T>
__device__ __forceinline__ float4 load4(const T* p);
template <>
__device__ __forceinline__ float4 load4(const float* p) {
  return *reinterpret_cast<const float4*>(p);
}
template <>
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p) {
  const uint2 x = *reinterpret_cast<const uint2*>(p);
  return make_float4(__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xffff0000u), __uint_as_float(x.y << 16),
                     __uint_as_float(x.y & 0xffff0000u));
}
__device__ __forceinline__ void store4(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
__device__ __forceinline__ void store4(__nv_bfloat16* p, float4 v) {
  __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
  *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<uint32_t*>(&a), *reinterpret_cast<uint32_t*>(&b));
}
// d += a b for pairs: one instruction.
__device__ __forceinline__ void fma2(float& d0, float& d1, float a0, float a1, float b0, float b1) {
  asm("{\n\t.reg .b64 ra, rb, rd;\n\tmov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %5};\n\tmov.b64 rd, {%0, %1};\n\t"
      "fma.rn.f32x2 rd, ra, rb, rd;\n\tmov.b64 {%0, %1}, rd;\n\t}"
      : "+f"(d0), "+f"(d1)
      : "f"(a0), "f"(a1), "f"(b0), "f"(b1));
}
// A sum of products in two halves, which are added at the end.
struct Sum2 {
  float a, b;
  __device__ __forceinline__ float all() const { return a + b; }
};
__device__ __forceinline__ void dot4(float4 x, float4 y, Sum2& s) {
  fma2(s.a, s.b, x.x, x.y, y.x, y.y);
  fma2(s.a, s.b, x.z, x.w, y.z, y.w);
}
__device__ __forceinline__ void axpy4(float w, float4 v, float* acc) {
  fma2(acc[0], acc[1], w, w, v.x, v.y);
  fma2(acc[2], acc[3], w, w, v.z, v.w);
}

template <typename T>
__device__ __forceinline__ const T* row_of(const View& x, int64_t b, int64_t h, int64_t n) {
  return static_cast<const T*>(x.p) + b * x.sb + h * x.sh + n * x.sn;
}

template <typename T, int DV>
__global__ void __launch_bounds__(kThreads)
window_delta_kernel(Params p, int64_t rows) {
  wait_for_previous();
  const int lane = threadIdx.x & 31;
  const int64_t r = int64_t(blockIdx.x) * 8 + (threadIdx.x >> 5);
  if (r >= rows) return;
  const int64_t per = int64_t(p.N) * p.G, bh = r / per, b = bh / p.Hk, h = bh - b * p.Hk;
  const int64_t at = r - bh * per, i = at / p.G, g = at - i * p.G, hq = h * p.G + g;
  float s = 0.f;
  if (lane * 4 < DV) {
    const float4 x = load4(row_of<T>(p.o, b, hq, i) + lane * 4), y = load4(row_of<T>(p.go, b, hq, i) + lane * 4);
    s = fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, x.w * y.w)));
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
  if (lane == 0) {
    const float l = p.lse[(b * p.Hk * p.G + hq) * p.N + i];
    p.delta[r] = s;
    p.nl[r] = l == -INFINITY ? -INFINITY : -l * kLog2e;
  }
}

// Four features from global into shared memory: asynchronously (fp32), or widened (bf16).  Absent ones are zeros.
__device__ __forceinline__ void fill4(float* dst, const float* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(uint32_t(__cvta_generic_to_shared(dst))), "l"(src),
               "r"(there ? 16 : 0)
               : "memory");
}
__device__ __forceinline__ void fill4(float* dst, const __nv_bfloat16* src, bool there) {
  *reinterpret_cast<float4*>(dst) = there ? load4(src) : make_float4(0.f, 0.f, 0.f, 0.f);
}
__device__ __forceinline__ void fill_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void fill_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// Rows r0 .. of X and Y of a key head into shared memory; rows past `rows` are zero.
template <typename T, int DX, int DY, int ROWS>
__device__ __forceinline__ void fill_rows(const View& x, const View& y, float* sx, float* sy, int b, int h, int G, int r0,
                                          int rows) {
  for (int r = threadIdx.x >> 4; r < ROWS; r += kThreads / 16) {
    const bool there = r0 + r < rows;
    const int at = there ? r0 + r : r0, i = int(unsigned(at) / unsigned(G));
    const int64_t hq = int64_t(h) * G + (at - i * G);
    const T *px = row_of<T>(x, b, hq, i), *py = row_of<T>(y, b, hq, i);
#pragma unroll
    for (int c = 4 * (threadIdx.x & 15); c < DX; c += 64) fill4(sx + r * (DX + 4) + c, px + c, there);
#pragma unroll
    for (int c = 4 * (threadIdx.x & 15); c < DY; c += 64) fill4(sy + r * (DY + 4) + c, py + c, there);
  }
}
// Tokens run.at(x0) .. alike.
template <typename T, int DK, int DV, int TOKENS>
__device__ __forceinline__ void fill_tokens(const View& k, const View& v, float* sk, float* sv, int b, int h, int x0,
                                            const win::Run& run) {
  for (int j = threadIdx.x >> 4; j < TOKENS; j += kThreads / 16) {
    const bool there = x0 + j < run.n;
    const int n = run.at(there ? x0 + j : x0);
    const T *pk = row_of<T>(k, b, h, n), *pv = row_of<T>(v, b, h, n);
#pragma unroll
    for (int c = 4 * (threadIdx.x & 15); c < DK; c += 64) fill4(sk + j * (DK + 4) + c, pk + c, there);
#pragma unroll
    for (int c = 4 * (threadIdx.x & 15); c < DV; c += 64) fill4(sv + j * (DV + 4) + c, pv + c, there);
  }
}

// The rows [ra, rz) that see a token of tile kt, or a piece of them (piece < 0: all); false: there is no such piece.
__device__ __forceinline__ bool rows_of_piece(const Params& p, int kt, int piece, int* ra, int* rz) {
  const int k0 = kt * kKeysKv, keys = p.Nk - k0 < kKeysKv ? p.Nk - k0 : kKeysKv, off = p.Nk - p.N;
  // from position k0 to the last token's window, or to the end
  const int64_t i0 = k0 > off ? int64_t(k0) - off : 0;
  int64_t i1 = p.N;
  if (k0 >= p.mask.sinks && p.mask.window != win::kNoWindow) {
    const int64_t n = int64_t(k0) + keys - 1 + p.mask.window - off;
    i1 = n < 0 ? 0 : n < i1 ? n : i1;
  }
  int64_t a = i0 * p.G, z = i1 * p.G;
  if (piece >= 0) {
    a += piece * p.piece_rows;
    if (a >= z) return false;
    if (a + p.piece_rows < z) z = a + p.piece_rows;
  }
  *ra = int(a), *rz = int(z);
  return true;
}

// Buffers of a step's rows or tokens: two where two CTAs still fit on an SM (8 warps alone left it waiting for shared memory
// half of the time: gradients of 2 x (6 / 3) heads x 517 x (128 / 64), window 100: 77 us, with all that is below 61, and with products in pairs 54).
__host__ __device__ constexpr int buffers(int dk, int dv) { return dk + dv <= 192 ? 2 : 1; }

template <int DK, int DV>
struct KvSmem {
  static constexpr int kLdW = kKeysKv + 4;
  static constexpr int kRows = kRowsKv * (DK + 4 + DV + 4);   // a step's queries and output gradients
  static constexpr int kFloats = kKeysKv * (DK + 4 + DV + 4) + buffers(DK, DV) * kRows + kRowsKv * kLdW;
};

// Which of a warp's eight tokens (rows) have a sum that is not finite: thread (ty, tx) holds N features of each of four, 4 ty + a.
template <int N>
__device__ __forceinline__ uint32_t odd_sums(const float (&sum)[4][N]) {
  float any = 0.f;
#pragma unroll
  for (int c = 0; c < N; ++c) any += (sum[0][c] * 0.f + sum[1][c] * 0.f) + (sum[2][c] * 0.f + sum[3][c] * 0.f);
  uint32_t bad = 0;
  if (!__any_sync(0xffffffffu, any != 0.f)) return bad;
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    float odd = 0.f;   // x * 0 + odd is NaN from the first x on that is not finite
#pragma unroll
    for (int c = 0; c < N; ++c) odd = fmaf(sum[a][c], 0.f, odd);
    const uint32_t which = __ballot_sync(0xffffffffu, odd != 0.f);
    bad |= uint32_t((which & 0xffffu) != 0) << a | uint32_t(which >> 16 != 0) << (a + 4);
  }
  return bad;
}

// dK (KEY) or dV of a warp's tokens `bad` once more, from what their rows see (window_again.cuh): sums that are not finite, as hidden
// pairs' may not be (0 * NaN).
template <typename T, int DK, int DV, bool KEY>
__device__ __forceinline__ void tokens_again(const Params& p, unsigned index, int warp, uint32_t bad) {
  const unsigned per = unsigned(p.cut * p.pieces + p.n_kt - p.cut);
  const int bh = int(index / per), item = int(index - unsigned(bh) * per);
  const bool whole = item >= p.cut * p.pieces;
  const int kt = whole ? item - p.cut * p.pieces + p.cut : item / p.pieces, piece = whole ? 0 : item - kt * p.pieces;
  const int b = bh / p.Hk, h = bh - b * p.Hk, k0 = kt * kKeysKv, off = p.Nk - p.N;
  const int keys = p.Nk - k0 < kKeysKv ? p.Nk - k0 : kKeysKv, first = 8 * warp;
  const int64_t rows = int64_t(p.N) * p.G;
  int ra, rz;
  rows_of_piece(p, kt, whole ? -1 : piece, &ra, &rz);
  if (keys - first < 8) bad &= keys > first ? (1u << (keys - first)) - 1 : 0u;
  const int G = p.G;
  const int64_t q_sh = p.q.sh, q_sn = p.q.sn, go_sh = p.go.sh, go_sn = p.go.sn;
  const T *q = row_of<T>(p.q, b, int64_t(h) * G, 0), *go = row_of<T>(p.go, b, int64_t(h) * G, 0);
  const float *nl = p.nl + bh * rows + ra, *delta = p.delta + bh * rows + ra;
  win::tokens_again<T, DK, DV, KEY>(
      bad, k0 + first, k0, k0 + keys - 1, rz - ra, p.mask, p.c_log2,
      win::Tokens<T>{row_of<T>(p.k, b, h, 0), row_of<T>(p.v, b, h, 0), p.k.sn, p.v.sn},
      [=](int x) {
        const int r = ra + x, i = int(unsigned(r) / unsigned(G)), g = r - i * G;
        return win::RowOf<T>{q + g * q_sh + i * q_sn, go + g * go_sh + i * go_sn, nl[x], delta[x], i + off, true};
      },
      [&](int j, int f, const float(&sum)[(KEY ? DK : DV) / 32]) {
        float* to = p.part + (((int64_t(bh) * p.cut + kt) * p.pieces + piece) * kKeysKv + (j - k0)) * (DK + DV) + (KEY ? 0 : DK) + f;
        T* dst = const_cast<T*>(row_of<T>(KEY ? p.dk : p.dv, b, h, j)) + f;
        const float mul = KEY ? p.scale : 1.f;
#pragma unroll
        for (int e = 0; e < (KEY ? DK : DV) / 32; ++e)
          if (whole)
            dst[e] = T(sum[e] * mul);
          else
            to[e] = sum[e];
      });
}

template <typename T, int DK, int DV>
__device__ __forceinline__ uint32_t dkdv_tile(const Params& p, unsigned index, float* smem) {
  using S = KvSmem<DK, DV>;
  constexpr int kLdW = S::kLdW, kBuf = buffers(DK, DV);
  float* sK = smem;
  float* sV = sK + kKeysKv * (DK + 4);
  float* sRows = sV + kKeysKv * (DV + 4);
  float* sP = sRows + kBuf * S::kRows;   // [rows][tokens]: the weights, then dS
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  // items of a key head: the pieces of its first `cut` tiles, then the other tiles
  const unsigned per = unsigned(p.cut * p.pieces + p.n_kt - p.cut);
  const int bh = int(index / per), b = bh / p.Hk, h = bh - b * p.Hk;
  const int item = int(index - unsigned(bh) * per);
  const bool whole = item >= p.cut * p.pieces;
  const int kt = whole ? item - p.cut * p.pieces + p.cut : item / p.pieces, piece = whole ? 0 : item - kt * p.pieces;
  const int k0 = kt * kKeysKv, off = p.Nk - p.N;   // row i's position: i + off
  const int keys = p.Nk - k0 < kKeysKv ? p.Nk - k0 : kKeysKv;
  const int64_t rows = int64_t(p.N) * p.G;
  int ra, rz;
  if (!rows_of_piece(p, kt, whole ? -1 : piece, &ra, &rz)) return 0;   // the join adds what pieces there are
  fill_tokens<T, DK, DV, kKeysKv>(p.k, p.v, sK, sV, b, h, k0, win::Run{p.Nk, p.Nk, p.Nk});
  if (ra < rz) fill_rows<T, DK, DV, kRowsKv>(p.q, p.go, sRows, sRows + kRowsKv * (DK + 4), b, h, p.G, ra, rz);
  fill_commit();
  float dv[4][DV / 16], dk[4][DK / 16];   // tokens 4 ty + a, features 64 c + 4 tx + e
#pragma unroll
  for (int a = 0; a < 4; ++a) {
#pragma unroll
    for (int c = 0; c < DV / 16; ++c) dv[a][c] = 0.f;
#pragma unroll
    for (int c = 0; c < DK / 16; ++c) dk[a][c] = 0.f;
  }
  for (int r0 = ra, step = 0; r0 < rz; r0 += kRowsKv, ++step) {
    const float* sQ = sRows + (step % kBuf) * S::kRows;
    const float* sG = sQ + kRowsKv * (DK + 4);
    float* next = sRows + ((step + 1) % kBuf) * S::kRows;
    if (kBuf == 2 && r0 + kRowsKv < rz)
      fill_rows<T, DK, DV, kRowsKv>(p.q, p.go, next, next + kRowsKv * (DK + 4), b, h, p.G, r0 + kRowsKv, rz);
    fill_commit();
    fill_wait<kBuf - 1>();
    __syncthreads();
    // A warp whose eight tokens no row of the step sees has nothing to add: beside a window's ends, and of the tokens
    // behind the sinks in all rows that only see those.
    const int p0 = int(unsigned(r0) / unsigned(p.G)) + off, r1 = r0 + kRowsKv < rz ? r0 + kRowsKv : rz;
    const int p1 = int(unsigned(r1 - 1) / unsigned(p.G)) + off, j0 = k0 + 8 * (threadIdx.x >> 5);
    if (j0 <= p1 && (p0 - (j0 + 7) < p.mask.window || j0 < p.mask.sinks)) {
      // rows tx, tx + 16 against tokens 4 ty + a
      Sum2 s2[4][2], e2[4][2];
#pragma unroll
      for (int a = 0; a < 4; ++a) s2[a][0] = s2[a][1] = e2[a][0] = e2[a][1] = Sum2{0.f, 0.f};
#pragma unroll 4
      for (int c = 0; c < DK; c += 4) {
        const float4 q0 = *reinterpret_cast<const float4*>(sQ + tx * (DK + 4) + c);
        const float4 q1 = *reinterpret_cast<const float4*>(sQ + (tx + 16) * (DK + 4) + c);
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const float4 kk = *reinterpret_cast<const float4*>(sK + (4 * ty + a) * (DK + 4) + c);
          dot4(q0, kk, s2[a][0]);
          dot4(q1, kk, s2[a][1]);
        }
      }
#pragma unroll 4
      for (int c = 0; c < DV; c += 4) {
        const float4 g0 = *reinterpret_cast<const float4*>(sG + tx * (DV + 4) + c);
        const float4 g1 = *reinterpret_cast<const float4*>(sG + (tx + 16) * (DV + 4) + c);
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const float4 vv = *reinterpret_cast<const float4*>(sV + (4 * ty + a) * (DV + 4) + c);
          dot4(g0, vv, e2[a][0]);
          dot4(g1, vv, e2[a][1]);
        }
      }
      float s[4][2], e[4][2];
#pragma unroll
      for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int x = 0; x < 2; ++x) s[a][x] = s2[a][x].all(), e[a][x] = e2[a][x].all();
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int r = r0 + tx + 16 * x;
        const bool live = r < rz;
        const int pos = int(unsigned(live ? r : rz - 1) / unsigned(p.G)) + off;
        const float nl = live ? p.nl[bh * rows + r] : -INFINITY, d = live ? p.delta[bh * rows + r] : 0.f;
        // the weights into s, dS into e
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const int j = k0 + 4 * ty + a;
          const bool seen = live && j <= pos && (pos - j < p.mask.window || j < p.mask.sinks) && j < p.Nk;
          s[a][x] = seen ? exp2f(fmaf(s[a][x], p.c_log2, nl)) : 0.f;
          e[a][x] = seen ? s[a][x] * (e[a][x] - d) : 0.f;
        }
        *reinterpret_cast<float4*>(sP + (tx + 16 * x) * kLdW + 4 * ty) = make_float4(s[0][x], s[1][x], s[2][x], s[3][x]);
      }
      __syncwarp();   // tokens 4 ty .. of all rows: written and read by the same half warp
#pragma unroll 4
      for (int r = 0; r < kRowsKv; ++r) {
        const float4 w = *reinterpret_cast<const float4*>(sP + r * kLdW + 4 * ty);
#pragma unroll
        for (int c = 0; c < DV / 64; ++c) {
          const float4 g = *reinterpret_cast<const float4*>(sG + r * (DV + 4) + 64 * c + 4 * tx);
          axpy4(w.x, g, dv[0] + 4 * c);
          axpy4(w.y, g, dv[1] + 4 * c);
          axpy4(w.z, g, dv[2] + 4 * c);
          axpy4(w.w, g, dv[3] + 4 * c);
        }
      }
      __syncwarp();
#pragma unroll
      for (int x = 0; x < 2; ++x)
        *reinterpret_cast<float4*>(sP + (tx + 16 * x) * kLdW + 4 * ty) = make_float4(e[0][x], e[1][x], e[2][x], e[3][x]);
      __syncwarp();
#pragma unroll 4
      for (int r = 0; r < kRowsKv; ++r) {
        const float4 w = *reinterpret_cast<const float4*>(sP + r * kLdW + 4 * ty);
#pragma unroll
        for (int c = 0; c < DK / 64; ++c) {
          const float4 q = *reinterpret_cast<const float4*>(sQ + r * (DK + 4) + 64 * c + 4 * tx);
          axpy4(w.x, q, dk[0] + 4 * c);
          axpy4(w.y, q, dk[1] + 4 * c);
          axpy4(w.z, q, dk[2] + 4 * c);
          axpy4(w.w, q, dk[3] + 4 * c);
        }
      }
    }
    __syncthreads();   // this step's rows make room for others
    if (kBuf == 1 && r0 + kRowsKv < rz)
      fill_rows<T, DK, DV, kRowsKv>(p.q, p.go, next, next + kRowsKv * (DK + 4), b, h, p.G, r0 + kRowsKv, rz);
  }
  fill_wait<0>();
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    const int j = 4 * ty + a;
    if (j >= keys) continue;
    if (!whole) {
      float* dst = p.part + (((int64_t(bh) * p.cut + kt) * p.pieces + piece) * kKeysKv + j) * (DK + DV);
#pragma unroll
      for (int c = 0; c < DK / 64; ++c)
        store4(dst + 64 * c + 4 * tx, make_float4(dk[a][4 * c], dk[a][4 * c + 1], dk[a][4 * c + 2], dk[a][4 * c + 3]));
#pragma unroll
      for (int c = 0; c < DV / 64; ++c)
        store4(dst + DK + 64 * c + 4 * tx, make_float4(dv[a][4 * c], dv[a][4 * c + 1], dv[a][4 * c + 2], dv[a][4 * c + 3]));
      continue;
    }
    T* ok = const_cast<T*>(row_of<T>(p.dk, b, h, k0 + j));
    T* ov = const_cast<T*>(row_of<T>(p.dv, b, h, k0 + j));
#pragma unroll
    for (int c = 0; c < DK / 64; ++c)
      store4(ok + 64 * c + 4 * tx, make_float4(dk[a][4 * c] * p.scale, dk[a][4 * c + 1] * p.scale, dk[a][4 * c + 2] * p.scale,
                                               dk[a][4 * c + 3] * p.scale));
#pragma unroll
    for (int c = 0; c < DV / 64; ++c)
      store4(ov + 64 * c + 4 * tx, make_float4(dv[a][4 * c], dv[a][4 * c + 1], dv[a][4 * c + 2], dv[a][4 * c + 3]));
  }
  return odd_sums(dk) | odd_sums(dv) << 8;
}

// Adds the pieces of cut tiles: four features of a token a thread.
template <typename T, int DK, int DV>
__global__ void __launch_bounds__(kThreads)
window_dkdv_join_kernel(Params p, int64_t n) {
  wait_for_previous();
  constexpr int kQuads = (DK + DV) / 4;
  const int64_t x = int64_t(blockIdx.x) * kThreads + threadIdx.x;
  if (x >= n) return;
  const int64_t row = x / kQuads, c = (x - row * kQuads) * 4;        // row: (key head, tile, token)
  const int64_t tile = row / kKeysKv, j = row - tile * kKeysKv;
  const int64_t bh = tile / p.cut, kt = tile - bh * p.cut, b = bh / p.Hk, h = bh - b * p.Hk;
  if (kt * kKeysKv + j >= p.Nk) return;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  int ra, rz;
  for (int i = 0; i < p.pieces && rows_of_piece(p, int(kt), i, &ra, &rz); ++i) {
    const float4 v = load4(p.part + ((tile * p.pieces + i) * kKeysKv + j) * (DK + DV) + c);
    s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
  }
  if (c < DK)
    store4(const_cast<T*>(row_of<T>(p.dk, b, h, kt * kKeysKv + j)) + c,
           make_float4(s.x * p.scale, s.y * p.scale, s.z * p.scale, s.w * p.scale));
  else
    store4(const_cast<T*>(row_of<T>(p.dv, b, h, kt * kKeysKv + j)) + (c - DK), s);
}

template <int DK, int DV>
struct QSmem {
  static constexpr int kLdW = kRowsQ + 4;
  static constexpr int kTokens = kKeysQ * (DK + 4 + DV + 4);   // a step's keys and values
  static constexpr int kFloats = kRowsQ * (DK + 4 + DV + 4) + buffers(DK, DV) * kTokens + kKeysQ * kLdW;
};

// dQ of a warp's rows `bad` once more, from the tokens that they see.
template <typename T, int DK, int DV>
__device__ __forceinline__ void rows_again(const Params& p, unsigned index, int warp, uint32_t bad) {
  const unsigned tile = index / unsigned(p.q_pieces), piece = index - tile * unsigned(p.q_pieces);
  const int bh = int(tile / unsigned(p.n_rt)), rt = p.n_rt - 1 - int(tile - unsigned(bh) * unsigned(p.n_rt));
  const int b = bh / p.Hk, h = bh - b * p.Hk, r0 = rt * kRowsQ, off = p.Nk - p.N, first = r0 + 8 * warp;
  const int64_t rows = int64_t(p.N) * p.G;
  const int live = int(rows - r0 < kRowsQ ? rows - r0 : kRowsQ), i0 = r0 / p.G, i1 = (r0 + live - 1) / p.G;
  const win::Run run = win::run_of(p.mask, p.Nk, p.N, i0, i1);
  const int all = (run.n + kKeysQ - 1) / kKeysQ;
  const int begin = int(int64_t(all) * piece / p.q_pieces) * kKeysQ, steps = int(int64_t(all) * (piece + 1) / p.q_pieces);
  const int end = int64_t(steps) * kKeysQ < run.n ? steps * kKeysQ : run.n;
  if (rows - first < 8) bad &= rows > first ? (1u << (rows - first)) - 1 : 0u;
  win::rows_again<T, DK, DV>(
      bad, i0 + off, i1 + off, end - begin, p.mask, p.c_log2,
      win::Tokens<T>{row_of<T>(p.k, b, h, 0), row_of<T>(p.v, b, h, 0), p.k.sn, p.v.sn},
      [&](int t) {
        const int r = first + t, i = r / p.G;
        const int64_t hq = int64_t(h) * p.G + (r - i * p.G);
        return win::RowOf<T>{row_of<T>(p.q, b, hq, i), row_of<T>(p.go, b, hq, i), p.nl[bh * rows + r], p.delta[bh * rows + r], i + off, true};
      },
      [=](int x) { return run.at(begin + x); },
      [&](int t, int f, const float(&sum)[DK / 32]) {
        const int r = first + t, i = r / p.G;
        float* to = p.part_q + (((int64_t(bh) * p.n_rt + rt) * p.q_pieces + piece) * kRowsQ + (r - r0)) * DK + f;
        T* dst = const_cast<T*>(row_of<T>(p.dq, b, int64_t(h) * p.G + (r - i * p.G), i)) + f;
#pragma unroll
        for (int e = 0; e < DK / 32; ++e)
          if (p.q_pieces > 1)
            to[e] = sum[e];
          else
            dst[e] = T(sum[e] * p.scale);
      });
}

template <typename T, int DK, int DV>
__device__ __forceinline__ uint32_t dq_tile(const Params& p, unsigned index, float* smem) {
  using S = QSmem<DK, DV>;
  constexpr int kLdW = S::kLdW, kBuf = buffers(DK, DV);
  float* sQ = smem;
  float* sG = sQ + kRowsQ * (DK + 4);
  float* sTokens = sG + kRowsQ * (DV + 4);
  float* sS = sTokens + kBuf * S::kTokens;   // [tokens][rows]
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const unsigned tile = index / unsigned(p.q_pieces), piece = index - tile * unsigned(p.q_pieces);
  const int bh = int(tile / unsigned(p.n_rt)), b = bh / p.Hk, h = bh - b * p.Hk;
  // the last rows, which see the most without a window, come first
  const int rt = p.n_rt - 1 - int(tile - unsigned(bh) * unsigned(p.n_rt)), r0 = rt * kRowsQ;
  const int64_t rows = int64_t(p.N) * p.G;
  const int live = int(rows - r0 < kRowsQ ? rows - r0 : kRowsQ);
  const int off = p.Nk - p.N;
  const int i0 = r0 / p.G, i1 = (r0 + live - 1) / p.G;
  // the tokens that they visit, 32 at a time, the sinks and the window's next to each other
  const win::Run run = win::run_of(p.mask, p.Nk, p.N, i0, i1);
  const int all = (run.n + kKeysQ - 1) / kKeysQ;
  const int begin = int(int64_t(all) * piece / p.q_pieces), steps = int(int64_t(all) * (piece + 1) / p.q_pieces);   // this piece's
  fill_rows<T, DK, DV, kRowsQ>(p.q, p.go, sQ, sG, b, h, p.G, r0, int(rows));
  float* buffer0 = sTokens + (begin % kBuf) * S::kTokens;
  if (begin < steps) fill_tokens<T, DK, DV, kKeysQ>(p.k, p.v, buffer0, buffer0 + kKeysQ * (DK + 4), b, h, begin * kKeysQ, run);
  fill_commit();
  float nl[4], d[4], dq[4][DK / 16];
  int pos[4];
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    const int r = r0 + 4 * ty + a;
    const bool in = r < rows;
    nl[a] = in ? p.nl[bh * rows + r] : -INFINITY;
    d[a] = in ? p.delta[bh * rows + r] : 0.f;
    pos[a] = in ? int(r / p.G) + off : -1;   // sees nothing
#pragma unroll
    for (int c = 0; c < DK / 16; ++c) dq[a][c] = 0.f;
  }
  // positions of the warp's rows
  const int wr = r0 + 8 * (threadIdx.x >> 5), wz = r0 + live < wr + 8 ? r0 + live : wr + 8;
  const int warp_first = wr / p.G + off, warp_last = wz > wr ? (wz - 1) / p.G + off : -1;
  for (int t = begin; t < steps; ++t) {
    const float* sK = sTokens + (t % kBuf) * S::kTokens;
    const float* sV = sK + kKeysQ * (DK + 4);
    float* next = sTokens + ((t + 1) % kBuf) * S::kTokens;
    if (kBuf == 2 && t + 1 < steps)
      fill_tokens<T, DK, DV, kKeysQ>(p.k, p.v, next, next + kKeysQ * (DK + 4), b, h, (t + 1) * kKeysQ, run);
    fill_commit();
    fill_wait<kBuf - 1>();
    __syncthreads();
    // A warp whose eight rows see no token of the step has nothing to add.
    const int x1 = (t + 1) * kKeysQ < run.n ? (t + 1) * kKeysQ - 1 : run.n - 1;
    const int first = run.at(t * kKeysQ), last = run.at(x1);   // tokens
    if (first <= warp_last && (warp_first - last < p.mask.window || first < p.mask.sinks)) {
      // tokens tx, tx + 16 against rows 4 ty + a
      Sum2 s2[4][2], e2[4][2];
#pragma unroll
      for (int a = 0; a < 4; ++a) s2[a][0] = s2[a][1] = e2[a][0] = e2[a][1] = Sum2{0.f, 0.f};
#pragma unroll 4
      for (int c = 0; c < DK; c += 4) {
        const float4 k0 = *reinterpret_cast<const float4*>(sK + tx * (DK + 4) + c);
        const float4 k1 = *reinterpret_cast<const float4*>(sK + (tx + 16) * (DK + 4) + c);
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const float4 q = *reinterpret_cast<const float4*>(sQ + (4 * ty + a) * (DK + 4) + c);
          dot4(q, k0, s2[a][0]);
          dot4(q, k1, s2[a][1]);
        }
      }
#pragma unroll 4
      for (int c = 0; c < DV; c += 4) {
        const float4 v0 = *reinterpret_cast<const float4*>(sV + tx * (DV + 4) + c);
        const float4 v1 = *reinterpret_cast<const float4*>(sV + (tx + 16) * (DV + 4) + c);
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const float4 g = *reinterpret_cast<const float4*>(sG + (4 * ty + a) * (DV + 4) + c);
          dot4(g, v0, e2[a][0]);
          dot4(g, v1, e2[a][1]);
        }
      }
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int at = t * kKeysQ + tx + 16 * x, j = at < run.n ? run.at(at) : 0x7fffffff;
        float4 ws;
        float* fs = reinterpret_cast<float*>(&ws);
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const bool seen = j <= pos[a] && (pos[a] - j < p.mask.window || j < p.mask.sinks);
          fs[a] = seen ? exp2f(fmaf(s2[a][x].all(), p.c_log2, nl[a])) * (e2[a][x].all() - d[a]) : 0.f;
        }
        *reinterpret_cast<float4*>(sS + (tx + 16 * x) * kLdW + 4 * ty) = ws;
      }
      __syncwarp();
#pragma unroll 4
      for (int j = 0; j < kKeysQ; ++j) {
        const float4 ws = *reinterpret_cast<const float4*>(sS + j * kLdW + 4 * ty);
#pragma unroll
        for (int c = 0; c < DK / 64; ++c) {
          const float4 k = *reinterpret_cast<const float4*>(sK + j * (DK + 4) + 64 * c + 4 * tx);
          axpy4(ws.x, k, dq[0] + 4 * c);
          axpy4(ws.y, k, dq[1] + 4 * c);
          axpy4(ws.z, k, dq[2] + 4 * c);
          axpy4(ws.w, k, dq[3] + 4 * c);
        }
      }
    }
    __syncthreads();   // this step's tokens make room for others
    if (kBuf == 1 && t + 1 < steps)
      fill_tokens<T, DK, DV, kKeysQ>(p.k, p.v, next, next + kKeysQ * (DK + 4), b, h, (t + 1) * kKeysQ, run);
  }
  fill_wait<0>();
#pragma unroll
  for (int a = 0; a < 4; ++a) {
    const int r = r0 + 4 * ty + a;
    if (r >= rows) continue;
    if (p.q_pieces > 1) {
      float* dst = p.part_q + (((int64_t(bh) * p.n_rt + rt) * p.q_pieces + piece) * kRowsQ + 4 * ty + a) * DK;
#pragma unroll
      for (int c = 0; c < DK / 64; ++c)
        store4(dst + 64 * c + 4 * tx, make_float4(dq[a][4 * c], dq[a][4 * c + 1], dq[a][4 * c + 2], dq[a][4 * c + 3]));
      continue;
    }
    const int i = r / p.G;
    const int64_t hq = int64_t(h) * p.G + (r - i * p.G);
    T* dst = const_cast<T*>(row_of<T>(p.dq, b, hq, i));
#pragma unroll
    for (int c = 0; c < DK / 64; ++c)
      store4(dst + 64 * c + 4 * tx, make_float4(dq[a][4 * c] * p.scale, dq[a][4 * c + 1] * p.scale, dq[a][4 * c + 2] * p.scale,
                                                dq[a][4 * c + 3] * p.scale));
  }
  return odd_sums(dq);
}

// Adds the pieces of dQ's tiles: four features of a row a thread.
template <typename T, int DK>
__global__ void __launch_bounds__(kThreads)
window_dq_join_kernel(const Params p, int64_t n) {
  wait_for_previous();
  const int64_t x = int64_t(blockIdx.x) * kThreads + threadIdx.x;
  if (x >= n) return;
  const int64_t row = x / (DK / 4), tile = row / kRowsQ, bh = tile / p.n_rt;   // row: (tile, row of the tile)
  const int c = int(x - row * (DK / 4)) * 4;
  const int64_t r = (tile - bh * p.n_rt) * kRowsQ + (row - tile * kRowsQ);
  if (r >= int64_t(p.N) * p.G) return;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i = 0; i < p.q_pieces; ++i) {
    const float4 v = load4(p.part_q + ((tile * p.q_pieces + i) * kRowsQ + (row - tile * kRowsQ)) * DK + c);
    s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
  }
  const int64_t b = bh / p.Hk, h = bh - b * p.Hk, i = r / p.G;
  store4(const_cast<T*>(row_of<T>(p.dq, b, h * p.G + (r - i * p.G), i)) + c,
         make_float4(s.x * p.scale, s.y * p.scale, s.z * p.scale, s.w * p.scale));
}

// CTAs below n_q: dQ; the others, whose pieces are shorter: dK and dV.
template <typename T, int DK, int DV>
__global__ void __launch_bounds__(kThreads, 2)
window_bwd_cc_kernel(const Params p, unsigned n_q) {
  extern __shared__ float smem[];
  wait_for_previous();
  const uint32_t odd = blockIdx.x < n_q ? dq_tile<T, DK, DV>(p, blockIdx.x, smem) : dkdv_tile<T, DK, DV>(p, blockIdx.x - n_q, smem);
  if (threadIdx.x % 32 == 0) p.odd[blockIdx.x * (kThreads / 32) + threadIdx.x / 32] = odd;
}

// The marked sums of all CTAs' warps, of which there are n, once more: neighbours by different warps.
template <typename T, int DK, int DV>
__global__ void __launch_bounds__(kThreads)
window_again_kernel(const Params p, unsigned n, unsigned n_q) {
  wait_for_previous();
  const unsigned lane = threadIdx.x % 32, warps = gridDim.x * (kThreads / 32), mine = blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
  for (unsigned base = mine; base < n; base += 32 * warps) {
    const uint64_t at = base + uint64_t(lane) * warps;
    const uint32_t odd = at < n ? p.odd[at] : 0u;
    uint32_t marked = __ballot_sync(0xffffffffu, odd != 0);
    while (marked != 0) {
      const int from = __ffs(marked) - 1;
      marked &= marked - 1;
      const uint32_t bad = __shfl_sync(0xffffffffu, odd, from);
      const unsigned which = base + unsigned(from) * warps, cta = which / (kThreads / 32);
      const int warp = int(which % (kThreads / 32));
      if (cta < n_q) {
        rows_again<T, DK, DV>(p, cta, warp, bad);
      } else {
        if ((bad & 0xffu) != 0) tokens_again<T, DK, DV, true>(p, cta - n_q, warp, bad & 0xffu);
        if (bad >> 8 != 0) tokens_again<T, DK, DV, false>(p, cta - n_q, warp, bad >> 8);
      }
    }
  }
}

// How token tiles are cut: pieces of a window's rows (of all rows without one), or of so few that there are two CTAs
// for each SM; the first `cut` tiles then come in up to `pieces` pieces.
struct Cut {
  int64_t n_kt, cut, pieces, piece_rows;
  int64_t q_tiles, q_pieces;   // dQ's tiles, and pieces of each one's tokens where there are few
};
Cut cut_of(const WindowBwdArgs& a) {
  const int64_t G = a.Hq / a.Hk, bh = a.B * a.Hk, rows = a.Nq * G;
  Cut c;
  c.n_kt = (a.Nk + kKeysKv - 1) / kKeysKv;
  const bool windowed = a.window != win::kNoWindow;
  int64_t usual = windowed ? (int64_t(a.window) + kKeysKv) * G : rows;
  if (usual > rows) usual = rows;
  int64_t want = usual;
  c.cut = windowed ? (int64_t(a.sinks) + kKeysKv - 1) / kKeysKv : 0;
  if (c.n_kt * bh < kMostPieces / 4) {
    // about the rows of all tiles: half of them without a window
    const int64_t all = bh * c.n_kt * (windowed ? usual : (usual + 1) / 2);
    const int64_t fine = all / (kMostPieces / 4);
    if (fine < usual) {
      want = fine;
      c.cut = c.n_kt;
    }
  }
  if (want < 3 * kRowsKv) want = 3 * kRowsKv;   // (2, 3, 4, 6 steps: 64, 61, 63, 75 us of the case above)
  c.piece_rows = (want + kRowsKv - 1) / kRowsKv * kRowsKv;
  if (c.cut > c.n_kt) c.cut = c.n_kt;
  // not more pieces than keep the machine busy: each is 64 rows of fp32 in the workspace (80 MB in all)
  const int64_t most = c.cut > 0 && bh * c.cut < kMostPieces ? kMostPieces / (bh * c.cut) : 1;
  if ((rows + c.piece_rows - 1) / c.piece_rows > most) c.piece_rows = ((rows + most - 1) / most + kRowsKv - 1) / kRowsKv * kRowsKv;
  c.pieces = (rows + c.piece_rows - 1) / c.piece_rows;
  if (c.pieces == 1) c.cut = 0;
  c.q_tiles = bh * ((rows + kRowsQ - 1) / kRowsQ);
  int64_t tokens = windowed ? int64_t(a.window) + kRowsQ / G + a.sinks : a.Nk;
  if (tokens > a.Nk) tokens = a.Nk;
  c.q_pieces = c.q_tiles < kMostPieces / 8 ? (kMostPieces / 4 + c.q_tiles - 1) / c.q_tiles : 1;
  // (pieces of eight steps at least: with two of three, the case above takes 71 us instead of 61)
  if (c.q_pieces > tokens / (8 * kKeysQ)) c.q_pieces = tokens / (8 * kKeysQ);
  if (c.q_pieces < 1) c.q_pieces = 1;
  return c;
}

// The workspace: -LSE log2 e and D of every row, the pieces, and the marks of sums that are not finite.
int64_t rows_bytes(const WindowBwdArgs& a) { return (a.B * a.Hq * a.Nq * 4 + 255) / 256 * 256; }

template <typename T, int DK, int DV>
int launch(const WindowBwdArgs& a, char* msg, size_t msglen) {
  const Cut cut = cut_of(a);
  const int64_t bh = a.B * a.Hk, G = a.Hq / a.Hk, rows = a.B * a.Hq * a.Nq;
  uint8_t* ws = static_cast<uint8_t*>(a.ws);
  Params p{};
  p.q = a.q, p.k = a.k, p.v = a.v, p.o = a.o, p.go = a.go, p.dq = a.dq, p.dk = a.dk_, p.dv = a.dv_;
  p.lse = a.lse;
  p.nl = reinterpret_cast<float*>(ws);
  p.delta = reinterpret_cast<float*>(ws + rows_bytes(a));
  p.part = reinterpret_cast<float*>(ws + 2 * rows_bytes(a));
  p.part_q = p.part + bh * cut.cut * cut.pieces * kKeysKv * (DK + DV);
  const int64_t items = bh * (cut.cut * cut.pieces + cut.n_kt - cut.cut), ctas = items + cut.q_tiles * cut.q_pieces;
  p.odd = reinterpret_cast<uint32_t*>(p.part_q + (cut.q_pieces > 1 ? cut.q_tiles * cut.q_pieces * kRowsQ * DK : 0));
  p.q_pieces = int(cut.q_pieces);
  p.Hk = int(a.Hk), p.N = int(a.Nq), p.G = int(G), p.Nk = int(a.Nk);
  p.mask = win::Mask{a.window, a.sinks, true};
  p.c_log2 = a.scale * kLog2e, p.scale = a.scale;
  p.n_kt = int(cut.n_kt), p.cut = int(cut.cut), p.pieces = int(cut.pieces), p.piece_rows = cut.piece_rows;
  p.n_rt = int((a.Nq * G + kRowsQ - 1) / kRowsQ);
  constexpr int kSmem = (KvSmem<DK, DV>::kFloats > QSmem<DK, DV>::kFloats ? KvSmem<DK, DV>::kFloats : QSmem<DK, DV>::kFloats) * 4;
  static_assert(kSmem <= 232448, "shared memory budget");
  auto kern = window_bwd_cc_kernel<T, DK, DV>;
  cudaError_t e = ensure_smem_limit(reinterpret_cast<const void*>(kern), kSmem);
  if (e == cudaSuccess)
    e = launch_overlapped(window_delta_kernel<T, DV>, dim3(unsigned((rows + 7) / 8)), dim3(kThreads), 0, a.stream, p, rows);
  if (e == cudaSuccess)
    e = launch_overlapped(kern, dim3(unsigned(ctas)), dim3(kThreads), size_t(kSmem), a.stream, p,
                          unsigned(cut.q_tiles * cut.q_pieces));
  const int64_t marks = ctas * (kThreads / 32), again = (marks + kThreads - 1) / kThreads;
  if (e == cudaSuccess)
    e = launch_overlapped(window_again_kernel<T, DK, DV>, dim3(unsigned(again < kMostAgain ? again : kMostAgain)), dim3(kThreads), 0,
                          a.stream, p, unsigned(marks), unsigned(cut.q_tiles * cut.q_pieces));
  const int64_t joined = bh * cut.cut * kKeysKv * ((DK + DV) / 4);
  if (e == cudaSuccess && joined > 0)
    e = launch_overlapped(window_dkdv_join_kernel<T, DK, DV>, dim3(unsigned((joined + kThreads - 1) / kThreads)), dim3(kThreads),
                          0, a.stream, p, joined);
  const int64_t q_joined = cut.q_tiles * kRowsQ * (DK / 4);
  if (e == cudaSuccess && cut.q_pieces > 1)
    e = launch_overlapped(window_dq_join_kernel<T, DK>, dim3(unsigned((q_joined + kThreads - 1) / kThreads)), dim3(kThreads), 0,
                          a.stream, p, q_joined);
  if (e != cudaSuccess) {
    snprintf(msg, msglen, "gradients of attention with a window: %s", cudaGetErrorString(e));
    return 5;
  }
  return 0;
}

template <typename T>
int launch_sizes(const WindowBwdArgs& a, char* msg, size_t msglen) {
  if (a.dk == 64) return a.dv == 64 ? launch<T, 64, 64>(a, msg, msglen) : launch<T, 64, 128>(a, msg, msglen);
  return a.dv == 64 ? launch<T, 128, 64>(a, msg, msglen) : launch<T, 128, 128>(a, msg, msglen);
}

}  // namespace

size_t window_bwd_cc_workspace(const WindowBwdArgs& a) {
  const Cut c = cut_of(a);
  const int64_t ctas = a.B * a.Hk * (c.cut * c.pieces + c.n_kt - c.cut) + c.q_tiles * c.q_pieces;
  return size_t(2 * rows_bytes(a) + a.B * a.Hk * c.cut * c.pieces * kKeysKv * (a.dk + a.dv) * 4 +
                (c.q_pieces > 1 ? c.q_tiles * c.q_pieces * kRowsQ * a.dk * 4 : 0) + ctas * (kThreads / 32) * 4);
}

int launch_window_bwd_cc(const WindowBwdArgs& a, char* msg, size_t msglen) {
  return a.f32 ? launch_sizes<float>(a, msg, msglen) : launch_sizes<__nv_bfloat16>(a, msg, msglen);
}

}  // namespace moa
