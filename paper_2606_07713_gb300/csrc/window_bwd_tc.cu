// Gradients of causal attention with a sliding window and first tokens that stay visible, bf16, on the
// fifth-generation tensor cores (tcgen05 + TMEM + TMA), sm_103a.
//
// Mathematics, with P_ij = 2^(c s_ij - LSE_i log2 e) for the tokens j that row i sees (window.cuh), 0 for the
// others, c = scale log2 e, and D_i = <dO_i, O_i>:
//     dV_j = sum_i P_ij dO_i,   dS_ij = P_ij (<dO_i, v_j> - D_i),
//     dQ_i = scale sum_j dS_ij k_j,   dK_j = scale sum_i dS_ij q_i,
// the sums over i also over the query heads that share the key head.  P and dS are rounded to bf16 (operands of the
// products), all sums are fp32 in TMEM.
//
//   delta  D and -LSE log2 e of every row, in tiles of 128 rows;
//   tiles  one launch, two kinds of CTAs.  dK and dV: 128 tokens of a key head and a piece of the row tiles that see them,
//            S^T = K Q^T, dP^T = V dO^T, P^T and dS^T back into TMEM as bf16, dV += P^T dO, dK += dS^T Q;
//          dQ: 128 rows, over the token tiles that they see,
//            S = Q K^T, dP = dO V^T, dS = P (dP - D), dQ += dS K;
//   join   adds the pieces of cut tiles, in order.
// dQ apart from dK and dV: seven tile products in place of five, but every sum stays within one CTA (no
// atomics, the same bits every time).
//
// Rows of a key head are counted position by position as in the forward kernel, here in halves of 64: row r of a half is
// position r / GC, query head r % GC of the group (TMA brings them in that order), so that a window's tiles hold few rows
// that are hidden; for a token the rows that see it are one range of a half's columns, for a row the tokens two ranges.
//
// Score tiles are 128 x 128 (M x N).  With d_k = d_v = 64 the products are short, and a tile's chain of product,
// exponentials, product, dS, product is what takes the time (213 us of 4 x 16 heads x 2048 x 64, causal): there N is 64, a CTA takes half of an SM's
// tensor and shared memory, and the chains of two CTAs an SM overlap (184 us).
//
// Pieces.  A token's rows are those of a window; a sink's are all later ones, which one CTA would walk over while the
// others are done: token tiles with more row tiles than `piece` are cut.  `piece` is a window's row tiles, or less
// where there are too few CTAs for the machine.  With few rows and many tokens dQ's tiles have their tokens cut alike.
//
// What bounds it: the same chain; 2 x (32 / 8) heads x 8192 x 128, window 1024: 993 us = 0.65 PFLOP/s of what the five products need,
// tensor pipe 49 %, no other unit half busy.  (16 compute warps: 1026 us in place of 996 at the time; score tiles of 64 columns in two
// buffers: 1364 in place of 1000.)
//
// What is not finite.  Hidden pairs have the weight zero, and zero times what is not finite reaches every output of a product.  So
// a tile with an output that is not finite is computed once more by its CTA at the end, unless nothing that is not finite is hidden from a
// part of it: step after step without overlap, hidden dS set to zero, what is not finite taken out of the operand in steps that are seen
// in part, and added at the end where it is seen.  (dq_again, dkdv_again.  That takes some five times as long; other calls pay nothing.)
//
// CTA organisation of both kinds: 8 compute warps (warp w: TMEM lanes 32 (w % 4) .., columns N / 2 (w / 4) .. of the score
// tiles; its bf16 values go back into the first half of its own columns), one warp for TMEM and the products, one for the
// copies.  Waits are bounded; on expiry MOA_ERR_DEVICE_TIMEOUT is recorded and
// every role leaves its loop.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdio>

#include "internal.h"
#include "ops_internal.h"
#include "ptx.cuh"
#include "tc_common.cuh"
#include "window.cuh"
#include "window_tc.cuh"

namespace moa {

__device__ unsigned int g_moa_window_bwd_status = 0;

namespace {

using namespace ptx;
using namespace tc;
using win::below, win::describable, win::map_stride, win::tma_load_4d, win::tma_load_5d;

constexpr int kBlk = 128;                // tokens of dK's and dV's tiles, rows of dQ's
constexpr int kHalf = 64;                // rows of half a row tile
constexpr int kPanelBytes = 128 * 128;   // 64 bf16 columns of 128 rows, 128-byte swizzle
constexpr float kLog2e = 1.4426950408889634f;

struct Params {
  View q, k, v, o, go, dq, dk, dv;
  const float* lse;
  float* nl;      // [half][64] -LSE log2 e; -infinity for rows that are not there or see nothing
  float* delta;   // alike: D
  float* part;    // [cut tile][piece][128][DK + DV]
  float* part_q;  // [pair of halves][piece][128][DK], if dQ's tiles come in pieces
  int B, Hk, G, N, Nk;
  int GC, chunks, PT;   // heads of a half, chunks of heads, positions of a half
  int n_ht;             // halves along the positions, an even number
  int n_kt;             // token tiles
  int cut, pieces, piece;   // the first `cut` token tiles come in up to `pieces` pieces of `piece` row tiles (of N rows)
  int q_pieces;         // pieces of a dQ tile's tokens
  int group;            // key heads whose token tiles are handed out in turn, longest first
  win::Mask mask;
  float c_log2, scale;
  uint64_t wait_limit_ns;
};

constexpr int kParts = 2, kComputeThreads = 256, kThreads = 320, kMmaWarp = 8, kLoadWarp = 9;
// Columns of the score tiles, CTAs of an SM, the ring's stages.
__host__ __device__ constexpr int width_of(int dk, int dv) { return dk + dv <= 128 ? 64 : 128; }
__host__ __device__ constexpr int ctas_of(int dk, int dv) { return dk + dv <= 128 ? 2 : 1; }
__host__ __device__ constexpr int ring_stages(int dk, int dv) { return dk + dv <= 128 ? 4 : (dk + dv <= 192 ? 3 : 2); }

// TMEM column of step kk (16 rows of the reduction axis) of a bf16 operand that the column parts wrote.
template <int COLS>
__device__ __forceinline__ uint32_t part_col(int kk) {
  return uint32_t((kk * 16 / COLS) * COLS + (kk * 16 % COLS) / 2);
}
template <int COLS>
__device__ __forceinline__ void tmem_load_part(uint32_t taddr, uint32_t* r) {
#pragma unroll
  for (int c = 0; c < COLS; c += 32) tmem_ld_32x32b_x32(taddr + c, r + c);
  tmem_wait_ld();
#pragma unroll
  for (int c = 0; c < COLS; c += 32) reg_anchor_x32(r + c);
}
// The same in steps of 32 columns: while one is worked on, the next is on its way.
template <int COLS, typename F>
__device__ __forceinline__ void tmem_each_32(uint32_t taddr, uint32_t* r, F&& work) {
  tmem_ld_32x32b_x32(taddr, r);
#pragma unroll
  for (int c = 0; c < COLS; c += 32) {
    tmem_wait_ld();
    reg_anchor_x32(r + c);
    if (c + 32 < COLS) tmem_ld_32x32b_x32(taddr + c + 32, r + c + 32);
    work(c);
  }
}
template <int COLS>
__device__ __forceinline__ void tmem_store_part(uint32_t taddr, const uint32_t* pk) {
  if constexpr (COLS == 64)
    tmem_st_32x32b_x32(taddr, pk);
  else
    tmem_st_32x32b_x16(taddr, pk);
}
__device__ __forceinline__ float4 lds_f32x4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
// NCOLS fp32 TMEM columns of this thread's lane, times mul: as bf16 to dst, or as they are to part.  Whether all are finite.
template <int NCOLS, bool ROLLED = false>
__device__ __forceinline__ bool store_row(uint32_t taddr, float mul, __nv_bfloat16* dst, float* part, bool valid) {
  constexpr int kUnroll = ROLLED ? 1 : NCOLS / 32;
  float odd[4] = {0.f, 0.f, 0.f, 0.f};   // x * 0 + odd is NaN from the first x on that is not finite
  const uint64_t none = pack_f32x2(0.f, 0.f);
#pragma unroll(kUnroll)
  for (int c = 0; c < NCOLS; c += 32) {
    uint32_t o[32];
    tmem_ld_32x32b_x32(taddr + c, o);
    tmem_wait_ld();
    reg_anchor_x32(o);
    if (!valid) continue;
#pragma unroll
    for (int i = 0; i < 32; i += 2)
      ffma2(odd[i & 2], odd[(i & 2) + 1], __uint_as_float(o[i]), __uint_as_float(o[i + 1]), none, pack_f32x2(odd[i & 2], odd[(i & 2) + 1]));
    if (part != nullptr) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        reinterpret_cast<float4*>(part + c)[i] = make_float4(__uint_as_float(o[4 * i]), __uint_as_float(o[4 * i + 1]),
                                                             __uint_as_float(o[4 * i + 2]), __uint_as_float(o[4 * i + 3]));
    } else {
      uint32_t w[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) w[i] = pack_bf16x2(__uint_as_float(o[2 * i]) * mul, __uint_as_float(o[2 * i + 1]) * mul);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        reinterpret_cast<uint4*>(dst + c)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    }
  }
  return (odd[0] + odd[1]) + (odd[2] + odd[3]) == 0.f;
}

// ------------------------------------------------------------------------------------------------
// What dkdv_again and dq_again share
// ------------------------------------------------------------------------------------------------
__device__ __forceinline__ bool odd_word(uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; }
template <int D>
__device__ __forceinline__ bool odd_row(const __nv_bfloat16* x) {
  bool odd = false;
#pragma unroll 4
  for (int c = 0; c < D; c += 8) {
    const uint4 w = *reinterpret_cast<const uint4*>(x + c);
    odd |= odd_word(w.x) || odd_word(w.y) || odd_word(w.z) || odd_word(w.w);
  }
  return odd;
}
// All compute threads; whether all of them say so.
__device__ __forceinline__ bool meet(bool yes) {
  uint32_t all;
  asm volatile("{\n\t.reg .pred a, b;\n\tsetp.ne.u32 a, %1, 0;\n\tbar.red.and.pred b, 1, %2, a;\n\tselp.u32 %0, 1, 0, b;\n\t}"
               : "=r"(all)
               : "r"(uint32_t(yes)), "n"(256)
               : "memory");
  return all != 0;
}
// Sets what is not finite in `rows` rows of D columns in shared memory, 64 a panel, to zero (all compute threads).
template <int D>
__device__ __forceinline__ void take_out(uint8_t* tile, int rows, int panel) {
#pragma unroll 1
  for (int x = threadIdx.x; x < rows * (D / 64); x += 256) {
    const int q = x / rows, r = x - q * rows;
#pragma unroll 2
    for (int e = 0; e < 8; ++e) {   // eight lanes in eight banks
      uint4* at = reinterpret_cast<uint4*>(tile + q * panel + r * 128 + ((e ^ r) & 7) * 16);
      const uint4 v = *at;
      if (!(odd_word(v.x) || odd_word(v.y) || odd_word(v.z) || odd_word(v.w))) continue;
      uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if ((w[i] & 0x7f80u) == 0x7f80u) w[i] &= 0xffff0000u;
        if ((w[i] & 0x7f800000u) == 0x7f800000u) w[i] &= 0xffffu;
      }
      *at = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}
// Whether some of a warp's 32 sums each, of outputs that are there, are numbers.
__device__ __forceinline__ bool any_number(const uint32_t (&o)[32], bool there) {
  bool any = false;
#pragma unroll
  for (int e = 0; e < 32; ++e) any |= __uint_as_float(o[e]) == __uint_as_float(o[e]);
  return __any_sync(0xffffffffu, any && there);
}
// Adds to 32 sums the members of the rows `odd` (a lane each, its row at x) that are not finite, where sees(lane) says that the
// thread's output sees the row; NAN_ONLY: as NaN, whatever they are.
template <bool NAN_ONLY, typename Sees>
__device__ __forceinline__ void add_odd(uint32_t (&o)[32], uint32_t odd, const __nv_bfloat16* x, Sees&& sees) {
  while (odd != 0) {
    const int b = __ffs(odd) - 1;
    odd &= odd - 1;
    const __nv_bfloat16* row =
        reinterpret_cast<const __nv_bfloat16*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(x), b));
    if (!sees(b)) continue;
#pragma unroll
    for (int e = 0; e < 32; ++e) {
      const float y = __bfloat162float(row[e]);
      if (!(fabsf(y) < INFINITY)) o[e] = __float_as_uint(__uint_as_float(o[e]) + (NAN_ONLY ? __int_as_float(0x7fffffff) : y));
    }
  }
}
__device__ __forceinline__ bool sees(const win::Mask& m, int pos, int j) { return j <= pos && (pos - j < m.window || j < m.sinks); }

__device__ __forceinline__ __nv_bfloat16* row_of(const View& x, int b, int h, int n) {
  return static_cast<__nv_bfloat16*>(x.p) + b * x.sb + h * x.sh + n * x.sn;
}

// Pair of halves t: its key head, chunk of heads and first position.
struct RowTile {
  int b, h, chunk, i0;
};
__device__ __forceinline__ RowTile row_tile(const Params& p, int64_t t) {
  RowTile r;
  const int64_t per = int64_t(p.chunks) * (p.n_ht / 2), bh = t / per;
  const int rest = int(t - bh * per);
  r.chunk = rest / (p.n_ht / 2);
  r.i0 = (rest - r.chunk * (p.n_ht / 2)) * 2 * p.PT;
  r.b = int(bh / p.Hk), r.h = int(bh - int64_t(r.b) * p.Hk);
  return r;
}
// Row r of a pair of halves: its head of the group and position, and whether it is there.
struct RowAt {
  int g, i;
  bool real;
};
__device__ __forceinline__ RowAt row_at(const Params& p, const RowTile& t, int r) {
  const int in_half = r % kHalf, pos = int(unsigned(in_half) / unsigned(p.GC));
  RowAt a;
  a.g = t.chunk * p.GC + (in_half - pos * p.GC);
  a.i = t.i0 + r / kHalf * p.PT + pos;
  a.real = pos < p.PT && a.g < p.G && a.i < p.N;
  return a;
}

// ------------------------------------------------------------------------------------------------
// D and -LSE log2 e: DV / 8 lanes a row
// ------------------------------------------------------------------------------------------------
// A CTA for two halves; its rows' loads are all on their way together.  Bound by memory: O and dO once.
template <int DV>
__global__ void __launch_bounds__(256)
window_delta_tc_kernel(const Params p) {
  constexpr int L = DV / 8, kStep = 256 / L, kIts = kBlk / kStep;
  wait_for_previous();
  const RowTile t = row_tile(p, blockIdx.x);
  const int gl = threadIdx.x % L, first = threadIdx.x / L;
  // four rows a thread on their way at a time (eight leave room for two CTAs an SM)
  constexpr int kBatch = kIts < 4 ? kIts : 4;
#pragma unroll 1
  for (int k0 = 0; k0 < kIts; k0 += kBatch) {
    uint4 ov[kBatch], gv[kBatch];
    float lse[kBatch];
    bool real[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const RowAt at = row_at(p, t, first + (k0 + k) * kStep);
      const int hq = t.h * p.G + at.g, i = at.i;
      real[k] = at.real;
      ov[k] = gv[k] = make_uint4(0, 0, 0, 0);
      lse[k] = -INFINITY;
      if (real[k]) {
        ov[k] = *reinterpret_cast<const uint4*>(row_of(p.o, t.b, hq, i) + gl * 8);
        gv[k] = *reinterpret_cast<const uint4*>(row_of(p.go, t.b, hq, i) + gl * 8);
        if (gl == 0) lse[k] = p.lse[(int64_t(t.b) * p.Hk * p.G + hq) * p.N + i];
      }
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const __nv_bfloat162* o2 = reinterpret_cast<const __nv_bfloat162*>(&ov[k]);
      const __nv_bfloat162* g2 = reinterpret_cast<const __nv_bfloat162*>(&gv[k]);
      float acc = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 of = __bfloat1622float2(o2[e]), gf = __bfloat1622float2(g2[e]);
        acc = fmaf(of.x, gf.x, acc);
        acc = fmaf(of.y, gf.y, acc);
      }
#pragma unroll
      for (int d = L / 2; d > 0; d >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, d);
      if (gl == 0) {
        const int64_t r = int64_t(blockIdx.x) * kBlk + first + (k0 + k) * kStep;
        p.nl[r] = lse[k] == -INFINITY ? -INFINITY : -lse[k] * kLog2e;
        p.delta[r] = acc;
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------
// dK and dV
// ------------------------------------------------------------------------------------------------
// The row tiles (of `positions` positions) that see a token of tile kt: [first, first + n) along the positions.
struct Range {
  int first, n;
};
__host__ __device__ __forceinline__ Range rows_of_tokens(const win::Mask& m, int kt, int N, int Nk, int positions) {
  const int off = Nk - N, k0 = kt * kBlk, k1 = k0 + kBlk < Nk ? k0 + kBlk : Nk;
  const int64_t i0 = k0 > off ? int64_t(k0) - off : 0;
  int64_t i1 = N;
  if (k0 >= m.sinks && m.window != win::kNoWindow) {
    const int64_t n = int64_t(k1) - 1 + m.window - off;
    i1 = n < 0 ? 0 : n < i1 ? n : i1;
  }
  Range r;
  r.first = int(i0 / positions);
  r.n = i1 > i0 ? int((i1 + positions - 1) / positions) - r.first : 0;
  return r;
}

template <int DK, int DV>
struct KvCfg {
  static constexpr int kN = width_of(DK, DV), kCols = kN / kParts, kHalves = kN / kHalf;
  static constexpr int kKBytes = kBlk * DK * 2, kVBytes = kBlk * DV * 2;
  static constexpr int kRowPanel = kN * 128;   // 64 columns of a row tile
  static constexpr int kQBytes = kN * DK * 2, kGBytes = kN * DV * 2, kVecBytes = kN * 4;
  // stage: Q tile, dO tile, -L and D of its rows
  static constexpr int kStageBytes = (kQBytes + kGBytes + 2 * kVecBytes + 1023) / 1024 * 1024;
  static constexpr int kStages = ring_stages(DK, DV);
  static constexpr int kOffK = 0, kOffV = kKBytes, kOffStage = kKBytes + kVBytes;
  // barriers: full[NS], empty[NS], kv_full, s_full, dp_full, p_ready, ds_ready, acc_done, again_loaded, again_done
  static constexpr int kNumBars = 2 * kStages + 8;
  static constexpr int kOffBar = kOffStage + kStages * kStageBytes;
  static constexpr int kOffMisc = kOffBar + kNumBars * 8;
  static constexpr int kSmemBytes = kOffMisc + 16 + 1024;
  static constexpr uint32_t kTmemS = 0, kTmemDP = kN, kTmemDV = 2 * kN, kTmemDK = 2 * kN + DV;
  static constexpr uint32_t kTmemCols = 512 / ctas_of(DK, DV);
  static_assert(kTmemDK + DK <= kTmemCols, "TMEM budget");
  static_assert((kSmemBytes + 1024) * ctas_of(DK, DV) <= 233472, "shared memory budget");
};

// A CTA's work: token tile kt of a key head, row tiles [t0, t0 + n) of the list (chunk after chunk).
struct KvItem {
  int b, h, kt, piece;
  bool whole;   // not cut: the result is written, not a piece of it
};
__host__ __device__ __forceinline__ KvItem kv_item(const Params& p, int64_t x) {
  // groups of key heads; within one, token tile after token tile (the first have the most rows), head after head
  const int per = p.cut * p.pieces + p.n_kt - p.cut;   // items of a key head
  const int64_t heads = int64_t(p.B) * p.Hk, first = x / (int64_t(per) * p.group) * p.group;
  const int64_t g = heads - first < p.group ? heads - first : p.group;
  const int64_t rest = x - first * per, item = rest / g, bh = first + (rest - item * g);
  KvItem k;
  k.b = int(bh / p.Hk), k.h = int(bh - int64_t(k.b) * p.Hk);
  const int64_t n_cut = int64_t(p.cut) * p.pieces;
  k.whole = item >= n_cut;
  k.kt = k.whole ? int(item - n_cut) + p.cut : int(item / p.pieces);
  k.piece = k.whole ? 0 : int(item - int64_t(k.kt) * p.pieces);
  return k;
}

// The products of a step: S^T = K Q^T (M = 128 tokens, N rows, both operands K-major), dP^T = V dO^T,
// dV += P^T dO and dK += dS^T Q (A from TMEM, B MN-major).
template <int DK, int DV>
__device__ __forceinline__ void issue_scores(uint32_t tS, uint32_t sK, uint32_t sQ) {
  using C = KvCfg<DK, DV>;
  constexpr uint32_t kIdesc = make_idesc(kBlk, C::kN, false);
#pragma unroll
  for (int kk = 0; kk < DK / 16; ++kk) {
    const uint32_t k = (kk >> 2) * kPanelBytes + (kk & 3) * 32, r = (kk >> 2) * C::kRowPanel + (kk & 3) * 32;
    mma_f16_ss(tS, make_sdesc_sw128(sK + k, 16, 1024), make_sdesc_sw128(sQ + r, 16, 1024), kIdesc, kk > 0 ? 1u : 0u);
  }
}
template <int DK, int DV>
__device__ __forceinline__ void issue_changes(uint32_t tDP, uint32_t sV, uint32_t sG) {
  using C = KvCfg<DK, DV>;
  constexpr uint32_t kIdesc = make_idesc(kBlk, C::kN, false);
#pragma unroll
  for (int kk = 0; kk < DV / 16; ++kk) {
    const uint32_t k = (kk >> 2) * kPanelBytes + (kk & 3) * 32, r = (kk >> 2) * C::kRowPanel + (kk & 3) * 32;
    mma_f16_ss(tDP, make_sdesc_sw128(sV + k, 16, 1024), make_sdesc_sw128(sG + r, 16, 1024), kIdesc, kk > 0 ? 1u : 0u);
  }
}
template <int DK, int DV>
__device__ __forceinline__ void issue_dv(uint32_t tDV, uint32_t tS, uint32_t sG, bool more) {
  using C = KvCfg<DK, DV>;
  constexpr uint32_t kIdesc = make_idesc(kBlk, DV, true);
#pragma unroll
  for (int kk = 0; kk < C::kN / 16; ++kk)
    mma_f16_ts(tDV, tS + part_col<C::kCols>(kk), make_sdesc_sw128(sG + kk * 2048, C::kRowPanel, 1024), kIdesc, (kk > 0 || more) ? 1u : 0u);
}
template <int DK, int DV>
__device__ __forceinline__ void issue_dk(uint32_t tDK, uint32_t tDP, uint32_t sQ, bool more) {
  using C = KvCfg<DK, DV>;
  constexpr uint32_t kIdesc = make_idesc(kBlk, DK, true);
#pragma unroll
  for (int kk = 0; kk < C::kN / 16; ++kk)
    mma_f16_ts(tDK, tDP + part_col<C::kCols>(kk), make_sdesc_sw128(sQ + kk * 2048, C::kRowPanel, 1024), kIdesc, (kk > 0 || more) ? 1u : 0u);
}

// A dK and dV tile once more, by the compute warps alone, if what is not finite may have come through a product.
template <int DK, int DV>
__device__ __noinline__ void dkdv_again(const CUtensorMap* tmQ, const CUtensorMap* tmG, const Params& p, unsigned index, uint8_t* smem, uint32_t tmem) {
  using C = KvCfg<DK, DV>;
  constexpr int kCols = C::kCols;
  const uint32_t sK = smem_u32(smem + C::kOffK), sV = smem_u32(smem + C::kOffV), sQ = smem_u32(smem + C::kOffStage), sG = sQ + C::kQBytes;
  const uint32_t loaded = smem_u32(smem + C::kOffBar) + 8u * (2 * C::kStages + 6), done = loaded + 8;
  const WaitCtl wc{reinterpret_cast<volatile int*>(smem + C::kOffMisc + 4), p.wait_limit_ns, 0u, &g_moa_window_bwd_status};
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = warp >> 2, lane_base = (warp & 3) * 32, row = lane_base + lane;
  const uint32_t lanes = uint32_t(lane_base) << 16;
  const uint32_t tS = tmem + C::kTmemS, tDP = tmem + C::kTmemDP, tDV = tmem + C::kTmemDV, tDK = tmem + C::kTmemDK;
  const KvItem it = kv_item(p, index);
  const int k0 = it.kt * kBlk, k1 = (k0 + kBlk < p.Nk ? k0 + kBlk : p.Nk) - 1, off = p.Nk - p.N, key = k0 + row;
  const Range range = rows_of_tokens(p.mask, it.kt, p.N, p.Nk, C::kHalves * p.PT);
  const int all = range.n * p.chunks, t0 = it.whole ? 0 : it.piece * p.piece;
  const int n_t = it.whole ? all : all - t0 < p.piece ? all - t0 : p.piece;
  const int64_t bh = int64_t(it.b) * p.Hk + it.h;
  struct Row {
    int hq, i;
    int64_t at;
    bool real;
  };
  auto tile_of = [&](int t, int* chunk) {   // the first half of row tile number t of the piece
    *chunk = (t0 + t) / range.n;
    return (range.first + (t0 + t) - *chunk * range.n) * C::kHalves;
  };
  auto row_of_tile = [&](int t, int r) {
    int chunk;
    const int half = tile_of(t, &chunk) + r / kHalf, in_half = r % kHalf, pos = in_half / p.GC, g = chunk * p.GC + in_half - pos * p.GC;
    const int i = half * p.PT + pos;
    return Row{it.h * p.G + g, i, (int64_t(bh * p.chunks + chunk) * p.n_ht + half) * kHalf + in_half, pos < p.PT && g < p.G && i < p.N};
  };
  // whether a token of the tile does not see some row of a row tile
  auto partly = [&](int t) {
    int chunk;
    const int half = tile_of(t, &chunk), p0 = half * p.PT + off, p1 = p0 + C::kHalves * p.PT - 1;
    return p0 < k1 || (p1 - k0 >= p.mask.window && k1 >= p.mask.sinks);
  };
  {
    bool odd = false;
    if (part == 0 && key < p.Nk) odd = odd_row<DK>(row_of(p.k, it.b, it.h, key)) || odd_row<DV>(row_of(p.v, it.b, it.h, key));
#pragma unroll 1
    for (int t = 0; t < n_t; ++t) {
      if (!partly(t) || int(threadIdx.x) >= C::kN) continue;
      const Row r = row_of_tile(t, threadIdx.x);
      if (!r.real) continue;
      odd |= !(p.nl[r.at] < INFINITY) || !(fabsf(p.delta[r.at]) < INFINITY) || odd_row<DK>(row_of(p.q, it.b, r.hq, r.i)) ||
             odd_row<DV>(row_of(p.go, it.b, r.hq, r.i));
    }
    if (meet(!odd)) return;
  }
  const bool first = threadIdx.x == 0, bounded = p.mask.window != win::kNoWindow && key >= p.mask.sinks;
  bool ok = true;
  uint32_t products = 0;
#pragma unroll 1
  for (int t = 0; t < n_t; ++t) {
    int chunk;
    const int half = tile_of(t, &chunk);
    ok = meet(ok);   // the row tile before is done with
    if (!ok) break;
    if (first) {
      mbar_arrive_expect_tx(loaded, C::kHalves * (DK + DV) * 2 * p.GC * p.PT + 2 * C::kVecBytes);
#pragma unroll 1
      for (int f = 0; f < C::kHalves; ++f) {
        const int i0 = (half + f) * p.PT;
#pragma unroll 1
        for (int q = 0; q < DK / 64; ++q)
          tma_load_5d(sQ + q * C::kRowPanel + f * kHalf * 128, tmQ, loaded, q * 64, chunk * p.GC, i0, it.h, it.b);
#pragma unroll 1
        for (int q = 0; q < DV / 64; ++q)
          tma_load_5d(sG + q * C::kRowPanel + f * kHalf * 128, tmG, loaded, q * 64, chunk * p.GC, i0, it.h, it.b);
      }
      const int64_t vrow = ((bh * p.chunks + chunk) * p.n_ht + half) * kHalf;
      bulk_load(sG + C::kGBytes, p.nl + vrow, C::kVecBytes, loaded);
      bulk_load(sG + C::kGBytes + C::kVecBytes, p.delta + vrow, C::kVecBytes, loaded);
    }
    ok = wait_bounded(loaded, uint32_t(t) & 1u, wc);
    if (first) {
      tc_fence_after_sync();
      issue_scores<DK, DV>(tS, sK, sQ);
      issue_changes<DK, DV>(tDP, sV, sG);
      mma_commit(done);
    }
    ok = wait_bounded(done, products++ & 1u, wc) && ok;
    tc_fence_after_sync();
    const int p0 = half * p.PT + part * kCols / kHalf * p.PT + off, ahead = key - p0;
    int from = ahead <= 0 ? 0 : ahead >= p.PT ? kHalf : ahead * p.GC, upto = kHalf;
    if (bounded) {
      const int64_t left = int64_t(ahead) + p.mask.window;
      upto = left <= 0 ? 0 : left >= p.PT ? kHalf : int(left) * p.GC;
    }
    from -= part * kCols % kHalf, upto -= part * kCols % kHalf;
    const uint32_t nl4 = sG + C::kGBytes + part * kCols * 4, d4 = nl4 + C::kVecBytes;
#pragma unroll 1
    for (int c = 0; c < kCols; c += 32) {
      const uint32_t bits = below(upto, c / 32) & ~below(from, c / 32);
      uint32_t r[32], pk[16];
      float w[32];
      tmem_ld_32x32b_x32(tS + lanes + part * kCols + c, r);
      tmem_wait_ld();
      reg_anchor_x32(r);
#pragma unroll
      for (int e = 0; e < 32; e += 4) {
        const float4 l = lds_f32x4(nl4 + (c + e) * 4);
        const float x[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
          w[e + i] = bits >> (e + i) & 1u ? ex2_approx(fmaf(__uint_as_float(r[e + i]), p.c_log2, x[i])) : 0.f;
      }
#pragma unroll
      for (int e = 0; e < 32; e += 2) pk[e >> 1] = pack_bf16x2(w[e], w[e + 1]);
      tmem_st_32x32b_x16(tS + lanes + part * kCols + c / 2, pk);
      tmem_ld_32x32b_x32(tDP + lanes + part * kCols + c, r);
      tmem_wait_ld();
      reg_anchor_x32(r);
#pragma unroll
      for (int e = 0; e < 32; e += 4) {
        const float4 d = lds_f32x4(d4 + (c + e) * 4);
        const float x[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) w[e + i] = bits >> (e + i) & 1u ? w[e + i] * (__uint_as_float(r[e + i]) - x[i]) : 0.f;
      }
#pragma unroll
      for (int e = 0; e < 32; e += 2) pk[e >> 1] = pack_bf16x2(w[e], w[e + 1]);
      tmem_st_32x32b_x16(tDP + lanes + part * kCols + c / 2, pk);
      tmem_wait_st();
    }
    if (partly(t)) {
      take_out<DK>(smem + C::kOffStage, C::kN, C::kRowPanel);
      take_out<DV>(smem + C::kOffStage + C::kQBytes, C::kN, C::kRowPanel);
      fence_proxy_async_smem();
    }
    tc_fence_before_sync();
    ok = meet(ok);
    if (first) {
      tc_fence_after_sync();
      issue_dv<DK, DV>(tDV, tS, sG, t > 0);
      issue_dk<DK, DV>(tDK, tDP, sQ, t > 0);
      mma_commit(done);
    }
    ok = wait_bounded(done, products++ & 1u, wc) && ok;
    tc_fence_after_sync();
  }
  ok = meet(ok);
  if (!ok) {   // the last copies and products end before the CTA does
    if (first) {
      wait_quiesce(loaded, uint32_t(n_t - 1) & 1u, wc.limit_ns, wc.status);
      wait_quiesce(done, (products - 1) & 1u, wc.limit_ns, wc.status);
    }
    return;
  }
  // what was taken out, to the tokens that it reaches
  const uint32_t acc = lanes + (part == 0 ? tDV : tDK);
#pragma unroll 1
  for (int c = 0; c < (part == 0 ? DV : DK); c += 32) {
    uint32_t o[32];
    tmem_ld_32x32b_x32(acc + c, o);
    tmem_wait_ld();
    reg_anchor_x32(o);
#pragma unroll 1
    for (int t = 0; t < n_t && any_number(o, key < p.Nk); ++t) {
      if (!partly(t)) continue;
#pragma unroll 1
      for (int r0 = 0; r0 < C::kN; r0 += 32) {
        const Row r = row_of_tile(t, r0 + lane);
        const __nv_bfloat16* x = r.real ? row_of(part == 0 ? p.go : p.q, it.b, r.hq, r.i) + c : nullptr;
        const uint32_t odd = __ballot_sync(0xffffffffu, x != nullptr && odd_row<32>(x));
        if (odd == 0) continue;
        auto seen = [&](int b) { return key < p.Nk && sees(p.mask, row_of_tile(t, r0 + b).i + off, key); };
        if (part == 0)
          add_odd<false>(o, odd, x, seen);
        else
          add_odd<true>(o, odd, x, seen);
      }
    }
    tmem_st_32x32b_x32(acc + c, o);
    tmem_wait_st();
  }
  const bool valid = key < p.Nk;
  float* piece = it.whole ? nullptr : p.part + (((bh * p.cut + it.kt) * p.pieces + it.piece) * kBlk + row) * (DK + DV);
  if (part == 0)
    store_row<DV, true>(acc, 1.f, row_of(p.dv, it.b, it.h, valid ? key : 0), piece ? piece + DK : nullptr, valid);
  else
    store_row<DK, true>(acc, p.scale, row_of(p.dk, it.b, it.h, valid ? key : 0), piece, valid);
  tc_fence_before_sync();
}

template <int DK, int DV>
__device__ __forceinline__ void dkdv_tile(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV,
                                          const CUtensorMap& tmG, const Params& p, unsigned index) {
  using C = KvCfg<DK, DV>;
  constexpr int kCols = C::kCols;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const uint32_t sK = smem_u32(smem + C::kOffK), sV = smem_u32(smem + C::kOffV), sStage = smem_u32(smem + C::kOffStage);
  const uint32_t bar0 = smem_u32(smem + C::kOffBar);
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (C::kStages + s); };
  const uint32_t kv_full = bar0 + 8u * (2 * C::kStages);
  const uint32_t s_full = kv_full + 8, dp_full = kv_full + 16, p_ready = kv_full + 24;
  const uint32_t ds_ready = kv_full + 32, acc_done = kv_full + 40;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::kOffMisc);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + C::kOffMisc + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const WaitCtl wc{abort_flag, p.wait_limit_ns, 0u, &g_moa_window_bwd_status};

  const KvItem it = kv_item(p, index);
  const int k0 = it.kt * kBlk;
  const Range range = rows_of_tokens(p.mask, it.kt, p.N, p.Nk, C::kHalves * p.PT);
  const int all = range.n * p.chunks;
  const int t0 = it.whole ? 0 : it.piece * p.piece;
  const int n_t = it.whole ? all : all - t0 < p.piece ? all - t0 : p.piece;
  if (n_t <= 0 && !it.whole) return;   // the join adds what pieces there are
  const int64_t bh = int64_t(it.b) * p.Hk + it.h;

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    mbar_init(kv_full, 1);
    mbar_init(s_full, 1);
    mbar_init(dp_full, 1);
    mbar_init(p_ready, kComputeThreads);
    mbar_init(ds_ready, kComputeThreads);
    mbar_init(acc_done, 1);
    *abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == kMmaWarp) {
    tmem_alloc(smem_u32(tmem_slot), C::kTmemCols);
    tmem_relinquish();
  }
  if (p.GC * p.PT < kHalf) {   // rows of a half that no copy fills
    for (int x = threadIdx.x; x < C::kStages * C::kStageBytes / 16; x += kThreads)
      reinterpret_cast<uint4*>(smem + C::kOffStage)[x] = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  bool bad = false;   // the thread's outputs are not all finite

  if (warp == kLoadWarp) {
    // ---------------------------------------------------------------- TMA producer
    if (lane == 0 && n_t > 0) {
      tma_prefetch_desc(&tmQ);
      tma_prefetch_desc(&tmK);
      tma_prefetch_desc(&tmV);
      tma_prefetch_desc(&tmG);
      mbar_arrive_expect_tx(kv_full, C::kKBytes + C::kVBytes);
#pragma unroll
      for (int f = 0; f < kBlk / C::kN; ++f) {
#pragma unroll
        for (int q = 0; q < DK / 64; ++q)
          tma_load_4d(sK + q * kPanelBytes + f * C::kRowPanel, &tmK, kv_full, q * 64, k0 + f * C::kN, it.h, it.b);
#pragma unroll
        for (int q = 0; q < DV / 64; ++q)
          tma_load_4d(sV + q * kPanelBytes + f * C::kRowPanel, &tmV, kv_full, q * 64, k0 + f * C::kN, it.h, it.b);
      }
      int slot = 0;
      uint32_t phase = 0, issued = 0, issued_phase = 0;
      bool aborted = false;
      int chunk = t0 / range.n, pt = range.first + (t0 - chunk * range.n);
      const uint32_t bytes = C::kHalves * (DK + DV) * 2 * p.GC * p.PT + 2 * C::kVecBytes;
      for (int i = 0; i < n_t; ++i) {
        if (!wait_bounded(empty_bar(slot), phase ^ 1u, wc)) {
          aborted = true;
          break;
        }
        issued |= 1u << slot;
        issued_phase = (issued_phase & ~(1u << slot)) | (phase << slot);
        const uint32_t st = sStage + slot * C::kStageBytes;
        mbar_arrive_expect_tx(full_bar(slot), bytes);
#pragma unroll
        for (int f = 0; f < C::kHalves; ++f) {
          const int i0 = (pt * C::kHalves + f) * p.PT;
#pragma unroll
          for (int q = 0; q < DK / 64; ++q)
            tma_load_5d(st + q * C::kRowPanel + f * kHalf * 128, &tmQ, full_bar(slot), q * 64, chunk * p.GC, i0, it.h, it.b);
#pragma unroll
          for (int q = 0; q < DV / 64; ++q)
            tma_load_5d(st + C::kQBytes + q * C::kRowPanel + f * kHalf * 128, &tmG, full_bar(slot), q * 64, chunk * p.GC, i0,
                        it.h, it.b);
        }
        const int64_t vrow = ((bh * p.chunks + chunk) * p.n_ht + pt * C::kHalves) * kHalf;
        bulk_load(st + C::kQBytes + C::kGBytes, p.nl + vrow, C::kVecBytes, full_bar(slot));
        bulk_load(st + C::kQBytes + C::kGBytes + C::kVecBytes, p.delta + vrow, C::kVecBytes, full_bar(slot));
        if (++pt == range.first + range.n) {
          pt = range.first;
          ++chunk;
        }
        if (++slot == C::kStages) {
          slot = 0;
          phase ^= 1u;
        }
      }
      if (aborted || *abort_flag) {
        wait_quiesce(kv_full, 0, p.wait_limit_ns, &g_moa_window_bwd_status);
        for (int sl = 0; sl < C::kStages; ++sl)
          if (issued & (1u << sl)) wait_quiesce(full_bar(sl), (issued_phase >> sl) & 1u, p.wait_limit_ns, &g_moa_window_bwd_status);
      }
    }
  } else if (warp == kMmaWarp) {
    // ---------------------------------------------------------------- MMA issuer
    if (lane == 0) {
      const uint32_t tS = tmem + C::kTmemS, tDP = tmem + C::kTmemDP;
      const uint32_t tDV = tmem + C::kTmemDV, tDK = tmem + C::kTmemDK;
      int slot = 0;
      uint32_t phase = 0;
      auto issue_s = [&](uint32_t sQ) {
        issue_scores<DK, DV>(tS, sK, sQ);
        mma_commit(s_full);
      };
      auto issue_dp = [&](uint32_t sG) {
        issue_changes<DK, DV>(tDP, sV, sG);
        mma_commit(dp_full);
      };
      auto stage = [&](int st) { return sStage + st * C::kStageBytes; };
      // S(0) dP(0) | dV(0) S(1) dK(0) dP(1) | dV(1) S(2) dK(1) dP(2) | ...: the scores of tile i + 1 are ready when
      // the compute warps finish dS of tile i.  S(i + 1) overwrites the columns of P^T(i) only after dV(i), and
      // dP(i + 1) those of dS^T(i) only after dK(i), both issued earlier (products of one CTA complete in order).
      bool ok = n_t > 0 && wait_bounded(kv_full, 0, wc) && wait_bounded(full_bar(0), 0, wc);
      if (ok) {
        tc_fence_after_sync();
        issue_s(stage(0));
        issue_dp(stage(0) + C::kQBytes);
      }
      for (int i = 0; ok && i < n_t; ++i) {
        const int st = slot;
        if (++slot == C::kStages) {
          slot = 0;
          phase ^= 1u;
        }
        const uint32_t sQ = stage(st), sG = sQ + C::kQBytes;
        const uint32_t par = uint32_t(i) & 1u;
        // dV += P^T dO: A from TMEM, B = dO tile MN-major
        ok = wait_bounded(p_ready, par, wc);
        if (!ok) break;
        tc_fence_after_sync();
        issue_dv<DK, DV>(tDV, tS, sG, i > 0);
        const bool more = i + 1 < n_t;
        if (more) {
          ok = wait_bounded(full_bar(slot), phase, wc);
          if (!ok) break;
          tc_fence_after_sync();
          issue_s(stage(slot));
        }
        // dK += dS^T Q (the scale comes at the end)
        ok = wait_bounded(ds_ready, par, wc);
        if (!ok) break;
        tc_fence_after_sync();
        issue_dk<DK, DV>(tDK, tDP, sQ, i > 0);
        mma_commit(empty_bar(st));
        if (more) issue_dp(stage(slot) + C::kQBytes);
      }
      // arrives once everything issued is complete, on the abort path too
      mma_commit(acc_done);
    }
  } else {
    // ---------------------------------------------------------------- compute warps
    const int part = warp >> 2;
    const int lane_base = (warp & 3) * 32, row = lane_base + lane;
    const uint32_t lanes = uint32_t(lane_base) << 16;
    const uint32_t tS = tmem + lanes + C::kTmemS + part * kCols;
    const uint32_t tDP = tmem + lanes + C::kTmemDP + part * kCols;
    const uint64_t cc = pack_f32x2(p.c_log2, p.c_log2);
    const int key = k0 + row;
    const bool bounded = p.mask.window != win::kNoWindow && key >= p.mask.sinks;   // seen by a window's rows only
    int slot = 0;
    uint32_t phase = 0;
    bool ok = true;
    int pt = n_t > 0 ? range.first + t0 % range.n : 0;
    auto wait_warp = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, wait_bounded(bar, parity, wc)) != 0; };
    for (int i = 0; ok && i < n_t; ++i) {
      const int st = slot;
      const uint32_t par = uint32_t(i) & 1u;
      // -L and D came with the tiles: the wait for the stage makes them visible to this thread
      // Waits that run out leave the loop together, at its end: until then what they would have brought is used as it is.
      ok = wait_bounded(full_bar(st), phase, wc) && wait_bounded(s_full, par, wc);
      if (++slot == C::kStages) {
        slot = 0;
        phase ^= 1u;
      }
      tc_fence_after_sync();
      const uint32_t nl4 = sStage + st * C::kStageBytes + C::kQBytes + C::kGBytes + part * kCols * 4;
      const uint32_t d4 = nl4 + C::kVecBytes;
      // the rows that see the token: columns [from, upto) of this part, which lies in one half
      const int p0 = pt * C::kHalves * p.PT + part * kCols / kHalf * p.PT + (p.Nk - p.N);
      if (++pt == range.first + range.n) pt = range.first;
      const int ahead = key - p0;   // positions of the half before the token's own
      int from = ahead <= 0 ? 0 : ahead >= p.PT ? kHalf : ahead * p.GC, upto = kHalf;
      if (bounded) {
        const int64_t left = int64_t(ahead) + p.mask.window;
        upto = left <= 0 ? 0 : left >= p.PT ? kHalf : int(left) * p.GC;
      }
      from -= part * kCols % kHalf, upto -= part * kCols % kHalf;
      const bool full = __all_sync(0xffffffffu, from <= 0 && upto >= kCols);
      uint32_t r[kCols];
      float w[kCols];
      uint32_t pk[kCols / 2];
      tmem_each_32<kCols>(tS, r, [&](int c) {
#pragma unroll
        for (int q = c; q < c + 32; q += 4) {
          const float4 l = lds_f32x4(nl4 + q * 4);
          ffma2(w[q], w[q + 1], __uint_as_float(r[q]), __uint_as_float(r[q + 1]), cc, pack_f32x2(l.x, l.y));
          ffma2(w[q + 2], w[q + 3], __uint_as_float(r[q + 2]), __uint_as_float(r[q + 3]), cc, pack_f32x2(l.z, l.w));
        }
        if (!full) {
          const uint32_t bits = below(upto, c / 32) & ~below(from, c / 32);
#pragma unroll
          for (int e = 0; e < 32; ++e) w[c + e] = bits >> e & 1u ? w[c + e] : -INFINITY;
        }
#pragma unroll
        for (int q = c; q < c + 32; q += 2) {
          w[q] = ex2_approx(w[q]);
          w[q + 1] = ex2_approx(w[q + 1]);
          pk[q >> 1] = pack_bf16x2(w[q], w[q + 1]);
        }
      });
      tmem_store_part<kCols>(tS, pk);
      tmem_wait_st();
      tc_fence_before_sync();
      mbar_arrive(p_ready);
      ok = wait_bounded(dp_full, par, wc) && ok;
      tc_fence_after_sync();
      tmem_each_32<kCols>(tDP, r, [&](int c) {
#pragma unroll
        for (int q = c; q < c + 32; q += 4) {
          const float4 d = lds_f32x4(d4 + q * 4);
          const float s0 = w[q] * (__uint_as_float(r[q]) - d.x);
          const float s1 = w[q + 1] * (__uint_as_float(r[q + 1]) - d.y);
          const float s2 = w[q + 2] * (__uint_as_float(r[q + 2]) - d.z);
          const float s3 = w[q + 3] * (__uint_as_float(r[q + 3]) - d.w);
          pk[q >> 1] = pack_bf16x2(s0, s1);
          pk[(q >> 1) + 1] = pack_bf16x2(s2, s3);
        }
      });
      tmem_store_part<kCols>(tDP, pk);
      tmem_wait_st();
      tc_fence_before_sync();
      mbar_arrive(ds_ready);
      ok = __all_sync(0xffffffffu, ok);
    }
    // The first part writes dV, the second scale dK.
    const bool valid = key < p.Nk;
    if (n_t <= 0) {   // tokens that no row sees
      if (valid) {
        uint4* dst = reinterpret_cast<uint4*>(row_of(part == 0 ? p.dv : p.dk, it.b, it.h, key));
        for (int e = 0; e < (part == 0 ? DV : DK) / 8; ++e) dst[e] = make_uint4(0, 0, 0, 0);
      }
    } else if (ok && wait_warp(acc_done, 0)) {
      tc_fence_after_sync();
      float* piece = it.whole ? nullptr : p.part + (((bh * p.cut + it.kt) * p.pieces + it.piece) * kBlk + row) * (DK + DV);
      bad = !(part == 0 ? store_row<DV>(tmem + lanes + C::kTmemDV, 1.f, row_of(p.dv, it.b, it.h, valid ? key : 0), piece ? piece + DK : nullptr, valid)
                        : store_row<DK>(tmem + lanes + C::kTmemDK, p.scale, row_of(p.dk, it.b, it.h, valid ? key : 0), piece, valid));
    }
  }

  if (warp == kMmaWarp && lane == 0) wait_quiesce(acc_done, 0, p.wait_limit_ns, &g_moa_window_bwd_status);
  tc_fence_before_sync();
  if (__syncthreads_or(bad)) {
    const bool dead = *abort_flag != 0;
    if (threadIdx.x == 0) {
      mbar_init(acc_done + 8, 1);
      mbar_init(acc_done + 8 + 8, 1);
      fence_barrier_init();
    }
    __syncthreads();
    if (!dead && warp < kMmaWarp) {
      tc_fence_after_sync();
      dkdv_again<DK, DV>(&tmQ, &tmG, p, index, smem, tmem);
    }
    tc_fence_before_sync();
    __syncthreads();
  }
  if (warp == kMmaWarp) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, C::kTmemCols);
  }
}

// Adds the pieces of cut token tiles: four features of a token a thread.
template <int DK, int DV>
__global__ void __launch_bounds__(256)
window_dkdv_tc_join_kernel(const Params p, int64_t n) {
  wait_for_previous();
  constexpr int kQuads = (DK + DV) / 4;
  const int64_t x = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (x >= n) return;
  const int64_t row = x / kQuads;   // (key head, tile, token)
  const int c = int(x - row * kQuads) * 4;
  const int64_t tile = row / kBlk, bh = tile / p.cut;
  const int j = int(row - tile * kBlk), kt = int(tile - bh * p.cut);
  const int b = int(bh / p.Hk), h = int(bh - int64_t(b) * p.Hk), key = kt * kBlk + j;
  if (key >= p.Nk) return;
  const int all = rows_of_tokens(p.mask, kt, p.N, p.Nk, width_of(DK, DV) / kHalf * p.PT).n * p.chunks;
  const int pieces = (all + p.piece - 1) / p.piece;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int i = 0; i < pieces; ++i) {
    const float4 v = *reinterpret_cast<const float4*>(p.part + ((tile * p.pieces + i) * kBlk + j) * (DK + DV) + c);
    s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
  }
  const float mul = c < DK ? p.scale : 1.f;
  __nv_bfloat16* dst = c < DK ? row_of(p.dk, b, h, key) + c : row_of(p.dv, b, h, key) + (c - DK);
  *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(s.x * mul, s.y * mul), pack_bf16x2(s.z * mul, s.w * mul));
}

// ------------------------------------------------------------------------------------------------
// dQ
// ------------------------------------------------------------------------------------------------
template <int DK, int DV>
struct QCfg {
  static constexpr int kN = width_of(DK, DV), kCols = kN / kParts;
  static constexpr int kQBytes = kBlk * DK * 2, kGBytes = kBlk * DV * 2;
  static constexpr int kTokenPanel = kN * 128;
  static constexpr int kKBytes = kN * DK * 2, kVBytes = kN * DV * 2;
  static constexpr int kStageBytes = kKBytes + kVBytes;
  static constexpr int kStages = ring_stages(DK, DV);
  static constexpr int kOffQ = 0, kOffG = kQBytes, kOffStage = kQBytes + kGBytes;
  // barriers: full[NS], empty[NS], q_full, s_full, dp_full, ds_ready, acc_done, s_free, again_loaded, again_done
  static constexpr int kNumBars = 2 * kStages + 8;
  static constexpr int kOffBar = kOffStage + kStages * kStageBytes;
  static constexpr int kOffMisc = kOffBar + kNumBars * 8;
  static constexpr int kSmemBytes = kOffMisc + 16 + 1024;
  static constexpr uint32_t kTmemS = 0, kTmemDP = kN, kTmemDQ = 2 * kN;
  static constexpr uint32_t kTmemCols = 512 / ctas_of(DK, DV);
  static_assert(kTmemDQ + DK <= kTmemCols, "TMEM budget");
  static_assert((kSmemBytes + 1024) * ctas_of(DK, DV) <= 233472, "shared memory budget");
};

// The products of a step: S = Q K^T, dP = dO V^T, dQ += dS K (A from TMEM, B MN-major).
template <int DK, int DV>
__device__ __forceinline__ void issue_row_scores(uint32_t tS, uint32_t sQ, uint32_t sK) {
  using C = QCfg<DK, DV>;
  constexpr uint32_t kIdesc = make_idesc(kBlk, C::kN, false);
#pragma unroll
  for (int kk = 0; kk < DK / 16; ++kk) {
    const uint32_t r = (kk >> 2) * kPanelBytes + (kk & 3) * 32, k = (kk >> 2) * C::kTokenPanel + (kk & 3) * 32;
    mma_f16_ss(tS, make_sdesc_sw128(sQ + r, 16, 1024), make_sdesc_sw128(sK + k, 16, 1024), kIdesc, kk > 0 ? 1u : 0u);
  }
}
template <int DK, int DV>
__device__ __forceinline__ void issue_row_changes(uint32_t tDP, uint32_t sG, uint32_t sV) {
  using C = QCfg<DK, DV>;
  constexpr uint32_t kIdesc = make_idesc(kBlk, C::kN, false);
#pragma unroll
  for (int kk = 0; kk < DV / 16; ++kk) {
    const uint32_t r = (kk >> 2) * kPanelBytes + (kk & 3) * 32, k = (kk >> 2) * C::kTokenPanel + (kk & 3) * 32;
    mma_f16_ss(tDP, make_sdesc_sw128(sG + r, 16, 1024), make_sdesc_sw128(sV + k, 16, 1024), kIdesc, kk > 0 ? 1u : 0u);
  }
}
template <int DK, int DV>
__device__ __forceinline__ void issue_dq(uint32_t tDQ, uint32_t tDP, uint32_t sK, bool more) {
  using C = QCfg<DK, DV>;
  constexpr uint32_t kIdesc = make_idesc(kBlk, DK, true);
#pragma unroll
  for (int kk = 0; kk < C::kN / 16; ++kk)
    mma_f16_ts(tDQ, tDP + part_col<C::kCols>(kk), make_sdesc_sw128(sK + kk * 2048, C::kTokenPanel, 1024), kIdesc, (kk > 0 || more) ? 1u : 0u);
}

// A dQ tile's work: the pair of halves, this piece's token tiles [j0, j0 + n) of the list.
struct QItem {
  int64_t tile;
  RowTile t;
  win::Tiles list;
  int piece, i1, j0, n;
};
template <int DK, int DV>
__device__ __forceinline__ QItem q_item(const Params& p, unsigned index) {
  QItem x;
  // the last positions, which see the most without a window, come first
  const unsigned which = index / unsigned(p.q_pieces);
  x.piece = int(index - which * unsigned(p.q_pieces));
  const int64_t per = int64_t(p.chunks) * (p.n_ht / 2), group = which / per;
  x.tile = group * per + (per - 1 - (which - group * per));
  x.t = row_tile(p, x.tile);
  // (a pair's positions may all lie past the end)
  x.i1 = x.t.i0 + 2 * p.PT - 1 < p.N ? x.t.i0 + 2 * p.PT - 1 : p.N - 1;
  x.list = win::tiles_of(p.mask, p.Nk, p.N, x.t.i0, x.i1, QCfg<DK, DV>::kN);
  x.j0 = int(int64_t(x.list.n) * x.piece / p.q_pieces);
  x.n = int(int64_t(x.list.n) * (x.piece + 1) / p.q_pieces) - x.j0;
  return x;
}

// A dQ tile once more, by the compute warps alone, if what is not finite may have come through a product.
template <int DK, int DV>
__device__ __noinline__ void dq_again(const CUtensorMap* tmK, const CUtensorMap* tmV, const Params& p, unsigned index, uint8_t* smem, uint32_t tmem) {
  using C = QCfg<DK, DV>;
  constexpr int kCols = C::kCols, wq = DK / kParts;
  const uint32_t sQ = smem_u32(smem + C::kOffQ), sG = smem_u32(smem + C::kOffG), sK = smem_u32(smem + C::kOffStage), sV = sK + C::kKBytes;
  const uint32_t loaded = smem_u32(smem + C::kOffBar) + 8u * (2 * C::kStages + 6), done = loaded + 8;
  const WaitCtl wc{reinterpret_cast<volatile int*>(smem + C::kOffMisc + 4), p.wait_limit_ns, 0u, &g_moa_window_bwd_status};
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = warp >> 2, lane_base = (warp & 3) * 32, row = lane_base + lane;
  const uint32_t lanes = uint32_t(lane_base) << 16;
  const uint32_t tS = tmem + C::kTmemS, tDP = tmem + C::kTmemDP, tDQ = tmem + C::kTmemDQ;
  const QItem x = q_item<DK, DV>(p, index);
  const RowAt at = row_at(p, x.t, row);
  const bool live = at.real;
  const float nl = p.nl[x.tile * kBlk + row], dd = p.delta[x.tile * kBlk + row];
  const int off = p.Nk - p.N, p0 = x.t.i0 + off, p1 = x.i1 + off, pos = at.i + off;
  const int lim = live ? win::row_end(p.mask, p.Nk, p.N, at.i) : 0, low = live ? win::row_low(p.mask, p.Nk, p.N, at.i) : 0;
  // whether a row of the tile does not see some token of the tile from n0 on
  auto partly = [&](int n0) { return n0 + C::kN - 1 > p0 || (p1 - n0 >= p.mask.window && n0 + C::kN > p.mask.sinks); };
  {
    // (a row that sees nothing, and is none, has what hidden tokens give only)
    bool odd = live && pos < 0 && (!(nl < INFINITY) || !(fabsf(dd) < INFINITY) || odd_row<DK>(row_of(p.q, x.t.b, x.t.h * p.G + at.g, at.i)));
#pragma unroll 1
    for (int j = 0; j < x.n; ++j) {
      const int n0 = x.list.at(x.j0 + j) * C::kN, token = n0 + int(threadIdx.x);
      if (!partly(n0) || int(threadIdx.x) >= C::kN || token >= p.Nk) continue;
      odd |= odd_row<DK>(row_of(p.k, x.t.b, x.t.h, token)) || odd_row<DV>(row_of(p.v, x.t.b, x.t.h, token));
    }
    if (meet(!odd)) return;
  }
  const bool first = threadIdx.x == 0;
  bool ok = true;
  uint32_t products = 0;
#pragma unroll 1
  for (int j = 0; j < x.n; ++j) {
    const int n0 = x.list.at(x.j0 + j) * C::kN;
    ok = meet(ok);   // the tile before is done with
    if (!ok) break;
    if (first) {
      mbar_arrive_expect_tx(loaded, C::kStageBytes);
#pragma unroll 1
      for (int q = 0; q < DK / 64; ++q) tma_load_4d(sK + q * C::kTokenPanel, tmK, loaded, q * 64, n0, x.t.h, x.t.b);
#pragma unroll 1
      for (int q = 0; q < DV / 64; ++q) tma_load_4d(sV + q * C::kTokenPanel, tmV, loaded, q * 64, n0, x.t.h, x.t.b);
    }
    ok = wait_bounded(loaded, uint32_t(j) & 1u, wc);
    if (first) {
      tc_fence_after_sync();
      issue_row_scores<DK, DV>(tS, sQ, sK);
      issue_row_changes<DK, DV>(tDP, sG, sV);
      mma_commit(done);
    }
    ok = wait_bounded(done, products++ & 1u, wc) && ok;
    tc_fence_after_sync();
#pragma unroll 1
    for (int c = 0; c < kCols; c += 32) {
      const int t0 = n0 + part * kCols + c;
      const uint32_t bits = below(lim - t0, 0) & (~below(low - t0, 0) | below(p.mask.sinks - t0, 0));
      uint32_t r[32], pk[16];
      float w[32];
      tmem_ld_32x32b_x32(tS + lanes + part * kCols + c, r);
      tmem_wait_ld();
      reg_anchor_x32(r);
#pragma unroll
      for (int e = 0; e < 32; ++e) w[e] = bits >> e & 1u ? ex2_approx(fmaf(__uint_as_float(r[e]), p.c_log2, nl)) : 0.f;
      tmem_ld_32x32b_x32(tDP + lanes + part * kCols + c, r);
      tmem_wait_ld();
      reg_anchor_x32(r);
#pragma unroll
      for (int e = 0; e < 32; ++e) w[e] = bits >> e & 1u ? w[e] * (__uint_as_float(r[e]) - dd) : 0.f;
#pragma unroll
      for (int e = 0; e < 32; e += 2) pk[e >> 1] = pack_bf16x2(w[e], w[e + 1]);
      tmem_st_32x32b_x16(tDP + lanes + part * kCols + c / 2, pk);
      tmem_wait_st();
    }
    if (partly(n0)) {
      take_out<DK>(smem + C::kOffStage, C::kN, C::kTokenPanel);
      fence_proxy_async_smem();
    }
    tc_fence_before_sync();
    ok = meet(ok);
    if (first) {
      tc_fence_after_sync();
      issue_dq<DK, DV>(tDQ, tDP, sK, j > 0);
      mma_commit(done);
    }
    ok = wait_bounded(done, products++ & 1u, wc) && ok;
    tc_fence_after_sync();
  }
  ok = meet(ok);
  if (!ok) {   // the last copies and products end before the CTA does
    if (first) {
      wait_quiesce(loaded, uint32_t(x.n - 1) & 1u, wc.limit_ns, wc.status);
      wait_quiesce(done, (products - 1) & 1u, wc.limit_ns, wc.status);
    }
    return;
  }
  // what was taken out, to the rows that see it
  const uint32_t acc = tDQ + lanes + part * wq;
#pragma unroll 1
  for (int c = 0; c < wq; c += 32) {
    uint32_t o[32];
    tmem_ld_32x32b_x32(acc + c, o);
    tmem_wait_ld();
    reg_anchor_x32(o);
#pragma unroll 1
    for (int j = 0; j < x.n && any_number(o, live); ++j) {
      const int n0 = x.list.at(x.j0 + j) * C::kN;
      if (!partly(n0)) continue;
#pragma unroll 1
      for (int r0 = 0; r0 < C::kN; r0 += 32) {
        const int token = n0 + r0 + lane;
        const __nv_bfloat16* k = token < p.Nk ? row_of(p.k, x.t.b, x.t.h, token) + part * wq + c : nullptr;
        const uint32_t odd = __ballot_sync(0xffffffffu, k != nullptr && odd_row<32>(k));
        if (odd != 0) add_odd<true>(o, odd, k, [&](int b) { return live && sees(p.mask, pos, n0 + r0 + b); });
      }
    }
    tmem_st_32x32b_x32(acc + c, o);
    tmem_wait_st();
  }
  store_row<wq, true>(acc, p.scale, row_of(p.dq, x.t.b, x.t.h * p.G + (live ? at.g : 0), live ? at.i : 0) + part * wq,
                      p.q_pieces > 1 ? p.part_q + ((x.tile * p.q_pieces + x.piece) * kBlk + row) * DK + part * wq : nullptr, live);
  tc_fence_before_sync();
}

template <int DK, int DV>
__device__ __forceinline__ void dq_tile(const CUtensorMap& tmQ, const CUtensorMap& tmK, const CUtensorMap& tmV,
                                        const CUtensorMap& tmG, const Params& p, unsigned index) {
  using C = QCfg<DK, DV>;
  constexpr int kCols = C::kCols;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const uint32_t sQ = smem_u32(smem + C::kOffQ), sG = smem_u32(smem + C::kOffG), sStage = smem_u32(smem + C::kOffStage);
  const uint32_t bar0 = smem_u32(smem + C::kOffBar);
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (C::kStages + s); };
  const uint32_t q_full = bar0 + 8u * (2 * C::kStages);
  const uint32_t s_full = q_full + 8, dp_full = q_full + 16, ds_ready = q_full + 24;
  const uint32_t acc_done = q_full + 32, s_free = q_full + 40;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::kOffMisc);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + C::kOffMisc + 4);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const WaitCtl wc{abort_flag, p.wait_limit_ns, 0u, &g_moa_window_bwd_status};

  const QItem x = q_item<DK, DV>(p, index);
  const RowTile& t = x.t;
  const win::Tiles& list = x.list;
  const int64_t tile_id = x.tile;
  const int piece = x.piece, j0 = x.j0, n_kt = x.n;
  if (n_kt == 0 && p.q_pieces > 1) return;   // the join adds what pieces there are

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    mbar_init(q_full, 1);
    mbar_init(s_full, 1);
    mbar_init(dp_full, 1);
    mbar_init(ds_ready, kComputeThreads);
    mbar_init(acc_done, 1);
    mbar_init(s_free, kComputeThreads);
    *abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == kMmaWarp) {
    tmem_alloc(smem_u32(tmem_slot), C::kTmemCols);
    tmem_relinquish();
  }
  if (p.GC * p.PT < kHalf) {   // rows that no copy fills
    for (int x = threadIdx.x; x < (C::kQBytes + C::kGBytes) / 16; x += kThreads)
      reinterpret_cast<uint4*>(smem)[x] = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  bool bad = false;   // the thread's outputs are not all finite

  if (warp == kLoadWarp) {
    // ---------------------------------------------------------------- TMA producer
    if (lane == 0 && n_kt > 0) {
      tma_prefetch_desc(&tmQ);
      tma_prefetch_desc(&tmK);
      tma_prefetch_desc(&tmV);
      tma_prefetch_desc(&tmG);
      mbar_arrive_expect_tx(q_full, 2 * (DK + DV) * 2 * p.GC * p.PT);
#pragma unroll
      for (int f = 0; f < 2; ++f) {
#pragma unroll
        for (int q = 0; q < DK / 64; ++q)
          tma_load_5d(sQ + q * kPanelBytes + f * kHalf * 128, &tmQ, q_full, q * 64, t.chunk * p.GC, t.i0 + f * p.PT, t.h, t.b);
#pragma unroll
        for (int q = 0; q < DV / 64; ++q)
          tma_load_5d(sG + q * kPanelBytes + f * kHalf * 128, &tmG, q_full, q * 64, t.chunk * p.GC, t.i0 + f * p.PT, t.h, t.b);
      }
      int slot = 0;
      uint32_t phase = 0, issued = 0, issued_phase = 0;
      bool aborted = false;
      for (int j = 0; j < n_kt; ++j) {
        if (!wait_bounded(empty_bar(slot), phase ^ 1u, wc)) {
          aborted = true;
          break;
        }
        issued |= 1u << slot;
        issued_phase = (issued_phase & ~(1u << slot)) | (phase << slot);
        const uint32_t st = sStage + slot * C::kStageBytes;
        mbar_arrive_expect_tx(full_bar(slot), C::kStageBytes);
        const int n0 = list.at(j0 + j) * C::kN;
#pragma unroll
        for (int q = 0; q < DK / 64; ++q) tma_load_4d(st + q * C::kTokenPanel, &tmK, full_bar(slot), q * 64, n0, t.h, t.b);
#pragma unroll
        for (int q = 0; q < DV / 64; ++q)
          tma_load_4d(st + C::kKBytes + q * C::kTokenPanel, &tmV, full_bar(slot), q * 64, n0, t.h, t.b);
        if (++slot == C::kStages) {
          slot = 0;
          phase ^= 1u;
        }
      }
      if (aborted || *abort_flag) {
        wait_quiesce(q_full, 0, p.wait_limit_ns, &g_moa_window_bwd_status);
        for (int sl = 0; sl < C::kStages; ++sl)
          if (issued & (1u << sl)) wait_quiesce(full_bar(sl), (issued_phase >> sl) & 1u, p.wait_limit_ns, &g_moa_window_bwd_status);
      }
    }
  } else if (warp == kMmaWarp) {
    // ---------------------------------------------------------------- MMA issuer
    if (lane == 0) {
      const uint32_t tS = tmem + C::kTmemS, tDP = tmem + C::kTmemDP, tDQ = tmem + C::kTmemDQ;
      int slot = 0;
      uint32_t phase = 0;
      auto stage = [&](int st) { return sStage + st * C::kStageBytes; };
      auto issue_s = [&](uint32_t sK) {
        issue_row_scores<DK, DV>(tS, sQ, sK);
        mma_commit(s_full);
      };
      auto issue_dp = [&](uint32_t sV) {
        issue_row_changes<DK, DV>(tDP, sG, sV);
        mma_commit(dp_full);
      };
      // S(0) dP(0) | S(1) dQ(0) dP(1) | S(2) dQ(1) dP(2) | ...: S(j + 1) goes as soon as the compute warps hold S(j)
      // in registers (s_free); dP(j + 1) overwrites the columns of dS(j) only after dQ(j), issued earlier.
      bool ok = n_kt > 0 && wait_bounded(q_full, 0, wc) && wait_bounded(full_bar(0), 0, wc);
      if (ok) {
        tc_fence_after_sync();
        issue_s(stage(0));
        issue_dp(stage(0) + C::kKBytes);
      }
      for (int j = 0; ok && j < n_kt; ++j) {
        const int st = slot;
        if (++slot == C::kStages) {
          slot = 0;
          phase ^= 1u;
        }
        const uint32_t par = uint32_t(j) & 1u;
        const bool more = j + 1 < n_kt;
        if (more) {
          ok = wait_bounded(full_bar(slot), phase, wc) && wait_bounded(s_free, par, wc);
          if (!ok) break;
          tc_fence_after_sync();
          issue_s(stage(slot));
        }
        // dQ += dS K (the scale comes at the end): A from TMEM, B = K tile MN-major
        ok = wait_bounded(ds_ready, par, wc);
        if (!ok) break;
        tc_fence_after_sync();
        issue_dq<DK, DV>(tDQ, tDP, stage(st), j > 0);
        mma_commit(empty_bar(st));
        if (more) issue_dp(stage(slot) + C::kKBytes);
      }
      mma_commit(acc_done);
    }
  } else {
    // ---------------------------------------------------------------- compute warps
    const int part = warp >> 2;
    const int lane_base = (warp & 3) * 32, row = lane_base + lane;
    const uint32_t lanes = uint32_t(lane_base) << 16;
    const uint32_t tS = tmem + lanes + C::kTmemS + part * kCols;
    const uint32_t tDP = tmem + lanes + C::kTmemDP + part * kCols;
    const float nl = p.nl[tile_id * kBlk + row], dd = p.delta[tile_id * kBlk + row];
    const uint64_t cc = pack_f32x2(p.c_log2, p.c_log2), nn = pack_f32x2(nl, nl);
    const RowAt at = row_at(p, t, row);
    const int g = at.g, i = at.i;
    const bool live = at.real;
    // rows that are not there weigh nothing anyway (their nl)
    const int lim = live ? win::row_end(p.mask, p.Nk, p.N, i) : 0x7fffffff, low = live ? win::row_low(p.mask, p.Nk, p.N, i) : 0;
    bool ok = true;
    auto wait_warp = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, wait_bounded(bar, parity, wc)) != 0; };
    for (int j = 0; ok && j < n_kt; ++j) {
      const uint32_t par = uint32_t(j) & 1u;
      ok = wait_bounded(s_full, par, wc);
      tc_fence_after_sync();
      uint32_t r[kCols];
      tmem_load_part<kCols>(tS, r);
      tc_fence_before_sync();
      mbar_arrive(s_free);
      const int n0 = list.at(j0 + j) * C::kN + part * kCols;
      float w[kCols];
#pragma unroll
      for (int k = 0; k < kCols; k += 2) ffma2(w[k], w[k + 1], __uint_as_float(r[k]), __uint_as_float(r[k + 1]), cc, nn);
      if (!__all_sync(0xffffffffu, lim - n0 >= kCols && (n0 >= low || n0 + kCols <= p.mask.sinks))) {
#pragma unroll
        for (int k = 0; k < kCols / 32; ++k) {
          const uint32_t bits = below(lim - n0, k) & (~below(low - n0, k) | below(p.mask.sinks - n0, k));
#pragma unroll
          for (int e = 0; e < 32; ++e) w[32 * k + e] = bits >> e & 1u ? w[32 * k + e] : -INFINITY;
        }
      }
#pragma unroll
      for (int k = 0; k < kCols; ++k) w[k] = ex2_approx(w[k]);
      ok = wait_bounded(dp_full, par, wc) && ok;
      tc_fence_after_sync();
      uint32_t pk[kCols / 2];
      tmem_each_32<kCols>(tDP, r, [&](int c) {
#pragma unroll
        for (int k = c; k < c + 32; k += 2)
          pk[k >> 1] = pack_bf16x2(w[k] * (__uint_as_float(r[k]) - dd), w[k + 1] * (__uint_as_float(r[k + 1]) - dd));
      });
      tmem_store_part<kCols>(tDP, pk);
      tmem_wait_st();
      tc_fence_before_sync();
      mbar_arrive(ds_ready);
      ok = __all_sync(0xffffffffu, ok);
    }
    // part q writes columns [wq q, wq q + wq)
    constexpr int wq = DK / kParts;
    {
      __nv_bfloat16* dst = row_of(p.dq, t.b, t.h * p.G + (live ? g : 0), live ? i : 0) + part * wq;
      if (n_kt == 0) {
        if (live)
          for (int e = 0; e < wq / 8; ++e) reinterpret_cast<uint4*>(dst)[e] = make_uint4(0, 0, 0, 0);
      } else if (ok && wait_warp(acc_done, 0)) {
        tc_fence_after_sync();
        bad = !store_row<wq>(tmem + lanes + C::kTmemDQ + part * wq, p.scale, dst,
                             p.q_pieces > 1 ? p.part_q + ((tile_id * p.q_pieces + piece) * kBlk + row) * DK + part * wq : nullptr, live);
      }
    }
  }

  if (warp == kMmaWarp && lane == 0) wait_quiesce(acc_done, 0, p.wait_limit_ns, &g_moa_window_bwd_status);
  tc_fence_before_sync();
  if (__syncthreads_or(bad)) {
    const bool dead = *abort_flag != 0;
    if (threadIdx.x == 0) {
      mbar_init(acc_done + 16, 1);
      mbar_init(acc_done + 16 + 8, 1);
      fence_barrier_init();
    }
    __syncthreads();
    if (!dead && warp < kMmaWarp) {
      tc_fence_after_sync();
      dq_again<DK, DV>(&tmK, &tmV, p, index, smem, tmem);
    }
    tc_fence_before_sync();
    __syncthreads();
  }
  if (warp == kMmaWarp) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, C::kTmemCols);
  }
}

// Adds the pieces of dQ's tiles: four features of a row a thread.
template <int DK, int DV>
__global__ void __launch_bounds__(256)
window_dq_tc_join_kernel(const Params p, int64_t n) {
  wait_for_previous();
  const int64_t x = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (x >= n) return;
  const int64_t row = x / (DK / 4), pair = row / kBlk;
  const int c = int(x - row * (DK / 4)) * 4, r = int(row - pair * kBlk);
  const RowTile t = row_tile(p, pair);
  const RowAt at = row_at(p, t, r);
  if (!at.real) return;
  const int i1 = t.i0 + 2 * p.PT - 1 < p.N ? t.i0 + 2 * p.PT - 1 : p.N - 1;
  const int tiles = win::tiles_of(p.mask, p.Nk, p.N, t.i0, i1, width_of(DK, DV)).n;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i = 0; i < p.q_pieces; ++i) {
    if (int64_t(tiles) * i / p.q_pieces == int64_t(tiles) * (i + 1) / p.q_pieces) continue;   // an empty piece
    const float4 v = *reinterpret_cast<const float4*>(p.part_q + ((pair * p.q_pieces + i) * kBlk + r) * DK + c);
    s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
  }
  *reinterpret_cast<uint2*>(row_of(p.dq, t.b, t.h * p.G + at.g, at.i) + c) =
      make_uint2(pack_bf16x2(s.x * p.scale, s.y * p.scale), pack_bf16x2(s.z * p.scale, s.w * p.scale));
}

// CTAs below n_kv: dK and dV; the others: dQ, which are shorter and fill the SMs that run out of the former.
template <int DK, int DV>
__global__ void __launch_bounds__(kThreads, ctas_of(DK, DV))
window_bwd_tc_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                     const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CUtensorMap tmG,
                     const __grid_constant__ Params p, unsigned n_kv) {
  wait_for_previous();
  if (blockIdx.x < n_kv)
    dkdv_tile<DK, DV>(tmQ, tmK, tmV, tmG, p, blockIdx.x);
  else
    dq_tile<DK, DV>(tmQ, tmK, tmV, tmG, p, blockIdx.x - n_kv);
}

// ------------------------------------------------------------------------------------------------
// Host side
// ------------------------------------------------------------------------------------------------
constexpr int kSms = 152;   // the pieces aim at two CTAs for each SM; results do not go by the device's count

struct Plan {
  int64_t GC, chunks, PT, n_ht, n_kt, pairs;   // pairs of halves
  int64_t cut, pieces, piece, items, q_pieces;
  explicit Plan(const WindowBwdArgs& a) {
    const int64_t G = a.Hq / a.Hk, bh = a.B * a.Hk;
    chunks = (G + kHalf - 1) / kHalf;
    GC = (G + chunks - 1) / chunks;
    PT = kHalf / GC;
    n_ht = (a.Nq + 2 * PT - 1) / (2 * PT) * 2;
    n_kt = (a.Nk + kBlk - 1) / kBlk;
    pairs = bh * chunks * (n_ht / 2);
    const win::Mask m{a.window, a.sinks, true};
    // positions of the row tiles that dK's and dV's CTAs step by, and those tiles along the positions
    const int64_t step = width_of(a.dk, a.dv) / kHalf * PT, n_pt = (a.Nq + step - 1) / step;
    // row tiles of a token tile: the most of any, and of one without sinks
    const int64_t top = rows_of_tokens(m, 0, int(a.Nq), int(a.Nk), int(step)).n * chunks;
    const int64_t sink_tiles = a.window == win::kNoWindow ? 0 : (int64_t(a.sinks) + kBlk - 1) / kBlk;
    int64_t usual = top;
    if (a.window != win::kNoWindow) {
      usual = (int64_t(a.window) + kBlk + 2 * step - 1) / step * chunks;
      if (usual > top) usual = top;
    }
    piece = usual;
    cut = sink_tiles;
    if (n_kt * bh < 2 * kSms) {   // too few token tiles for the machine: all are cut
      int64_t total = 0;
      for (int64_t t = 0; t < n_kt; ++t) total += rows_of_tokens(m, int(t), int(a.Nq), int(a.Nk), int(step)).n * chunks;
      const int64_t want = (total * bh + 2 * kSms - 1) / (2 * kSms);
      if (want < usual) {
        piece = want;
        cut = n_kt;
      }
    }
    if (piece < 4) piece = 4;
    if (cut > n_kt) cut = n_kt;
    // not more pieces than keep the machine busy: each is 128 rows of fp32 in the workspace (160 MB in all)
    const int64_t most = cut > 0 && bh * cut < 8 * kSms ? 8 * kSms / (bh * cut) : 1;
    if ((chunks * n_pt + piece - 1) / piece > most) piece = (chunks * n_pt + most - 1) / most;
    pieces = (chunks * n_pt + piece - 1) / piece;
    if (pieces <= 1) cut = 0, pieces = 1;
    items = bh * (cut * pieces + n_kt - cut);
    // dQ's tiles: pieces of four token tiles at least, until there are two CTAs for each SM
    const int64_t width = width_of(a.dk, a.dv);
    int64_t tiles = (a.Nk + width - 1) / width;
    if (a.window != win::kNoWindow) {
      const int64_t seen = (int64_t(a.window) + 2 * PT + a.sinks + 3 * width) / width;
      if (seen < tiles) tiles = seen;
    }
    q_pieces = (2 * kSms + pairs - 1) / pairs;
    if (q_pieces > tiles / 4) q_pieces = tiles / 4;
    if (q_pieces < 1 || pairs >= kSms) q_pieces = 1;
  }
};

// The workspace: -LSE log2 e and D of every row of every half, then the pieces.
struct Work {
  int64_t nl, delta, part, part_q, bytes;
  Work(const WindowBwdArgs& a, const Plan& p) {
    nl = 0;
    delta = p.pairs * kBlk * 4;
    part = 2 * delta;
    part_q = part + a.B * a.Hk * p.cut * p.pieces * kBlk * (a.dk + a.dv) * 4;
    bytes = part_q + (p.q_pieces > 1 ? p.pairs * p.q_pieces * kBlk * a.dk * 4 : 0);
  }
};

template <int DK, int DV>
int launch(const WindowBwdArgs& a, char* msg, size_t msglen) {
  using CK = KvCfg<DK, DV>;
  using CQ = QCfg<DK, DV>;
  auto kern = window_bwd_tc_kernel<DK, DV>;
  constexpr int kSmem = CK::kSmemBytes > CQ::kSmemBytes ? CK::kSmemBytes : CQ::kSmemBytes;
  cudaError_t e = ensure_smem_limit(reinterpret_cast<const void*>(kern), kSmem);
  const Plan plan(a);
  const Work w(a, plan);
  uint8_t* ws = static_cast<uint8_t*>(a.ws);
  const int64_t G = a.Hq / a.Hk, bh = a.B * a.Hk;
  Params p{};
  p.q = a.q, p.k = a.k, p.v = a.v, p.o = a.o, p.go = a.go, p.dq = a.dq, p.dk = a.dk_, p.dv = a.dv_;
  p.lse = a.lse;
  p.nl = reinterpret_cast<float*>(ws + w.nl);
  p.delta = reinterpret_cast<float*>(ws + w.delta);
  p.part = reinterpret_cast<float*>(ws + w.part);
  p.part_q = reinterpret_cast<float*>(ws + w.part_q);
  p.q_pieces = int(plan.q_pieces);
  p.B = int(a.B), p.Hk = int(a.Hk), p.G = int(G), p.N = int(a.Nq), p.Nk = int(a.Nk);
  p.GC = int(plan.GC), p.chunks = int(plan.chunks), p.PT = int(plan.PT);
  p.n_ht = int(plan.n_ht), p.n_kt = int(plan.n_kt);
  p.cut = int(plan.cut), p.pieces = int(plan.pieces), p.piece = int(plan.piece);
  // as many key heads side by side as leave their queries and output gradients in L2
  const int64_t head = a.Nq * G * (DK + DV) * 2;
  p.group = int((int64_t(48) << 20) / head < 1 ? 1 : (int64_t(48) << 20) / head > bh ? bh : (int64_t(48) << 20) / head);
  p.mask = win::Mask{a.window, a.sinks, true};
  p.c_log2 = a.scale * kLog2e, p.scale = a.scale;
  p.wait_limit_ns = wait_limit_ns();
  CUtensorMap mq, mk, mv, mg;
  const uint64_t q_dims[5] = {DK, uint64_t(G), uint64_t(a.Nq), uint64_t(a.Hk), uint64_t(a.B)};
  const uint64_t g_dims[5] = {DV, uint64_t(G), uint64_t(a.Nq), uint64_t(a.Hk), uint64_t(a.B)};
  const uint64_t q_str[4] = {map_stride(a.q.sh, G), map_stride(a.q.sn, a.Nq), map_stride(G * a.q.sh, a.Hk), map_stride(a.q.sb, a.B)};
  const uint64_t g_str[4] = {map_stride(a.go.sh, G), map_stride(a.go.sn, a.Nq), map_stride(G * a.go.sh, a.Hk),
                             map_stride(a.go.sb, a.B)};
  const uint32_t row_box[5] = {64, uint32_t(plan.GC), uint32_t(plan.PT), 1, 1};
  const uint64_t k_dims[4] = {DK, uint64_t(a.Nk), uint64_t(a.Hk), uint64_t(a.B)};
  const uint64_t v_dims[4] = {DV, uint64_t(a.Nk), uint64_t(a.Hk), uint64_t(a.B)};
  const uint64_t k_str[3] = {map_stride(a.k.sn, a.Nk), map_stride(a.k.sh, a.Hk), map_stride(a.k.sb, a.B)};
  const uint64_t v_str[3] = {map_stride(a.v.sn, a.Nk), map_stride(a.v.sh, a.Hk), map_stride(a.v.sb, a.B)};
  const uint32_t kv_box[4] = {64, width_of(DK, DV), 1, 1};
  if (!encode_bf16_map_nd(&mq, a.q.p, 5, q_dims, q_str, row_box, msg, msglen) ||
      !encode_bf16_map_nd(&mg, a.go.p, 5, g_dims, g_str, row_box, msg, msglen) ||
      !encode_bf16_map_nd(&mk, a.k.p, 4, k_dims, k_str, kv_box, msg, msglen) ||
      !encode_bf16_map_nd(&mv, a.v.p, 4, v_dims, v_str, kv_box, msg, msglen))
    return 5;
  if (e == cudaSuccess)
    e = launch_overlapped(window_delta_tc_kernel<DV>, dim3(unsigned(plan.pairs)), dim3(256), 0, a.stream, p);
  if (e == cudaSuccess)
    e = launch_overlapped(kern, dim3(unsigned(plan.items + plan.pairs * plan.q_pieces)), dim3(kThreads), kSmem, a.stream, mq, mk, mv, mg, p,
                          unsigned(plan.items));
  const int64_t joined = bh * plan.cut * kBlk * ((DK + DV) / 4);
  if (e == cudaSuccess && joined > 0)
    e = launch_overlapped(window_dkdv_tc_join_kernel<DK, DV>, dim3(unsigned((joined + 255) / 256)), dim3(256), 0, a.stream, p,
                          joined);
  const int64_t q_joined = plan.pairs * kBlk * (DK / 4);
  if (e == cudaSuccess && plan.q_pieces > 1)
    e = launch_overlapped(window_dq_tc_join_kernel<DK, DV>, dim3(unsigned((q_joined + 255) / 256)), dim3(256), 0, a.stream, p, q_joined);
  if (e != cudaSuccess) {
    snprintf(msg, msglen, "gradients of attention with a window: %s", cudaGetErrorString(e));
    return 5;
  }
  return 0;
}

}  // namespace

bool window_bwd_tc_takes(const WindowBwdArgs& a) {
  const int64_t G = a.Hq / a.Hk;
  auto rows = [&](const View& x) {
    return describable(x.sh, G) && describable(G * x.sh, a.Hk) && describable(x.sn, a.Nq) && describable(x.sb, a.B);
  };
  auto keys = [&](const View& x) { return describable(x.sn, a.Nk) && describable(x.sh, a.Hk) && describable(x.sb, a.B); };
  return !a.f32 && rows(a.q) && rows(a.go) && keys(a.k) && keys(a.v);
}

size_t window_bwd_tc_workspace(const WindowBwdArgs& a) { return size_t(Work(a, Plan(a)).bytes); }

int launch_window_bwd_tc(const WindowBwdArgs& a, char* msg, size_t msglen) {
  if (a.dk == 64) return a.dv == 64 ? launch<64, 64>(a, msg, msglen) : launch<64, 128>(a, msg, msglen);
  return a.dv == 64 ? launch<128, 64>(a, msg, msglen) : launch<128, 128>(a, msg, msglen);
}

cudaError_t window_bwd_read_and_clear_status(unsigned* value) {
  cudaError_t e = cudaMemcpyFromSymbol(value, g_moa_window_bwd_status, sizeof(unsigned));
  if (e != cudaSuccess || *value == 0) return e;
  const unsigned zero = 0;
  return cudaMemcpyToSymbol(g_moa_window_bwd_status, &zero, sizeof(unsigned));
}

}  // namespace moa
