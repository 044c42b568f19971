// Attention of many query rows over the 4-bit paged cache (a chunk of a prompt) on the
// fifth-generation tensor cores (tcgen05 + TMEM + TMA), sm_103a.
//
// Mathematics: that of kv4_attn.cu (scores, softmax, empty rows, joined pieces).  With many query
// rows the two products are the cost, and each cached token meets every block of 256 query rows:
// so the cache is widened once, by a kernel of its own, into 16-bit keys and values in the
// workspace (read through L2 by all query blocks), instead of once in every block.
//
//   widen    one CTA for 128 tokens of a head.  Keys become fp16: code * scale has at most 3 + 8
//            significant bits, so with the tile's power of two 2^E taken out (E from its largest
//            scale) the products are exact while the scales are within 2^28 of each other; 2^E goes
//            into the tile's softmax factor.  A tile with scales further apart is marked, and its
//            scores are computed from the codes in fp32 instead (exact_scores: 0.3 ms a tile, for keys that
//            a trained model does not have).  Values become bf16, rounded once.  Tokens past the end, and
//            pages that are not there, become zeros (the rows' limits, and a mark beside the factor, hide
//            them).
//            A value group that is not finite gets zeros, and a bit in its block's mask: the rows
//            that see it are made NaN in that group at the end (0 * NaN would reach all rows through the
//            second product).
//   attend   query rows, as fp16 with each row's power of two taken out (members within 2^-31 of the
//            row's largest fit exactly, smaller ones are rounded to 2^-40 of it), against 128-token tiles: S = Q K^T (fp16), running maximum and sum per row, O += P V
//            (bf16) in TMEM.  Maximum, exponentials, sum in fp32.  P and V in fp16 (11 bits, V then
//            exact) would halve the rounding of ordinary rows, but weights below 2^-31 of the largest
//            would be lost, and they are all there is of a feature that the larger ones leave at zero.
//   join     the pieces of cut work items.
//
// Rows of a key head are counted head by head: row r is query r % N of query head r / N of the
// group, so 256 rows are neighbours in position and a causal block ends early.
//
// What bounds it: the second and first products' tensor time and, beside it, a softmax warp's chain of
// score load, maximum, 128 exponentials and stores.  Measured, 2048 causal queries of 32 heads against
// 16384 tokens of 8 key heads, d = 128: 346 us in all in replayed graphs = 1.49 PFLOP/s (measured
// matrix-product rate: 1.89), of them about 315 us the attention, tensor pipe 70 % active, issue 44 %; the
// widening 15 to 20 us, the join the rest.  The attention's time moves by 3 % with the compiler's schedule
// of its softmax loop, whatever else changes: 346 to 362 us in all have been seen of the same loop.
//
// Work items (key head, block of 256 rows) count in units of 128-token tiles; the units of all items
// are cut into equal shares, one for each SM (one CTA fills an SM): with 256 items on 152 SMs whole
// items would leave a sixth of the machine idle.  A CTA walks over the items of its share.
//
// CTA organisation (12 warps): warps 0-3 and 4-7 softmax and epilogue of row tiles 0 and 1 (thread
// = row), warp 8 TMEM allocation and the products of tile 0, warp 9 TMA, warp 10 the products of
// tile 1, warp 11 the share's items, one after another, for the other roles.  TMEM columns: two
// S, P and O at d_v = 64; one S for both tiles at d_v = 128.  K and V tiles stream through a
// shared-memory ring in the order of use, K0 K1 V0 K2 V1 ...
// Waits are bounded: on expiry MOA_ERR_DEVICE_TIMEOUT is recorded and every role leaves its loop.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cfloat>
#include <cstdio>

#include "internal.h"
#include "kv4.cuh"
#include "ops_internal.h"
#include "ptx.cuh"
#include "tc_common.cuh"

namespace moa {

__device__ unsigned int g_moa_kv4_tc_status = 0;

namespace {

using namespace kv4;
using namespace ptx;
using namespace tc;

constexpr int kBM = 128;              // query rows of a row tile (= TMEM lanes)
constexpr int kRows = 2 * kBM;        // query rows of a work item
constexpr int kBN = 128;              // tokens of a tile
// A work item costs about as much as this many tiles besides its own (queries, the pipeline's filling,
// its output): it counts for that many more, which come first and hold no tokens (256 items of 128 tiles:
// 357 us with 0, 355 with 4 and 8; it matters more to short items).
constexpr int kItemUnits = 4;
constexpr int kThreads = 384;
constexpr int kMmaWarp0 = 8, kLoadWarp = 9, kMmaWarp1 = 10, kWalkWarp = 11;
constexpr float kRescaleLog2 = 8.f;   // the running maximum may lag by this: weights up to 2^8
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

template <int DK, int DV>
struct Cfg {
  // 256 kRegsSoftmax + 128 kRegsCtrl is what the launch allocates (the host checks it).  At 168 registers
  // the compiler spills 8 to 20 bytes, which it reloads in many places
  static constexpr int kRegsLaunch = 168, kRegsSoftmax = 208, kRegsCtrl = 88;
  static_assert(256 * kRegsSoftmax + 128 * kRegsCtrl <= kThreads * kRegsLaunch, "register split");
  static constexpr int kPanelBytes = 128 * 128;   // 64 columns of 128 rows, 128-byte swizzle
  static constexpr int kQTileBytes = kBM * DK * 2;
  static constexpr int kKTileBytes = kBN * DK * 2, kVTileBytes = kBN * DV * 2;
  static constexpr int kStageBytes = kKTileBytes > kVTileBytes ? kKTileBytes : kVTileBytes;
  static constexpr bool kSharedS = DV == 128;
  static constexpr int kStages = DK == 64 ? (DV == 64 ? 8 : 6) : (DV == 64 ? 4 : 5);
  static constexpr int kOffKV = 2 * kQTileBytes;
  static constexpr int kOffBar = kOffKV + kStages * kStageBytes;
  // barriers: full[NS], empty[NS], q_full, s_full[2], p_ready[2], o_done[2], s_free[2], p_free[2], drain,
  // item_full[2], item_empty[2]
  static constexpr int kNumBars = 2 * kStages + 16;
  static constexpr int kOffMisc = kOffBar + kNumBars * 8;
  static constexpr int kOffItems = (kOffMisc + 8 + 15) / 16 * 16;    // two items, then scan[12] and found[2]
  static constexpr int kSmemBytes = kOffItems + 2 * 16 + 14 * 8 + 1024;
  // exponentials, in chunks of 32 tokens, before the wait for the buffer of P: 2, 3, 4 of 4 at d_v = 128 363, 356,
  // 354 us (the chunk above); at 64 one to four 283, 279, 278, 278 us
  static constexpr int kEarlyChunks = DV == 64 ? 2 : 4;
  static constexpr uint32_t kTmemCols = 512;
  static constexpr uint32_t kTmemS0 = 0, kTmemS1 = kSharedS ? 0 : 128;
  static constexpr uint32_t kTmemP0 = kSharedS ? 128 : 256, kTmemP1 = kSharedS ? 192 : 320;
  static constexpr uint32_t kTmemO0 = kSharedS ? 256 : 384, kTmemO1 = kTmemO0 + DV;
  static_assert(kTmemO1 + DV <= kTmemCols, "TMEM budget");
  static_assert(kSmemBytes <= 232448, "shared memory budget");
};

struct Params {
  int64_t q_sb, q_sh, q_sn, o_sb, o_sh, o_sn;
  int64_t n_pages, max_pages;
  int N, max_len;
  int Hk, G, blocks_per_page;
  int bh0, n_bh;       // the heads (b * Hk + h) of this launch
  int n_tiles;         // work items of a head
  int tiles_pad;       // 128-token tiles of a head in the workspace
  float c_log2;        // |scale| log2 e
  bool negate, causal;
  uint64_t wait_limit_ns;
};

__device__ __forceinline__ int length_of(const int32_t* lens, int b, const Params& p, bool report) {
  const int len = lens[b];
  if (len >= 0 && len <= p.max_len) return len;
  if (report) atomicExch(&g_moa_kv4_tc_status, kErrIndex);
  return len < 0 ? 0 : p.max_len;
}
__device__ __forceinline__ int limit_of(int len, int i, const Params& p) {
  if (!p.causal) return len;
  const int n = len - p.N + i + 1;
  return n < 0 ? 0 : n;
}
// Tiles that work item `item` sees: at least one, so that every item is written.
__device__ __forceinline__ int units_of(const int32_t* lens, int item, const Params& p, bool report) {
  const int bh = int(unsigned(item) / unsigned(p.n_tiles)), r0 = (item - bh * p.n_tiles) * kRows;
  const int rows = p.N * p.G, r1 = r0 + kRows < rows ? r0 + kRows : rows;
  const int first = int(unsigned(r0) / unsigned(p.N)), last = int(unsigned(r1 - 1) / unsigned(p.N));
  // the latest query of the rows: the last of a head if they reach into the next one
  const int i = first != last ? p.N - 1 : r1 - 1 - first * p.N;
  const int n = limit_of(length_of(lens, int(unsigned(p.bh0 + bh) / unsigned(p.Hk)), p, report), i, p);
  return n <= kBN ? 1 : (n + kBN - 1) / kBN;
}

// Equal shares of `total` units: share c begins at start(c).
struct Shares {
  int64_t each;
  uint32_t rest, n;
  __device__ __forceinline__ Shares(int64_t total, uint32_t ctas) {
    n = total < ctas ? uint32_t(total) : ctas;
    each = total / n;
    rest = uint32_t(total - each * n);
  }
  __device__ __forceinline__ int64_t start(uint32_t c) const { return each * c + rest * c / n; }
};

// An item cut by CTA c's share, begun by it and not ended: its pieces lie with CTAs c, c + 1, ...
struct Cut {
  int item;
  int pieces;   // 0: none
};

// ------------------------------------------------------------------------------------------------
// Widening
// ------------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  const __half2 x = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&x);
}
__device__ __forceinline__ float bf16_value(const uint8_t* p) {
  return __uint_as_float(uint32_t(*reinterpret_cast<const uint16_t*>(p)) << 16);
}

// 2^e, -126 <= e <= 127, and the exponent that brings a largest scale (its bits) into [2^to, 2^(to + 1)).
__device__ __forceinline__ float power_of(int e) { return __uint_as_float(uint32_t(127 + e) << 23); }
__device__ __forceinline__ int tile_exponent(uint32_t top, int to) {
  return top == 0 ? 0 : max(int(top >> 23) - 127 - to, -126);
}
// Of tiles with scales far apart: room for queries below 2^15, codes and 128 products above, and for
// scales down to 2^-186 of the largest below.
constexpr int kMixedTop = 60;
// The power of two that a row's largest magnitude (its bf16 bits) is brought into [2^14, 2^15) by.
__device__ __forceinline__ int row_exponent(uint32_t top) {
  return top == 0 || top >= 0x7f80u ? 0 : max(int(top >> 7) - 127 - 14, -126);
}

// What a tile's factor carries beside its power of two: a bit for each 16-token block whose page is not
// there, whether the tile's scores have to be computed in fp32, and whether a value is not finite (the
// blocks' masks are only written then).
constexpr uint32_t kGoneBlocks = 0xffu, kMixedKeys = 0x100u, kBadValues = 0x200u;

// Bound by its stores into L2 and the latency of a warp's one block: 2304 bytes in, 8 KB out.  Words
// asked for before the scales are looked at, and products in pairs: 5 us less than one after the other
// (128 tiles of 8 heads, of 355 us).
template <int DK, int DV>
__global__ void __launch_bounds__(256)
kv4_widen_kernel(const uint8_t* pool, const int32_t* table,
                 const int32_t* lens, __half* __restrict__ wk, __nv_bfloat16* __restrict__ wv,
                 float2* __restrict__ factor, uint64_t* __restrict__ bad_values, Params p) {
  constexpr int GK = DK / 32, GV = DV / 32;
  __shared__ uint32_t s_max[8], s_min[8], s_marks[8];
  wait_for_previous();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int tile = int(blockIdx.x), bh = int(blockIdx.y);
  const int b = int(unsigned(p.bh0 + bh) / unsigned(p.Hk)), h = p.bh0 + bh - b * p.Hk;
  const int len = length_of(lens, b, p, tile == 0 && threadIdx.x == 0);
  if (tile > 0 && tile * kBN >= len) return;
  // warp w: the tile's block w
  const int blk = tile * (kBN / kBlock) + warp;
  const uint8_t* src = nullptr;
  if (blk * kBlock < len) {
    const int slot = int(unsigned(blk) / unsigned(p.blocks_per_page));
    const int pg = table[b * p.max_pages + slot];
    if (pg >= 0 && pg < p.n_pages)
      src = pool + ((int64_t(pg) * p.Hk + h) * p.blocks_per_page + (blk - slot * p.blocks_per_page)) * block_bytes(DK, DV);
    else if (lane == 0)
      atomicExch(&g_moa_kv4_tc_status, kErrIndex);
  }
  const int n_tok = src == nullptr ? 0 : min(kBlock, len - blk * kBlock);
  // the lane's words, on their way while the scales are looked at.  Keys: a word is eight neighbouring
  // features of a token.  Values: two words are eight neighbouring features of two tokens.
  constexpr int kChunks = DK / 8, kChunksV = DV / 8, kItsK = kBlock * kChunks / 32, kItsV = kBlock / 2 * kChunksV / 32;
  uint32_t kw[kItsK], vw[kItsV][2];
#pragma unroll
  for (int it = 0; it < kItsK; ++it) {
    const int i = it * 32 + lane, token = i / kChunks, f8 = i % kChunks;
    kw[it] = token < n_tok ? *reinterpret_cast<const uint32_t*>(src + key_word(token, f8 & 3, f8 >> 2, GK)) : 0x88888888u;
  }
#pragma unroll
  for (int it = 0; it < kItsV; ++it) {
    const int i = it * 32 + lane, token = 2 * (i / kChunksV), f8 = i % kChunksV;
#pragma unroll
    for (int k = 0; k < 2; ++k)
      vw[it][k] = token < n_tok ? *reinterpret_cast<const uint32_t*>(src + value_word(DK, token, (f8 & 3) * 2 + k, f8 >> 2, GV))
                                : 0x88888888u;
  }
  // the largest and the smallest key scale that is a number and not zero (their bits are in the same
  // order), and the value groups that are not finite: bit GV token + group
  uint32_t top_bits = 0, low_bits = 0x7f800000u;
  uint64_t bad = 0;
  bool huge = false;   // a value may round to infinity: seven times the largest scale there is, 1.140625 * 2^125
  if (src != nullptr) {
    for (int i = lane; i < kBlock * GK; i += 32) {
      const float s = bf16_value(src + key_scales(DK, DV) + 2 * i);
      if (i / GK < n_tok && s > 0.f && s < INFINITY)
        top_bits = max(top_bits, __float_as_uint(s)), low_bits = min(low_bits, __float_as_uint(s));
    }
#pragma unroll
    for (int i = 0; i < kBlock * GV; i += 32) {
      const float s = bf16_value(src + value_scales(DK, DV) + 2 * (i + lane));
      bad |= uint64_t(__ballot_sync(0xffffffffu, (i + lane) / GV < n_tok && !(s < INFINITY))) << i;
      huge |= s >= 0x1.24p125f;
    }
  }
  huge = __any_sync(0xffffffffu, huge);
  top_bits = __reduce_max_sync(0xffffffffu, top_bits);
  low_bits = __reduce_min_sync(0xffffffffu, low_bits);
  if (lane == 0) {
    s_max[warp] = top_bits;
    s_min[warp] = low_bits;
    s_marks[warp] = (src == nullptr && blk * kBlock < len ? 1u << warp : 0u) | (bad != 0 ? kBadValues : 0u);
  }
  __syncthreads();
  uint32_t marks = 0;
#pragma unroll
  for (int w = 0; w < 8; ++w) {
    top_bits = max(top_bits, s_max[w]);
    low_bits = min(low_bits, s_min[w]);
    marks |= s_marks[w];
  }
  // 2^E with the largest scale times 2^-E in [2^11, 2^12); eight bits of a scale then end above 2^-24, the
  // spacing of the smallest fp16, if it is 2^-17 or more
  const int e = tile_exponent(top_bits, 11);
  const float down = power_of(-e);
  const bool mixed = low_bits < 0x7f800000u && __uint_as_float(low_bits) * down < 0x1p-17f;
  if (mixed) marks |= kMixedKeys;
  const int64_t at = int64_t(bh) * p.tiles_pad + tile;
  if (threadIdx.x == 0)
    factor[at] = make_float2(power_of(mixed ? tile_exponent(top_bits, kMixedTop) : e), __uint_as_float(marks));
  if ((marks & kBadValues) && lane == 0) bad_values[at * 8 + warp] = bad;

  const int64_t row0 = at * kBN + warp * kBlock;
#pragma unroll
  for (int it = 0; it < kItsK; ++it) {
    const int i = it * 32 + lane, token = i / kChunks, f8 = i % kChunks, g = f8 >> 2;
    float s = 0.f;
    if (token < n_tok) s = bf16_value(src + key_scales(DK, DV) + (token * GK + g) * 2) * down;
    // codes as 1024 + n, less 1032
    const __half2 s2 = __float2half2_rn(s), bias = __float2half2_rn(1032.f);
    uint32_t o[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t x = (kw[it] >> (4 * j) & 0x000f000fu) | 0x64006400u;
      const __half2 y = __hmul2(__hsub2(*reinterpret_cast<const __half2*>(&x), bias), s2);
      o[j] = *reinterpret_cast<const uint32_t*>(&y);
    }
    *reinterpret_cast<uint4*>(wk + (row0 + token) * DK + f8 * 8) = make_uint4(o[0], o[1], o[2], o[3]);
  }
#pragma unroll
  for (int it = 0; it < kItsV; ++it) {
    const int i = it * 32 + lane, f8 = i % kChunksV, g = f8 >> 2, token = 2 * (i / kChunksV);
    uint32_t s = 0;   // the two tokens' scales
#pragma unroll
    for (int k = 0; k < 2; ++k)
      if (token + k < n_tok && !(bad >> (GV * (token + k) + g) & 1u))
        s |= uint32_t(*reinterpret_cast<const uint16_t*>(src + value_scales(DK, DV) + ((token + k) * GV + g) * 2)) << (16 * k);
    const __nv_bfloat162 s2 = *reinterpret_cast<const __nv_bfloat162*>(&s), bias = __float2bfloat162_rn(136.f);
    uint32_t y[8];   // a feature of both tokens: codes as 128 + n, less 136; the product is rounded once
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t x = (vw[it][j >> 2] >> (4 * (j & 3)) & 0x000f000fu) | 0x43004300u;
      __nv_bfloat162 z = __hmul2(__hsub2(*reinterpret_cast<const __nv_bfloat162*>(&x), bias), s2);
      if (huge) {   // the largest number instead, half a unit away: infinity times a hidden token's zero is NaN
        const __nv_bfloat162 most = __halves2bfloat162(__ushort_as_bfloat16(0x7f7f), __ushort_as_bfloat16(0x7f7f));
        z = __hmax2(__hmin2(z, most), __hneg2(most));
      }
      y[j] = *reinterpret_cast<const uint32_t*>(&z);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      uint32_t o[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = __byte_perm(y[2 * j], y[2 * j + 1], k ? 0x7632 : 0x5410);
      *reinterpret_cast<uint4*>(wv + (row0 + token + k) * DV + f8 * 8) = make_uint4(o[0], o[1], o[2], o[3]);
    }
  }
}

// ------------------------------------------------------------------------------------------------
// Attention
// ------------------------------------------------------------------------------------------------
// Maximum of 128 values with four independent 3-input chains.
__device__ __forceinline__ float row_max128(const float* s) {
  float a0 = s[0], a1 = s[1], a2 = s[2], a3 = s[3];
#pragma unroll
  for (int i = 4; i < 124; i += 8) {
    a0 = max3f(a0, s[i], s[i + 1]);
    a1 = max3f(a1, s[i + 2], s[i + 3]);
    a2 = max3f(a2, s[i + 4], s[i + 5]);
    a3 = max3f(a3, s[i + 6], s[i + 7]);
  }
  a0 = max3f(a0, s[124], s[125]);
  a1 = max3f(a1, s[126], s[127]);
  return max3f(a0, a1, fmaxf(a2, a3));
}

// Multiplies DV fp32 TMEM columns of this thread's lane by alpha (warp-collective).
template <int DV>
__device__ __forceinline__ void tmem_scale_row(uint32_t taddr, float alpha) {
#pragma unroll
  for (int c = 0; c < DV; c += 32) {
    uint32_t o[32];
    tmem_ld_32x32b_x32(taddr + c, o);
    tmem_wait_ld();
    reg_anchor_x32(o);
#pragma unroll
    for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
    tmem_st_32x32b_x32(taddr + c, o);
  }
  tmem_wait_st();
}

// Instruction descriptor of tcgen05.mma kind::f16 with fp16 operands (format 0), both K-major.
__host__ __device__ constexpr uint32_t make_idesc_f16(int M, int N) {
  return (1u << 4) | (uint32_t(N >> 3) << 17) | (uint32_t(M >> 4) << 24);
}

// A thread's query row and where its head's codes lie.
struct Codes {
  const __nv_bfloat16* q;   // null: no row
  const uint8_t* pool;      // the head's place in page 0
  const int32_t* pages;     // of the sequence
  int64_t page_bytes, n_pages;
  int blocks_per_page, len;
  float sign;               // of the scale
  const uint64_t* bad;      // the masks of value groups that are not finite, of the sequence's blocks
};

// The value groups that are not finite in the first `valid` tokens of a tile, from its blocks' masks.
template <int GV>
__device__ uint32_t bad_groups(const uint64_t* bad, int valid) {
  uint64_t all = 0;
  for (int k = 0; k < kBN / kBlock; ++k) {
    const int bits = GV * min(max(valid - k * kBlock, 0), kBlock);
    all |= bits == 64 ? bad[k] : bad[k] & ((uint64_t(1) << bits) - 1);
  }
#pragma unroll
  for (int d = 32; d >= GV; d >>= 1) all |= all >> d;
  return uint32_t(all) & ((1u << GV) - 1);
}

// The scores of a thread's row against a tile whose key scales lie too far apart for fp16, into its TMEM
// lane (warp-collective), in fp32 from the cache's codes: the row with its power of two taken out, as in
// the product, the scales times `down`.  Tokens that are not there get zeros; the caller hides them.
template <int DK, int DV>
__device__ void exact_scores(uint32_t tS, const Codes& a, int tile, float down) {
  constexpr int GK = DK / 32;
  uint32_t top = 0;
  for (int i = 0; a.q != nullptr && i < DK; ++i)
    top = max(top, uint32_t(reinterpret_cast<const uint16_t*>(a.q)[i]) & 0x7fffu);
  const float row_down = top >= 0x7f80u ? __int_as_float(0x7fc00000) : power_of(-row_exponent(top)) * a.sign;
#pragma unroll 1
  for (int k = 0; k < kBN / kBlock; ++k) {
    const int blk = tile * (kBN / kBlock) + k, slot = int(unsigned(blk) / unsigned(a.blocks_per_page));
    const int pg = blk * kBlock < a.len ? a.pages[slot] : -1;
    float s[kBlock];
#pragma unroll
    for (int u = 0; u < kBlock; ++u) s[u] = 0.f;
    if (a.q != nullptr && pg >= 0 && pg < a.n_pages) {
      const uint8_t* src = a.pool + pg * a.page_bytes + (blk - slot * a.blocks_per_page) * block_bytes(DK, DV);
#pragma unroll 1
      for (int g = 0; g < GK; ++g) {
        float part[kBlock];
#pragma unroll
        for (int u = 0; u < kBlock; ++u) part[u] = 0.f;
#pragma unroll 1
        for (int t = 0; t < 4; ++t) {
          float x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = __bfloat162float(a.q[32 * g + 8 * t + e]) * row_down;
#pragma unroll
          for (int u = 0; u < kBlock; ++u) {
            const uint32_t w = *reinterpret_cast<const uint32_t*>(src + key_word(u, t, g, GK));
#pragma unroll
            for (int e = 0; e < 8; ++e)
              part[u] += x[e] * float(int(w >> (16 * (e & 1) + 4 * (e >> 1)) & 15u) - 8);
          }
        }
#pragma unroll
        for (int u = 0; u < kBlock; ++u) s[u] += part[u] * (bf16_value(src + key_scales(DK, DV) + (u * GK + g) * 2) * down);
      }
    }
    uint32_t r[kBlock];
#pragma unroll
    for (int u = 0; u < kBlock; ++u) r[u] = __float_as_uint(s[u]);
    __syncwarp();
    tmem_st_32x32b_x16(tS + kBlock * k, r);
  }
  tmem_wait_st();
}

// What a softmax thread of row tile j works with in an item: its lane of the TMEM buffers, barriers, the
// tiles' factors from the sequence's first on, the tokens that its row sees, its tiles, its row's factor.
struct Tiles {
  uint32_t tS, tO, tP;
  uint32_t s_full, s_free, p_ready, p_free;
  const float2* fac;
  int lim, u0, u1;
  float c_row;
};

// The softmax of an item's tiles: maximum m and sum l of the thread's row.  `t`: the tiles of the CTA
// before them.  ODD: some carry marks; `bad`: the value groups that make the row NaN.  False if a wait
// ran out.
template <int DK, int DV, bool ODD>
__device__ __forceinline__ bool item_tiles(const Tiles& x, const Codes* codes, uint32_t t, float& m, float& l,
                                           [[maybe_unused]] uint32_t& bad, const WaitCtl& wc) {
  using C = Cfg<DK, DV>;
  float2 f_next = x.fac[x.u0];
  for (int n = x.u0; n < x.u1; ++n, ++t) {
    const float c = fmaxf(x.c_row * f_next.x, FLT_MIN);   // not zero: c * -infinity hides a token
    const uint32_t marks = ODD ? __float_as_uint(f_next.y) : 0;
    [[maybe_unused]] const float up = f_next.x;
    if (n + 1 < x.u1) f_next = x.fac[n + 1];
    if (!wait_bounded(x.s_full, t & 1u, wc)) return false;
    tc_fence_after_sync();
    if constexpr (ODD) {
      if (marks & kMixedKeys) exact_scores<DK, DV>(x.tS, *codes, n, 1.f / up);
      if (marks & kBadValues) bad |= bad_groups<DV / 32>(codes->bad + n * int64_t(kBN / kBlock), x.lim - n * kBN);
    }
    uint32_t sr[128];
    tmem_load_row128(x.tS, sr);
    tc_fence_before_sync();
    mbar_arrive(x.s_free);
    float* s = reinterpret_cast<float*>(sr);
    const int valid = x.lim - n * kBN;   // of this row
    const bool full = __all_sync(0xffffffffu, valid >= kBN) && marks == 0;
    if (!full) {   // hidden tokens: -infinity, and the rest is the same code
#pragma unroll
      for (int i = 0; i < kBN; ++i) s[i] = i < valid && !(marks & kGoneBlocks & 1u << i / kBlock) ? s[i] : -INFINITY;
    }
    const float m_tile = c * row_max128(s);
    bool rescale = false;   // warp-uniform
    float alpha = 1.f;
    if (n == x.u0) {
      m = m_tile;
    } else if (__any_sync(0xffffffffu, m_tile > m + kRescaleLog2)) {
      const float m_new = fmaxf(m, m_tile);
      alpha = m == -INFINITY ? 0.f : ex2_approx(m - m_new);
      l *= alpha;
      m = m_new;
      rescale = true;
    }
    const float base = m == -INFINITY ? 0.f : m;
    const uint64_t cc = pack_f32x2(c, c);
    const uint64_t mm = pack_f32x2(-base, -base);
    float l0 = 0.f, l1 = 0.f, l2 = 0.f, l3 = 0.f;
    auto exp_chunk = [&](int ch, uint32_t* pk) {
#pragma unroll
      for (int i = 0; i < 32; i += 4) {
        const int k = 32 * ch + i;
        float x0, x1, x2, x3;
        ffma2(x0, x1, s[k], s[k + 1], cc, mm);
        ffma2(x2, x3, s[k + 2], s[k + 3], cc, mm);
        const float p0 = ex2_approx(x0), p1 = ex2_approx(x1), p2 = ex2_approx(x2), p3 = ex2_approx(x3);
        fadd2(l0, l1, p0, p1);
        fadd2(l2, l3, p2, p3);
        pk[i >> 1] = pack_bf16x2(p0, p1);
        pk[(i >> 1) + 1] = pack_bf16x2(p2, p3);
      }
    };
    auto store_chunk = [&](int ch, const uint32_t* pk) { tmem_st_32x32b_x16(x.tP + 16 * ch, pk); };
    constexpr int kEarly = C::kEarlyChunks;
    uint32_t pe[16 * kEarly];
#pragma unroll
    for (int ch = 0; ch < kEarly; ++ch) exp_chunk(ch, pe + 16 * ch);
    // P_j's buffer is free, and O_j may be rescaled, once the previous tile's product is done
    if (t > 0 && !wait_bounded(x.p_free, (t - 1) & 1u, wc)) return false;
    tc_fence_after_sync();
#pragma unroll
    for (int ch = 0; ch < kEarly; ++ch) store_chunk(ch, pe + 16 * ch);
#pragma unroll
    for (int ch = kEarly; ch < 4; ++ch) {
      uint32_t pk[16];
      exp_chunk(ch, pk);
      store_chunk(ch, pk);
    }
    l += (l0 + l1) + (l2 + l3);
    if (rescale) tmem_scale_row<DV>(x.tO, alpha);
    tmem_wait_st();
    tc_fence_before_sync();
    mbar_arrive(x.p_ready);
  }
  return true;
}
// Items with marks, which are rare, in a function of their own: in the one loop for all items, the call of
// exact_scores cost that 3 to 5 %.
struct Row {
  float m, l;
  uint32_t bad;
  bool ok;
};
template <int DK, int DV>
__device__ __noinline__ Row odd_item_tiles(const Tiles& x, const Codes& codes, uint32_t t, const WaitCtl& wc) {
  Row r{-INFINITY, 0.f, 0u, true};
  r.ok = item_tiles<DK, DV, true>(x, &codes, t, r.m, r.l, r.bad, wc);
  return r;
}

// One item of a CTA's share: its tiles [u0, u1) of `units` are this CTA's.  item < 0: no more.
struct Item {
  int item, u0, u1, units;
};

template <int DK, int DV>
__global__ void __launch_bounds__(kThreads, 1)
kv4_attn_tc_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                   const __nv_bfloat16* Q, const uint8_t* pool,
                   const int32_t* table, const float2* factor,
                   const uint64_t* bad_values,
                   const int32_t* lens, __nv_bfloat16* __restrict__ O, float* __restrict__ lse,
                   float* __restrict__ part_o, float2* __restrict__ part_ml, Cut* __restrict__ cuts, Params p) {
  using C = Cfg<DK, DV>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const uint32_t sQ = smem_u32(smem), sKV = smem_u32(smem + C::kOffKV), bar0 = smem_u32(smem + C::kOffBar);
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (C::kStages + s); };
  const uint32_t q_full = bar0 + 8u * (2 * C::kStages);
  auto s_full = [&](int j) { return bar0 + 8u * (2 * C::kStages + 1 + j); };
  auto p_ready = [&](int j) { return bar0 + 8u * (2 * C::kStages + 3 + j); };
  auto o_done = [&](int j) { return bar0 + 8u * (2 * C::kStages + 5 + j); };
  auto s_free = [&](int j) { return bar0 + 8u * (2 * C::kStages + 7 + j); };
  auto p_free = [&](int j) { return bar0 + 8u * (2 * C::kStages + 9 + j); };
  const uint32_t drain = bar0 + 8u * (2 * C::kStages + 11);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::kOffMisc);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + C::kOffMisc + 4);
  auto item_full = [&](int i) { return bar0 + 8u * (2 * C::kStages + 12 + i); };
  auto item_empty = [&](int i) { return bar0 + 8u * (2 * C::kStages + 14 + i); };
  volatile Item* items = reinterpret_cast<volatile Item*>(smem + C::kOffItems);
  int64_t* scan = reinterpret_cast<int64_t*>(smem + C::kOffItems + 2 * sizeof(Item));   // warp sums
  int64_t* found = scan + 12;                                                           // item, its first unit
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const WaitCtl wc{abort_flag, p.wait_limit_ns, 0u, &g_moa_kv4_tc_status};

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 2);   // one commit from each issuer
    }
    mbar_init(q_full, 256);
    mbar_init(drain, 2);
    for (int i = 0; i < 2; ++i) {
      mbar_init(item_full(i), 1);
      mbar_init(item_empty(i), 11);   // the softmax warps, both issuers, the loads
    }
    for (int j = 0; j < 2; ++j) {
      mbar_init(s_full(j), 1);
      mbar_init(p_ready(j), 128);
      mbar_init(o_done(j), 1);
      mbar_init(s_free(j), 128);
      mbar_init(p_free(j), 1);
    }
    *abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == kMmaWarp0) {
    tmem_alloc(smem_u32(tmem_slot), C::kTmemCols);
    tmem_relinquish();
  }
  wait_for_previous();
  // this CTA's share of all units, and the item in which it begins
  const int n_items = p.n_bh * p.n_tiles;
  int64_t sum = 0;
  for (int i = threadIdx.x; i < n_items; i += kThreads) sum += units_of(lens, i, p, true) + kItemUnits;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if (lane == 0) scan[warp] = sum;
  __syncthreads();
  int64_t total = 0;
#pragma unroll
  for (int w = 0; w < 12; ++w) total += scan[w];
  const Shares shares(total, gridDim.x);
  const int64_t first_unit = blockIdx.x < shares.n ? shares.start(blockIdx.x) : total;
  const int64_t stop = blockIdx.x < shares.n ? shares.start(blockIdx.x + 1) : total;
  int64_t done = 0;
  for (int base = 0; first_unit < stop; base += kThreads) {
    const int i = base + threadIdx.x;
    const int64_t mine = i < n_items ? units_of(lens, i, p, false) + kItemUnits : 0;
    int64_t incl = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t o = __shfl_up_sync(0xffffffffu, incl, d);
      if (lane >= d) incl += o;
    }
    __syncthreads();
    if (lane == 31) scan[warp] = incl;
    __syncthreads();
    int64_t all = 0;
#pragma unroll
    for (int w = 0; w < 12; ++w) {
      if (w < warp) incl += scan[w];
      all += scan[w];
    }
    incl += done;
    done += all;
    if (first_unit >= incl - mine && first_unit < incl) {
      found[0] = i;
      found[1] = incl - mine;
    }
    if (first_unit < done) break;
  }
  if (threadIdx.x == 0) cuts[blockIdx.x].pieces = 0;
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  // Item number i of the share, as every role sees it: valid until the role's release.
  auto get_item = [&](uint32_t i, bool& ok) {
    ok = ok && wait_bounded(item_full(i & 1), i >> 1 & 1u, wc);
    const volatile Item& x = items[i & 1];
    return ok ? Item{x.item, x.u0, x.u1, x.units} : Item{-1, 0, 0, 0};
  };

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kRegsCtrl));
    if (warp == kLoadWarp) {
      // ------------------------------------------------------------ TMA producer
      if (lane == 0) {
        tma_prefetch_desc(&tmK);
        tma_prefetch_desc(&tmV);
        int slot = 0;
        uint32_t phase = 0, issued = 0, issued_phase = 0;
        bool ok = true;
        for (uint32_t seg = 0; ok; ++seg) {
          const Item x = get_item(seg, ok);
          if (x.item < 0) break;
          mbar_arrive(item_empty(seg & 1));
          const int bh = int(unsigned(x.item) / unsigned(p.n_tiles)), n_kt = x.u1 - x.u0;
          for (int t = 0; t < 2 * n_kt; ++t) {
            // K0 K1 V0 K2 V1 ... (tile n + 1's scores come before tile n's P V)
            const int u = t - 1, nn = u >> 1;
            const bool is_k = t == 0 || ((u & 1) == 0 && nn + 1 < n_kt);
            const int n = t == 0 ? 0 : is_k ? nn + 1 : nn;
            if (!wait_bounded(empty_bar(slot), phase ^ 1u, wc)) {
              ok = false;
              break;
            }
            issued |= 1u << slot;
            issued_phase = (issued_phase & ~(1u << slot)) | (phase << slot);
            const uint32_t dst = sKV + slot * C::kStageBytes;
            const int row = (x.u0 + n) * kBN;
            mbar_arrive_expect_tx(full_bar(slot), is_k ? C::kKTileBytes : C::kVTileBytes);
            if (is_k) {
#pragma unroll
              for (int q = 0; q < DK / 64; ++q)
                tma_load_3d(dst + q * C::kPanelBytes, &tmK, full_bar(slot), q * 64, row, bh);
            } else {
#pragma unroll
              for (int q = 0; q < DV / 64; ++q)
                tma_load_3d(dst + q * C::kPanelBytes, &tmV, full_bar(slot), q * 64, row, bh);
            }
            if (++slot == C::kStages) {
              slot = 0;
              phase ^= 1u;
            }
          }
        }
        if (!ok || *abort_flag) {   // let every copy land before the CTA can exit
          for (int sl = 0; sl < C::kStages; ++sl)
            if (issued & (1u << sl))
              wait_quiesce(full_bar(sl), (issued_phase >> sl) & 1u, p.wait_limit_ns, &g_moa_kv4_tc_status);
        }
      }
    } else if (warp == kMmaWarp0 || warp == kMmaWarp1) {
      // ------------------------------------------------------------ MMA issuers, one for each row tile
      if (lane == 0) {
        const int j = warp == kMmaWarp0 ? 0 : 1;
        constexpr uint32_t kIdescQK = make_idesc_f16(kBM, kBN);
        constexpr uint32_t kIdescPV = make_idesc(kBM, DV, true);
        const uint32_t tS = tmem + (j ? C::kTmemS1 : C::kTmemS0);
        const uint32_t tP = tmem + (j ? C::kTmemP1 : C::kTmemP0);
        const uint32_t tO = tmem + (j ? C::kTmemO1 : C::kTmemO0);
        const uint32_t sQj = sQ + j * C::kQTileBytes;
        int slot = 0;
        uint32_t phase = 0;
        uint32_t t = 0;   // tiles so far: the phases of the barriers between the roles
        auto next = [&]() {
          if (++slot == C::kStages) {
            slot = 0;
            phase ^= 1u;
          }
        };
        auto issue_qk = [&](uint32_t kb) {
#pragma unroll
          for (int kk = 0; kk < DK / 16; ++kk) {
            const uint32_t off = (kk >> 2) * C::kPanelBytes + (kk & 3) * 32;
            mma_f16_ss(tS, make_sdesc_sw128(sQj + off, 16, 1024), make_sdesc_sw128(kb + off, 16, 1024), kIdescQK,
                       kk > 0 ? 1u : 0u);
          }
        };
        auto issue_pv = [&](uint32_t vb, uint32_t acc_first) {
#pragma unroll
          for (int kk = 0; kk < kBN / 16; ++kk)
            mma_f16_ts(tO, tP + kk * 8, make_sdesc_sw128(vb + kk * 2048, C::kPanelBytes, 1024), kIdescPV,
                       kk > 0 ? 1u : acc_first);
        };
        // The S buffer may take tile u's scores once its last reader holds what it has: this row
        // tile's softmax (tile u - 1), or with one buffer for both, the other one's (tile u - 1 for
        // row tile 0, tile u for row tile 1).
        auto s_buffer = [&](uint32_t u) {
          if (C::kSharedS) return j ? wait_bounded(s_free(0), u & 1u, wc) : u == 0 || wait_bounded(s_free(1), (u - 1) & 1u, wc);
          return u == 0 || wait_bounded(s_free(j), (u - 1) & 1u, wc);
        };
        bool ok = true;
        for (uint32_t seg = 0; ok; ++seg) {
          const Item x = get_item(seg, ok);
          if (x.item < 0) break;
          mbar_arrive(item_empty(seg & 1));
          const int n_kt = x.u1 - x.u0;
          ok = wait_bounded(q_full, seg & 1u, wc) && wait_bounded(full_bar(slot), phase, wc) && s_buffer(t);
          if (ok) {
            tc_fence_after_sync();
            const int ks = slot;
            next();
            issue_qk(sKV + ks * C::kStageBytes);
            mma_commit(s_full(j));
            mma_commit(empty_bar(ks));
          }
          for (int n = 0; ok && n < n_kt; ++n, ++t) {
            if (n + 1 < n_kt) {
              const int ks = slot;
              ok = wait_bounded(full_bar(slot), phase, wc) && s_buffer(t + 1);
              next();
              if (!ok) break;
              tc_fence_after_sync();
              issue_qk(sKV + ks * C::kStageBytes);
              mma_commit(s_full(j));
              mma_commit(empty_bar(ks));
            }
            const int vs = slot;
            ok = wait_bounded(full_bar(slot), phase, wc) && wait_bounded(p_ready(j), t & 1u, wc);
            next();
            if (!ok) break;
            tc_fence_after_sync();
            issue_pv(sKV + vs * C::kStageBytes, n > 0 ? 1u : 0u);
            mma_commit(p_free(j));
            mma_commit(empty_bar(vs));
          }
          // arrives when the item's products are complete
          mma_commit(o_done(j));
        }
        mma_commit(drain);
      }
    } else if (warp == kWalkWarp && lane == 0) {
      // ------------------------------------------------------------ the items of the share
      int64_t at = first_unit, before = 0;
      int item = 0;
      if (at < stop) {
        item = int(found[0]);
        before = found[1];
      }
      for (uint32_t seg = 0;; ++seg) {
        int units = 0, u0 = 0, u1 = 0, which = -1;
        while (at < stop && u0 == u1) {   // (nothing of an item's tiles: the next CTA begins it)
          units = units_of(lens, item, p, false);
          const int64_t end = before + units + kItemUnits, upto = end < stop ? end : stop;
          u0 = max(0, int(at - before) - kItemUnits), u1 = max(0, int(upto - before) - kItemUnits);
          if (u0 < u1) which = item;
          if (u0 == 0 && u1 > 0 && u1 < units) {   // begun here, ended by a later CTA
            uint32_t c = blockIdx.x;
            while (shares.start(c + 1) < end) ++c;
            cuts[blockIdx.x] = Cut{item, int(c - blockIdx.x) + 1};
          }
          at = upto;
          before = end;
          ++item;
        }
        // the wait lasts as long as the item before this one takes: up to 0.3 ms a tile (exact_scores)
        const WaitCtl wi{abort_flag, p.wait_limit_ns + uint64_t(p.tiles_pad) * 1000000u, 0u, &g_moa_kv4_tc_status};
        if (seg >= 2 && !wait_bounded(item_empty(seg & 1), ((seg >> 1) - 1) & 1u, wi)) break;
        volatile Item& x = items[seg & 1];
        x.item = which, x.u0 = u0, x.u1 = u1, x.units = units;
        mbar_arrive(item_full(seg & 1));
        if (which < 0) break;
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kRegsSoftmax));
    // -------------------------------------------------------------- softmax warpgroups
    const int j = warp >> 2;
    const int lane_base = (warp & 3) * 32, row = lane_base + lane;
    const uint32_t tS = tmem + (uint32_t(lane_base) << 16) + (j ? C::kTmemS1 : C::kTmemS0);
    const uint32_t tO = tmem + (uint32_t(lane_base) << 16) + (j ? C::kTmemO1 : C::kTmemO0);
    const uint32_t tP = tmem + (uint32_t(lane_base) << 16) + (j ? C::kTmemP1 : C::kTmemP0);
    bool ok = true;
    uint32_t t = 0;
    for (uint32_t seg = 0;; ++seg) {
      const Item x0 = get_item(seg, ok);
      if (x0.item < 0) break;
      const int u0 = x0.u0, u1 = x0.u1;
      // where the thread's row lies: row r of key head bh is query ri of its query head rh
      struct Place {
        int r, b, h, rh, ri;
        bool live;
      };
      auto place = [&](int item) {
        Place w;
        const int bh = int(unsigned(item) / unsigned(p.n_tiles));
        w.r = (item - bh * p.n_tiles) * kRows + j * kBM + row;
        w.b = int(unsigned(p.bh0 + bh) / unsigned(p.Hk)), w.h = p.bh0 + bh - w.b * p.Hk;
        w.rh = int(unsigned(w.r) / unsigned(p.N)), w.ri = w.r - w.rh * p.N;
        w.live = w.r < p.N * p.G;
        return w;
      };
      int lim;
      float c_row = p.c_log2;
      const float2* fac;
      {
        const Place w = place(x0.item);
        lim = w.live ? limit_of(length_of(lens, w.b, p, false), w.ri, p) : 0;
        fac = factor + int64_t(w.b * p.Hk + w.h - p.bh0) * p.tiles_pad;
        // the row as fp16, its power of two taken out, into the swizzled tile
        uint4 x[DK / 8];
        const __nv_bfloat16* src = Q + int64_t(w.b) * p.q_sb + (int64_t(w.h) * p.G + w.rh) * p.q_sh + int64_t(w.ri) * p.q_sn;
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < DK / 8; ++i) {
          x[i] = w.live ? *reinterpret_cast<const uint4*>(src + 8 * i) : make_uint4(0, 0, 0, 0);
          const uint32_t q[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            top = max(top, q[k] & 0x7fffu);
            top = max(top, (q[k] >> 16) & 0x7fffu);
          }
        }
        // a row with a member that is not finite gets a NaN: scores of -infinity would hide its tokens
        if (top >= 0x7f80u) x[0].x = 0x7fc07fc0u;
        const int e = row_exponent(top);
        const float down = power_of(-e) * (p.negate ? -1.f : 1.f);
        c_row *= power_of(e);
#pragma unroll
        for (int i = 0; i < DK / 8; ++i) {
          const uint32_t q[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
          uint32_t o[4];
#pragma unroll
          for (int k = 0; k < 4; ++k)
            o[k] = pack_f16x2(__uint_as_float(q[k] << 16) * down, __uint_as_float(q[k] & 0xffff0000u) * down);
          *reinterpret_cast<uint4*>(smem + j * C::kQTileBytes + (i >> 3) * C::kPanelBytes + row * 128 +
                                    (((i & 7) ^ (row & 7)) << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
        }
        fence_proxy_async_smem();
        mbar_arrive(q_full);
      }
      bool odd = false;   // a tile of the item is marked (looked for while the first product runs)
      for (int n = u0 + lane; n < u1; n += 32) odd |= __float_as_uint(fac[n].y) != 0;
      odd = __any_sync(0xffffffffu, odd);
      float m = -INFINITY, l = 0.f;
      uint32_t bad = 0;    // value groups that make the row NaN
      const Tiles x{tS, tO, tP, s_full(j), s_free(j), p_ready(j), p_free(j), fac, lim, u0, u1, c_row};
      if (odd) {
        const Place w = place(items[seg & 1].item);
        const __nv_bfloat16* q = Q + int64_t(w.b) * p.q_sb + (int64_t(w.h) * p.G + w.rh) * p.q_sh + int64_t(w.ri) * p.q_sn;
        const int64_t head_bytes = int64_t(p.blocks_per_page) * block_bytes(DK, DV);
        const Codes codes{w.live ? q : nullptr, pool + w.h * head_bytes, table + w.b * p.max_pages, p.Hk * head_bytes,
                          p.n_pages, p.blocks_per_page, length_of(lens, w.b, p, false), p.negate ? -1.f : 1.f,
                          bad_values + (fac - factor) * (kBN / kBlock)};
        const Tiles x_there = x;   // copies, so that what is in registers needs no address
        const WaitCtl wc_there = wc;
        const Row r = odd_item_tiles<DK, DV>(x_there, codes, t, wc_there);
        m = r.m, l = r.l, bad = r.bad, ok = r.ok;
      } else {
        ok = item_tiles<DK, DV, false>(x, nullptr, t, m, l, bad, wc);
      }
      t += u1 - u0;
      if (!ok || !wait_bounded(o_done(j), seg & 1u, wc)) break;
      tc_fence_after_sync();
      // the item is written, or this CTA's piece of it
      const volatile Item& xi = items[seg & 1];
      const Place w = place(xi.item);
      const bool first_piece = xi.u0 == 0, whole = first_piece && xi.u1 == xi.units;
      if (!whole) {
        const int64_t at = (int64_t(blockIdx.x) * 2 + first_piece) * kRows + j * kBM + row;
#pragma unroll
        for (int c = 0; c < DV; c += 16) {
          uint32_t o[16];
          tmem_ld_32x32b_x16(tO + c, o);
          tmem_wait_ld();
          reg_anchor_x16(o);
          if (bad >> (c / 32) & 1u) {
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] = 0x7fc00000u;
          }
          float4* dst = reinterpret_cast<float4*>(part_o + at * DV + c);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            dst[i] = make_float4(__uint_as_float(o[4 * i]), __uint_as_float(o[4 * i + 1]), __uint_as_float(o[4 * i + 2]),
                                 __uint_as_float(o[4 * i + 3]));
        }
        part_ml[at] = make_float2(m, l);
      } else {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        __nv_bfloat16* orow = O + int64_t(w.b) * p.o_sb + (int64_t(w.h) * p.G + w.rh) * p.o_sh + int64_t(w.ri) * p.o_sn;
        if (lse != nullptr && w.live)
          lse[(int64_t(w.b) * p.Hk * p.G + int64_t(w.h) * p.G + w.rh) * p.N + w.ri] = l == 0.f ? -INFINITY : (m + lg2_approx(l)) * kLn2;
#pragma unroll
        for (int c = 0; c < DV; c += 16) {
          uint32_t o[16];
          tmem_ld_32x32b_x16(tO + c, o);
          tmem_wait_ld();
          reg_anchor_x16(o);
          if (bad >> (c / 32) & 1u) {
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] = 0x7fc00000u;
          }
          if (w.live) {
            uint32_t y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
              y[i] = pack_bf16x2(__uint_as_float(o[2 * i]) * inv, __uint_as_float(o[2 * i + 1]) * inv);
            reinterpret_cast<uint4*>(orow + c)[0] = make_uint4(y[0], y[1], y[2], y[3]);
            reinterpret_cast<uint4*>(orow + c)[1] = make_uint4(y[4], y[5], y[6], y[7]);
          }
        }
      }
      tc_fence_before_sync();   // O is read: the next item's first product (after p_ready) may write it
      __syncwarp();
      if (lane == 0) mbar_arrive(item_empty(seg & 1));
    }
  }

  // Teardown: the tensor core is quiet before TMEM is freed, on the abort path too.  Only the lane of the role
  // waits: the others come here at the start, and their time would run out in a kernel longer than the limit.
  if (warp == kMmaWarp0 && lane == 0) wait_quiesce(drain, 0, p.wait_limit_ns, &g_moa_kv4_tc_status);
  tc_fence_before_sync();
  __syncthreads();
  if (warp == kMmaWarp0) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, C::kTmemCols);
  }
}

// Joins the pieces of cut items: one warp a row, eight rows a CTA.  A launch of its own has all SMs for
// it: done by the CTA that ends an item last, 100 queries against 9000 tokens took 59.8 us instead of 42.8.
template <int DV>
__global__ void __launch_bounds__(256)
kv4_attn_tc_join_kernel(const float* part_o, const float2* part_ml,
                        const Cut* cuts, __nv_bfloat16* __restrict__ O, float* __restrict__ lse, Params p) {
  wait_for_previous();
  const Cut cut = cuts[blockIdx.x];
  if (cut.pieces == 0) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int bh = int(unsigned(cut.item) / unsigned(p.n_tiles)), row = int(blockIdx.y) * 8 + warp;
  const int r = (cut.item - bh * p.n_tiles) * kRows + row;
  if (r >= p.N * p.G) return;
  auto place = [&](int i) -> int64_t { return ((int64_t(blockIdx.x) + i) * 2 + (i == 0)) * kRows + row; };
  float M = -INFINITY;
  for (int i = lane; i < cut.pieces; i += 32) M = fmaxf(M, part_ml[place(i)].x);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, d));
  const float base = M == -INFINITY ? 0.f : M;
  float L = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int i = 0; i < cut.pieces; ++i) {
    const float2 ml = part_ml[place(i)];
    const float f = ex2_approx(ml.x - base);
    L += f * ml.y;
    if (lane * 4 < DV) {
      const float4 v = *reinterpret_cast<const float4*>(part_o + place(i) * DV + lane * 4);
      x[0] += f * v.x, x[1] += f * v.y, x[2] += f * v.z, x[3] += f * v.w;
    }
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  const int b = int(unsigned(p.bh0 + bh) / unsigned(p.Hk)), h = p.bh0 + bh - b * p.Hk;
  const int rh = int(unsigned(r) / unsigned(p.N)), ri = r - rh * p.N;
  if (lane * 4 < DV)
    *reinterpret_cast<uint2*>(O + int64_t(b) * p.o_sb + (int64_t(h) * p.G + rh) * p.o_sh + int64_t(ri) * p.o_sn + lane * 4) =
        make_uint2(pack_bf16x2(x[0] * inv, x[1] * inv), pack_bf16x2(x[2] * inv, x[3] * inv));
  if (lse != nullptr && lane == 0)
    lse[(int64_t(b) * p.Hk * p.G + int64_t(h) * p.G + rh) * p.N + ri] = L == 0.f ? -INFINITY : (M + lg2_approx(L)) * kLn2;
}

// ------------------------------------------------------------------------------------------------
// Host side
// ------------------------------------------------------------------------------------------------
constexpr int64_t kWidenedMost = int64_t(1) << 30;   // bytes of widened heads at a time (one head may take more)

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// The workspace: widened keys and values of `heads` heads, the tiles' factors and masks, pieces, cuts.
struct Work {
  int64_t tiles_pad, heads;
  int64_t k, v, factor, bad, part_o, part_ml, cuts, bytes;   // offsets, and the sum
  Work(int64_t bh, int64_t max_len, int64_t dk, int64_t dv, int sms) {
    tiles_pad = (max_len + kBN - 1) / kBN;
    const int64_t head = tiles_pad * kBN * (dk + dv) * 2;
    heads = kWidenedMost / head;
    heads = heads < 1 ? 1 : heads > bh ? bh : heads;
    if (heads > 65535) heads = 65535;
    k = 0;
    v = k + heads * tiles_pad * kBN * dk * 2;
    factor = v + heads * tiles_pad * kBN * dv * 2;
    bad = factor + round_up(heads * tiles_pad * 8, 256);
    part_o = bad + heads * tiles_pad * (kBN / kBlock) * 8;
    part_ml = part_o + int64_t(sms) * 2 * kRows * dv * 4;
    cuts = part_ml + int64_t(sms) * 2 * kRows * 8;
    bytes = cuts + round_up(int64_t(sms) * sizeof(Cut), 256);
  }
};

template <int DK, int DV>
int launch(const Kv4AttnArgs& a, int sms, char* msg, size_t msglen) {
  using C = Cfg<DK, DV>;
  auto kern = kv4_attn_tc_kernel<DK, DV>;
  cudaError_t e = ensure_smem_limit(reinterpret_cast<const void*>(kern), C::kSmemBytes);
  static std::atomic<int> regs{-1};
  if (e == cudaSuccess && regs.load(std::memory_order_relaxed) < 0) {
    cudaFuncAttributes fa;
    e = cudaFuncGetAttributes(&fa, reinterpret_cast<const void*>(kern));
    if (e == cudaSuccess) regs.store(fa.numRegs, std::memory_order_relaxed);
  }
  if (e != cudaSuccess) {
    snprintf(msg, msglen, "cache attention: function attributes: %s", cudaGetErrorString(e));
    return 5;
  }
  if (regs.load(std::memory_order_relaxed) * kThreads < 256 * C::kRegsSoftmax + 128 * C::kRegsCtrl) {
    snprintf(msg, msglen, "cache attention: %d registers per thread, short of the register split", regs.load());
    return 5;
  }
  const int64_t bh = a.B * a.c.H;
  const Work w(bh, a.max_len, DK, DV, sms);
  uint8_t* ws = static_cast<uint8_t*>(a.ws);
  __half* wk = reinterpret_cast<__half*>(ws + w.k);
  __nv_bfloat16* wv = reinterpret_cast<__nv_bfloat16*>(ws + w.v);
  float2* factor = reinterpret_cast<float2*>(ws + w.factor);
  uint64_t* bad = reinterpret_cast<uint64_t*>(ws + w.bad);
  float* part_o = reinterpret_cast<float*>(ws + w.part_o);
  float2* part_ml = reinterpret_cast<float2*>(ws + w.part_ml);
  Cut* cuts = reinterpret_cast<Cut*>(ws + w.cuts);
  Params p{};
  p.q_sb = a.q.sb, p.q_sh = a.q.sh, p.q_sn = a.q.sn;
  p.o_sb = a.o.sb, p.o_sh = a.o.sh, p.o_sn = a.o.sn;
  p.n_pages = a.c.n_pages, p.max_pages = a.c.max_pages;
  p.N = int(a.N), p.max_len = int(a.max_len);
  p.Hk = a.c.H, p.G = int(a.Hq / a.c.H), p.blocks_per_page = a.c.page / kBlock;
  p.n_tiles = int((a.N * p.G + kRows - 1) / kRows);
  p.tiles_pad = int(w.tiles_pad);
  p.c_log2 = (a.scale < 0.f ? -a.scale : a.scale) * kLog2e;
  p.negate = a.scale < 0.f, p.causal = a.causal;
  p.wait_limit_ns = wait_limit_ns();
  for (int64_t first = 0; first < bh; first += w.heads) {
    p.bh0 = int(first);
    p.n_bh = int(bh - first < w.heads ? bh - first : w.heads);
    CUtensorMap mk, mv;
    if (!encode_bf16_map(&mk, wk, p.n_bh, w.tiles_pad * kBN, DK, msg, msglen)) return 5;
    if (!encode_bf16_map(&mv, wv, p.n_bh, w.tiles_pad * kBN, DV, msg, msglen)) return 5;
    const int64_t most = int64_t(p.n_bh) * p.n_tiles * w.tiles_pad;   // tiles of tokens, if all are as long as max_len
    const unsigned ctas = unsigned(most < sms ? most : sms);
    e = launch_overlapped(kv4_widen_kernel<DK, DV>, dim3(unsigned(w.tiles_pad), unsigned(p.n_bh)), dim3(256), 0, a.stream,
                          static_cast<const uint8_t*>(a.c.pool), a.c.table, a.lens, wk, wv, factor, bad, p);
    if (e == cudaSuccess)
      e = launch_overlapped(kern, dim3(ctas), dim3(kThreads), C::kSmemBytes, a.stream, mk, mv,
                            static_cast<const __nv_bfloat16*>(a.q.p), static_cast<const uint8_t*>(a.c.pool), a.c.table,
                            factor, bad, a.lens, static_cast<__nv_bfloat16*>(a.o.p),
                            a.lse, part_o, part_ml, cuts, p);
    if (e == cudaSuccess)
      e = launch_overlapped(kv4_attn_tc_join_kernel<DV>, dim3(ctas, kRows / 8), dim3(256), 0, a.stream, part_o, part_ml,
                            cuts, static_cast<__nv_bfloat16*>(a.o.p), a.lse, p);
    if (e != cudaSuccess) {
      snprintf(msg, msglen, "cache attention launch: %s", cudaGetErrorString(e));
      return 5;
    }
  }
  return 0;
}

}  // namespace

size_t kv4_attn_tc_workspace(int64_t bh, int64_t max_len, int64_t dk, int64_t dv, int sms) {
  return size_t(Work(bh, max_len, dk, dv, sms).bytes);
}

int launch_kv4_attn_tc(const Kv4AttnArgs& a, char* msg, size_t msglen) {
  int sms = 0;
  const cudaError_t e = device_sm_count(&sms);
  if (e != cudaSuccess) {
    snprintf(msg, msglen, "cache attention: SM count: %s", cudaGetErrorString(e));
    return 5;
  }
  if (a.c.dk == 64)
    return a.c.dv == 64 ? launch<64, 64>(a, sms, msg, msglen) : launch<64, 128>(a, sms, msg, msglen);
  return a.c.dv == 64 ? launch<128, 64>(a, sms, msg, msglen) : launch<128, 128>(a, sms, msg, msglen);
}

cudaError_t kv4_tc_read_and_clear_status(unsigned* value) {
  cudaError_t e = cudaMemcpyFromSymbol(value, g_moa_kv4_tc_status, sizeof(unsigned));
  if (e != cudaSuccess || *value == 0) return e;
  const unsigned zero = 0;
  return cudaMemcpyToSymbol(g_moa_kv4_tc_status, &zero, sizeof(unsigned));
}

}  // namespace moa
