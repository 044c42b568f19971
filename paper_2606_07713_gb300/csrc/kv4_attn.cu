// Attention over the 4-bit paged cache (kv4.cuh), sm_103a.
//
// Mathematics.  Query row (head, i) of sequence b, key head h = head / G, sees the first
// n = len_b - N + i + 1 cached tokens (causal) or all len_b:
//     s_j = scale * sum_c q_c k_jc,    o = sum_j e^(s_j - m) v_j / sum_j e^(s_j - m),  m = max s_j.
// With k_jc = sk_j,g code_jc the inner sum is, group by group of 32 features, an integer-valued
// product scaled afterwards: s_j = scale * sum_g sk_j,g (sum_{c in g} q_c code_jc).  The values'
// scales go into the weights: o_c = sum_j (p_j sv_j,g) code_jc.  So codes enter the matrix
// instructions as exact small integers in bf16 and the cache is never widened in memory.  One
// pass over the tokens with the running maximum and sum; partial results of token ranges are
// joined by o = sum_s e^(m_s - M) o_s / sum_s e^(m_s - M) l_s.
//
// Rounding: bf16 queries (below 2^120) enter exactly; the weights p sv are rounded to bf16 once (relative
// 2^-8, as in the other bf16 forward).  fp32 queries and weights enter as three bf16 terms each
// (24 bits), so the fp32 form is fp32-accurate on the same instructions.  Scores, maxima, sums
// and outputs accumulate in fp32.
//
// What bounds it: for single tokens chains of dependent instructions at the three warps a scheduler that
// the registers allow (fixed latency is the largest stall).  No unit is full: memory 56 to 60 %, the ALU
// pipe, which widens codes, half, issue 57 %.  The floor is the cache's bytes, 9/16 a value.  Measured,
// single bf16 tokens, d = 128: 131072 + 42256 cached tokens of 8 key heads under 64 query heads 45.4 us =
// 4.4 TB/s of the cache; 48 uneven sequences up to 16384 under 32 query heads 71.5 us = 4.8 TB/s (measured
// copy bandwidth: 6.8).  From 17 to some 1000 query rows of a key head it is far from a floor: see
// widening_pays below.
// Tokens lie on the 16 rows of mma.m16n8k16 and queries on its 8 columns: a decoding step has few
// queries, and the other way round half of the tensor work would be padding.  (A byte form, codes as
// fp8 and queries as two fp8 terms, took fewer instructions and a fifth more time.)
//
// Layout of the work: a work item is a tile of up to 8 NT query rows of one key head of one
// sequence; its visible tokens count in units of 64.  The units of all items, in a row, are cut into
// equal shares, one for each resident CTA, so uneven lengths leave no SM idle; a CTA walks over the
// items of its share.  An item inside one share is written at once; the pieces of a cut item go to
// the workspace and a second kernel joins them.  Within a CTA four warps take turns at tiles of
// kSub blocks, each with its own ring of bulk copies, running maximum, sum and output, joined
// through shared memory at the end of the item.  Tiles are worked on two blocks at a time, two chains of
// dependent instructions beside each other.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdio>
#include <type_traits>

#include "internal.h"
#include "kv4.cuh"
#include "ops_internal.h"
#include "ptx.cuh"
#include "tc_common.cuh"

namespace moa {

__device__ unsigned int g_moa_kv4_attn_status = 0;

namespace {

using namespace kv4;
using namespace ptx;
using namespace tc;

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// D += A B, 16 x 8 x 16, bf16 in, fp32 accumulation.
__device__ __forceinline__ void mma_16816(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7},"
      " {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// D = A B: the same without an addend.
__device__ __forceinline__ void mma_16816_first(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7},"
      " {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
// Transpose of an 8 x 8 matrix of 16-bit values held one row (two values a lane) per four lanes.
__device__ __forceinline__ uint32_t transpose8(uint32_t a) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
// Four pairs of codes of a word as bf16 pairs of code / 64.  The bits 0 .. 255 of a bf16 are the
// numbers 0 .. 255 times 2^-133 (subnormals and the first binade share their spacing), so a nibble
// n = code + 8 masked out at bits 0-3 is n 2^-133 and at bits 4-7 is n 2^-129: one fused multiply-add
// makes (n - 8) / 64 of either, exactly, and half of the nibbles need no shift.
constexpr float kCodeUnit = 64.f;
__device__ __forceinline__ void widen(uint32_t w, uint32_t* r) {
  const __nv_bfloat162 low = __halves2bfloat162(__ushort_as_bfloat16(0x7f00), __ushort_as_bfloat16(0x7f00));    // 2^127
  const __nv_bfloat162 high = __halves2bfloat162(__ushort_as_bfloat16(0x7d00), __ushort_as_bfloat16(0x7d00));   // 2^123
  const __nv_bfloat162 bias = __halves2bfloat162(__ushort_as_bfloat16(0xbe00), __ushort_as_bfloat16(0xbe00));   // -1/8
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t x = (j < 2 ? w : w >> 8) & (j % 2 ? 0x00f000f0u : 0x000f000fu);
    const __nv_bfloat162 y = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&x), j % 2 ? high : low, bias);
    r[j] = *reinterpret_cast<const uint32_t*>(&y);
  }
}
// The same without the multiply-add: n 2^-133 and n 2^-129, for keys against bf16 queries, which are
// brought up by a power of two and hold the 16 and the 8 (see the queries).
__device__ __forceinline__ void widen_raw(uint32_t w, uint32_t* r) {
#pragma unroll
  for (int j = 0; j < 4; ++j) r[j] = (j < 2 ? w : w >> 8) & (j % 2 ? 0x00f000f0u : 0x000f000fu);
}
// 2^e, -126 <= e <= 127, and the exponent of a number (0 for zero and what is not finite).
__device__ __forceinline__ float power_of(int e) { return __uint_as_float(uint32_t(127 + e) << 23); }
__device__ __forceinline__ int exponent_of(float x) {
  return x == 0.f || !(x < INFINITY) ? 0 : int(__float_as_uint(x) >> 23) - 127;
}
// A query row is multiplied by 2^row_shift: its largest magnitude is then in [2^100, 2^101), so that
// n 2^-133 times it is an ordinary number; rows from 2^93 on by 2^7, which keeps 2^(133 - shift), the
// scores' unit, one too.
__device__ __forceinline__ int row_shift(float top) { return max(100 - exponent_of(top), 7); }
__device__ __forceinline__ float bf16_bits(uint32_t b) { return __uint_as_float(b << 16); }

template <int G>
__device__ __forceinline__ void load_words(uint32_t* w, const uint8_t* p) {
  if constexpr (G == 1) {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  } else if constexpr (G == 4) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
  } else {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    w[0] = v.x, w[1] = v.y;
  }
}
// G bf16 scales of one token as floats.
template <int G>
__device__ __forceinline__ void load_scales(float* s, const uint8_t* p) {
  if constexpr (G == 4) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    s[0] = bf16_bits(v.x), s[1] = __uint_as_float(v.x & 0xffff0000u);
    s[2] = bf16_bits(v.y), s[3] = __uint_as_float(v.y & 0xffff0000u);
  } else {
    const uint32_t v = *reinterpret_cast<const uint32_t*>(p);
    s[0] = bf16_bits(v), s[1] = __uint_as_float(v & 0xffff0000u);
  }
}

// The terms of a pair of fp32 values as bf16 pairs: one rounding, or three terms of 24 bits.
template <int TERMS>
__device__ __forceinline__ void split_pair(float x, float y, uint32_t* t) {
#pragma unroll
  for (int i = 0; i < TERMS; ++i) {
    t[i] = pack_bf16x2(x, y);
    if (i + 1 < TERMS) {
      x -= bf16_bits(t[i]);
      y -= __uint_as_float(t[i] & 0xffff0000u);
    }
  }
}

constexpr int kUnit = 64;              // tokens of a unit of work
constexpr int kUnitBlocks = kUnit / kBlock;
// An item costs about as much as this many units besides its tokens (places, queries, the join of
// the warps): it counts for that many more, which come first and hold no tokens.  Without them a
// share of short items takes several times as long as one of long items (48 sequences of 0 to 16384
// tokens: 87 us with 0, 72 with 6, 74 with 12; 131072 + 42256: 47.6, 45.5, 45.1).
constexpr int kItemUnits = 6;
constexpr float kSlack = 8.f;          // the running maximum may lag by this (log2): weights up to 2^8

struct Params {
  int64_t q_sb, q_sh, q_sn, o_sb, o_sh, o_sn;
  int64_t n_pages, max_pages;
  int64_t N;
  int max_len;
  int n_tiles, n_pairs;                // query tiles of a key head; B * n_tiles
  int Hk, G, blocks_per_page;
  float scale;
  bool causal;
  uint64_t wait_limit_ns;
};

// An item for the joining kernel: the list has one for every item if there are no more items than
// CTAs, else one for every CTA (the item that it begins and does not end).
struct Cut {
  int pair, h;
  int first;    // the CTA of its first piece
  int pieces;   // 0: written whole, nothing to join
};

template <int DK, int DV, int NT, int TERMS>
struct Cfg {
  static constexpr int kSub = NT == 4 ? 1 : 2;                  // 16-token blocks of a tile
  static constexpr int kPair = NT == 1 ? 2 : 1;                 // blocks taken at once (independent chains)
  static_assert(kSub % kPair == 0, "whole pairs in a tile");
  static constexpr int kBytes = block_bytes(DK, DV);
  static constexpr int kStages = (NT * TERMS == 1 ? 13824 : 18432) / (kSub * kBytes);
  static constexpr int kBatch = 32 / kSub;                      // tiles whose places are looked up at once
  static constexpr int kRing = kSub * kStages * kBytes;         // one warp's ring
  static constexpr int kOStride = DV + 4;                       // padded row of the final join
  static constexpr int kJoin = kWarps * 8 * NT * (kOStride + 2) * 4;
  static constexpr int kData = kWarps * kRing > kJoin ? kWarps * kRing : kJoin;
  static constexpr bool kQRegs = NT * TERMS == 1;               // queries in registers
  // queries in the order of the matrix operands: [nt][term][group][lane] 16 bytes
  static constexpr int kQ = kQRegs ? 0 : NT * TERMS * (DK / 32) * 32 * 16;
  static constexpr int kOffQ = kData;
  static constexpr bool kQSmem = !kQRegs && TERMS == 1;
  static constexpr int kOffBias = kOffQ + kQ;                   // [nt][lane] 8 bytes (bf16 queries)
  static constexpr int kOffTop = kOffBias + (kQSmem ? NT * 32 * 8 : 0);   // [nt][8] rows' largest
  static constexpr int kOffBar = kOffTop + (kQSmem ? NT * 8 * 4 : 0);
  static constexpr int kOffMisc = kOffBar + kWarps * kStages * 8;
  static constexpr int kSmem = kOffMisc + 64;
  // resident CTAs: registers (168 or 255 a thread; 32-row tiles spill all the same, at d = 128 132 bytes
  // with bf16 queries and 104 with fp32 ones) and 228 KB of shared memory
  static constexpr int kCtas = NT * TERMS == 1 ? 3 : 2;
  static_assert(kBytes % 16 == 0, "bulk copies are whole 16-byte units");
  static_assert(8 + 8 * kWarps <= 64, "the warps' sums fit behind the abort flag");
  static_assert(kCtas * (kSmem + 1024) <= 233472, "shared memory of the resident CTAs");
};

template <typename T>
__device__ __forceinline__ void store4(T* p, const float* x);
template <>
__device__ __forceinline__ void store4(float* p, const float* x) {
  *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
}
template <>
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float* x) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
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

// The cached tokens of sequence b, its length clamped to what the call allows.
__device__ __forceinline__ int length_of(const int32_t* lens, int64_t b, const Params& p, bool report) {
  const int len = lens[b];
  if (len >= 0 && len <= p.max_len) return len;
  if (report) atomicExch(&g_moa_kv4_attn_status, kErrIndex);
  return len < 0 ? 0 : p.max_len;
}
// Tokens that row r of a sequence of `len` tokens sees.
__device__ __forceinline__ int limit_of(int len, int r, const Params& p) {
  if (!p.causal) return len;
  const int n = len - int(p.N) + int(unsigned(r) / unsigned(p.G)) + 1;
  return n < 0 ? 0 : n;
}
__device__ __forceinline__ int sequence_of(int pair, const Params& p) {
  return p.n_tiles == 1 ? pair : int(unsigned(pair) / unsigned(p.n_tiles));
}
// Units of tokens of an item of a pair (sequence, query tile): at least one, so that every item is
// written.
template <int NT>
__device__ __forceinline__ int units_of(const int32_t* lens, int pair, const Params& p, bool report) {
  const int rows = int(p.N) * p.G, b = sequence_of(pair, p);
  const int last = (pair - b * p.n_tiles + 1) * (8 * NT) - 1;
  const int n = limit_of(length_of(lens, b, p, report), last < rows ? last : rows - 1, p);
  return n <= kUnit ? 1 : (n + kUnit - 1) / kUnit;
}

// Equal shares of `total` units: share c begins at start(c).
struct Shares {
  int64_t each;
  uint32_t rest, n;
  __device__ __forceinline__ Shares(int64_t total, uint32_t ctas) {
    n = total < ctas ? uint32_t(total) : ctas;   // none without a unit
    each = total < 0x7fffffff ? int64_t(uint32_t(total) / n) : total / n;
    rest = uint32_t(total - each * n);
  }
  __device__ __forceinline__ int64_t start(uint32_t c) const { return each * c + rest * c / n; }
};

template <typename T, int DK, int DV, int NT, int TERMS>
__global__ void __launch_bounds__(kThreads, Cfg<DK, DV, NT, TERMS>::kCtas)
kv4_attn_kernel(const T* Q, const uint8_t* pool,
                const int32_t* table, const int32_t* lens,
                T* __restrict__ O, float* __restrict__ lse, float* __restrict__ part_o,
                float* __restrict__ part_ml, Cut* __restrict__ cuts, Params p) {
  using C = Cfg<DK, DV, NT, TERMS>;
  constexpr int GK = DK / 32, GV = DV / 32;
  extern __shared__ __align__(128) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, t = lane & 3;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + C::kOffMisc);
  int64_t* scan = reinterpret_cast<int64_t*>(smem + C::kOffMisc + 8);   // [kWarps], then a pair found
  const WaitCtl wc{abort_flag, p.wait_limit_ns, 0u, &g_moa_kv4_attn_status};

  uint8_t* ring = smem + warp * C::kRing;
  const uint32_t ring_s = smem_u32(ring);
  const uint32_t bars = smem_u32(smem + C::kOffBar) + warp * C::kStages * 8;
  if (lane == 0) {
    for (int s = 0; s < C::kStages; ++s) mbar_init(bars + 8 * s, 1);
    fence_barrier_init();
  }
  if (threadIdx.x == 0) *abort_flag = 0;
  wait_for_previous();

  // this CTA's share of all units, and the pair in which it begins
  int64_t sum = 0;
  for (int i = threadIdx.x; i < p.n_pairs; i += kThreads) sum += units_of<NT>(lens, i, p, true) + kItemUnits;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
  if (lane == 0) scan[warp] = sum;
  __syncthreads();
  int64_t total = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) total += scan[w];
  total *= p.Hk;
  const Shares shares(total, gridDim.x);
  int64_t at = blockIdx.x < shares.n ? shares.start(blockIdx.x) : total;
  const int64_t stop = blockIdx.x < shares.n ? shares.start(blockIdx.x + 1) : total;
  int pair = 0;
  int64_t before = 0;   // the pair of unit `at`, the units of all heads in the pairs before it
  int64_t done = 0;
  for (int base = 0; p.n_pairs > 1 && at < stop; base += kThreads) {
    const int i = base + threadIdx.x;
    const int64_t mine = i < p.n_pairs ? int64_t(units_of<NT>(lens, i, p, false) + kItemUnits) * p.Hk : 0;
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
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) incl += scan[w];
      all += scan[w];
    }
    incl += done;
    done += all;
    __syncthreads();
    if (at >= incl - mine && at < incl) {
      scan[0] = i;
      scan[1] = incl - mine;
    }
    if (at < done) {
      __syncthreads();
      pair = int(scan[0]);
      before = scan[1];
      break;
    }
  }

  const bool by_item = int64_t(p.n_pairs) * p.Hk <= gridDim.x;
  if (threadIdx.x == 0 && !by_item) cuts[blockIdx.x].pieces = 0;
  const int rows = int(p.N) * p.G;
  uint32_t count = 0;     // tiles this warp has taken so far: its place in the ring and the phases
  bool ok = true;
  while (at < stop) {
    // the item and this CTA's units of it: u0 to u1 of its units of tokens
    const int units = units_of<NT>(lens, pair, p, false), counted = units + kItemUnits;
    const uint32_t local = uint32_t(at - before);
    const int h = int(local / uint32_t(counted));
    const int64_t item = before + int64_t(h) * counted;      // its first unit
    const int64_t upto = item + counted < stop ? item + counted : stop;
    const int u0 = max(0, int(at - item) - kItemUnits), u1 = max(0, int(upto - item) - kItemUnits);
    at = upto;
    const int this_pair = pair;
    if (at == before + int64_t(counted) * p.Hk) {
      before = at;
      ++pair;
    }
    if (u0 == u1) continue;   // nothing of its tokens: the next CTA begins it
    const int64_t b = sequence_of(this_pair, p);
    const int r0 = (this_pair - int(b) * p.n_tiles) * (8 * NT);
    const int len = length_of(lens, b, p, false);
    const int last_row = r0 + 8 * NT < rows ? r0 + 8 * NT - 1 : rows - 1;
    const int all_limit = limit_of(len, r0, p);          // every row sees these
    const int any_limit = limit_of(len, last_row, p);    // no row sees more
    const int n_blocks = (any_limit + kBlock - 1) / kBlock;
    const int first = u0 * kUnitBlocks;
    const int end = u1 * kUnitBlocks < n_blocks ? u1 * kUnitBlocks : n_blocks;

    // This warp's tiles: kSub blocks each, every kWarps-th one.  Places are looked up for kBatch
    // tiles at once: lane i finds where block i of the batch lies, and starts its copy when the
    // turn of its tile comes.
    const int n_tiles = end <= first ? 0 : (end - first + C::kSub - 1) / C::kSub;
    const int my_tiles = ok && n_tiles > warp ? (n_tiles - warp + kWarps - 1) / kWarps : 0;
    const int32_t* pages = table + b * p.max_pages;
    const uint8_t* src = nullptr;      // this lane's block of the batch being started
    uint32_t dst = 0, bar = 0, here = 0, here_next = 0;   // blocks that are there: batch in use, batch started
    auto look_up = [&](int batch) {
      const int i = batch * C::kBatch + lane / C::kSub;
      const int blk = first + (warp + i * kWarps) * C::kSub + lane % C::kSub;
      src = nullptr;
      if (blk < end) {
        const int slot = blk / p.blocks_per_page;
        const int pg = pages[slot];
        if (pg >= 0 && pg < p.n_pages)
          src = pool + ((int64_t(pg) * p.Hk + h) * p.blocks_per_page + (blk - slot * p.blocks_per_page)) * C::kBytes;
        else
          atomicExch(&g_moa_kv4_attn_status, kErrIndex);
      }
      const uint32_t st = (count + i) % C::kStages;
      dst = ring_s + (st * C::kSub + lane % C::kSub) * C::kBytes;
      bar = bars + 8 * st;
      here_next = __ballot_sync(0xffffffffu, src != nullptr);
    };
    constexpr uint32_t kTileBits = (1u << C::kSub) - 1;
    auto start = [&](int it) {         // starts the copies of tile `it`, of the batch looked up last
      const int j = it % C::kBatch;
      const uint32_t bytes = __popc(here_next >> (j * C::kSub) & kTileBits) * C::kBytes;
      if (lane == j * C::kSub) mbar_arrive_expect_tx(bar, bytes);
      __syncwarp();
      if (lane / C::kSub == j && src != nullptr) bulk_load(dst, src, C::kBytes, bar);
    };
    int issued = 0;
    if (my_tiles > 0) {
      look_up(0);
      here = here_next;
      for (; issued < my_tiles && issued < C::kStages; ++issued) start(issued);
      static_assert(C::kStages <= C::kBatch, "the first tiles are of one batch");
    }

    // Queries: registers or shared memory, in operand order; a negative scale turns their signs.
    // bf16: a row times a power of two, its largest magnitude then in [2^100, 2^101), and -8 2^-133
    // sum q of each group as bf16 terms beside it (see widen_raw).  fp32: three bf16 terms.
    uint4 qreg[C::kQRegs ? GK : 1];
    uint2 qbias = make_uint2(0, 0);
    float c2[NT][2], slack[NT][2];   // log2 units of a score, and kSlack in scores
    if constexpr (TERMS == 1) {
      for (int nt = C::kQRegs ? 0 : warp; nt < NT; nt += C::kQRegs ? 1 : kWarps) {
        const int r = r0 + nt * 8 + g, i_n = int(unsigned(r) / unsigned(p.G));
        const T* src = Q + b * p.q_sb + (int64_t(h) * p.G + r - i_n * p.G) * p.q_sh + i_n * p.q_sn + 8 * t;
        float x[GK][8];
        float top = 0.f;
#pragma unroll
        for (int gi = 0; gi < GK; ++gi) {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[gi][e] = 0.f;
          if (r < rows) load8(src + 32 * gi, x[gi]);
#pragma unroll
          for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[gi][e]));
        }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // in two factors: it may be above the largest number
        const int up = row_shift(top);
        const float up0 = power_of(up / 2) * (p.scale < 0.f ? -1.f : 1.f), up1 = power_of(up - up / 2);
        float part[GK];
#pragma unroll
        for (int gi = 0; gi < GK; ++gi) {
          float q = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            x[gi][e] = x[gi][e] * up0 * up1;
            q += x[gi][e] * power_of(-100);
          }
          q += __shfl_xor_sync(0xffffffffu, q, 1);
          q += __shfl_xor_sync(0xffffffffu, q, 2);
          part[gi] = q * -power_of(100 + 3 - 133);
          // features 0 1 and 4 5 meet nibbles as they are, 2 3 and 6 7 nibbles times 16
          const uint4 w = make_uint4(pack_bf16x2(x[gi][0], x[gi][1]), pack_bf16x2(x[gi][2] * 0.0625f, x[gi][3] * 0.0625f),
                                     pack_bf16x2(x[gi][4], x[gi][5]), pack_bf16x2(x[gi][6] * 0.0625f, x[gi][7] * 0.0625f));
          if constexpr (C::kQRegs) qreg[gi] = w;
          else *reinterpret_cast<uint4*>(smem + C::kOffQ + ((nt * GK + gi) * 32 + lane) * 16) = w;
        }
        // index k = GK term + group of the bias product: a lane's pairs are k = 2t, 2t + 1 and 2t + 8, 2t + 9
        uint32_t terms[3][GK / 2];
#pragma unroll
        for (int i = 0; i < GK / 2; ++i) {
          uint32_t s3[3];
          split_pair<3>(part[2 * i], part[2 * i + 1], s3);
          terms[0][i] = s3[0], terms[1][i] = s3[1], terms[2][i] = s3[2];
        }
        uint2 bias = make_uint2(0, 0);
        if constexpr (GK == 4) {
          const int i = t & 1;
          bias.x = t < 2 ? (i ? terms[0][GK / 2 - 1] : terms[0][0]) : (i ? terms[1][GK / 2 - 1] : terms[1][0]);
          bias.y = t < 2 ? (i ? terms[2][GK / 2 - 1] : terms[2][0]) : 0u;
        } else {
          bias.x = t == 0 ? terms[0][0] : t == 1 ? terms[1][0] : t == 2 ? terms[2][0] : 0u;
        }
        if constexpr (C::kQRegs) {
          qbias = bias;
#pragma unroll
          for (int c = 0; c < 2; ++c) c2[0][c] = __shfl_sync(0xffffffffu, top, 8 * t + 4 * c);
        } else {
          *reinterpret_cast<uint2*>(smem + C::kOffBias + (nt * 32 + lane) * 8) = bias;
          if (t == 0) reinterpret_cast<float*>(smem + C::kOffTop)[nt * 8 + g] = top;
        }
      }
      if constexpr (!C::kQRegs) {
        __syncthreads();
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int c = 0; c < 2; ++c) c2[n][c] = reinterpret_cast<const float*>(smem + C::kOffTop)[n * 8 + 2 * t + c];
      }
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const float top = c2[n][c];   // not finite: neither are the row's scores
          c2[n][c] = top < INFINITY ? fabsf(p.scale) * kLog2e * power_of(133 - row_shift(top)) : __int_as_float(0x7fc00000);
        }
    } else {
      const uint32_t sign = p.scale < 0.f ? 0x80008000u : 0u;
      for (int i = threadIdx.x; i < NT * GK * 32; i += kThreads) {
        const int gi = (i >> 5) % GK, nt = (i >> 5) / GK;
        const int r = r0 + nt * 8 + g, i_n = int(unsigned(r) / unsigned(p.G));
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 0.f;
        if (r < rows)
          load8(Q + b * p.q_sb + (int64_t(h) * p.G + r - i_n * p.G) * p.q_sh + i_n * p.q_sn + 32 * gi + 8 * t, x);
        uint32_t w[4][TERMS];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          split_pair<TERMS>(x[2 * e], x[2 * e + 1], w[e]);
#pragma unroll
          for (int k = 0; k < TERMS; ++k) w[e][k] ^= sign;
        }
#pragma unroll
        for (int k = 0; k < TERMS; ++k)
          *reinterpret_cast<uint4*>(smem + C::kOffQ + (((nt * TERMS + k) * GK + gi) * 32 + lane) * 16) =
              make_uint4(w[0][k], w[1][k], w[2][k], w[3][k]);
      }
      __syncthreads();
#pragma unroll
      for (int n = 0; n < NT; ++n) c2[n][0] = c2[n][1] = fabsf(p.scale) * kLog2e * kCodeUnit;
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int c = 0; c < 2; ++c) slack[n][c] = c2[n][c] > 0.f ? kSlack / c2[n][c] : INFINITY;

    float o[NT][DV / 16][4];
    // maximum, sum, where the maximum has to move, and what weights subtract: -m c2
    float m[NT][2], l[NT][2], above[NT][2], mb[NT][2];
    int lim[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        m[n][c] = above[n][c] = -INFINITY;
        l[n][c] = mb[n][c] = 0.f;
        const int r = r0 + n * 8 + 2 * t + c;
        lim[n][c] = r < rows ? limit_of(len, r, p) : any_limit;
      }
#pragma unroll
      for (int i = 0; i < DV / 16; ++i) o[n][i][0] = o[n][i][1] = o[n][i][2] = o[n][i][3] = 0.f;
    }

    // kPair blocks of 16 tokens.  PLAIN: they are there and every row sees every token of them.
    // `there`: one bit a block.
    auto blocks = [&](auto plain_tag, const uint8_t* blk, int tok0, uint32_t there) {
      constexpr bool PLAIN = decltype(plain_tag)::value;
      // scores: sc[block][nt]: (token g, rows 2t, 2t+1), (token g+8, ...)
      float sc[C::kPair][NT][4];
#pragma unroll
      for (int u = 0; u < C::kPair; ++u) {
        const uint8_t* at_blk = blk + u * C::kBytes;
        uint32_t kw[2][GK];
        uint32_t sw[2][GK / 2];      // scales, two groups a word
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          load_words<GK>(kw[r], at_blk + ((g + 8 * r) * 4 + t) * GK * 4);
          load_words<GK / 2>(sw[r], at_blk + key_scales(DK, DV) + (g + 8 * r) * GK * 2);
        }
        if constexpr (TERMS == 1) {
          // what code + 8 is too much: sum_g ks (-8 sum q), one product over groups and terms
          const uint32_t s0 = GK == 4 && (t & 1) ? sw[0][GK / 2 - 1] : sw[0][0];
          const uint32_t s1 = GK == 4 && (t & 1) ? sw[1][GK / 2 - 1] : sw[1][0];
          const uint32_t a[4] = {s0, s1, s0, s1};
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            uint2 qb = qbias;
            if constexpr (!C::kQRegs) qb = *reinterpret_cast<const uint2*>(smem + C::kOffBias + (n * 32 + lane) * 8);
            mma_16816_first(sc[u][n], a, qb.x, qb.y);
          }
        }
#pragma unroll
        for (int gi = 0; gi < GK; ++gi) {
          float ks[2];
#pragma unroll
          for (int r = 0; r < 2; ++r)
            ks[r] = gi & 1 ? __uint_as_float(sw[r][gi / 2] & 0xffff0000u) : bf16_bits(sw[r][gi / 2]);
          uint32_t lo[4], hi[4];
          if constexpr (TERMS == 1) {
            widen_raw(kw[0][gi], lo);
            widen_raw(kw[1][gi], hi);
          } else {
            widen(kw[0][gi], lo);
            widen(kw[1][gi], hi);
          }
          const uint32_t a0[4] = {lo[0], hi[0], lo[1], hi[1]}, a1[4] = {lo[2], hi[2], lo[3], hi[3]};
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            float acc[4];
#pragma unroll
            for (int k = 0; k < TERMS; ++k) {
              uint4 q;
              if constexpr (C::kQRegs) q = qreg[gi];
              else q = *reinterpret_cast<const uint4*>(smem + C::kOffQ + (((n * TERMS + k) * GK + gi) * 32 + lane) * 16);
              if (k == 0) mma_16816_first(acc, a0, q.x, q.y);
              else mma_16816(acc, a0, q.x, q.y);
              mma_16816(acc, a1, q.z, q.w);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
              sc[u][n][e] = TERMS > 1 && gi == 0 ? ks[e >> 1] * acc[e] : fmaf(ks[e >> 1], acc[e], sc[u][n][e]);
          }
        }
        if constexpr (!PLAIN) {
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (!(there >> u & 1u) || tok0 + u * kBlock + g + (e >> 1) * 8 >= lim[n][e & 1]) sc[u][n][e] = -INFINITY;
        }
      }
      // The maximum moves only when a score passes it by more than kSlack (in log2): until then
      // the weights stay below 2^kSlack and nothing is rescaled.
      float top[NT][2];
      bool moves = false;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          top[n][c] = fmaxf(sc[0][n][c], sc[0][n][2 + c]);
#pragma unroll
          for (int u = 1; u < C::kPair; ++u) top[n][c] = max3f(top[n][c], sc[u][n][c], sc[u][n][2 + c]);
          moves |= top[n][c] > above[n][c];
        }
      if (__any_sync(0xffffffffu, moves)) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float x = top[n][c];
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
            const float mn = fmaxf(m[n][c], x);
            const float alpha = m[n][c] == -INFINITY ? 0.f : ex2_approx((m[n][c] - mn) * c2[n][c]);
            m[n][c] = mn;
            above[n][c] = mn == -INFINITY ? -INFINITY : mn + slack[n][c];
            mb[n][c] = mn == -INFINITY ? 0.f : -mn * c2[n][c];
            l[n][c] *= alpha;
#pragma unroll
            for (int i = 0; i < DV / 16; ++i) {
              o[n][i][c] *= alpha;
              o[n][i][2 + c] *= alpha;
            }
          }
      }
#pragma unroll
      for (int u = 0; u < C::kPair; ++u)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float w = ex2_approx(fmaf(sc[u][n][e], c2[n][e & 1], mb[n][e & 1]));
            if (!PLAIN && sc[u][n][e] == -INFINITY) w = -0.f;   // hidden; a small visible weight ends as +0
            sc[u][n][e] = w;
            l[n][e & 1] += w;
          }
      // o += (p sv) codes
#pragma unroll
      for (int u = 0; u < C::kPair; ++u) {
        const uint8_t* at_blk = blk + u * C::kBytes;
        uint32_t vw[2][GV];
        float vs[2][GV];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          load_words<GV>(vw[r], at_blk + value_codes(DK) + ((r * 8 + g) * 4 + t) * GV * 4);
          load_scales<GV>(vs[r], at_blk + value_scales(DK, DV) + (g + 8 * r) * GV * 2);
        }
#pragma unroll
        for (int gi = 0; gi < GV; ++gi) {
          uint32_t lo[4], hi[4];
          widen(vw[0][gi], lo);
          widen(vw[1][gi], hi);
          const uint32_t a0[4] = {lo[0], lo[1], hi[0], hi[1]}, a1[4] = {lo[2], lo[3], hi[2], hi[3]};
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            float w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              w[e] = sc[u][n][e] * vs[e >> 1][gi];
              // a hidden token's scale may be anything: its weight is zero whatever that is
              if (!PLAIN && __float_as_uint(sc[u][n][e]) == 0x80000000u) w[e] = 0.f;
            }
            uint32_t p0[TERMS], p1[TERMS];
            split_pair<TERMS>(w[0], w[1], p0);
            split_pair<TERMS>(w[2], w[3], p1);
#pragma unroll
            for (int k = 0; k < TERMS; ++k) {
              const uint32_t b0 = transpose8(p0[k]), b1 = transpose8(p1[k]);
              mma_16816(o[n][2 * gi], a0, b0, b1);
              mma_16816(o[n][2 * gi + 1], a1, b0, b1);
            }
          }
        }
      }
    };

    uint32_t s = count % C::kStages, phase = count / C::kStages & 1u;
    for (int it = 0; it < my_tiles; ++it) {
      ok = wait_bounded(bars + 8 * s, phase, wc);
      if (__any_sync(0xffffffffu, !ok)) {
        ok = false;
        break;
      }
      const uint8_t* st = ring + s * C::kSub * C::kBytes;
      const int tok0 = (first + (warp + it * kWarps) * C::kSub) * kBlock;
      const uint32_t got = here >> (it % C::kBatch * C::kSub) & kTileBits;
      constexpr uint32_t kPairBits = (1u << C::kPair) - 1;
#pragma unroll 1
      for (int sub = 0; sub < C::kSub; sub += C::kPair) {
        const int tok = tok0 + sub * kBlock;
        const uint32_t there = got >> sub & kPairBits;
        if (there == kPairBits && tok + C::kPair * kBlock <= all_limit)
          blocks(std::true_type{}, st + sub * C::kBytes, tok, there);
        else
          blocks(std::false_type{}, st + sub * C::kBytes, tok, there);
      }
      if (it % C::kBatch == C::kBatch - 1) here = here_next;
      // the stage is free again: start its next tile
      __syncwarp();
      if (issued < my_tiles) {
        if (issued % C::kBatch == 0) look_up(issued / C::kBatch);
        start(issued);
        ++issued;
      }
      if (++s == C::kStages) {
        s = 0;
        phase ^= 1u;
      }
    }
    if (!ok) {  // a wait ran out: let the copies in flight land before the memory is reused
      for (int i = issued > C::kStages ? issued - C::kStages : 0; i < issued; ++i)
        wait_quiesce(bars + 8 * ((count + i) % C::kStages), (count + i) / C::kStages & 1u, p.wait_limit_ns,
                     &g_moa_kv4_attn_status);
    }
    count += my_tiles;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) l[n][c] += __shfl_xor_sync(0xffffffffu, l[n][c], d);

    // join the warps; maxima in log2 from here on
    __syncthreads();
    float* jo = reinterpret_cast<float*>(smem);                      // [warp][row][kOStride]
    float* jm = jo + kWarps * 8 * NT * C::kOStride;                  // [warp][row]
    float* jl = jm + kWarps * 8 * NT;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int row = warp * 8 * NT + n * 8 + 2 * t + c;
        if (g == 0) {
          jm[row] = m[n][c] == -INFINITY ? -INFINITY : m[n][c] * c2[n][c];
          jl[row] = l[n][c];
        }
#pragma unroll
        for (int gi = 0; gi < GV; ++gi)
          *reinterpret_cast<float4*>(jo + row * C::kOStride + 32 * gi + 4 * g) = make_float4(
              o[n][2 * gi][c], o[n][2 * gi][2 + c], o[n][2 * gi + 1][c], o[n][2 * gi + 1][2 + c]);
      }
    __syncthreads();
    const bool whole = u0 == 0 && u1 == units;
    // pieces of a cut item: the first one in the CTA's second place, others in the first
    const int64_t place = (int64_t(blockIdx.x) * 2 + (u0 == 0)) * (8 * NT);
    for (int i = threadIdx.x; i < 8 * NT * (DV / 4); i += kThreads) {
      const int row = i / (DV / 4), col = i % (DV / 4) * 4;
      const int r = r0 + row;
      if (r >= rows) continue;
      float M = -INFINITY, L = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWarps; ++w) M = fmaxf(M, jm[w * 8 * NT + row]);
      const float base = M == -INFINITY ? 0.f : M;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float f = ex2_approx(jm[w * 8 * NT + row] - base);
        const float4 v = *reinterpret_cast<const float4*>(jo + (w * 8 * NT + row) * C::kOStride + col);
        L += f * jl[w * 8 * NT + row];
        x[0] += f * v.x, x[1] += f * v.y, x[2] += f * v.z, x[3] += f * v.w;
      }
      if (!whole) {
        store4(part_o + (place + row) * DV + col, x);
        if (col == 0) *reinterpret_cast<float2*>(part_ml + 2 * (place + row)) = make_float2(M, L);
      } else {
        const float inv = L == 0.f ? 0.f : kCodeUnit / L;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] *= inv;
        const int64_t i_n = unsigned(r) / unsigned(p.G), head = int64_t(h) * p.G + r - i_n * p.G;
        store4(O + b * p.o_sb + head * p.o_sh + i_n * p.o_sn + col, x);
        if (lse != nullptr && col == 0)
          lse[(b * p.Hk * p.G + head) * p.N + i_n] = L == 0.f ? -INFINITY : (M + lg2_approx(L)) * kLn2;
      }
    }
    if (u0 == 0 && (by_item || !whole) && threadIdx.x == 0) {
      // the CTA that has the item's last unit
      uint32_t c = blockIdx.x;
      while (shares.start(c + 1) < item + counted) ++c;
      cuts[by_item ? uint32_t(this_pair) * p.Hk + h : blockIdx.x] =
          Cut{this_pair, h, int(blockIdx.x), whole ? 0 : int(c - blockIdx.x) + 1};
    }
    // the joined values have been read: copies may write the memory again
    __syncthreads();
    fence_proxy_async_smem();
  }
}

// Joins the pieces of cut items: CTA (item, row); its warps share the pieces, each with its first
// ones on their way before the largest maximum is known (the call is all latency).  Eight warps for
// items of many pieces, two where most have a few (then the CTAs are many and short).
template <typename T, int DV, int ROWS, int kJoinWarps>
__global__ void __launch_bounds__(32 * kJoinWarps)
kv4_attn_join_kernel(const float* part_o, const float* part_ml,
                     const Cut* cuts, T* __restrict__ O, float* __restrict__ lse, Params p) {
  constexpr int kAhead = kJoinWarps == 8 ? 8 : 2;
  __shared__ float so[kJoinWarps][DV], sl[kJoinWarps];
  wait_for_previous();
  const Cut cut = cuts[blockIdx.x];
  if (cut.pieces == 0) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t b = sequence_of(cut.pair, p);
  const int row = int(blockIdx.y), r = (cut.pair - int(b) * p.n_tiles) * ROWS + row;
  if (r >= int(p.N) * p.G) return;
  // piece 0 lies in its CTA's second place, the others in the first
  auto place = [&](int i) -> int64_t { return (int64_t(cut.first + i) * 2 + (i == 0)) * ROWS + row; };
  float4 v[kAhead];
  float2 ml[kAhead];
#pragma unroll
  for (int j = 0; j < kAhead; ++j) {
    const int i = warp + j * kJoinWarps;
    ml[j] = make_float2(-INFINITY, 0.f);
    v[j] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (i < cut.pieces) {
      ml[j] = *reinterpret_cast<const float2*>(part_ml + 2 * place(i));
      if (lane * 4 < DV) v[j] = *reinterpret_cast<const float4*>(part_o + place(i) * DV + lane * 4);
    }
  }
  float M = -INFINITY;
  for (int i = lane; i < cut.pieces; i += 32) M = fmaxf(M, part_ml[2 * place(i)]);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, d));
  const float base = M == -INFINITY ? 0.f : M;
  float L = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int j = 0; j < kAhead; ++j) {
    const float f = ex2_approx(ml[j].x - base);
    L += f * ml[j].y;
    x[0] += f * v[j].x, x[1] += f * v[j].y, x[2] += f * v[j].z, x[3] += f * v[j].w;
  }
#pragma unroll 4
  for (int i = warp + kAhead * kJoinWarps; i < cut.pieces; i += kJoinWarps) {
    const int64_t at = place(i);
    const float2 q = *reinterpret_cast<const float2*>(part_ml + 2 * at);
    const float f = ex2_approx(q.x - base);
    L += f * q.y;
    if (lane * 4 < DV) {
      const float4 u = *reinterpret_cast<const float4*>(part_o + at * DV + lane * 4);
      x[0] += f * u.x, x[1] += f * u.y, x[2] += f * u.z, x[3] += f * u.w;
    }
  }
  if (lane * 4 < DV) *reinterpret_cast<float4*>(&so[warp][lane * 4]) = make_float4(x[0], x[1], x[2], x[3]);
  if (lane == 0) sl[warp] = L;
  __syncthreads();
  if (warp != 0) return;
  L = 0.f;
#pragma unroll
  for (int w = 0; w < kJoinWarps; ++w) L += sl[w];
  const float inv = L == 0.f ? 0.f : kCodeUnit / L;
  const int64_t i_n = unsigned(r) / unsigned(p.G), head = int64_t(cut.h) * p.G + r - i_n * p.G;
  if (lane * 4 < DV) {
    x[0] = x[1] = x[2] = x[3] = 0.f;
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) {
      const float4 u = *reinterpret_cast<const float4*>(&so[w][lane * 4]);
      x[0] += u.x, x[1] += u.y, x[2] += u.z, x[3] += u.w;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] *= inv;
    store4(O + b * p.o_sb + head * p.o_sh + i_n * p.o_sn + lane * 4, x);
  }
  if (lse != nullptr && lane == 0)
    lse[(b * p.Hk * p.G + head) * p.N + i_n] = L == 0.f ? -INFINITY : (M + lg2_approx(L)) * kLn2;
}

// Workspace: the pieces' rows, their maxima and sums, and the list of cut items.
struct Work {
  size_t o, ml, cuts;   // bytes of each
  Work(int64_t ctas, int64_t rows, int64_t dv)
      : o(size_t(ctas) * 2 * rows * dv * 4), ml(size_t(ctas) * 2 * rows * 8), cuts(size_t(ctas) * sizeof(Cut)) {}
  size_t bytes() const { return o + ml + cuts; }
};

template <typename T, int DK, int DV, int NT, int TERMS>
cudaError_t run(const Kv4AttnArgs& a, const Kv4Plan& plan, const Params& p) {
  using C = Cfg<DK, DV, NT, TERMS>;
  const void* f = reinterpret_cast<const void*>(kv4_attn_kernel<T, DK, DV, NT, TERMS>);
  cudaError_t e = ensure_smem_limit(f, C::kSmem);
  if (e != cudaSuccess) return e;
  const Work w(plan.ctas, plan.rows_tile, DV);
  uint8_t* ws = static_cast<uint8_t*>(a.ws);
  float* part_o = reinterpret_cast<float*>(ws);
  float* part_ml = reinterpret_cast<float*>(ws + w.o);
  Cut* cuts = reinterpret_cast<Cut*>(ws + w.o + w.ml);
  e = launch_overlapped(kv4_attn_kernel<T, DK, DV, NT, TERMS>, dim3(unsigned(plan.ctas)), dim3(kThreads), C::kSmem,
                        a.stream, static_cast<const T*>(a.q.p), static_cast<const uint8_t*>(a.c.pool), a.c.table,
                        a.lens, static_cast<T*>(a.o.p), a.lse, part_o, part_ml, cuts, p);
  if (e != cudaSuccess) return e;
  const int64_t items = a.B * a.c.H * plan.n_tiles, rows = a.N * (a.Hq / a.c.H);
  const dim3 grid(unsigned(items < plan.ctas ? items : plan.ctas), unsigned(rows < 8 * NT ? rows : 8 * NT));
  // few items of many pieces: eight warps share the pieces.  16 items on 456 CTAs 45.6 us (49.6 with two
  // warps); 48 x 8 items 75.0 us (71.6 with two)
  const bool many = plan.ctas >= 8 * items;
  return launch_overlapped(many ? kv4_attn_join_kernel<T, DV, 8 * NT, 8> : kv4_attn_join_kernel<T, DV, 8 * NT, 2>, grid,
                           dim3(many ? 256 : 64), 0, a.stream, part_o, part_ml, cuts, static_cast<T*>(a.o.p), a.lse, p);
}

template <typename T, int DK, int DV, int TERMS>
cudaError_t run_nt(const Kv4AttnArgs& a, const Kv4Plan& plan, const Params& p) {
  switch (plan.rows_tile) {
    case 8: return run<T, DK, DV, 1, TERMS>(a, plan, p);
    case 16: return run<T, DK, DV, 2, TERMS>(a, plan, p);
    default: return run<T, DK, DV, 4, TERMS>(a, plan, p);
  }
}

template <typename T, int TERMS>
cudaError_t run_d(const Kv4AttnArgs& a, const Kv4Plan& plan, const Params& p) {
  if (a.c.dk == 64)
    return a.c.dv == 64 ? run_nt<T, 64, 64, TERMS>(a, plan, p) : run_nt<T, 64, 128, TERMS>(a, plan, p);
  return a.c.dv == 64 ? run_nt<T, 128, 64, TERMS>(a, plan, p) : run_nt<T, 128, 128, TERMS>(a, plan, p);
}

}  // namespace

// Whether many query rows are faster through kv4_attn_tc.cu.  This file's kernel widens codes once for
// every 32 rows: 8 us + 0.08 ns for each cached token of a head and 32 rows.  The other one widens
// once for all, in a launch of its own: 20 us + 0.13 ns for each, + 0.076 ns for each 256 rows.
// Measured, 8 key heads (this file's, the other's, us): 64 rows x 8192 tokens 22, 36; 128 x 8192 34,
// 35; 128 x 65536 165, 127; 256 x 8192 51, 38; 512 x 600 22, 25; 2048 x 600 42, 32 (all causal, d = 128:
// the heads' sizes and the mask do not enter the rule).  Either way this range is 7 to 15 times above its
// floors, in the same order 1.4, 2.3, 18, 4.5 and 0.7 us: codes are widened too often here, and there it
// takes three launches, 16-bit copies of all keys and values, and items of 256 rows.
bool widening_pays(int64_t heads, int64_t rows, int64_t max_len) {
  const double tokens = double(heads) * double(max_len);
  const double n32 = double((rows + 31) / 32), n256 = double((rows + 255) / 256);
  return tokens * (0.08 * n32 - 0.13 - 0.076 * n256) > 14000.0;
}

Kv4Plan kv4_attn_plan(int64_t B, int64_t Hk, int64_t G, int64_t N, int64_t max_len, bool f32, int sms) {
  Kv4Plan p;
  const int64_t rows = G * N;
  p.tc = !f32 && widening_pays(B * Hk, rows, max_len);
  p.rows_tile = rows <= 8 ? 8 : rows <= 16 ? 16 : 32;
  p.n_tiles = (rows + p.rows_tile - 1) / p.rows_tile;
  // resident CTAs, but none with less than two units if every length is max_len
  const int64_t resident = int64_t(sms) * (p.rows_tile == 8 && !f32 ? 3 : 2);
  const int64_t units = (max_len + kUnit - 1) / kUnit;
  const int64_t items = B * Hk * p.n_tiles;
  const int64_t most = items * ((units + 1) / 2);
  p.ctas = most < resident ? most : resident;
  return p;
}

size_t kv4_attn_workspace(int64_t B, int64_t Hk, int64_t max_len, int64_t dk, int64_t dv, const Kv4Plan& p, int sms) {
  return p.tc ? kv4_attn_tc_workspace(B * Hk, max_len, dk, dv, sms) : Work(p.ctas, p.rows_tile, dv).bytes();
}

int launch_kv4_attn(const Kv4AttnArgs& a, const Kv4Plan& plan, char* msg, size_t msglen) {
  if (plan.tc) return launch_kv4_attn_tc(a, msg, msglen);
  Params p{};
  p.q_sb = a.q.sb, p.q_sh = a.q.sh, p.q_sn = a.q.sn;
  p.o_sb = a.o.sb, p.o_sh = a.o.sh, p.o_sn = a.o.sn;
  p.n_pages = a.c.n_pages, p.max_pages = a.c.max_pages;
  p.N = a.N, p.max_len = int(a.max_len);
  p.Hk = a.c.H, p.G = int(a.Hq / a.c.H);
  p.blocks_per_page = a.c.page / kv4::kBlock;
  p.n_tiles = int(plan.n_tiles), p.n_pairs = int(a.B * plan.n_tiles);
  if ((a.max_len / kUnit + 1 + kItemUnits) * a.c.H > 0x7fffffffLL) {
    snprintf(msg, msglen, "cache attention: max_len times the key heads is too large");
    return 3;
  }
  p.scale = a.scale;
  p.causal = a.causal;
  p.wait_limit_ns = wait_limit_ns();
  const cudaError_t e = a.f32 ? run_d<float, 3>(a, plan, p) : run_d<__nv_bfloat16, 1>(a, plan, p);
  if (e != cudaSuccess) {
    snprintf(msg, msglen, "cache attention launch: %s", cudaGetErrorString(e));
    return 5;
  }
  return 0;
}

cudaError_t kv4_attn_read_and_clear_status(unsigned* value) {
  cudaError_t e = cudaMemcpyFromSymbol(value, g_moa_kv4_attn_status, sizeof(unsigned));
  if (e != cudaSuccess || *value == 0) return e;
  const unsigned zero = 0;
  return cudaMemcpyToSymbol(g_moa_kv4_attn_status, &zero, sizeof(unsigned));
}

}  // namespace moa
