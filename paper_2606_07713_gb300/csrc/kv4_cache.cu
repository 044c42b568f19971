// Writing keys and values into the 4-bit cache, and reading them back, sm_103a.
//
// Mathematics and layout: kv4.cuh.  Write: per row and 32 features, s = bf16(max|x| / 7),
// code = rint(x / s) (ties to even; for bf16 inputs the same codes as in exact arithmetic).  Read:
// code * s in fp32, rounded once to the output's type.
//
// What bounds it: memory, and in the write the instructions of a code (figures at the kernels).  A bf16
// value is 2 bytes on one side and 9/16 on the other.
//
// Layout of the work: a unit is 16 tokens of a sequence that fall into one 16-token block of the cache
// when the call's positions are consecutive (a prompt): a head's block is then put together (or taken
// apart) in shared memory and crosses to or from global memory in whole 16-byte pieces.  Rows that do
// not fill a block (single tokens, the ends of a prompt, positions in another order) go straight to
// their places, in 2- and 4-byte pieces.  A CTA takes a unit through a range of heads: its places are
// looked up once, and the next head's rows are on their way while one is worked on.  8 or 16 lanes own
// one row, eight features a lane, so the four lanes of a scale group are neighbours.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdio>

#include "internal.h"
#include "kv4.cuh"
#include "ops_internal.h"

namespace moa {

__device__ unsigned int g_moa_kv4_status = 0;

namespace {

using namespace kv4;

constexpr int kThreads = 256;

// A lane's eight features as they lie in memory.
template <typename T>
struct Raw {
  uint4 w[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < int(sizeof(T) / 2); ++i) w[i] = p ? reinterpret_cast<const uint4*>(p)[i] : make_uint4(0, 0, 0, 0);
  }
  __device__ __forceinline__ void widen(float* x) const {
    if constexpr (sizeof(T) == 2) {
      const uint32_t v[4] = {w[0].x, w[0].y, w[0].z, w[0].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(v[i] << 16);
        x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
      }
    } else {
      const uint32_t v[8] = {w[0].x, w[0].y, w[0].z, w[0].w, w[1].x, w[1].y, w[1].z, w[1].w};
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(v[i]);
    }
  }
  // The largest magnitude's bits, as a float's: a NaN's are above every number's.
  __device__ __forceinline__ uint32_t top() const {
    if constexpr (sizeof(T) == 2) {
      uint32_t m = w[0].x;   // of each half's magnitudes (the sign is no use); a NaN in either operand gives a NaN
      const uint32_t v[3] = {w[0].y, w[0].z, w[0].w};
#pragma unroll
      for (int i = 0; i < 3; ++i) asm("max.NaN.xorsign.abs.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(v[i]));
      return max(m << 16 & 0x7fff0000u, m & 0x7fff0000u);
    } else {
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 2; ++i)
        m = max(max(m, max(w[i].x & 0x7fffffffu, w[i].y & 0x7fffffffu)), max(w[i].z & 0x7fffffffu, w[i].w & 0x7fffffffu));
      return m;
    }
  }
};
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float* x) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<uint32_t*>(&v);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(float* p, const float* x) {
  *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}

// Two floats in a register pair, and arithmetic on both at once (each rounded as by itself).
__device__ __forceinline__ uint64_t pair(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
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

// Codes + 8 of this lane's eight features, and the group's scale (bits of a bf16).
// The quotient of bf16 inputs: x (1/s), rounded to a multiple of 2^-11 by the sum with 1.5 * 2^12, then
// to an integer.  x and s have 8 significant bits, so a quotient that is not a half-integer is 2^-10 or
// more away from one, and x (1/s) is within 2^-20 of the quotient: on that grid it falls on a
// half-integer if and only if the quotient is one, and the code is that of the exact quotient.  fp32
// inputs take the IEEE division.
// `code` holds them as integers plus a multiple of 2^16 (of 2^20 and more once shifted): only the low
// 16 bits of a sum of four, shifted by nibbles, count.
template <typename T>
__device__ __forceinline__ uint32_t quantise8(const Raw<T>& raw, uint32_t* code) {
  uint32_t m = raw.top();
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
  const bool finite = m < 0x7f800000u;
  float s;
  uint32_t bits;
  {
    // bf16: m / 7 is never within 2^-12 of a boundary between bf16 values (7 times one of those has
    // 9 bits and a factor of 7, m has 8 bits), so the rounded reciprocal gives the same
    const float top = __uint_as_float(m);
    const __nv_bfloat16 h = __float2bfloat16_rn(sizeof(T) == 2 ? top * (1.f / 7.f) : __fdiv_rn(top, 7.f));
    bits = finite ? __bfloat16_as_ushort(h) : 0x7fc0u;
    s = finite ? __bfloat162float(h) : 0.f;
  }
  float x[8];
  raw.widen(x);
  // rint and the bias of 8 at once: 1.5 * 2^23 + 8 makes an integer of the sum, ties to even
  constexpr float kRound = 12582920.f;
  if (sizeof(T) == 2 && s > 1.2e-38f && s < 8.0e37f) {   // 1/s is a normal number
    float inv;   // within 2^-22 of 1/s
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
    constexpr float kGrid = 6144.f;
    const uint64_t inv2 = pair(inv, inv), grid2 = pair(kGrid, kGrid), round2 = pair(kRound - kGrid, kRound - kGrid);
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      // |x / s| <= 7 (1 + 2^-8): the code needs no bound
      const uint64_t c2 = add2(fma2(pair(x[i], x[i + 1]), inv2, grid2), round2);
      code[i] = uint32_t(c2), code[i + 1] = uint32_t(c2 >> 32);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float q = s > 0.f ? __fdiv_rn(x[i], s) : 0.f;
      code[i] = __float_as_uint(fminf(fmaxf(q, -7.f), 7.f) + kRound);
    }
  }
  return bits;
}
// Four codes as a 16-bit word.
__device__ __forceinline__ uint32_t pack4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return a + (b << 4) + (c << 8) + (d << 12);
}

struct Dims {
  int64_t B, N;
  int64_t n_pages, max_pages;
  uint32_t units;   // of a sequence: 16 tokens each, the first one short of the first position's offset
  uint32_t all;     // units of all sequences
  bool flat;        // short sequences: a unit is 16 tokens of any
  int H, page, dk, dv;
  int hp;           // heads of a CTA
};

// A thread's row: which unit of the CTA, which row of the unit, where it lies in the cache.
template <int LPR>
struct Row {
  static constexpr int kUnits = kThreads / (kBlock * LPR);   // units of a CTA
  int lane, i, unit;        // lane of the row, row of the unit, unit of the CTA
  bool live;                // the row exists
  bool whole;               // the unit is one whole block
  int64_t b, n;
  int tok;
  int32_t at;
  uint8_t* block;           // of head 0; null: padding or (with the status word set) no such place
  __device__ __forceinline__ Row(uint8_t* pool, const int32_t* table, const int32_t* pos, const Dims& p) {
    __shared__ const uint8_t* s_block[kUnits][kBlock];
    lane = threadIdx.x % LPR;
    i = threadIdx.x / LPR % kBlock;
    unit = threadIdx.x / (LPR * kBlock);
    const uint32_t u = blockIdx.x * kUnits + unit;
    if (p.flat) {
      const uint64_t token = uint64_t(u) * kBlock + i;
      live = token < uint64_t(p.B) * p.N;
      b = live ? uint32_t(token) / uint32_t(p.N) : 0;
      n = live ? int64_t(token) - b * p.N : 0;
    } else {
      b = u / p.units;
      live = u < p.all;
      // where in its block the first row would lie, going by the last row if that has a position (padding
      // comes first where the rows are a chunk's queries), else by the first
      const int32_t first = live ? pos[b * p.N] : 0, last = live ? pos[b * p.N + p.N - 1] : 0;
      const uint32_t from = last >= 0 ? uint32_t(last) - uint32_t(p.N - 1) : uint32_t(first);
      n = int64_t(u - uint32_t(b) * p.units) * kBlock - int(from & (kBlock - 1)) + i;
      live = live && n >= 0 && n < p.N;
    }
    at = live ? pos[b * p.N + n] : -1;
    tok = at & (kBlock - 1);
    block = nullptr;
    if (at >= 0) {
      const uint32_t slot = uint32_t(at) / uint32_t(p.page);
      int32_t page = -1;
      if (slot < p.max_pages) page = table[b * p.max_pages + slot];
      if (page >= 0 && page < p.n_pages)
        block = pool + (int64_t(page) * p.H * (p.page / kBlock) + (uint32_t(at) - slot * p.page) / kBlock) * block_bytes(p.dk, p.dv);
      else if (lane == 0)
        atomicExch(&g_moa_kv4_status, kErrIndex);
    }
    // whole: each of the 16 rows in its own place of the same block
    if (lane == 0) s_block[unit][i] = tok == i ? block : nullptr;
    __syncthreads();
    whole = s_block[unit][0] != nullptr;
#pragma unroll
    for (int k = 1; k < kBlock; ++k) whole = whole && s_block[unit][k] == s_block[unit][0];
  }
};

constexpr int kMostBytes = block_bytes(128, 128);
static_assert(8 * kBlock * 16 >= block_bytes(64, 64) && 16 * kBlock * 16 >= kMostBytes, "a thread for each 16 bytes of a block");

// Keys' and values' words of a lane's codes, to their places in a block.
struct Places {
  int k, ks, v, v1, vs;
};
template <typename T>
__device__ __forceinline__ void put(uint8_t* to, const Places& at, const Raw<T>& k, const Raw<T>& v, bool mine_k,
                                    bool mine_v, bool first) {
  uint32_t c[8];
  uint32_t s = quantise8<T>(k, c);
  if (mine_k) {
    *reinterpret_cast<uint32_t*>(to + at.k) = __byte_perm(pack4(c[0], c[2], c[4], c[6]), pack4(c[1], c[3], c[5], c[7]), 0x5410);
    if (first) *reinterpret_cast<uint16_t*>(to + at.ks) = uint16_t(s);
  }
  s = quantise8<T>(v, c);
  if (mine_v) {
    *reinterpret_cast<uint16_t*>(to + at.v) = uint16_t(pack4(c[0], c[1], c[2], c[3]));
    *reinterpret_cast<uint16_t*>(to + at.v1) = uint16_t(pack4(c[4], c[5], c[6], c[7]));
    if (first) *reinterpret_cast<uint16_t*>(to + at.vs) = uint16_t(s);
  }
}

// Two heads of bf16 at a time share a barrier.  Measured on bf16 keys and values, 3 x 8 x 16001 x (128 +
// 128): 52.3 us = 4.8 TB/s with four CTAs on an SM (64 registers, 20
// bytes spilled); with three 58, with five 60; one head at a time 55.1.  The instructions of the codes fill about 70 % of the issue
// slots, the rest waits for rows and barriers.
template <typename T, int LPR>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 4 : 3)
kv4_write_kernel(View k, View v, uint8_t* pool, const int32_t* table, const int32_t* pos, Dims p) {
  constexpr int kUnits = Row<LPR>::kUnits, kTeam = LPR * kBlock;   // threads of a unit
  constexpr int kStep = sizeof(T) == 2 ? 2 : 1;                    // heads at a time
  __shared__ __align__(16) uint8_t s_bytes[2][kStep][kUnits][kMostBytes];
  wait_for_previous();
  const Row<LPR> r(pool, table, pos, p);
  const int f0 = r.lane * 8, g = r.lane >> 2, t = r.lane & 3;
  const int bytes = block_bytes(p.dk, p.dv), gk = p.dk / kGroup, gv = p.dv / kGroup;
  const int64_t head_bytes = int64_t(p.page / kBlock) * bytes;
  const bool mine_k = r.block != nullptr && f0 < p.dk, mine_v = r.block != nullptr && f0 < p.dv;
  const int h0 = int(blockIdx.y) * p.hp, h1 = min(h0 + p.hp, p.H);
  const T* from_k = static_cast<const T*>(k.p) + r.b * k.sb + r.n * k.sn + f0 + h0 * k.sh;
  const T* from_v = static_cast<const T*>(v.p) + r.b * v.sb + r.n * v.sn + f0 + h0 * v.sh;
  const Places at{key_word(r.tok, t, g, gk), key_scales(p.dk, p.dv) + (r.tok * gk + g) * 2,
                  value_word(p.dk, r.tok, 2 * t, g, gv) + (r.tok & 1) * 2,
                  value_word(p.dk, r.tok, 2 * t + 1, g, gv) + (r.tok & 1) * 2,
                  value_scales(p.dk, p.dv) + (r.tok * gv + g) * 2};
  Raw<T> xk[kStep], xv[kStep];
  auto fetch = [&](int h) {   // heads h, ..., h + kStep - 1, and on to the next ones
#pragma unroll
    for (int u = 0; u < kStep; ++u) {
      xk[u].load(mine_k && h + u < h1 ? from_k : nullptr);
      xv[u].load(mine_v && h + u < h1 ? from_v : nullptr);
      from_k += k.sh, from_v += v.sh;
    }
  };
  fetch(h0);
  uint8_t* block = r.block + h0 * head_bytes;
  if (r.whole) {
    // a team has at least as many threads as a block has 16-byte pieces
    const int piece = (threadIdx.x % kTeam) * 16;
    const bool copies = piece < bytes;
    int side = 0;
    for (int h = h0; h < h1; h += kStep, side ^= 1) {
      Raw<T> ck[kStep], cv[kStep];
#pragma unroll
      for (int u = 0; u < kStep; ++u) ck[u] = xk[u], cv[u] = xv[u];
      if (h + kStep < h1) fetch(h + kStep);
#pragma unroll
      for (int u = 0; u < kStep; ++u)
        put<T>(s_bytes[side][u][r.unit], at, ck[u], cv[u], f0 < p.dk, f0 < p.dv, t == 0);
      // the team's blocks are together (the other side's copies were read before this)
      asm volatile("bar.sync %0, %1;" ::"r"(1 + r.unit), "n"(kTeam) : "memory");
#pragma unroll
      for (int u = 0; u < kStep; ++u, block += head_bytes)
        if (copies && h + u < h1)
          *reinterpret_cast<uint4*>(block + piece) = *reinterpret_cast<const uint4*>(s_bytes[side][u][r.unit] + piece);
    }
  } else {
    for (int h = h0; h < h1; h += kStep) {
#pragma unroll
      for (int u = 0; u < kStep; ++u, block += head_bytes)
        put<T>(block, at, xk[u], xv[u], mine_k && h + u < h1, mine_v && h + u < h1, t == 0);
      if (h + kStep < h1) fetch(h + kStep);
    }
  }
}

// Code pairs (nibbles 4 j and 4 j + 16 of w, less 8) times the scale, rounded to bf16 once: the codes
// are exact in bf16, and the product of two bf16 values is rounded from the exact one.
__device__ __forceinline__ uint32_t scaled_pair(uint32_t w, int j, __nv_bfloat162 s) {
  uint32_t x = (w >> (4 * j) & 0x000f000fu) | 0x43004300u;   // 128 + n
  const __nv_bfloat162 bias = __halves2bfloat162(__ushort_as_bfloat16(0x4308), __ushort_as_bfloat16(0x4308));
  const __nv_bfloat162 y = __hmul2(__hsub2(*reinterpret_cast<__nv_bfloat162*>(&x), bias), s);
  return *reinterpret_cast<const uint32_t*>(&y);
}
// Eight features of w's nibbles in the keys' order (even features in the low half) to p.
__device__ __forceinline__ void store_scaled(__nv_bfloat16* p, uint32_t w, uint32_t s) {
  const __nv_bfloat162 s2 = __halves2bfloat162(__ushort_as_bfloat16(uint16_t(s)), __ushort_as_bfloat16(uint16_t(s)));
  *reinterpret_cast<uint4*>(p) =
      make_uint4(scaled_pair(w, 0, s2), scaled_pair(w, 1, s2), scaled_pair(w, 2, s2), scaled_pair(w, 3, s2));
}
__device__ __forceinline__ void store_scaled(float* p, uint32_t w, uint32_t s) {
  const float scale = __uint_as_float(s << 16);
  float x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = float(int((w >> (16 * (e & 1) + 4 * (e >> 1))) & 15u) - 8) * scale;
  store8(p, x);
}
// The same order from the values' two 16-bit words (features 0-3 and 4-7): evens low, odds high.
__device__ __forceinline__ uint32_t reorder(uint32_t a, uint32_t b) {
  const uint32_t even = (a & 0x000fu) | (a >> 4 & 0x00f0u) | (b & 0x000fu) << 8 | (b >> 4 & 0x00f0u) << 8;
  const uint32_t odd = (a >> 4 & 0x000fu) | (a >> 8 & 0x00f0u) | (b >> 4 & 0x000fu) << 8 | (b >> 8 & 0x00f0u) << 8;
  return even | odd << 16;
}
__device__ __forceinline__ void store_all(__nv_bfloat16* p, float x) {
  const float y[8] = {x, x, x, x, x, x, x, x};
  store8(p, y);
}
__device__ __forceinline__ void store_all(float* p, float x) {
  const float y[8] = {x, x, x, x, x, x, x, x};
  store8(p, y);
}

// Bound by the stores of the widened rows: 3 x 8 x 16001 x (128 + 128) 48.2 us = 5.2 TB/s, the same with
// five or six CTAs on an SM instead of four.
template <typename T, int LPR>
__global__ void __launch_bounds__(kThreads)
kv4_read_kernel(View k, View v, uint8_t* pool, const int32_t* table, const int32_t* pos, Dims p) {
  constexpr int kUnits = Row<LPR>::kUnits, kTeam = LPR * kBlock;
  __shared__ __align__(16) uint8_t s_bytes[2][2][kUnits][kMostBytes];
  wait_for_previous();
  const Row<LPR> r(pool, table, pos, p);
  const int f0 = r.lane * 8, g = r.lane >> 2, t = r.lane & 3;
  const int bytes = block_bytes(p.dk, p.dv), gk = p.dk / kGroup, gv = p.dv / kGroup;
  const int64_t head_bytes = int64_t(p.page / kBlock) * bytes;
  const int h0 = int(blockIdx.y) * p.hp, h1 = min(h0 + p.hp, p.H);
  T* to_k = static_cast<T*>(k.p) + r.b * k.sb + r.n * k.sn + f0;
  T* to_v = static_cast<T*>(v.p) + r.b * v.sb + r.n * v.sn + f0;
  const bool mine_k = r.live && f0 < p.dk, mine_v = r.live && f0 < p.dv;
  const int at_k = key_word(r.tok, t, g, gk), at_ks = key_scales(p.dk, p.dv) + (r.tok * gk + g) * 2;
  const int at_v = value_word(p.dk, r.tok, 2 * t, g, gv) + (r.tok & 1) * 2;
  const int at_v1 = value_word(p.dk, r.tok, 2 * t + 1, g, gv) + (r.tok & 1) * 2;
  const int at_vs = value_scales(p.dk, p.dv) + (r.tok * gv + g) * 2;
  // whole blocks, two heads at a time: 16 bytes a thread of each, the next ones on their way while
  // these are taken apart (a team has at least as many threads as a block has such pieces)
  const int piece = (threadIdx.x % kTeam) * 16;
  const bool copies = r.whole && piece < bytes;
  const uint8_t* block = r.block + h0 * head_bytes;
  to_k += h0 * k.sh, to_v += h0 * v.sh;
  uint4 a[2];
  auto fetch = [&](const uint8_t* from, int h) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
      if (copies && h + u < h1) a[u] = *reinterpret_cast<const uint4*>(from + u * head_bytes + piece);
  };
  fetch(block, h0);
  for (int h = h0; h < h1; h += 2) {
    uint8_t* mid = s_bytes[(h - h0) >> 1 & 1][0][r.unit];
    if (copies) {
#pragma unroll
      for (int u = 0; u < 2; ++u) *reinterpret_cast<uint4*>(mid + u * kUnits * kMostBytes + piece) = a[u];
      fetch(block + 2 * head_bytes, h + 2);
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      if (h + u >= h1) break;
      if (r.block == nullptr) {   // padding: zeros; no such place: NaN
        const float fill = r.at < 0 ? 0.f : __int_as_float(0x7fc00000);
        if (mine_k) store_all(to_k, fill);
        if (mine_v) store_all(to_v, fill);
      } else {
        const uint8_t* from = r.whole ? mid + u * kUnits * kMostBytes : block;
        if (mine_k) store_scaled(to_k, *reinterpret_cast<const uint32_t*>(from + at_k), *reinterpret_cast<const uint16_t*>(from + at_ks));
        if (mine_v)
          store_scaled(to_v, reorder(*reinterpret_cast<const uint16_t*>(from + at_v), *reinterpret_cast<const uint16_t*>(from + at_v1)),
                       *reinterpret_cast<const uint16_t*>(from + at_vs));
      }
      block += head_bytes, to_k += k.sh, to_v += v.sh;
    }
  }
}

template <typename T, int LPR>
cudaError_t run(const Kv4MoveArgs& a, const Dims& p, bool write, dim3 grid) {
  uint8_t* pool = static_cast<uint8_t*>(a.c.pool);
  return launch_overlapped(write ? kv4_write_kernel<T, LPR> : kv4_read_kernel<T, LPR>, grid,
                           dim3(kThreads), 0, a.stream, a.k, a.v, pool, a.c.table, a.pos, p);
}

int launch(const Kv4MoveArgs& a, bool write, char* msg, size_t msglen) {
  int sms = 0;
  cudaError_t e = device_sm_count(&sms);
  if (e != cudaSuccess) {
    snprintf(msg, msglen, "cache: SM count: %s", cudaGetErrorString(e));
    return 5;
  }
  // Sequences shorter than two blocks hardly fill any: their tokens are taken 16 at a time whosever
  // they are.  Positions that begin inside a block may need one unit more.
  const bool flat = a.N < 2 * kBlock;
  const int64_t units = flat ? 0 : (a.N + 2 * kBlock - 2) / kBlock;
  const int64_t all = flat ? (a.B * a.N + kBlock - 1) / kBlock : a.B * units;
  const int lpr = a.c.dk <= 64 && a.c.dv <= 64 ? 8 : 16;
  const int64_t per = kThreads / (lpr * kBlock), x = (all + per - 1) / per;
  if (all > 0x7fffffffLL || (flat && a.B * a.N > 0x7fffffffLL)) {
    snprintf(msg, msglen, "cache: too many rows for one launch");
    return 3;
  }
  // heads of a CTA: all of them, unless that leaves SMs with less than eight CTAs
  int hp = a.c.H;
  while (hp > 1 && x * ((a.c.H + hp - 1) / hp) < int64_t(sms) * 8) hp = (hp + 1) / 2;
  while ((a.c.H + hp - 1) / hp > 65535) hp *= 2;
  const Dims p{a.B, a.N, a.c.n_pages, a.c.max_pages, uint32_t(units), uint32_t(all), flat, a.c.H, a.c.page, a.c.dk, a.c.dv, hp};
  const dim3 grid(unsigned(x), unsigned((a.c.H + hp - 1) / hp));
  if (a.f32)
    e = lpr == 8 ? run<float, 8>(a, p, write, grid) : run<float, 16>(a, p, write, grid);
  else
    e = lpr == 8 ? run<__nv_bfloat16, 8>(a, p, write, grid) : run<__nv_bfloat16, 16>(a, p, write, grid);
  if (e != cudaSuccess) {
    snprintf(msg, msglen, "cache launch: %s", cudaGetErrorString(e));
    return 5;
  }
  return 0;
}

}  // namespace

int launch_kv4_write(const Kv4MoveArgs& a, char* msg, size_t msglen) {
  return launch(a, true, msg, msglen);
}
int launch_kv4_read(const Kv4MoveArgs& a, char* msg, size_t msglen) {
  return launch(a, false, msg, msglen);
}

cudaError_t kv4_read_and_clear_status(unsigned* value) {
  cudaError_t e = cudaMemcpyFromSymbol(value, g_moa_kv4_status, sizeof(unsigned));
  if (e != cudaSuccess || *value == 0) return e;
  const unsigned zero = 0;
  return cudaMemcpyToSymbol(g_moa_kv4_status, &zero, sizeof(unsigned));
}

}  // namespace moa
