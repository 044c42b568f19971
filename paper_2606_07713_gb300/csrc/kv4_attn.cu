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
// Rounding: bf16 queries enter exactly; the weights p sv are rounded to bf16 once (relative
// 2^-9, as in the other bf16 forward).  fp32 queries and weights enter as three bf16 terms each
// (24 bits), so the fp32 form is fp32-accurate on the same instructions.  Scores, maxima, sums
// and outputs accumulate in fp32.
//
// What bounds it: for single tokens the cache's bytes, 9/16 a value, and close behind it the
// instructions that widen codes (about two a value and lane).  Tokens lie on the 16 rows of
// mma.m16n8k16 and queries on its 8 columns: a decoding step has few queries, and the other way
// round half of the tensor work would be padding.
//
// Layout of the work: a CTA owns up to 8 NT query rows of one key head and a range of 16-token
// blocks; its four warps take turns at tiles of SUB blocks, each with its own ring of bulk copies,
// running maximum, sum and output, joined through shared memory at the end.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdio>

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
// Transpose of an 8 x 8 matrix of 16-bit values held one row (two values a lane) per four lanes.
__device__ __forceinline__ uint32_t transpose8(uint32_t a) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
// Four pairs of codes of a word as bf16 pairs of integers -8 .. 7: 0x4300 | n is 128 + n.
__device__ __forceinline__ void widen(uint32_t w, uint32_t* r) {
  const __nv_bfloat162 bias = __halves2bfloat162(__ushort_as_bfloat16(0x4308), __ushort_as_bfloat16(0x4308));
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    uint32_t x = ((w >> (4 * j)) & 0x000f000fu) | 0x43004300u;
    const __nv_bfloat162 y = __hsub2(*reinterpret_cast<__nv_bfloat162*>(&x), bias);
    r[j] = *reinterpret_cast<const uint32_t*>(&y);
  }
}
__device__ __forceinline__ float bf16_bits(uint32_t b) { return __uint_as_float(b << 16); }

template <int G>
__device__ __forceinline__ void load_words(uint32_t* w, const uint8_t* p) {
  if constexpr (G == 4) {
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

struct Params {
  int64_t q_sb, q_sh, q_sn, o_sb, o_sh, o_sn;
  int64_t n_pages, max_pages;
  int64_t N, max_len;
  int Hk, G, blocks_per_page;
  int n_splits, chunk_blocks;
  int64_t n_tiles;
  float scale;
  bool causal;
  uint64_t wait_limit_ns;
};

template <int DK, int DV, int NT, int TERMS>
struct Cfg {
  static constexpr int kSub = NT == 1 ? 4 : NT == 2 ? 2 : 1;  // 16-token blocks of a tile
  static constexpr int kBytes = block_bytes(DK, DV);
  static constexpr int kStages = 12 / kSub;
  static constexpr int kRing = kSub * kStages * kBytes;         // one warp's ring
  static constexpr int kOStride = DV + 4;                       // padded row of the final join
  static constexpr int kJoin = kWarps * 8 * NT * (kOStride + 2) * 4;
  static constexpr int kData = kWarps * kRing > kJoin ? kWarps * kRing : kJoin;
  // queries in the order of the matrix operands: [nt][term][group][lane] 16 bytes
  static constexpr int kQ = NT * TERMS * (DK / 32) * 32 * 16;
  static constexpr int kOffQ = kData;
  static constexpr int kOffBar = kOffQ + kQ;
  static constexpr int kOffMisc = kOffBar + kWarps * kStages * 8;
  static constexpr int kSmem = kOffMisc + 16;
  static_assert(kBytes % 16 == 0, "bulk copies are whole 16-byte units");
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

template <typename T, int DK, int DV, int NT, int TERMS>
__global__ void __launch_bounds__(kThreads)
kv4_attn_kernel(const T* __restrict__ Q, const uint8_t* __restrict__ pool,
                const int32_t* __restrict__ table, const int32_t* __restrict__ lens,
                T* __restrict__ O, float* __restrict__ lse, float* __restrict__ part_o,
                float* __restrict__ part_ml, Params p) {
  using C = Cfg<DK, DV, NT, TERMS>;
  constexpr int GK = DK / 32, GV = DV / 32;
  extern __shared__ __align__(128) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, t = lane & 3;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + C::kOffMisc);
  const WaitCtl wc{abort_flag, p.wait_limit_ns, 0u, &g_moa_kv4_attn_status};

  const int split = int(blockIdx.x % unsigned(p.n_splits));
  const int64_t item = blockIdx.x / unsigned(p.n_splits);
  const int64_t tile = item % p.n_tiles;
  const int h = int(item / p.n_tiles % p.Hk);
  const int64_t b = item / p.n_tiles / p.Hk;
  const int64_t rows = p.N * p.G;
  const int64_t r0 = tile * (8 * NT);

  // tokens that the tile's rows may see
  int64_t len = lens[b];
  if (len < 0 || len > p.max_len) {
    if (threadIdx.x == 0) atomicExch(&g_moa_kv4_attn_status, kErrIndex);
    len = len < 0 ? 0 : p.max_len;
  }
  auto limit = [&](int64_t r) -> int64_t {  // visible tokens of row r
    if (!p.causal) return len;
    const int64_t n = len - p.N + r / p.G + 1;
    return n < 0 ? 0 : n;
  };
  const int64_t last_row = r0 + 8 * NT < rows ? r0 + 8 * NT - 1 : rows - 1;
  const int all_limit = int(limit(r0));          // every row sees these
  const int any_limit = int(limit(last_row));    // no row sees more
  const int n_blocks = (any_limit + kBlock - 1) / kBlock;
  const int first = split * p.chunk_blocks;
  const int end = first + p.chunk_blocks < n_blocks ? first + p.chunk_blocks : n_blocks;

  uint8_t* ring = smem + warp * C::kRing;
  const uint32_t ring_s = smem_u32(ring);
  const uint32_t bars = smem_u32(smem + C::kOffBar) + warp * C::kStages * 8;
  if (lane == 0) {
    for (int s = 0; s < C::kStages; ++s) mbar_init(bars + 8 * s, 1);
    fence_barrier_init();
  }
  if (threadIdx.x == 0) *abort_flag = 0;
  // queries -> shared memory, split into their terms, in operand order
  for (int i = threadIdx.x; i < NT * GK * 32; i += kThreads) {
    const int ln = i & 31, gi = (i >> 5) % GK, nt = (i >> 5) / GK;
    const int64_t r = r0 + nt * 8 + (ln >> 2);
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 0.f;
    if (r < rows) {
      const T* src = Q + b * p.q_sb + (int64_t(h) * p.G + r % p.G) * p.q_sh + (r / p.G) * p.q_sn +
                     32 * gi + 8 * (ln & 3);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = float(src[e]);
    }
    uint32_t w[4][TERMS];
#pragma unroll
    for (int e = 0; e < 4; ++e) split_pair<TERMS>(x[2 * e], x[2 * e + 1], w[e]);
#pragma unroll
    for (int k = 0; k < TERMS; ++k)
      *reinterpret_cast<uint4*>(smem + C::kOffQ + (((nt * TERMS + k) * GK + gi) * 32 + ln) * 16) =
          make_uint4(w[0][k], w[1][k], w[2][k], w[3][k]);
  }
  __syncthreads();

  float o[NT][DV / 16][4];
  float m[NT][2], l[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    m[n][0] = m[n][1] = -INFINITY;
    l[n][0] = l[n][1] = 0.f;
#pragma unroll
    for (int i = 0; i < DV / 16; ++i) o[n][i][0] = o[n][i][1] = o[n][i][2] = o[n][i][3] = 0.f;
  }
  int lim[NT][2];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int64_t r = r0 + n * 8 + 2 * t + c;
      lim[n][c] = r < rows ? int(limit(r)) : any_limit;
    }

  const int n_mine = end - first;                       // blocks of this CTA's range
  const int n_tiles = n_mine <= 0 ? 0 : (n_mine + C::kSub - 1) / C::kSub;
  const float c2 = p.scale * kLog2e;
  const int32_t* pages = table + b * p.max_pages;
  // The page of block `lane` (< kSub) of this warp's tile number `it` (0, 1, ...), -1 if none.
  auto page_of = [&](int it) -> int {
    const int blk = first + (warp + it * kWarps) * C::kSub + lane;
    if (lane >= C::kSub || blk >= end) return -2;
    const int pg = pages[blk / p.blocks_per_page];
    if (pg < 0 || pg >= p.n_pages) {
      atomicExch(&g_moa_kv4_attn_status, kErrIndex);
      return -1;
    }
    return pg;
  };
  // Starts the copies of tile `it` into its stage; returns the blocks copied, one bit each.
  auto issue = [&](int it, int pg) -> uint32_t {
    const uint32_t got = __ballot_sync(0xffffffffu, pg >= 0);
    const int s = it % C::kStages;
    if (lane == 0) mbar_arrive_expect_tx(bars + 8 * s, __popc(got) * C::kBytes);
    __syncwarp();
    if (pg >= 0) {
      const int blk = first + (warp + it * kWarps) * C::kSub + lane;
      const int64_t at = (int64_t(pg) * p.Hk + h) * p.blocks_per_page + blk % p.blocks_per_page;
      bulk_load(ring_s + (s * C::kSub + lane) * C::kBytes, pool + at * C::kBytes, C::kBytes, bars + 8 * s);
    }
    return got;
  };
  const int my_tiles = n_tiles > warp ? (n_tiles - warp + kWarps - 1) / kWarps : 0;
  uint64_t present = 0;  // copied blocks of the tiles in flight, kSub bits a stage
  int issued = 0;
  for (; issued < my_tiles && issued < C::kStages; ++issued)
    present |= uint64_t(issue(issued, page_of(issued))) << (issued * C::kSub);
  int next_page = issued < my_tiles ? page_of(issued) : -2;

  bool ok = true;
  for (int it = 0; it < my_tiles; ++it) {
    const int s = it % C::kStages;
    ok = wait_bounded(bars + 8 * s, uint32_t(it / C::kStages) & 1u, wc);
    ok = __all_sync(0xffffffffu, ok);
    if (!ok) break;
    const uint8_t* st = ring + s * C::kSub * C::kBytes;
    const int tok0 = (first + (warp + it * kWarps) * C::kSub) * kBlock;
    const uint32_t got = uint32_t(present >> (s * C::kSub)) & ((1u << C::kSub) - 1);
    const bool plain = got == (1u << C::kSub) - 1 && tok0 + C::kSub * kBlock <= all_limit;

    // scores of the tile, in log2 units: sc[sub][nt]: (token g, rows 2t, 2t+1), (token g+8, ...)
    float sc[C::kSub][NT][4];
#pragma unroll
    for (int sub = 0; sub < C::kSub; ++sub) {
      const uint8_t* blk = st + sub * C::kBytes;
      uint32_t kw[2][GK];
      float ks[2][GK];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        load_words<GK>(kw[r], blk + ((g + 8 * r) * 4 + t) * GK * 4);
        load_scales<GK>(ks[r], blk + key_scales(DK, DV) + (g + 8 * r) * GK * 2);
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) sc[sub][n][0] = sc[sub][n][1] = sc[sub][n][2] = sc[sub][n][3] = 0.f;
#pragma unroll
      for (int gi = 0; gi < GK; ++gi) {
        uint32_t lo[4], hi[4];
        widen(kw[0][gi], lo);
        widen(kw[1][gi], hi);
        const uint32_t a0[4] = {lo[0], hi[0], lo[1], hi[1]}, a1[4] = {lo[2], hi[2], lo[3], hi[3]};
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = 0; k < TERMS; ++k) {
            const uint4 q = *reinterpret_cast<const uint4*>(
                smem + C::kOffQ + (((n * TERMS + k) * GK + gi) * 32 + lane) * 16);
            mma_16816(acc, a0, q.x, q.y);
            mma_16816(acc, a1, q.z, q.w);
          }
          sc[sub][n][0] += ks[0][gi] * acc[0];
          sc[sub][n][1] += ks[0][gi] * acc[1];
          sc[sub][n][2] += ks[1][gi] * acc[2];
          sc[sub][n][3] += ks[1][gi] * acc[3];
        }
      }
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) sc[sub][n][e] *= c2;
      if (!plain) {
        const int tok = tok0 + sub * kBlock + g;
        const bool here = (got >> sub) & 1u;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!here || tok + (e >> 1) * 8 >= lim[n][e & 1]) sc[sub][n][e] = -INFINITY;
      }
    }
    // running maximum and sum
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float x = -INFINITY;
#pragma unroll
        for (int sub = 0; sub < C::kSub; ++sub) x = fmaxf(x, fmaxf(sc[sub][n][c], sc[sub][n][2 + c]));
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
        const float mn = fmaxf(m[n][c], x);
        const float base = mn == -INFINITY ? 0.f : mn;  // no visible token yet: weights stay 0
        const float alpha = ex2_approx(m[n][c] - base);
        m[n][c] = mn;
        float sum = 0.f;
#pragma unroll
        for (int sub = 0; sub < C::kSub; ++sub)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const float e = ex2_approx(sc[sub][n][2 * r + c] - base);
            sc[sub][n][2 * r + c] = e;
            sum += e;
          }
        l[n][c] = l[n][c] * alpha + sum;
#pragma unroll
        for (int i = 0; i < DV / 16; ++i) {
          o[n][i][c] *= alpha;
          o[n][i][2 + c] *= alpha;
        }
      }
    // o += (p sv) codes
#pragma unroll
    for (int sub = 0; sub < C::kSub; ++sub) {
      const uint8_t* blk = st + sub * C::kBytes;
      uint32_t vw[2][GV];
      float vs[2][GV];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        load_words<GV>(vw[r], blk + value_codes(DK) + ((r * 8 + g) * 4 + t) * GV * 4);
        load_scales<GV>(vs[r], blk + value_scales(DK, DV) + (g + 8 * r) * GV * 2);
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
            w[e] = sc[sub][n][e] * vs[e >> 1][gi];
            // a hidden token's scale may be anything: its weight is zero whatever that is
            if (!plain && sc[sub][n][e] == 0.f) w[e] = 0.f;
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
    // the stage is free again: start its next tile
    __syncwarp();
    if (issued < my_tiles) {
      const uint64_t bits = ((uint64_t(1) << C::kSub) - 1) << (s * C::kSub);
      present = (present & ~bits) | (uint64_t(issue(issued, next_page)) << (s * C::kSub));
      ++issued;
      next_page = issued < my_tiles ? page_of(issued) : -2;
    }
  }
  if (!ok) {  // a wait ran out: let the copies in flight land before the memory is reused
    for (int s = 0; s < C::kStages; ++s) {
      const int it = issued - 1 - ((issued - 1 - s) % C::kStages + C::kStages) % C::kStages;
      if (it >= 0) wait_quiesce(bars + 8 * s, uint32_t(it / C::kStages) & 1u, p.wait_limit_ns, &g_moa_kv4_attn_status);
    }
  }
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) l[n][c] += __shfl_xor_sync(0xffffffffu, l[n][c], d);

  // join the warps
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
        jm[row] = m[n][c];
        jl[row] = l[n][c];
      }
#pragma unroll
      for (int gi = 0; gi < GV; ++gi)
        *reinterpret_cast<float4*>(jo + row * C::kOStride + 32 * gi + 4 * g) = make_float4(
            o[n][2 * gi][c], o[n][2 * gi][2 + c], o[n][2 * gi + 1][c], o[n][2 * gi + 1][2 + c]);
    }
  __syncthreads();
  for (int i = threadIdx.x; i < 8 * NT * (DV / 4); i += kThreads) {
    const int row = i / (DV / 4), col = i % (DV / 4) * 4;
    const int64_t r = r0 + row;
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
    if (p.n_splits > 1) {
      const int64_t at = (item * p.n_splits + split) * (8 * NT) + row;
      store4(part_o + at * DV + col, x);
      if (col == 0) {
        part_ml[2 * at] = M;
        part_ml[2 * at + 1] = L;
      }
    } else {
      const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] *= inv;
      const int64_t head = int64_t(h) * p.G + r % p.G, i_n = r / p.G;
      store4(O + b * p.o_sb + head * p.o_sh + i_n * p.o_sn + col, x);
      if (lse != nullptr && col == 0)
        lse[(b * p.Hk * p.G + head) * p.N + i_n] = L == 0.f ? -INFINITY : (M + lg2_approx(L)) * kLn2;
    }
  }
}

// Joins the ranges of one query row: one warp a row.
template <typename T, int DV>
__global__ void __launch_bounds__(128)
kv4_attn_join_kernel(const float* __restrict__ part_o, const float* __restrict__ part_ml,
                     T* __restrict__ O, float* __restrict__ lse, int rows_tile, int64_t n_rows_all,
                     Params p) {
  const int64_t id = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (id >= n_rows_all) return;
  const int64_t rows = p.N * p.G;
  const int64_t r = id % rows, bh = id / rows;
  const int h = int(bh % p.Hk);
  const int64_t b = bh / p.Hk;
  const int64_t item = bh * p.n_tiles + r / rows_tile;
  const int64_t at0 = item * p.n_splits * rows_tile + r % rows_tile;
  float M = -INFINITY;
  for (int s = lane; s < p.n_splits; s += 32) M = fmaxf(M, part_ml[2 * (at0 + int64_t(s) * rows_tile)]);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, d));
  const float base = M == -INFINITY ? 0.f : M;
  float L = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
  for (int s = 0; s < p.n_splits; ++s) {
    const int64_t at = at0 + int64_t(s) * rows_tile;
    const float f = ex2_approx(part_ml[2 * at] - base);
    L += f * part_ml[2 * at + 1];
    if (lane * 4 < DV) {
      const float4 v = *reinterpret_cast<const float4*>(part_o + at * DV + lane * 4);
      x[0] += f * v.x, x[1] += f * v.y, x[2] += f * v.z, x[3] += f * v.w;
    }
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] *= inv;
  const int64_t head = int64_t(h) * p.G + r % p.G, i_n = r / p.G;
  if (lane * 4 < DV) store4(O + b * p.o_sb + head * p.o_sh + i_n * p.o_sn + lane * 4, x);
  if (lse != nullptr && lane == 0)
    lse[(b * p.Hk * p.G + head) * p.N + i_n] = L == 0.f ? -INFINITY : (M + lg2_approx(L)) * kLn2;
}

template <typename T, int DK, int DV, int NT, int TERMS>
cudaError_t run(const Kv4AttnArgs& a, const Kv4Plan& plan, const Params& p) {
  using C = Cfg<DK, DV, NT, TERMS>;
  const void* f = reinterpret_cast<const void*>(kv4_attn_kernel<T, DK, DV, NT, TERMS>);
  cudaError_t e = ensure_smem_limit(f, C::kSmem);
  if (e != cudaSuccess) return e;
  const int64_t items = a.B * a.c.H * plan.n_tiles;
  float* part_o = static_cast<float*>(a.ws);
  float* part_ml = part_o + items * plan.n_splits * plan.rows_tile * DV;
  kv4_attn_kernel<T, DK, DV, NT, TERMS><<<unsigned(items * plan.n_splits), kThreads, C::kSmem, a.stream>>>(
      static_cast<const T*>(a.q.p), static_cast<const uint8_t*>(a.c.pool), a.c.table, a.lens,
      static_cast<T*>(a.o.p), a.lse, part_o, part_ml, p);
  e = cudaGetLastError();
  if (e != cudaSuccess || plan.n_splits == 1) return e;
  const int64_t n_rows = a.B * a.Hq * a.N;
  kv4_attn_join_kernel<T, DV><<<unsigned((n_rows + 3) / 4), 128, 0, a.stream>>>(
      part_o, part_ml, static_cast<T*>(a.o.p), a.lse, plan.rows_tile, n_rows, p);
  return cudaGetLastError();
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

Kv4Plan kv4_attn_plan(int64_t B, int64_t Hk, int64_t G, int64_t N, int64_t max_len, int sms) {
  Kv4Plan p;
  const int64_t rows = G * N;
  p.rows_tile = rows <= 8 ? 8 : rows <= 16 ? 16 : 32;
  p.n_tiles = (rows + p.rows_tile - 1) / p.rows_tile;
  const int64_t items = B * Hk * p.n_tiles;
  const int64_t blocks = (max_len + kv4::kBlock - 1) / kv4::kBlock;
  // enough ranges for four CTAs on every SM, none shorter than one tile of 64 tokens a warp
  int64_t splits = (int64_t(sms) * 4 + items - 1) / items;
  const int64_t most = (blocks + 15) / 16;
  splits = splits < 1 ? 1 : splits > most ? most : splits;
  if (splits < 1) splits = 1;
  int64_t chunk = (blocks + splits - 1) / splits;
  chunk = (chunk + 3) / 4 * 4;
  if (chunk < 1) chunk = 1;
  p.chunk_blocks = int(chunk);
  p.n_splits = int((blocks + chunk - 1) / chunk);
  if (p.n_splits < 1) p.n_splits = 1;
  return p;
}

size_t kv4_attn_workspace(int64_t B, int64_t Hk, int64_t dv, const Kv4Plan& p) {
  if (p.n_splits <= 1) return 0;
  return size_t(B) * Hk * p.n_tiles * p.n_splits * p.rows_tile * (4 * dv + 8);
}

int launch_kv4_attn(const Kv4AttnArgs& a, const Kv4Plan& plan, char* msg, size_t msglen) {
  Params p{};
  p.q_sb = a.q.sb, p.q_sh = a.q.sh, p.q_sn = a.q.sn;
  p.o_sb = a.o.sb, p.o_sh = a.o.sh, p.o_sn = a.o.sn;
  p.n_pages = a.c.n_pages, p.max_pages = a.c.max_pages;
  p.N = a.N, p.max_len = a.max_len;
  p.Hk = a.c.H, p.G = int(a.Hq / a.c.H);
  p.blocks_per_page = a.c.page / kv4::kBlock;
  p.n_splits = plan.n_splits, p.chunk_blocks = plan.chunk_blocks;
  p.n_tiles = plan.n_tiles;
  p.scale = a.scale;
  p.causal = a.causal;
  p.wait_limit_ns = wait_limit_ns();
  if (a.B * a.c.H * plan.n_tiles > 0x7fffffffLL / plan.n_splits || (a.B * a.Hq * a.N + 3) / 4 > 0x7fffffffLL) {
    snprintf(msg, msglen, "cache attention: too many query rows for one launch");
    return 3;
  }
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
