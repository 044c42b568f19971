// Causal attention with a sliding window and first tokens that stay visible, bf16, on the fifth-generation
// tensor cores (tcgen05 + TMEM + TMA), sm_103a.  Keys and values lie in dense tensors or in the pages of a
// cache; any number of query rows, from a decoding step's to a training batch's.
//
// Mathematics: o_i = sum_j p_ij v_j / l_i over the tokens j that row i sees (window.cuh), p_ij = 2^(c s_ij - m_i),
// c = scale log2 e, running maximum m_i and sum l_i: one pass over the tokens.  S = Q K^T and O += P V are
// 128 x 128 tiles in TMEM; maximum, exponentials and sums are fp32, P is rounded to bf16 (the operand type).
//
// Rows of a key head are counted position by position: row r of a 128-row tile is position r / GC and query
// head r % GC of the group (GC = min(G, 128) heads), so that a tile covers few positions: a window then needs few
// tiles of tokens, and a decoding step's heads share one tile.  TMA puts them in that order itself (a
// five-dimensional map: feature, head of the group, position, key head, sequence); heads and positions past the
// end are zeros.  Keys and values come by TMA as well, a page (or the part of it that divides 128) a copy, straight from
// the pool: a row's 128-byte panels lie side by side for every eight tokens, so that one copy brings all of them (with a
// copy for each panel, 2048 queries against 16384 tokens in pages of 16 took 460 us instead of 345, 48 single tokens against
// 8192 each 327 instead of 288).  A page that no row of the work item sees is asked for past the pool's end, which fills zeros: its
// entry in the table may be anything.
//
// Work items (key head, chunk of heads, 128 QT rows) count in 128-token tiles; all items' tiles are cut into equal
// shares, one for each SM (one CTA fills an SM), and a CTA walks over its share.  Cut items are joined by a
// second kernel.  Few items (of one row tile then) go to a cluster each, whose CTAs join them in the same launch.  QT = 2 where there are more rows than a tile holds (and no clusters): keys and values in shared memory then serve
// twice the rows.
//
// Hidden tokens: a tile that some row sees only in part is masked by words of bits, -infinity in place of the
// score.  Past a sequence's end the cache may hold anything: the softmax threads zero the values' rows there in
// shared memory before the product.  Any other hidden value that is not finite reaches all rows of the product (0 * NaN).  So an
// item with an output that is not finite, though its row's sum of weights is a number, is computed once more when the CTA is done
// with the others (redo_piece): tile after tile without overlap, with the values of its partly hidden tiles looked through in shared
// memory; those that are not finite are taken out before the product, and added at the end to the rows that do see them.  A call all of
// whose values are infinite or NaN takes some five times as long as one without; other calls pay nothing.
//
// What bounds it.  Many rows: a softmax warp's chain of score load, maximum, 128 exponentials and stores beside the products
// (32768 tokens, 32 / 8 heads of 128, window 4096: 1515 us = 1.36 PFLOP/s of what is seen, tensor pipe 64 %; 2048 queries against 16384 cached
// tokens: 352 us = 1.46 PFLOP/s).  Few rows: memory (48 sequences, 1.2 GB of keys and values: 190 us, 6.3 TB/s), or latency (one
// token, window 1024: 10.7 us).
//
// CTA organisation (QT = 2): warps 0-3 and 4-7 softmax and epilogue of row tiles 0 and 1 (thread = row), then the
// products of tile 0 (and TMEM allocation), TMA, the products of tile 1, the share's items for the other roles.
// QT = 1: warps 0-3, then four such warps of which one idles.  K and V tiles stream through a ring in the
// order of use, K0 K1 V0 K2 V1 ...  Waits are bounded: on expiry MOA_ERR_DEVICE_TIMEOUT is recorded and every
// role leaves its loop.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cfloat>
#include <cstdio>

#include "internal.h"
#include "ops_internal.h"
#include "ptx.cuh"
#include "tc_common.cuh"
#include "window.cuh"
#include "window_tc.cuh"

namespace moa {

__device__ unsigned int g_moa_window_tc_status = 0;

namespace {

using namespace ptx;
using namespace tc;
using win::below, win::describable, win::map_stride, win::tma_load_4d, win::tma_load_5d;

constexpr int kBM = 128;              // rows of a row tile (= TMEM lanes)
constexpr int kBN = 128;              // tokens of a tile
// What an item costs besides its tiles, in tiles (48 sequences of one query with 0, 1, 2, 4: 204, 195, 189, 192 us; 4 x 16 heads x
// 2048 x 64, causal, with 1, 2, 3, 4: 66.7, 64.7, 65.2, 66.7, a chunk of 2048 queries 363, 364, 361, 363).
__host__ __device__ constexpr int item_units(int QT) { return QT == 2 ? 3 : 2; }
constexpr int kAgain = 256;           // pieces of a share that are marked one by one; the last bit is for all that follow
constexpr float kRescaleLog2 = 8.f;   // the running maximum may lag by this: weights up to 2^8
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

template <int DK, int DV, int QT>
struct Cfg {
  static constexpr int kSoftmax = 128 * QT, kThreads = kSoftmax + 128;
  static constexpr int kRows = kBM * QT;
  static constexpr int kMmaWarp0 = 4 * QT, kLoadWarp = kMmaWarp0 + 1, kMmaWarp1 = kMmaWarp0 + 2, kWalkWarp = kMmaWarp0 + 3;
  // QT = 2: 256 kRegsSoftmax + 128 kRegsCtrl is what the launch allocates (the host checks it)
  static constexpr int kRegsLaunch = 168, kRegsSoftmax = 208, kRegsCtrl = 88;
  static_assert(256 * kRegsSoftmax + 128 * kRegsCtrl <= 384 * kRegsLaunch, "register split");
  static constexpr int kPanelBytes = 128 * 128;   // 64 columns of 128 rows, 128-byte swizzle
  static constexpr int kQTileBytes = kBM * DK * 2;
  static constexpr int kKTileBytes = kBN * DK * 2, kVTileBytes = kBN * DV * 2;
  static constexpr int kStageBytes = kKTileBytes > kVTileBytes ? kKTileBytes : kVTileBytes;
  static constexpr bool kSharedS = DV == 128 && QT == 2;   // one S for both row tiles
  static constexpr int kOffKV = QT * kQTileBytes;
  static constexpr int kStages = (229376 - kOffKV) / kStageBytes < 8 ? (229376 - kOffKV) / kStageBytes : 8;
  static constexpr int kOffBar = kOffKV + kStages * kStageBytes;
  // barriers: full[NS], empty[NS], q_full, q_empty, drain, s_full[2], p_ready[2], o_done[2], s_free[2], p_free[2],
  // item_full[2], item_empty[2], redo_loaded, redo_done
  static constexpr int kNumBars = 2 * kStages + 19;
  static constexpr int kOffMisc = kOffBar + kNumBars * 8;
  static constexpr int kOffItems = (kOffMisc + 16 + 15) / 16 * 16;   // two items, then scan[12] and the share's beginning
  static constexpr int kOffAgain = kOffItems + 2 * 32 + 15 * 8;      // kAgain bits: pieces of the share to compute once more
  static constexpr int kOffSums = (kOffAgain + kAgain / 8 + 15) / 16 * 16;   // m and l of a row, for the cluster (QT = 1)
  static constexpr int kSmemBytes = kOffSums + (QT == 1 ? kBM * 8 : 0) + 1024;
  // Exponentials, in chunks of 32 tokens, before the wait for P's buffer (2, 3, 4 of 4 at d_v = 128: 1566, 1525, 1545 us of 32768
  // tokens; 1 to 4 at d_v = 64: 65.2, 64.5, 65.1, 67.0 us of 4 x 16 heads x 2048, causal).
  static constexpr int kEarlyChunks = DV == 64 ? 2 : 3;
  static constexpr uint32_t kTmemCols = 512;
  static constexpr uint32_t kTmemS0 = 0, kTmemS1 = kSharedS ? 0 : 128;
  static constexpr uint32_t kTmemP0 = kSharedS ? 128 : 256, kTmemP1 = kSharedS ? 192 : 320;
  static constexpr uint32_t kTmemO0 = kSharedS ? 256 : 384, kTmemO1 = kTmemO0 + (QT == 2 ? DV : 0);
  static_assert(QT == 2 || (2 * kStageBytes >= kBM * DV * 4 && kStages >= 6), "parts of a cluster's rows beside two tiles");
  static_assert(kTmemO1 + DV <= kTmemCols, "TMEM budget");
  static_assert(kSmemBytes <= 232448, "shared memory budget");
};

// Where a tile's panels of 64 columns and its groups of eight tokens lie in shared memory, in bytes from one to the next.  (A
// template's constants: as variables of the products' descriptors, 32768 tokens take 4 % longer.)
template <int D, bool PAGED>
struct Layout {
  static constexpr uint32_t kPanel = PAGED ? 1024 : 128 * 128, kGroup = PAGED ? D / 64 * 1024 : 1024;
};

struct Params {
  int64_t o_sb, o_sh, o_sn;
  KvSource kv;
  const int32_t* lens;   // null: every sequence has max_len tokens
  int N, max_len, Hk, G;
  int GC, chunks, PT;    // heads of a tile, chunks of heads, positions of a tile
  int n_tiles;           // work items of a key head
  int n_items;
  int columns, tall, height;   // the items' order in the shares (where_of)
  int box;               // tokens of a TMA copy
  int page_groups;       // groups of eight tokens of a page and head
  int all_groups;        // of the pool
  int cluster;           // CTAs for each work item, joined in the same launch; 0: equal shares of all items
  win::Mask mask;
  float c_log2;          // scale log2 e, >= 0
  uint64_t wait_limit_ns;
};

__device__ __forceinline__ int length_of(const Params& p, int b, bool report) {
  if (p.lens == nullptr) return p.max_len;
  const int len = p.lens[b];
  if (len >= 0 && len <= p.max_len) return len;
  if (report) atomicExch(&g_moa_window_tc_status, win::kErrIndex);
  return len < 0 ? 0 : p.max_len;
}

// A work item: its key head, chunk of heads and positions.
struct Where {
  int b, h, chunk, i0, i1;   // the last position is i1
};
// Items in the order of the shares: what the CTAs work on at one time is neighbouring items (positions of one key head),
// whose tokens they share in L2.  The order is that of a table read column by column, a column a CTA; the first `tall` columns
// have height + 1 items.  Where all CTAs' tokens fit into L2 the items are taken in order of place (columns = 0).  32768 tokens of 8
// key heads of 128, window 4096: in order of place the tokens come 12 times from memory, 5.1 GB, and the call takes 4 % longer
// (1717 us instead of 1653 before the softmax loop's last steps); 4 x 16 heads x 2048 x 64, causal: 66 us instead of 68.
template <int QT>
__device__ __forceinline__ Where where_of(const Params& p, int item) {
  Where w;
  if (p.columns > 0) {
    const int split = p.tall * (p.height + 1), x = item < split ? item : item - split;
    const int h = item < split ? p.height + 1 : p.height, c = int(unsigned(x) / unsigned(h));
    item = (x - c * h) * p.columns + (item < split ? c : c + p.tall);
  }
  const int bh = int(unsigned(item) / unsigned(p.n_tiles)), rest = item - bh * p.n_tiles;
  const int tile = int(unsigned(rest) / unsigned(p.chunks));
  w.chunk = rest - tile * p.chunks;
  w.b = int(unsigned(bh) / unsigned(p.Hk)), w.h = bh - w.b * p.Hk;
  w.i0 = tile * QT * p.PT;
  const int64_t last = int64_t(w.i0) + QT * p.PT - 1;
  w.i1 = last < p.N ? int(last) : p.N - 1;
  return w;
}
// Tiles of tokens that it counts for: at least one, so that every item is written.
template <int QT>
__device__ __forceinline__ int units_of(const Params& p, int item, bool report) {
  const Where w = where_of<QT>(p, item);
  const int n = win::tiles_of(p.mask, length_of(p, w.b, report), p.N, w.i0, w.i1, kBN).n;
  return n < 1 ? 1 : n;
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

// One item of a CTA's share: its tiles [u0, u1) of `units` are this CTA's; tile t is token tile
// list.at(t).  item < 0: no more.
struct Item {
  int item, u0, u1, units;
  int first, from, len;
};

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

// Zeros in rows `row`, row + step, ... of a values' tile (of pages) that has arrived, from row `gone` on; false if it has not.  (A
// function of its own: an item's last tile only.)
template <int DV>
__device__ __noinline__ bool zero_rows(uint8_t* tile, int row, int step, int gone, uint32_t full, uint32_t parity,
                                       const WaitCtl& wc) {
  using L = Layout<DV, true>;
  const bool ok = wait_bounded(full, parity, wc);
  for (; row < kBN; row += step) {
    if (row < gone) continue;
#pragma unroll
    for (int q = 0; q < DV / 64; ++q)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        reinterpret_cast<uint4*>(tile + q * L::kPanel + (row >> 3) * L::kGroup + (row & 7) * 128)[e] = make_uint4(0, 0, 0, 0);
  }
  fence_proxy_async_smem();
  return ok;
}

// What a CTA needs to find its share again, in shared memory: the item in which it begins, that item's first unit, all units.
struct Begin {
  int64_t item, unit, total;
};

// A cluster's item: CTA (r / 4) % size joins row r.  Every CTA leaves its part of the row there, in the last two stages of the
// ring, which a cluster does not use for tiles: [CTA][row of the owner][DV], and m and l.  (Parts fetched by the owner instead
// took 3 us more: two round trips and a second barrier.)
struct Owner {
  int rank, row;
};
__device__ __forceinline__ Owner owner_of(int r, int size) { return Owner{(r >> 2) % size, (r >> 2) / size * 4 + (r & 3)}; }

template <int DV>
__device__ __noinline__ void cluster_rows(__nv_bfloat16* O, float* lse, const Params& p, const float* sum,
                                          const float2* stat) {
  // eight lanes a row
  constexpr int kQuads = DV / 32;
  const int lane = threadIdx.x & 31, sub = lane & 7, rows = kBM / p.cluster;
  const Where w = where_of<1>(p, int(blockIdx.x));
  for (int base = 0; base < rows; base += 16) {
    const int at = base + int(threadIdx.x >> 3), r = ((at >> 2) * p.cluster + int(blockIdx.y)) * 4 + (at & 3);
    const int pos = int(unsigned(r) / unsigned(p.GC)), g = w.chunk * p.GC + r - pos * p.GC, i = w.i0 + pos, hq = w.h * p.G + g;
    const bool live = at < rows && pos < p.PT && i <= w.i1 && g < p.G;
    if (!__any_sync(0xffffffffu, live)) continue;
    float M = -INFINITY, L = 0.f;
    float4 x[kQuads];
#pragma unroll
    for (int q = 0; q < kQuads; ++q) x[q] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (live) {
      for (int k = 0; k < p.cluster; ++k) M = fmaxf(M, stat[k * rows + at].x);
#pragma unroll 2
      for (int k = 0; k < p.cluster; ++k) {
        const float2 ml = stat[k * rows + at];
        if (ml.x == -INFINITY && ml.y == 0.f) continue;   // its tiles held nothing that the row sees, or it had none
        const float f = ex2_approx(ml.x - M);
        L += f * ml.y;
#pragma unroll
        for (int q = 0; q < kQuads; ++q) {
          const float4 v = *reinterpret_cast<const float4*>(sum + (k * rows + at) * DV + (sub + 8 * q) * 4);
          x[q].x += f * v.x, x[q].y += f * v.y, x[q].z += f * v.z, x[q].w += f * v.w;
        }
      }
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;
    __nv_bfloat16* o = O + int64_t(w.b) * p.o_sb + int64_t(hq) * p.o_sh + int64_t(i) * p.o_sn;
#pragma unroll
    for (int q = 0; q < kQuads; ++q) {
      x[q].x *= inv, x[q].y *= inv, x[q].z *= inv, x[q].w *= inv;
      if (live)
        *reinterpret_cast<uint2*>(o + (sub + 8 * q) * 4) = make_uint2(pack_bf16x2(x[q].x, x[q].y), pack_bf16x2(x[q].z, x[q].w));
    }
    if (lse != nullptr && live && sub == 0)
      lse[(int64_t(w.b) * p.Hk * p.G + hq) * p.N + i] = L == 0.f ? -INFINITY : (M + lg2_approx(L)) * kLn2;
  }
}

// Looks through rows `row`, row + step, ... of a values' tile that has arrived.  From row `gone` on they become zeros; values
// of the others that are not finite become zeros and set *odd to `mark`.  False if the tile has not arrived.  (In the softmax loop this
// would cost 4 to 10 % of long calls; it is for redo_piece.)
template <int DV, bool PAGED>
__device__ __noinline__ bool look_through(uint8_t* tile, int row, int step, int gone, uint32_t full, uint32_t parity, volatile int* odd,
                                          int mark, const WaitCtl& wc) {
  using L = Layout<DV, PAGED>;
  const bool ok = wait_bounded(full, parity, wc);
  for (; row < kBN; row += step) {
    // the row's 16-byte words, eight lanes in eight banks at a time
    uint8_t* at = tile + (row >> 3) * L::kGroup + (row & 7) * 128;
    auto word = [&](int q, int e) { return reinterpret_cast<uint4*>(at + q * L::kPanel + ((e ^ row) & 7) * 16); };
    if (row >= gone) {
#pragma unroll
      for (int q = 0; q < DV / 64; ++q)
#pragma unroll
        for (int e = 0; e < 8; ++e) *word(q, e) = make_uint4(0, 0, 0, 0);
      continue;
    }
    // x * 0 + sum is NaN from the first x on that is not finite
    const __nv_bfloat162 zero = __floats2bfloat162_rn(0.f, 0.f);
    __nv_bfloat162 sum[4] = {zero, zero, zero, zero};
#pragma unroll
    for (int q = 0; q < DV / 64; ++q)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint4 x = *word(q, e);
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&w[i]), zero, sum[i]);
      }
    const __nv_bfloat162 all = __hadd2(__hadd2(sum[0], sum[1]), __hadd2(sum[2], sum[3]));
    if (__low2float(all) == 0.f && __high2float(all) == 0.f) continue;
    *odd = mark;
    __threadfence_block();   // (the other row tile's warps may find the zeros)
#pragma unroll 1
    for (int e = 0; e < DV / 8; ++e) {
      uint32_t* w = reinterpret_cast<uint32_t*>(word(e >> 3, e));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if ((w[i] & 0x7f80u) == 0x7f80u) w[i] &= 0xffff0000u;
        if ((w[i] & 0x7f800000u) == 0x7f800000u) w[i] &= 0xffffu;
      }
    }
  }
  fence_proxy_async_smem();
  return ok;
}

// Tiles of an item in which a token is hidden from one of its rows: end0 the end of its first row, low1 the beginning of its last one's
// window.
struct Partly {
  int end0, low1;
  __device__ __forceinline__ Partly(const win::Mask& m, int len, int N, int i0, int i1)
      : end0(win::row_end(m, len, N, i0)), low1(win::row_low(m, len, N, i1)) {}
  __device__ __forceinline__ bool operator()(int n0, int sinks) const {
    return end0 - n0 < kBN || (n0 < low1 && n0 + kBN > sinks);
  }
};

// Where token t's values lie; null: a page outside the pool.
__device__ __forceinline__ const __nv_bfloat16* values_of(const Params& p, int b, int h, int t) {
  int64_t at = b, place = t;
  if (p.kv.table != nullptr) {
    const int slot = int(unsigned(t) / unsigned(p.kv.page));
    at = p.kv.table[b * p.kv.max_pages + slot];
    place = t - slot * p.kv.page;
    if (at < 0 || at >= p.kv.n_pages) return nullptr;
  }
  return static_cast<const __nv_bfloat16*>(p.kv.v) + at * p.kv.v_sb + h * p.kv.v_sh + place * p.kv.v_sn;
}
__device__ __forceinline__ bool odd_pair(uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; }

// Adds, to the sums in TMEM of a warp's rows, the values that look_through took out of tiles [u0, u1) and that the rows see: tokens below
// lim from low on, or below the sinks.  Rows that are not `live` are left.  A row that has nothing but NaN is done.
template <int DV>
__device__ __noinline__ void add_odd_values(uint32_t tO, const Params& p, int b, int h, int len, int i0, int i1, const win::Tiles& list, int u0,
                                            int u1, int lim, int low, bool live) {
  const int lane = threadIdx.x & 31;
  const Partly partly(p.mask, len, p.N, i0, i1);
#pragma unroll 1
  for (int c = 0; c < DV; c += 32) {
    uint32_t o[32];
    tmem_ld_32x32b_x32(tO + c, o);
    tmem_wait_ld();
    reg_anchor_x32(o);
    auto open = [&]() {
      bool any = false;
#pragma unroll
      for (int e = 0; e < 32; ++e) any |= __uint_as_float(o[e]) == __uint_as_float(o[e]);
      return __any_sync(0xffffffffu, any && live);
    };
#pragma unroll 1
    for (int n = u0; n < u1 && open(); ++n) {
      const int n0 = list.at(n) * kBN;
      if (!partly(n0, p.mask.sinks)) continue;
#pragma unroll 1
      for (int t0 = n0; t0 < n0 + kBN && t0 < len; t0 += 32) {
        // a token a lane
        const __nv_bfloat16* v = t0 + lane < len ? values_of(p, b, h, t0 + lane) : nullptr;
        bool odd = false;
        if (v != nullptr) {
          v += c;
#pragma unroll
          for (int e = 0; e < 32; e += 2) odd |= odd_pair(*reinterpret_cast<const uint32_t*>(v + e));
        }
        uint32_t rest = __ballot_sync(0xffffffffu, odd);
        while (rest != 0) {
          const int from = __ffs(rest) - 1, token = t0 + from;
          rest &= rest - 1;
          const __nv_bfloat16* x = reinterpret_cast<const __nv_bfloat16*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(v), from));
          if (live && token < lim && (token >= low || token < p.mask.sinks)) {
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              const float y = __bfloat162float(x[e]);
              if (!(fabsf(y) < INFINITY)) o[e] = __float_as_uint(__uint_as_float(o[e]) + y);
            }
          }
        }
      }
    }
    tmem_st_32x32b_x32(tO + c, o);
    tmem_wait_st();
  }
}

// A row's place.
struct Place {
  int b, hq, i;
  bool live;
};
template <int QT>
__device__ __forceinline__ Place place_of(const Params& p, int item, int j, int row_pos, int row_head) {
  const Where w = where_of<QT>(p, item);
  const int g = w.chunk * p.GC + row_head, i = w.i0 + j * p.PT + row_pos;
  return Place{w.b, w.h * p.G + g, i, row_pos < p.PT && g < p.G && i < p.N};
}

// Where an item's rows go.
struct Out {
  __nv_bfloat16* O;
  float* lse;
  float* part_o;
  float2* part_ml;
};
// Writes a warp's rows of an item: the output, or this CTA's piece, or to the CTA of the cluster that joins the row.  Returns whether some
// row has a sum that is not finite though its weights are numbers.
template <int DK, int DV, int QT, bool ROLLED>
__device__ __forceinline__ bool write_rows(const Params& p, const Out& out, const Place& w, uint32_t tO, uint32_t parts, int j, int row, float m,
                                           float l, bool first_piece, bool whole) {
  using C = Cfg<DK, DV, QT>;
  constexpr int kUnroll = ROLLED ? 1 : DV / 16;
  float top[4] = {0.f, 0.f, 0.f, 0.f};   // x * 0 + top is NaN from the first x on that is not finite
  if (QT == 1 && p.cluster > 1) {   // the row's sums, to the CTA that joins it
    const Owner own = owner_of(row, p.cluster);
    const uint32_t sum = smem_of_cta(parts + ((int(blockIdx.y) * (kBM / p.cluster) + own.row) * DV) * 4, own.rank);
#pragma unroll(kUnroll)
    for (int d = 0; d < DV; d += 16) {
      uint32_t o[16];
      tmem_ld_32x32b_x16(tO + d, o);
      tmem_wait_ld();
      reg_anchor_x16(o);
      if (w.live) {
#pragma unroll
        for (int e = 0; e < 4; ++e) store4_to_cta(sum + (d + 4 * e) * 4, o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) top[e & 3] = fmaf(__uint_as_float(o[e]), 0.f, top[e & 3]);
    }
  } else if (!whole) {
    const int64_t at = (int64_t(blockIdx.x) * 2 + first_piece) * C::kRows + j * kBM + row;
#pragma unroll(kUnroll)
    for (int d = 0; d < DV; d += 16) {
      uint32_t o[16];
      tmem_ld_32x32b_x16(tO + d, o);
      tmem_wait_ld();
      reg_anchor_x16(o);
#pragma unroll
      for (int e = 0; e < 16; ++e) top[e & 3] = fmaf(__uint_as_float(o[e]), 0.f, top[e & 3]);
      if (w.live) {
        float4* dst = reinterpret_cast<float4*>(out.part_o + at * DV + d);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          dst[e] = make_float4(__uint_as_float(o[4 * e]), __uint_as_float(o[4 * e + 1]), __uint_as_float(o[4 * e + 2]),
                               __uint_as_float(o[4 * e + 3]));
      }
    }
    if (w.live) out.part_ml[at] = make_float2(m, l);
  } else {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    __nv_bfloat16* orow = out.O + int64_t(w.b) * p.o_sb + int64_t(w.hq) * p.o_sh + int64_t(w.i) * p.o_sn;
    if (out.lse != nullptr && w.live)
      out.lse[(int64_t(w.b) * p.Hk * p.G + w.hq) * p.N + w.i] = l == 0.f ? -INFINITY : (m + lg2_approx(l)) * kLn2;
#pragma unroll(kUnroll)
    for (int d = 0; d < DV; d += 16) {
      uint32_t o[16];
      tmem_ld_32x32b_x16(tO + d, o);
      tmem_wait_ld();
      reg_anchor_x16(o);
      uint32_t z[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float y0 = __uint_as_float(o[2 * e]) * inv, y1 = __uint_as_float(o[2 * e + 1]) * inv;
        top[2 * e & 3] = fmaf(y0, 0.f, top[2 * e & 3]);
        top[(2 * e + 1) & 3] = fmaf(y1, 0.f, top[(2 * e + 1) & 3]);
        z[e] = pack_bf16x2(y0, y1);
      }
      if (w.live) {
        reinterpret_cast<uint4*>(orow + d)[0] = make_uint4(z[0], z[1], z[2], z[3]);
        reinterpret_cast<uint4*>(orow + d)[1] = make_uint4(z[4], z[5], z[6], z[7]);
      }
    }
  }
  return __any_sync(0xffffffffu, w.live && (top[0] + top[1]) + (top[2] + top[3]) != 0.f && l == l);
}

// The lane's copy of the tile of tokens from t0 (its own first token) on of a paged item: the first group of eight tokens of the pool.
__device__ __forceinline__ int page_source(const Params& p, const Where& w, int t0, int end, int low) {
  if (t0 < end && (t0 > low - p.box || t0 < p.mask.sinks)) {
    const int at = int(unsigned(t0) / unsigned(p.kv.page));
    const int pg = p.kv.table[w.b * p.kv.max_pages + at];
    if (pg >= 0 && pg < p.kv.n_pages) return (pg * p.Hk + w.h) * p.page_groups + ((t0 - at * p.kv.page) >> 3);
    atomicExch(&g_moa_window_tc_status, win::kErrIndex);
  }
  return p.all_groups;   // past the pool: zeros
}

// The products of a row tile: S = Q K^T, O (+)= P V.
template <int DK, bool PAGED>
__device__ __forceinline__ void issue_scores(uint32_t tS, uint32_t q, uint32_t k) {
  using L = Layout<DK, PAGED>;
  constexpr uint32_t kIdesc = make_idesc(kBM, kBN, false);
#pragma unroll
  for (int kk = 0; kk < DK / 16; ++kk)
    mma_f16_ss(tS, make_sdesc_sw128(q + (kk >> 2) * (128 * 128) + (kk & 3) * 32, 16, 1024),
               make_sdesc_sw128(k + (kk >> 2) * L::kPanel + (kk & 3) * 32, 16, L::kGroup), kIdesc, kk > 0 ? 1u : 0u);
}
template <int DV, bool PAGED>
__device__ __forceinline__ void issue_outputs(uint32_t tO, uint32_t tP, uint32_t v, uint32_t acc_first) {
  using L = Layout<DV, PAGED>;
  constexpr uint32_t kIdesc = make_idesc(kBM, DV, true);
#pragma unroll
  for (int kk = 0; kk < kBN / 16; ++kk)
    mma_f16_ts(tO, tP + kk * 8, make_sdesc_sw128(v + 2 * kk * L::kGroup, L::kPanel, L::kGroup), kIdesc, kk > 0 ? 1u : acc_first);
}

// What redo_piece works with.
struct Again {
  const CUtensorMap *q, *k, *v;
  uint8_t* kv;             // the ring: a tile of keys in its first stage, of values in its second
  uint32_t tmem, sQ;
  uint32_t loaded, done;   // barriers: copies, products
  volatile int* odd;
  uint32_t loads, products;   // so far
};

// Tiles [u0, u1) of an item once more, by the softmax warps alone, with values that are not finite taken out of the tiles that
// some row does not see all of, if there are any.  False if a wait ran out.
template <int DK, int DV, int QT, bool PAGED>
__device__ __forceinline__ bool redo_piece(Again& a, const Params& p, const Out& out, int item, int u0, int u1, const WaitCtl& wc) {
  using C = Cfg<DK, DV, QT>;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, j = warp >> 2, row = (warp & 3) * 32 + lane;
  const uint32_t lanes = a.tmem + (uint32_t((warp & 3) * 32) << 16);
  const uint32_t tS = lanes + (j ? C::kTmemS1 : C::kTmemS0), tP = lanes + (j ? C::kTmemP1 : C::kTmemP0);
  const uint32_t tO = lanes + (j ? C::kTmemO1 : C::kTmemO0), sK = smem_u32(a.kv), sV = sK + C::kStageBytes;
  const bool first = threadIdx.x == 0;
  // all softmax threads; whether all of them say so
  auto meet = [](bool yes) {
    uint32_t all;
    asm volatile("{\n\t.reg .pred a, b;\n\tsetp.ne.u32 a, %1, 0;\n\tbar.red.and.pred b, 1, %2, a;\n\tselp.u32 %0, 1, 0, b;\n\t}"
                 : "=r"(all)
                 : "r"(uint32_t(yes)), "n"(C::kSoftmax)
                 : "memory");
    return all != 0;
  };
  const Where w = where_of<QT>(p, item);
  const int len = length_of(p, w.b, false);
  const win::Tiles list = win::tiles_of(p.mask, len, p.N, w.i0, w.i1, kBN);
  const int end = win::row_end(p.mask, len, p.N, w.i1), begin = win::row_low(p.mask, len, p.N, w.i0);
  const Partly partly(p.mask, len, p.N, w.i0, w.i1);
  const int row_pos = int(unsigned(row) / unsigned(p.GC));
  const Place at = place_of<QT>(p, item, j, row_pos, row - row_pos * p.GC);
  const int lim = at.live ? win::row_end(p.mask, len, p.N, at.i) : 0, low = at.live ? win::row_low(p.mask, len, p.N, at.i) : 0;
  const float c = fmaxf(p.c_log2, FLT_MIN);
  const int gone = PAGED ? len : 0x7fffffff;
  // nothing to take out: what is not finite is what the rows see
  bool odd = false;
#pragma unroll 1
  for (int n = u0; n < u1; ++n) {
    const int n0 = list.at(n) * kBN;
    if (!partly(n0, p.mask.sinks)) continue;
    for (int x = threadIdx.x; x < kBN * (DV / 8); x += C::kSoftmax) {
      const int t = n0 + x / (DV / 8);
      const __nv_bfloat16* v = t < len ? values_of(p, w.b, w.h, t) : nullptr;
      if (v == nullptr) continue;
      const uint4 y = *reinterpret_cast<const uint4*>(v + x % (DV / 8) * 8);
      odd |= odd_pair(y.x) || odd_pair(y.y) || odd_pair(y.z) || odd_pair(y.w);
    }
  }
  if (meet(!odd)) return true;
  float m = -INFINITY, l = 0.f;
  if (first) {
    *a.odd = 0;
    mbar_arrive_expect_tx(a.loaded, QT * DK * 2 * p.GC * p.PT);
#pragma unroll 1
    for (int x = 0; x < QT * (DK / 64); ++x) {
      const int t = x / (DK / 64), q = x % (DK / 64);
      tma_load_5d(a.sQ + t * C::kQTileBytes + q * C::kPanelBytes, a.q, a.loaded, q * 64, w.chunk * p.GC, w.i0 + t * p.PT, w.h, w.b);
    }
  }
  bool ok = wait_bounded(a.loaded, a.loads++ & 1u, wc);
#pragma unroll 1
  for (int n = u0; n < u1; ++n) {
    const int n0 = list.at(n) * kBN;
    ok = meet(ok);   // the tile before is done with
    if (!ok) break;
    if (first) {
      mbar_arrive_expect_tx(a.loaded, C::kKTileBytes + C::kVTileBytes);
      if constexpr (PAGED) {
#pragma unroll 1
        for (int t = 0; t < kBN; t += p.box) {
          const int s = page_source(p, w, n0 + t, end, begin);
          tma_load_4d(sK + t / 8 * Layout<DK, true>::kGroup, a.k, a.loaded, 0, 0, 0, s);
          tma_load_4d(sV + t / 8 * Layout<DV, true>::kGroup, a.v, a.loaded, 0, 0, 0, s);
        }
      } else {
#pragma unroll 1
        for (int q = 0; q < DK / 64; ++q) tma_load_4d(sK + q * C::kPanelBytes, a.k, a.loaded, q * 64, n0, w.h, w.b);
#pragma unroll 1
        for (int q = 0; q < DV / 64; ++q) tma_load_4d(sV + q * C::kPanelBytes, a.v, a.loaded, q * 64, n0, w.h, w.b);
      }
    }
    const uint32_t arrived = a.loads++ & 1u;
    ok = wait_bounded(a.loaded, arrived, wc);
#pragma unroll 1
    for (int t = 0; t < QT; ++t) {   // (both row tiles may have one buffer of scores)
      if (first) {
        tc_fence_after_sync();
        issue_scores<DK, PAGED>(a.tmem + (t ? C::kTmemS1 : C::kTmemS0), a.sQ + t * C::kQTileBytes, sK);
        mma_commit(a.done);
      }
      ok = wait_bounded(a.done, a.products++ & 1u, wc) && ok;
      tc_fence_after_sync();
      if (j == t) {
        // 32 tokens at a time, twice: their scores, -infinity for those that the row does not see
        uint32_t sr[32];
        auto scores = [&](int k) {
          tmem_ld_32x32b_x32(tS + 32 * k, sr);
          tmem_wait_ld();
          reg_anchor_x32(sr);
          const uint32_t bits = below(lim - n0, k) & (~below(low - n0, k) | below(p.mask.sinks - n0, k));
#pragma unroll
          for (int e = 0; e < 32; ++e) sr[e] = bits >> e & 1u ? sr[e] : 0xff800000u;
        };
        float top = -INFINITY;
#pragma unroll 1
        for (int k = 0; k < 4; ++k) {
          scores(k);
#pragma unroll
          for (int e = 0; e < 32; ++e) top = fmaxf(top, __uint_as_float(sr[e]));
        }
        top *= c;
        if (__any_sync(0xffffffffu, top > m)) {
          const float m_new = fmaxf(m, top), alpha = m == -INFINITY ? 0.f : ex2_approx(m - m_new);
          l *= alpha;
          m = m_new;
          if (n > u0) tmem_scale_row<DV>(tO, alpha);
        }
        const float base = m == -INFINITY ? 0.f : m;
#pragma unroll 1
        for (int k = 0; k < 4; ++k) {
          scores(k);
          uint32_t pk[16];
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const float p0 = ex2_approx(fmaf(__uint_as_float(sr[e]), c, -base)), p1 = ex2_approx(fmaf(__uint_as_float(sr[e + 1]), c, -base));
            l += p0 + p1;
            pk[e >> 1] = pack_bf16x2(p0, p1);
          }
          tmem_st_32x32b_x16(tP + 16 * k, pk);
        }
        tmem_wait_st();
      }
      tc_fence_before_sync();
      ok = meet(ok);
    }
    if (partly(n0, p.mask.sinks))
      ok = look_through<DV, PAGED>(a.kv + C::kStageBytes, int(threadIdx.x), C::kSoftmax, gone - n0, a.loaded, arrived, a.odd, 1, wc) && ok;
    ok = meet(ok);
    if (first) {
      tc_fence_after_sync();
#pragma unroll 1
      for (int t = 0; t < QT; ++t)
        issue_outputs<DV, PAGED>(a.tmem + (t ? C::kTmemO1 : C::kTmemO0), a.tmem + (t ? C::kTmemP1 : C::kTmemP0), sV, n > u0 ? 1u : 0u);
      mma_commit(a.done);
    }
    ok = wait_bounded(a.done, a.products++ & 1u, wc) && ok;
    tc_fence_after_sync();
  }
  ok = meet(ok);
  if (!ok) {   // the last copies and products end before the CTA does
    if (first) {
      wait_quiesce(a.loaded, (a.loads - 1) & 1u, wc.limit_ns, wc.status);
      if (a.products > 0) wait_quiesce(a.done, (a.products - 1) & 1u, wc.limit_ns, wc.status);
    }
    return false;
  }
  if (*a.odd != 0) add_odd_values<DV>(tO, p, w.b, w.h, len, w.i0, w.i1, list, u0, u1, lim, low, at.live && l == l);
  const int units = list.n < 1 ? 1 : list.n;
  write_rows<DK, DV, QT, true>(p, out, at, tO, sK + (C::kStages - 2) * C::kStageBytes, j, row, m, l, u0 == 0, u0 == 0 && u1 == units);
  if (QT == 1 && p.cluster > 1) {
    const Owner own = owner_of(row, p.cluster);
    store2_to_cta(smem_of_cta(sK - C::kOffKV + C::kOffSums + (int(blockIdx.y) * (kBM / p.cluster) + own.row) * 8, own.rank),
                  at.live ? m : -INFINITY, at.live ? l : 0.f);
  }
  tc_fence_before_sync();
  return meet(true);
}

// The marked pieces of a CTA's share, as the walk had them, or its part of a cluster's item.  (All that it needs it finds again: what
// a call kept for it would cost the softmax loop registers.)
template <int DK, int DV, int QT, bool PAGED>
__device__ __noinline__ void redo_share(const CUtensorMap* tmQ, const CUtensorMap* tmK, const CUtensorMap* tmV, const Params& p, const Out& out,
                                        uint8_t* smem, uint32_t tmem) {
  using C = Cfg<DK, DV, QT>;
  const volatile Item* items = reinterpret_cast<const volatile Item*>(smem + C::kOffItems);
  const uint32_t* again = reinterpret_cast<const uint32_t*>(smem + C::kOffAgain);
  const Begin* found = reinterpret_cast<const Begin*>(smem + C::kOffItems + 64 + 12 * 8);
  const uint32_t bars = smem_u32(smem + C::kOffBar) + 8u * (2 * C::kStages + 17);
  const WaitCtl wc{reinterpret_cast<volatile int*>(smem + C::kOffMisc + 4), p.wait_limit_ns, 0u, &g_moa_window_tc_status};
  Again a{tmQ, tmK, tmV, smem + C::kOffKV, tmem, smem_u32(smem), bars, bars + 8, reinterpret_cast<volatile int*>(smem + C::kOffMisc + 12), 0, 0};
  int64_t at = 0, stop = 0, before = 0;
  int item = 0;
  if (p.cluster == 0) {
    const Shares shares(found->total, gridDim.x);
    at = shares.start(blockIdx.x), stop = shares.start(blockIdx.x + 1);
    item = int(found->item), before = found->unit;
  }
  for (uint32_t seg = 0; p.cluster != 0 ? seg == 0 : at < stop; ++item) {
    int u0 = items[0].u0, u1 = items[0].u1, which = items[0].item;   // of a cluster
    if (p.cluster == 0) {
      which = item;
      const int64_t end = before + units_of<QT>(p, item, false) + item_units(QT), upto = end < stop ? end : stop;
      u0 = max(0, int(at - before) - item_units(QT)), u1 = max(0, int(upto - before) - item_units(QT));
      at = upto;
      before = end;
      if (u0 >= u1) continue;
    }
    const uint32_t bit = seg < kAgain - 1 ? seg : kAgain - 1;
    if ((again[bit / 32] >> (bit & 31) & 1u) != 0 && !redo_piece<DK, DV, QT, PAGED>(a, p, out, which, u0, u1, wc)) return;
    ++seg;
  }
}

// ------------------------------------------------------------------------------------------------
// Attention
// ------------------------------------------------------------------------------------------------
template <int DK, int DV, int QT, bool PAGED>
__global__ void __launch_bounds__(Cfg<DK, DV, QT>::kThreads, 1)
window_tc_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                 const __grid_constant__ CUtensorMap tmV, const __grid_constant__ Out out, Cut* cuts,
                 const __grid_constant__ Params p) {
  using C = Cfg<DK, DV, QT>;
  using KL = Layout<DK, PAGED>;
  using VL = Layout<DV, PAGED>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const uint32_t sQ = smem_u32(smem), sKV = smem_u32(smem + C::kOffKV), bar0 = smem_u32(smem + C::kOffBar);
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (C::kStages + s); };
  const uint32_t q_full = bar0 + 8u * (2 * C::kStages), q_empty = q_full + 8, drain = q_full + 16;
  auto s_full = [&](int j) { return q_full + 8u * (3 + j); };
  auto p_ready = [&](int j) { return q_full + 8u * (5 + j); };
  auto o_done = [&](int j) { return q_full + 8u * (7 + j); };
  auto s_free = [&](int j) { return q_full + 8u * (9 + j); };
  auto p_free = [&](int j) { return q_full + 8u * (11 + j); };
  auto item_full = [&](int i) { return q_full + 8u * (13 + i); };
  auto item_empty = [&](int i) { return q_full + 8u * (15 + i); };
  const uint32_t redo_loaded = q_full + 8u * 17, redo_done = q_full + 8u * 18;   // (redo_share)
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + C::kOffMisc);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + C::kOffMisc + 4);
  volatile int* any_again = reinterpret_cast<volatile int*>(smem + C::kOffMisc + 8);   // a piece is to be computed once more
  uint32_t* again = reinterpret_cast<uint32_t*>(smem + C::kOffAgain);
  volatile Item* items = reinterpret_cast<volatile Item*>(smem + C::kOffItems);
  int64_t* scan = reinterpret_cast<int64_t*>(smem + C::kOffItems + 64);   // warp sums
  Begin* found = reinterpret_cast<Begin*>(scan + 12);
  constexpr int kWarps = C::kThreads / 32;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const WaitCtl wc{abort_flag, p.wait_limit_ns, 0u, &g_moa_window_tc_status};

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), QT);   // one commit from each issuer
    }
    mbar_init(q_full, 1);
    mbar_init(q_empty, QT);
    mbar_init(drain, QT);
    for (int i = 0; i < 2; ++i) {
      mbar_init(item_full(i), 1);
      mbar_init(item_empty(i), 5 * QT + 1);   // the softmax warps, the issuers, the loads
    }
    for (int j = 0; j < QT; ++j) {
      mbar_init(s_full(j), 1);
      mbar_init(p_ready(j), 128);
      mbar_init(o_done(j), 1);
      mbar_init(s_free(j), 128);
      mbar_init(p_free(j), 1);
    }
    *abort_flag = 0;
    *any_again = 0;
    fence_barrier_init();
  }
  if (threadIdx.x < kAgain / 32) again[threadIdx.x] = 0;
  if (warp == C::kLoadWarp && lane == 0) {
    tma_prefetch_desc(&tmQ);
    tma_prefetch_desc(&tmK);
    tma_prefetch_desc(&tmV);
  }
  if (warp == C::kMmaWarp0) {
    tmem_alloc(smem_u32(tmem_slot), C::kTmemCols);
    tmem_relinquish();
  }
  if (p.GC * p.PT < kBM) {   // rows of a tile that no copy fills
    for (int x = threadIdx.x; x < QT * C::kQTileBytes / 16; x += C::kThreads)
      reinterpret_cast<uint4*>(smem)[x] = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();
  }
  wait_for_previous();
  int64_t total = 1, first_unit = 0, stop = 0;
  if (p.cluster != 0) {
    if (warp == C::kWalkWarp && lane == 0) {   // one item, of which the cluster's CTAs take equal parts
      const Where w = where_of<QT>(p, int(blockIdx.x));
      const int len = length_of(p, w.b, blockIdx.y == 0);
      const win::Tiles list = win::tiles_of(p.mask, len, p.N, w.i0, w.i1, kBN);
      const int units = list.n < 1 ? 1 : list.n;
      volatile Item& x = items[0];
      x.u0 = units * int(blockIdx.y) / p.cluster, x.u1 = units * (int(blockIdx.y) + 1) / p.cluster;
      x.item = x.u0 < x.u1 ? int(blockIdx.x) : -1;
      x.units = units, x.first = list.first, x.from = list.from, x.len = len;
    }
  } else {
    // this CTA's share of all units, and the item in which it begins: the sum of all units, then their running sum
    // (the same pass where there is an item for each thread at most)
    auto block_scan = [&](int64_t mine, int64_t* all) {
      int64_t incl = mine;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int64_t o = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += o;
      }
      __syncthreads();
      if (lane == 31) scan[warp] = incl;
      __syncthreads();
      *all = 0;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        if (w < warp) incl += scan[w];
        *all += scan[w];
      }
      return incl;
    };
    const bool one_pass = p.n_items <= C::kThreads;
    int64_t mine = 0;
    for (int i = threadIdx.x; i < p.n_items; i += C::kThreads) mine += units_of<QT>(p, i, true) + item_units(QT);
    int64_t incl = block_scan(mine, &total);
    const Shares shares(total, gridDim.x);
    first_unit = blockIdx.x < shares.n ? shares.start(blockIdx.x) : total;
    stop = blockIdx.x < shares.n ? shares.start(blockIdx.x + 1) : total;
    int64_t done = 0;
    for (int base = 0; first_unit < stop; base += C::kThreads) {
      const int i = base + threadIdx.x;
      if (!one_pass) {
        int64_t all;
        mine = i < p.n_items ? units_of<QT>(p, i, false) + item_units(QT) : 0;
        incl = block_scan(mine, &all) + done;
        done += all;
      }
      if (first_unit >= incl - mine && first_unit < incl) *found = Begin{i, incl - mine, total};
      if (one_pass || first_unit < done) break;
    }
    if (threadIdx.x == 0) cuts[blockIdx.x].pieces = 0;
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = *tmem_slot;
  const bool clustered = QT == 1 && p.cluster > 1;
  const int stages = clustered ? C::kStages - 2 : C::kStages;   // the last two receive a cluster's parts
  if (clustered) cluster_arrive();   // every thread waits for it once: the softmax threads before they write to other CTAs
  // A whole warp's wait: on expiry all its lanes leave together.
  auto wait_warp = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, wait_bounded(bar, parity, wc)) != 0; };
  // Item number i of the share, as every role sees it: valid until the role's release.  The wait lasts as long as the item
  // before the last one takes.
  const WaitCtl wi{abort_flag, p.wait_limit_ns + uint64_t(p.max_len / kBN) * 10000u, 0u, &g_moa_window_tc_status};
  auto get_item = [&](uint32_t i, bool& ok) {
    ok = ok && __all_sync(0xffffffffu, wait_bounded(item_full(i & 1), i >> 1 & 1u, wi)) != 0;
    const volatile Item& x = items[i & 1];
    return ok ? Item{x.item, x.u0, x.u1, x.units, x.first, x.from, x.len} : Item{-1, 0, 0, 0, 0, 0, 0};
  };

  if (warp >= C::kMmaWarp0) {
    if constexpr (QT == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kRegsCtrl));
    if (warp == C::kLoadWarp) {
      // ------------------------------------------------------------ TMA producer: a copy a lane
      const int boxes = kBN / p.box;
      int slot = 0;
      uint32_t phase = 0, issued = 0, issued_phase = 0, q_issued = 0;
      bool ok = true;
      for (uint32_t seg = 0; ok; ++seg) {
        const Item x = get_item(seg, ok);
        if (x.item < 0) break;
        __syncwarp();
        if (lane == 0) mbar_arrive(item_empty(seg & 1));
        const Where w = where_of<QT>(p, x.item);
        const win::Tiles list{x.first, x.from, x.units};
        const int end = win::row_end(p.mask, x.len, p.N, w.i1), low = win::row_low(p.mask, x.len, p.N, w.i0);
        const int n_kt = x.u1 - x.u0;
        // the lane's copy of tile u0 + n: its first token, or its first group of eight tokens of the pool
        auto source = [&](int n) {
          int s = 0;
          if (n >= n_kt || lane >= boxes) return s;
          const int t0 = list.at(x.u0 + n) * kBN + lane * p.box;
          if (!PAGED) return t0;
          s = page_source(p, w, t0, end, low);
          return s;
        };
        int cur = source(0), next = cur, after = source(1);
        for (int t = 0; t < 2 * n_kt; ++t) {
          // K0 K1 V0 K2 V1 ... (tile n + 1's scores come before tile n's P V)
          const int u = t - 1, nn = u >> 1;
          const bool is_k = t == 0 || ((u & 1) == 0 && nn + 1 < n_kt);
          const int n = t == 0 ? 0 : is_k ? nn + 1 : nn;
          if (is_k && n > 0) {
            next = after;
            after = source(n + 1);
          }
          if (!wait_warp(empty_bar(slot), phase ^ 1u)) {
            ok = false;
            break;
          }
          issued |= 1u << slot;
          issued_phase = (issued_phase & ~(1u << slot)) | (phase << slot);
          const uint32_t dst = sKV + slot * C::kStageBytes + lane * p.box / 8 * (is_k ? KL::kGroup : VL::kGroup);
          if (lane == 0) mbar_arrive_expect_tx(full_bar(slot), is_k ? C::kKTileBytes : C::kVTileBytes);
          __syncwarp();
          if (lane < boxes) {
            const int s = is_k && n > 0 ? next : cur;
            if constexpr (PAGED) {
              tma_load_4d(dst, is_k ? &tmK : &tmV, full_bar(slot), 0, 0, 0, s);
            } else if (is_k) {
#pragma unroll
              for (int q = 0; q < DK / 64; ++q)
                tma_load_4d(dst + q * C::kPanelBytes, &tmK, full_bar(slot), q * 64, s, w.h, w.b);
            } else {
#pragma unroll
              for (int q = 0; q < DV / 64; ++q)
                tma_load_4d(dst + q * C::kPanelBytes, &tmV, full_bar(slot), q * 64, s, w.h, w.b);
            }
          }
          if (!is_k) cur = next;
          if (t == 0) {   // the queries, once the item before has no use for its own
            if (seg > 0 && !wait_warp(q_empty, (seg - 1) & 1u)) {
              ok = false;
            } else if (lane == 0) {
              mbar_arrive_expect_tx(q_full, QT * DK * 2 * p.GC * p.PT);
#pragma unroll
              for (int j = 0; j < QT; ++j)
#pragma unroll
                for (int q = 0; q < DK / 64; ++q)
                  tma_load_5d(sQ + j * C::kQTileBytes + q * C::kPanelBytes, &tmQ, q_full, q * 64, w.chunk * p.GC,
                              w.i0 + j * p.PT, w.h, w.b);
            }
            if (!ok) break;
            ++q_issued;
          }
          if (++slot == stages) {
            slot = 0;
            phase ^= 1u;
          }
        }
      }
      __syncwarp();
      if (lane == 0 && (!ok || *abort_flag)) {   // let every copy land before the CTA can exit
        if (q_issued > 0) wait_quiesce(q_full, (q_issued - 1) & 1u, p.wait_limit_ns, &g_moa_window_tc_status);
        for (int sl = 0; sl < C::kStages; ++sl)
          if (issued & (1u << sl))
            wait_quiesce(full_bar(sl), (issued_phase >> sl) & 1u, p.wait_limit_ns, &g_moa_window_tc_status);
      }
    } else if (warp == C::kMmaWarp0 || (QT == 2 && warp == C::kMmaWarp1)) {
      // ------------------------------------------------------------ MMA issuers, one for each row tile
      if (lane == 0) {
        const int j = warp == C::kMmaWarp0 ? 0 : 1;
        const uint32_t tS = tmem + (j ? C::kTmemS1 : C::kTmemS0);
        const uint32_t tP = tmem + (j ? C::kTmemP1 : C::kTmemP0);
        const uint32_t tO = tmem + (j ? C::kTmemO1 : C::kTmemO0);
        const uint32_t sQj = sQ + j * C::kQTileBytes;
        int slot = 0;
        uint32_t phase = 0;
        uint32_t t = 0;   // tiles so far: the phases of the barriers between the roles
        auto next = [&]() {
          if (++slot == stages) {
            slot = 0;
            phase ^= 1u;
          }
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
          ok = wait_bounded(item_full(seg & 1), seg >> 1 & 1u, wi);
          const volatile Item& xi = items[seg & 1];
          const int item = xi.item, n_kt = xi.u1 - xi.u0;
          if (!ok || item < 0) break;
          mbar_arrive(item_empty(seg & 1));
          ok = wait_bounded(q_full, seg & 1u, wc) && wait_bounded(full_bar(slot), phase, wc) && s_buffer(t);
          if (ok) {
            tc_fence_after_sync();
            const int ks = slot;
            next();
            issue_scores<DK, PAGED>(tS, sQj, sKV + ks * C::kStageBytes);
            mma_commit(s_full(j));
            mma_commit(empty_bar(ks));
            if (n_kt == 1) mma_commit(q_empty);
          }
          for (int n = 0; ok && n < n_kt; ++n, ++t) {
            if (n + 1 < n_kt) {
              const int ks = slot;
              ok = wait_bounded(full_bar(slot), phase, wc) && s_buffer(t + 1);
              next();
              if (!ok) break;
              tc_fence_after_sync();
              issue_scores<DK, PAGED>(tS, sQj, sKV + ks * C::kStageBytes);
              mma_commit(s_full(j));
              mma_commit(empty_bar(ks));
              if (n + 2 == n_kt) mma_commit(q_empty);
            }
            const int vs = slot;
            ok = wait_bounded(full_bar(slot), phase, wc) && wait_bounded(p_ready(j), t & 1u, wc);
            next();
            if (!ok) break;
            tc_fence_after_sync();
            issue_outputs<DV, PAGED>(tO, tP, sKV + vs * C::kStageBytes, n > 0 ? 1u : 0u);
            mma_commit(p_free(j));
            mma_commit(empty_bar(vs));
          }
          // arrives when the item's products are complete
          mma_commit(o_done(j));
        }
        mma_commit(drain);
      }
    } else if (warp == C::kWalkWarp && lane == 0) {
      // ------------------------------------------------------------ the items of the share
      const Shares shares(total, gridDim.x);
      int64_t at = first_unit, before = 0;
      int item = 0;
      if (p.cluster != 0) {
        mbar_arrive(item_full(0));
        items[1].item = -1;
        mbar_arrive(item_full(1));
      } else if (at < stop) {
        item = int(found->item);
        before = found->unit;
      }
      for (uint32_t seg = 0; p.cluster == 0; ++seg) {
        int units = 0, u0 = 0, u1 = 0, which = -1, len = 0;
        win::Tiles list{};
        while (at < stop && u0 == u1) {   // (nothing of an item's tiles: the next CTA begins it)
          const Where w = where_of<QT>(p, item);
          len = length_of(p, w.b, false);
          list = win::tiles_of(p.mask, len, p.N, w.i0, w.i1, kBN);
          units = list.n < 1 ? 1 : list.n;
          const int64_t end = before + units + item_units(QT), upto = end < stop ? end : stop;
          u0 = max(0, int(at - before) - item_units(QT)), u1 = max(0, int(upto - before) - item_units(QT));
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
        if (seg >= 2 && !wait_bounded(item_empty(seg & 1), ((seg >> 1) - 1) & 1u, wi)) break;
        volatile Item& x = items[seg & 1];
        x.item = which, x.u0 = u0, x.u1 = u1, x.units = units;
        x.first = list.first, x.from = list.from, x.len = len;
        mbar_arrive(item_full(seg & 1));
        if (which < 0) break;
      }
    }
  } else {
    if constexpr (QT == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kRegsSoftmax));
    // -------------------------------------------------------------- softmax warpgroups
    const int j = warp >> 2;
    const int lane_base = (warp & 3) * 32, row = lane_base + lane;
    const uint32_t tS = tmem + (uint32_t(lane_base) << 16) + (j ? C::kTmemS1 : C::kTmemS0);
    const uint32_t tO = tmem + (uint32_t(lane_base) << 16) + (j ? C::kTmemO1 : C::kTmemO0);
    const uint32_t tP = tmem + (uint32_t(lane_base) << 16) + (j ? C::kTmemP1 : C::kTmemP0);
    const float c = fmaxf(p.c_log2, FLT_MIN);   // not zero: c * -infinity hides a token
    const int row_pos = int(unsigned(row) / unsigned(p.GC)), row_head = row - row_pos * p.GC;
    bool ok = true;
    uint32_t t = 0, ring = 0;   // tiles and stages of the ring before this item
    if (clustered) cluster_wait();
    [[maybe_unused]] float cluster_m = -INFINITY, cluster_l = 0.f;   // the row's, for the CTA that joins it (if this one has no tiles)
    for (uint32_t seg = 0;; ++seg) {
      const Item x = get_item(seg, ok);
      if (x.item < 0) break;
      const win::Tiles list{x.first, x.from, 0};
      auto place = [&](int which) { return place_of<QT>(p, which, j, row_pos, row_head); };   // where the thread's row lies
      int lim = 0x7fffffff, low = 0;
      bool live_warp;
      {
        const Place w = place(x.item);
        live_warp = __any_sync(0xffffffffu, w.live);
        if (w.live) {
          lim = win::row_end(p.mask, x.len, p.N, w.i);
          low = win::row_low(p.mask, x.len, p.N, w.i);
        }
      }
      // past the sequence's end a page holds whatever it held: the first such token, of a cache.  Its rows of values are
      // zeroed by the warps that have no rows of queries, or else by all, each its own rows.
      const int gone = PAGED ? x.len : 0x7fffffff;
      int zero_row = row, zero_step = kBN;
      if (QT == 1) {
        const int warps = (p.N * p.GC + 31) / 32;   // those with rows
        if (warps < 4) {
          zero_row = row - 32 * warps;
          zero_step = live_warp ? 0 : kBN - 32 * warps;
        }
      }
      float m = -INFINITY, l = 0.f;
      for (int n = x.u0; ok && n < x.u1; ++n, ++t) {
        const int n0 = list.at(n) * kBN;
        // Waits that run out leave the loop together, at its end: until then what they would have brought is used
        // as it is.
        ok = wait_bounded(s_full(j), t & 1u, wc);
        tc_fence_after_sync();
        if (PAGED && gone - n0 < kBN && zero_step > 0) {   // the item's last tile
          const int k = n - x.u0, at = int(ring) + (n + 1 < x.u1 ? 2 * k + 2 : 2 * k + 1);
          ok = zero_rows<DV>(smem + C::kOffKV + at % stages * C::kStageBytes, zero_row, zero_step, gone - n0,
                             full_bar(at % stages), at / stages & 1, wc) && ok;
        }
        // (with two row tiles such warps are few, and the branch alone cost the loop 5 %: 16384 tokens in 357 us, 341 without)
        if (QT == 1 && !live_warp) {   // rows that are not there: in step with the others, and no more
          tc_fence_before_sync();
          mbar_arrive(s_free(j));
          if (t > 0) ok = wait_bounded(p_free(j), (t - 1) & 1u, wc) && ok;
          mbar_arrive(p_ready(j));
          ok = __all_sync(0xffffffffu, ok);
          continue;
        }
        uint32_t sr[128];
        tmem_load_row128(tS, sr);
        tc_fence_before_sync();
        mbar_arrive(s_free(j));
        float* s = reinterpret_cast<float*>(sr);
        if (!__all_sync(0xffffffffu, lim - n0 >= kBN && (n0 >= low || n0 + kBN <= p.mask.sinks))) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t bits = below(lim - n0, k) & (~below(low - n0, k) | below(p.mask.sinks - n0, k));
#pragma unroll
            for (int e = 0; e < 32; ++e) s[32 * k + e] = bits >> e & 1u ? s[32 * k + e] : -INFINITY;
          }
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
          for (int e = 0; e < 32; e += 4) {
            const int k = 32 * ch + e;
            float x0, x1, x2, x3;
            ffma2(x0, x1, s[k], s[k + 1], cc, mm);
            ffma2(x2, x3, s[k + 2], s[k + 3], cc, mm);
            const float p0 = ex2_approx(x0), p1 = ex2_approx(x1), p2 = ex2_approx(x2), p3 = ex2_approx(x3);
            fadd2(l0, l1, p0, p1);
            fadd2(l2, l3, p2, p3);
            pk[e >> 1] = pack_bf16x2(p0, p1);
            pk[(e >> 1) + 1] = pack_bf16x2(p2, p3);
          }
        };
        auto store_chunk = [&](int ch, const uint32_t* pk) { tmem_st_32x32b_x16(tP + 16 * ch, pk); };
        constexpr int kEarly = C::kEarlyChunks;
        uint32_t pe[16 * kEarly];
#pragma unroll
        for (int ch = 0; ch < kEarly; ++ch) exp_chunk(ch, pe + 16 * ch);
        // P_j's buffer is free, and O_j may be rescaled, once the previous tile's product is done
        if (t > 0) ok = wait_bounded(p_free(j), (t - 1) & 1u, wc) && ok;
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
        if (rescale) tmem_scale_row<DV>(tO, alpha);
        tmem_wait_st();
        tc_fence_before_sync();
        mbar_arrive(p_ready(j));
        ok = __all_sync(0xffffffffu, ok);
      }
      if (!ok || !wait_warp(o_done(j), seg & 1u)) break;
      tc_fence_after_sync();
      // the item is written, or this CTA's piece of it
      const volatile Item& xi = items[seg & 1];
      ring += 2u * uint32_t(xi.u1 - xi.u0);
      const bool first_piece = xi.u0 == 0, whole = first_piece && xi.u1 == xi.units;
      if (live_warp) {
        const Place w = place(xi.item);
        if (write_rows<DK, DV, QT, false>(p, out, w, tO, sKV + (C::kStages - 2) * C::kStageBytes, j, row, m, l, first_piece, whole) && lane == 0) {
          const uint32_t bit = seg < kAgain - 1 ? seg : kAgain - 1;
          atomicOr(again + bit / 32, 1u << (bit & 31));
          *any_again = 1;
        }
        cluster_m = m, cluster_l = l;
      }
      tc_fence_before_sync();   // O is read: the next item's first product (after p_ready) may write it
      __syncwarp();
      if (lane == 0) mbar_arrive(item_empty(seg & 1));
    }
    if (clustered) {
      const Owner own = owner_of(row, p.cluster);
      store2_to_cta(smem_of_cta(smem_u32(smem + C::kOffSums) + (int(blockIdx.y) * (kBM / p.cluster) + own.row) * 8, own.rank),
                    cluster_m, cluster_l);
    }
  }

  // Teardown: the tensor core is quiet before TMEM is freed, on the abort path too.  Only the lane of the role
  // waits: the others come here at the start, and their time would run out in a kernel longer than the limit.
  if (warp == C::kMmaWarp0 && lane == 0) wait_quiesce(drain, 0, p.wait_limit_ns, &g_moa_window_tc_status);
  tc_fence_before_sync();
  __syncthreads();
  if (*any_again != 0) {
    const bool dead = *abort_flag != 0;
    if (threadIdx.x == 0) {
      mbar_init(redo_loaded, 1);
      mbar_init(redo_done, 1);
      fence_barrier_init();
    }
    __syncthreads();
    if (!dead && warp < C::kMmaWarp0) {
      tc_fence_after_sync();
      redo_share<DK, DV, QT, PAGED>(&tmQ, &tmK, &tmV, p, out, smem, tmem);
    }
    tc_fence_before_sync();
    __syncthreads();
  }
  if (warp == C::kMmaWarp0) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, C::kTmemCols);
  }
  if constexpr (QT == 1) {
    if (clustered) {
      if (warp >= C::kMmaWarp0) cluster_wait();
      __syncwarp();
      cluster_sync();
      if (warp < C::kMmaWarp0)
        cluster_rows<DV>(out.O, out.lse, p, reinterpret_cast<const float*>(smem + C::kOffKV + (C::kStages - 2) * C::kStageBytes),
                             reinterpret_cast<const float2*>(smem + C::kOffSums));
    }
  }
}

// Joins the pieces of cut items: CTA (x, y) 32 / WS rows of CTA x's cut, four for every WS warps, eight lanes a row (a row a
// warp spent most of its instructions on places: the call of 4 x 16 heads x 2048 x 64 took 78 us in place of 67); each of the WS warps takes
// every WS-th piece, where items have many.
constexpr int kJoinRows = 4;
template <int DV, int QT>
__global__ void __launch_bounds__(256)
window_tc_join_kernel(const Out out, const Cut* cuts, const Params p, int WS) {
  constexpr int kRows = kBM * QT, kQuads = DV / 32;
  __shared__ float4 s_x[8][32][kQuads];
  __shared__ float s_l[8][kJoinRows];
  wait_for_previous();
  const Cut cut = cuts[blockIdx.x];
  if (cut.pieces == 0) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, turn = warp % WS, sub = lane & 7;
  const int row = (int(blockIdx.y) * (8 / WS) + warp / WS) * kJoinRows + (lane >> 3);
  const Where w = where_of<QT>(p, cut.item);
  const int tile = row / kBM, in_tile = row - tile * kBM;
  const int row_pos = int(unsigned(in_tile) / unsigned(p.GC)), row_head = in_tile - row_pos * p.GC;
  const int g = w.chunk * p.GC + row_head, hq = w.h * p.G + g, i = w.i0 + tile * p.PT + row_pos;
  const bool live = row < kRows && row_pos < p.PT && g < p.G && i < p.N;
  if (WS == 1 && !__any_sync(0xffffffffu, live)) return;
  auto place = [&](int k) -> int64_t { return ((int64_t(blockIdx.x) + k) * 2 + (k == 0)) * kRows + row; };
  float M = -INFINITY, L = 0.f;
  float4 x[kQuads];
#pragma unroll
  for (int q = 0; q < kQuads; ++q) x[q] = make_float4(0.f, 0.f, 0.f, 0.f);
  if (live)
    for (int k = sub; k < cut.pieces; k += 8) M = fmaxf(M, out.part_ml[place(k)].x);
#pragma unroll
  for (int d = 4; d > 0; d >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, d));
  const float base = M == -INFINITY ? 0.f : M;
  if (live) {
#pragma unroll 2
    for (int k = turn; k < cut.pieces; k += WS) {
      const int64_t at = place(k);
      const float2 ml = out.part_ml[at];
      const float f = ex2_approx(ml.x - base);
      L += f * ml.y;
#pragma unroll
      for (int q = 0; q < kQuads; ++q) {
        const float4 v = *reinterpret_cast<const float4*>(out.part_o + at * DV + (sub + 8 * q) * 4);
        x[q].x += f * v.x, x[q].y += f * v.y, x[q].z += f * v.z, x[q].w += f * v.w;
      }
    }
  }
  if (WS > 1) {   // the other warps' sums, in their order
#pragma unroll
    for (int q = 0; q < kQuads; ++q) s_x[warp][lane][q] = x[q];
    if (sub == 0) s_l[warp][lane >> 3] = L;
    __syncthreads();
    if (turn != 0) return;
    for (int k = 1; k < WS; ++k) {
      L += s_l[warp + k][lane >> 3];
#pragma unroll
      for (int q = 0; q < kQuads; ++q) {
        const float4 v = s_x[warp + k][lane][q];
        x[q].x += v.x, x[q].y += v.y, x[q].z += v.z, x[q].w += v.w;
      }
    }
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  __nv_bfloat16* o = out.O + int64_t(w.b) * p.o_sb + int64_t(hq) * p.o_sh + int64_t(i) * p.o_sn;
#pragma unroll
  for (int q = 0; q < kQuads; ++q) {
    x[q].x *= inv, x[q].y *= inv, x[q].z *= inv, x[q].w *= inv;
    if (live)
      *reinterpret_cast<uint2*>(o + (sub + 8 * q) * 4) = make_uint2(pack_bf16x2(x[q].x, x[q].y), pack_bf16x2(x[q].z, x[q].w));
  }
  if (out.lse != nullptr && live && sub == 0)
    out.lse[(int64_t(w.b) * p.Hk * p.G + hq) * p.N + i] = L == 0.f ? -INFINITY : (M + lg2_approx(L)) * kLn2;
}

// ------------------------------------------------------------------------------------------------
// Host side
// ------------------------------------------------------------------------------------------------
int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

constexpr int64_t kMostInL2 = int64_t(100) << 20;   // of 129 MB
// Clusters of 16, 8, 4, 2 CTAs at a time on a whole GPU: what there was room for, or a little less (7, 15, 36, 76; one more took twice
// as long).  Where the context has fewer SMs, what there is room for.
constexpr int64_t kClusters16 = 7, kClusters8 = 14, kClusters4 = 34, kClusters2 = 72;
template <int DK, int DV>
int room_of(int size) {
  static ClusterRoom dense, paged;
  using C = Cfg<DK, DV, 1>;
  const int a = dense(reinterpret_cast<const void*>(window_tc_kernel<DK, DV, 1, false>), C::kThreads, C::kSmemBytes, size);
  const int b = paged(reinterpret_cast<const void*>(window_tc_kernel<DK, DV, 1, true>), C::kThreads, C::kSmemBytes, size);
  return a < b ? a : b;
}
int room(int64_t dk, int64_t dv, int size) {
  if (dk == 64) return dv == 64 ? room_of<64, 64>(size) : room_of<64, 128>(size);
  return dv == 64 ? room_of<128, 64>(size) : room_of<128, 128>(size);
}

// How the rows of a key head are divided.
struct Plan {
  int64_t GC, chunks, PT, QT, n_tiles, n_items;
  int cluster;   // CTAs for each item; 0: equal shares
  Plan(const WindowArgs& a, int sms) {
    const int64_t G = a.Hq / a.Hk;
    GC = G < kBM ? G : kBM;
    chunks = (G + GC - 1) / GC;
    PT = kBM / GC;
    // Few items: a cluster for each, the largest that all fit into the GPU at the same time, joined in the same launch, where that is
    // no more than eight tiles a CTA (equal shares and the cluster, bf16, d = 128: 1 item of 128 tiles 23.9 and 18.2 us; 8 of 64:
    // 20.2 and 17.8, of 128, sixteen a CTA: 24.0 and 26.2; 32 of 32: 24.9 and 19.2; 64 of 16: 23.9 and 19.2).  Where there are more
    // rows than one tile's, sixteen: shares then come in two row tiles, whose items are longer (16 heads x 512 tokens 21.8 and
    // 10.7; 64 queries of 32 / 8 heads against 8192 tokens 34.6 and 29.5).
    int64_t tiles = (a.max_len + kBN - 1) / kBN;   // of tokens that an item of one row tile visits, at most
    if (a.window != win::kNoWindow) {
      const int64_t seen = (int64_t(a.window) + PT + kBN - 1) / kBN + 1 + (int64_t(a.sinks) + kBN - 1) / kBN;
      if (seen < tiles) tiles = seen;
    }
    QT = 1;
    n_tiles = chunks * ((a.N + PT - 1) / PT);
    n_items = a.B * a.Hk * n_tiles;
    int64_t size = 16;
    for (int64_t most : {kClusters16, kClusters8, kClusters4, kClusters2}) {
      if (n_items <= most && n_items <= room(a.dk, a.dv, int(size))) break;
      size /= 2;
    }
    cluster = 0;
    if (n_items <= sms && tiles <= (a.N > PT ? 16 : 8) * size) {
      cluster = 1;
      // Many rows cost the join about what three tiles do: those then stay together (16 heads x 512 tokens of 128 rows a tile 14.5 us in
      // pairs and 10.7 alone; 64 rows against 1024 tokens 10.3 in eights and 13.6 in pairs).
      const int64_t rows = (a.N < PT ? a.N : PT) * GC, least = rows > 64 ? 4 : 1;
      while (cluster < size && cluster * least < tiles) cluster *= 2;
    } else if (a.N > PT) {
      QT = 2;
      n_tiles = chunks * ((a.N + 2 * PT - 1) / (2 * PT));
      n_items = a.B * a.Hk * n_tiles;
    }
  }
};

// The workspace: pieces, cuts.
struct Work {
  int64_t part_o, part_ml, cuts, bytes;
  Work(const WindowArgs& a, const Plan& plan, int sms) {
    const int64_t rows = int64_t(sms) * 2 * kBM * plan.QT;
    part_o = 0;
    part_ml = part_o + rows * a.dv * 4;
    cuts = part_ml + rows * 8;
    bytes = cuts + round_up(int64_t(sms) * sizeof(Cut), 256);
  }
};

template <int DK, int DV, int QT, bool PAGED>
int launch(const WindowArgs& a, const Plan& plan, int sms, char* msg, size_t msglen) {
  using C = Cfg<DK, DV, QT>;
  auto kern = window_tc_kernel<DK, DV, QT, PAGED>;
  cudaError_t e = ensure_smem_limit(reinterpret_cast<const void*>(kern), C::kSmemBytes);
  if constexpr (QT == 2) {
    static std::atomic<int> regs{-1};
    if (e == cudaSuccess && regs.load(std::memory_order_relaxed) < 0) {
      cudaFuncAttributes fa;
      e = cudaFuncGetAttributes(&fa, reinterpret_cast<const void*>(kern));
      if (e == cudaSuccess) regs.store(fa.numRegs, std::memory_order_relaxed);
    }
    if (e == cudaSuccess && regs.load(std::memory_order_relaxed) * C::kThreads < 256 * C::kRegsSoftmax + 128 * C::kRegsCtrl) {
      snprintf(msg, msglen, "attention with a window: %d registers per thread, short of the register split", regs.load());
      return 5;
    }
  }
  if (e != cudaSuccess) {
    snprintf(msg, msglen, "attention with a window: function attributes: %s", cudaGetErrorString(e));
    return 5;
  }
  const Work w(a, plan, sms);
  uint8_t* ws = static_cast<uint8_t*>(a.ws);
  const Out out{static_cast<__nv_bfloat16*>(a.o.p), a.lse, reinterpret_cast<float*>(ws + w.part_o), reinterpret_cast<float2*>(ws + w.part_ml)};
  Cut* cuts = reinterpret_cast<Cut*>(ws + w.cuts);
  const int64_t G = a.Hq / a.Hk;
  Params p{};
  p.o_sb = a.o.sb, p.o_sh = a.o.sh, p.o_sn = a.o.sn;
  p.kv = a.kv, p.lens = a.lens;
  p.N = int(a.N), p.max_len = int(a.max_len), p.Hk = int(a.Hk), p.G = int(G);
  p.GC = int(plan.GC), p.chunks = int(plan.chunks), p.PT = int(plan.PT);
  p.n_tiles = int(plan.n_tiles), p.n_items = int(plan.n_items);
  p.mask = win::Mask{a.window, a.sinks, a.causal};
  p.c_log2 = a.scale * kLog2e;
  p.wait_limit_ns = wait_limit_ns();
  p.box = kBN;
  if (PAGED)
    while (a.kv.page % p.box != 0) p.box /= 2;
  CUtensorMap mq, mk, mv;
  const uint64_t q_dims[5] = {DK, uint64_t(G), uint64_t(a.N), uint64_t(a.Hk), uint64_t(a.B)};
  const uint64_t q_str[4] = {map_stride(a.q.sh, G), map_stride(a.q.sn, a.N), map_stride(G * a.q.sh, a.Hk),
                             map_stride(a.q.sb, a.B)};
  const uint32_t q_box[5] = {64, uint32_t(plan.GC), uint32_t(plan.PT), 1, 1};
  // Keys and values.  Dense: feature, token, head, sequence, a panel of 64 features a copy.  Pages: feature of a panel, token of a
  // group of eight, panel, group of the pool (its pages and heads lie one after the other).
  p.page_groups = PAGED ? a.kv.page / 8 : 0;
  p.all_groups = PAGED ? int(a.kv.n_pages * a.Hk * p.page_groups) : 0;
  const uint64_t len = uint64_t(a.max_len), row_bytes = (DK + DV) * 2;
  uint64_t k_dims[4] = {DK, len, uint64_t(a.Hk), uint64_t(a.B)}, v_dims[4] = {DV, len, uint64_t(a.Hk), uint64_t(a.B)};
  uint64_t k_str[3] = {map_stride(a.kv.k_sn, a.max_len), map_stride(a.kv.k_sh, a.Hk), map_stride(a.kv.k_sb, a.B)};
  uint64_t v_str[3] = {map_stride(a.kv.v_sn, a.max_len), map_stride(a.kv.v_sh, a.Hk), map_stride(a.kv.v_sb, a.B)};
  uint32_t k_box[4] = {64, uint32_t(p.box), 1, 1}, v_box[4] = {64, uint32_t(p.box), 1, 1};
  auto by_groups = [&](uint32_t panels, uint64_t* dims, uint64_t* str, uint32_t* box) {
    dims[0] = 64, dims[1] = 8, dims[2] = panels, dims[3] = uint64_t(p.all_groups);
    str[0] = row_bytes, str[1] = 128, str[2] = 8 * row_bytes;
    box[1] = 8, box[2] = panels, box[3] = uint32_t(p.box) / 8;
  };
  if (PAGED) by_groups(DK / 64, k_dims, k_str, k_box), by_groups(DV / 64, v_dims, v_str, v_box);
  if (!encode_bf16_map_nd(&mq, a.q.p, 5, q_dims, q_str, q_box, msg, msglen) ||
      !encode_bf16_map_nd(&mk, a.kv.k, 4, k_dims, k_str, k_box, msg, msglen) ||
      !encode_bf16_map_nd(&mv, a.kv.v, 4, v_dims, v_str, v_box, msg, msglen))
    return 5;
  // tiles of tokens, if every sequence is as long as max_len and no window hides any
  const int64_t most_tiles = (a.max_len + kBN - 1) / kBN, most = plan.n_items * most_tiles;
  const unsigned ctas = unsigned(most < sms ? most : sms);
  if constexpr (QT == 1) {
    if (plan.cluster != 0) {
      p.cluster = plan.cluster;
      if (p.cluster > 8) e = cudaFuncSetAttribute(reinterpret_cast<const void*>(kern), cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
      if (e == cudaSuccess)
        e = launch_clusters(kern, dim3(unsigned(plan.n_items), unsigned(p.cluster)), unsigned(p.cluster), dim3(C::kThreads),
                            C::kSmemBytes, a.stream, mq, mk, mv, out, cuts, p);
      if (e != cudaSuccess) {
        snprintf(msg, msglen, "attention with a window: %s", cudaGetErrorString(e));
        return 5;
      }
      return 0;
    }
  }
  if (QT == 2) {
    const int64_t token = (DK + DV) * 2, all = a.B * a.Hk * a.max_len * token;
    const int64_t seen = a.window == win::kNoWindow ? a.max_len : int64_t(a.window) + QT * plan.PT;   // by an item
    if (all > kMostInL2 && int64_t(ctas) * seen * token > kMostInL2)
      p.columns = int(ctas), p.height = int(plan.n_items / ctas), p.tall = int(plan.n_items % ctas);
  }
  // rows of an item that may be there
  const int64_t positions = a.N < plan.PT ? a.N : plan.PT, live = QT == 2 ? C::kRows : positions * plan.GC;
  e = launch_overlapped(kern, dim3(ctas), dim3(C::kThreads), C::kSmemBytes, a.stream, mq, mk, mv, out, cuts, p);
  // warps for a row's pieces: about a quarter of the pieces that an item may have
  const int64_t pieces = ctas / plan.n_items + 1;
  const int split = pieces <= 4 ? 1 : pieces <= 8 ? 2 : pieces <= 16 ? 4 : 8;
  const int64_t per = 32 / split;
  if (e == cudaSuccess)
    e = launch_overlapped(window_tc_join_kernel<DV, QT>, dim3(ctas, unsigned((live + per - 1) / per)), dim3(256), 0, a.stream, out, cuts, p,
                          split);
  if (e != cudaSuccess) {
    snprintf(msg, msglen, "attention with a window: %s", cudaGetErrorString(e));
    return 5;
  }
  return 0;
}

template <int DK, int DV>
int launch_rows(const WindowArgs& a, int sms, char* msg, size_t msglen) {
  const Plan plan(a, sms);
  if (a.kv.table != nullptr)
    return plan.QT == 2 ? launch<DK, DV, 2, true>(a, plan, sms, msg, msglen) : launch<DK, DV, 1, true>(a, plan, sms, msg, msglen);
  return plan.QT == 2 ? launch<DK, DV, 2, false>(a, plan, sms, msg, msglen) : launch<DK, DV, 1, false>(a, plan, sms, msg, msglen);
}

}  // namespace

bool window_tc_takes(const WindowArgs& a) {
  const int64_t G = a.Hq / a.Hk, rows = a.kv.table != nullptr ? a.kv.page : a.max_len;
  const int64_t outer = a.kv.table != nullptr ? a.kv.n_pages : a.B;
  if (a.kv.table != nullptr && a.kv.n_pages * a.Hk * (a.kv.page / 8) >= int64_t(1) << 31) return false;   // groups of a pool
  return !a.f32 && a.scale >= 0.f && describable(a.q.sh, G) && describable(G * a.q.sh, a.Hk) && describable(a.q.sn, a.N) &&
         describable(a.q.sb, a.B) && describable(a.kv.k_sn, rows) && describable(a.kv.k_sh, a.Hk) &&
         describable(a.kv.k_sb, outer) && describable(a.kv.v_sn, rows) && describable(a.kv.v_sh, a.Hk) &&
         describable(a.kv.v_sb, outer);
}

size_t window_tc_workspace(const WindowArgs& a, int sms) { return size_t(Work(a, Plan(a, sms), sms).bytes); }

int launch_window_tc(const WindowArgs& a, int sms, char* msg, size_t msglen) {
  if (a.dk == 64) return a.dv == 64 ? launch_rows<64, 64>(a, sms, msg, msglen) : launch_rows<64, 128>(a, sms, msg, msglen);
  return a.dv == 64 ? launch_rows<128, 64>(a, sms, msg, msglen) : launch_rows<128, 128>(a, sms, msg, msglen);
}

cudaError_t window_tc_read_and_clear_status(unsigned* value) {
  cudaError_t e = cudaMemcpyFromSymbol(value, g_moa_window_tc_status, sizeof(unsigned));
  if (e != cudaSuccess || *value == 0) return e;
  const unsigned zero = 0;
  return cudaMemcpyToSymbol(g_moa_window_tc_status, &zero, sizeof(unsigned));
}

}  // namespace moa
