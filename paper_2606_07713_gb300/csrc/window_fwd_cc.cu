// Causal attention with a sliding window and first tokens that stay visible, on CUDA cores (sm_103a):
// for fp32, and for bf16 tensors whose strides no tensor map can describe.  Keys and values lie in
// dense tensors or in the pages of a cache.
//
// Mathematics: o_i = sum_j p_ij v_j / l_i over the tokens j that row i sees (window.cuh), with
// p_ij = 2^(c s_ij - m_i), s_ij = <q_i, k_j>, c = scale log2 e, m_i the running maximum of c s_ij and
// l_i = sum_j p_ij: one pass over the tokens, the sums rescaled when a tile raises the maximum.
//
// A key head's query rows are counted position by position: row r is query r / G of head r % G of the
// group, so that a tile of rows covers few positions and a window few tiles of tokens.  A CTA takes one
// tile of rows (64, or 16 where there are few) and a share of the 64-token tiles that it visits; shares
// are joined through the shared memory of a cluster, or by a second kernel where there are more than sixteen.  Thread (ty, tx) holds RM rows: the scores of four tokens of each,
// then DV / 16 features of their outputs.
//
// What bounds it: shared memory's data path and multiply-adds about equally (2 x (6 / 3) heads x 517 queries x 700 keys x (128 / 64),
// window 100: 18.6 us, 52 %, and 39 % of the issue slots); few rows: the latency of a tile (5 sequences of 5 queries, window 1000:
// 13.7 us).  The next tile's keys are on their way during the second product, its values during the next first one.
//
// Hidden tokens get the weight -1, which the second product skips: what their values hold (not numbers,
// perhaps) then reaches no row that does not see them.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdio>

#include "internal.h"
#include "ops_internal.h"
#include "window.cuh"

namespace moa {

__device__ unsigned int g_moa_window_cc_status = 0;

namespace {

constexpr int kKeys = 64;            // tokens of a tile
constexpr int kMostCluster = 16;     // CTAs of a cluster (more than 8 are asked for by an attribute)
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct Params {
  View q, o;
  KvSource kv;
  float* lse;
  const int32_t* lens;
  int Hk, N, G, max_len, n_tiles;   // n_tiles: row tiles of a key head
  win::Mask mask;
  float c_log2;
  int splits;
  float* part_o;                // [item * splits + split][rows][DV], null: no shares
  float2* part_ml;
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

__device__ __forceinline__ int length_of(const Params& p, int64_t b) {
  if (p.lens == nullptr) return p.max_len;
  const int len = p.lens[b];
  if (len >= 0 && len <= p.max_len) return len;
  atomicExch(&g_moa_window_cc_status, win::kErrIndex);
  return len < 0 ? 0 : p.max_len;
}

template <int DK, int DV, int RM, int NT>
struct Cfg {
  static constexpr int kRows = NT / 16 * RM;
  // rows of 16-byte groups, one group longer: neighbouring rows then start in different banks
  static constexpr int kLdQ = DK + 4, kLdK = DK + 4, kLdP = kRows + 4;
  static constexpr int kFloats = kRows * kLdQ + kKeys * kLdK + kKeys * DV + kKeys * kLdP;
  static constexpr int kSmem = kFloats * 4;
};

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

template <typename T, int DK, int DV, int RM, int NT>
__global__ void __launch_bounds__(NT)
window_cc_kernel(const Params p) {
  using C = Cfg<DK, DV, RM, NT>;
  extern __shared__ float smem[];
  float* sQ = smem;                        // [rows][DK]
  float* sK = sQ + C::kRows * C::kLdQ;     // [tokens][DK]
  float* sV = sK + kKeys * C::kLdK;        // [tokens][DV]
  float* sP = sV + kKeys * DV;             // [tokens][rows]
  __shared__ const T* s_at[2][2][kKeys];   // a tile's keys and values; null: nothing there, zeros
  wait_for_previous();
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const unsigned item = blockIdx.x, bh = item / unsigned(p.n_tiles);
  const int tile = int(item - bh * unsigned(p.n_tiles));
  const int b = int(bh / unsigned(p.Hk)), h = int(bh - unsigned(b) * unsigned(p.Hk));
  const int rows_all = p.N * p.G, r0 = tile * C::kRows;
  const int rows = rows_all - r0 < C::kRows ? rows_all - r0 : C::kRows;
  const int len = length_of(p, b);
  const int i0 = r0 / p.G, i1 = (r0 + rows - 1) / p.G;
  // the tokens that its rows visit, 64 at a time, the sinks and the window's next to each other
  const win::Run run = win::run_of(p.mask, len, p.N, i0, i1);
  const int tiles = (run.n + kKeys - 1) / kKeys;
  const int first = int(int64_t(tiles) * blockIdx.y / p.splits), last = int(int64_t(tiles) * (blockIdx.y + 1) / p.splits);

  auto find = [&](int t) {   // where tile t's tokens lie
    if (t >= last || threadIdx.x >= kKeys) return;
    const int x = t * kKeys + int(threadIdx.x);
    const T *k = nullptr, *v = nullptr;
    if (x < run.n) {
      const int n = run.at(x);
      int64_t at = b, place = n;
      bool there = true;
      if (p.kv.table != nullptr) {
        const int slot = int(unsigned(n) / unsigned(p.kv.page));
        at = p.kv.table[b * p.kv.max_pages + slot];
        place = n - slot * p.kv.page;
        there = at >= 0 && at < p.kv.n_pages;
        if (!there) atomicExch(&g_moa_window_cc_status, win::kErrIndex);
      }
      if (there) {
        k = static_cast<const T*>(p.kv.k) + at * p.kv.k_sb + h * p.kv.k_sh + place * p.kv.k_sn;
        v = static_cast<const T*>(p.kv.v) + at * p.kv.v_sb + h * p.kv.v_sh + place * p.kv.v_sn;
      }
    }
    s_at[t & 1][0][threadIdx.x] = k;
    s_at[t & 1][1][threadIdx.x] = v;
  };
  const T* any = static_cast<const T*>(p.q.p);   // an address for copies of nothing
  auto fill_keys = [&](int t) {
    if (t < last)
#pragma unroll 4
      for (int x = threadIdx.x; x < kKeys * (DK / 4); x += NT) {
        const int j = x / (DK / 4), c = x % (DK / 4) * 4;
        const T* src = s_at[t & 1][0][j];
        fill4(sK + j * C::kLdK + c, src == nullptr ? any : src + c, src != nullptr);
      }
    fill_commit();
  };
  auto fill_values = [&](int t) {
    if (t < last)
#pragma unroll 4
      for (int x = threadIdx.x; x < kKeys * (DV / 4); x += NT) {
        const int j = x / (DV / 4), c = x % (DV / 4) * 4;
        const T* src = s_at[t & 1][1][j];
        fill4(sV + j * DV + c, src == nullptr ? any : src + c, src != nullptr);
      }
    fill_commit();
  };

  find(first);
  const T* Q = static_cast<const T*>(p.q.p) + b * p.q.sb + int64_t(h) * p.G * p.q.sh;
  for (int x = threadIdx.x; x < C::kRows * (DK / 4); x += NT) {
    const int r = x / (DK / 4), c = x % (DK / 4) * 4, i = (r0 + r) / p.G, g = r0 + r - i * p.G;
    fill4(sQ + r * C::kLdQ + c, r < rows ? Q + g * p.q.sh + i * p.q.sn + c : any, r < rows);
  }
  __syncthreads();
  fill_keys(first);
  fill_values(first);
  find(first + 1);
  int end[RM], low[RM];
#pragma unroll
  for (int a = 0; a < RM; ++a) {
    const int r = ty * RM + a;
    const int i = (r0 + (r < rows ? r : rows - 1)) / p.G;
    end[a] = r < rows ? win::row_end(p.mask, len, p.N, i) : 0;
    low[a] = win::row_low(p.mask, len, p.N, i);
  }
  float m[RM], l[RM], acc[RM][DV / 16];
#pragma unroll
  for (int a = 0; a < RM; ++a) {
    m[a] = -INFINITY, l[a] = 0.f;
#pragma unroll
    for (int c = 0; c < DV / 16; ++c) acc[a][c] = 0.f;
  }
  // the next tile's keys are on their way during the second product, its values during the next first one
  for (int t = first; t < last; ++t) {
    fill_wait<1>();
    __syncthreads();
    // scores of tokens tx, tx + 16, ... : a quarter warp's rows of sK then lie in all banks
    float2 s[RM][4];   // in two halves
#pragma unroll
    for (int a = 0; a < RM; ++a)
#pragma unroll
      for (int k = 0; k < 4; ++k) s[a][k] = make_float2(0.f, 0.f);
#pragma unroll 4
    for (int c = 0; c < DK; c += 4) {
      float4 q[RM], kk[4];
#pragma unroll
      for (int a = 0; a < RM; ++a) q[a] = *reinterpret_cast<const float4*>(sQ + (ty * RM + a) * C::kLdQ + c);
#pragma unroll
      for (int k = 0; k < 4; ++k) kk[k] = *reinterpret_cast<const float4*>(sK + (tx + 16 * k) * C::kLdK + c);
#pragma unroll
      for (int a = 0; a < RM; ++a)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          fma2(s[a][k].x, s[a][k].y, q[a].x, q[a].y, kk[k].x, kk[k].y);
          fma2(s[a][k].x, s[a][k].y, q[a].z, q[a].w, kk[k].z, kk[k].w);
        }
    }
    float w[RM][4];
    int token[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) token[k] = t * kKeys + tx + 16 * k < run.n ? run.at(t * kKeys + tx + 16 * k) : 0x7fffffff;
#pragma unroll
    for (int a = 0; a < RM; ++a) {
      bool seen[4];
      float top = -INFINITY;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        seen[k] = token[k] < end[a] && (token[k] >= low[a] || token[k] < p.mask.sinks);
        w[a][k] = (s[a][k].x + s[a][k].y) * p.c_log2;
        if (seen[k]) top = fmaxf(top, w[a][k]);
      }
#pragma unroll
      for (int d = 8; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
      const float m_new = fmaxf(m[a], top), base = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = exp2f(m[a] - base);   // 0 before the first token
      float sum = 0.f;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        w[a][k] = seen[k] ? exp2f(w[a][k] - base) : -1.f;
        if (seen[k]) sum += w[a][k];
      }
#pragma unroll
      for (int d = 8; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
      l[a] = l[a] * alpha + sum;
      m[a] = m_new;
#pragma unroll
      for (int c = 0; c < DV / 16; ++c) acc[a][c] *= alpha;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int a = 0; a < RM; ++a) sP[(tx + 16 * k) * C::kLdP + ty * RM + a] = w[a][k];
    __syncthreads();
    fill_keys(t + 1);
    fill_wait<1>();
    __syncthreads();
#pragma unroll 4
    for (int j = 0; j < kKeys; ++j) {
      float pw[RM];
#pragma unroll
      for (int a = 0; a < RM; ++a) pw[a] = sP[j * C::kLdP + ty * RM + a];
#pragma unroll
      for (int c = 0; c < DV / 64; ++c) {
        const float4 v = *reinterpret_cast<const float4*>(sV + j * DV + c * 64 + tx * 4);
#pragma unroll
        for (int a = 0; a < RM; ++a) {
          if (pw[a] >= 0.f || pw[a] != pw[a]) {
            fma2(acc[a][4 * c], acc[a][4 * c + 1], pw[a], pw[a], v.x, v.y);
            fma2(acc[a][4 * c + 2], acc[a][4 * c + 3], pw[a], pw[a], v.z, v.w);
          }
        }
      }
    }
    __syncthreads();
    fill_values(t + 1);
    find(t + 2);
  }
  fill_wait<0>();

  if (p.splits > 1 && p.part_o == nullptr) {
    // The shares are the CTAs of a cluster: each leaves its rows' sums in shared memory (where keys were) and joins every
    // splits-th row from all of them.
    float4* sum = reinterpret_cast<float4*>(sK);                                   // [rows][DV / 4]
    float4* stat = reinterpret_cast<float4*>(sK + C::kRows * DV);                  // [rows] m, l
    __syncthreads();
#pragma unroll
    for (int a = 0; a < RM; ++a) {
      const int r = ty * RM + a;
#pragma unroll
      for (int c = 0; c < DV / 64; ++c)
        sum[r * (DV / 4) + c * 16 + tx] = make_float4(acc[a][4 * c], acc[a][4 * c + 1], acc[a][4 * c + 2], acc[a][4 * c + 3]);
      if (tx == 0) stat[r] = make_float4(m[a], l[a], 0.f, 0.f);
    }
    cluster_sync();
    for (int x = threadIdx.x; x < (rows + p.splits - 1) / p.splits * (DV / 4); x += NT) {
      const int r = x / (DV / 4) * p.splits + int(blockIdx.y), c = x % (DV / 4);
      if (r >= rows) continue;
      float M = -INFINITY, L = 0.f;
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
      for (int k = 0; k < p.splits; ++k) M = fmaxf(M, load_of_cta(stat + r, k).x);
      const float base = M == -INFINITY ? 0.f : M;
#pragma unroll 4
      for (int k = 0; k < p.splits; ++k) {
        const float4 ml = load_of_cta(stat + r, k), v = load_of_cta(sum + r * (DV / 4) + c, k);
        const float f = exp2f(ml.x - base);
        L += f * ml.y;
        o.x += f * v.x, o.y += f * v.y, o.z += f * v.z, o.w += f * v.w;
      }
      const float inv = L == 0.f ? 0.f : 1.f / L;
      const int i = (r0 + r) / p.G, g = r0 + r - i * p.G;
      store4(static_cast<T*>(p.o.p) + b * p.o.sb + (int64_t(h) * p.G + g) * p.o.sh + i * p.o.sn + c * 4,
             make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
      if (p.lse != nullptr && c == 0)
        p.lse[((int64_t(b) * p.Hk + h) * p.G + g) * p.N + i] = L == 0.f ? -INFINITY : (M + log2f(L)) * kLn2;
    }
    cluster_sync();   // no CTA leaves while others read from it
    return;
  }
#pragma unroll
  for (int a = 0; a < RM; ++a) {
    const int r = ty * RM + a;
    if (r >= rows) continue;
    if (p.part_o != nullptr) {
      const int64_t at = (int64_t(item) * p.splits + blockIdx.y) * C::kRows + r;
#pragma unroll
      for (int c = 0; c < DV / 64; ++c)
        store4(p.part_o + at * DV + c * 64 + tx * 4,
               make_float4(acc[a][4 * c], acc[a][4 * c + 1], acc[a][4 * c + 2], acc[a][4 * c + 3]));
      if (tx == 0) p.part_ml[at] = make_float2(m[a], l[a]);
      continue;
    }
    const int i = (r0 + r) / p.G, g = r0 + r - i * p.G;
    const float inv = m[a] == -INFINITY && l[a] == 0.f ? 0.f : 1.f / l[a];
    T* o = static_cast<T*>(p.o.p) + b * p.o.sb + (int64_t(h) * p.G + g) * p.o.sh + i * p.o.sn;
#pragma unroll
    for (int c = 0; c < DV / 64; ++c)
      store4(o + c * 64 + tx * 4, make_float4(acc[a][4 * c] * inv, acc[a][4 * c + 1] * inv, acc[a][4 * c + 2] * inv,
                                              acc[a][4 * c + 3] * inv));
    if (p.lse != nullptr && tx == 0)
      p.lse[((int64_t(b) * p.Hk + h) * p.G + g) * p.N + i] = l[a] == 0.f ? -INFINITY : (m[a] + log2f(l[a])) * kLn2;
  }
}

// Joins the shares of a row: one warp a row, eight rows a CTA.
template <typename T, int DV>
__global__ void __launch_bounds__(256)
window_cc_join_kernel(Params p, int tile_rows) {
  wait_for_previous();
  const int lane = threadIdx.x & 31;
  const int64_t item = blockIdx.x, bh = unsigned(blockIdx.x) / unsigned(p.n_tiles);
  const int r = int(blockIdx.y) * 8 + (threadIdx.x >> 5);
  const int64_t row = (item - bh * p.n_tiles) * tile_rows + r;
  if (row >= int64_t(p.N) * p.G) return;
  auto place = [&](int k) { return (item * p.splits + k) * tile_rows + r; };
  float M = -INFINITY;
  for (int k = lane; k < p.splits; k += 32) M = fmaxf(M, p.part_ml[place(k)].x);
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, d));
  const float base = M == -INFINITY ? 0.f : M;
  float L = 0.f;
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int k = 0; k < p.splits; ++k) {
    const float2 ml = p.part_ml[place(k)];
    const float f = exp2f(ml.x - base);   // 0 of a share that saw nothing
    L += f * ml.y;
    if (lane * 4 < DV) {
      const float4 v = load4(p.part_o + place(k) * DV + lane * 4);
      x.x += f * v.x, x.y += f * v.y, x.z += f * v.z, x.w += f * v.w;
    }
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  const int64_t b = unsigned(bh) / unsigned(p.Hk), h = bh - b * p.Hk, i = unsigned(row) / unsigned(p.G), g = row - i * p.G;
  if (lane * 4 < DV)
    store4(static_cast<T*>(p.o.p) + b * p.o.sb + (h * p.G + g) * p.o.sh + i * p.o.sn + lane * 4,
           make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv));
  if (p.lse != nullptr && lane == 0)
    p.lse[((b * p.Hk + h) * p.G + g) * p.N + i] = L == 0.f ? -INFINITY : (M + log2f(L)) * kLn2;
}

template <typename T, int DK, int DV, int RM, int NT>
int launch(const WindowArgs& a, const WindowCcPlan& plan, char* msg, size_t msglen) {
  using C = Cfg<DK, DV, RM, NT>;
  auto kern = window_cc_kernel<T, DK, DV, RM, NT>;
  cudaError_t e = ensure_smem_limit(reinterpret_cast<const void*>(kern), C::kSmem);
  Params p{};
  p.q = a.q, p.o = a.o, p.kv = a.kv, p.lse = a.lse, p.lens = a.lens;
  p.Hk = int(a.Hk), p.N = int(a.N), p.G = int(a.Hq / a.Hk), p.max_len = int(a.max_len);
  p.n_tiles = int(plan.items / (a.B * a.Hk));
  p.mask = win::Mask{a.window, a.sinks, a.causal};
  p.c_log2 = a.scale * kLog2e;
  p.splits = int(plan.splits);
  if (plan.splits > 1 && !plan.cluster) {
    p.part_o = static_cast<float*>(a.ws);
    p.part_ml = reinterpret_cast<float2*>(p.part_o + plan.items * plan.splits * C::kRows * DV);
  }
  static_assert(C::kRows * DV + 4 * C::kRows <= kKeys * C::kLdK + kKeys * DV, "the sums lie where keys and values were");
  const dim3 grid(unsigned(plan.items), unsigned(plan.splits));
  if (e == cudaSuccess && plan.cluster && plan.splits > 8)
    e = cudaFuncSetAttribute(reinterpret_cast<const void*>(kern), cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e == cudaSuccess)
    e = plan.cluster ? launch_clusters(kern, grid, unsigned(plan.splits), dim3(NT), C::kSmem, a.stream, p)
                     : launch_overlapped(kern, grid, dim3(NT), C::kSmem, a.stream, p);
  if (e == cudaSuccess && plan.splits > 1 && !plan.cluster)
    e = launch_overlapped(window_cc_join_kernel<T, DV>, dim3(unsigned(plan.items), C::kRows / 8), dim3(256), 0, a.stream, p,
                          int(C::kRows));
  if (e != cudaSuccess) {
    snprintf(msg, msglen, "attention with a window: %s", cudaGetErrorString(e));
    return 5;
  }
  return 0;
}

template <typename T, int DK, int DV>
int launch_rows(const WindowArgs& a, const WindowCcPlan& plan, char* msg, size_t msglen) {
  return plan.rows == 16 ? launch<T, DK, DV, 2, 128>(a, plan, msg, msglen) : launch<T, DK, DV, 4, 256>(a, plan, msg, msglen);
}
template <typename T>
int launch_sizes(const WindowArgs& a, const WindowCcPlan& plan, char* msg, size_t msglen) {
  if (a.dk == 64)
    return a.dv == 64 ? launch_rows<T, 64, 64>(a, plan, msg, msglen) : launch_rows<T, 64, 128>(a, plan, msg, msglen);
  return a.dv == 64 ? launch_rows<T, 128, 64>(a, plan, msg, msglen) : launch_rows<T, 128, 128>(a, plan, msg, msglen);
}

// The most CTAs of a cluster that has room on the device: 1, where no cluster has.
template <typename T, int DK, int DV, int RM, int NT>
int most_cluster() {
  static ClusterRoom room;
  int size = kMostCluster;
  while (size > 1 && room(reinterpret_cast<const void*>(window_cc_kernel<T, DK, DV, RM, NT>), NT, Cfg<DK, DV, RM, NT>::kSmem, size) < 1)
    size /= 2;
  return size;
}
template <typename T, int DK, int DV>
int most_cluster(int64_t rows) {
  return rows == 16 ? most_cluster<T, DK, DV, 2, 128>() : most_cluster<T, DK, DV, 4, 256>();
}
template <typename T>
int most_cluster(const WindowArgs& a, int64_t rows) {
  if (a.dk == 64) return a.dv == 64 ? most_cluster<T, 64, 64>(rows) : most_cluster<T, 64, 128>(rows);
  return a.dv == 64 ? most_cluster<T, 128, 64>(rows) : most_cluster<T, 128, 128>(rows);
}

}  // namespace

// Tiles of 16 rows where 64 would be mostly empty, or too few for the machine; shares of a tile's
// tokens until there are two CTAs for each SM, none of less than one tile of tokens.
WindowCcPlan window_cc_plan(const WindowArgs& a, int sms) {
  const int64_t G = a.Hq / a.Hk, rows = a.N * G, bh = a.B * a.Hk;
  WindowCcPlan p;
  const int64_t big = bh * ((rows + 63) / 64);
  p.rows = rows <= 32 || big < sms ? 16 : 64;
  const int64_t tiles = (rows + p.rows - 1) / p.rows;
  p.items = bh * tiles;
  // most tiles of tokens that a row tile visits
  int64_t most = (a.max_len + kKeys - 1) / kKeys;
  if (a.window != win::kNoWindow) {
    const int64_t seen = (int64_t(a.window) + p.rows / G + 2 + a.sinks + kKeys - 1) / kKeys;
    if (seen < most) most = seen;
  }
  p.splits = p.items >= 2 * sms ? 1 : (2 * sms + p.items - 1) / p.items;
  if (p.splits > most) p.splits = most;
  if (p.splits < 1) p.splits = 1;
  // joined by clusters where a cluster's CTAs have no more than three tiles each
  p.cluster = false;
  if (p.splits > 1) {
    const int64_t size = a.f32 ? most_cluster<float>(a, p.rows) : most_cluster<__nv_bfloat16>(a, p.rows);
    p.cluster = size > 1 && (p.splits <= size || most <= 3 * size);
    if (p.cluster && p.splits > size) p.splits = size;
  }
  return p;
}

size_t window_cc_workspace(const WindowArgs& a, const WindowCcPlan& p) {
  return p.splits > 1 && !p.cluster ? size_t(p.items * p.splits * p.rows) * size_t(a.dv * 4 + 8) : 0;
}

int launch_window_cc(const WindowArgs& a, const WindowCcPlan& plan, char* msg, size_t msglen) {
  return a.f32 ? launch_sizes<float>(a, plan, msg, msglen) : launch_sizes<__nv_bfloat16>(a, plan, msg, msglen);
}

cudaError_t window_cc_read_and_clear_status(unsigned* value) {
  cudaError_t e = cudaMemcpyFromSymbol(value, g_moa_window_cc_status, sizeof(unsigned));
  if (e != cudaSuccess || *value == 0) return e;
  const unsigned zero = 0;
  return cudaMemcpyToSymbol(g_moa_window_cc_status, &zero, sizeof(unsigned));
}

}  // namespace moa
