// New keys and values into a paged 16- or 32-bit cache, keys (and the queries beside them) rotated on the
// way (sm_103a).
//
// The pool is [n_pages, H, page, d_k + d_v]: a token's key and value of one head lie next to each other, so
// that a decoding step writes whole rows, and a page of a head is one run of memory for the attention.
//
// Mathematics: each pair (a, b) of a row's first d_rot features becomes (a cos - b sin, b cos + a sin) of
// its position's angles, in fp32, rounded once to the row's type; the others, and values, are copied.
//
// What bounds it: memory.  A thread keeps the 8 angles of its 16 features (8 pairs) of one token and walks
// over heads, several rows on their way at a time; a token's angles are then read once for a group of heads.
// Few tokens: each head is a group of its own, which leaves the latency of position, then angles and page.  3 x (16 + 8 + 8) x 16001 x 128:
// 125 us, 6.4 TB/s; 64 x (32 + 8 + 8) x 1 x 128: 2.5 us in a replayed graph.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdio>

#include "internal.h"
#include "ops_internal.h"
#include "window.cuh"

namespace moa {

__device__ unsigned int g_moa_kv_append_status = 0;

namespace {

constexpr int kThreads = 256;
constexpr int kBatch = 4;   // rows of a thread on their way at a time

struct Params {
  View q, oq, k, v;
  void* pool;
  const int32_t* table;
  const int32_t* pos;
  const float* cosines;
  const float* sines;
  int64_t tokens, N, n_pages, max_pages, n_pos;
  int Hq, Hk, page, dk, dv, half;   // half: d_rot / 2, 0 for no rotation
  int chunks;                       // of 16 features, of the longer of key and value rows
  int slots;                        // query heads, key heads, value heads
  int group;                        // slots of a CTA
};

// 16 features: 8 at p and 8 at p + gap.
struct Feat {
  float a[8], b[8];
};
template <typename T>
struct Raw;
template <>
struct Raw<__nv_bfloat16> {
  uint4 x, y;
  __device__ __forceinline__ void load(const __nv_bfloat16* p, int gap) {
    x = *reinterpret_cast<const uint4*>(p);
    y = *reinterpret_cast<const uint4*>(p + gap);
  }
  __device__ __forceinline__ void store(__nv_bfloat16* p, int gap) const {
    *reinterpret_cast<uint4*>(p) = x;
    *reinterpret_cast<uint4*>(p + gap) = y;
  }
  static __device__ __forceinline__ void wide(const uint4& u, float* f) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 narrow(const float* f) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 t = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&t);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ __forceinline__ Feat get() const {
    Feat f;
    wide(x, f.a);
    wide(y, f.b);
    return f;
  }
  __device__ __forceinline__ void set(const Feat& f) {
    x = narrow(f.a);
    y = narrow(f.b);
  }
};
template <>
struct Raw<float> {
  float4 x[2], y[2];
  __device__ __forceinline__ void load(const float* p, int gap) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      x[i] = reinterpret_cast<const float4*>(p)[i];
      y[i] = reinterpret_cast<const float4*>(p + gap)[i];
    }
  }
  __device__ __forceinline__ void store(float* p, int gap) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      reinterpret_cast<float4*>(p)[i] = x[i];
      reinterpret_cast<float4*>(p + gap)[i] = y[i];
    }
  }
  __device__ __forceinline__ Feat get() const {
    Feat f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      f.a[4 * i] = x[i].x, f.a[4 * i + 1] = x[i].y, f.a[4 * i + 2] = x[i].z, f.a[4 * i + 3] = x[i].w;
      f.b[4 * i] = y[i].x, f.b[4 * i + 1] = y[i].y, f.b[4 * i + 2] = y[i].z, f.b[4 * i + 3] = y[i].w;
    }
    return f;
  }
  __device__ __forceinline__ void set(const Feat& f) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      x[i] = make_float4(f.a[4 * i], f.a[4 * i + 1], f.a[4 * i + 2], f.a[4 * i + 3]);
      y[i] = make_float4(f.b[4 * i], f.b[4 * i + 1], f.b[4 * i + 2], f.b[4 * i + 3]);
    }
  }
};

template <typename T, bool PAIRS>
__global__ void __launch_bounds__(kThreads)
kv_append_kernel(Params p) {
  wait_for_previous();
  const int per = kThreads / p.chunks;   // tokens of a CTA
  const int64_t token = int64_t(blockIdx.x) * per + threadIdx.x / p.chunks;
  const int chunk = threadIdx.x % p.chunks;
  if (token >= p.tokens) return;
  const int64_t b = token / p.N, n = token - b * p.N;
  const int pos = p.pos[token];
  const int s0 = int(blockIdx.y) * p.group, s1 = min(s0 + p.group, p.slots);
  // where the token's rows go
  T* row = nullptr;
  bool known = true;   // its angles are in the tables
  if (pos >= 0) {
    const int slot = pos / p.page;
    known = p.half == 0 || pos < p.n_pos;
    int pg = -1;
    if (slot < p.max_pages) pg = p.table[b * p.max_pages + slot];
    if (known && pg >= 0 && pg < p.n_pages)
      row = static_cast<T*>(p.pool) + (int64_t(pg) * p.Hk * p.page + (pos - slot * p.page)) * (p.dk + p.dv);
    else if (chunk == 0)
      atomicExch(&g_moa_kv_append_status, win::kErrIndex);
  }
  const int64_t head_step = int64_t(p.page) * (p.dk + p.dv);
  // the thread's 16 features of a query or key row: 8 pairs, or 16 that pass
  const int rot_chunks = p.half / 8;
  const bool turns = chunk < rot_chunks;
  const int at = PAIRS || !turns ? 16 * chunk : 8 * chunk, gap = PAIRS || !turns ? 8 : p.half;
  float c[8], s[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = 1.f, s[i] = 0.f;
  if (turns && pos >= 0) {
    if (known) {
      const float* pc = p.cosines + int64_t(pos) * p.half + 8 * chunk;
      const float* ps = p.sines + int64_t(pos) * p.half + 8 * chunk;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float4 x = reinterpret_cast<const float4*>(pc)[i], y = reinterpret_cast<const float4*>(ps)[i];
        c[4 * i] = x.x, c[4 * i + 1] = x.y, c[4 * i + 2] = x.z, c[4 * i + 3] = x.w;
        s[4 * i] = y.x, s[4 * i + 1] = y.y, s[4 * i + 2] = y.z, s[4 * i + 3] = y.w;
      }
    }
  }
  for (int first = s0; first < s1; first += kBatch) {
    Raw<T> x[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int slot = first + u;
      if (slot >= s1) continue;
      const int kind = slot < p.Hq ? 0 : slot < p.Hq + p.Hk ? 1 : 2;
      const int h = kind == 0 ? slot : kind == 1 ? slot - p.Hq : slot - p.Hq - p.Hk;
      const View& src = kind == 0 ? p.q : kind == 1 ? p.k : p.v;
      if (16 * chunk < (kind == 2 ? p.dv : p.dk))
        x[u].load(static_cast<const T*>(src.p) + b * src.sb + h * src.sh + n * src.sn + (kind == 2 ? 16 * chunk : at),
                  kind == 2 ? 8 : gap);
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int slot = first + u;
      if (slot >= s1) continue;
      const int kind = slot < p.Hq ? 0 : slot < p.Hq + p.Hk ? 1 : 2;
      const int h = kind == 0 ? slot : kind == 1 ? slot - p.Hq : slot - p.Hq - p.Hk;
      if (16 * chunk >= (kind == 2 ? p.dv : p.dk) || (kind != 0 && row == nullptr)) continue;
      if (kind == 2) {
        x[u].store(row + h * head_step + p.dk + 16 * chunk, 8);
        continue;
      }
      if (turns || (kind == 0 && (pos < 0 || !known))) {
        Feat f = x[u].get(), y;
        if (PAIRS) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            y.a[2 * i] = f.a[2 * i] * c[i] - f.a[2 * i + 1] * s[i];
            y.a[2 * i + 1] = f.a[2 * i + 1] * c[i] + f.a[2 * i] * s[i];
            y.b[2 * i] = f.b[2 * i] * c[4 + i] - f.b[2 * i + 1] * s[4 + i];
            y.b[2 * i + 1] = f.b[2 * i + 1] * c[4 + i] + f.b[2 * i] * s[4 + i];
          }
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            y.a[i] = f.a[i] * c[i] - f.b[i] * s[i];
            y.b[i] = f.b[i] * c[i] + f.a[i] * s[i];
          }
        }
        if (kind == 0 && (pos < 0 || !known)) {   // padding, or a position without angles
#pragma unroll
          for (int i = 0; i < 8; ++i) y.a[i] = y.b[i] = pos < 0 ? 0.f : __int_as_float(0x7fc00000);
        }
        x[u].set(y);
      }
      T* dst = kind == 0 ? static_cast<T*>(p.oq.p) + b * p.oq.sb + h * p.oq.sh + n * p.oq.sn : row + h * head_step;
      x[u].store(dst + at, gap);
    }
  }
}

template <typename T>
int launch(const KvAppendArgs& a, int sms, char* msg, size_t msglen) {
  Params p{};
  p.q = a.q, p.oq = a.oq, p.k = a.k, p.v = a.v;
  p.pool = a.pool, p.table = a.table, p.pos = a.pos, p.cosines = a.cosines, p.sines = a.sines;
  p.tokens = a.B * a.N, p.N = a.N, p.n_pages = a.n_pages, p.max_pages = a.max_pages, p.n_pos = a.n_pos;
  p.Hq = a.q.p == nullptr ? 0 : int(a.Hq), p.Hk = int(a.Hk);
  p.page = a.page, p.dk = a.dk, p.dv = a.dv, p.half = a.d_rot / 2;
  p.chunks = (a.dk > a.dv ? a.dk : a.dv) / 16;
  p.slots = p.Hq + 2 * p.Hk;
  const int64_t per = kThreads / p.chunks, ctas = (p.tokens + per - 1) / per;
  // groups of heads: as many as give every SM eight CTAs, of a batch's rows at least where there are more tokens
  int64_t groups = (8 * sms + ctas - 1) / ctas;
  groups = groups > p.slots ? p.slots : groups;
  p.group = int((p.slots + groups - 1) / groups);
  if (p.group > 1) p.group = (p.group + kBatch - 1) / kBatch * kBatch;
  const dim3 grid(unsigned(ctas), unsigned((p.slots + p.group - 1) / p.group));
  const cudaError_t e = a.pairs ? launch_overlapped(kv_append_kernel<T, true>, grid, dim3(kThreads), 0, a.stream, p)
                                : launch_overlapped(kv_append_kernel<T, false>, grid, dim3(kThreads), 0, a.stream, p);
  if (e != cudaSuccess) {
    snprintf(msg, msglen, "cache append: %s", cudaGetErrorString(e));
    return 5;
  }
  return 0;
}

}  // namespace

int launch_kv_append(const KvAppendArgs& a, char* msg, size_t msglen) {
  int sms = 0;
  const cudaError_t e = device_sm_count(&sms);
  if (e != cudaSuccess) {
    snprintf(msg, msglen, "cache append: SM count: %s", cudaGetErrorString(e));
    return 5;
  }
  return a.f32 ? launch<float>(a, sms, msg, msglen) : launch<__nv_bfloat16>(a, sms, msg, msglen);
}

cudaError_t kv_append_read_and_clear_status(unsigned* value) {
  cudaError_t e = cudaMemcpyFromSymbol(value, g_moa_kv_append_status, sizeof(unsigned));
  if (e != cudaSuccess || *value == 0) return e;
  const unsigned zero = 0;
  return cudaMemcpyToSymbol(g_moa_kv_append_status, &zero, sizeof(unsigned));
}

}  // namespace moa
