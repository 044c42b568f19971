// Writing keys and values into the 4-bit cache, and reading them back, sm_103a.
//
// Mathematics and layout: kv4.cuh.  Write: per row and 32 features, s = bf16(max|x| / 7),
// code = rint(x / s) (ties to even, IEEE division: the same codes as the definition in exact
// arithmetic for bf16 inputs).  Read: code * s in fp32, rounded once to the output's type.
//
// What bounds it: memory.  A bf16 value is 2 bytes on one side and 9/16 on the other.
//
// Layout of the work: 8 or 16 lanes own one row (head, token), eight features a lane, so that the
// four lanes of a scale group are neighbours.
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

// Codes + 8 of this lane's eight features, and the group's scale (bits of a bf16).
__device__ __forceinline__ uint32_t quantise8(const float* x, uint32_t* code) {
  // the maximum of the magnitudes' bits: a NaN's are above every number's
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t a = __float_as_uint(x[i]) & 0x7fffffffu;
    m = a > m ? a : m;
  }
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) {
    const uint32_t a = __shfl_xor_sync(0xffffffffu, m, o);
    m = a > m ? a : m;
  }
  uint32_t bits = 0x7fc0u;
  float s = 0.f;
  if (m < 0x7f800000u) {
    const __nv_bfloat16 h = __float2bfloat16_rn(__fdiv_rn(__uint_as_float(m), 7.f));
    bits = __bfloat16_as_ushort(h);
    s = __bfloat162float(h);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float c = 0.f;
    if (s > 0.f) c = fminf(fmaxf(rintf(__fdiv_rn(x[i], s)), -7.f), 7.f);
    code[i] = uint32_t(int(c) + 8);
  }
  return bits;
}

struct Dims {
  int64_t B, N;
  int64_t n_pages, max_pages;
  int64_t rows;     // B * H * N
  int H, page, dk, dv;
};

// The 16-token block that holds position `at` of sequence b for head h, or null: at < 0 (padding)
// or, with the status word set, a position or page outside its table.
__device__ __forceinline__ uint8_t* find_block(uint8_t* pool, const int32_t* table, const Dims& p,
                                               int64_t b, int h, int32_t at, bool report) {
  if (at < 0) return nullptr;
  const int64_t slot = at / p.page;
  int32_t page = -1;
  if (slot < p.max_pages) page = table[b * p.max_pages + slot];
  if (page < 0 || page >= p.n_pages) {
    if (report) atomicExch(&g_moa_kv4_status, kErrIndex);
    return nullptr;
  }
  const int64_t blocks = p.page / kBlock;
  const int64_t i = (int64_t(page) * p.H + h) * blocks + (at - int32_t(slot) * p.page) / kBlock;
  return pool + i * block_bytes(p.dk, p.dv);
}

template <typename T, int LPR>
__global__ void __launch_bounds__(kThreads)
kv4_write_kernel(View k, View v, uint8_t* pool, const int32_t* table, const int32_t* pos, Dims p) {
  wait_for_previous();
  const int lane = threadIdx.x % LPR;
  const int64_t row = int64_t(blockIdx.x) * (kThreads / LPR) + threadIdx.x / LPR;
  const bool live = row < p.rows;
  const int64_t n = live ? row % p.N : 0, bh = live ? row / p.N : 0;
  const int h = int(bh % p.H);
  const int64_t b = bh / p.H;
  const int32_t at = live ? pos[b * p.N + n] : -1;
  uint8_t* block = find_block(pool, table, p, b, h, at, lane == 0);
  const int tok = at & (kBlock - 1);
  const int f0 = lane * 8, g = lane >> 2, t = lane & 3;
  float x[8];
  uint32_t c[8];
  {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = 0.f;
    const bool mine = block != nullptr && f0 < p.dk;
    if (mine) load8(static_cast<const T*>(k.p) + b * k.sb + h * k.sh + n * k.sn + f0, x);
    const uint32_t s = quantise8(x, c);
    if (mine) {
      const int groups = p.dk / kGroup;
      *reinterpret_cast<uint32_t*>(block + key_word(tok, t, g, groups)) =
          c[0] | c[2] << 4 | c[4] << 8 | c[6] << 12 | c[1] << 16 | c[3] << 20 | c[5] << 24 | c[7] << 28;
      if (t == 0)
        *reinterpret_cast<uint16_t*>(block + key_scales(p.dk, p.dv) + (tok * groups + g) * 2) = uint16_t(s);
    }
  }
  {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = 0.f;
    const bool mine = block != nullptr && f0 < p.dv;
    if (mine) load8(static_cast<const T*>(v.p) + b * v.sb + h * v.sh + n * v.sn + f0, x);
    const uint32_t s = quantise8(x, c);
    if (mine) {
      const int groups = p.dv / kGroup;
      uint8_t* w = block + value_word(p.dk, tok, 2 * t, g, groups) + (tok & 1) * 2;
      *reinterpret_cast<uint16_t*>(w) = uint16_t(c[0] | c[1] << 4 | c[2] << 8 | c[3] << 12);
      w = block + value_word(p.dk, tok, 2 * t + 1, g, groups) + (tok & 1) * 2;
      *reinterpret_cast<uint16_t*>(w) = uint16_t(c[4] | c[5] << 4 | c[6] << 8 | c[7] << 12);
      if (t == 0)
        *reinterpret_cast<uint16_t*>(block + value_scales(p.dk, p.dv) + (tok * groups + g) * 2) = uint16_t(s);
    }
  }
}

template <typename T, int LPR>
__global__ void __launch_bounds__(kThreads)
kv4_read_kernel(View k, View v, uint8_t* pool, const int32_t* table, const int32_t* pos, Dims p) {
  wait_for_previous();
  const int lane = threadIdx.x % LPR;
  const int64_t row = int64_t(blockIdx.x) * (kThreads / LPR) + threadIdx.x / LPR;
  if (row >= p.rows) return;
  const int64_t n = row % p.N, bh = row / p.N;
  const int h = int(bh % p.H);
  const int64_t b = bh / p.H;
  const int32_t at = pos[b * p.N + n];
  const uint8_t* block = find_block(pool, table, p, b, h, at, lane == 0);
  const int tok = at & (kBlock - 1);
  const int f0 = lane * 8, g = lane >> 2, t = lane & 3;
  const float fill = at < 0 ? 0.f : __int_as_float(0x7fc00000);  // padding, or no such place
  float x[8];
  if (f0 < p.dk) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = fill;
    if (block != nullptr) {
      const int groups = p.dk / kGroup;
      const uint32_t w = *reinterpret_cast<const uint32_t*>(block + key_word(tok, t, g, groups));
      const uint32_t s = *reinterpret_cast<const uint16_t*>(block + key_scales(p.dk, p.dv) + (tok * groups + g) * 2);
      const float scale = __uint_as_float(s << 16);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        x[e] = float(int((w >> (16 * (e & 1) + 4 * (e >> 1))) & 15u) - 8) * scale;
    }
    store8(static_cast<T*>(k.p) + b * k.sb + h * k.sh + n * k.sn + f0, x);
  }
  if (f0 < p.dv) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = fill;
    if (block != nullptr) {
      const int groups = p.dv / kGroup;
      const uint32_t s = *reinterpret_cast<const uint16_t*>(block + value_scales(p.dk, p.dv) + (tok * groups + g) * 2);
      const float scale = __uint_as_float(s << 16);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const uint32_t w = *reinterpret_cast<const uint16_t*>(
            block + value_word(p.dk, tok, 2 * t + c, g, groups) + (tok & 1) * 2);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[4 * c + j] = float(int((w >> (4 * j)) & 15u) - 8) * scale;
      }
    }
    store8(static_cast<T*>(v.p) + b * v.sb + h * v.sh + n * v.sn + f0, x);
  }
}

template <typename T, int LPR>
cudaError_t run(const Kv4MoveArgs& a, const Dims& p, bool write, int64_t grid) {
  uint8_t* pool = static_cast<uint8_t*>(a.c.pool);
  return launch_overlapped(write ? kv4_write_kernel<T, LPR> : kv4_read_kernel<T, LPR>, dim3(unsigned(grid)),
                           dim3(kThreads), 0, a.stream, a.k, a.v, pool, a.c.table, a.pos, p);
}

int launch(const Kv4MoveArgs& a, bool write, char* msg, size_t msglen) {
  Dims p{a.B, a.N, a.c.n_pages, a.c.max_pages, a.B * a.c.H * a.N, a.c.H, a.c.page, a.c.dk, a.c.dv};
  const int lpr = a.c.dk <= 64 && a.c.dv <= 64 ? 8 : 16;
  const int64_t grid = (p.rows + kThreads / lpr - 1) / (kThreads / lpr);
  if (grid > 0x7fffffffLL) {
    snprintf(msg, msglen, "cache: too many rows for one launch");
    return 3;
  }
  cudaError_t e;
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
