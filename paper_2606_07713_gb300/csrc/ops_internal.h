// Declarations shared by the translation units of the operators around attention: per-head norms
// with rotation, the 4-bit cache and attention over it.
#pragma once
#include <cstddef>
#include <cstdint>
#include <cuda_runtime.h>
#include <utility>

namespace moa {

// Launches a kernel that may be set up while the kernel before it on the stream still runs.  Every
// thread of such a kernel calls wait_for_previous() before its first access to global memory.
template <typename... P, typename... A>
cudaError_t launch_overlapped(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t stream, A&&... args) {
  cudaLaunchAttribute attr{};
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t c{};
  c.gridDim = grid;
  c.blockDim = block;
  c.dynamicSmemBytes = smem;
  c.stream = stream;
  c.attrs = &attr;
  c.numAttrs = 1;
  return cudaLaunchKernelEx(&c, kernel, P(std::forward<A>(args))...);
}
#ifdef __CUDACC__
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
#endif

// Defined beside the attention entry points: the per-thread error text, and MOA_DEBUG_SYNC.
int api_fail(int code, const char* fmt, ...);
void api_clear();
int api_debug_check(void* stream);

// A [B, H, N, d] tensor with unit stride along d; strides in elements.
struct View {
  void* p;
  int64_t sb, sh, sn;
};

struct NormRopeArgs {
  View q, k;             // inputs
  View gq, gk;           // backward: gradients of the outputs
  View oq, ok;           // outputs (backward: dQ, dK)
  const void* wq;        // [d], the element type of q
  const void* wk;
  const float* cosines;  // [n_pos, d_rot / 2]
  const float* sines;
  const int32_t* pos;    // [B, N]
  float* dwq;            // backward only, [d]
  float* dwk;
  float* partial;        // backward only, norm_rope_partial_rows() x d
  int64_t B, Hq, Hk, N, n_pos;
  int d, d_rot;
  float eps;
  bool pairs;            // (2i, 2i+1) instead of (i, i + d_rot/2)
  bool f32;
  cudaStream_t stream;
};
int launch_norm_rope(const NormRopeArgs& a, char* msg, size_t msglen);
int launch_norm_rope_bwd(const NormRopeArgs& a, char* msg, size_t msglen);
// Rows of d floats the backward writes before its last sum.
int64_t norm_rope_partial_rows(int64_t B, int64_t Hq, int64_t Hk, int64_t N, int64_t d, int sms);

// The 4-bit cache (layout: kv4.cuh): a pool [n_pages, H, page / 16 blocks of 9 (dk + dv) bytes]
// and a table [B, max_pages] of page numbers.
struct Kv4Cache {
  void* pool;
  const int32_t* table;
  int64_t n_pages, max_pages;
  int page, H, dk, dv;
};
struct Kv4MoveArgs {
  Kv4Cache c;
  View k, v;             // rows written to the cache, or read from it
  const int32_t* pos;    // [B, N]
  int64_t B, N;
  bool f32;
  cudaStream_t stream;
};
int launch_kv4_write(const Kv4MoveArgs& a, char* msg, size_t msglen);
int launch_kv4_read(const Kv4MoveArgs& a, char* msg, size_t msglen);

struct Kv4AttnArgs {
  Kv4Cache c;
  View q, o;
  float* lse;            // [B, Hq, N] or null
  const int32_t* lens;   // [B]
  int64_t B, Hq, N, max_len;
  float scale;
  bool causal, f32;
  void* ws;
  cudaStream_t stream;
};
// How the work is divided: tiles of the G * N query rows of one key head, and the CTAs that share
// the tokens of all tiles.
struct Kv4Plan {
  bool tc = false;          // many rows: kv4_attn_tc.cu (the rest of the plan is then unused)
  int rows_tile = 8;        // query rows of one tile
  int64_t n_tiles = 1;
  int64_t ctas = 1;
};
Kv4Plan kv4_attn_plan(int64_t B, int64_t Hk, int64_t G, int64_t N, int64_t max_len, bool f32, int sms);
size_t kv4_attn_workspace(int64_t B, int64_t Hk, int64_t max_len, int64_t dk, int64_t dv, const Kv4Plan& p, int sms);
size_t kv4_attn_tc_workspace(int64_t bh, int64_t max_len, int64_t dk, int64_t dv, int sms);
int launch_kv4_attn_tc(const Kv4AttnArgs& a, char* msg, size_t msglen);
int launch_kv4_attn(const Kv4AttnArgs& a, const Kv4Plan& p, char* msg, size_t msglen);

// Status words of the four translation units (0, MOA_ERR_DEVICE_TIMEOUT or
// MOA_ERR_DEVICE_INDEX); read and cleared after a synchronisation.
cudaError_t norm_read_and_clear_status(unsigned* value);
cudaError_t kv4_read_and_clear_status(unsigned* value);
cudaError_t kv4_attn_read_and_clear_status(unsigned* value);
cudaError_t kv4_tc_read_and_clear_status(unsigned* value);

}  // namespace moa
