// Declarations shared by the translation units of the operators around attention: per-head norms
// with rotation, the 4-bit cache and attention over it.
#pragma once
#include <atomic>
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
// The same with clusters of `cluster` CTAs along the grid's y axis.
template <typename... P, typename... A>
cudaError_t launch_clusters(void (*kernel)(P...), dim3 grid, unsigned cluster, dim3 block, size_t smem, cudaStream_t stream,
                            A&&... args) {
  cudaLaunchAttribute attr[2]{};
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 1;
  attr[1].val.clusterDim.y = cluster;
  attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t c{};
  c.gridDim = grid;
  c.blockDim = block;
  c.dynamicSmemBytes = smem;
  c.stream = stream;
  c.attrs = attr;
  c.numAttrs = 2;
  return cudaLaunchKernelEx(&c, kernel, P(std::forward<A>(args))...);
}
// Clusters of `size` CTAs (1, 2, 4, 8, 16) of a kernel that the current device, or what the context has of it, takes at the same
// time: 0 if a launch of one would fail.  Asked once for each device and size.
class ClusterRoom {
 public:
  int operator()(const void* kernel, int threads, int bytes, int size);

 private:
  std::atomic<int> known_[64][5]{};   // [device][log2 size]: what was asked, and 1
};
void limit_clusters(int most);   // as if no cluster of more than `most` CTAs fitted (0: as it is)

#ifdef __CUDACC__
// The cluster's barrier in two halves: a CTA's shared memory may be written from others once all have arrived.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
// All threads of all CTAs of the cluster; what they wrote before is seen after.
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The address in CTA `rank`'s shared memory of what lies at `at` in this CTA's, and stores there.
__device__ __forceinline__ uint32_t smem_of_cta(uint32_t at, unsigned rank) {
  uint32_t there;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(rank));
  return there;
}
__device__ __forceinline__ void store4_to_cta(uint32_t there, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(there), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void store2_to_cta(uint32_t there, float a, float b) {
  asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(there), "f"(a), "f"(b) : "memory");
}
// Four floats of CTA `rank`'s shared memory, at the place that `p` has in this CTA's.
__device__ __forceinline__ float4 load_of_cta(const float4* p, unsigned rank) {
  const uint32_t at = smem_of_cta(uint32_t(__cvta_generic_to_shared(p)), rank);
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
  return v;
}
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

// Where keys and values of attention with a window lie: token t of sequence b and key head h at
// k + b * k_sb + h * k_sh + t * k_sn (and v alike), or, with a page table, page table[b, t / page] in
// the place of b and t % page in that of t.  Strides in elements.
struct KvSource {
  const void* k;
  const void* v;
  int64_t k_sb, k_sh, k_sn, v_sb, v_sh, v_sn;
  const int32_t* table;   // null: no pages
  int64_t n_pages, max_pages;
  int page;
};
// Attention of the last N of each sequence's tokens with a window and sinks (window.cuh).
struct WindowArgs {
  View q, o;
  KvSource kv;
  float* lse;            // [B, Hq, N] or null
  const int32_t* lens;   // [B], or null: every sequence has max_len tokens
  int64_t B, Hq, Hk, N, max_len;
  int dk, dv;
  int window, sinks;     // window: win::kNoWindow for none
  float scale;
  bool causal, f32;
  void* ws;
  cudaStream_t stream;
};
// CUDA cores: fp32, and bf16 tensors that no tensor map describes (window_fwd_cc.cu).
struct WindowCcPlan {
  int rows;              // query rows of a tile
  int64_t items;         // tiles of all key heads
  int64_t splits;        // shares of a tile's tokens, joined at the end
  bool cluster;          // by the CTAs of a cluster, in the same launch
};
WindowCcPlan window_cc_plan(const WindowArgs& a, int sms);   // (on the current device)
size_t window_cc_workspace(const WindowArgs& a, const WindowCcPlan& p);
int launch_window_cc(const WindowArgs& a, const WindowCcPlan& p, char* msg, size_t msglen);

// Tensor cores: bf16 (window_fwd_tc.cu).  Whether it takes a call: tensor maps describe its tensors (no strides that
// are zero or negative), and the scale is not negative.
bool window_tc_takes(const WindowArgs& a);
size_t window_tc_workspace(const WindowArgs& a, int sms);
int launch_window_tc(const WindowArgs& a, int sms, char* msg, size_t msglen);

// Gradients of attention with a window (dense keys and values).
struct WindowBwdArgs {
  View q, k, v, o, go;   // inputs
  const float* lse;      // [B, Hq, Nq]
  View dq, dk_, dv_;     // outputs
  int64_t B, Hq, Hk, Nq, Nk;
  int dk, dv;
  int window, sinks;
  float scale;
  bool f32;
  void* ws;
  cudaStream_t stream;
};
size_t window_bwd_cc_workspace(const WindowBwdArgs& a);
int launch_window_bwd_cc(const WindowBwdArgs& a, char* msg, size_t msglen);
// Tensor cores: bf16 tensors that tensor maps describe (window_bwd_tc.cu).
bool window_bwd_tc_takes(const WindowBwdArgs& a);
size_t window_bwd_tc_workspace(const WindowBwdArgs& a);
int launch_window_bwd_tc(const WindowBwdArgs& a, char* msg, size_t msglen);

// New keys and values into a 16- or 32-bit paged cache [n_pages, H, page, dk + dv], keys (and
// queries, into oq) rotated on the way.
struct KvAppendArgs {
  View q, oq;            // q.p null: no queries
  View k, v;
  void* pool;
  const int32_t* table;  // [B, max_pages]
  const int32_t* pos;    // [B, N]
  const float* cosines;  // [n_pos, d_rot / 2], null: no rotation
  const float* sines;
  int64_t B, Hq, Hk, N, n_pages, max_pages, n_pos;
  int page, dk, dv, d_rot;
  bool pairs, f32;
  cudaStream_t stream;
};
int launch_kv_append(const KvAppendArgs& a, char* msg, size_t msglen);

cudaError_t window_tc_read_and_clear_status(unsigned* value);
cudaError_t window_bwd_read_and_clear_status(unsigned* value);
cudaError_t window_cc_read_and_clear_status(unsigned* value);
cudaError_t kv_append_read_and_clear_status(unsigned* value);

// Status words of the translation units above (0, MOA_ERR_DEVICE_TIMEOUT or
// MOA_ERR_DEVICE_INDEX); read and cleared after a synchronisation.
cudaError_t norm_read_and_clear_status(unsigned* value);
cudaError_t kv4_read_and_clear_status(unsigned* value);
cudaError_t kv4_attn_read_and_clear_status(unsigned* value);
cudaError_t kv4_tc_read_and_clear_status(unsigned* value);

}  // namespace moa
