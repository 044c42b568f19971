// C ABI of the operators around attention: argument checks and dispatch.  The contract of every
// entry point is documented in include/moa_attn.h.
#include <cuda_runtime.h>

#include <atomic>
#include <cmath>
#include <cstdint>
#include <exception>
#include <utility>

#include "../../include/moa_attn.h"
#include "internal.h"
#include "ops_internal.h"
#include "window.cuh"

namespace moa {
namespace {
std::atomic<int> g_most_cluster{0};
}  // namespace

void limit_clusters(int most) { g_most_cluster.store(most, std::memory_order_relaxed); }

int ClusterRoom::operator()(const void* kernel, int threads, int bytes, int size) {
  const int most = g_most_cluster.load(std::memory_order_relaxed);
  int dev = -1, at = 0;
  if ((most > 0 && size > most) || cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
  while ((1 << at) < size) ++at;
  const int known = known_[dev][at].load(std::memory_order_relaxed);
  if (known > 0) return known - 1;
  int n = 0;
  cudaError_t e = ensure_smem_limit(kernel, bytes);
  if (e == cudaSuccess && size > 8) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e == cudaSuccess) {
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = 1;
    attr.val.clusterDim.y = unsigned(size);
    attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t c{};
    c.gridDim = dim3(1, unsigned(size));
    c.blockDim = dim3(unsigned(threads));
    c.dynamicSmemBytes = size_t(bytes);
    c.attrs = &attr;
    c.numAttrs = 1;
    e = cudaOccupancyMaxActiveClusters(&n, kernel, &c);
  }
  if (e != cudaSuccess) {   // no error of the call, which takes smaller clusters or none
    cudaGetLastError();
    n = 0;
  }
  known_[dev][at].store(n + 1, std::memory_order_relaxed);
  return n;
}

namespace {

constexpr int64_t kMax31 = 0x7fffffffLL;
constexpr int64_t kMaxElements = INT64_MAX / 16;

// An exception must not cross the C boundary.
template <typename F>
int guarded(F&& f) {
  try {
    return f();
  } catch (const std::exception& e) {
    return api_fail(MOA_ERR_CUDA, "internal error: %s", e.what());
  } catch (...) {
    return api_fail(MOA_ERR_CUDA, "internal error");
  }
}

bool mul(int64_t a, int64_t b, int64_t* r) {
  return !__builtin_mul_overflow(a, b, r) && *r <= kMaxElements && *r >= -kMaxElements;
}

// Bytes [lo, hi) from the tensor's pointer that its rows span.
struct Span {
  uintptr_t lo, hi;
};
bool overlap(const Span& a, const Span& b) { return a.lo < b.hi && b.lo < a.hi; }

struct Shape {
  int64_t B, H, N, d;
};

// Checks pointer, strides and alignment of a [B, H, N, d] tensor and computes its span.
int check_view(const char* name, const View& v, const Shape& s, int64_t elt, bool output, Span* span) {
  if (v.p == nullptr) return api_fail(MOA_ERR_INVALID_ARG, "null pointer %s", name);
  const uintptr_t p = reinterpret_cast<uintptr_t>(v.p);
  if (p % 16 != 0) return api_fail(MOA_ERR_MISALIGNED, "%s is not 16-byte aligned", name);
  const int64_t size[3] = {s.B, s.H, s.N}, stride[3] = {v.sb, v.sh, v.sn};
  int64_t lo = 0, hi = 0;
  for (int i = 0; i < 3; ++i) {
    if (size[i] == 1) continue;
    if (stride[i] < -kMaxElements || stride[i] > kMaxElements || stride[i] * elt % 16 != 0)
      return api_fail(MOA_ERR_MISALIGNED, "%s: stride %lld is not a multiple of 16 bytes", name,
                      (long long)stride[i]);
    int64_t far;
    if (!mul(stride[i], size[i] - 1, &far)) return api_fail(MOA_ERR_UNSUPPORTED_SHAPE, "%s: strides overflow", name);
    if (far < 0) lo += far; else hi += far;
    if (lo < -kMaxElements || hi > kMaxElements) return api_fail(MOA_ERR_UNSUPPORTED_SHAPE, "%s: strides overflow", name);
  }
  if (output) {
    // rows apart from one another: each stride, in rising order, at least the extent below it
    int order[3] = {0, 1, 2};
    auto mag = [&](int i) { return stride[i] < 0 ? -stride[i] : stride[i]; };
    for (int i = 0; i < 3; ++i)
      for (int j = i + 1; j < 3; ++j)
        if (mag(order[j]) < mag(order[i])) {
          const int t = order[i];
          order[i] = order[j];
          order[j] = t;
        }
    int64_t extent = s.d;
    for (int i : order) {
      if (size[i] == 1) continue;
      if (mag(i) < extent) return api_fail(MOA_ERR_INVALID_ARG, "%s: an output's rows overlap one another", name);
      extent += mag(i) * (size[i] - 1);
    }
  }
  span->lo = p + uintptr_t(lo * elt);
  span->hi = p + uintptr_t((hi + s.d) * elt);
  return MOA_OK;
}

Span flat(const void* p, int64_t bytes) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p);
  return Span{a, a + uintptr_t(bytes)};
}

bool same_view(const View& a, const View& b) {
  return a.p == b.p && a.sb == b.sb && a.sh == b.sh && a.sn == b.sn;
}

// Whether two tensors of the same B and N whose spans meet are slices of one buffer that share no
// element: equal strides along B and N, and heads that lie apart.  The buffer's dimensions may be in any
// order: with k of B and N (those of the smaller strides) inside a head, a head is a piece of `in_a` or
// `in_b` elements (rows may differ in length); the two tensors' pieces must lie apart, one tensor's after the
// other's or in turn, and all of them within the strides of the dimensions outside.
bool disjoint_slices(const View& a, const Shape& sa, const View& b, const Shape& sb, int64_t elt) {
  if ((sa.B > 1 && a.sb != b.sb) || (sa.N > 1 && a.sn != b.sn)) return false;
  if (a.sh < 0 || b.sh < 0 || a.sn < 0 || a.sb < 0) return false;
  const intptr_t bytes = reinterpret_cast<intptr_t>(b.p) - reinterpret_cast<intptr_t>(a.p);
  if (bytes % elt != 0) return false;
  const int64_t off = bytes / elt;   // of b's first element from a's
  int64_t size[2] = {sa.N, sa.B}, stride[2] = {sa.N > 1 ? a.sn : 0, sa.B > 1 ? a.sb : 0};
  if (stride[0] > stride[1]) {
    std::swap(stride[0], stride[1]);
    std::swap(size[0], size[1]);
  }
  int64_t in_a = sa.d, in_b = sb.d;
  for (int k = 0; k <= 2; ++k) {
    if (k > 0) {
      if (size[k - 1] > 1 && (stride[k - 1] < in_a || stride[k - 1] < in_b)) return false;   // rows on one another
      in_a += (size[k - 1] - 1) * stride[k - 1];
      in_b += (size[k - 1] - 1) * stride[k - 1];
    }
    if ((sa.H > 1 && a.sh < in_a) || (sb.H > 1 && b.sh < in_b)) continue;
    const int64_t end_a = (sa.H - 1) * a.sh + in_a, end_b = off + (sb.H - 1) * b.sh + in_b;
    bool apart = end_a <= off || end_b <= 0;
    if (!apart && sa.H > 1 && sb.H > 1 && a.sh == b.sh) {
      const int64_t turn = (off % a.sh + a.sh) % a.sh;   // where b's pieces lie between a's
      apart = turn >= in_a && turn + in_b <= a.sh;
    }
    if (!apart) continue;
    int64_t whole = (end_a > end_b ? end_a : end_b) - (off < 0 ? off : 0);
    bool nested = true;
    for (int i = k; i < 2; ++i) {
      if (size[i] == 1) continue;
      nested = nested && stride[i] >= whole;
      whole += (size[i] - 1) * stride[i];
    }
    if (nested) return true;
  }
  return false;
}

int check_dtype(int dtype) {
  if (dtype != MOA_FP32 && dtype != MOA_BF16) return api_fail(MOA_ERR_UNSUPPORTED_DTYPE, "unknown dtype %d", dtype);
  return MOA_OK;
}

// ---------------------------------------------------------------------------------------------
// Norm and rotation
// ---------------------------------------------------------------------------------------------
struct Named {
  const char* name;
  const View* v;
  bool keys;     // H_k heads
  bool output;
  int alias;     // index of the input that this output may be, or -1
};

int norm_call(NormRopeArgs& a, int64_t d, int64_t d_rot, int dtype, bool bwd, size_t workspace_bytes) {
  int rc = check_dtype(dtype);
  if (rc != MOA_OK) return rc;
  if (a.B < 1 || a.Hq < 1 || a.Hk < 1 || a.N < 1 || a.n_pos < 1)
    return api_fail(MOA_ERR_INVALID_ARG, "sizes must be >= 1");
  if (a.Hq > 65535 || a.Hk > 65535 || a.Hq + a.Hk > 65535)
    return api_fail(MOA_ERR_UNSUPPORTED_SHAPE, "at most 65535 heads");
  int64_t tokens, all;
  if (!mul(a.B, a.N, &tokens) || !mul(tokens, (a.Hq + a.Hk) * 256, &all) || tokens > kMax31 * 4)
    return api_fail(MOA_ERR_UNSUPPORTED_SHAPE, "too many tokens");
  if (d < 8 || d > 256 || d % 8 != 0)
    return api_fail(MOA_ERR_UNSUPPORTED_SHAPE, "d must be a multiple of 8 up to 256; got %lld", (long long)d);
  if (d_rot < 16 || d_rot > d || d_rot % 16 != 0)
    return api_fail(MOA_ERR_UNSUPPORTED_SHAPE, "d_rot must be a multiple of 16 up to d; got %lld", (long long)d_rot);
  if (a.n_pos > kMax31) return api_fail(MOA_ERR_UNSUPPORTED_SHAPE, "n_pos must be below 2^31");
  if (!std::isfinite(a.eps) || !(a.eps > 0.f)) return api_fail(MOA_ERR_INVALID_ARG, "eps must be positive and finite");
  const int64_t elt = dtype == MOA_FP32 ? 4 : 2;
  a.d = int(d), a.d_rot = int(d_rot), a.f32 = dtype == MOA_FP32;
  struct Flat {
    const char* name;
    const void* p;
    int64_t bytes;
    int align;
    bool output;
  };
  // the workspace's size goes by the current device; without one its place is still checked
  size_t need = 0;
  cudaError_t device = cudaSuccess;
  if (bwd) {
    int sms = 0;
    device = device_sm_count(&sms);
    need = size_t(norm_rope_partial_rows(a.B, a.Hq, a.Hk, a.N, d, device == cudaSuccess ? sms : 1)) * d * 4;
  }
  const Flat flats[] = {{"W_q", a.wq, d * elt, 16, false},
                        {"W_k", a.wk, d * elt, 16, false},
                        {"cos", a.cosines, a.n_pos * d_rot * 2, 16, false},
                        {"sin", a.sines, a.n_pos * d_rot * 2, 16, false},
                        {"pos", a.pos, tokens * 4, 4, false},
                        {"dW_q", a.dwq, d * 4, 4, true},
                        {"dW_k", a.dwk, d * 4, 4, true},
                        {"workspace", a.partial, int64_t(need), 16, true}};
  const int n_flat = bwd ? 8 : 5;
  for (int i = 0; i < n_flat; ++i) {
    if (flats[i].p == nullptr) return api_fail(MOA_ERR_INVALID_ARG, "null pointer %s", flats[i].name);
    if (reinterpret_cast<uintptr_t>(flats[i].p) % flats[i].align != 0)
      return api_fail(MOA_ERR_MISALIGNED, "%s is not %d-byte aligned", flats[i].name, flats[i].align);
  }
  const Named fwd_t[] = {{"Q", &a.q, false, false, -1}, {"K", &a.k, true, false, -1},
                         {"Qo", &a.oq, false, true, 0}, {"Ko", &a.ok, true, true, 1}};
  const Named bwd_t[] = {{"Q", &a.q, false, false, -1},    {"K", &a.k, true, false, -1},
                         {"dQo", &a.gq, false, false, -1}, {"dKo", &a.gk, true, false, -1},
                         {"dQ", &a.oq, false, true, 2},    {"dK", &a.ok, true, true, 3}};
  const Named* t = bwd ? bwd_t : fwd_t;
  const int n_t = bwd ? 6 : 4;
  Span span[6];
  Shape shape[6];
  for (int i = 0; i < n_t; ++i) {
    shape[i] = Shape{a.B, t[i].keys ? a.Hk : a.Hq, a.N, d};
    rc = check_view(t[i].name, *t[i].v, shape[i], elt, t[i].output, &span[i]);
    if (rc != MOA_OK) return rc;
  }
  for (int i = 0; i < n_t; ++i) {
    if (!t[i].output) continue;
    for (int j = 0; j < n_t; ++j) {
      if (j == i || (t[j].output && j < i) || !overlap(span[i], span[j])) continue;
      if (j == t[i].alias && same_view(*t[i].v, *t[j].v)) continue;
      if (disjoint_slices(*t[i].v, shape[i], *t[j].v, shape[j], elt)) continue;
      return api_fail(MOA_ERR_INVALID_ARG, "%s overlaps %s", t[i].name, t[j].name);
    }
    for (int j = 0; j < n_flat; ++j)
      if (overlap(span[i], flat(flats[j].p, flats[j].bytes)))
        return api_fail(MOA_ERR_INVALID_ARG, "%s overlaps %s", t[i].name, flats[j].name);
  }
  for (int i = 0; i < n_flat; ++i) {
    if (!flats[i].output) continue;
    const Span s = flat(flats[i].p, flats[i].bytes);
    for (int j = 0; j < n_t; ++j)
      if (!t[j].output && overlap(s, span[j]))
        return api_fail(MOA_ERR_INVALID_ARG, "%s overlaps %s", flats[i].name, t[j].name);
    for (int j = 0; j < n_flat; ++j)
      if (j != i && overlap(s, flat(flats[j].p, flats[j].bytes)))
        return api_fail(MOA_ERR_INVALID_ARG, "%s overlaps %s", flats[i].name, flats[j].name);
  }
  if (device != cudaSuccess)
    return api_fail(MOA_ERR_CUDA, "SM count of the current device: %s", cudaGetErrorString(device));
  if (workspace_bytes < need)
    return api_fail(MOA_ERR_INVALID_ARG, "workspace too small: need %zu bytes, got %zu", need, workspace_bytes);
  char msg[256] = {0};
  rc = bwd ? launch_norm_rope_bwd(a, msg, sizeof(msg)) : launch_norm_rope(a, msg, sizeof(msg));
  if (rc != MOA_OK) return api_fail(rc, "%s", msg);
  api_clear();
  return api_debug_check(a.stream);
}

// A read-only tensor in the form the launchers take.
View view(const void* p, const int64_t* s) { return View{const_cast<void*>(p), s[0], s[1], s[2]}; }

// ---------------------------------------------------------------------------------------------
// The cache
// ---------------------------------------------------------------------------------------------
bool pool_bytes(int64_t n_pages, int64_t H, int64_t page, int64_t dk, int64_t dv, int64_t* bytes) {
  if (n_pages < 1 || H < 1 || page < 16 || page % 16 != 0) return false;
  if ((dk != 64 && dk != 128) || (dv != 64 && dv != 128)) return false;
  int64_t x;
  return mul(n_pages, H, &x) && mul(x, page / 16, &x) && mul(x, 9 * (dk + dv), bytes);
}

int check_cache(Kv4Cache& c, const void* pool, const int32_t* pages, int64_t B, int64_t H, int64_t d_k,
                int64_t d_v, int64_t n_pages, int64_t page_tokens, int64_t max_pages, Span* pool_span,
                Span* pages_span) {
  if (!pool || !pages) return api_fail(MOA_ERR_INVALID_ARG, "null pool or pages pointer");
  if (B < 1 || H < 1 || n_pages < 1 || max_pages < 1 || page_tokens < 1)
    return api_fail(MOA_ERR_INVALID_ARG, "sizes must be >= 1");
  if (page_tokens % 16 != 0 || page_tokens > (1 << 20))
    return api_fail(MOA_ERR_UNSUPPORTED_SHAPE, "page_tokens must be a multiple of 16 up to 2^20; got %lld",
                    (long long)page_tokens);
  if ((d_k != 64 && d_k != 128) || (d_v != 64 && d_v != 128))
    return api_fail(MOA_ERR_UNSUPPORTED_SHAPE, "the cache needs d_k, d_v in {64, 128}; got %lld, %lld",
                    (long long)d_k, (long long)d_v);
  int64_t bytes, table;
  if (H > kMax31 || n_pages > kMax31 || !pool_bytes(n_pages, H, page_tokens, d_k, d_v, &bytes) ||
      !mul(B, max_pages, &table) || max_pages > kMax31)
    return api_fail(MOA_ERR_UNSUPPORTED_SHAPE, "the pool or its table is too large");
  if (reinterpret_cast<uintptr_t>(pool) % 16 != 0) return api_fail(MOA_ERR_MISALIGNED, "pool is not 16-byte aligned");
  if (reinterpret_cast<uintptr_t>(pages) % 4 != 0) return api_fail(MOA_ERR_MISALIGNED, "pages is not 4-byte aligned");
  c = Kv4Cache{const_cast<void*>(pool), pages, n_pages, max_pages, int(page_tokens), int(H), int(d_k), int(d_v)};
  *pool_span = flat(pool, bytes);
  *pages_span = flat(pages, table * 4);
  return MOA_OK;
}

int move_call(const void* K, const void* V, const void* pool, const int32_t* pages, const int32_t* pos,
              int64_t B, int64_t H, int64_t N, int64_t d_k, int64_t d_v, int64_t n_pages,
              int64_t page_tokens, int64_t max_pages, const int64_t* strides, int dtype, void* stream,
              bool write) {
  int rc = check_dtype(dtype);
  if (rc != MOA_OK) return rc;
  Kv4MoveArgs a{};
  Span pool_s, pages_s, ks, vs;
  rc = check_cache(a.c, pool, pages, B, H, d_k, d_v, n_pages, page_tokens, max_pages, &pool_s, &pages_s);
  if (rc != MOA_OK) return rc;
  if (!pos || !strides) return api_fail(MOA_ERR_INVALID_ARG, "null pos or strides pointer");
  if (reinterpret_cast<uintptr_t>(pos) % 4 != 0) return api_fail(MOA_ERR_MISALIGNED, "pos is not 4-byte aligned");
  if (N < 1) return api_fail(MOA_ERR_INVALID_ARG, "sizes must be >= 1");
  int64_t rows;
  if (!mul(B, H, &rows) || !mul(rows, N, &rows) || !mul(rows, 128, &rows))
    return api_fail(MOA_ERR_UNSUPPORTED_SHAPE, "too many rows");
  const int64_t elt = dtype == MOA_FP32 ? 4 : 2;
  a.k = view(K, strides), a.v = view(V, strides + 3);
  const Shape sk{B, H, N, d_k}, sv{B, H, N, d_v};
  rc = check_view("K", a.k, sk, elt, !write, &ks);
  if (rc != MOA_OK) return rc;
  rc = check_view("V", a.v, sv, elt, !write, &vs);
  if (rc != MOA_OK) return rc;
  const Span pos_s = flat(pos, B * N * 4);
  if (overlap(pool_s, ks) || overlap(pool_s, vs) || overlap(pool_s, pages_s) || overlap(pool_s, pos_s))
    return api_fail(MOA_ERR_INVALID_ARG, "the pool overlaps a tensor");
  if (!write) {
    if (overlap(ks, vs) && !disjoint_slices(a.k, sk, a.v, sv, elt))
      return api_fail(MOA_ERR_INVALID_ARG, "K overlaps V");
    for (const Span& s : {ks, vs})
      if (overlap(s, pages_s) || overlap(s, pos_s))
        return api_fail(MOA_ERR_INVALID_ARG, "an output overlaps pages or pos");
  }
  a.pos = pos;
  a.B = B, a.N = N;
  a.f32 = dtype == MOA_FP32;
  a.stream = static_cast<cudaStream_t>(stream);
  char msg[256] = {0};
  rc = write ? launch_kv4_write(a, msg, sizeof(msg)) : launch_kv4_read(a, msg, sizeof(msg));
  if (rc != MOA_OK) return api_fail(rc, "%s", msg);
  api_clear();
  return api_debug_check(stream);
}

int attn_call(const void* Q, const void* pool, const int32_t* pages, const int32_t* lens, void* O,
              float* LSE, int64_t B, int64_t H_q, int64_t H_k, int64_t N, int64_t d_k, int64_t d_v,
              int64_t n_pages, int64_t page_tokens, int64_t max_pages, int64_t max_len,
              const int64_t* strides, float scale, int causal, int dtype, void* workspace,
              size_t workspace_bytes, void* stream) {
  int rc = check_dtype(dtype);
  if (rc != MOA_OK) return rc;
  Kv4AttnArgs a{};
  Span pool_s, pages_s, qs, os;
  rc = check_cache(a.c, pool, pages, B, H_k, d_k, d_v, n_pages, page_tokens, max_pages, &pool_s, &pages_s);
  if (rc != MOA_OK) return rc;
  if (!lens || !strides) return api_fail(MOA_ERR_INVALID_ARG, "null lens or strides pointer");
  if (reinterpret_cast<uintptr_t>(lens) % 4 != 0) return api_fail(MOA_ERR_MISALIGNED, "lens is not 4-byte aligned");
  if (N < 1 || H_q < 1 || max_len < 1) return api_fail(MOA_ERR_INVALID_ARG, "sizes must be >= 1");
  if (H_q % H_k != 0)
    return api_fail(MOA_ERR_UNSUPPORTED_SHAPE, "H_q must be a multiple of H_k; got %lld, %lld",
                    (long long)H_q, (long long)H_k);
  if (max_len > max_pages * page_tokens || max_len > kMax31 - 64)
    return api_fail(MOA_ERR_INVALID_ARG, "max_len %lld is more than the page table or the kernels take", (long long)max_len);
  int64_t rows;
  if (!mul(B, H_q, &rows) || !mul(rows, N, &rows) || rows > kMax31)
    return api_fail(MOA_ERR_UNSUPPORTED_SHAPE, "B * H_q * N must be below 2^31");
  if (!std::isfinite(scale)) return api_fail(MOA_ERR_INVALID_ARG, "scale must be finite");
  const int64_t elt = dtype == MOA_FP32 ? 4 : 2;
  a.q = view(Q, strides), a.o = view(O, strides + 3);
  rc = check_view("Q", a.q, Shape{B, H_q, N, d_k}, elt, false, &qs);
  if (rc != MOA_OK) return rc;
  rc = check_view("O", a.o, Shape{B, H_q, N, d_v}, elt, true, &os);
  if (rc != MOA_OK) return rc;
  if (reinterpret_cast<uintptr_t>(LSE) % 4 != 0) return api_fail(MOA_ERR_MISALIGNED, "LSE is not 4-byte aligned");
  const Span in[4] = {qs, pool_s, pages_s, flat(lens, B * 4)};
  const Span lse_s = flat(LSE, LSE ? rows * 4 : 0);
  for (const Span& s : in)
    if (overlap(os, s) || (LSE != nullptr && overlap(lse_s, s)))
      return api_fail(MOA_ERR_INVALID_ARG, "an output overlaps an input");
  if (LSE != nullptr && overlap(os, lse_s)) return api_fail(MOA_ERR_INVALID_ARG, "O overlaps LSE");
  int sms = 0;
  const cudaError_t e = device_sm_count(&sms);
  if (e != cudaSuccess)
    return api_fail(MOA_ERR_CUDA, "SM count of the current device: %s", cudaGetErrorString(e));
  const Kv4Plan plan = kv4_attn_plan(B, H_k, H_q / H_k, N, max_len, dtype == MOA_FP32, sms);
  const size_t need = kv4_attn_workspace(B, H_k, max_len, d_k, d_v, plan, sms);
  if (need > 0) {
    if (workspace == nullptr || workspace_bytes < need)
      return api_fail(MOA_ERR_INVALID_ARG, "workspace too small: need %zu bytes, got %zu", need,
                      workspace == nullptr ? size_t(0) : workspace_bytes);
    if (reinterpret_cast<uintptr_t>(workspace) % 16 != 0)
      return api_fail(MOA_ERR_MISALIGNED, "workspace is not 16-byte aligned");
    const Span ws = flat(workspace, int64_t(need));
    for (const Span& s : in)
      if (overlap(ws, s)) return api_fail(MOA_ERR_INVALID_ARG, "the workspace overlaps an input");
    if (overlap(ws, os) || (LSE != nullptr && overlap(ws, lse_s)))
      return api_fail(MOA_ERR_INVALID_ARG, "the workspace overlaps an output");
  }
  a.lse = LSE;
  a.lens = lens;
  a.B = B, a.Hq = H_q, a.N = N, a.max_len = max_len;
  a.scale = scale;
  a.causal = causal != 0, a.f32 = dtype == MOA_FP32;
  a.ws = workspace;
  a.stream = static_cast<cudaStream_t>(stream);
  char msg[256] = {0};
  rc = launch_kv4_attn(a, plan, msg, sizeof(msg));
  if (rc != MOA_OK) return api_fail(rc, "%s", msg);
  api_clear();
  return api_debug_check(stream);
}

// ---------------------------------------------------------------------------------------------
// Attention with a window, its gradients, and the 16- and 32-bit cache
// ---------------------------------------------------------------------------------------------
// Rows and tokens stay this far below 2^31: the kernels look ahead by a tile or two in 32 bits.
constexpr int64_t kMostRows = kMax31 - 1024;
constexpr float kMostScale = 2e38f;   // times log2 e still finite

// Two tensors that may share a buffer without sharing an element.
bool apart(const View& a, const Shape& sa, const View& b, const Shape& sb, int64_t elt) {
  return sa.N == sb.N && sa.B == sb.B && disjoint_slices(a, sa, b, sb, elt);
}

struct Tensor {
  const char* name;
  const View* v;
  Shape shape;
  bool output;
  int alias;   // index of the input that this output may be, or -1
};
struct Buffer {
  const char* name;
  const void* p;
  int64_t bytes;
  int align;
  bool output;
};

// Every tensor and buffer by itself, then no output on anything else.
template <int NT, int NB>
int check_operands(const Tensor (&t)[NT], const Buffer (&f)[NB], int64_t elt) {
  Span span[NT];
  for (int i = 0; i < NB; ++i) {
    if (f[i].p == nullptr) return api_fail(MOA_ERR_INVALID_ARG, "null pointer %s", f[i].name);
    if (reinterpret_cast<uintptr_t>(f[i].p) % f[i].align != 0)
      return api_fail(MOA_ERR_MISALIGNED, "%s is not %d-byte aligned", f[i].name, f[i].align);
  }
  for (int i = 0; i < NT; ++i) {
    const int rc = check_view(t[i].name, *t[i].v, t[i].shape, elt, t[i].output, &span[i]);
    if (rc != MOA_OK) return rc;
  }
  for (int i = 0; i < NT; ++i) {
    if (!t[i].output) continue;
    for (int j = 0; j < NT; ++j) {
      if (j == i || (t[j].output && j < i) || !overlap(span[i], span[j])) continue;
      if (j == t[i].alias && same_view(*t[i].v, *t[j].v)) continue;
      if (apart(*t[i].v, t[i].shape, *t[j].v, t[j].shape, elt)) continue;
      return api_fail(MOA_ERR_INVALID_ARG, "%s overlaps %s", t[i].name, t[j].name);
    }
    for (int j = 0; j < NB; ++j)
      if (overlap(span[i], flat(f[j].p, f[j].bytes)))
        return api_fail(MOA_ERR_INVALID_ARG, "%s overlaps %s", t[i].name, f[j].name);
  }
  for (int i = 0; i < NB; ++i) {
    if (!f[i].output) continue;
    const Span s = flat(f[i].p, f[i].bytes);
    for (int j = 0; j < NT; ++j)
      if (!t[j].output && overlap(s, span[j])) return api_fail(MOA_ERR_INVALID_ARG, "%s overlaps %s", f[i].name, t[j].name);
    for (int j = 0; j < NB; ++j)
      if (j != i && overlap(s, flat(f[j].p, f[j].bytes)))
        return api_fail(MOA_ERR_INVALID_ARG, "%s overlaps %s", f[i].name, f[j].name);
  }
  return MOA_OK;
}

// Sizes and settings that windowed attention, its gradients and cache attention share.
int check_window(int64_t B, int64_t Hq, int64_t Hk, int64_t N, int64_t dk, int64_t dv, int64_t window, int64_t sinks,
                 float scale) {
  if (B < 1 || Hq < 1 || Hk < 1 || N < 1) return api_fail(MOA_ERR_INVALID_ARG, "sizes must be >= 1");
  if (Hq % Hk != 0)
    return api_fail(MOA_ERR_UNSUPPORTED_SHAPE, "H_q must be a multiple of H_k; got %lld, %lld", (long long)Hq, (long long)Hk);
  if ((dk != 64 && dk != 128) || (dv != 64 && dv != 128))
    return api_fail(MOA_ERR_UNSUPPORTED_SHAPE, "d_k, d_v must be 64 or 128; got %lld, %lld", (long long)dk, (long long)dv);
  int64_t rows;
  if (!mul(B, Hq, &rows) || !mul(rows, N, &rows) || rows > kMostRows)
    return api_fail(MOA_ERR_UNSUPPORTED_SHAPE, "B * H_q * N must be at most 2^31 - 1025");
  if (window < 0 || sinks < 0) return api_fail(MOA_ERR_INVALID_ARG, "window and sinks must not be negative");
  if (!(std::fabs(scale) <= kMostScale)) return api_fail(MOA_ERR_INVALID_ARG, "scale must be finite, and 2e38 at most");
  return MOA_OK;
}

// A window as the kernels take it: one that reaches past every token is none, and then nothing but the
// sequence's beginning is a sink.
void set_window(WindowArgs& a, int64_t window, int64_t sinks) {
  a.window = window == 0 || window >= a.max_len ? win::kNoWindow : int(window);
  a.sinks = int(a.window == win::kNoWindow ? 0 : sinks < a.max_len ? sinks : a.max_len);
}

// What either kernel needs: a workspace's size does not go by strides.
size_t window_workspace(const WindowArgs& a, int sms) {
  const size_t cc = window_cc_workspace(a, window_cc_plan(a, sms)), tc = a.f32 ? 0 : window_tc_workspace(a, sms);
  return cc > tc ? cc : tc;
}
int launch_window(const WindowArgs& a, int sms, char* msg, size_t msglen) {
  if (window_tc_takes(a)) return launch_window_tc(a, sms, msg, msglen);
  return launch_window_cc(a, window_cc_plan(a, sms), msg, msglen);
}

// The workspace of a call: as large as it has to be, aligned, and on nothing else.
int run_window(WindowArgs& a, const Span* in, int n_in, const Span& out, void* workspace, size_t workspace_bytes) {
  int64_t rows = a.B * a.Hq * a.N;
  if (reinterpret_cast<uintptr_t>(a.lse) % 4 != 0) return api_fail(MOA_ERR_MISALIGNED, "LSE is not 4-byte aligned");
  const Span lse_s = flat(a.lse, a.lse ? rows * 4 : 0);
  for (int i = 0; i < n_in; ++i)
    if (overlap(out, in[i]) || (a.lse != nullptr && overlap(lse_s, in[i])))
      return api_fail(MOA_ERR_INVALID_ARG, "an output overlaps an input");
  if (a.lse != nullptr && overlap(out, lse_s)) return api_fail(MOA_ERR_INVALID_ARG, "O overlaps LSE");
  int sms = 0;
  const cudaError_t e = device_sm_count(&sms);
  if (e != cudaSuccess) return api_fail(MOA_ERR_CUDA, "SM count of the current device: %s", cudaGetErrorString(e));
  const size_t need = window_workspace(a, sms);
  if (need > 0) {
    if (workspace == nullptr || workspace_bytes < need)
      return api_fail(MOA_ERR_INVALID_ARG, "workspace too small: need %zu bytes, got %zu", need,
                      workspace == nullptr ? size_t(0) : workspace_bytes);
    if (reinterpret_cast<uintptr_t>(workspace) % 16 != 0) return api_fail(MOA_ERR_MISALIGNED, "workspace is not 16-byte aligned");
    const Span ws = flat(workspace, int64_t(need));
    for (int i = 0; i < n_in; ++i)
      if (overlap(ws, in[i])) return api_fail(MOA_ERR_INVALID_ARG, "the workspace overlaps an input");
    if (overlap(ws, out) || (a.lse != nullptr && overlap(ws, lse_s)))
      return api_fail(MOA_ERR_INVALID_ARG, "the workspace overlaps an output");
  }
  a.ws = workspace;
  char msg[256] = {0};
  const int rc = launch_window(a, sms, msg, sizeof(msg));
  if (rc != MOA_OK) return api_fail(rc, "%s", msg);
  api_clear();
  return api_debug_check(a.stream);
}

int check_keys(int64_t B, int64_t Hk, int64_t Nk) {
  if (Nk < 1) return api_fail(MOA_ERR_INVALID_ARG, "sizes must be >= 1");
  int64_t rows;
  if (!mul(B, Hk, &rows) || !mul(rows, Nk, &rows) || rows > kMostRows)
    return api_fail(MOA_ERR_UNSUPPORTED_SHAPE, "B * H_k * N_k must be at most 2^31 - 1025");
  return MOA_OK;
}

int window_call(const void* Q, const void* K, const void* V, void* O, float* LSE, int64_t B, int64_t H_q, int64_t H_k,
                int64_t N_q, int64_t N_k, int64_t d_k, int64_t d_v, int64_t window, int64_t sinks, const int64_t* strides,
                float scale, int dtype, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_dtype(dtype);
  if (rc == MOA_OK) rc = check_window(B, H_q, H_k, N_q, d_k, d_v, window, sinks, scale);
  if (rc == MOA_OK) rc = check_keys(B, H_k, N_k);
  if (rc != MOA_OK) return rc;
  if (!strides) return api_fail(MOA_ERR_INVALID_ARG, "null strides pointer");
  const int64_t elt = dtype == MOA_FP32 ? 4 : 2;
  WindowArgs a{};
  const View k = view(K, strides + 3), v = view(V, strides + 6);
  a.q = view(Q, strides), a.o = view(O, strides + 9);
  Span in[3], out;
  rc = check_view("Q", a.q, Shape{B, H_q, N_q, d_k}, elt, false, &in[0]);
  if (rc == MOA_OK) rc = check_view("K", k, Shape{B, H_k, N_k, d_k}, elt, false, &in[1]);
  if (rc == MOA_OK) rc = check_view("V", v, Shape{B, H_k, N_k, d_v}, elt, false, &in[2]);
  if (rc == MOA_OK) rc = check_view("O", a.o, Shape{B, H_q, N_q, d_v}, elt, true, &out);
  if (rc != MOA_OK) return rc;
  a.kv = KvSource{K, V, k.sb, k.sh, k.sn, v.sb, v.sh, v.sn, nullptr, B, 0, 0};
  a.lse = LSE, a.lens = nullptr;
  a.B = B, a.Hq = H_q, a.Hk = H_k, a.N = N_q, a.max_len = N_k;
  a.dk = int(d_k), a.dv = int(d_v);
  set_window(a, window, sinks);
  a.scale = scale, a.causal = true, a.f32 = dtype == MOA_FP32;
  a.stream = static_cast<cudaStream_t>(stream);
  return run_window(a, in, 3, out, workspace, workspace_bytes);
}

bool kv_pool_size(int64_t n_pages, int64_t H, int64_t page, int64_t dk, int64_t dv, int64_t elt, int64_t* bytes) {
  if (n_pages < 1 || H < 1 || page < 16 || page % 16 != 0) return false;
  if ((dk != 64 && dk != 128) || (dv != 64 && dv != 128)) return false;
  int64_t x;
  return mul(n_pages, H, &x) && mul(x, page, &x) && mul(x, (dk + dv) * elt, bytes);
}

// The pool, its table, and their sizes.
int check_pool(const void* pool, const int32_t* pages, int64_t B, int64_t H, int64_t d_k, int64_t d_v, int64_t n_pages,
               int64_t page_tokens, int64_t max_pages, int64_t elt, Span* pool_span, Span* pages_span) {
  if (!pool || !pages) return api_fail(MOA_ERR_INVALID_ARG, "null pool or pages pointer");
  if (n_pages < 1 || max_pages < 1 || page_tokens < 1) return api_fail(MOA_ERR_INVALID_ARG, "sizes must be >= 1");
  if (page_tokens % 16 != 0 || page_tokens > (1 << 20))
    return api_fail(MOA_ERR_UNSUPPORTED_SHAPE, "page_tokens must be a multiple of 16 up to 2^20; got %lld",
                    (long long)page_tokens);
  int64_t bytes, table;
  if (H > kMax31 || n_pages > kMax31 - 1 || !kv_pool_size(n_pages, H, page_tokens, d_k, d_v, elt, &bytes) ||
      !mul(B, max_pages, &table) || max_pages > kMax31)
    return api_fail(MOA_ERR_UNSUPPORTED_SHAPE, "the pool or its table is too large");
  if (reinterpret_cast<uintptr_t>(pool) % 16 != 0) return api_fail(MOA_ERR_MISALIGNED, "pool is not 16-byte aligned");
  if (reinterpret_cast<uintptr_t>(pages) % 4 != 0) return api_fail(MOA_ERR_MISALIGNED, "pages is not 4-byte aligned");
  *pool_span = flat(pool, bytes);
  *pages_span = flat(pages, table * 4);
  return MOA_OK;
}

int cache_call(const void* Q, const void* pool, const int32_t* pages, const int32_t* lens, void* O, float* LSE, int64_t B,
               int64_t H_q, int64_t H_k, int64_t N, int64_t d_k, int64_t d_v, int64_t n_pages, int64_t page_tokens,
               int64_t max_pages, int64_t max_len, int64_t window, int64_t sinks, const int64_t* strides, float scale,
               int causal, int dtype, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = check_dtype(dtype);
  if (rc == MOA_OK) rc = check_window(B, H_q, H_k, N, d_k, d_v, window, sinks, scale);
  if (rc != MOA_OK) return rc;
  const int64_t elt = dtype == MOA_FP32 ? 4 : 2;
  Span in[4], out;
  rc = check_pool(pool, pages, B, H_k, d_k, d_v, n_pages, page_tokens, max_pages, elt, &in[1], &in[2]);
  if (rc != MOA_OK) return rc;
  if (!lens || !strides) return api_fail(MOA_ERR_INVALID_ARG, "null lens or strides pointer");
  if (reinterpret_cast<uintptr_t>(lens) % 4 != 0) return api_fail(MOA_ERR_MISALIGNED, "lens is not 4-byte aligned");
  if (max_len < 1) return api_fail(MOA_ERR_INVALID_ARG, "sizes must be >= 1");
  if (max_len > max_pages * page_tokens || max_len > kMostRows)
    return api_fail(MOA_ERR_INVALID_ARG, "max_len %lld is more than the page table or the kernels take", (long long)max_len);
  WindowArgs a{};
  a.q = view(Q, strides), a.o = view(O, strides + 3);
  rc = check_view("Q", a.q, Shape{B, H_q, N, d_k}, elt, false, &in[0]);
  if (rc == MOA_OK) rc = check_view("O", a.o, Shape{B, H_q, N, d_v}, elt, true, &out);
  if (rc != MOA_OK) return rc;
  in[3] = flat(lens, B * 4);
  const int64_t row = d_k + d_v;
  a.kv = KvSource{pool, static_cast<const char*>(pool) + d_k * elt, H_k * page_tokens * row, page_tokens * row, row,
                  H_k * page_tokens * row, page_tokens * row, row, pages, n_pages, max_pages, int(page_tokens)};
  a.lse = LSE, a.lens = lens;
  a.B = B, a.Hq = H_q, a.Hk = H_k, a.N = N, a.max_len = max_len;
  a.dk = int(d_k), a.dv = int(d_v);
  set_window(a, window, sinks);
  a.scale = scale, a.causal = causal != 0, a.f32 = dtype == MOA_FP32;
  a.stream = static_cast<cudaStream_t>(stream);
  return run_window(a, in, 4, out, workspace, workspace_bytes);
}

size_t window_bwd_workspace(const WindowBwdArgs& a) {
  const size_t cc = window_bwd_cc_workspace(a), tc = a.f32 ? 0 : window_bwd_tc_workspace(a);
  return cc > tc ? cc : tc;
}

void set_bwd_window(WindowBwdArgs& a, int64_t window, int64_t sinks) {
  a.window = window == 0 || window >= a.Nk ? win::kNoWindow : int(window);
  a.sinks = int(a.window == win::kNoWindow ? 0 : sinks < a.Nk ? sinks : a.Nk);
}

int window_bwd_call(WindowBwdArgs& a, int64_t window, int64_t sinks, int dtype, size_t workspace_bytes) {
  const int64_t elt = dtype == MOA_FP32 ? 4 : 2;
  set_bwd_window(a, window, sinks);
  const size_t need = window_bwd_workspace(a);
  const Shape q{a.B, a.Hq, a.Nq, a.dk}, k{a.B, a.Hk, a.Nk, a.dk}, v{a.B, a.Hk, a.Nk, a.dv}, o{a.B, a.Hq, a.Nq, a.dv};
  const Tensor t[] = {{"Q", &a.q, q, false, -1},  {"K", &a.k, k, false, -1},   {"V", &a.v, v, false, -1},
                      {"O", &a.o, o, false, -1},  {"dO", &a.go, o, false, -1}, {"dQ", &a.dq, q, true, -1},
                      {"dK", &a.dk_, k, true, -1}, {"dV", &a.dv_, v, true, -1}};
  const Buffer f[] = {{"LSE", a.lse, a.B * a.Hq * a.Nq * 4, 4, false}, {"workspace", a.ws, int64_t(need), 16, true}};
  int rc = check_operands(t, f, elt);
  if (rc != MOA_OK) return rc;
  if (workspace_bytes < need)
    return api_fail(MOA_ERR_INVALID_ARG, "workspace too small: need %zu bytes, got %zu", need, workspace_bytes);
  char msg[256] = {0};
  rc = window_bwd_tc_takes(a) ? launch_window_bwd_tc(a, msg, sizeof(msg)) : launch_window_bwd_cc(a, msg, sizeof(msg));
  if (rc != MOA_OK) return api_fail(rc, "%s", msg);
  api_clear();
  return api_debug_check(a.stream);
}

int append_call(KvAppendArgs& a, int64_t d_k, int64_t d_v, int64_t d_rot, int64_t page_tokens, int dtype) {
  const int64_t elt = dtype == MOA_FP32 ? 4 : 2;
  const bool with_q = a.q.p != nullptr, turns = a.cosines != nullptr;
  if (a.B < 1 || a.Hk < 1 || a.N < 1 || (with_q && a.Hq < 1)) return api_fail(MOA_ERR_INVALID_ARG, "sizes must be >= 1");
  if ((d_k != 64 && d_k != 128) || (d_v != 64 && d_v != 128))
    return api_fail(MOA_ERR_UNSUPPORTED_SHAPE, "d_k, d_v must be 64 or 128; got %lld, %lld", (long long)d_k, (long long)d_v);
  if (!with_q) a.Hq = 0;
  if (a.Hq > 65535 || a.Hk > 65535) return api_fail(MOA_ERR_UNSUPPORTED_SHAPE, "at most 65535 heads");
  int64_t tokens, all;
  if (!mul(a.B, a.N, &tokens) || !mul(tokens, (a.Hq + 2 * a.Hk) * 128, &all) || tokens > kMax31)
    return api_fail(MOA_ERR_UNSUPPORTED_SHAPE, "too many tokens");
  if (turns != (a.sines != nullptr)) return api_fail(MOA_ERR_INVALID_ARG, "cos and sin go together");
  if (with_q && !turns) return api_fail(MOA_ERR_INVALID_ARG, "queries are only passed to be rotated: cos and sin are null");
  if (turns) {
    if (a.n_pos < 1) return api_fail(MOA_ERR_INVALID_ARG, "sizes must be >= 1");
    if (a.n_pos > kMax31) return api_fail(MOA_ERR_UNSUPPORTED_SHAPE, "n_pos must be below 2^31");
    if (d_rot < 16 || d_rot > d_k || d_rot % 16 != 0)
      return api_fail(MOA_ERR_UNSUPPORTED_SHAPE, "d_rot must be a multiple of 16 up to d_k; got %lld", (long long)d_rot);
  }
  Span pool_s, pages_s;
  int rc = check_pool(a.pool, a.table, a.B, a.Hk, d_k, d_v, a.n_pages, page_tokens, a.max_pages, elt, &pool_s, &pages_s);
  if (rc != MOA_OK) return rc;
  a.page = int(page_tokens), a.dk = int(d_k), a.dv = int(d_v), a.d_rot = turns ? int(d_rot) : 0;
  a.f32 = dtype == MOA_FP32;
  const Shape q{a.B, a.Hq, a.N, d_k}, k{a.B, a.Hk, a.N, d_k}, v{a.B, a.Hk, a.N, d_v};
  const Buffer pool{"the pool", a.pool, int64_t(pool_s.hi - pool_s.lo), 16, true};
  const Buffer pages{"pages", a.table, int64_t(pages_s.hi - pages_s.lo), 4, false}, pos{"pos", a.pos, tokens * 4, 4, false};
  const Tensor tk{"K", &a.k, k, false, -1}, tv{"V", &a.v, v, false, -1};
  if (turns) {
    const Buffer f[] = {pool, pages, pos, {"cos", a.cosines, a.n_pos * d_rot * 2, 16, false},
                        {"sin", a.sines, a.n_pos * d_rot * 2, 16, false}};
    if (with_q) {
      const Tensor t[] = {{"Q", &a.q, q, false, -1}, {"Qo", &a.oq, q, true, 0}, tk, tv};
      rc = check_operands(t, f, elt);
    } else {
      const Tensor t[] = {tk, tv};
      rc = check_operands(t, f, elt);
    }
  } else {
    const Buffer f[] = {pool, pages, pos};
    const Tensor t[] = {tk, tv};
    rc = check_operands(t, f, elt);
  }
  if (rc != MOA_OK) return rc;
  char msg[256] = {0};
  rc = launch_kv_append(a, msg, sizeof(msg));
  if (rc != MOA_OK) return api_fail(rc, "%s", msg);
  api_clear();
  return api_debug_check(a.stream);
}

}  // namespace
}  // namespace moa

extern "C" {

int moa_qk_norm_rope(const void* Q, const void* K, const void* W_q, const void* W_k,
                     const float* cos, const float* sin, const int32_t* pos, void* Qo, void* Ko,
                     int64_t B, int64_t H_q, int64_t H_k, int64_t N, int64_t d, int64_t d_rot,
                     int64_t n_pos, const int64_t* strides, float eps, int interleaved, int dtype,
                     void* stream) {
  return moa::guarded([&] {
    if (!strides) return moa::api_fail(MOA_ERR_INVALID_ARG, "null strides pointer");
    moa::NormRopeArgs a{};
    a.q = moa::view(Q, strides), a.k = moa::view(K, strides + 3);
    a.oq = moa::view(Qo, strides + 6), a.ok = moa::view(Ko, strides + 9);
    a.wq = W_q, a.wk = W_k, a.cosines = cos, a.sines = sin, a.pos = pos;
    a.B = B, a.Hq = H_q, a.Hk = H_k, a.N = N, a.n_pos = n_pos;
    a.eps = eps, a.pairs = interleaved != 0;
    a.stream = static_cast<cudaStream_t>(stream);
    return moa::norm_call(a, d, d_rot, dtype, false, 0);
  });
}

int moa_qk_norm_rope_bwd(const void* Q, const void* K, const void* W_q, const void* W_k,
                         const float* cos, const float* sin, const int32_t* pos, const void* dQo,
                         const void* dKo, void* dQ, void* dK, float* dW_q, float* dW_k, int64_t B,
                         int64_t H_q, int64_t H_k, int64_t N, int64_t d, int64_t d_rot,
                         int64_t n_pos, const int64_t* strides, float eps, int interleaved,
                         int dtype, void* workspace, size_t workspace_bytes, void* stream) {
  return moa::guarded([&] {
    if (!strides) return moa::api_fail(MOA_ERR_INVALID_ARG, "null strides pointer");
    moa::NormRopeArgs a{};
    a.q = moa::view(Q, strides), a.k = moa::view(K, strides + 3);
    a.gq = moa::view(dQo, strides + 6), a.gk = moa::view(dKo, strides + 9);
    a.oq = moa::view(dQ, strides + 12), a.ok = moa::view(dK, strides + 15);
    a.wq = W_q, a.wk = W_k, a.cosines = cos, a.sines = sin, a.pos = pos;
    a.dwq = dW_q, a.dwk = dW_k, a.partial = static_cast<float*>(workspace);
    a.B = B, a.Hq = H_q, a.Hk = H_k, a.N = N, a.n_pos = n_pos;
    a.eps = eps, a.pairs = interleaved != 0;
    a.stream = static_cast<cudaStream_t>(stream);
    return moa::norm_call(a, d, d_rot, dtype, true, workspace_bytes);
  });
}

size_t moa_qk_norm_rope_bwd_workspace_bytes(int64_t B, int64_t H_q, int64_t H_k, int64_t N,
                                            int64_t d) {
  if (B < 1 || H_q < 1 || H_k < 1 || N < 1 || d < 8 || d > 256 || H_q > 65535 || H_k > 65535) return 0;
  int64_t tokens, all;
  if (!moa::mul(B, N, &tokens) || !moa::mul(tokens, (H_q + H_k) * 256, &all)) return 0;
  int sms = 0;
  if (moa::device_sm_count(&sms) != cudaSuccess) return 0;
  return size_t(moa::norm_rope_partial_rows(B, H_q, H_k, N, d, sms)) * size_t(d) * 4;
}

size_t moa_kv4_pool_bytes(int64_t n_pages, int64_t H, int64_t page_tokens, int64_t d_k, int64_t d_v) {
  int64_t bytes;
  return moa::pool_bytes(n_pages, H, page_tokens, d_k, d_v, &bytes) ? size_t(bytes) : 0;
}

int moa_kv4_write(const void* K, const void* V, void* pool, const int32_t* pages,
                  const int32_t* pos, int64_t B, int64_t H, int64_t N, int64_t d_k, int64_t d_v,
                  int64_t n_pages, int64_t page_tokens, int64_t max_pages, const int64_t* strides,
                  int dtype, void* stream) {
  return moa::guarded([&] {
    return moa::move_call(K, V, pool, pages, pos, B, H, N, d_k, d_v, n_pages, page_tokens, max_pages,
                          strides, dtype, stream, true);
  });
}

int moa_kv4_read(void* K, void* V, const void* pool, const int32_t* pages, const int32_t* pos,
                 int64_t B, int64_t H, int64_t N, int64_t d_k, int64_t d_v, int64_t n_pages,
                 int64_t page_tokens, int64_t max_pages, const int64_t* strides, int dtype,
                 void* stream) {
  return moa::guarded([&] {
    return moa::move_call(K, V, pool, pages, pos, B, H, N, d_k, d_v, n_pages, page_tokens, max_pages,
                          strides, dtype, stream, false);
  });
}

int moa_kv4_attn(const void* Q, const void* pool, const int32_t* pages, const int32_t* lens, void* O,
                 float* LSE, int64_t B, int64_t H_q, int64_t H_k, int64_t N, int64_t d_k,
                 int64_t d_v, int64_t n_pages, int64_t page_tokens, int64_t max_pages,
                 int64_t max_len, const int64_t* strides, float scale, int causal, int dtype,
                 void* workspace, size_t workspace_bytes, void* stream) {
  return moa::guarded([&] {
    return moa::attn_call(Q, pool, pages, lens, O, LSE, B, H_q, H_k, N, d_k, d_v, n_pages, page_tokens,
                          max_pages, max_len, strides, scale, causal, dtype, workspace, workspace_bytes,
                          stream);
  });
}

size_t moa_kv4_attn_workspace_bytes(int64_t B, int64_t H_q, int64_t H_k, int64_t N, int64_t d_k,
                                    int64_t d_v, int64_t max_len, int dtype) {
  if ((dtype != MOA_BF16 && dtype != MOA_FP32) || B < 1 || H_q < 1 || H_k < 1 || N < 1 || max_len < 1) return 0;
  if (H_q % H_k != 0 || (d_k != 64 && d_k != 128) || (d_v != 64 && d_v != 128) || max_len > moa::kMax31 - 64) return 0;
  int64_t rows;
  if (!moa::mul(B, H_q, &rows) || !moa::mul(rows, N, &rows) || rows > moa::kMax31) return 0;
  int sms = 0;
  if (moa::device_sm_count(&sms) != cudaSuccess) return 0;
  return moa::kv4_attn_workspace(B, H_k, max_len, d_k, d_v,
                                 moa::kv4_attn_plan(B, H_k, H_q / H_k, N, max_len, dtype == MOA_FP32, sms), sms);
}

int moa_window_attn(const void* Q, const void* K, const void* V, void* O, float* LSE, int64_t B, int64_t H_q, int64_t H_k,
                    int64_t N_q, int64_t N_k, int64_t d_k, int64_t d_v, int64_t window, int64_t sinks,
                    const int64_t* strides, float scale, int dtype, void* workspace, size_t workspace_bytes,
                    void* stream) {
  return moa::guarded([&] {
    return moa::window_call(Q, K, V, O, LSE, B, H_q, H_k, N_q, N_k, d_k, d_v, window, sinks, strides, scale, dtype,
                            workspace, workspace_bytes, stream);
  });
}

size_t moa_window_attn_workspace_bytes(int64_t B, int64_t H_q, int64_t H_k, int64_t N_q, int64_t N_k, int64_t d_k,
                                       int64_t d_v, int64_t window, int64_t sinks, int dtype) {
  return moa_kv_attn_workspace_bytes(B, H_q, H_k, N_q, d_k, d_v, N_k, window, sinks, dtype);
}

int moa_window_attn_bwd(const void* Q, const void* K, const void* V, const void* O, const void* dO, const float* LSE,
                        void* dQ, void* dK, void* dV, int64_t B, int64_t H_q, int64_t H_k, int64_t N_q, int64_t N_k,
                        int64_t d_k, int64_t d_v, int64_t window, int64_t sinks, const int64_t* strides, float scale,
                        int dtype, void* workspace, size_t workspace_bytes, void* stream) {
  return moa::guarded([&] {
    int rc = moa::check_dtype(dtype);
    if (rc == MOA_OK) rc = moa::check_window(B, H_q, H_k, N_q, d_k, d_v, window, sinks, scale);
    if (rc == MOA_OK) rc = moa::check_keys(B, H_k, N_k);
    if (rc != MOA_OK) return rc;
    if (!strides) return moa::api_fail(MOA_ERR_INVALID_ARG, "null strides pointer");
    moa::WindowBwdArgs a{};
    const moa::View x[] = {moa::view(Q, strides), moa::view(K, strides + 3), moa::view(V, strides + 6),
                           moa::view(O, strides + 9), moa::view(dO, strides + 12), moa::view(dQ, strides + 15),
                           moa::view(dK, strides + 18), moa::view(dV, strides + 21)};
    a.q = x[0], a.k = x[1], a.v = x[2], a.o = x[3], a.go = x[4], a.dq = x[5], a.dk_ = x[6], a.dv_ = x[7];
    a.lse = LSE;
    a.B = B, a.Hq = H_q, a.Hk = H_k, a.Nq = N_q, a.Nk = N_k, a.dk = int(d_k), a.dv = int(d_v);
    a.scale = scale, a.f32 = dtype == MOA_FP32;
    a.ws = workspace;
    a.stream = static_cast<cudaStream_t>(stream);
    return moa::window_bwd_call(a, window, sinks, dtype, workspace_bytes);
  });
}

size_t moa_window_attn_bwd_workspace_bytes(int64_t B, int64_t H_q, int64_t H_k, int64_t N_q, int64_t N_k, int64_t d_k,
                                           int64_t d_v, int64_t window, int64_t sinks, int dtype) {
  if ((dtype != MOA_BF16 && dtype != MOA_FP32) || B < 1 || H_q < 1 || H_k < 1 || N_q < 1 || N_k < 1) return 0;
  if (H_q % H_k != 0 || (d_k != 64 && d_k != 128) || (d_v != 64 && d_v != 128) || window < 0 || sinks < 0) return 0;
  int64_t rows;
  if (!moa::mul(B, H_q, &rows) || !moa::mul(rows, N_q, &rows) || rows > moa::kMostRows) return 0;
  if (!moa::mul(B, H_k, &rows) || !moa::mul(rows, N_k, &rows) || rows > moa::kMostRows) return 0;
  moa::WindowBwdArgs a{};
  a.B = B, a.Hq = H_q, a.Hk = H_k, a.Nq = N_q, a.Nk = N_k, a.dk = int(d_k), a.dv = int(d_v);
  a.f32 = dtype == MOA_FP32;
  moa::set_bwd_window(a, window, sinks);
  return moa::window_bwd_workspace(a);
}

int moa_selftest_cluster_limit(int most) {
  if (most != 0 && most != 1 && most != 2 && most != 4 && most != 8 && most != 16)
    return moa::api_fail(MOA_ERR_INVALID_ARG, "the limit must be 0, 1, 2, 4, 8 or 16; got %d", most);
  moa::limit_clusters(most);
  moa::api_clear();
  return MOA_OK;
}

size_t moa_kv_pool_bytes(int64_t n_pages, int64_t H, int64_t page_tokens, int64_t d_k, int64_t d_v, int dtype) {
  int64_t bytes;
  if (dtype != MOA_BF16 && dtype != MOA_FP32) return 0;
  return moa::kv_pool_size(n_pages, H, page_tokens, d_k, d_v, dtype == MOA_FP32 ? 4 : 2, &bytes) ? size_t(bytes) : 0;
}

int moa_kv_append(const void* Q, const void* K, const void* V, const float* cos, const float* sin, void* pool,
                  const int32_t* pages, const int32_t* pos, void* Qo, int64_t B, int64_t H_q, int64_t H_k, int64_t N,
                  int64_t d_k, int64_t d_v, int64_t d_rot, int64_t n_pos, int64_t n_pages, int64_t page_tokens,
                  int64_t max_pages, const int64_t* strides, int interleaved, int dtype, void* stream) {
  return moa::guarded([&] {
    const int rc = moa::check_dtype(dtype);
    if (rc != MOA_OK) return rc;
    if (!strides) return moa::api_fail(MOA_ERR_INVALID_ARG, "null strides pointer");
    if ((Q == nullptr) != (Qo == nullptr)) return moa::api_fail(MOA_ERR_INVALID_ARG, "Q and Qo go together");
    moa::KvAppendArgs a{};
    a.q = moa::view(Q, strides), a.k = moa::view(K, strides + 3), a.v = moa::view(V, strides + 6);
    a.oq = moa::view(Qo, strides + 9);
    a.pool = pool, a.table = pages, a.pos = pos, a.cosines = cos, a.sines = sin;
    a.B = B, a.Hq = H_q, a.Hk = H_k, a.N = N, a.n_pages = n_pages, a.max_pages = max_pages, a.n_pos = n_pos;
    a.pairs = interleaved != 0;
    a.stream = static_cast<cudaStream_t>(stream);
    return moa::append_call(a, d_k, d_v, d_rot, page_tokens, dtype);
  });
}

int moa_kv_attn(const void* Q, const void* pool, const int32_t* pages, const int32_t* lens, void* O, float* LSE, int64_t B,
                int64_t H_q, int64_t H_k, int64_t N, int64_t d_k, int64_t d_v, int64_t n_pages, int64_t page_tokens,
                int64_t max_pages, int64_t max_len, int64_t window, int64_t sinks, const int64_t* strides, float scale,
                int causal, int dtype, void* workspace, size_t workspace_bytes, void* stream) {
  return moa::guarded([&] {
    return moa::cache_call(Q, pool, pages, lens, O, LSE, B, H_q, H_k, N, d_k, d_v, n_pages, page_tokens, max_pages, max_len,
                           window, sinks, strides, scale, causal, dtype, workspace, workspace_bytes, stream);
  });
}

size_t moa_kv_attn_workspace_bytes(int64_t B, int64_t H_q, int64_t H_k, int64_t N, int64_t d_k, int64_t d_v,
                                   int64_t max_len, int64_t window, int64_t sinks, int dtype) {
  if ((dtype != MOA_BF16 && dtype != MOA_FP32) || B < 1 || H_q < 1 || H_k < 1 || N < 1 || max_len < 1) return 0;
  if (H_q % H_k != 0 || (d_k != 64 && d_k != 128) || (d_v != 64 && d_v != 128) || max_len > moa::kMostRows) return 0;
  int64_t rows;
  if (window < 0 || sinks < 0 || !moa::mul(B, H_q, &rows) || !moa::mul(rows, N, &rows) || rows > moa::kMostRows) return 0;
  int sms = 0;
  if (moa::device_sm_count(&sms) != cudaSuccess) return 0;
  moa::WindowArgs a{};
  a.B = B, a.Hq = H_q, a.Hk = H_k, a.N = N, a.max_len = max_len, a.dk = int(d_k), a.dv = int(d_v);
  a.f32 = dtype == MOA_FP32;
  moa::set_window(a, window, sinks);
  return moa::window_workspace(a, sms);
}

}  // extern "C"
