// C ABI of the operators around attention: argument checks and dispatch.  The contract of every
// entry point is documented in include/moa_attn.h.
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>
#include <exception>
#include <utility>

#include "../../include/moa_attn.h"
#include "internal.h"
#include "ops_internal.h"

namespace moa {
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

// Whether two tensors of the same B, N and d whose spans meet are slices of one buffer that share no
// element: equal strides along B and N, and heads that lie apart.  The buffer's dimensions may be in any
// order: with k of B and N (those of the smaller strides) inside a head, a head is a piece of `inner`
// elements; the two tensors' pieces must lie apart, one tensor's after the other's or in turn, and all of
// them within the strides of the dimensions outside.
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
  int64_t inner = sa.d;
  for (int k = 0; k <= 2; ++k) {
    if (k > 0) {
      if (size[k - 1] > 1 && stride[k - 1] < inner) return false;   // rows on one another
      inner += (size[k - 1] - 1) * stride[k - 1];
    }
    if ((sa.H > 1 && a.sh < inner) || (sb.H > 1 && b.sh < inner)) continue;
    const int64_t end_a = (sa.H - 1) * a.sh + inner, end_b = off + (sb.H - 1) * b.sh + inner;
    bool apart = end_a <= off || end_b <= 0;
    if (!apart && sa.H > 1 && sb.H > 1 && a.sh == b.sh) {
      const int64_t turn = (off % a.sh + a.sh) % a.sh;   // where b's pieces lie between a's
      apart = turn >= inner && turn + inner <= a.sh;
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

}  // extern "C"
