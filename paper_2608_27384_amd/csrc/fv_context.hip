// The C boundary of the observation context's operators: what the host can see
// of a call is checked here, before anything is enqueued.
#include "fv_context.h"

#include <cmath>
#include <exception>
#include <new>
#include <string>

#include "fv_error.h"

namespace fv {
namespace {

thread_local std::string context_error;

template <typename Fn>
fv_status guarded(Fn&& fn) noexcept {
  try {
    try {
      fn();
      context_error.clear();
      return FV_OK;
    } catch (const FvError& e) {
      context_error = e.msg;
      return e.st;
    } catch (const std::bad_alloc&) {
      context_error = "host allocation failed";
      return FV_ERR_OOM;
    } catch (const std::exception& e) {
      context_error = e.what();
      return FV_ERR_INTERNAL;
    }
  } catch (...) {  // also a message that could not be stored
    return FV_ERR_INTERNAL;
  }
}

[[noreturn]] void bad(const std::string& m) { fail(FV_ERR_INVALID_ARG, m); }

void aligned(const void* p, size_t to, const char* what) {
  need(p, what);
  if (reinterpret_cast<uintptr_t>(p) % to)
    bad(std::string(what) + " must be " + std::to_string(to) + "-byte aligned");
}

size_t type_size(int dtype) {
  if (dtype != FV_BF16 && dtype != FV_FP32) bad("dtype must be FV_BF16 or FV_FP32");
  return dtype == FV_BF16 ? 2 : 4;
}

void check_heads(int hq, int hkv, int dh) {
  if (dh != 64 && dh != 128 && dh != 192 && dh != 256) bad("head_dim must be 64, 128, 192 or 256");
  if (hkv < 1 || hq < 1 || hq > 1024 || hq % hkv)
    bad("n_q_heads must be a multiple of n_kv_heads, from 1 to 1024");
}

void check_cache(const fv_pages* c) {
  need(c, "cache");
  type_size(c->dtype);
  check_heads(c->n_kv_heads, c->n_kv_heads, c->head_dim);
  if (c->n_layers < 1 || c->n_layers > 1024) bad("n_layers must be 1 to 1024");
  if (c->page_len < 16 || c->page_len > 256 || c->page_len % 16)
    bad("page_len must be a multiple of 16, at most 256");
  if (c->n_pages < 1 || c->n_pages > (1 << 20)) bad("n_pages must be 1 to 2^20");
  if (c->max_seqs < 1 || c->max_seqs > 65536) bad("max_seqs must be 1 to 65536");
  if (c->max_pages < 1 || c->max_pages > 65536) bad("max_pages must be 1 to 65536");
  aligned(c->k, 16, "cache k");
  aligned(c->v, 16, "cache v");
  aligned(c->table, 4, "cache table");
  aligned(c->len, 4, "cache len");
  aligned(c->refs, 4, "cache refs");
}

// A strided operand: rows of `row` bytes, `ld` bytes apart, from lo to hi.
struct Span {
  uintptr_t lo = 0, hi = 0, row = 0, ld = 0;
};
Span operand(const void* p, int n, int ld, int row, size_t e, const char* what) {
  aligned(p, 16, what);
  if (ld < row || ld > (1 << 20) || (size_t)ld * e % 16)
    bad(std::string("leading dimension of ") + what + " must be at least " + std::to_string(row) +
        ", at most 2^20 and a multiple of 16 bytes");
  const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
  return Span{lo, lo + (n > 0 ? ((size_t)(n - 1) * ld + row) * e : 0), (size_t)row * e, (size_t)ld * e};
}
// Columns of one packed matrix are apart though their spans are not.
void apart(const Span& a, const Span& b, const char* what) {
  if (a.lo >= b.hi || b.lo >= a.hi) return;
  if (a.ld == b.ld) {
    const uintptr_t d = a.lo < b.lo ? (b.lo - a.lo) % a.ld : (a.lo - b.lo) % a.ld;
    if (a.lo < b.lo ? d >= a.row && d + b.row <= a.ld : d >= b.row && d + a.row <= a.ld) return;
  }
  bad(std::string(what) + " must not overlap");
}

// One run of `n` times `bytes` bytes (a size past 64 bits reaches the end of memory).
Span run_of(const void* p, size_t n, size_t bytes) {
  const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
  uintptr_t size, hi;
  if (__builtin_mul_overflow(n, bytes, &size) || __builtin_add_overflow(lo, size, &hi)) {
    hi = UINTPTR_MAX;
    size = hi - lo;
  }
  return Span{lo, hi, size, size};
}
// The pages of a layer in the pool p, and those of all layers.
size_t layer_bytes(const fv_pages& c) {
  return page_row(c.n_pages, c.n_kv_heads, 0, c.page_len) * c.head_dim * type_size(c.dtype);
}
Span layer_of(const void* p, const fv_pages& c, int layer) {
  return run_of(static_cast<const char*>(p) + layer * layer_bytes(c), 1, layer_bytes(c));
}
Span pool_of(const void* p, const fv_pages& c) { return run_of(p, c.n_layers, layer_bytes(c)); }

// A launch holds less than 2^32 threads in x and 2^16 workgroups in y and z.  The bounds of n,
// n * heads and n_seqs * heads in the calls below keep x under that: the most are the 256
// threads of 2^23 + 2^22 row tiles and spare slots of prompt attention, the 512 of 2^22 rows
// that paged attention joins and the rotary tokens, whose number a workgroup follows n
// (rope_tokens).  y and z count layers (1024 at most, 2049 with keys and values apart) or are cut
// to fit.
void check_launch() {
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) fail(FV_ERR_HIP, std::string("kernel launch: ") + hipGetErrorString(e));
}

// The stream's device for the duration of a call, and no earlier error left to be
// taken for the launch's.
int stream_device(hipStream_t s) {
  int dev = 0;
  if (s)
    FV_HIP(hipStreamGetDevice(s, &dev));
  else
    FV_HIP(hipGetDevice(&dev));
  return dev;
}
struct OnStream {
  DeviceScope scope;
  explicit OnStream(hipStream_t s) : scope(stream_device(s)) { (void)hipGetLastError(); }
};

void check_paged(const fv_paged_args* a, const fv_pages* c) {
  need(a, "args");
  check_cache(c);
  check_heads(a->n_q_heads, c->n_kv_heads, c->head_dim);
  if (a->n < 0 || a->n > 65536) bad("n must be 0 to 65536");
  if ((int64_t)a->n * a->n_q_heads > 1 << 22) bad("n * n_q_heads must be at most 2^22");
  if (a->max_len < 0) bad("max_len must not be negative");
  if (a->layer < 0 || a->layer >= c->n_layers) bad("layer out of range");
}

PagedPlan paged_plan(const fv_paged_args& a, const fv_pages& c) {
  const int holds = c.max_pages * c.page_len;
  const int keys = a.max_len > 0 && a.max_len < holds ? a.max_len : holds;
  return plan_paged(a.n, a.n_q_heads, c.n_kv_heads, c.head_dim, keys, c.dtype == FV_BF16);
}

void check_list(const fv_pages* c, const void* p, int n, const char* what) {
  check_cache(c);
  if (n < 0 || n > c->max_seqs) bad("n must be 0 to max_seqs");
  if (n) aligned(p, 4, what);
}

}  // namespace
}  // namespace fv

using namespace fv;

extern "C" {

const char* fv_context_error(void) { return context_error.c_str(); }

fv_status fv_rope_append(const fv_rope_args* a, const fv_pages* c, void* stream) {
  return guarded([&] {
    need(a, "args");
    const size_t e = type_size(a->dtype);
    check_heads(a->n_q_heads, a->n_kv_heads, a->head_dim);
    if (a->n < 0 || a->n > 1 << 26) bad("n must be 0 to 2^26");
    if (a->n_axes < 1 || a->n_axes > 4) bad("n_axes must be 1 to 4");
    int64_t pairs = 0;
    for (int i = 0; i < a->n_axes; ++i) {
      if (a->sections[i] < 0) bad("sections must not be negative");
      pairs += a->sections[i];
    }
    if (pairs != a->head_dim / 2) bad("sections must add up to head_dim/2");
    if (!(a->theta > 0.f) || !std::isfinite(a->theta)) bad("theta must be positive and finite");
    if (c) {
      check_cache(c);
      if (c->dtype != a->dtype || c->head_dim != a->head_dim || c->n_kv_heads != a->n_kv_heads)
        bad("the cache has another dtype, head_dim or n_kv_heads");
      if (a->layer < 0 || a->layer >= c->n_layers) bad("layer out of range");
    }
    if (a->n == 0) return;
    const int rq = a->n_q_heads * a->head_dim, rk = a->n_kv_heads * a->head_dim;
    const Span q = operand(a->q, a->n, a->ldq, rq, e, "q");
    const Span k = operand(a->k, a->n, a->ldk, rk, e, "k");
    const Span v = c ? operand(a->v, a->n, a->ldv, rk, e, "v") : Span{};
    const Span qo = operand(a->q_out, a->n, a->ldq_out, rq, e, "q_out");
    // an output may be its own input, and nothing else that the call reads or writes
    const bool q_in_place = a->q_out == a->q && a->ldq_out == a->ldq;
    if (!q_in_place) apart(qo, q, "q_out and q");
    if (!q_in_place || c || a->k_out) apart(qo, k, "q_out and k");
    apart(qo, v, "q_out and v");
    Span ko;
    if (a->k_out) {
      ko = operand(a->k_out, a->n, a->ldk_out, rk, e, "k_out");
      if (!(a->k_out == a->k && a->ldk_out == a->ldk)) apart(ko, k, "k_out and k");
      apart(ko, q, "k_out and q");
      apart(ko, v, "k_out and v");
      apart(ko, qo, "k_out and q_out");
    }
    if (c) {
      const Span pk = layer_of(c->k, *c, a->layer), pv = layer_of(c->v, *c, a->layer);
      apart(pk, pv, "cache k and v");
      for (const Span& p : {pk, pv}) {
        apart(qo, p, "q_out and the cache's pages");
        apart(ko, p, "k_out and the cache's pages");
      }
    }
    aligned(a->pos, 4, "pos");
    if (c) {
      aligned(a->seqs, 4, "seqs");
      aligned(a->at, 4, "at");
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    OnStream on(s);
    if (a->dtype == FV_BF16)
      launch_rope_append<bf16_t>(*a, c, s);
    else
      launch_rope_append<float>(*a, c, s);
    check_launch();
  });
}

fv_status fv_prompt_attention(const fv_prompt_args* a, void* stream) {
  return guarded([&] {
    need(a, "args");
    const size_t e = type_size(a->dtype);
    check_heads(a->n_q_heads, a->n_kv_heads, a->head_dim);
    if (a->n_seqs < 0 || a->n_seqs > 65536) bad("n_seqs must be 0 to 65536");
    if (a->n_q < 0 || a->n_k < 0) bad("n_q and n_k must not be negative");
    if (a->causal != 0 && a->causal != 1) bad("causal must be 0 or 1");
    if (!(a->scale > 0.f) || !std::isfinite(a->scale)) bad("scale must be positive and finite");
    if (a->n_seqs == 0 || a->n_q == 0) return;
    if ((int64_t)a->n_q * a->n_q_heads > 1 << 30) bad("n_q * n_q_heads must be at most 2^30");
    if ((int64_t)a->n_seqs * a->n_kv_heads > 1 << 22)
      bad("n_seqs * n_kv_heads must be at most 2^22");
    const int rq = a->n_q_heads * a->head_dim, rk = a->n_kv_heads * a->head_dim;
    const Span q = operand(a->q, a->n_q, a->ldq, rq, e, "q");
    const Span o = operand(a->out, a->n_q, a->ldo, rq, e, "out");
    apart(o, q, "out and q");
    if (a->n_k) {
      apart(o, operand(a->k, a->n_k, a->ldk, rk, e, "k"), "out and k");
      apart(o, operand(a->v, a->n_k, a->ldv, rk, e, "v"), "out and v");
    }
    aligned(a->cu_q, 4, "cu_q");
    aligned(a->cu_k, 4, "cu_k");
    hipStream_t s = static_cast<hipStream_t>(stream);
    OnStream on(s);
    if (a->dtype == FV_BF16)
      launch_prompt<bf16_t>(*a, s);
    else
      launch_prompt<float>(*a, s);
    check_launch();
  });
}

fv_status fv_paged_attention_workspace(const fv_paged_args* a, const fv_pages* c, size_t* bytes) {
  return guarded([&] {
    need(bytes, "bytes");
    check_paged(a, c);
    *bytes = a->n ? paged_plan(*a, *c).work_bytes : 0;
  });
}

fv_status fv_paged_attention(const fv_paged_args* a, const fv_pages* c, void* stream) {
  return guarded([&] {
    check_paged(a, c);
    if (!(a->scale > 0.f) || !std::isfinite(a->scale)) bad("scale must be positive and finite");
    if (a->n == 0) return;
    const size_t e = type_size(c->dtype);
    const int row = a->n_q_heads * c->head_dim;
    const Span out = operand(a->out, a->n, a->ldo, row, e, "out");
    const Span q = operand(a->q, a->n, a->ldq, row, e, "q");
    const Span pk = layer_of(c->k, *c, a->layer), pv = layer_of(c->v, *c, a->layer);
    apart(out, q, "out and q");
    apart(out, pk, "out and the cache's pages");
    apart(out, pv, "out and the cache's pages");
    aligned(a->seqs, 4, "seqs");
    const PagedPlan p = paged_plan(*a, *c);
    if (p.work_bytes) {
      aligned(a->work, 16, "work");
      if (a->work_bytes < p.work_bytes)
        bad("work holds " + std::to_string(a->work_bytes) + " bytes, " +
            std::to_string(p.work_bytes) + " are needed");
      const Span w = run_of(a->work, 1, p.work_bytes);
      apart(w, out, "work and out");
      apart(w, q, "work and q");
      apart(w, pk, "work and the cache's pages");
      apart(w, pv, "work and the cache's pages");
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    OnStream on(s);
    if (c->dtype == FV_BF16)
      launch_paged<bf16_t>(*a, *c, p, s);
    else
      launch_paged<float>(*a, *c, p, s);
    check_launch();
  });
}

fv_status fv_pages_workspace(const fv_pages* c, size_t* bytes) {
  return guarded([&] {
    need(bytes, "bytes");
    check_cache(c);
    *bytes = pages_work_ints(*c) * 4;
  });
}

fv_status fv_pages_grow(const fv_pages* c, const int32_t* seqs, const int32_t* add, int32_t n,
                        int32_t* status, void* work, void* stream) {
  return guarded([&] {
    check_list(c, seqs, n, "seqs");
    if (n) aligned(add, 4, "add");
    aligned(status, 4, "status");
    aligned(work, 16, "work");
    hipStream_t s = static_cast<hipStream_t>(stream);
    OnStream on(s);
    launch_pages_grow(*c, seqs, add, n, status, static_cast<int*>(work), s);
    check_launch();
  });
}

fv_status fv_pages_fork(const fv_pages* c, const int32_t* parents, const int32_t* children,
                        int32_t n, int32_t* status, void* work, void* stream) {
  return guarded([&] {
    check_list(c, parents, n, "parents");
    if (n) aligned(children, 4, "children");
    aligned(status, 4, "status");
    aligned(work, 16, "work");
    hipStream_t s = static_cast<hipStream_t>(stream);
    OnStream on(s);
    launch_pages_fork(*c, parents, children, n, status, static_cast<int*>(work), s);
    check_launch();
  });
}

fv_status fv_pages_free(const fv_pages* c, const int32_t* seqs, int32_t n, int32_t* status,
                        void* stream) {
  return guarded([&] {
    check_list(c, seqs, n, "seqs");
    aligned(status, 4, "status");
    hipStream_t s = static_cast<hipStream_t>(stream);
    OnStream on(s);
    launch_pages_free(*c, seqs, n, status, s);
    check_launch();
  });
}

fv_status fv_pages_compact(const fv_pages* c, int32_t* used, void* work, void* stream) {
  return guarded([&] {
    check_cache(c);
    aligned(used, 4, "used");
    aligned(work, 16, "work");
    hipStream_t s = static_cast<hipStream_t>(stream);
    OnStream on(s);
    launch_pages_compact(*c, used, static_cast<int*>(work), s);
    check_launch();
  });
}

fv_status fv_pages_gather(const fv_pages* c, const int32_t* seqs, int32_t n, int32_t ld,
                          void* k_out, void* v_out, void* stream) {
  return guarded([&] {
    check_cache(c);
    if (n < 0 || n > 65536) bad("n must be 0 to 65536");
    if (ld < 0) bad("ld must not be negative");
    if (n == 0 || ld == 0) return;
    aligned(seqs, 4, "seqs");
    aligned(k_out, 16, "k_out");
    aligned(v_out, 16, "v_out");
    // bytes of a row, of all heads: at most 2^20
    const size_t row = (size_t)c->n_kv_heads * c->head_dim * type_size(c->dtype);
    const size_t rows = (size_t)c->n_layers * n * ld;
    const Span ko = run_of(k_out, rows, row), vo = run_of(v_out, rows, row);
    apart(ko, vo, "k_out and v_out");
    for (const void* pool : {c->k, c->v}) {
      apart(ko, pool_of(pool, *c), "k_out and the cache's pages");
      apart(vo, pool_of(pool, *c), "v_out and the cache's pages");
    }
    hipStream_t s = static_cast<hipStream_t>(stream);
    OnStream on(s);
    launch_pages_gather(*c, seqs, n, ld, k_out, v_out, s);
    check_launch();
  });
}

}  // extern "C"
