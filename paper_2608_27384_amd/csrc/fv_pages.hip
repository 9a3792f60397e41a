// The paged cache of the observation context: rotary positions fused with the
// append to its pages, and its upkeep (grow, fork, free, compact, gather).
//
// All of it moves data: nothing here is bound by arithmetic.  The bookkeeping
// (table, lengths, holders) lives on the device, so a captured graph can change
// it; each change is decided as a whole by one workgroup (plan kernels: checks,
// then page numbers) and carried out by as many as the data wants.
#include "fv_context.h"

namespace fv {
namespace {

// ------------------------------------------------------------ rotary append

struct RopeCall {
  fv_rope_args a;
  fv_pages c;
  int has_cache, tokens;  // tokens of a workgroup
  double log2_theta;
};

// A workgroup first forms the cosines and sines of its tokens, once for all
// heads (RopeAngles).  Then each thread takes 16 bytes of a head's first half and
// the 16 that they are paired with.  Memory bounds it: 38 thousand tokens, heads 8/1 of 256,
// 78 us (388 MB, 4.9 TB/s, as a copy has);
// 64 tokens 3.8 us, a launch and one trip to memory.
template <typename T, int DH>
__global__ __launch_bounds__(kRopeThreads) void rope_append_kernel(RopeCall r) {
  constexpr int HALF = DH / 2;
  constexpr int VE = 16 / (int)sizeof(T);
  constexpr int PIECES = HALF / VE;           // 16-byte pieces of half a head
  __shared__ __attribute__((aligned(16))) float cs[kRopeTokens][HALF], sn[kRopeTokens][HALF];
  __shared__ long long slot[kRopeTokens];     // row of the token's place for kv head 0, or -1

  const fv_rope_args& a = r.a;
  const int tid = threadIdx.x;
  const int t0 = blockIdx.x * r.tokens;
  const int nt = min(r.tokens, a.n - t0);

  if (tid < nt && r.has_cache) {
    const int s = a.seqs[t0 + tid], at = a.at[t0 + tid];
    long long row = -1;
    if (s >= 0 && s < r.c.max_seqs && at >= 0 && at < r.c.max_pages * r.c.page_len) {
      const int page = r.c.table[(size_t)s * r.c.max_pages + at / r.c.page_len];
      if (page >= 0 && page < r.c.n_pages)
        row = (long long)page_row(page, a.n_kv_heads, 0, r.c.page_len) + at % r.c.page_len;
    }
    slot[tid] = row;
  }
  RopeAngles<DH>(a, r.log2_theta, kRopeThreads).form(t0, 0, nt, cs, sn);
  __syncthreads();

  const int hk = a.n_q_heads, hv = hk + a.n_kv_heads;
  const int heads = r.has_cache ? hv + a.n_kv_heads : (a.k_out ? hv : hk);
  const T* q = static_cast<const T*>(a.q);
  const T* k = static_cast<const T*>(a.k);
  const T* v = static_cast<const T*>(a.v);
  const size_t layer = (size_t)a.layer * r.c.n_pages * r.c.n_kv_heads * r.c.page_len * DH;
  for (int idx = tid; idx < nt * heads * PIECES; idx += kRopeThreads) {
    const int piece = idx % PIECES, th = idx / PIECES;
    const int t = th / heads, h = th - t * heads;
    const size_t tok = t0 + t;
    const T* src = h < hk ? q + tok * a.ldq + h * DH
                   : h < hv ? k + tok * a.ldk + (h - hk) * DH
                            : v + tok * a.ldv + (h - hv) * DH;
    u32x4 lo = *reinterpret_cast<const u32x4*>(src + piece * VE);
    u32x4 hi = *reinterpret_cast<const u32x4*>(src + HALF + piece * VE);
    if (h < hv) {
      T x[VE], y[VE];
      __builtin_memcpy(x, &lo, 16);
      __builtin_memcpy(y, &hi, 16);
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const float c = cs[t][piece * VE + e], s = sn[t][piece * VE + e];
        const float xf = to_f32(x[e]), yf = to_f32(y[e]);
        x[e] = from_f32<T>(xf * c - yf * s);
        y[e] = from_f32<T>(yf * c + xf * s);
      }
      __builtin_memcpy(&lo, x, 16);
      __builtin_memcpy(&hi, y, 16);
      T* out = h < hk ? static_cast<T*>(a.q_out) + tok * a.ldq_out + h * DH
               : a.k_out ? static_cast<T*>(a.k_out) + tok * a.ldk_out + (h - hk) * DH : nullptr;
      if (out) {
        *reinterpret_cast<u32x4*>(out + piece * VE) = lo;
        *reinterpret_cast<u32x4*>(out + HALF + piece * VE) = hi;
      }
    }
    if (h >= hk && r.has_cache) {
      const long long row = slot[t];
      if (row >= 0) {
        const int g = h < hv ? h - hk : h - hv;
        T* dst = static_cast<T*>(h < hv ? r.c.k : r.c.v) + layer +
                 ((size_t)row + (size_t)g * r.c.page_len) * DH;
        *reinterpret_cast<u32x4*>(dst + piece * VE) = lo;
        *reinterpret_cast<u32x4*>(dst + HALF + piece * VE) = hi;
      }
    }
  }
}

// ------------------------------------------------------------------- upkeep

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / 64;
// Pages looked at between two barriers: 64 J of each wave, J at most 16 and no more
// than needed (a wave takes about a hundred cycles for each 64).
__device__ __forceinline__ int scan_groups(const fv_pages& c) {
  return min(16, (c.n_pages + kPlanThreads - 1) / kPlanThreads);
}

struct PlanShared {
  int wave[2][kPlanWaves];
  int bad;
  uint32_t seen[65536 / 32];
};

__device__ __forceinline__ int pages_of(int len, int page_len) {
  return (len + page_len - 1) / page_len;
}
__device__ __forceinline__ bool is_page(const fv_pages& c, int p) { return p >= 0 && p < c.n_pages; }

// A plan kernel is one workgroup, bound by its trips to memory one after another: 7.4
// us to fork and 6.7 to grow by 32 children, 10.3 to compact a cache of 4564 pages.
// Exclusive sum over the workgroup; *total is the whole.
__device__ int block_scan(int x, int* wave_sums, int* total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int inc = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(inc, d);
    if (lane >= d) inc += y;
  }
  __syncthreads();
  if (lane == 63) wave_sums[w] = inc;
  __syncthreads();
  int before = 0, all = 0;
  for (int i = 0; i < kPlanWaves; ++i) {
    before += i < w ? wave_sums[i] : 0;
    all += wave_sums[i];
  }
  *total = all;
  return before + inc - x;
}

__device__ void clear_seen(PlanShared& sh, int max_seqs) {
  if (threadIdx.x == 0) sh.bad = 0;
  for (int i = threadIdx.x; i < (max_seqs + 31) / 32; i += kPlanThreads) sh.seen[i] = 0;
  __syncthreads();
}
// Marks sequence s; whether it had been marked.
__device__ bool mark(PlanShared& sh, int s) {
  const uint32_t bit = 1u << (s & 31);
  return atomicOr(&sh.seen[s >> 5], bit) & bit;
}

// A wave's pages first + 64 j + lane, j < J: their holders, which of them `pick` takes.
struct Holders {
  int refs[16];
  __device__ __forceinline__ void load(const fv_pages& c, int first, int J) {
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const int p = first + 64 * j + (int)(threadIdx.x & 63);
      refs[j] = j < J && p < c.n_pages ? c.refs[p] : 0;
    }
  }
};
template <typename Pick>
__device__ __forceinline__ int pick_pages(const fv_pages& c, const Holders& h, int first, int J,
                                          uint64_t (&m)[16], Pick pick) {
  const int lane = threadIdx.x & 63;
  int n = 0;
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    const int p = first + 64 * j + lane;
    m[j] = j < J ? __ballot(p < c.n_pages && pick(p, h.refs[j])) : 0;
    n += __popcll(m[j]);
  }
  return n;
}
__device__ __forceinline__ void list_pages(const uint64_t (&m)[16], int first, int J, int at, int limit,
                                           int* list) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    if (j < J) {
      const int rank = at + __popcll(m[j] & ((1ull << lane) - 1));
      if ((m[j] >> lane & 1) && rank < limit) list[rank] = first + 64 * j + lane;
      at += __popcll(m[j]);
    }
  }
}

// The lowest `want` free pages into list; how many there are, at most want.  h: the
// wave's holders of the first pages, loaded while the call was being checked.
__device__ int take_free(const fv_pages& c, Holders& h, int want, int* list, PlanShared& sh) {
  const int w = threadIdx.x >> 6, J = scan_groups(c);
  int found = 0;
  for (int p0 = 0; p0 < c.n_pages && found < want; p0 += kPlanThreads * J) {
    const int first = p0 + w * 64 * J;
    if (p0) h.load(c, first, J);
    uint64_t m[16];
    const int n = pick_pages(c, h, first, J, m, [](int, int refs) { return refs <= 0; });
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.wave[0][w] = n;
    __syncthreads();
    int before = 0, all = 0;
    for (int i = 0; i < kPlanWaves; ++i) {
      before += i < w ? sh.wave[0][i] : 0;
      all += sh.wave[0][i];
    }
    if (found + before < want) list_pages(m, first, J, found + before, want, list);
    found += all;
  }
  __syncthreads();
  return found < want ? found : want;
}

__device__ __forceinline__ void verdict(int st, int* status, int* work) {
  if (threadIdx.x == 0) {
    *status = st;
    if (work) work[0] = st;
  }
}

// Entries that a plan kernel carries out by itself: a launch of its own costs 3.4 us of
// the host.  us on the GPU by itself and with a second launch: grown by a page each, 64
// sequences 6.0 and 7.9, 1024 8.0 and 9.5; by 51 pages each, 64 sequences 7.7 and 8.6, 512
// 18 and 14; freed, with 408 table entries 2.2 and 4.0, with 8192 4.9 and 4.0.
constexpr int kInline = kPlanThreads;  // sequences of a grow or free
constexpr int kInlineRows = 8192;      // table entries of a free
__host__ __device__ __forceinline__ bool free_inline(const fv_pages& c, int n) {
  return n <= kInline && (long long)n * c.max_pages <= kInlineRows;
}
constexpr int kBatch = 4;  // entries of a thread under way at a time

// Workspace: [0] the call's status; lists A, B, C of `list` ints each.
// A: pages taken.  B[i]: how many were taken for the entries before i.

__global__ __launch_bounds__(kPlanThreads) void grow_plan_kernel(fv_pages c, const int* seqs,
                                                                 const int* add, int n,
                                                                 int* status, int* work,
                                                                 int list) {
  __shared__ PlanShared sh;
  __shared__ int first[kInline];       // of a request's pages: in A
  __shared__ uint32_t place[kInline];  // and in the table
  int* A = work + kPagesHeader;
  int* B = A + list;
  Holders h;
  h.load(c, (threadIdx.x >> 6) * 64 * scan_groups(c), scan_groups(c));
  clear_seen(sh, c.max_seqs);
  long long total = 0;
  int mine = -1, now = 0;  // the thread's sequence, if the lists are short, and its length to be
  for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
    const int i = i0 + threadIdx.x;
    int need = 0, have = 0;
    if (i < n) {
      const int s = seqs[i];
      bool ok = s >= 0 && s < c.max_seqs && !mark(sh, s);
      if (ok) {
        const int len = c.len[s], more = add[i], holds = c.max_pages * c.page_len;
        ok = len >= 0 && len <= holds && more >= 0 && more <= holds - len;
        if (ok && more > 0 && len % c.page_len) {
          const int last = c.table[(size_t)s * c.max_pages + len / c.page_len];
          ok = is_page(c, last) && c.refs[last] == 1;
        }
        if (ok) {
          have = pages_of(len, c.page_len);
          need = pages_of(len + more, c.page_len) - have;
          mine = s;
          now = len + more;
        }
      }
      if (!ok) sh.bad = 1;
    }
    int all;
    const int before = block_scan(need, sh.wave[1], &all);
    if (i < n) {
      B[i] = (int)(total + before);
      if (n <= kInline) {
        first[i] = before;
        place[i] = (uint32_t)mine * c.max_pages + have;
      }
    }
    total += all;
  }
  __syncthreads();
  if (sh.bad) return verdict(FV_PAGES_BAD, status, work);
  if (total > c.n_pages || take_free(c, h, (int)total, A, sh) < total)
    return verdict(FV_PAGES_FULL, status, work);
  verdict(FV_PAGES_OK, status, work);
  if (n > kInline) return;
  if (total <= kPlanThreads) {  // a page a thread
    const int t = threadIdx.x;
    if (t < (int)total) {
      const int page = A[t];
      int lo = 0, hi = n;  // the last request whose pages start at t or before
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= t)
          lo = mid;
        else
          hi = mid;
      }
      c.table[(size_t)place[lo] + (t - first[lo])] = page;
      c.refs[page] = 1;
    }
  } else {  // 16 lanes a request: no search, which 52 thousand pages would spend 45 us on
    constexpr int LANES = 16, GROUPS = kPlanThreads / LANES;
    for (int i0 = threadIdx.x / LANES; i0 < n; i0 += kBatch * GROUPS) {
      int at[kBatch], end[kBatch], most = 0;
      uint32_t to[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int i = i0 + u * GROUPS, r = min(i, n - 1);
        at[u] = first[r];
        end[u] = i >= n ? at[u] : r + 1 < n ? first[r + 1] : (int)total;
        to[u] = place[r];
        most = max(most, end[u] - at[u]);
      }
      for (int j = threadIdx.x % LANES; j < most; j += LANES) {
        int page[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) page[u] = at[u] + j < end[u] ? A[at[u] + j] : -1;
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
          if (page[u] >= 0) {
            c.table[(size_t)to[u] + j] = page[u];
            c.refs[page[u]] = 1;
          }
      }
    }
  }
  if (mine >= 0) c.len[mine] = now;
}

__global__ __launch_bounds__(64) void grow_apply_kernel(fv_pages c, const int* seqs, const int* add,
                                                        const int* work, int list) {
  if (work[0] != FV_PAGES_OK) return;
  const int i = blockIdx.x, s = seqs[i];
  const int* A = work + kPagesHeader;
  const int at = A[list + i];
  const int len = c.len[s], now = len + add[i];
  const int have = pages_of(len, c.page_len), need = pages_of(now, c.page_len) - have;
  int* row = c.table + (size_t)s * c.max_pages + have;
  for (int j = threadIdx.x; j < need; j += 64) {
    const int page = A[at + j];
    row[j] = page;
    c.refs[page] = 1;
  }
  if (threadIdx.x == 0) c.len[s] = now;
}

__global__ __launch_bounds__(kPlanThreads) void fork_plan_kernel(fv_pages c, const int* parents,
                                                                 const int* children, int n,
                                                                 int* status, int* work,
                                                                 int list) {
  __shared__ PlanShared sh;
  int* A = work + kPagesHeader;
  int* B = A + list;
  Holders h;
  h.load(c, (threadIdx.x >> 6) * 64 * scan_groups(c), scan_groups(c));
  clear_seen(sh, c.max_seqs);
  const int holds = c.max_pages * c.page_len;
  int total = 0;
  for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
    const int i = i0 + threadIdx.x;
    int need = 0;
    if (i < n) {
      const int cs = children[i], ps = parents[i];
      bool ok = cs >= 0 && cs < c.max_seqs && ps >= 0 && ps < c.max_seqs;
      if (ok) {
        const int empty = c.len[cs], len = c.len[ps];
        ok = !mark(sh, cs) && empty == 0 && len >= 0 && len <= holds;
        need = ok && len % c.page_len;
      }
      if (!ok) sh.bad = 1;
    }
    int all;
    const int before = block_scan(need, sh.wave[1], &all);
    if (i < n) B[i] = total + before;
    total += all;
  }
  // every child is marked: no parent is one, and its entries in use are pages
  for (int i = threadIdx.x >> 6; i < n; i += kPlanWaves) {
    const int s = parents[i];
    if (s < 0 || s >= c.max_seqs) continue;
    if (sh.seen[s >> 5] >> (s & 31) & 1) sh.bad = 1;
    const int pages = pages_of(min(max(c.len[s], 0), holds), c.page_len);
    const int* row = c.table + (size_t)s * c.max_pages;
    for (int j = threadIdx.x & 63; j < pages; j += 64)
      if (!is_page(c, row[j])) sh.bad = 1;
  }
  __syncthreads();
  if (sh.bad) return verdict(FV_PAGES_BAD, status, work);
  if (total > c.n_pages || take_free(c, h, total, A, sh) < total)
    return verdict(FV_PAGES_FULL, status, work);
  verdict(FV_PAGES_OK, status, work);
}

// Block (i, 0) writes the child's bookkeeping; blocks (i, 1 + 2 l + kv) copy the
// rows in use of the parent's part-filled last page, in layer l: in 8 bits the blocks of
// 16 that hold them, and their scales.
__global__ __launch_bounds__(256) void fork_apply_kernel(fv_pages c, const int* parents,
                                                         const int* children, const int* work,
                                                         int list, int row16, Scales q) {
  if (work[0] != FV_PAGES_OK) return;
  const int i = blockIdx.x, tid = threadIdx.x;
  const int ps = parents[i], len = c.len[ps];
  const int full = len / c.page_len, part = len % c.page_len;
  const int* A = work + kPagesHeader;
  const int* from = c.table + (size_t)ps * c.max_pages;
  if (blockIdx.y == 0) {
    const int cs = children[i];
    int* to = c.table + (size_t)cs * c.max_pages;
    for (int j = tid; j < c.max_pages; j += 256) {
      int page = -1;
      if (j < full) {
        page = from[j];
        atomicAdd(&c.refs[page], 1);
      } else if (j == full && part) {
        page = A[A[list + i]];
        c.refs[page] = 1;
      }
      to[j] = page;
    }
    if (tid == 0) c.len[cs] = len;
    return;
  }
  if (!part) return;
  const int l = (blockIdx.y - 1) >> 1;
  u32x4* pool = static_cast<u32x4*>((blockIdx.y - 1) & 1 ? c.v : c.k);
  const size_t base = (size_t)l * c.n_pages;
  const size_t page16 = (size_t)c.n_kv_heads * c.page_len * row16;  // 16-byte pieces of a page
  const size_t src_page = base + from[full], dst_page = base + A[A[list + i]];
  const u32x4* src = pool + src_page * page16;
  u32x4* dst = pool + dst_page * page16;
  const int blocks = (part + 15) / 16;
  const int run = (q.k ? 16 * blocks : part) * row16;  // pieces in use of one head
  for (int x = tid; x < run * c.n_kv_heads; x += 256) {
    const int h = x / run;
    const size_t at = (size_t)h * c.page_len * row16 + (x - h * run);
    dst[at] = src[at];
  }
  if (q.k) {
    uint8_t* scales = (blockIdx.y - 1) & 1 ? q.v : q.k;
    const int per = c.page_len / 16, all = c.n_kv_heads * per;
    for (int x = tid; x < all; x += 256)
      if (x % per < blocks) scales[dst_page * all + x] = scales[src_page * all + x];
  }
}

__global__ __launch_bounds__(kPlanThreads) void free_plan_kernel(fv_pages c, const int* seqs, int n,
                                                                 int* status) {
  __shared__ PlanShared sh;
  __shared__ uint32_t place[kInline];  // of a sequence's table row
  __shared__ int held[kInline];        // its pages
  const bool here = free_inline(c, n);
  clear_seen(sh, c.max_seqs);
  int mine = -1;
  for (int i = threadIdx.x; i < n; i += kPlanThreads) {
    const int s = seqs[i];
    if (s < 0 || s >= c.max_seqs || mark(sh, s)) {
      sh.bad = 1;
    } else if (here) {
      mine = s;
      place[i] = (uint32_t)s * c.max_pages;
      held[i] = pages_of(min(max(c.len[s], 0), c.max_pages * c.page_len), c.page_len);
    }
  }
  __syncthreads();
  verdict(sh.bad ? FV_PAGES_BAD : FV_PAGES_OK, status, nullptr);
  if (sh.bad || !here) return;
  const int rows = n * c.max_pages;
  for (int t0 = threadIdx.x; t0 < rows; t0 += kBatch * kPlanThreads) {
    int* at[kBatch];
    int page[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int t = min(t0 + u * kPlanThreads, rows - 1), i = t / c.max_pages, j = t - i * c.max_pages;
      at[u] = c.table + (size_t)place[i] + j;
      page[u] = *at[u];
      if (j >= held[i]) page[u] = -1;
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u)
      if (t0 + u * kPlanThreads < rows) {
        if (is_page(c, page[u])) atomicSub(&c.refs[page[u]], 1);
        *at[u] = -1;
      }
  }
  if (mine >= 0) c.len[mine] = 0;
}

__global__ __launch_bounds__(256) void free_apply_kernel(fv_pages c, const int* seqs,
                                                         const int* status) {
  if (*status != FV_PAGES_OK) return;
  const int s = seqs[blockIdx.x];
  int* row = c.table + (size_t)s * c.max_pages;
  const int pages = pages_of(min(max(c.len[s], 0), c.max_pages * c.page_len), c.page_len);
  __syncthreads();  // len is read before it is cleared
  for (int j = threadIdx.x; j < c.max_pages; j += 256) {
    const int p = row[j];
    if (j < pages && is_page(c, p)) atomicSub(&c.refs[p], 1);
    row[j] = -1;
  }
  if (threadIdx.x == 0) c.len[s] = 0;
}

// Workspace: [0] moves, [1] pages in use; A[i] <- B[i] are the moves and C[B[i]] = i.
// C is written for the pages that move and no others: an entry of it counts where B
// says that it is that page's.
__global__ __launch_bounds__(kPlanThreads) void compact_plan_kernel(fv_pages c, int* used,
                                                                    int* work, int list) {
  __shared__ PlanShared sh;
  int* A = work + kPagesHeader;
  int* B = A + list;
  int* C = B + list;
  const int w = threadIdx.x >> 6, J = scan_groups(c);
  int mine = 0;
  Holders h;
  for (int p0 = 0; p0 < c.n_pages; p0 += kPlanThreads * J) {
    const int first = p0 + w * 64 * J;
    uint64_t m[16];
    h.load(c, first, J);
    mine += pick_pages(c, h, first, J, m, [](int, int refs) { return refs > 0; });
  }
  if ((threadIdx.x & 63) == 0) sh.wave[0][w] = mine;
  __syncthreads();
  int u = 0;
  for (int i = 0; i < kPlanWaves; ++i) u += sh.wave[0][i];
  int holes = 0, movers = 0;
  for (int p0 = 0; p0 < c.n_pages; p0 += kPlanThreads * J) {
    const int first = p0 + w * 64 * J;
    uint64_t mh[16], mm[16];
    if (c.n_pages > kPlanThreads * J) h.load(c, first, J);
    const int nh = pick_pages(c, h, first, J, mh, [u](int p, int refs) { return p < u && refs <= 0; });
    const int nm = pick_pages(c, h, first, J, mm, [u](int p, int refs) { return p >= u && refs > 0; });
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
      sh.wave[0][w] = nh;
      sh.wave[1][w] = nm;
    }
    __syncthreads();
    int bh = 0, bm = 0, ah = 0, am = 0;
    for (int i = 0; i < kPlanWaves; ++i) {
      bh += i < w ? sh.wave[0][i] : 0;
      bm += i < w ? sh.wave[1][i] : 0;
      ah += sh.wave[0][i];
      am += sh.wave[1][i];
    }
    list_pages(mh, first, J, holes + bh, list, A);
    list_pages(mm, first, J, movers + bm, list, B);
    holes += ah;
    movers += am;
  }
  __syncthreads();  // the lists are complete; holes == movers
  for (int i = threadIdx.x; i < movers; i += kPlanThreads) {
    const int src = B[i], dst = A[i];
    C[src] = i;
    c.refs[dst] = c.refs[src];
    c.refs[src] = 0;
  }
  if (threadIdx.x == 0) {
    work[0] = movers;
    work[1] = u;
    *used = u;
  }
}

// Blocks (x, 0) rewrite the table; blocks (x, 1 + 2 l + kv) move pages of layer l, a
// page at a time, which a few hundred kilobytes in flight a CU keep at the rate of a
// copy: 672 MB in 132 us (5.1 TB/s).
template <bool STREAM>
__global__ __launch_bounds__(256) void compact_apply_kernel(fv_pages c, const int* work, int list,
                                                            int row16, Scales q) {
  const int moves = work[0], tid = threadIdx.x;
  const int* A = work + kPagesHeader;
  if (blockIdx.y == 0) {
    const int u = work[1];
    const int *B = A + list, *C = B + list;
    for (int s = blockIdx.x; s < c.max_seqs; s += gridDim.x) {
      int* row = c.table + (size_t)s * c.max_pages;
      const int pages = pages_of(min(max(c.len[s], 0), c.max_pages * c.page_len), c.page_len);
      for (int j = tid; j < pages; j += 256) {
        const int p = row[j];
        if (p < u || !is_page(c, p)) continue;
        const int i = C[p];
        if (i >= 0 && i < moves && B[i] == p) row[j] = A[i];  // a page that nobody holds stays
      }
    }
    return;
  }
  const int* B = A + list;
  const int l = (blockIdx.y - 1) >> 1;
  u32x4* pool = static_cast<u32x4*>((blockIdx.y - 1) & 1 ? c.v : c.k);
  const size_t base = (size_t)l * c.n_pages;
  const int page16 = c.n_kv_heads * c.page_len * row16;
  for (int i = blockIdx.x; i < moves; i += gridDim.x) {
    const u32x4* src = pool + (base + B[i]) * page16;
    u32x4* dst = pool + (base + A[i]) * page16;
    for (int x = tid; x < page16; x += 256) store_piece<STREAM>(dst + x, load_piece<STREAM>(src + x));
    if (q.k) {
      uint8_t* scales = (blockIdx.y - 1) & 1 ? q.v : q.k;
      const int all = c.n_kv_heads * (c.page_len / 16);
      for (int x = tid; x < all; x += 256) scales[(base + A[i]) * all + x] = scales[(base + B[i]) * all + x];
    }
  }
}

// Block (page, entry, layer): the rows of one page of one sequence, keys and values.
// A copy: 5.0 to 5.5 TB/s at 64 sequences of 300 to 816 tokens, 18 layers, heads of 64
// to 256.
template <bool STREAM>
__global__ __launch_bounds__(256) void gather_kernel(fv_pages c, const int* seqs, int n, int ld,
                                                     u32x4* k_out, u32x4* v_out, int row16) {
  const int l = blockIdx.z, pg = blockIdx.x, tid = threadIdx.x;
  const int wide = c.n_kv_heads * row16;  // 16-byte pieces of a token
  for (int i = blockIdx.y; i < n; i += gridDim.y) {
    const int s = seqs[i];
    if (s < 0 || s >= c.max_seqs) continue;
    const int rows = min(min(min(c.len[s], c.max_pages * c.page_len), ld) - pg * c.page_len, c.page_len);
    if (rows <= 0) continue;
    const int page = c.table[(size_t)s * c.max_pages + pg];
    if (!is_page(c, page)) continue;
    const size_t from = ((size_t)l * c.n_pages + page) * c.page_len * wide;
    const size_t to = (((size_t)l * n + i) * ld + (size_t)pg * c.page_len) * wide;
    const u32x4* k = static_cast<const u32x4*>(c.k) + from;
    const u32x4* v = static_cast<const u32x4*>(c.v) + from;
    for (int x = tid; x < rows * wide; x += 256) {
      const int r = x / wide, y = x - r * wide, h = y / row16;
      const int at = (h * c.page_len + r) * row16 + (y - h * row16);
      store_piece<STREAM>(k_out + to + x, load_piece<STREAM>(k + at));
      store_piece<STREAM>(v_out + to + x, load_piece<STREAM>(v + at));
    }
  }
}

int row_pieces(const fv_pages& c, const Scales& q = {}) {
  return c.head_dim * (q.k ? 1 : c.dtype == FV_BF16 ? 2 : 4) / 16;
}
// Keys and values of n tokens in every layer.
size_t token_bytes(const fv_pages& c, size_t n, const Scales& q = {}) {
  return 2 * n * c.n_layers * c.n_kv_heads * row_pieces(c, q) * 16;
}

template <typename T, int DH>
void rope_at(const RopeCall& r, hipStream_t s) {
  const int blocks = (int)(((int64_t)r.a.n + r.tokens - 1) / r.tokens);
  hipLaunchKernelGGL((rope_append_kernel<T, DH>), dim3(blocks), dim3(kRopeThreads), 0, s, r);
}

}  // namespace

// Angles are shared by a token's heads, so one token a workgroup loses nothing; more
// of them amortise the 64-bit exponentials once the chip is full, the more the less
// there is to move.  us with 1 | 2 | 8 tokens a workgroup, heads 8/1 of 256 (5 KB a
// token): 3.4 | 3.8 | 5.8 at 64 tokens, 10.7 | 8.9 | 9.8 at 4096, 77 | 61 | 57 at
// 32768; 8/2 of 64 (1.5 KB), 42 | 28 | 18 at 32768; 32/8 of 128 (12 KB), 30.9 | 29.9 |
// 30.5 at 8192, 130 | 135 | 150 at 32768.
// From 2^24 workgroups on the grid would have the 2^32 threads that no launch takes.
int rope_tokens(int n, size_t row) {
  int tokens = n >= 8192 && row < 6 << 10 ? kRopeTokens : 2;
  if (n < 2048 || (n >= 16384 && row >= 10 << 10)) tokens = 1;
  while (((int64_t)n + tokens - 1) / tokens * kRopeThreads >= (int64_t)1 << 32) tokens *= 2;
  return tokens;
}

template <typename T>
void launch_rope_append(const fv_rope_args& a, const fv_pages* c, hipStream_t s) {
  RopeCall r{};
  r.a = a;
  if (c) r.c = *c;
  r.has_cache = c != nullptr;
  r.log2_theta = log2((double)a.theta);
  const int heads = a.n_q_heads + (c || a.k_out ? a.n_kv_heads : 0) + (c ? a.n_kv_heads : 0);
  r.tokens = rope_tokens(a.n, (size_t)heads * a.head_dim * sizeof(T));
  switch (a.head_dim) {
    case 64: return rope_at<T, 64>(r, s);
    case 128: return rope_at<T, 128>(r, s);
    case 192: return rope_at<T, 192>(r, s);
    default: return rope_at<T, 256>(r, s);
  }
}
template void launch_rope_append<bf16_t>(const fv_rope_args&, const fv_pages*, hipStream_t);
template void launch_rope_append<float>(const fv_rope_args&, const fv_pages*, hipStream_t);

void launch_pages_grow(const fv_pages& c, const int* seqs, const int* add, int n, int* status,
                       int* work, hipStream_t s) {
  const int list = (int)pages_list(c);
  hipLaunchKernelGGL(grow_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, c, seqs, add, n, status,
                     work, list);
  if (n > kInline)
    hipLaunchKernelGGL(grow_apply_kernel, dim3(n), dim3(64), 0, s, c, seqs, add, work, list);
}

void launch_pages_fork(const fv_pages& c, const int* parents, const int* children, int n,
                       int* status, int* work, hipStream_t s, const Scales& q) {
  const int list = (int)pages_list(c);
  hipLaunchKernelGGL(fork_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, c, parents, children, n,
                     status, work, list);
  if (n)
    hipLaunchKernelGGL(fork_apply_kernel, dim3(n, 1 + 2 * c.n_layers), dim3(256), 0, s, c, parents,
                       children, work, list, row_pieces(c, q), q);
}

void launch_pages_free(const fv_pages& c, const int* seqs, int n, int* status, hipStream_t s) {
  hipLaunchKernelGGL(free_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, c, seqs, n, status);
  if (!free_inline(c, n))
    hipLaunchKernelGGL(free_apply_kernel, dim3(n), dim3(256), 0, s, c, seqs, status);
}

void launch_pages_compact(const fv_pages& c, int* used, int* work, hipStream_t s, const Scales& q) {
  const int list = (int)pages_list(c);
  hipLaunchKernelGGL(compact_plan_kernel, dim3(1), dim3(kPlanThreads), 0, s, c, used, work, list);
  const int most = c.n_pages / 2 > 1 ? c.n_pages / 2 : 1;  // no more pages than holes can move
  // at most half of the pages are read and as many written
  const bool stream = token_bytes(c, (size_t)c.n_pages * c.page_len, q) > kStreamBytes;
  hipLaunchKernelGGL(stream ? compact_apply_kernel<true> : compact_apply_kernel<false>,
                     dim3(most < 1024 ? most : 1024, 1 + 2 * c.n_layers), dim3(256), 0, s, c, work,
                     list, row_pieces(c, q), q);
}

void launch_pages_gather(const fv_pages& c, const int* seqs, int n, int ld, void* k_out,
                         void* v_out, hipStream_t s) {
  const int holds = c.max_pages * c.page_len;
  const int pages = ((ld < holds ? ld : holds) + c.page_len - 1) / c.page_len;
  const bool stream = 2 * token_bytes(c, (size_t)n * pages * c.page_len) > kStreamBytes;
  hipLaunchKernelGGL(stream ? gather_kernel<true> : gather_kernel<false>, dim3(pages, n < 65535 ? n : 65535, c.n_layers), dim3(256), 0, s,
                     c, seqs, n, ld, static_cast<u32x4*>(k_out), static_cast<u32x4*>(v_out),
                     row_pieces(c));
}

}  // namespace fv
