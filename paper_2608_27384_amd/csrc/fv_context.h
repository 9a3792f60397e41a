// Internal declarations of the observation context's operators (rotary append,
// prompt attention, paged attention, the cache's upkeep).
#pragma once

#include "fv_internal.h"

namespace fv {

constexpr float kLog2e = 1.4426950408889634f;

// First of the `group` kv heads' rows: the pools are [layer][page][kv head][row][dh].
__host__ __device__ __forceinline__ size_t page_row(int page, int n_kv, int head, int page_len) {
  return ((size_t)page * n_kv + head) * page_len;
}

// Data that no cache holds until it is used again (the last level has 256 MiB) is moved past
// them: above twice that size a call's loads and stores are marked as streaming.  Paged
// attention, 192 rows of 1 to 8191 keys, 32/8 heads of 128 (3.2 GB), 574 us, streaming 526;
// 64 of 500 to 3001, fp32, 8/1 of 256 (0.2 GB), called again and again, 65 and 79.  Gathering
// 64 sequences of 300 to 816 in 18 layers (1.3 GB moved) 243 and 228.
constexpr size_t kStreamBytes = (size_t)512 << 20;
template <bool STREAM, typename V> __device__ __forceinline__ V load_piece(const V* p) {
  if constexpr (STREAM) return __builtin_nontemporal_load(p);
  return *p;
}
template <bool STREAM, typename V> __device__ __forceinline__ void store_piece(V* p, V x) {
  if constexpr (STREAM)
    __builtin_nontemporal_store(x, p);
  else
    *p = x;
}

// The angles of a thread of the workgroup: pair i turns by pos * theta^(-2i/DH), taken in turns
// (over 2 pi) in 64 bits, of which only the fraction is rounded to fp32.
template <int DH> struct RopeAngles {
  static constexpr int HALF = DH / 2;
  const int* pos;  // of the pair's axis
  double turns;
  int i, at, step;  // the pair, the first token of the thread, tokens a pass
  // threads: of the workgroup, at least HALF
  __device__ __forceinline__ RopeAngles(const fv_rope_args& a, double log2_theta, int threads) {
    step = threads / HALF;
    i = threadIdx.x % HALF;
    at = threadIdx.x < step * HALF ? threadIdx.x / HALF : 1 << 30;
    int axis = 0, end = a.sections[0];
    while (axis < a.n_axes - 1 && i >= end) end += a.sections[++axis];
    pos = a.pos + (size_t)axis * a.n;
    turns = exp2(-log2_theta * (2.0 * i / DH)) * 0.15915494309189535;
  }
  // Cosine and sine of x turns, |x| <= 1/2, as 64 bits give them: off by no more than fp32's own
  // rounding, where the fp32 function of the rounded angle is off by several times that.  What is
  // quantised lands on the other side of a tie that much less often.  Their series within an eighth
  // of a turn, whose first terms left out are below 2^-33.
  static __device__ __forceinline__ void fine(double x, float& c, float& s) {
    const double quarter = rint(4 * x), t = (x - 0.25 * quarter) * 6.283185307179586, z = t * t;
    const float a = (float)(t * (1 + z * (-1. / 6 + z * (1. / 120 + z * (-1. / 5040 + z * (1. / 362880 + z * (-1. / 39916800)))))));
    const float b = (float)(1 + z * (-1. / 2 + z * (1. / 24 + z * (-1. / 720 + z * (1. / 40320 + z * (-1. / 3628800))))));
    const int n = (int)quarter;
    c = n & 1 ? a : b;
    s = n & 1 ? b : a;
    if ((n + 1) & 2) c = -c;
    if (n & 2) s = -s;
  }
  // Of the tokens from `from` to `to` behind t0.
  template <bool FINE = false>
  __device__ __forceinline__ void form(int t0, int from, int to, float (*cs)[HALF], float (*sn)[HALF]) const {
    for (int t = from + at; t < to; t += step) {
      double x = (double)pos[t0 + t] * turns;
      x -= rint(x);
      float s, c;
      if (FINE)
        fine(x, c, s);
      else
        sincospif(2.0f * (float)x, &s, &c);
      cs[t][i] = c;
      sn[t][i] = s;
    }
  }
};

constexpr int kRopeThreads = 256;
constexpr int kRopeTokens = 8;  // most tokens of a workgroup
// Tokens of a workgroup that rotates n tokens of `row` bytes to be rotated or stored.
int rope_tokens(int n, size_t row);

// The launches take validated arguments.
template <typename T>
void launch_rope_append(const fv_rope_args& a, const fv_pages* c, hipStream_t s);
// The kernel of a prompt attention: few rows, halved keys or whole tiles.
enum { kFew, kHalves, kTiles };
int prompt_form(const fv_prompt_args& a);
template <typename T>
void launch_prompt(const fv_prompt_args& a, hipStream_t s);

// How a paged attention is laid out for up to `keys` keys: chunks of `chunk`, at most n_chunks
// a sequence, each with one workgroup per kv head and tile of 16 query heads.
struct PagedPlan {
  int keys, chunk, n_chunks;
  size_t work_bytes;  // partial outputs and softmax statistics; 0 with one chunk
};
PagedPlan plan_paged(int n, int n_q_heads, int n_kv_heads, int head_dim, int max_keys, bool bf16);
template <typename T>
void launch_paged(const fv_paged_args& a, const fv_pages& c, const PagedPlan& p, hipStream_t s);

// int32 values of the upkeep's workspace: a header, then three lists.
constexpr int kPagesHeader = 64;
inline size_t pages_list(const fv_pages& c) {
  return (size_t)(c.n_pages > c.max_seqs ? c.n_pages : c.max_seqs);
}
inline size_t pages_work_ints(const fv_pages& c) { return kPagesHeader + 3 * pages_list(c); }
// The scales of a cache in 8 bits, whose pages then hold a byte an element; none otherwise.
struct Scales {
  uint8_t *k = nullptr, *v = nullptr;
};
void launch_pages_grow(const fv_pages& c, const int* seqs, const int* add, int n, int* status,
                       int* work, hipStream_t s);
void launch_pages_fork(const fv_pages& c, const int* parents, const int* children, int n,
                       int* status, int* work, hipStream_t s, const Scales& q = {});
void launch_pages_free(const fv_pages& c, const int* seqs, int n, int* status, hipStream_t s);
void launch_pages_compact(const fv_pages& c, int* used, int* work, hipStream_t s, const Scales& q = {});
void launch_pages_gather(const fv_pages& c, const int* seqs, int n, int ld, void* k_out,
                         void* v_out, hipStream_t s);

}  // namespace fv
