// What the attentions over pages share, of one new token a sequence with pages of the dtype
// (fv_paged.hip) and in 8 bits (fv_quant_attn.hip), of several (fv_quant_part.hip): the call,
// and the join of its chunks.
#pragma once

#include "fv_context.h"

namespace fv {

constexpr int kPagedWaves = 4;

// Largest of the lanes l, l ^ 16, l ^ 32, l ^ 48.
__device__ __forceinline__ float max_xor16_32(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const float y = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(y), __float_as_uint(y), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

struct PagedCall {
  const void *q, *k, *v;  // the pools of the layer
  const uint8_t *k_scale, *v_scale;  // its scales, in 8 bits
  void* out;
  const int *seqs, *table, *len;
  const int* cu;  // of several rows an entry (fv_quant_part.hip): their offsets; else NULL
  int n_entries;
  float* part;  // [n][n_chunks][heads][DH] sums, then [n][n_chunks][heads][2] maximum and sum
  float* stat;
  int ldq, ldo, n, heads, n_kv, group, q_tiles, page_len, n_pages, max_seqs, max_pages;
  uint32_t per_page;  // 2^31 over a page's runs of 16 rows, rounded up
  int chunk, n_chunks;
  float scale;  // of the scores, in log2 units
};

// Sums that say why a row's chunk has none: it saw no key; its entry names no sequence.
constexpr float kNoKey = -1.f, kNoEntry = -2.f;

// Chunks of a sequence that hold keys.  The last workgroup takes what lies past
// the planned bound, should a sequence be longer.
__device__ __forceinline__ int chunks_of(int len, int chunk, int n_chunks) {
  const int c = (len + chunk - 1) / chunk;
  return c < n_chunks ? c : n_chunks;
}
__device__ __forceinline__ int length_of(const PagedCall& a, int s) {
  return min(max(a.len[s], 0), a.max_pages * a.page_len);
}

// The call of validated arguments, without its pools.
PagedCall paged_call(const fv_paged_args& x, const fv_pages& c, const PagedPlan& p);
// The kernel that joins a call's chunks, if it has several.
template <typename T>
void launch_paged_join(const PagedCall& a, int head_dim, hipStream_t s);

}  // namespace fv
