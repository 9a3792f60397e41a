// Internal declarations of the cache in 8 bits (append, read back, attention).
#pragma once

#include "fv_context.h"

#include <type_traits>

namespace fv {

// A block: 16 positions of a kv head, in slabs of 64 elements.  A kilobyte is a slab: of keys
// [16 positions][64], of values [4 runs of 4 positions][16][4][4 positions], so that the 16
// bytes at 16 l of a slab are what lane l of a wave multiplies (keys: row l / 4; values: the
// elements l % 16 + 16 c, c < 4, at four positions of run l / 16).
constexpr int kBlock = 16;
constexpr int kLeastScale = 10, kMostScale = 246;  // bytes: 2^-117 to 2^119

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__host__ __device__ __forceinline__ size_t block_of(int page, int n_kv, int head, int page_len, int block) {
  return ((size_t)page * n_kv + head) * (page_len / kBlock) + block;
}
__device__ __forceinline__ int scale_exponent(uint8_t b) {
  return min(max((int)b, kLeastScale), kMostScale) - 127;
}
// 2^e, -126 <= e <= 127
__device__ __forceinline__ float power_of(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Two e4m3 codes (the lower or the upper ones of w) times a power of two, as bf16 numbers:
// exact, 4 cycles a wave.
template <bool UP> __device__ __forceinline__ uint32_t to_bf16(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, UP));
}
// Eight codes as an MFMA operand.
__device__ __forceinline__ u32x4 to_bf16x8(uint32_t lo, uint32_t hi, float scale) {
  return u32x4{to_bf16<false>(lo, scale), to_bf16<true>(lo, scale), to_bf16<false>(hi, scale),
               to_bf16<true>(hi, scale)};
}

// x as PARTS numbers of bf16, one in each of `at`: its upper bits, and what they leave.
template <int PARTS>
__device__ __forceinline__ void split(float x, bf16_t (&at)[PARTS]) {
#pragma unroll
  for (int i = 0; i < PARTS - 1; ++i) {
    const uint32_t top = __float_as_uint(x) & 0xffff0000u;
    at[i] = (bf16_t)(top >> 16);
    x -= __uint_as_float(top);
  }
  at[PARTS - 1] = f32_to_bf16(x);
}
// Eight elements as operands.
__device__ __forceinline__ void query8(const bf16_t* p, u32x4 (&q)[1]) { q[0] = *reinterpret_cast<const u32x4*>(p); }
__device__ __forceinline__ void query8(const float* p, u32x4 (&q)[3]) {
  u16x8 w[3];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    bf16_t at[3];
    split<3>(p[e], at);
#pragma unroll
    for (int i = 0; i < 3; ++i) w[i][e] = at[i];
  }
#pragma unroll
  for (int i = 0; i < 3; ++i) q[i] = __builtin_bit_cast(u32x4, w[i]);
}

// Eight elements, rounded once.
__device__ __forceinline__ void store8(bf16_t* p, const float (&x)[8]) {
  u16x8 v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = f32_to_bf16(x[e]);
  *reinterpret_cast<u16x8*>(p) = v;
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  store4(p, x[0], x[1], x[2], x[3]);
  store4(p + 4, x[4], x[5], x[6], x[7]);
}

// Sizes and bookkeeping as those of pages of the dtype, for what reads nothing else.
inline fv_pages as_pages(const fv_quant_pages& c) {
  return fv_pages{c.dtype, c.n_layers, c.n_kv_heads, c.head_dim, c.page_len, c.n_pages, c.max_seqs,
                  c.max_pages, c.k, c.v, c.table, c.len, c.refs};
}

inline Scales scales_of(const fv_quant_pages& c) {
  return Scales{static_cast<uint8_t*>(c.k_scale), static_cast<uint8_t*>(c.v_scale)};
}

// The launches take validated arguments.
template <typename T>
void launch_quant_append(const fv_rope_args& a, const fv_quant_pages& c, hipStream_t s);
// Tokens of a workgroup of the append, and workgroups that share the same ones.
struct QuantShare {
  int tokens, parts;
};
QuantShare quant_share(int n, int n_kv_heads);
template <typename T>
void launch_quant_gather(const fv_quant_pages& c, const int* seqs, int n, int ld, void* k_out, void* v_out,
                         hipStream_t s);
PagedPlan plan_quant(int n, int n_q_heads, int n_kv_heads, int head_dim, int max_keys, bool bf16);
template <typename T>
void launch_quant_paged(const fv_paged_args& a, const fv_quant_pages& c, const PagedPlan& p, hipStream_t s);

// How an attention of several tokens a sequence is laid out: row tiles of `rows` (token, head)
// pairs, keys in n_chunks chunks of `chunk`.
struct PartPlan {
  int rows, chunk, n_chunks;
  size_t work_bytes;
};
PartPlan plan_part(const fv_part_args& a, const fv_quant_pages& c, int max_keys);
template <typename T>
void launch_quant_part(const fv_part_args& a, const fv_quant_pages& c, const PartPlan& p, hipStream_t s);

}  // namespace fv
