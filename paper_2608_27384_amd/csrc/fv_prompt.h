// What the attentions over packed rows share, keys and values dense (fv_prompt.hip) or in pages
// of 8 bits (fv_quant_part.hip): 32x32 products, loads to LDS, the softmax of 32 keys, and which
// entry a row tile belongs to.
#pragma once

#include "fv_context.h"

namespace fv {

// A row's reference stays until a score is this much (in log2) above it: the
// probabilities are then at most 2^8, the same to every rounding, and the output
// is rescaled a few times instead of with every new maximum.
constexpr float kSlack = 8.0f;

typedef short s16x4 __attribute__((ext_vector_type(4)));

// In a group of 16 lanes, lane i gives the address of 4 elements of row i / 4
// (columns 4 (i % 4) on) of a 4x16 block and gets column i, rows 0..3.
__device__ __forceinline__ u32x2 read_transposed(const unsigned char* p) {
  const s16x4 r = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) s16x4*)(p));
  return __builtin_bit_cast(u32x2, r);
}

// A direct-to-LDS load (see lds_dma16) that the compiler does not know of: it waits
// for all those it knows of before a transposing read, the next tile's among them.
// Whoever reads the data waits for the loads itself.  The place in LDS goes by m0, an
// operand, so that the compiler knows what that holds.
__device__ __forceinline__ u32x4 dma_source(const void* base) {
  const uint64_t p = reinterpret_cast<uint64_t>(base);
  return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)p),
               (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(p >> 32)), 0x7fffffffu, 0x00020000u};
}
__device__ __forceinline__ uint32_t lds_address(const unsigned char* p) {
  return (uint32_t)reinterpret_cast<uintptr_t>((const __attribute__((address_space(3))) unsigned char*)p);
}
__device__ __forceinline__ void dma16(u32x4 src, uint32_t lds, int off) {
  asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"{m0}"(
                   __builtin_amdgcn_readfirstlane((int)lds)),
               "v"(off), "s"(src)
               : "memory");
}
__device__ __forceinline__ void dma16(u32x4 src, const unsigned char* lds, int off) {
  dma16(src, lds_address(lds), off);
}

// 32x32 products over two 16-byte pieces a row (one of each lane half).
__device__ __forceinline__ f32x16 mma32(u32x4 x, u32x4 y, f32x16 c, bf16_t) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x),
                                                 __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma32(u32x4 x, u32x4 y, f32x16 c, float) {
#pragma unroll
  for (int e = 0; e < 4; ++e)
    c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(x[e]), __uint_as_float(y[e]), c, 0, 0, 0);
  return c;
}

__device__ __forceinline__ float other_half_max(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float other_half_sum(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// Values at the edge, where a wave's rows differ in what they see.  A weight of
// zero does not silence a value that is not finite, so such values are taken out
// of the product there and added afterwards to the sums of the rows that see them
// (add_unruly), which makes the infinity or NaN that the formula has.
// odd(x): high bits for bf16 pairs (or an fp32 value) whose exponent is all ones.
__device__ __forceinline__ uint32_t odd(uint32_t x, bf16_t) { return (x & 0x7f807f80u) + 0x00800080u; }
__device__ __forceinline__ uint32_t odd(uint32_t x, float) { return (x & 0x7f800000u) + 0x00800000u; }
__device__ __forceinline__ bool any_odd(uint32_t odds, bf16_t) { return __any(odds & 0x80008000u); }
__device__ __forceinline__ bool any_odd(uint32_t odds, float) { return __any(odds >> 31); }
__device__ __forceinline__ uint32_t even(uint32_t x, bf16_t t) {  // without the odd ones
  const uint32_t b = odd(x, t) & 0x80008000u;
  return x & ~(b | (b - (b >> 15)));
}
__device__ __forceinline__ uint32_t even(uint32_t x, float t) { return odd(x, t) >> 31 ? 0u : x; }
// Operands of V.
template <typename T> __device__ __forceinline__ uint32_t odds_of(u32x4 v, T t) {
  return odd(v[0], t) | odd(v[1], t) | odd(v[2], t) | odd(v[3], t);
}
template <typename T> __device__ __forceinline__ uint32_t odds_of(float v, T t) { return odd(__float_as_uint(v), t); }
template <typename T> __device__ __forceinline__ u32x4 even_of(u32x4 v, T t) {
  return u32x4{even(v[0], t), even(v[1], t), even(v[2], t), even(v[3], t)};
}
template <typename T> __device__ __forceinline__ float even_of(float v, T t) {
  return __uint_as_float(even(__float_as_uint(v), t));
}
__device__ __forceinline__ f32x16 zeros16() {
  f32x16 z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.f;
  return z;
}

__device__ __forceinline__ int clamped(const int* cu, int s, int n) { return min(max(cu[s], 0), n); }

// The prompt that row tile `slot` belongs to.  Prompt s has the slots from
// g(s) = floor(row0(s) / R) + s on, row0(s) being its first row: enough for its
// ceil(rows / R) tiles, with at most one to spare, and known without a sum over
// the prompts before it.  64 candidates at a time.
template <int R, typename Call>
__device__ __forceinline__ int prompt_of(const Call& a, int slot, int* first) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = a.n_seqs;
  while (n > 1) {
    const int step = (n + 63) / 64, i = lane * step;
    bool le = false;
    if (i < n)
      le = (long long)clamped(a.cu_q, lo + i, a.n_q) * a.group / R + lo + i <= slot;
    const int c = max(1, (int)__popcll(__ballot(le)));
    lo += (c - 1) * step;
    n = min(step, n - (c - 1) * step);
  }
  lo = __builtin_amdgcn_readfirstlane(lo);
  *first = (int)((long long)clamped(a.cu_q, lo, a.n_q) * a.group / R) + lo;
  return lo;
}

// O^T += V^T P^T for operand c of V, of the probabilities p (pf: as bf16 operands).
__device__ __forceinline__ f32x16 product(u32x4 v, const f32x16&, const u32x4 (&pf)[2], int c, f32x16 o) {
  return mma32(v, pf[c], o, bf16_t{});
}
__device__ __forceinline__ f32x16 product(float v, const f32x16& p, const u32x4 (&)[2], int c, f32x16 o) {
  return __builtin_amdgcn_mfma_f32_32x32x2f32(v, p[c], o, 0, 0, 0);
}
// bf16 operands of 32 probabilities, each rounded once (2^-8 at most), as the result is
// afterwards; their sum is of the unrounded ones.  The error against 64 bits is 1.2 to 1.4
// times that of exact probabilities.  Operands of 16 bits, in two parts, make half as
// many products again, which here nothing hides: us with one part and with two, one prompt
// of 560, heads 8/1 of 256, 15.6 and 17.0; 64 of 300 to 816 196 and 258; one of 28672 2634
// and 3770; 7 of 1 to 4111, 32/8 of 128, 599 and 857.
__device__ __forceinline__ void as_operands(const f32x16& p, u32x4 (&pf)[2]) {
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    u16x8 w;
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = f32_to_bf16(p[8 * c + e]);
    pf[c] = __builtin_bit_cast(u32x4, w);
  }
}
// Scores past what the lane's row sees (keys from lim on) to -inf.
__device__ __forceinline__ void hide(f32x16& sc, int key0, int lh, int lim) {
#pragma unroll
  for (int r = 0; r < 16; ++r)
    if (key0 + 8 * (r >> 2) + 4 * lh + (r & 3) >= lim) sc[r] = -INFINITY;
}
__device__ __forceinline__ float highest(const f32x16& sc) {
  float top = sc[0];
#pragma unroll
  for (int r = 1; r < 16; ++r) top = fmaxf(top, sc[r]);
  return other_half_max(top);
}
// Scores of 32 keys to probabilities (pf: as bf16 operands), with the row's
// reference m and sum l; calls rescale(f) where the reference moves, and tick(r)
// after the r-th of 16 probabilities.
template <typename T, typename Rescale, typename Tick>
__device__ __forceinline__ void softmax(f32x16& sc, bool edge, int key0, int lh, int lim, float scale,
                                        float& m, float& l, u32x4 (&pf)[2], Rescale rescale, Tick tick) {
  if (edge) hide(sc, key0, lh, lim);
  const float top = highest(sc) * scale;
  const bool raise = top > m + kSlack;
  if (__any(raise)) {
    const float now = raise ? top : m;  // its own scores alone move a row's reference
    const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - now);
    m = now;
    l *= f;
    rescale(f);
  }
  const float ref = m == -INFINITY ? 0.f : -m;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    sc[r] = __builtin_amdgcn_exp2f(fmaf(sc[r], scale, ref));
    l += sc[r];
    tick(r);
  }
  if constexpr (sizeof(T) == 2) as_operands(sc, pf);
}
// The same without a maximum on the usual path: probabilities against the row's
// reference as it is, whose sum says whether it will do.  A row whose sum (of
// either half's keys) is past kLimit, or none, takes its maximum as the reference and
// everything again.  `minus`: minus the reference, kNoRef for a row without one,
// against which any visible score is infinite and a hidden one still nothing.
// Leaves the scores as they are, which takes 16 more registers.  With heads of 128 the
// vector unit is busy 58 % of the time and the matrix unit 62 %, and a wave uses one after
// the other: 16 maxima less, and the kept load offsets, brought eight prompts of 2000
// tokens, every key seen, heads 32/8 of 128, from 519 to 485 us (1.08 PFLOP/s).
constexpr float kLimit = 1024.0f;  // sums stay within 2^10 of the largest value's size
constexpr float kNoRef = 3.402823466e38f;
template <typename Rescale>
__device__ __forceinline__ void softmax_by_sum(f32x16& sc, bool edge, int key0, int lh, int lim,
                                               float scale, float& minus, float& l, u32x4 (&pf)[2],
                                               Rescale rescale) {
  if (edge) hide(sc, key0, lh, lim);
  f32x16 p;
  auto weigh = [&] {
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      p[r] = __builtin_amdgcn_exp2f(fmaf(sc[r], scale, minus));
      sum += p[r];
    }
    return sum;
  };
  float sum = weigh();
  if (__builtin_expect(__any(!(sum <= kLimit)), 0)) {
    const bool raise = !(other_half_max(sum <= kLimit ? 0.f : 1.f) == 0.f);
    const float top = highest(sc) * scale;
    // NaN scores have no maximum: the reference stays, and the sum is NaN
    const float now = raise && top > -INFINITY ? -top : minus;
    const float f = minus == kNoRef ? (now == kNoRef ? 1.f : 0.f) : __builtin_amdgcn_exp2f(now - minus);
    minus = now;
    l *= f;
    rescale(f);
    sum = weigh();
  }
  l += sum;
  as_operands(p, pf);
}
// No key seen: zeros; keys that all score -inf: 0/0, as the formula has it.
__device__ __forceinline__ float inverse(float l, int lim) {
  return lim > 0 ? 1.0f / other_half_sum(l) : 0.f;
}

}  // namespace fv
