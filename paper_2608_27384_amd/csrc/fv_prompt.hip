// Attention over whole prompts: packed sequences of different lengths, grouped
// heads, causal or not.
//
// The query rows of one (prompt, kv head) are its (token, head) pairs, token
// major, so the heads that share a kv head share its key and value tiles and the
// causal edge of a workgroup spans few tokens.  A workgroup takes 32 rows a wave
// and walks the keys once, with the running maximum and sum of a softmax.
// Key and value tiles go from memory straight into LDS, one tile ahead.
//
// Per 32 keys: S^T = K Q^T by 32x32 MFMA, so a lane holds 16 scores of one query
// and the row maximum is 15 register maxima and one exchange of lane halves; the
// probabilities are, without data movement, the operand of O^T += V^T P^T, and
// the row's rescaling factor is the lane's own.  V^T comes out of the row-major
// LDS tile by transposing reads.
#include "fv_context.h"

#include <type_traits>

namespace fv {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
// A row's reference stays until a score is this much (in log2) above it: the
// probabilities are then at most 2^8, the same to every rounding, and the output
// is rescaled a few times instead of with every new maximum.
constexpr float kSlack = 8.0f;

struct PromptCall {
  const void *q, *k, *v;
  void* out;
  const int *cu_q, *cu_k;
  int ldq, ldk, ldv, ldo, n_seqs, n_q, n_k, n_kv, group, causal, n_slots;
  float scale;  // of the scores, in log2 units
};

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
__device__ __forceinline__ void dma16(u32x4 src, const unsigned char* lds, int off) {
  const uint32_t to = (uint32_t)reinterpret_cast<uintptr_t>(
      (const __attribute__((address_space(3))) unsigned char*)lds);
  asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"{m0}"(
                   __builtin_amdgcn_readfirstlane((int)to)),
               "v"(off), "s"(src)
               : "memory");
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

// 16-byte piece c of LDS row r is stored at c ^ swizzle(r): the 16 rows that a
// read of K touches at one piece, and the 4 rows by 64 bytes that a transposing
// read of V touches, fall on different banks.
template <typename T, int DH> __device__ __forceinline__ int swizzle(int r) {
  if (sizeof(T) == 4) return ((r >> 2) & 1) << 3 | (r & 3) << 1 | ((r >> 3) & 1);
  if (DH % 128 == 0) return (r & 3) << 2 | ((r >> 2) & 3);
  return ((r >> 1) & 1) << 2 | ((r >> 2) & 3);  // rows of 8 or 24 pieces: within 8
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
// Adds the odd values of the keys [from, to) (rows of v, ldv apart) to the staged
// results of a wave's 32 rows that see them; lane l holds the view of row l % 32,
// and at(row, d) is the place of a result.
template <int DH, typename T, typename At>
__device__ __forceinline__ void add_unruly(const T* v, int ldv, int from, int to, int lim, At at) {
  for (int key = from; key < to; ++key)
    for (int d = threadIdx.x & 63; d < DH; d += 64) {
      const float x = to_f32(v[(size_t)key * ldv + d]);
      const bool skip = fabsf(x) < INFINITY;
      if (!__any(!skip)) continue;
      for (int r = 0; r < 32; ++r) {
        const bool sees = key < __shfl(lim, r);
        if (sees && !skip) {
          auto* p = at(r, d);
          typedef typename std::remove_pointer<decltype(p)>::type O;
          *p = from_f32<O>(to_f32(*p) + x);
        }
      }
    }
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
template <int R>
__device__ __forceinline__ int prompt_of(const PromptCall& a, int slot, int* first) {
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
// Leaves the scores as they are, which takes 16 more registers: for head dims up to
// 192.  At 128 the vector unit is busy 58 % of the time and the matrix unit 62 %, and a
// wave uses one after the other: 16 maxima less, and the kept load offsets, brought eight
// prompts of 2000 tokens, every key seen, heads 32/8 of 128, from 519 to 485 us (1.08
// PFLOP/s).
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

// Row and byte in it of a lane's 16 bytes in the n-th kilobyte of a staged tile.
// Where a kilobyte is whole rows, both are the lane's of the first one moved by
// constants (the swizzle is linear over exclusive or).
template <typename T, int DH> struct Slots {
  static constexpr int PIECES = DH * (int)sizeof(T) / 16, PER = 64 / PIECES;
  static constexpr bool WHOLE = PIECES <= 64 && (PIECES & (PIECES - 1)) == 0;
  int lane, row0, byte0;
  __device__ __forceinline__ explicit Slots(int l) : lane(l) {
    row0 = l / PIECES;
    byte0 = ((l % PIECES) ^ swizzle<T, DH>(row0)) << 4;
  }
  __device__ __forceinline__ void find(int n, int& row, int& byte) const {
    if constexpr (WHOLE) {
      row = PER * n + row0;
      byte = byte0 ^ (swizzle<T, DH>(PER * n) << 4);
    } else {
      const int u = 64 * n + lane;
      row = u / PIECES;
      byte = ((u % PIECES) ^ swizzle<T, DH>(row)) << 4;
    }
  }
};

// What a workgroup of R rows knows of its prompt.
template <typename T, int DH, int R>
struct Rows {
  static constexpr int E = (int)sizeof(T);
  static constexpr int NK = DH * E / 32;  // K operands of 32 keys
  static constexpr int ND = DH / 32;      // 32-row tiles of O^T

  const PromptCall& a;
  int lane, wave, l32, lh, kh, q0, k0, nk, rows, row0, diff;

  __device__ __forceinline__ explicit Rows(const PromptCall& call) : a(call) {
    lane = threadIdx.x & 63;
    wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    l32 = lane & 31;
    lh = lane >> 5;
    // within a causal prompt the heaviest tiles, its last ones, go first; the prompts go in
    // the reverse of the caller's order
    const int slot = a.n_slots - 1 - (int)(blockIdx.x / a.n_kv);
    kh = blockIdx.x % a.n_kv;
    int first;
    const int s = prompt_of<R>(a, slot, &first);
    q0 = clamped(a.cu_q, s, a.n_q);
    k0 = clamped(a.cu_k, s, a.n_k);
    const int nq = max(0, clamped(a.cu_q, s + 1, a.n_q) - q0);
    nk = max(0, clamped(a.cu_k, s + 1, a.n_k) - k0);
    rows = nq * a.group;
    row0 = (slot - first) * R;
    diff = nk - nq + 1;
  }
  // False: a spare slot, or one that no prompt has (offsets that do not ascend from 0).
  __device__ __forceinline__ bool any() const { return row0 >= 0 && row0 < rows; }
  // A row sees the keys [0, limit), which do not fall from one row to the next.
  __device__ __forceinline__ int limit(int row) const {
    return a.causal ? min(max(diff + min(row, rows - 1) / a.group, 0), nk) : nk;
  }
  // The lane's query of the 32 rows from r0 on, as products' operands, and its
  // place in the output.  A lane wants a row of its own, which as loads is 32 bytes
  // of each of 32 rows at a time (4 times the cycles of whole rows): the rows go
  // whole to `lds` (32 of them) and from there to the lanes, shared by `waves` waves.
  template <bool KNOWN>  // loads that the compiler knows of
  __device__ __forceinline__ long long query(int r0, u32x4 (&qf)[NK], unsigned char* lds, int waves) const {
    constexpr int ROW = DH * E, SW = E == 4 || DH % 128 == 0 ? 16 : 8, N = 32 * ROW / 1024;
    const int row = min(r0 + l32, rows - 1);
    const int tok = row / a.group, head = kh * a.group + row - tok * a.group;
    const int tok0 = __builtin_amdgcn_readfirstlane(tok);
    const T* from = static_cast<const T*>(a.q) + (size_t)(q0 + tok0) * a.ldq;
    const int off = ((tok - tok0) * a.ldq + head * DH) * E;
    const Slots<T, DH> at(lane);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // what was there has been read
#pragma unroll
    for (int n = 0; n < N; ++n) {
      if (waves > 1 && n % waves != wave) continue;
      int r, byte;
      at.find(n, r, byte);
      if constexpr (KNOWN)
        lds_dma16(lds_source(from), lds + 1024 * n, __shfl(off, r) + byte, 0);
      else
        dma16(dma_source(from), lds + 1024 * n, __shfl(off, r) + byte);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (waves > 1) {
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    }
    const int base = l32 * ROW + ((lh ^ swizzle<T, DH>(l32)) << 4);
#pragma unroll
    for (int p = 0; p < NK; ++p)
      qf[p] = *reinterpret_cast<const u32x4*>(lds + (base ^ ((2 * p & (SW - 1)) << 4)) + 2 * p / SW * SW * 16);
    return (long long)(q0 + tok) * a.ldo + head * DH;
  }
};

// The walk over the keys with tiles staged in LDS, 128 rows a workgroup.  KG 1:
// four waves of 32 rows, tiles of 32 keys.  KG 2 (bf16): eight waves, tiles of 64
// keys, of which half the waves take the first 32 and half the others; they join
// at the end.  A workgroup's walk then has half the steps, for where there are not
// enough of them to fill the chip.
template <typename T, int DH, int KG>
struct Walk : Rows<T, DH, 128> {
  typedef Rows<T, DH, 128> Base;
  using Base::a, Base::lane, Base::wave, Base::l32, Base::lh, Base::kh, Base::k0, Base::nk, Base::rows,
      Base::row0, Base::limit, Base::E, Base::NK, Base::ND;
  static constexpr int R = 128, WAVES = 4 * KG;
  static constexpr int KT = 32 * KG;                           // keys of a tile
  static constexpr int ROW = DH * E, PIECES = ROW / 16;
  static constexpr int BYTES = KT * ROW;                       // of a K tile, and of a V tile
  static constexpr int SW = E == 4 || DH % 128 == 0 ? 16 : 8;  // pieces that a swizzle permutes
  static constexpr int NI = BYTES / 1024 / WAVES;              // direct loads of a wave per tensor and tile
  static constexpr int PV = E == 2 ? 2 : 16;                   // V operands of 32 keys and 32 elements
  static_assert(NI * 1024 * WAVES == BYTES && 32 * WAVES * ROW <= 4 * BYTES, "tile split");
  static_assert(KG == 1 || (KG == 2 && 4 * 32 * DH * 4 <= 4 * BYTES), "join");
  typedef typename std::conditional<E == 2, u32x4, float>::type vop;

  unsigned char* ring;  // two stages of K and V
  int wrow, half, tiles, kaddr, vaddr;

  __device__ __forceinline__ Walk(const PromptCall& call, unsigned char* lds) : Base(call), ring(lds) {
    half = wave / 4;
    wrow = row0 + 32 * (wave % 4);
    tiles = (limit(row0 + R - 1) + KT - 1) / KT;
    // LDS addresses of the operands: one register each for K and V and a constant
    // exclusive or (the swizzle), so that they cost an instruction and no registers.
    kaddr = (32 * half + l32) * ROW + ((lh ^ swizzle<T, DH>(l32)) << 4);
    const int i16 = lane & 15, r = 4 * lh + (i16 >> 2);
    vaddr = E == 2 ? BYTES + (32 * half + r) * ROW +
                         (((2 * ((lane >> 4) & 1) + ((i16 >> 1) & 1)) ^ swizzle<T, DH>(r)) << 4) +
                         (i16 & 1) * 8
                   : BYTES + 4 * lh * ROW + (((l32 >> 2) ^ (lh << 3)) << 4) + (l32 & 3) * 4;
  }
  // Direct loads of key tile kt: slot u, 16 bytes, is piece u % PIECES of row u / PIECES.
  // offs: the offsets of a whole tile (Offsets), which the narrower heads have the
  // registers to keep, and whose vector instructions they have few products to hide behind.
  static constexpr bool KEEP = E == 2 && DH <= 128;
  struct Offsets {
    int k[KEEP ? NI : 1], v[KEEP ? NI : 1];
  };
  __device__ __forceinline__ void find(Offsets& offs) const {
    if constexpr (KEEP) {
      const Slots<T, DH> at(lane);
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        int row, byte;
        at.find(NI * wave + i, row, byte);
        offs.k[i] = __umul24(row, a.ldk * E) + byte;
        offs.v[i] = __umul24(row, a.ldv * E) + byte;
      }
    }
  }
  __device__ __forceinline__ void issue(int kt, int stage, const Offsets& offs) const {
    unsigned char* to = ring + stage * 2 * BYTES + wave * NI * 1024;
    const u32x4 ks = dma_source(static_cast<const T*>(a.k) + (size_t)(k0 + kt * KT) * a.ldk + kh * DH);
    const u32x4 vs = dma_source(static_cast<const T*>(a.v) + (size_t)(k0 + kt * KT) * a.ldv + kh * DH);
    const int most = nk - 1 - kt * KT;  // rows past the prompt's last repeat it
    if constexpr (KEEP) {
      if (most >= KT - 1) {
#pragma unroll
        for (int i = 0; i < NI; ++i) {
          dma16(ks, to + 1024 * i, offs.k[i]);
          dma16(vs, to + BYTES + 1024 * i, offs.v[i]);
        }
        return;
      }
    }
    int mine = lane;
    asm volatile("" : "+v"(mine));  // not 2 NI offsets kept over the loop
    const Slots<T, DH> at(mine);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      int row, byte;
      at.find(NI * wave + i, row, byte);
      row = min(row, most);
      dma16(ks, to + 1024 * i, __umul24(row, a.ldk * E) + byte);
      dma16(vs, to + BYTES + 1024 * i, __umul24(row, a.ldv * E) + byte);
    }
  }
  // Every wave's loads have landed, every wave's reads are done.
  __device__ __forceinline__ void meet() const {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  }
  __device__ __forceinline__ u32x4 kread(int base, int p) const {
    return *reinterpret_cast<const u32x4*>(ring + (base ^ ((2 * p & (SW - 1)) << 4)) +
                                           2 * p / SW * SW * 16);
  }
  // Operand c of V for the elements from 32 d on of the head: 16 keys from 16 c on
  // (bf16), the keys of score register c (fp32).
  __device__ __forceinline__ vop vread(int base, int d, int c) const {
    if constexpr (E == 2) {
      const unsigned char* p = ring + 16 * c * ROW + 4 * d / SW * SW * 16;
      const int x = base ^ ((4 * d & (SW - 1)) << 4);
      const u32x2 lo = read_transposed(p + x), hi = read_transposed(p + (x ^ 32) + 8 * ROW);
      return u32x4{lo[0], lo[1], hi[0], hi[1]};
    } else {
      const int j = c >> 2, r = c & 3;
      const int x = base ^ ((8 * d & 15) << 4) ^ (r << 5) ^ ((j & 1) << 4);
      return *reinterpret_cast<const float*>(ring + x + (8 * j + r) * ROW + 8 * d / 16 * 256);
    }
  }
  // stats: LDS for the maximum and sum of the waves that give theirs to others.
  __device__ __forceinline__ void run(float* stats) const {
    constexpr int AHEAD = 3;  // operands read ahead of their product
    u32x4 qf[NK];
    const long long mine = this->template query<false>(wrow, qf, ring + wave * 32 * ROW, 1);
    const int lim = limit(wrow + l32);
    meet();  // the ring is the tiles' from here on
    const int end = wrow < rows ? limit(wrow + 31) : 0;
    constexpr bool BY_SUM = E == 2 && DH <= 192;
    f32x16 o[ND];
    float m = BY_SUM ? kNoRef : -INFINITY, l = 0.f;  // l over the lane half's keys only
    uint32_t odds = 0;
#pragma unroll
    for (int d = 0; d < ND; ++d) o[d] = zeros16();
    // 32 keys.  EDGE: some row may not see them all, and values there are sifted.
    auto step = [&](auto at_edge, int kt) __attribute__((always_inline)) {
      constexpr bool EDGE = decltype(at_edge)::value;
      const int key0 = kt * KT + 32 * half;
      int kb = kaddr + (kt & 1) * 2 * BYTES, vb = vaddr + (kt & 1) * 2 * BYTES;
      asm volatile("" : "+v"(kb), "+v"(vb));  // not 16 addresses kept over the loop

      // Each product and the read that takes its place are pinned in this order:
      // left alone, the scheduler reads just before it multiplies.
      f32x16 sc = zeros16();
      u32x4 kf[AHEAD];
#pragma unroll
      for (int p = 0; p < AHEAD; ++p) kf[p] = kread(kb, p);
      __builtin_amdgcn_s_setprio(1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int p = 0; p < NK; ++p) {
        sc = mma32(kf[p % AHEAD], qf[p], sc, T{});
        if (p + AHEAD < NK) kf[p % AHEAD] = kread(kb, p + AHEAD);
        __builtin_amdgcn_sched_barrier(0);
      }
      __builtin_amdgcn_s_setprio(0);
      vop vf[AHEAD];
#pragma unroll
      for (int n = 0; n < AHEAD; ++n) vf[n] = vread(vb, n / PV, n % PV);
      __builtin_amdgcn_sched_barrier(0);

      u32x4 pf[2];
      auto rescale = [&](float f) __attribute__((always_inline)) {
#pragma unroll
        for (int d = 0; d < ND; ++d) o[d] *= f;
      };
      if constexpr (BY_SUM)
        softmax_by_sum(sc, EDGE, key0, lh, lim, a.scale, m, l, pf, rescale);
      else
        softmax<T>(sc, EDGE, key0, lh, lim, a.scale, m, l, pf, rescale, [](int) {});
      __builtin_amdgcn_s_setprio(1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int n = 0; n < ND * PV; ++n) {
        vop v = vf[n % AHEAD];
        if (EDGE) {
          odds |= odds_of(v, T{});
          v = even_of(v, T{});
        }
        o[n / PV] = product(v, sc, pf, n % PV, o[n / PV]);
        if (n + AHEAD < ND * PV) vf[n % AHEAD] = vread(vb, (n + AHEAD) / PV, (n + AHEAD) % PV);
        __builtin_amdgcn_sched_barrier(0);
      }
      __builtin_amdgcn_s_setprio(0);
    };
    const int whole = limit(row0) / KT;  // tiles that every row of the workgroup sees
    Offsets offs;
    find(offs);
    if (tiles > 0) issue(0, 0, offs);
    for (int kt = 0; kt < whole; ++kt) {
      meet();  // tile kt is there and tile kt - 1 is done with
      if (kt + 1 < tiles) issue(kt + 1, (kt + 1) & 1, offs);
      step(std::false_type{}, kt);
    }
    for (int kt = whole; kt < tiles; ++kt) {
      meet();
      if (kt + 1 < tiles) issue(kt + 1, (kt + 1) & 1, offs);
      if (kt * KT + 32 * half < end) step(std::true_type{}, kt);
    }
    bool unruly = any_odd(odds, T{});
    if (BY_SUM) m = m == kNoRef ? -INFINITY : -m;
    meet();
    if constexpr (KG == 2) {
      f32x4* so = reinterpret_cast<f32x4*>(ring) + (wave % 4) * (4 * ND * 64) + lane;
      float* st = stats + (wave % 4) * 128 + lane;
      if (half) {
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            so[(4 * d + j) * 64] = f32x4{o[d][4 * j], o[d][4 * j + 1], o[d][4 * j + 2], o[d][4 * j + 3]};
        st[0] = m;
        st[64] = l;
        if (lane == 0) stats[512 + wave % 4] = unruly;
      }
      meet();
      if (!half) {
        unruly |= stats[512 + wave] != 0.f;
        const float other = st[0], now = fmaxf(m, other), ref = now == -INFINITY ? 0.f : now;
        const float f = __builtin_amdgcn_exp2f(m - ref), g = __builtin_amdgcn_exp2f(other - ref);
        l = l * f + st[64] * g;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const f32x4 x = so[(4 * d + j) * 64];
#pragma unroll
            for (int e = 0; e < 4; ++e) o[d][4 * j + e] = o[d][4 * j + e] * f + x[e] * g;
          }
      }
      meet();
      if (half) return;
    }
    // rows go out whole, through LDS
    unsigned char* so = ring + wave * 32 * ROW;
    const float inv = inverse(l, lim);
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int at = 32 * d + 8 * j + 4 * lh;  // first of four elements
        T* p = reinterpret_cast<T*>(so + l32 * ROW + (((at * E >> 4) ^ (l32 & 7)) << 4) + (at * E & 15));
        const f32x16& x = o[d];
        store4(p, x[4 * j] * inv, x[4 * j + 1] * inv, x[4 * j + 2] * inv, x[4 * j + 3] * inv);
      }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (unruly) {
      add_unruly<DH>(static_cast<const T*>(a.v) + (size_t)k0 * a.ldv + kh * DH, a.ldv, whole * KT,
                     min(end, nk), lim, [&](int r, int d) {
                       return reinterpret_cast<T*>(so + r * ROW + (((d * E >> 4) ^ (r & 7)) << 4) + (d * E & 15));
                     });
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
    for (int u = lane; u < 32 * PIECES; u += 64) {
      const int r = u / PIECES, c = u % PIECES;
      const long long at = __shfl(mine, r);
      if (wrow + r < rows)
        *reinterpret_cast<u32x4*>(static_cast<T*>(a.out) + at + c * (16 / E)) =
            *reinterpret_cast<const u32x4*>(so + r * ROW + ((c ^ (r & 7)) << 4));
    }
  }
};

template <typename T, int DH, int KG>
__global__ __launch_bounds__(256 * KG, DH * sizeof(T) > 512 ? 1 : 2) void prompt_kernel(PromptCall a) {
  typedef Walk<T, DH, KG> W;
  __shared__ __attribute__((aligned(1024))) unsigned char ring[4 * W::BYTES];
  __shared__ float stats[KG == 2 ? 516 : 1];
  const W w(a, ring);
  if (w.any()) w.run(stats);
}

// Keys of V from memory into registers.  A lane takes W = DH/32 consecutive
// elements of each of its 16 keys (those of its score registers), a whole row by
// 32 lanes; row i of O^T's tile j is then the head's element W i + j.  bf16 wants
// all 16 at once (ROWS), fp32 one after another.
template <typename T, int DH> struct FewV {
  static constexpr int W = DH / 32, DW = W * (int)sizeof(T) / 4, ROWS = sizeof(T) == 2 ? 16 : 4;
  uint32_t w[ROWS][DW];
  // Row x: `off` bytes past the source.
  __device__ __forceinline__ void load(int row, lds_src src, int off) {
    const int x = row % ROWS;
    constexpr int B = DW / 4 * 4;
#pragma unroll
    for (int i = 0; i < B; i += 4) {
      const auto y = __builtin_amdgcn_raw_buffer_load_b128(src, off + 4 * i, 0, 0);
#pragma unroll
      for (int e = 0; e < 4; ++e) w[x][i + e] = y[e];
    }
    if constexpr (DW % 4 == 3) {
      const auto y = __builtin_amdgcn_raw_buffer_load_b96(src, off + 4 * B, 0, 0);
#pragma unroll
      for (int e = 0; e < 3; ++e) w[x][B + e] = y[e];
    } else if constexpr (DW % 4 == 2) {
      const auto y = __builtin_amdgcn_raw_buffer_load_b64(src, off + 4 * B, 0, 0);
#pragma unroll
      for (int e = 0; e < 2; ++e) w[x][B + e] = y[e];
    } else if constexpr (DW % 4 == 1) {
      w[x][B] = __builtin_amdgcn_raw_buffer_load_b32(src, off + 4 * B, 0, 0);
    }
  }
  // Takes what is not finite out of the rows [first, last); whether there was any.
  __device__ __forceinline__ bool sift(int first, int last) {
    uint32_t odds = 0;
#pragma unroll
    for (int x = first; x < last; ++x)
#pragma unroll
      for (int i = 0; i < DW; ++i) odds |= odd(w[x % ROWS][i], T{});
    if (__builtin_expect(!any_odd(odds, T{}), 1)) return false;
#pragma unroll
    for (int x = first; x < last; ++x)
#pragma unroll
      for (int i = 0; i < DW; ++i) w[x % ROWS][i] = even(w[x % ROWS][i], T{});
    return true;
  }
  // Operand c of tile j: 16 keys from 16 c on (bf16, a turned 8 x 2 block), the
  // keys of score register c (fp32).
  __device__ __forceinline__ auto operand(int j, int c) const {
    if constexpr (sizeof(T) == 2) {
      u32x4 r;
#pragma unroll
      for (int y = 0; y < 4; ++y)
        r[y] = __builtin_amdgcn_perm(w[8 * c + 2 * y + 1][j >> 1], w[8 * c + 2 * y][j >> 1],
                                     j & 1 ? 0x07060302u : 0x05040100u);
      return r;
    } else {
      return __uint_as_float(w[c % ROWS][j]);
    }
  }
};

// Few rows: 32 of them a workgroup, whose waves share the keys out and join in
// LDS.  Waves do not wait for each other before that.  Values come from the caches
// straight into registers, whole rows by 32 lanes; keys, of which a lane wants a
// row of its own (32 bytes of each of 32 rows a load), through a wave's own LDS in
// bf16, one step ahead, and into registers in fp32, whose products take 16 times as
// long and need no more than a few operands at a time.
constexpr int kFewWaves = 4;
template <typename T, int DH>
__global__ __launch_bounds__(64 * kFewWaves, 1) void prompt_few_kernel(PromptCall a) {
  typedef Rows<T, DH, 32> Base;
  constexpr int E = Base::E, NK = Base::NK, ND = Base::ND, PV = E == 2 ? 2 : 16, W = DH / 32;
  constexpr int PITCH = DH + 4;
  constexpr int ROW = DH * E, SW = DH % 128 == 0 ? 16 : 8, NI = 32 * ROW / 1024;
  constexpr int KEYS = E == 2 ? 2 * 32 * ROW : 0, JOIN = 32 * PITCH * 4;  // bytes of a wave
  __shared__ float sm[kFewWaves][32], sl[kFewWaves][32];
  __shared__ long long place[32];
  constexpr int WORK = kFewWaves * (KEYS > JOIN ? KEYS : JOIN);
  __shared__ __attribute__((aligned(1024))) unsigned char lds[WORK + (E == 2 ? 32 * ROW : 0)];
  unsigned char* queries = lds + (E == 2 ? WORK : 0);
  const Base b(a);
  if (!b.any()) return;
  const int l32 = b.l32, lh = b.lh, wave = b.wave;
  const int whole = b.limit(b.row0) / 32, steps = (b.limit(b.row0 + 31) + 31) / 32;
  const T* kbase = static_cast<const T*>(a.k) + (size_t)b.k0 * a.ldk + b.kh * DH;
  const T* vbase = static_cast<const T*>(a.v) + (size_t)b.k0 * a.ldv + b.kh * DH;
  unsigned char* ring = lds + wave * KEYS;
  const int kaddr = l32 * ROW + ((lh ^ swizzle<T, DH>(l32)) << 4);
  // Part n of NI of the keys of step i (bf16); of no step, past the last.
  auto load_keys = [&](int i, int stage, int n) __attribute__((always_inline)) {
    lds_src src = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<T*>(kbase + (size_t)32 * min(i, steps - 1) * a.ldk), 0, i < steps ? 0x7fffffff : 0, 0x00020000);
    const Slots<T, DH> at(b.lane);
    int row, byte;
    at.find(n, row, byte);
    lds_dma16(src, ring + stage * 32 * ROW + 1024 * n, __umul24(min(row, b.nk - 1 - 32 * i), a.ldk * E) + byte, 0);
  };
  if (E == 2 && wave < steps) {
#pragma unroll
    for (int n = 0; n < NI; ++n) load_keys(wave, 0, n);
  }
  u32x4 qf[NK];
  const long long mine = b.template query<true>(b.row0, qf, queries, kFewWaves);
  const int lim = b.limit(b.row0 + l32);
  f32x16 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) o[d] = zeros16();
  float m = -INFINITY, l = 0.f;  // l over the lane half's keys only
  bool unruly = false;
  int stage = 0;
  for (int i = wave; i < steps; i += kFewWaves, stage ^= 1) {
    const bool edge = i >= whole;
    FewV<T, DH> v;
    const lds_src vs = lds_source(vbase + (size_t)32 * i * a.ldv);
    const int most = b.nk - 1 - 32 * i;  // rows past the prompt's last repeat it
    auto load_value = [&](int x) __attribute__((always_inline)) {
      v.load(x, vs, __umul24(min(8 * (x >> 2) + (x & 3) + 4 * lh, most), a.ldv * E) + W * E * l32);
    };
    f32x16 sc = zeros16();
    u32x4 pf[2];
    auto rescale = [&](float f) __attribute__((always_inline)) {
#pragma unroll
      for (int d = 0; d < ND; ++d) o[d] *= f;
    };
    if constexpr (E == 2) {
      // A load holds its wave up for 16 cycles and more when four waves load: the
      // values' go out among the scores' products, the next keys' among the softmax.
      __builtin_amdgcn_s_waitcnt(0x7 << 4);  // this step's keys are there, nothing is under way
      __builtin_amdgcn_sched_barrier(0);
      f32x16 sc1 = zeros16();  // two chains of products
      int kb = kaddr + stage * 32 * ROW;
      asm volatile("" : "+v"(kb));
      auto key = [&](int p) __attribute__((always_inline)) {
        return *reinterpret_cast<const u32x4*>(ring + (kb ^ ((2 * p & (SW - 1)) << 4)) + 2 * p / SW * SW * 16);
      };
      u32x4 kr[3];
#pragma unroll
      for (int p = 0; p < 3; ++p) kr[p] = key(p);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int p = 0; p < NK; ++p) {
        if (p & 1)
          sc1 = mma32(kr[p % 3], qf[p], sc1, T{});
        else
          sc = mma32(kr[p % 3], qf[p], sc, T{});
        if (p + 3 < NK) kr[p % 3] = key(p + 3);
#pragma unroll
        for (int x = 16 * p / NK; x < 16 * (p + 1) / NK; ++x) load_value(x);
        __builtin_amdgcn_sched_barrier(0);
      }
      sc += sc1;
      softmax<T>(sc, edge, 32 * i, lh, lim, a.scale, m, l, pf, rescale, [&](int r) __attribute__((always_inline)) {
        if (r < NI) load_keys(i + kFewWaves, stage ^ 1, r);
      });
      if (edge && v.sift(0, 16)) unruly = true;
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int c = 0; c < PV; ++c) o[d] = product(v.operand(d, c), sc, pf, c, o[d]);
    } else {
      constexpr int AHEAD = 6;
      const T* row = kbase + (size_t)min(32 * i + l32, b.nk - 1) * a.ldk;
      auto key = [&](int p) __attribute__((always_inline)) {
        return *reinterpret_cast<const u32x4*>(row + (2 * p + lh) * (16 / E));
      };
      u32x4 kr[AHEAD];
#pragma unroll
      for (int p = 0; p < AHEAD; ++p) kr[p] = key(p);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int p = 0; p < NK; ++p) {
        sc = mma32(kr[p % AHEAD], qf[p], sc, T{});
        if (p + AHEAD < NK) kr[p % AHEAD] = key(p + AHEAD);
        if (p >= NK - FewV<T, DH>::ROWS) load_value(p - NK + FewV<T, DH>::ROWS);
        __builtin_amdgcn_sched_barrier(0);
      }
      softmax<T>(sc, edge, 32 * i, lh, lim, a.scale, m, l, pf, rescale, [](int) {});
#pragma unroll
      for (int c = 0; c < PV; ++c) {
        if (edge && v.sift(c, c + 1)) unruly = true;
#pragma unroll
        for (int d = 0; d < ND; ++d) o[d] = product(v.operand(d, c), sc, pf, c, o[d]);
        if (c + FewV<T, DH>::ROWS < PV) load_value(c + FewV<T, DH>::ROWS);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }

  // The waves' sums, brought to the rows' common reference, join in LDS.
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  l = other_half_sum(l);
  if (lh == 0) {
    sm[wave][l32] = m;
    sl[wave][l32] = l;
    if (wave == 0) place[l32] = mine;
  }
  __syncthreads();  // and every wave is done with its keys
  float f, all = 0.f, top = -INFINITY;
#pragma unroll
  for (int w = 0; w < kFewWaves; ++w) top = fmaxf(top, sm[w][l32]);
  const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
  for (int w = 0; w < kFewWaves; ++w) all += __builtin_amdgcn_exp2f(sm[w][l32] - ref) * sl[w][l32];
  f = lim > 0 ? __builtin_amdgcn_exp2f(m - ref) / all : 0.f;  // no key seen: zeros
  float* so = reinterpret_cast<float*>(lds) + wave * 32 * PITCH;
#pragma unroll
  for (int j = 0; j < 16; ++j)
#pragma unroll
    for (int d = 0; d < ND; ++d) so[l32 * PITCH + W * (8 * (j >> 2) + 4 * lh + (j & 3)) + d] = o[d][j] * f;
  if (unruly) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    for (int i = wave; i < steps; i += kFewWaves)
      if (i >= whole)
        add_unruly<DH>(vbase, a.ldv, 32 * i, min(32 * i + 32, b.nk), lim,
                       [&](int r, int d) { return so + r * PITCH + d; });
  }
  __syncthreads();
  constexpr int PER = 32 * (DH / 4) / (64 * kFewWaves);
#pragma unroll
  for (int n = 0; n < PER; ++n) {
    const int u = threadIdx.x + n * 64 * kFewWaves, r = u / (DH / 4), d = 4 * (u % (DH / 4));
    f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w)
      acc += *reinterpret_cast<const f32x4*>(reinterpret_cast<float*>(lds) + (w * 32 + r) * PITCH + d);
    if (b.row0 + r < b.rows)
      store4(static_cast<T*>(a.out) + place[r] + d, acc[0], acc[1], acc[2], acc[3]);
  }
}

template <typename T, int DH>
void prompt_at(PromptCall& a, int form, hipStream_t s) {
  const int R = form == kFew ? 32 : 128;
  a.n_slots = (int)((int64_t)a.n_q * a.group / R + a.n_seqs);
  const dim3 grid((unsigned)(a.n_slots * a.n_kv));
  if (form == kFew)
    hipLaunchKernelGGL((prompt_few_kernel<T, DH>), grid, dim3(64 * kFewWaves), 0, s, a);
  else if (form == kTiles)
    hipLaunchKernelGGL((prompt_kernel<T, DH, 1>), grid, dim3(256), 0, s, a);
  else if constexpr (sizeof(T) == 2)
    hipLaunchKernelGGL((prompt_kernel<T, DH, 2>), grid, dim3(512), 0, s, a);
}

}  // namespace

// Which kernel, by the 32-row tiles of the call (256 CUs; a CU holds one or two
// workgroups).  us at prompts of 560 tokens (one prompt), heads 8/1 of 256: kFew 17
// (22), kHalves 22 (33), kTiles 24 (39) at 280 tiles; 41 (95), 25 (81), 26 (104) at
// 840; 75 (314), 42 (184), 33 (231) at 1680; 191 (1971), 87 (1164), 67 (1105) at
// 4480.  Heads 32/8 of 128: 20 (20), 14 (15), 15 (15) at 560; 49 (73), 23 (32), 20 (38)
// at 1680; 125 (363), 47 (173), 37 (161) at 4480.  A long causal prompt's last tiles
// outlast the others, which halving the walk of each makes up for until the chip is
// full.  In fp32, where products are 16 times as long and the loads of few rows no
// matter, kFew and kTiles take: heads of 256, 81 (207) and 161 (583) at 560, 279 (2592)
// and 309 (2862) at 2240, 541 (10082) and 527 (10700) at 4480; of 128, 44 (44) and 81
// (80), 154 (390) and 133 (432), 298 (1425) and 240 (1260).  Long prompts favour kFew: 16
// of 4000, heads 4/2 of 192 (8000 tiles), 3376 and 4078; 8 of 2400, 8/1 of 256 (4800),
// 1668 and 1814; but heads of 64, 16 of 4000 (16000), 2400 and 2250.  So does the causal
// edge, most at 128: 4 prompts of 800, heads 8/2 (800), 74 and 111, all keys seen 137 and
// 112.
// Swept again over 122 calls (head dims 64 to 256, 140 to 8000 tiles, prompts of 128 to
// 16000): the kernel taken is the fastest or within 6 % of it in 114; the others are bf16
// heads of 64 at 560 to 600 tiles (one prompt of 2400: 28 and 22 with kFew; four of 560: 11.0 and
// 10.3) and of 128 with prompts under 200 (11.4 and 9.6 with kTiles), fp32 heads of 64 at
// 4050 to 7800 tiles (142 and 125, 817 and 752) and of 128, every key seen (287 and 262).
int prompt_form(const fv_prompt_args& x) {
  const int64_t tiles = (int64_t)x.n_q * x.n_q_heads / 32;
  const bool far = x.n_k / x.n_seqs >= 2048;  // long prompts
  if (x.dtype == FV_FP32) {
    int most = 4096;
    if (x.head_dim >= 192 && far) most = 8192;
    if (x.head_dim == 128 && !far) most = x.causal ? 2048 : 768;
    return tiles <= most ? kFew : kTiles;
  }
  if (tiles < 384) return kFew;
  return tiles <= (x.causal && far ? 2560 : 1024) ? kHalves : kTiles;
}

template <typename T>
void launch_prompt(const fv_prompt_args& x, hipStream_t s) {
  PromptCall a{};
  a.q = x.q;
  a.k = x.k;
  a.v = x.v;
  a.out = x.out;
  a.cu_q = x.cu_q;
  a.cu_k = x.cu_k;
  a.ldq = x.ldq;
  a.ldk = x.ldk;
  a.ldv = x.ldv;
  a.ldo = x.ldo;
  a.n_seqs = x.n_seqs;
  a.n_q = x.n_q;
  a.n_k = x.n_k;
  a.n_kv = x.n_kv_heads;
  a.group = x.n_q_heads / x.n_kv_heads;
  a.causal = x.causal;
  a.scale = x.scale * kLog2e;
  const int form = prompt_form(x);
  switch (x.head_dim) {
    case 64: return prompt_at<T, 64>(a, form, s);
    case 128: return prompt_at<T, 128>(a, form, s);
    case 192: return prompt_at<T, 192>(a, form, s);
    default: return prompt_at<T, 256>(a, form, s);
  }
}
template void launch_prompt<bf16_t>(const fv_prompt_args&, hipStream_t);
template void launch_prompt<float>(const fv_prompt_args&, hipStream_t);

}  // namespace fv
