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

__device__ __forceinline__ f32x16 zeros16() {
  f32x16 z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.f;
  return z;
}

// Values at the edge, where a wave's rows differ in what they see.  A weight of
// zero does not silence a value that is not finite, so such values are taken out
// of the product there; afterwards, products of ones in their place (for +inf, for
// -inf, for both where the value is NaN) with the rows' view say which sums they
// make infinite.
__device__ __forceinline__ bool is_unruly(u32x4 x, bf16_t) {
  bool any = false;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    any |= (x[i] & 0x7f80u) == 0x7f80u || (x[i] & 0x7f800000u) == 0x7f800000u;
  return any;
}
__device__ __forceinline__ bool is_unruly(float x, float) { return !(fabsf(x) < INFINITY); }
// The operand without them.
__device__ __forceinline__ u32x4 ruly(u32x4 x, bf16_t) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if ((x[i] & 0x7f80u) == 0x7f80u) x[i] &= 0xffff0000u;
    if ((x[i] & 0x7f800000u) == 0x7f800000u) x[i] &= 0x0000ffffu;
  }
  return x;
}
__device__ __forceinline__ float ruly(float x, float) { return is_unruly(x, x) ? 0.f : x; }
// Ones for the values of SIGN times infinity, or NaN.
template <int SIGN> __device__ __forceinline__ u32x4 ones_for(u32x4 x, bf16_t) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r[i] = 0;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const uint32_t b = x[i] >> (16 * half) & 0xffffu;
      if ((b & 0x7fffu) > 0x7f80u || b == (SIGN > 0 ? 0x7f80u : 0xff80u)) r[i] |= 0x3f80u << (16 * half);
    }
  }
  return r;
}
template <int SIGN> __device__ __forceinline__ float ones_for(float x, float) {
  return x != x || x == SIGN * INFINITY ? 1.f : 0.f;
}
template <int SIGN> __device__ __forceinline__ void add_infinities(f32x16& o, const f32x16& seen) {
#pragma unroll
  for (int r = 0; r < 16; ++r) o[r] += seen[r] > 0.f ? SIGN * INFINITY : 0.f;
}
// For operand c of V (see vread) and a lane whose row sees the keys below lim.
template <int SIGN>
__device__ __forceinline__ void add_unruly(u32x4 v, int c, int key0, int lh, int lim, f32x16& o, bf16_t) {
  u16x8 seen;
#pragma unroll
  for (int e = 0; e < 8; ++e)
    seen[e] = key0 + 16 * c + 8 * (e >> 2) + 4 * lh + (e & 3) < lim ? 0x3f80 : 0;
  add_infinities<SIGN>(o, mma32(ones_for<SIGN>(v, bf16_t{}), __builtin_bit_cast(u32x4, seen), zeros16(),
                                bf16_t{}));
}
template <int SIGN>
__device__ __forceinline__ void add_unruly(float v, int c, int key0, int lh, int lim, f32x16& o, float) {
  const float seen = key0 + 8 * (c >> 2) + 4 * lh + (c & 3) < lim ? 1.f : 0.f;
  add_infinities<SIGN>(o, __builtin_amdgcn_mfma_f32_32x32x2f32(ones_for<SIGN>(v, v), seen, zeros16(), 0, 0, 0));
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

// One workgroup's walk over the keys of its rows: RT 32-row tiles a wave (with
// two, every operand read from LDS serves two products).
template <typename T, int DH, int WAVES, int RT>
struct Walk {
  static constexpr int E = (int)sizeof(T);
  static constexpr int KT = E == 2 && WAVES == 8 ? 64 : 32;    // keys of a tile
  static constexpr int ROW = DH * E, PIECES = ROW / 16;
  static constexpr int BYTES = KT * ROW;                       // of a K tile, and of a V tile
  static constexpr int SW = E == 4 || DH % 128 == 0 ? 16 : 8;  // pieces that a swizzle permutes
  static constexpr int R = 32 * RT * WAVES;                    // rows of a workgroup
  static constexpr int ND = DH / 32;                           // 32-row tiles of O^T
  static constexpr int NI = BYTES / 1024 / WAVES;              // direct loads of a wave per tensor and tile
  static constexpr int NK = PIECES / 2;                        // K operands of 32 keys
  static constexpr int PV = E == 2 ? 2 : 16;                   // V operands of 32 keys and 32 elements
  static_assert(NI * 1024 * WAVES == BYTES && 32 * WAVES * ROW <= 4 * BYTES, "tile split");
  typedef typename std::conditional<E == 2, u32x4, float>::type vop;

  const PromptCall& a;
  unsigned char* ring;  // two stages of K and V
  int lane, wave, l32, lh, kh, q0, k0, nk, rows, row0, wrow, diff, tiles, kaddr, vaddr;

  __device__ __forceinline__ Walk(const PromptCall& call, unsigned char* lds) : a(call), ring(lds) {
    lane = threadIdx.x & 63;
    wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    l32 = lane & 31;
    lh = lane >> 5;
    // the heaviest tiles of a causal prompt, its last ones, go first
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
    wrow = row0 + 32 * RT * wave;
    diff = nk - nq + 1;
    tiles = (limit(row0 + R - 1) + KT - 1) / KT;
    // LDS addresses of the operands: one register each for K and V and a constant
    // exclusive or (the swizzle), so that they cost an instruction and no registers.
    kaddr = l32 * ROW + ((lh ^ swizzle<T, DH>(l32)) << 4);
    const int i16 = lane & 15, r = 4 * lh + (i16 >> 2);
    vaddr = E == 2 ? BYTES + r * ROW +
                         (((2 * ((lane >> 4) & 1) + ((i16 >> 1) & 1)) ^ swizzle<T, DH>(r)) << 4) +
                         (i16 & 1) * 8
                   : BYTES + 4 * lh * ROW + (((l32 >> 2) ^ (lh << 3)) << 4) + (l32 & 3) * 4;
  }
  // A row sees the keys [0, limit), which do not fall from one row to the next.
  __device__ __forceinline__ int limit(int row) const {
    return a.causal ? min(max(diff + min(row, rows - 1) / a.group, 0), nk) : nk;
  }
  // The lane's query of row tile t, as products' operands, and its place in the output.
  __device__ __forceinline__ long long query(int t, u32x4 (&qf)[NK]) const {
    const int row = min(wrow + 32 * t + l32, rows - 1);
    const int tok = row / a.group, head = kh * a.group + row - tok * a.group;
    const T* q = static_cast<const T*>(a.q) + (size_t)(q0 + tok) * a.ldq + head * DH;
#pragma unroll
    for (int p = 0; p < NK; ++p)
      qf[p] = *reinterpret_cast<const u32x4*>(q + (2 * p + lh) * (16 / E));
    return (long long)(q0 + tok) * a.ldo + head * DH;
  }
  // Direct loads of key tile kt: slot u, 16 bytes, is piece u % PIECES of row u / PIECES.
  __device__ __forceinline__ void issue(int kt, int stage) const {
    unsigned char* to = ring + stage * 2 * BYTES + wave * NI * 1024;
    const lds_src ks = lds_source(static_cast<const T*>(a.k) + (size_t)(k0 + kt * KT) * a.ldk + kh * DH);
    const lds_src vs = lds_source(static_cast<const T*>(a.v) + (size_t)(k0 + kt * KT) * a.ldv + kh * DH);
    const int most = nk - 1 - kt * KT;  // rows past the prompt's last repeat it
    int mine = lane;
    asm volatile("" : "+v"(mine));  // not 2 NI offsets kept over the loop
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int u = 64 * (NI * wave + i) + mine, r = u / PIECES;
      const int c = (u % PIECES) ^ swizzle<T, DH>(r), rr = min(r, most);
      lds_dma16(ks, to + 1024 * i, rr * a.ldk * E + 16 * c, 0);
      lds_dma16(vs, to + BYTES + 1024 * i, rr * a.ldv * E + 16 * c, 0);
    }
  }
  // Every wave's loads have landed, every wave's reads are done.
  __device__ __forceinline__ void meet() const {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  }
  __device__ __forceinline__ u32x4 kread(int base, int sub, int p) const {
    return *reinterpret_cast<const u32x4*>(ring + (base ^ ((2 * p & (SW - 1)) << 4)) +
                                           32 * sub * ROW + 2 * p / SW * SW * 16);
  }
  // Operand c of V for the elements from 32 d on of the head: 16 keys from 16 c on
  // (bf16), the keys of score register c (fp32).
  __device__ __forceinline__ vop vread(int base, int sub, int d, int c) const {
    if constexpr (E == 2) {
      const unsigned char* p = ring + (32 * sub + 16 * c) * ROW + 4 * d / SW * SW * 16;
      const int x = base ^ ((4 * d & (SW - 1)) << 4);
      const u32x2 lo = read_transposed(p + x), hi = read_transposed(p + (x ^ 32) + 8 * ROW);
      return u32x4{lo[0], lo[1], hi[0], hi[1]};
    } else {
      const int j = c >> 2, r = c & 3;
      const int x = base ^ ((8 * d & 15) << 4) ^ (r << 5) ^ ((j & 1) << 4);
      return *reinterpret_cast<const float*>(ring + x + (32 * sub + 8 * j + r) * ROW + 8 * d / 16 * 256);
    }
  }
  static __device__ __forceinline__ f32x16 product(vop v, const f32x16& p, const u32x4 (&pf)[2], int c,
                                                   f32x16 o) {
    if constexpr (E == 2)
      return mma32(v, pf[c], o, T{});
    else
      return __builtin_amdgcn_mfma_f32_32x32x2f32(v, p[c], o, 0, 0, 0);
  }
  // Scores of 32 keys to probabilities (pf: as bf16 operands), with the row's
  // reference m and sum l; calls rescale(f) where the reference moves.
  template <bool EDGE, typename Rescale>
  __device__ __forceinline__ void softmax(f32x16& sc, int key0, int lim, float& m, float& l,
                                          u32x4 (&pf)[2], Rescale rescale) const {
    if (EDGE) {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (key0 + 8 * (r >> 2) + 4 * lh + (r & 3) >= lim) sc[r] = -INFINITY;
    }
    float top = sc[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(top, sc[r]);
    top = other_half_max(top) * a.scale;
    if (__any(top > m + kSlack)) {
      const float now = fmaxf(m, top);
      const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - now);
      m = now;
      l *= f;
      rescale(f);
    }
    const float ref = m == -INFINITY ? 0.f : -m;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      sc[r] = __builtin_amdgcn_exp2f(fmaf(sc[r], a.scale, ref));
      l += sc[r];
    }
    if constexpr (E == 2) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        u16x8 w;
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = f32_to_bf16(sc[8 * c + e]);
        pf[c] = __builtin_bit_cast(u32x4, w);
      }
    }
  }
  // No key seen: zeros; keys that all score -inf: 0/0, as the formula has it.
  static __device__ __forceinline__ float inverse(float l, int lim) {
    return lim > 0 ? 1.0f / other_half_sum(l) : 0.f;
  }

  // *again: a word of LDS, cleared by the caller.
  __device__ __forceinline__ void run(int* again) const {
    constexpr int AHEAD = RT == 2 ? 2 : 3;  // operands read ahead of their product
    int lim[RT];
    long long mine[RT];
    u32x4 qf[RT][NK];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      lim[t] = limit(wrow + 32 * t + l32);
      mine[t] = query(t, qf[t]);
    }
    const int end = wrow < rows ? limit(wrow + 32 * RT - 1) : 0;
    f32x16 o[RT][ND];
    float m[RT], l[RT];  // l over the lane half's keys only
    bool unruly = false;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      m[t] = -INFINITY;
      l[t] = 0.f;
#pragma unroll
      for (int d = 0; d < ND; ++d) o[t][d] = zeros16();
    }
    // 32 keys.  EDGE: some row may not see them all, and values there are sifted.
    auto step = [&](auto at_edge, int kt, int sub) __attribute__((always_inline)) {
      constexpr bool EDGE = decltype(at_edge)::value;
      const int key0 = kt * KT + 32 * sub;
      int kb = kaddr + (kt & 1) * 2 * BYTES, vb = vaddr + (kt & 1) * 2 * BYTES;
      asm volatile("" : "+v"(kb), "+v"(vb));  // not 16 addresses kept over the loop

      // Each product and the read that takes its place are pinned in this order:
      // left alone, the scheduler reads just before it multiplies.
      f32x16 sc[RT];
#pragma unroll
      for (int t = 0; t < RT; ++t) sc[t] = zeros16();
      u32x4 kf[AHEAD];
#pragma unroll
      for (int p = 0; p < AHEAD; ++p) kf[p] = kread(kb, sub, p);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int p = 0; p < NK; ++p) {
#pragma unroll
        for (int t = 0; t < RT; ++t) sc[t] = mma32(kf[p % AHEAD], qf[t][p], sc[t], T{});
        if (p + AHEAD < NK) kf[p % AHEAD] = kread(kb, sub, p + AHEAD);
        __builtin_amdgcn_sched_barrier(0);
      }
      vop vf[AHEAD];
#pragma unroll
      for (int n = 0; n < AHEAD; ++n) vf[n] = vread(vb, sub, n / PV, n % PV);
      __builtin_amdgcn_sched_barrier(0);

      u32x4 pf[RT][2];
#pragma unroll
      for (int t = 0; t < RT; ++t)
        softmax<EDGE>(sc[t], key0, lim[t], m[t], l[t], pf[t], [&](float f) {
#pragma unroll
          for (int d = 0; d < ND; ++d) o[t][d] *= f;
        });
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int n = 0; n < ND * PV; ++n) {
        vop v = vf[n % AHEAD];
        if (EDGE) {
          unruly |= __any(is_unruly(v, T{}));
          v = ruly(v, T{});
        }
#pragma unroll
        for (int t = 0; t < RT; ++t) o[t][n / PV] = product(v, sc[t], pf[t], n % PV, o[t][n / PV]);
        if (n + AHEAD < ND * PV) vf[n % AHEAD] = vread(vb, sub, (n + AHEAD) / PV, (n + AHEAD) % PV);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    const int whole = limit(row0) / KT;  // tiles that every row of the workgroup sees
    if (tiles > 0) issue(0, 0);
    for (int kt = 0; kt < whole; ++kt) {
      meet();  // tile kt is there and tile kt - 1 is done with
      if (kt + 1 < tiles) issue(kt + 1, (kt + 1) & 1);
#pragma unroll
      for (int sub = 0; sub < KT / 32; ++sub) step(std::false_type{}, kt, sub);
    }
    for (int kt = whole; kt < tiles; ++kt) {
      meet();
      if (kt + 1 < tiles) issue(kt + 1, (kt + 1) & 1);
      for (int sub = 0; sub < KT / 32; ++sub)
        if (kt * KT + 32 * sub < end) step(std::true_type{}, kt, sub);
    }
    if (unruly) *again = 1;
    meet();
    // What the values left out of the edges make of the sums of rows that see them.
    if (__builtin_amdgcn_readfirstlane(*again))
      for (int kt = whole; kt < tiles; ++kt) {
        issue(kt, 0);
        meet();
        for (int sub = 0; sub < KT / 32; ++sub) {
          const int key0 = kt * KT + 32 * sub;
          if (key0 >= end) continue;
#pragma unroll
          for (int d = 0; d < ND; ++d)
#pragma unroll 1
            for (int c = 0; c < PV; ++c) {
              const vop v = vread(vaddr, sub, d, c);
              if (!__any(is_unruly(v, T{}))) continue;
#pragma unroll
              for (int t = 0; t < RT; ++t) {
                add_unruly<1>(v, c, key0, lh, lim[t], o[t][d], T{});
                add_unruly<-1>(v, c, key0, lh, lim[t], o[t][d], T{});
              }
            }
        }
        meet();
      }

    // rows go out whole, through LDS
    unsigned char* so = ring + wave * 32 * ROW;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const float inv = inverse(l[t], lim[t]);
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int at = 32 * d + 8 * j + 4 * lh;  // first of four elements
          T* p = reinterpret_cast<T*>(so + l32 * ROW + (((at * E >> 4) ^ (l32 & 7)) << 4) + (at * E & 15));
          const f32x16& x = o[t][d];
          store4(p, x[4 * j] * inv, x[4 * j + 1] * inv, x[4 * j + 2] * inv, x[4 * j + 3] * inv);
        }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      for (int u = lane; u < 32 * PIECES; u += 64) {
        const int r = u / PIECES, c = u % PIECES;
        const long long at = __shfl(mine[t], r);
        if (wrow + 32 * t + r < rows)
          *reinterpret_cast<u32x4*>(static_cast<T*>(a.out) + at + c * (16 / E)) =
              *reinterpret_cast<const u32x4*>(so + r * ROW + ((c ^ (r & 7)) << 4));
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
  }
};

template <typename T, int DH, int WAVES, int RT>
__global__ __launch_bounds__(64 * WAVES, 2) void prompt_kernel(PromptCall a) {
  typedef Walk<T, DH, WAVES, RT> W;
  __shared__ __attribute__((aligned(1024))) unsigned char ring[4 * W::BYTES];
  __shared__ int again;
  if (threadIdx.x == 0) again = 0;
  const W w(a, ring);
  if (w.row0 < w.rows) w.run(&again);
}

template <typename T, int DH, int WAVES, int RT>
void prompt_at(PromptCall& a, hipStream_t s) {
  const int64_t slots = (int64_t)a.n_q * a.group / (32 * RT * WAVES) + a.n_seqs;
  a.n_slots = (int)slots;
  hipLaunchKernelGGL((prompt_kernel<T, DH, WAVES, RT>), dim3((unsigned)(slots * a.n_kv)),
                     dim3(64 * WAVES), 0, s, a);
}

}  // namespace

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
  if constexpr (sizeof(T) == 2) {
    switch (x.head_dim) {
      case 64: return prompt_at<T, 64, 4, 2>(a, s);
      case 128: return prompt_at<T, 128, 4, 2>(a, s);
      case 192: return prompt_at<T, 192, 8, 1>(a, s);
      default: return prompt_at<T, 256, 8, 1>(a, s);
    }
  } else {
    switch (x.head_dim) {
      case 64: return prompt_at<T, 64, 4, 1>(a, s);
      case 128: return prompt_at<T, 128, 4, 1>(a, s);
      case 192: return prompt_at<T, 192, 4, 1>(a, s);
      default: return prompt_at<T, 256, 4, 1>(a, s);
    }
  }
}
template void launch_prompt<bf16_t>(const fv_prompt_args&, hipStream_t);
template void launch_prompt<float>(const fv_prompt_args&, hipStream_t);

}  // namespace fv
