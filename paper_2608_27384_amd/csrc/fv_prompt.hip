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

// Value operands of keys that only some rows of a wave see.  A weight of zero
// does not silence a value that is not finite, so such values are taken out of
// the product; `plus` and `minus` hold a one for +inf and -inf, both for NaN.
struct Unruly {
  u32x4 plus, minus;
};
__device__ __forceinline__ bool has_unruly(u32x4 x, bf16_t) {
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    any |= ((x[i] & 0x7f80u) == 0x7f80u) | ((x[i] & 0x7f800000u) == 0x7f800000u);
  return __any(any);
}
__device__ __forceinline__ Unruly take_unruly(u32x4& x, bf16_t) {
  Unruly u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t keep = 0, plus = 0, minus = 0;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const uint32_t b = x[i] >> (16 * half) & 0xffffu;
      const bool bad = (b & 0x7f80u) == 0x7f80u, nan = (b & 0x7fffu) > 0x7f80u;
      keep |= (bad ? 0u : b) << (16 * half);
      plus |= (bad && (nan || b == 0x7f80u) ? 0x3f80u : 0u) << (16 * half);
      minus |= (bad && (nan || b == 0xff80u) ? 0x3f80u : 0u) << (16 * half);
    }
    x[i] = keep;
    u.plus[i] = plus;
    u.minus[i] = minus;
  }
  return u;
}
// Adds what the seen ones among them make of the sums: an infinity, or NaN.
__device__ __forceinline__ void add_unruly(f32x16& o, const f32x16& plus, const f32x16& minus) {
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    o[r] += plus[r] > 0.f ? INFINITY : 0.f;
    o[r] -= minus[r] > 0.f ? INFINITY : 0.f;
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

template <typename T, int DH> struct PromptTile {
  static constexpr int KT = sizeof(T) == 2 ? 64 : 32;  // keys of a tile
  static constexpr int PIECES = DH * (int)sizeof(T) / 16;
  static constexpr int ROW = DH * (int)sizeof(T);
  static constexpr int BYTES = KT * ROW;  // of K, and of V
};

template <typename T, int DH, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void prompt_kernel(PromptCall a) {
  using G = PromptTile<T, DH>;
  constexpr int KT = G::KT, PIECES = G::PIECES, ROW = G::ROW, BYTES = G::BYTES;
  constexpr int R = 32 * WAVES;
  constexpr int ND = DH / 32;                      // 32-row tiles of O^T
  constexpr int NI = BYTES / 1024 / WAVES;         // direct loads of a wave per tensor and tile
  constexpr int E = (int)sizeof(T);
  static_assert(NI * 1024 * WAVES == BYTES && R * ROW <= 4 * BYTES, "tile split");
  __shared__ __attribute__((aligned(1024))) unsigned char ring[4 * BYTES];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int l32 = lane & 31, lh = lane >> 5;
  // the heaviest tiles of a causal prompt, its last ones, go first
  const int kh = blockIdx.x % a.n_kv, slot = a.n_slots - 1 - (int)(blockIdx.x / a.n_kv);
  int first;
  const int s = prompt_of<R>(a, slot, &first);
  const int q0 = clamped(a.cu_q, s, a.n_q), k0 = clamped(a.cu_k, s, a.n_k);
  const int nq = max(0, clamped(a.cu_q, s + 1, a.n_q) - q0);
  const int nk = max(0, clamped(a.cu_k, s + 1, a.n_k) - k0);
  const int rows = nq * a.group, row0 = (slot - first) * R;
  if (row0 >= rows) return;

  // visible keys [0, lim) of the lane's row, of the wave's first and last, of the block's last
  const int wrow = row0 + 32 * wave;
  const int diff = nk - nq + 1;
  auto limit = [&](int row) {
    return a.causal ? min(max(diff + min(row, rows - 1) / a.group, 0), nk) : nk;
  };
  const int row = min(wrow + l32, rows - 1), tok = row / a.group, head = kh * a.group + row - tok * a.group;
  const int lim = limit(row);
  const int full = limit(wrow), wend = wrow < rows ? limit(wrow + 31) : 0;
  const int tiles = (limit(row0 + R - 1) + KT - 1) / KT;

  u32x4 qf[PIECES / 2];
  {
    const T* q = static_cast<const T*>(a.q) + (size_t)(q0 + tok) * a.ldq + head * DH;
#pragma unroll
    for (int p = 0; p < PIECES / 2; ++p)
      qf[p] = *reinterpret_cast<const u32x4*>(q + (2 * p + lh) * (16 / E));
  }

  // Direct loads: slot u of a tile, 16 bytes, is piece u % PIECES of row u / PIECES.
  const T* kbase = static_cast<const T*>(a.k) + (size_t)k0 * a.ldk + kh * DH;
  const T* vbase = static_cast<const T*>(a.v) + (size_t)k0 * a.ldv + kh * DH;
  auto issue = [&](int t, int stage) __attribute__((always_inline)) {
    unsigned char* to = ring + stage * 2 * BYTES + wave * NI * 1024;
    const lds_src ks = lds_source(kbase + (size_t)t * KT * a.ldk);
    const lds_src vs = lds_source(vbase + (size_t)t * KT * a.ldv);
    const int most = nk - 1 - t * KT;  // rows past the prompt's last repeat it
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int u = 64 * (NI * wave + i) + lane, r = u / PIECES;
      const int c = (u % PIECES) ^ swizzle<T, DH>(r), rr = min(r, most);
      lds_dma16(ks, to + 1024 * i, rr * a.ldk * E + 16 * c, 0);
      lds_dma16(vs, to + BYTES + 1024 * i, rr * a.ldv * E + 16 * c, 0);
    }
  };

  f32x16 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
  float m = -INFINITY, l = 0.f;  // l over the lane half's keys only

  const int ksw = swizzle<T, DH>(l32);
  if (tiles > 0) issue(0, 0);
  for (int t = 0; t < tiles; ++t) {
    // this wave's part of tile t has landed and its reads of tile t - 1 are
    // done; past the barrier both hold for every wave
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (t + 1 < tiles) issue(t + 1, (t + 1) & 1);
    const unsigned char* sk = ring + (t & 1) * 2 * BYTES;
    const unsigned char* sv = sk + BYTES;
#pragma unroll
    for (int sub = 0; sub < KT / 32; ++sub) {
      const int key0 = t * KT + 32 * sub;
      if (key0 >= wend) break;
      f32x16 sc;
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[r] = 0.f;
#pragma unroll
      for (int p = 0; p < PIECES / 2; ++p) {
        const u32x4 kf = *reinterpret_cast<const u32x4*>(sk + (32 * sub + l32) * ROW +
                                                         (((2 * p + lh) ^ ksw) << 4));
        sc = mma32(kf, qf[p], sc, T{});
      }
      const bool edge = key0 + 32 > full;  // some row of the wave does not see all 32 keys
      if (edge) {
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
#pragma unroll
        for (int d = 0; d < ND; ++d) o[d] *= f;
      }
      const float ref = m == -INFINITY ? 0.f : -m;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        sc[r] = __builtin_amdgcn_exp2f(fmaf(sc[r], a.scale, ref));
        l += sc[r];
      }
      if constexpr (E == 2) {
        u32x4 pf[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          u16x8 w;
#pragma unroll
          for (int e = 0; e < 8; ++e) w[e] = f32_to_bf16(sc[8 * c + e]);
          pf[c] = __builtin_bit_cast(u32x4, w);
        }
        const int i = lane & 15, grp = (lane >> 4) & 1;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const int key = 32 * sub + 16 * c + 4 * lh + (i >> 2);
            const int piece = 4 * d + 2 * grp + ((i >> 1) & 1);
            const u32x2 a0 = read_transposed(sv + key * ROW + ((piece ^ swizzle<T, DH>(key)) << 4) + (i & 1) * 8);
            const u32x2 a1 = read_transposed(sv + (key + 8) * ROW + ((piece ^ swizzle<T, DH>(key + 8)) << 4) + (i & 1) * 8);
            u32x4 vf = u32x4{a0[0], a0[1], a1[0], a1[1]};
            if (edge && has_unruly(vf, T{})) {
              const Unruly bad = take_unruly(vf, T{});
              u16x8 seen;
#pragma unroll
              for (int e = 0; e < 8; ++e)
                seen[e] = key0 + 16 * c + 8 * (e >> 2) + 4 * lh + (e & 3) < lim ? 0x3f80 : 0;
              const u32x4 w = __builtin_bit_cast(u32x4, seen);
              add_unruly(o[d], mma32(bad.plus, w, zeros16(), T{}), mma32(bad.minus, w, zeros16(), T{}));
            }
            o[d] = mma32(vf, pf[c], o[d], T{});
          }
      } else {
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int key = 8 * (r >> 2) + 4 * lh + (r & 3);
            const int at = 32 * d + l32;
            float x = *reinterpret_cast<const float*>(
                sv + key * ROW + (((at >> 2) ^ swizzle<T, DH>(key)) << 4) + (at & 3) * 4);
            if (edge && __any(!(fabsf(x) < INFINITY))) {
              const float w = key0 + key < lim ? 1.f : 0.f;
              const bool ok = fabsf(x) < INFINITY;
              const float plus = !ok && !(x < 0.f) ? 1.f : 0.f, minus = !ok && !(x > 0.f) ? 1.f : 0.f;
              add_unruly(o[d], __builtin_amdgcn_mfma_f32_32x32x2f32(plus, w, zeros16(), 0, 0, 0),
                         __builtin_amdgcn_mfma_f32_32x32x2f32(minus, w, zeros16(), 0, 0, 0));
              x = ok ? x : 0.f;
            }
            o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, sc[r], o[d], 0, 0, 0);
          }
      }
    }
  }

  // Rows go out whole, through LDS.  No key seen: zeros; keys that all score
  // -inf: 0/0, as the formula has it.
  l = other_half_sum(l);
  const float inv = lim > 0 ? 1.0f / l : 0.f;
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  unsigned char* so = ring + wave * 32 * ROW;
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int at = 32 * d + 8 * j + 4 * lh;  // first of four elements
      T* p = reinterpret_cast<T*>(so + l32 * ROW + (((at * E >> 4) ^ (l32 & 7)) << 4) + (at * E & 15));
      store4(p, o[d][4 * j] * inv, o[d][4 * j + 1] * inv, o[d][4 * j + 2] * inv, o[d][4 * j + 3] * inv);
    }
  const long long mine = (long long)(q0 + tok) * a.ldo + head * DH;
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  for (int u = lane; u < 32 * PIECES; u += 64) {
    const int r = u / PIECES, c = u % PIECES;
    const long long at = __shfl(mine, r);
    if (wrow + r < rows)
      *reinterpret_cast<u32x4*>(static_cast<T*>(a.out) + at + c * (16 / E)) =
          *reinterpret_cast<const u32x4*>(so + r * ROW + ((c ^ (r & 7)) << 4));
  }
}

template <typename T, int DH, int WAVES>
void prompt_at(PromptCall& a, hipStream_t s) {
  const int64_t slots = (int64_t)a.n_q * a.group / (32 * WAVES) + a.n_seqs;
  a.n_slots = (int)slots;
  hipLaunchKernelGGL((prompt_kernel<T, DH, WAVES>), dim3((unsigned)(slots * a.n_kv)),
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
  constexpr int W = sizeof(T) == 2 ? 8 : 4;
  switch (x.head_dim) {
    case 64: return prompt_at<T, 64, W>(a, s);
    case 128: return prompt_at<T, 128, W>(a, s);
    case 192: return prompt_at<T, 192, W>(a, s);
    default: return prompt_at<T, 256, W>(a, s);
  }
}
template void launch_prompt<bf16_t>(const fv_prompt_args&, hipStream_t);
template void launch_prompt<float>(const fv_prompt_args&, hipStream_t);

}  // namespace fv
