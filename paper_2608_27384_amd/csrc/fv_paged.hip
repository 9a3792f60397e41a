// Attention of one new token a sequence over the pages of a cache.
//
// Every key and value is read once and used for the few query heads that share
// its kv head, so memory bounds it: the kernel is built around many wide loads
// in flight.  A sequence's keys are split into chunks, one workgroup each (per
// kv head and tile of 16 query heads), and a chunk's tiles among four waves that
// do not wait for each other: every wave runs its own softmax (running maximum
// and sum) over its own tiles, from memory straight into registers.  The waves
// join in LDS at the end, the chunks in a second kernel, both in a fixed order.
//
// Per tile S^T = K Q^T by MFMA (the queries are the columns, 16 of them, padded),
// so a lane holds scores of one query head for four consecutive keys of each 16,
// which is, without data movement, the operand that O^T += V^T P^T wants.  V^T
// needs keys along a lane: a lane loads 16 bytes (8 bf16 elements) of each of
// its own 8 keys, one 256-byte row per 16 lanes, and turns the 8x8 block over in
// registers (32 byte permutes, nothing beside the loads); which element of the
// head a matrix row stands for is free, and chosen so that this works out.
// bf16 values meet each probability in two parts, its upper 8 bits and what they
// leave, so that 16 bits count (2^-16 of it is lost, 2^-8 with one part: the error
// against 64 bits was 1.2 to 1.3 times that of exact probabilities).  A lowest bit
// that is always set keeps the second part above zero, where an infinite value would
// lose its infinity to 0 * inf.  Half as many products again, us with one part and with
// two: 64 rows of 816 keys 14.3 and 14.8, 32 of 1000 to 4000 23.9 and 24.3 (heads 8/1 of
// 256), 192 of 1 to 8191 522 and 522 (32/8 of 128).
//
// Measured (a read of memory alone reaches 6.2 TB/s): 192 rows of 1 to 8191 keys, heads
// 32/8 of 128, 524 us (6.2 TB/s); 192 of 1 to 16000, 8/1 of 256, 290 us (5.5); 64 of 816,
// 14 us; 1 of 816, 11 us, as a caller sees them.
#include "fv_context.h"

namespace fv {
namespace {

constexpr int kPagedWaves = 4;
constexpr float kLog2e = 1.4426950408889634f;

// Largest of the lanes l, l ^ 16, l ^ 32, l ^ 48.
__device__ __forceinline__ float max_xor16_32(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const float y = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(y), __float_as_uint(y), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

struct PagedCall {
  const void *q, *k, *v;  // the pools of the layer
  void* out;
  const int *seqs, *table, *len;
  float* part;  // [n][n_chunks][heads][DH] sums, then [n][n_chunks][heads][2] maximum and sum
  float* stat;
  int ldq, ldo, n, heads, n_kv, group, q_tiles, page_len, n_pages, max_seqs, max_pages;
  uint32_t per_page;  // 2^31 over a page's runs of 16 rows, rounded up
  int chunk, n_chunks;
  float scale;  // of the scores, in log2 units
};

// Chunks of a sequence that hold keys.  The last workgroup takes what lies past
// the planned bound, should a sequence be longer.
__device__ __forceinline__ int chunks_of(int len, int chunk, int n_chunks) {
  const int c = (len + chunk - 1) / chunk;
  return c < n_chunks ? c : n_chunks;
}
__device__ __forceinline__ int length_of(const PagedCall& a, int s) {
  return min(max(a.len[s], 0), a.max_pages * a.page_len);
}

// A V tile in registers, and its matrix operands.  bf16: 32 keys, 8 a lane
// (4g .. 4g+3 of either half); the head's 128-element blocks 8 elements a lane,
// a last block of 64 four.  fp32: 16 keys, 4 a lane, blocks of 64, 4 elements.
template <typename T, int DH, bool STREAM> struct VTile;

template <int DH, bool STREAM> struct VTile<bf16_t, DH, STREAM> {
  static constexpr int B8 = DH / 128, B4 = (DH % 128) / 64;
  u32x4 w[B8 > 0 ? B8 : 1][8];
  u32x2 n[8];
  __device__ __forceinline__ void load(const bf16_t* const (&row)[2], int l16, int lg) {
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      const bf16_t* p = row[x >> 2] + (size_t)(4 * lg + (x & 3)) * DH;
#pragma unroll
      for (int b = 0; b < B8; ++b) w[b][x] = load_piece<STREAM>(reinterpret_cast<const u32x4*>(p + 128 * b + 8 * l16));
      if (B4) n[x] = load_piece<STREAM>(reinterpret_cast<const u32x2*>(p + 128 * B8 + 4 * l16));
    }
  }
  __device__ __forceinline__ void drop(int x) {  // key x of the lane is not there
#pragma unroll
    for (int b = 0; b < B8; ++b) w[b][x] = u32x4{0, 0, 0, 0};
    if (B4) n[x] = u32x2{0, 0};
  }
  // operand of tile t: element t % 8 of the lane's in block t / 8 (t % 4 of the last 64)
  __device__ __forceinline__ u32x4 operand(int t) const {
    const int b = t / 8, j = b < B8 ? t % 8 : t - 8 * B8;
    const uint32_t sel = j & 1 ? 0x07060302u : 0x05040100u;
    u32x4 r;
#pragma unroll
    for (int y = 0; y < 4; ++y)
      r[y] = b < B8 ? __builtin_amdgcn_perm(w[b < B8 ? b : 0][2 * y + 1][j >> 1],
                                            w[b < B8 ? b : 0][2 * y][j >> 1], sel)
                    : __builtin_amdgcn_perm(n[2 * y + 1][(j >> 1) & 1], n[2 * y][(j >> 1) & 1], sel);
    return r;
  }
};

template <int DH, bool STREAM> struct VTile<float, DH, STREAM> {
  u32x4 w[DH / 64][4];
  __device__ __forceinline__ void load(const float* const (&row)[1], int l16, int lg) {
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int b = 0; b < DH / 64; ++b)
        w[b][x] = load_piece<STREAM>(
            reinterpret_cast<const u32x4*>(row[0] + (size_t)(4 * lg + x) * DH + 64 * b + 4 * l16));
  }
  __device__ __forceinline__ void drop(int x) {
#pragma unroll
    for (int b = 0; b < DH / 64; ++b) w[b][x] = u32x4{0, 0, 0, 0};
  }
  __device__ __forceinline__ u32x4 operand(int t) const {
    return u32x4{w[t / 4][0][t % 4], w[t / 4][1][t % 4], w[t / 4][2][t % 4], w[t / 4][3][t % 4]};
  }
};

// Head element of matrix row i of tile t.
template <typename T, int DH> __device__ __forceinline__ int element_of(int t, int i) {
  if (sizeof(T) == 4) return 64 * (t / 4) + 4 * i + t % 4;
  constexpr int B8 = DH / 128;
  return t / 8 < B8 ? 128 * (t / 8) + 8 * i + t % 8 : 128 * B8 + 4 * i + (t - 8 * B8);
}

template <typename T, int DH, bool STREAM>
__global__ __launch_bounds__(64 * kPagedWaves, 2) void paged_kernel(PagedCall a) {
  constexpr int NH = sizeof(T) == 2 ? 2 : 1;       // 16-key halves of a tile
  constexpr int KT = 16 * NH;                      // keys of a tile
  constexpr int KB = DH * (int)sizeof(T) / 64;     // 64-byte blocks of a head
  constexpr int EB = 64 / (int)sizeof(T);          // elements of one
  constexpr int NT = DH / 16;                      // tiles of O^T
  __shared__ float sm[kPagedWaves][16], sl[kPagedWaves][16];
  __shared__ __attribute__((aligned(16))) float so[kPagedWaves][16][DH + 4];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int l16 = lane & 15, lg = lane >> 4;
  int id = blockIdx.x;
  const int qt = id % a.q_tiles;
  id /= a.q_tiles;
  const int kh = id % a.n_kv;
  id /= a.n_kv;
  // Workgroups go to the eight dies in turn, and a sequence's last chunks are often empty: each
  // row begins one chunk further on, or a number of chunks that eight divides would leave some
  // dies with full chunks only (64 rows of 500..3001 keys, fp32 x 256: 85 us so, 68 with it).
  const int row = id / a.n_chunks, ch = (id + row) % a.n_chunks;
  const int s = a.seqs[row];
  if (s < 0 || s >= a.max_seqs) return;
  const int k0 = ch * a.chunk;
  const int* table = a.table + (size_t)s * a.max_pages;
  // Page number of the 16 keys from `key` on, a multiple of 16 below 2^25: with m = page_len / 16
  // up to 16, the rounded up quotient is exact while key / 16 * (m - 1) stays below 2^31.
  auto page_of = [&](int key) __attribute__((always_inline)) { return (int)__umulhi(key >> 3, a.per_page); };
  auto page_at = [&](int key) __attribute__((always_inline)) {
    const int p = page_of(key);
    return p < a.max_pages ? table[p] : -1;
  };
  // First key of the half that a lane looks up (below), past that of its wave's tile `base`; in
  // one register, which the compiler would make two.
  int ahead = kPagedWaves * (lane / NH) * KT + 16 * (lane % NH);
  asm volatile("" : "+v"(ahead));
  // the first page numbers are fetched together with the length
  int page = page_at(k0 + wave * KT + ahead);
  const int len = length_of(a, s);
  const int chunks = chunks_of(len, a.chunk, a.n_chunks);
  if (ch >= chunks && ch > 0) return;
  const int k1 = ch == a.n_chunks - 1 ? len : min(len, k0 + a.chunk);

  // queries: the head of column l16, zeros past the group
  const int head = qt * 16 + l16;
  u32x4 qf[KB];
  {
    const T* q = static_cast<const T*>(a.q) + (size_t)row * a.ldq + (kh * a.group + head) * DH;
#pragma unroll
    for (int b = 0; b < KB; ++b)
      qf[b] = head < a.group
                  ? *reinterpret_cast<const u32x4*>(q + EB * b + (EB / 4) * lg)
                  : u32x4{0, 0, 0, 0};
  }

  f32x4 o[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;  // of the lane's query; l over the lane's keys only
  bool any = false;              // a key was seen

  const T* kp = static_cast<const T*>(a.k);
  const T* vp = static_cast<const T*>(a.v);
  const int tiles = (k1 - k0 + KT - 1) / KT;
  // Page numbers 64 halves at a time: lane i holds half i % NH of the wave's tile base + i / NH.
  constexpr int GO = 64 / NH;
  for (int base = wave; base < tiles; base += kPagedWaves * GO) {
    const int myKey = k0 + base * KT + ahead;
    if (base != wave) page = page_at(myKey);
    // page and row / 16 in one register (a page has at most 256 rows), -1: no keys
    const int half = myKey >= k1 || page < 0 || page >= a.n_pages ? -1 : page << 4 | (myKey - page_of(myKey) * a.page_len) >> 4;
    const int here = min(GO, (tiles - base + kPagedWaves - 1) / kPagedWaves);
    // first rows of a tile's halves, and how many of their keys are there
    auto rows = [&](int it, const T* pool, const T* (&row)[NH], int (&left)[NH]) __attribute__((always_inline)) {
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        const int at = __builtin_amdgcn_readlane(half, it * NH + h);
        left[h] = at < 0 ? 0 : min(16, k1 - (k0 + (base + kPagedWaves * it) * KT + 16 * h));
        row[h] = pool + (page_row(max(at, 0) >> 4, a.n_kv, kh, a.page_len) + 16 * (max(at, 0) & 15)) * DH;
      }
    };
    u32x4 kf[NH][KB];
    auto load_keys = [&](int it) __attribute__((always_inline)) {
      const T* row[NH];
      int left[NH];
      rows(it, kp, row, left);
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int b = 0; b < KB; ++b)
          kf[h][b] = load_piece<STREAM>(
              reinterpret_cast<const u32x4*>(row[h] + (size_t)l16 * DH + EB * b + (EB / 4) * lg));
    };
    load_keys(0);
    for (int it = 0; it < here; ++it) {
      const T* vrow[NH];
      int left[NH];
      rows(it, vp, vrow, left);
      VTile<T, DH, STREAM> vt;
      vt.load(vrow, l16, lg);

      f32x4 sc[NH];
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        sc[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int b = 0; b < KB; ++b) sc[h] = mma64(kf[h][b], qf[b], sc[h], T{});
      }
      __builtin_amdgcn_sched_barrier(0);
      if (it + 1 < here) load_keys(it + 1);  // while the softmax and the values are at work
      bool whole = true;
#pragma unroll
      for (int h = 0; h < NH; ++h) {
        whole = whole && left[h] == 16;
        any = any || left[h] > 0;
      }
      if (!whole) {  // keys that are not there: no weight, and values that hold nothing
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (4 * lg + r >= left[h]) {
              sc[h][r] = -INFINITY;
              vt.drop(4 * h + r);
            }
      }
      float top = -INFINITY;
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          sc[h][r] *= a.scale;
          top = fmaxf(top, sc[h][r]);
        }
      top = max_xor16_32(top);
      if (__any(top > m)) {
        const float now = fmaxf(m, top);
        const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - now);
        m = now;
        l *= f;
#pragma unroll
        for (int t = 0; t < NT; ++t) o[t] *= f;
      }
      const float ref = m == -INFINITY ? 0.f : m;
      u32x4 pf, rest;
      if constexpr (sizeof(T) == 2) {
        u16x8 pb, rb;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const uint32_t p = __float_as_uint(__builtin_amdgcn_exp2f(sc[h][r] - ref)) | 1;
            l += __uint_as_float(p);
            pb[4 * h + r] = (bf16_t)(p >> 16);
            rb[4 * h + r] = f32_to_bf16(__uint_as_float(p) - __uint_as_float(p & 0xffff0000u));
          }
        pf = __builtin_bit_cast(u32x4, pb);
        rest = __builtin_bit_cast(u32x4, rb);
      } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float p = __builtin_amdgcn_exp2f(sc[0][r] - ref);
          l += p;
          pf[r] = __float_as_uint(p);
        }
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const u32x4 v = vt.operand(t);
        o[t] = mma64(v, pf, o[t], T{});
        if constexpr (sizeof(T) == 2) o[t] = mma64(v, rest, o[t], T{});
      }
    }
  }

  // join the waves
  l = sum_xor16_32(l);
  if (lg == 0) {
    sm[wave][l16] = m;
    // a sequence of keys that all score -inf has no softmax: NaN, as 0/0
    sl[wave][l16] = any && m == -INFINITY ? 0.f : l;
  }
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) so[wave][l16][element_of<T, DH>(t, 4 * lg + r)] = o[t][r];
  __shared__ int seen[kPagedWaves];
  if (lane == 0) seen[wave] = any;
  __syncthreads();
  const int tid = threadIdx.x;
  const int heads_here = min(16, a.group - qt * 16);
  bool some = false;
#pragma unroll
  for (int w = 0; w < kPagedWaves; ++w) some = some || seen[w];
  for (int idx = tid; idx < heads_here * (DH / 4); idx += 64 * kPagedWaves) {
    const int hd = idx / (DH / 4), d = 4 * (idx % (DH / 4));
    float mm = -INFINITY;
#pragma unroll
    for (int w = 0; w < kPagedWaves; ++w) mm = fmaxf(mm, sm[w][hd]);
    const float ref = mm == -INFINITY ? 0.f : mm;
    float ll = 0.f;
    f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kPagedWaves; ++w) {
      const float f = __builtin_amdgcn_exp2f(sm[w][hd] - ref);
      ll += f * sl[w][hd];
      acc += f * *reinterpret_cast<const f32x4*>(&so[w][hd][d]);
    }
    const int qh = kh * a.group + qt * 16 + hd;
    if (a.n_chunks == 1) {
      const float inv = some ? 1.0f / ll : 0.f;
      store4(static_cast<T*>(a.out) + (size_t)row * a.ldo + qh * DH + d, acc[0] * inv, acc[1] * inv,
             acc[2] * inv, acc[3] * inv);
    } else {
      const size_t at = ((size_t)row * a.n_chunks + ch) * a.heads + qh;
      *reinterpret_cast<f32x4*>(a.part + at * DH + d) = acc;
      if (d == 0) {
        a.stat[2 * at] = some ? mm : -INFINITY;
        // no key at all: a sum of -1, which no other chunk has
        a.stat[2 * at + 1] = some ? ll : -1.f;
      }
    }
  }
}

// Joins a row's chunks: a workgroup per (row, head), its WAVES waves taking every
// WAVES-th chunk, four elements a lane.  The first chunks' sums are fetched together
// with the length, before it is known which of them hold anything; chunk c's maximum
// and sum are a lane's, which makes the chunk's weight of them.
template <typename T, int DH, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void paged_join_kernel(PagedCall a) {
  constexpr int FIRST = 8;
  __shared__ float weight[WAVES][64];
  __shared__ float sm[WAVES], sl[WAVES];
  __shared__ __attribute__((aligned(16))) float so[WAVES][DH];
  const int row = blockIdx.x / a.heads, qh = blockIdx.x - row * a.heads;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int s = a.seqs[row];
  const size_t at = (size_t)row * a.n_chunks * a.heads + qh;  // of chunk 0; the next is `heads` on
  const int d = 4 * lane < DH ? 4 * lane : 0;
  auto part = [&](int c) __attribute__((always_inline)) {
    return *reinterpret_cast<const f32x4*>(a.part + (at + (size_t)c * a.heads) * DH + d);
  };
  f32x4 x[FIRST];
#pragma unroll
  for (int i = 0; i < FIRST; ++i) x[i] = part(min(wave + i * WAVES, a.n_chunks - 1));
  if (s < 0 || s >= a.max_seqs) return;
  const int chunks = max(1, chunks_of(length_of(a, s), a.chunk, a.n_chunks));
  const int mine = (chunks - wave + WAVES - 1) / WAVES;  // chunks of this wave, may be none

  float m = -INFINITY, l = -1.f;  // a sum of -1: no key
  f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int i0 = 0; i0 < mine; i0 += 64) {
    const int n = min(64, mine - i0);
    float mc = -INFINITY, lc = -1.f;
    if (lane < n) {
      const float* st = a.stat + 2 * (at + (size_t)(wave + (i0 + lane) * WAVES) * a.heads);
      mc = st[0];
      lc = st[1];
    }
    const bool here = lc != -1.f;
    if (!__any(here)) continue;
    float now = fmaxf(m, mc);
#pragma unroll
    for (int y = 1; y < 64; y <<= 1) now = fmaxf(now, __shfl_xor(now, y));
    const float ref = now == -INFINITY ? 0.f : now;
    const float old = l == -1.f ? 0.f : __builtin_amdgcn_exp2f(m - ref);
    const float f = here ? __builtin_amdgcn_exp2f(mc - ref) : 0.f;
    l = (l == -1.f ? 0.f : l * old) + wave_sum(here ? f * lc : 0.f);
    m = now;
    acc *= old;
    weight[wave][lane] = here ? f : -1.f;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (i0 == 0) {
#pragma unroll
      for (int i = 0; i < FIRST; ++i)
        if (i < n && weight[wave][i] != -1.f) acc += weight[wave][i] * x[i];
    }
#pragma unroll 8
    for (int i = i0 == 0 ? FIRST : 0; i < n; ++i) {
      const float w = weight[wave][i];
      const f32x4 y = part(wave + (i0 + i) * WAVES);
      if (w != -1.f) acc += w * y;
    }
  }
  if constexpr (WAVES > 1) {
    if (lane == 0) {
      sm[wave] = m;
      sl[wave] = l;
    }
    if (4 * lane < DH) *reinterpret_cast<f32x4*>(&so[wave][d]) = acc;
    __syncthreads();
    if (wave) return;
    m = -INFINITY;
    for (int w = 0; w < WAVES; ++w) m = fmaxf(m, sm[w]);
    const float ref = m == -INFINITY ? 0.f : m;
    l = -1.f;
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < WAVES; ++w)
      if (sl[w] != -1.f) {
        const float f = __builtin_amdgcn_exp2f(sm[w] - ref);
        l = (l == -1.f ? 0.f : l) + f * sl[w];
        acc += f * *reinterpret_cast<const f32x4*>(&so[w][d]);
      }
  }
  if (4 * lane >= DH) return;
  const float inv = l == -1.f ? 0.f : 1.0f / l;
  store4(static_cast<T*>(a.out) + (size_t)row * a.ldo + qh * DH + d, acc[0] * inv, acc[1] * inv,
         acc[2] * inv, acc[3] * inv);
}

template <typename T, int DH>
void paged_at(const PagedCall& a, size_t bytes, hipStream_t s) {
  const int blocks = a.n * a.n_chunks * a.n_kv * a.q_tiles;
  if (bytes > kStreamBytes)
    hipLaunchKernelGGL((paged_kernel<T, DH, true>), dim3(blocks), dim3(64 * kPagedWaves), 0, s, a);
  else
    hipLaunchKernelGGL((paged_kernel<T, DH, false>), dim3(blocks), dim3(64 * kPagedWaves), 0, s, a);
  // us of both kernels with eight waves and with one: 10.3 and 9.6 at 7 chunks, 10.6 and
  // 10.3 at 16, 10.8 and 11.5 at 32, 15 and 28 at 219 (one row, 8/1 of 256).
  if (a.n_chunks > 16)
    hipLaunchKernelGGL((paged_join_kernel<T, DH, 8>), dim3(a.n * a.heads), dim3(512), 0, s, a);
  else if (a.n_chunks > 1)
    hipLaunchKernelGGL((paged_join_kernel<T, DH, 1>), dim3(a.n * a.heads), dim3(64), 0, s, a);
}

}  // namespace

PagedPlan plan_paged(int n, int n_q_heads, int n_kv_heads, int head_dim, int max_keys, bool bf16) {
  PagedPlan p{};
  const int64_t cols = (int64_t)n * n_kv_heads * ((n_q_heads / n_kv_heads + 15) / 16);
  // 2048 workgroups fill the chip (two to four a CU at a time) and leave room for ragged
  // lengths: 64 rows of 1 to 8000 keys, heads 4/2 of 192, 83 us, with 1024 of them 91; 64 of 500
  // to 3001, fp32, 8/1 of 256, 65 and 76; 192 of 1 to 16000, 292 and 335; alike lengths want fewer
  // (256 of 8000 362 and 336).  A chunk is at least one tile of each wave and at most 2048 keys:
  // 192 rows of 1 to 8191 keys, 32/8 of 128, 526 us, with at most 512, 1024 and 4096 keys 564,
  // 551 and 657; 192 of 1 to 16000, 8/1 of 256, 292, and 320, 296 and 292.
  const int least = kPagedWaves * (bf16 ? 32 : 16);
  int64_t chunk = ((int64_t)max_keys * cols + 2047) / 2048;
  chunk = (chunk + least - 1) / least * least;
  if (chunk < least) chunk = least;
  if (chunk > 2048) chunk = 2048;
  int64_t chunks = (max_keys + chunk - 1) / chunk;
  if (chunks < 1) chunks = 1;
  while (chunks > 1 && chunks * cols > 1 << 23) chunks /= 2;  // the grid's limit: longer last chunks
  p.keys = max_keys;
  p.chunk = (int)chunk;
  p.n_chunks = (int)chunks;
  if (chunks > 1) {
    const size_t rows = (size_t)n * chunks * n_q_heads;
    p.work_bytes = rows * (head_dim + 2) * 4;
  }
  return p;
}

template <typename T>
void launch_paged(const fv_paged_args& x, const fv_pages& c, const PagedPlan& p, hipStream_t s) {
  PagedCall a{};
  const size_t layer = (size_t)x.layer * page_row(c.n_pages, c.n_kv_heads, 0, c.page_len) * c.head_dim;
  a.q = x.q;
  a.k = static_cast<const T*>(c.k) + layer;
  a.v = static_cast<const T*>(c.v) + layer;
  a.out = x.out;
  a.seqs = x.seqs;
  a.table = c.table;
  a.len = c.len;
  a.part = static_cast<float*>(x.work);
  a.stat = a.part + (size_t)x.n * p.n_chunks * x.n_q_heads * c.head_dim;
  a.ldq = x.ldq;
  a.ldo = x.ldo;
  a.n = x.n;
  a.heads = x.n_q_heads;
  a.n_kv = c.n_kv_heads;
  a.group = x.n_q_heads / c.n_kv_heads;
  a.q_tiles = (a.group + 15) / 16;
  a.page_len = c.page_len;
  a.per_page = (uint32_t)(((1ull << 31) + c.page_len / 16 - 1) / (c.page_len / 16));
  a.n_pages = c.n_pages;
  a.max_seqs = c.max_seqs;
  a.max_pages = c.max_pages;
  a.chunk = p.chunk;
  a.n_chunks = p.n_chunks;
  a.scale = x.scale * kLog2e;
  // what the call may read: the keys and values planned for, which a layer's pages bound
  const size_t key = 2 * (size_t)c.n_kv_heads * c.head_dim * sizeof(T);
  const size_t planned = (size_t)x.n * p.keys * key, pages = (size_t)c.n_pages * c.page_len * key;
  const size_t bytes = planned < pages ? planned : pages;
  switch (c.head_dim) {
    case 64: return paged_at<T, 64>(a, bytes, s);
    case 128: return paged_at<T, 128>(a, bytes, s);
    case 192: return paged_at<T, 192>(a, bytes, s);
    default: return paged_at<T, 256>(a, bytes, s);
  }
}
template void launch_paged<bf16_t>(const fv_paged_args&, const fv_pages&, const PagedPlan&, hipStream_t);
template void launch_paged<float>(const fv_paged_args&, const fv_pages&, const PagedPlan&, hipStream_t);

}  // namespace fv
