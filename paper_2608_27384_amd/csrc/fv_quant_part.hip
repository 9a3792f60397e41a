// Attention of several new tokens a sequence over the pages of a cache in 8 bits: parts of
// prompts, chunks of actions.
//
// The query rows of one (entry, kv head) are its (token, head) pairs, token major, as in the
// attention over whole prompts (fv_prompt.hip): the heads that share a kv head share its
// keys, and the causal edge of a row tile spans few tokens.  Where there are few rows the keys
// are split into chunks, whose results a second kernel joins (fv_paged.hip's).
//
// Per 32 keys: S^T = K Q^T by 32x32 MFMA, so a lane holds 16 scores of one query; the
// probabilities are, without data movement, the operand of O^T += V^T P^T.  Codes become bf16
// operands by an exact conversion that applies the block's scale.  fp32 queries and
// probabilities go in as three parts of bf16 each, 24 bits.  In bf16 the queries are exact.  A
// probability is two parts, 16 bits, where there are few rows (50 tokens on 866 keys, heads 8/1
// of 256: 14.3 us, with one part 14.0).  In the kernels of 64 and 128 rows nothing would hide the
// products of a second part, and it is one bf16 number, off by up to 2^-8 of it: us with one and
// with two, the same heads, 64 parts of 1 to 61 tokens on 300 to 866 keys 32.4 and 45.5, 500 tokens
// on 8000 keys 54 and 67, 4096 on 28672 785 and 1087.  (The unit's products of codes as they are, at
// twice the rate, are not used: their inner sums are off by 2^-12 of the largest term, which scores
// of large keys cannot bear, and queries would need several parts.)
#include "fv_paged.h"
#include "fv_prompt.h"
#include "fv_quant.h"

#include <type_traits>

namespace fv {
namespace {

struct PartCall {
  const void* q;
  const unsigned char *k, *v;         // the pools of the layer
  const uint8_t *k_scale, *v_scale;   // and its scales
  void* out;
  const int *cu_q, *seqs, *table, *len;
  float *part, *stat;  // see PagedCall
  int ldq, ldo, n_seqs, n_q, heads, n_kv, group, causal, n_slots;
  int page_len, n_pages, max_seqs, max_pages, chunk, n_chunks;
  uint32_t per_page;  // 2^31 over a page's blocks, rounded up
  float scale;        // of the scores, in log2 units
};

// Codes of NaN in four of them, as a set highest bit each; the codes without them.
__device__ __forceinline__ uint32_t nans(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
__device__ __forceinline__ uint32_t without(uint32_t w, uint32_t n) { return w & ~(n | (n - (n >> 7))); }

// What a workgroup of R rows knows of its entry, and of the chunk of keys that is its own.
template <int R> struct PartRows {
  const PartCall& a;
  int lane, wave, l32, lh, kh, ch, q0, nq, nk, rows, row0, k0, k1;
  bool named;  // the entry names a sequence
  const int* table;
  int page0;   // of the chunk's key `at`: on its way while the length is

  __device__ __forceinline__ PartRows(const PartCall& call, int at) : a(call) {
    lane = threadIdx.x & 63;
    wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    l32 = lane & 31;
    lh = lane >> 5;
    // the heaviest tiles of a causal part, its last ones, go first
    int id = blockIdx.x;
    ch = id % a.n_chunks;
    id /= a.n_chunks;
    kh = id % a.n_kv;
    const int slot = a.n_slots - 1 - id / a.n_kv;
    int first, entry, q1, s;
    if (a.n_seqs < 64) {  // every offset and sequence in a lane
      const int cu = min(max(a.cu_q[min(lane, a.n_seqs)], 0), a.n_q), seq = a.seqs[min(lane, a.n_seqs - 1)];
      const int from = (int)((long long)cu * a.group / R) + lane;  // see prompt_of
      entry = max(1, (int)__popcll(__ballot(lane < a.n_seqs && from <= slot))) - 1;
      first = __builtin_amdgcn_readlane(from, entry);
      q0 = __builtin_amdgcn_readlane(cu, entry);
      q1 = __builtin_amdgcn_readlane(cu, entry + 1);
      s = __builtin_amdgcn_readlane(seq, entry);
    } else {
      entry = prompt_of<R>(a, slot, &first);
      q0 = clamped(a.cu_q, entry, a.n_q);
      q1 = clamped(a.cu_q, entry + 1, a.n_q);
      s = a.seqs[entry];
    }
    nq = max(0, q1 - q0);
    rows = nq * a.group;
    row0 = (slot - first) * R;
    named = s >= 0 && s < a.max_seqs;
    table = a.table + (size_t)(named ? s : 0) * a.max_pages;
    k0 = ch * a.chunk;
    page0 = page_at(k0 + at);
    nk = named ? min(max(a.len[s], 0), a.max_pages * a.page_len) : 0;
    k1 = min(ch == a.n_chunks - 1 ? nk : min(nk, k0 + a.chunk), limit(row0 + R - 1));
  }
  // False: a spare slot, or one that no entry has (offsets that do not ascend from 0).
  __device__ __forceinline__ bool any() const { return row0 >= 0 && row0 < rows; }
  // A row sees the keys [0, limit), which do not fall from one row to the next.
  __device__ __forceinline__ int limit(int row) const {
    return a.causal ? min(max(nk - nq + 1 + min(row, rows - 1) / a.group, 0), nk) : nk;
  }
  // Token and query head of a row.
  __device__ __forceinline__ void of(int row, int& tok, int& head) const {
    row = min(row, rows - 1);
    tok = row / a.group;
    head = kh * a.group + row - tok * a.group;
  }
  __device__ __forceinline__ size_t partial(int tok, int head) const {
    return ((size_t)(q0 + tok) * a.n_chunks + ch) * a.heads + head;
  }
  __device__ __forceinline__ void state(int tok, int head, float m, float l) const {
    const size_t at = partial(tok, head);
    a.stat[2 * at] = m;
    a.stat[2 * at + 1] = l;
  }
  // The chunk has keys for no row: says so, where there are several.
  __device__ __forceinline__ bool idle() const {
    if (k1 > k0 || (a.n_chunks == 1 && named)) return false;
    if (a.n_chunks > 1)
      for (int r = threadIdx.x; r < R; r += blockDim.x)
        if (row0 + r < rows) {
          int tok, head;
          of(row0 + r, tok, head);
          state(tok, head, -INFINITY, named ? kNoKey : kNoEntry);
        }
    return true;
  }
  // The pool's block of the 16 keys from `key` on (page and its block), or -1.  In two steps: the
  // table's entry can be on its way before the length is known.
  __device__ __forceinline__ int page_at(int key) const {
    const int p = (int)__umulhi(key >> 3, a.per_page);
    return p < a.max_pages ? table[p] : -1;
  }
  __device__ __forceinline__ int block_at(int key, int page) const {
    const int p = (int)__umulhi(key >> 3, a.per_page);
    return key >= k1 || page < 0 || page >= a.n_pages ? -1 : page << 4 | (key - p * a.page_len) >> 4;
  }
  __device__ __forceinline__ int block_at(int key) const { return key < k1 ? block_at(key, page_at(key)) : -1; }
  __device__ __forceinline__ size_t place(int at) const {
    return block_of(max(at, 0) >> 4, a.n_kv, kh, a.page_len, max(at, 0) & 15);
  }
  // Whether the value of position `key` is NaN at element d of the head.
  __device__ __forceinline__ bool is_nan(size_t block, int key, int d, int DH) const {
    const unsigned char* p = a.v + block * (16 * DH) + 256 * (key % 16 / 4) + key % 4;
    return (p[1024 * (d / 64) + 16 * (d % 16) + 4 * (d % 64 / 16)] & 127) == 127;
  }
};

// 16 probabilities as bf16 operands, in PARTS parts.
template <int PARTS>
__device__ __forceinline__ void probabilities(const f32x16& p, u32x4 (&pf)[2][PARTS]) {
  u16x8 w[2][PARTS];
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    bf16_t at[PARTS];
    split<PARTS>(p[r], at);
#pragma unroll
    for (int x = 0; x < PARTS; ++x) w[r / 8][x][r % 8] = at[x];
  }
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int x = 0; x < PARTS; ++x) pf[c][x] = __builtin_bit_cast(u32x4, w[c][x]);
}

constexpr int kPartWaves = 4;

// 32 rows a workgroup, whose waves share a chunk's keys out, straight from memory into registers,
// the next step's codes under way in the one before, and join in LDS.  For where there are so few
// rows that the time is the chain of trips to memory (offsets, the table with the length, scales
// and codes, then the join's): 50 tokens on 866 keys, 8 query heads and 1 kv head of 256, bf16, are
// 14.3 us with the join, of which two launches are 8; under 2 us of it are products.
template <typename T, int DH>
__global__ __launch_bounds__(64 * kPartWaves, 1) void quant_part_kernel(PartCall a) {
  constexpr int SLABS = DH / 64, NK = DH / 16, ND = DH / 32, PITCH = DH + 4;
  constexpr int PARTS = sizeof(T) == 2 ? 1 : 3, PP = sizeof(T) == 2 ? 2 : 3;  // of queries, of probabilities
  // fp32 queries of long heads are 144 or 192 registers in parts: they stay in LDS, where `so` comes
  // later.  50 tokens on 866 keys, 8/1 heads of 256, 16.5 us, in registers 20.0; 4/2 of 192 13.3, 14.2.
  constexpr bool PUT = PARTS == 3 && DH >= 192;
  __shared__ float sm[kPartWaves][32], sl[kPartWaves][32];
  __shared__ int seen_by[kPartWaves][32];
  __shared__ __attribute__((aligned(16))) float so[kPartWaves][32 * PITCH];
  u32x4* const put = reinterpret_cast<u32x4*>(&so[0][0]);
  // Lane l looks up the block of the wave's step l / 2, half l % 2; the wave's steps are
  // kPartWaves apart, so this is 32 of them.
  const int ahead = 32 * ((int)threadIdx.x >> 6) + 16 * ((int)threadIdx.x & 1) + 32 * kPartWaves * (((int)threadIdx.x & 63) >> 1);
  const PartRows<32> b(a, ahead);
  if (!b.any() || b.idle()) return;
  const int lane = b.lane, wave = b.wave, l32 = b.l32, lh = b.lh, row0 = b.row0, rows = b.rows, k0 = b.k0, k1 = b.k1;
  const int steps = max(0, (k1 - k0 + 31) / 32);
  int at = b.block_at(k0 + ahead, b.page0);
  auto scales_at = [&](int at) __attribute__((always_inline)) {
    const size_t x = b.place(at);
    return (uint32_t)a.k_scale[x] | (uint32_t)a.v_scale[x] << 8;
  };
  uint32_t scales = scales_at(at);
  int tok, head;
  b.of(row0 + l32, tok, head);
  const int lim = b.limit(row0 + l32);
  const int whole = b.limit(row0);  // keys that every row of the tile sees
  struct Tile {
    int at[2];
    uint32_t scales[2];
    u32x4 k[2 * SLABS];
    u32x2 v[SLABS][2][2];  // of block c, the positions from 4 lh + 8 h on
  };
  // A step that some row does not see whole, or whose keys are not all there: its values are sifted.
  auto is_edge = [&](int key0, int at0, int at1) __attribute__((always_inline)) {
    return key0 + 32 > whole || key0 + 32 > k1 || at0 < 0 || at1 < 0;
  };
  auto fetch = [&](int i, Tile& t) __attribute__((always_inline)) {
    const int j = 2 * (i / kPartWaves % 32);
    if (j == 0 && i >= kPartWaves) {
      at = b.block_at(k0 + 32 * (i - wave) + ahead);
      scales = scales_at(at);
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) t.at[c] = __builtin_amdgcn_readlane(at, j + c);
    const size_t p0 = b.place(t.at[0]), p1 = b.place(t.at[1]);
    const unsigned char* kp = a.k + (l32 < 16 ? p0 : p1) * (16 * DH) + 64 * (l32 & 15) + 16 * lh;
#pragma unroll
    for (int x = 0; x < 2 * SLABS; ++x) t.k[x] = *reinterpret_cast<const u32x4*>(kp + 1024 * (x / 2) + 32 * (x % 2));
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const unsigned char* vp = a.v + (c ? p1 : p0) * (16 * DH) + 256 * lh + 16 * (l32 & 15) + 8 * (l32 >> 4);
#pragma unroll
      for (int x = 0; x < SLABS; ++x)
#pragma unroll
        for (int h = 0; h < 2; ++h) t.v[x][c][h] = *reinterpret_cast<const u32x2*>(vp + 1024 * x + 512 * h);
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) t.scales[c] = __builtin_amdgcn_readlane((int)scales, j + c);
    __builtin_amdgcn_sched_barrier(0);
  };
  Tile now, next;
  if (wave < steps) fetch(wave, next);
  u32x4 qf[NK][PARTS];
  {
    const T* q = static_cast<const T*>(a.q) + (size_t)(b.q0 + tok) * a.ldq + head * DH;
#pragma unroll
    for (int p = 0; p < NK; ++p) {
      if (PUT && p % kPartWaves != wave) continue;
      query8(q + 64 * (p / 4) + 32 * (p / 2 % 2) + 16 * lh + 8 * (p % 2), qf[p]);
      if (PUT)
#pragma unroll
        for (int x = 0; x < PARTS; ++x) put[(p * PARTS + x) * 64 + lane] = qf[p][x];
    }
    if (PUT) __syncthreads();
  }
  f32x16 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) o[d] = zeros16();
  float m = -INFINITY, l = 0.f;  // l over the lane half's keys only
  bool unruly = false, seen = false;
  for (int i = wave; i < steps; i += kPartWaves) {
    now = next;
    if (i + kPartWaves < steps) fetch(i + kPartWaves, next);
    const int key0 = k0 + 32 * i, at0 = now.at[0], at1 = now.at[1];
    const bool edge = is_edge(key0, at0, at1);
    const float ks = power_of(scale_exponent((uint8_t)(l32 < 16 ? now.scales[0] : now.scales[1])));
    const float vs[2] = {power_of(scale_exponent((uint8_t)(now.scales[0] >> 8))),
                         power_of(scale_exponent((uint8_t)(now.scales[1] >> 8)))};
    auto& kf = now.k;
    auto& vf = now.v;
    f32x16 sc = zeros16();
#pragma unroll
    for (int p = 0; p < NK; ++p) {
      const u32x4 k = to_bf16x8(kf[p / 2][2 * (p % 2)], kf[p / 2][2 * (p % 2) + 1], ks);
#pragma unroll
      for (int x = 0; x < PARTS; ++x) sc = mma32(k, PUT ? put[(p * PARTS + x) * 64 + lane] : qf[p][x], sc, bf16_t{});
    }
    if (edge) {
      uint32_t odd = 0;
#pragma unroll
      for (int x = 0; x < SLABS; ++x)
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint32_t n = nans(vf[x][c][h][e]);
              odd |= n;
              vf[x][c][h][e] = without(vf[x][c][h][e], n);
            }
      unruly = unruly || __any(odd != 0);
      hide(sc, key0, lh, lim);
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if ((r < 8 ? at0 : at1) < 0) sc[r] = -INFINITY;
    }
    seen = seen || (at0 >= 0 && key0 < lim) || (at1 >= 0 && key0 + 16 < lim);
    u32x4 unused[2];
    softmax<float>(sc, false, key0, lh, lim, a.scale, m, l, unused,
                   [&](float f) __attribute__((always_inline)) {
#pragma unroll
                     for (int d = 0; d < ND; ++d) o[d] *= f;
                   },
                   [](int) {});
    u32x4 pf[2][PP];
    probabilities<PP>(sc, pf);
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const uint32_t lo = vf[d / 2][c][0][d % 2], hi = vf[d / 2][c][1][d % 2];
        const u32x4 v = u32x4{to_bf16<false>(lo, vs[c]), to_bf16<true>(lo, vs[c]), to_bf16<false>(hi, vs[c]),
                              to_bf16<true>(hi, vs[c])};
#pragma unroll
        for (int x = 0; x < PP; ++x) o[d] = mma32(v, pf[c][x], o[d], bf16_t{});
      }
  }

  // the waves' sums, brought to the rows' common reference, join in LDS
  l = other_half_sum(l);
  if (lh == 0) {
    sm[wave][l32] = m;
    sl[wave][l32] = l;
    seen_by[wave][l32] = seen;
  }
  __syncthreads();
  float all = 0.f, top = -INFINITY;
  bool any = false;
#pragma unroll
  for (int w = 0; w < kPartWaves; ++w) {
    top = fmaxf(top, sm[w][l32]);
    any = any || seen_by[w][l32];
  }
  const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
  for (int w = 0; w < kPartWaves; ++w) all += __builtin_amdgcn_exp2f(sm[w][l32] - ref) * sl[w][l32];
  const bool last = a.n_chunks == 1;
  // a row that sees no key: zeros; keys that all score -inf: 0/0, as the formula has it
  float f = __builtin_amdgcn_exp2f(m - ref);
  if (last) f = any ? f / all : 0.f;
  float* mine = so[wave];
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int at = 64 * (d / 2) + 16 * (2 * (j >> 1) + d % 2) + 8 * (j & 1) + 4 * lh;
      *reinterpret_cast<f32x4*>(mine + l32 * PITCH + at) =
          f32x4{o[d][4 * j] * f, o[d][4 * j + 1] * f, o[d][4 * j + 2] * f, o[d][4 * j + 3] * f};
    }
  if (unruly) {  // NaN among the values that were sifted: of the rows that see them
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    for (int i = wave; i < steps; i += kPartWaves) {
      const int from = k0 + 32 * i;
      const int at0 = __builtin_amdgcn_readfirstlane(b.block_at(from));
      const int at1 = __builtin_amdgcn_readfirstlane(b.block_at(from + 16));
      if (!is_edge(from, at0, at1)) continue;
      for (int key = from; key < min(from + 32, k1); ++key) {
        const int at = key < from + 16 ? at0 : at1;
        if (at < 0) continue;
        for (int d = lane; d < DH; d += 64) {
          const bool odd = b.is_nan(b.place(at), key, d, DH);
          if (!__any(odd)) continue;
          for (int r = 0; r < 32; ++r)
            if (key < __shfl(lim, r) && odd) mine[r * PITCH + d] = __builtin_nanf("");
        }
      }
    }
  }
  __syncthreads();
  constexpr int OUT = 32 * (DH / 4) / (64 * kPartWaves);
  f32x4 sum[OUT];
#pragma unroll
  for (int j = 0; j < OUT; ++j) {
    const int u = threadIdx.x + 64 * kPartWaves * j;
    const float* x = so[0] + u / (DH / 4) * PITCH + 4 * (u % (DH / 4));
    sum[j] = *reinterpret_cast<const f32x4*>(x);
#pragma unroll
    for (int w = 1; w < kPartWaves; ++w) sum[j] += *reinterpret_cast<const f32x4*>(x + w * 32 * PITCH);
  }
#pragma unroll
  for (int j = 0; j < OUT; ++j) {
    const int u = threadIdx.x + 64 * kPartWaves * j, r = u / (DH / 4), d = 4 * (u % (DH / 4));
    if (row0 + r >= rows) continue;
    int t, h;
    b.of(row0 + r, t, h);
    if (last)
      store4(static_cast<T*>(a.out) + (size_t)(b.q0 + t) * a.ldo + h * DH + d, sum[j][0], sum[j][1], sum[j][2], sum[j][3]);
    else
      *reinterpret_cast<f32x4*>(a.part + b.partial(t, h) * DH + d) = sum[j];
  }
  if (!last && wave == 0 && lh == 0 && row0 + l32 < rows)
    b.state(tok, head, any ? top : -INFINITY, any ? all : kNoKey);
}

// Four waves with 32 rows each share the keys: tiles of 32 KG, as codes, go from memory straight
// into LDS, STAGES - 1 tiles ahead, and every wave converts what it multiplies (an LDS read of
// codes is half that of bf16, and a product hides four conversions).  KG 1: 128 rows, every
// wave takes every key.  KG 2: 64 rows, half of the waves take the first 32 keys of a tile and
// half the others, and they join at the end, for where there are not enough row tiles to fill the
// chip.  Which blocks a tile has, and their scales, stands in LDS for 256 blocks at a time, the
// next ones looked up meanwhile.
// 4096 tokens on 28672 keys, 8 query heads and 1 kv head of 256, causal, bf16 (KG 1, two chunks): 779 us,
// 1.15 PFLOP/s, where a library product of 8192^3 reaches 1.21: bounded by the matrix unit, which
// the conversions (4 cycles each, four beside a product of 32) and the softmax of the other
// wave of a SIMD leave busy.  64 parts of 1 to 61 tokens on 300 to 866 keys (KG 2): 33 us, of which
// 10 to 13 steps of 64 keys are 16 to 20; the rest is the lookup, the queries, the first tile and the
// join of the two halves.  277 workgroups then share 256 CUs, and those that share one end last.
constexpr int kList = 256;  // blocks of a list: a thread each
template <typename T, int DH, int KG>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void quant_walk_kernel(PartCall a) {
  constexpr int SLABS = DH / 64, NK = DH / 16, ND = DH / 32, RG = 4 / KG, KT = 32 * KG;
  constexpr int PARTS = sizeof(T) == 2 ? 1 : 3;
  constexpr int BLOCK = kBlock * DH, HALF = 2 * KG * BLOCK, STAGE = 2 * HALF;  // bytes: of a block, a tile's keys, both
  constexpr int STAGES = 65536 / STAGE > 4 ? 4 : 65536 / STAGE;
  constexpr int LT = kList / (2 * KG);  // tiles of a list
  constexpr bool BY_SUM = sizeof(T) == 2;  // no maximum in the loop: 789 us where 803 with it
  constexpr int JOIN = KG == 2 ? 2 * 32 * DH * 4 : 0;
  constexpr int RING = STAGES * STAGE > JOIN ? STAGES * STAGE : JOIN;
  static_assert(STAGES >= 2, "a tile ahead");
  __shared__ __attribute__((aligned(1024))) unsigned char ring[RING];
  // Blocks: where they begin in either pool (64 bits), and their scales, of keys and, from bit 8 on,
  // of values; bit 31: there is none.
  __shared__ __attribute__((aligned(16))) u32x4 list[2][kList];
  __shared__ float stats[KG == 2 ? 4 * 192 : 1];
  __shared__ int found;  // NaN among the values that were sifted
  const PartRows<32 * RG> b(a, 16 * threadIdx.x);
  if (!b.any() || b.idle()) return;
  const int lane = b.lane, wave = b.wave, l32 = b.l32, lh = b.lh, rows = b.rows, k0 = b.k0, k1 = b.k1;
  const int rg = wave % RG, kg = wave / RG;
  const int wrow = b.row0 + 32 * rg;
  const int tiles = (k1 - k0 + KT - 1) / KT;
  const int whole = (min(b.limit(b.row0), k1) - k0) / KT;  // tiles that every row sees (negative: none)
  // The thread, anew wherever it is used, so that nothing made of it is kept over the loop.
  auto self = [&]() __attribute__((always_inline)) {
    int x = threadIdx.x;
    asm volatile("" : "+v"(x));
    return x;
  };
  auto entry_of = [&](int at) __attribute__((always_inline)) {
    const size_t x = b.place(at), from = x * BLOCK;
    return u32x4{(uint32_t)from, (uint32_t)(from >> 32),
                 (uint32_t)(scale_exponent(a.k_scale[x]) + 127) | (uint32_t)(scale_exponent(a.v_scale[x]) + 127) << 8 |
                     (at < 0 ? 1u << 31 : 0u), 0};
  };
  auto look_up = [&](int n) __attribute__((always_inline)) {  // the list of blocks from number n on
    const int x = self();
    list[n / kList & 1][x] = entry_of(b.block_at(k0 + 16 * (n + x)));
  };

  const u32x4 entry = entry_of(b.block_at(k0 + 16 * threadIdx.x, b.page0));
  __builtin_amdgcn_sched_barrier(0);  // its loads before the queries'
  u32x4 qf[NK][PARTS];
  {
    int tok, head;
    b.of(wrow + l32, tok, head);
    const T* q = static_cast<const T*>(a.q) + (size_t)(b.q0 + tok) * a.ldq + head * DH;
#pragma unroll
    for (int p = 0; p < NK; ++p) query8(q + 64 * (p / 4) + 32 * (p / 2 % 2) + 16 * lh + 8 * (p % 2), qf[p]);
  }
  list[0][threadIdx.x] = entry;
  f32x16 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) o[d] = zeros16();
  float m = BY_SUM ? kNoRef : -INFINITY, l = 0.f;  // l over the lane half's keys only
  bool seen = false;
  if (threadIdx.x == 0) found = 0;

  // Waves 0 and 1 bring half of a tile's keys each, 2 and 3 of its values: KG blocks.  A kilobyte
  // of keys is 16 positions of 64 bytes, of which piece c lies at c ^ position / 4: the 16 positions
  // that a read touches at one piece then lie on different banks.
  int from = wave < 2 ? 64 * (lane >> 2) + 16 * ((lane & 3) ^ (lane >> 4)) : 16 * lane;
  const unsigned char* pool = wave < 2 ? a.k : a.v;
  const uint32_t ring0 = lds_address(ring) + wave * KG * BLOCK;
  auto issue = [&](int t, const uint64_t (&at)[KG]) __attribute__((always_inline)) {
    const uint32_t to = ring0 + t % STAGES * STAGE;
#pragma unroll
    for (int i = 0; i < KG; ++i) {
      const u32x4 src = dma_source(pool + at[i]);
#pragma unroll
      for (int x = 0; x < SLABS; ++x) dma16(src, to + i * BLOCK + 1024 * x, from + 1024 * x);
    }
  };
  int kaddr = (2 * kg + (l32 >> 4)) * BLOCK + 64 * (l32 & 15) + 16 * (lh ^ (l32 >> 2 & 3));
  int vaddr = HALF + 2 * kg * BLOCK + 256 * lh + 16 * (l32 & 15) + 8 * (l32 >> 4);
  asm volatile("" : "+v"(kaddr), "+v"(vaddr), "+v"(from));  // three registers, not what they are made of

  // Of the list, the same in every lane: the scales of the wave's two blocks of a tile, and where the
  // blocks begin that the wave brings for a later one.  Read during a softmax, used after it.
  struct Entries {
    uint32_t scales[2];
    uint64_t from[KG];
    bool holes;  // a block of the tile is not there
  };
  uint32_t read_scales[2 * KG];  // the wave's two first
  u32x2 read_from[KG];
  auto read_bases = [&](int t) __attribute__((always_inline)) {
    const u32x4* x = &list[t / LT & 1][2 * KG * t % kList + (wave & 1) * KG];
#pragma unroll
    for (int i = 0; i < KG; ++i) read_from[i] = *reinterpret_cast<const u32x2*>(x + i);
  };
  auto read = [&](int t) __attribute__((always_inline)) {  // of tile t, and of the one that it brings
    const u32x4* x = &list[t / LT & 1][2 * KG * t % kList];
#pragma unroll
    for (int i = 0; i < 2 * KG; ++i) read_scales[i] = reinterpret_cast<const uint32_t*>(x + (i ^ 2 * kg))[2];
    read_bases(t + STAGES - 1);
  };
  auto bases = [&](uint64_t (&from)[KG]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < KG; ++i)
      from[i] = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)read_from[i][1]) << 32 |
                (uint32_t)__builtin_amdgcn_readfirstlane((int)read_from[i][0]);
  };
  auto settled = [&]() __attribute__((always_inline)) {
    Entries e;
#pragma unroll
    for (int i = 0; i < 2; ++i) e.scales[i] = (uint32_t)__builtin_amdgcn_readfirstlane((int)read_scales[i]);
    e.holes = (int)(e.scales[0] | e.scales[1]) < 0;
    if (KG == 2)
      e.holes = e.holes || __builtin_amdgcn_readfirstlane((int)(read_scales[2 * KG - 2] | read_scales[2 * KG - 1])) < 0;
    bases(e.from);
    return e;
  };
  // 32 keys.  EDGE: some row may not see them all, or they are not all there.
  // Returns the entries of the next tile.
  auto step = [&](auto at_edge, int t, const Entries& at, int lim) __attribute__((always_inline)) {
    constexpr bool EDGE = decltype(at_edge)::value;
    const int key0 = k0 + KT * t + 32 * kg;
    const unsigned char* tile = ring + t % STAGES * STAGE;
    const float ks = __uint_as_float(((l32 < 16 ? at.scales[0] : at.scales[1]) & 255) << 23);
    const float vs[2] = {__uint_as_float((at.scales[0] >> 8 & 255) << 23), __uint_as_float((at.scales[1] >> 8 & 255) << 23)};
    auto key = [&](int x) __attribute__((always_inline)) {  // slab x / 2, half x % 2
      return *reinterpret_cast<const u32x4*>(tile + (x & 1 ? kaddr ^ 32 : kaddr) + 1024 * (x / 2));
    };
    auto value = [&](int x, int h) __attribute__((always_inline)) {  // slab x / 2, block x % 2
      return *reinterpret_cast<const u32x2*>(tile + vaddr + x % 2 * BLOCK + 1024 * (x / 2) + 512 * h);
    };
    f32x16 sc = zeros16();
    u32x4 raw[2] = {key(0), key(1)};
    u32x4 op = to_bf16x8(raw[0][0], raw[0][1], ks);
    __builtin_amdgcn_s_setprio(1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int p = 0; p < NK; ++p) {
      u32x4 next = op;
      if (p + 1 < NK) next = to_bf16x8(raw[(p + 1) / 2 % 2][2 * ((p + 1) % 2)], raw[(p + 1) / 2 % 2][2 * ((p + 1) % 2) + 1], ks);
#pragma unroll
      for (int x = 0; x < PARTS; ++x) sc = mma32(op, qf[p][x], sc, bf16_t{});
      if (p % 2 == 0 && p / 2 + 2 < NK / 2) raw[p / 2 % 2] = key(p / 2 + 2);
      __builtin_amdgcn_sched_barrier(0);
      op = next;
    }
    __builtin_amdgcn_s_setprio(0);
    u32x2 vr[2][2];
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int h = 0; h < 2; ++h) vr[x][h] = value(x, h);
    __builtin_amdgcn_sched_barrier(0);
    if (EDGE) {
      // What is seen is a branch ahead of the scores, and the compiler, where a long and a short path
      // lead from a product to its use, counts its wait along the long one: here it is in full.
      asm volatile("s_nop 11");
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if ((int)at.scales[r / 8] < 0) sc[r] = -INFINITY;
      hide(sc, key0, lh, lim);
      seen = seen || ((int)at.scales[0] >= 0 && key0 < lim) || ((int)at.scales[1] >= 0 && key0 + 16 < lim);
    } else {
      seen = true;
    }
    auto rescale = [&](float f) __attribute__((always_inline)) {
#pragma unroll
      for (int d = 0; d < ND; ++d) o[d] *= f;
    };
    u32x4 pf[2][PARTS];
    if constexpr (BY_SUM) {
      u32x4 one[2];
      softmax_by_sum(sc, false, key0, lh, lim, a.scale, m, l, one, rescale);
      pf[0][0] = one[0];
      pf[1][0] = one[1];
    } else {
      u32x4 unused[2];
      softmax<float>(sc, false, key0, lh, lim, a.scale, m, l, unused, rescale, [](int) {});
      probabilities<PARTS>(sc, pf);
    }
    read(t + 1);
    __builtin_amdgcn_s_setprio(1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int x = 0; x < 2 * SLABS; ++x) {
      const int c = x % 2;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const u32x4 v = u32x4{to_bf16<false>(vr[c][0][e], vs[c]), to_bf16<true>(vr[c][0][e], vs[c]),
                              to_bf16<false>(vr[c][1][e], vs[c]), to_bf16<true>(vr[c][1][e], vs[c])};
#pragma unroll
        for (int y = 0; y < PARTS; ++y) o[x / 2 * 2 + e] = mma32(v, pf[c][y], o[x / 2 * 2 + e], bf16_t{});
        if (e == 1 && x + 2 < 2 * SLABS) {
          vr[c][0] = value(x + 2, 0);
          vr[c][1] = value(x + 2, 1);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    __builtin_amdgcn_s_setprio(0);
    return settled();
  };

  __syncthreads();  // the list is there
  Entries now;
  for (int t = 0; t < STAGES - 1 && t < tiles; ++t) {
    read_bases(t);
    bases(now.from);
    issue(t, now.from);
  }
  read(0);
  now = settled();
  // Takes the NaN out of a tile's values: a weight of zero does not silence them.
  auto sift = [&](int t) __attribute__((always_inline)) {
    unsigned char* v = ring + t % STAGES * STAGE + HALF;
    for (int x = 16 * self(); x < HALF; x += 16 * 256) {
      u32x4 w = *reinterpret_cast<const u32x4*>(v + x);
      uint32_t odd = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t n = nans(w[i]);
        odd |= n;
        w[i] = without(w[i], n);
      }
      if (odd) {
        *reinterpret_cast<u32x4*>(v + x) = w;
        found = 1;
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  // Waits for tile t, brings a later one, looks up the next list.
  auto begin = [&](int t) __attribute__((always_inline)) {
    if (t + STAGES - 1 <= tiles)
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((STAGES - 2) * KG * SLABS) : "memory");
    else
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();  // every wave's part is there, and tile t - 1 done with
    asm volatile("" ::: "memory");
    if (t + STAGES - 1 < tiles) issue(t + STAGES - 1, now.from);
    const int n = t / LT + 1, at = t % LT;
    if (n * LT < tiles) {
      if (at == LT / 2) look_up(n * kList);
    }
  };
  int t = 0;
  // The queries are there: the compiler would wait for them at their use, in every turn of the
  // loop, and with them for the tiles that are under way.
#pragma unroll
  for (int i = 0; i < NK; ++i)
#pragma unroll
    for (int x = 0; x < PARTS; ++x) asm volatile("" : "+v"(qf[i][x]));
  // Whole tiles; from the first one on that some row does not see whole, or that has a hole, values
  // are sifted.
  if (wrow >= rows) {  // a wave without rows only does its part for the others
    for (bool sifting = false; t < tiles; ++t) {
      begin(t);
      sifting = sifting || t >= whole || now.holes;
      if (sifting) sift(t);
      read(t + 1);
      now = settled();
    }
  } else {
    for (; t < tiles; ++t) {
      begin(t);
      if (t >= whole || now.holes) break;
      now = step(std::false_type{}, t, now, 0);
    }
  }
  const int edge = t;
  // again from here on, so that nothing of it is kept over the whole tiles
  int row = wrow + l32, tok, head;
  asm volatile("" : "+v"(row));
  b.of(row, tok, head);
  const int lim = b.limit(row);
  while (t < tiles) {
    sift(t);
    now = step(std::true_type{}, t, now, lim);
    if (++t < tiles) begin(t);
  }
  // Every load has landed and every read is done: the ring is free.
  auto meet = [] __device__() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  meet();
  if (BY_SUM) m = m == kNoRef ? -INFINITY : -m;
  l = other_half_sum(l);
  const bool unruly = found;
  constexpr int OUT = ND / KG;  // of o, that the wave writes: from number kg OUT on, in front after this
  if constexpr (KG == 2) {
    // the two waves of the rows give each other half of their sums
    f32x4* so = reinterpret_cast<f32x4*>(ring) + lane;
    float* st = stats + lane;
    auto give = [&](int from) __attribute__((always_inline)) {
#pragma unroll
      for (int d = 0; d < OUT; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f32x16& x = o[from + d];
          so[((wave * OUT + d) * 4 + j) * 64] = f32x4{x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]};
        }
    };
    if (kg)
      give(0);
    else
      give(OUT);
    st[192 * wave] = m;
    st[192 * wave + 64] = l;
    st[192 * wave + 128] = seen;
    meet();
    const int with = wave ^ RG;
    const float other = st[192 * with], top = fmaxf(m, other), ref = top == -INFINITY ? 0.f : top;
    const float f = __builtin_amdgcn_exp2f(m - ref), g = __builtin_amdgcn_exp2f(other - ref);
    m = top;
    l = l * f + st[192 * with + 64] * g;
    seen = seen || st[192 * with + 128] != 0.f;
    auto take = [&](int from) __attribute__((always_inline)) {
#pragma unroll
      for (int d = 0; d < OUT; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f32x4 x = so[((with * OUT + d) * 4 + j) * 64];
#pragma unroll
          for (int e = 0; e < 4; ++e) o[d][4 * j + e] = o[from + d][4 * j + e] * f + x[e] * g;
        }
    };
    if (kg)
      take(OUT);
    else
      take(0);
  }
  if (wrow >= rows) return;
  const bool last = a.n_chunks == 1;
  // a row that sees no key: zeros; keys that all score -inf: 0/0, as the formula has it
  const float f = last ? (seen ? 1.0f / l : 0.f) : 1.0f;
  const size_t mine = last ? (size_t)(b.q0 + tok) * a.ldo + head * DH : b.partial(tok, head) * DH;
  // Lane halves exchange so that a lane has 8 elements of its row side by side.
  if (row < rows) {
#pragma unroll
    for (int d = 0; d < OUT; ++d)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int n = (KG == 2 ? kg * OUT : 0) + d;
        const size_t to = mine + 64 * (n / 2) + 16 * (2 * j + n % 2) + 8 * lh;
        float x[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(o[d][8 * j + e] * f),
                                                          __float_as_uint(o[d][8 * j + 4 + e] * f), false, false);
          x[e] = __uint_as_float(y[0]);
          x[4 + e] = __uint_as_float(y[1]);
        }
        if (last) {
          store8(static_cast<T*>(a.out) + to, x);
        } else {
          store8(a.part + to, x);
        }
      }
  }
  if (unruly) {  // NaN among the values at the edge: of the rows that see them
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    for (int key = k0 + KT * edge; key < min(b.limit(wrow + 31), k1); ++key) {
      const int at = __builtin_amdgcn_readfirstlane(b.block_at(key & ~15));
      if (at < 0) continue;
      for (int d = lane; d < DH; d += 64) {
        const bool odd = (KG == 1 || (2 * (d / 64) + d / 16 % 2) / OUT == kg) && b.is_nan(b.place(at), key, d, DH);
        if (!__any(odd)) continue;
        for (int r = 0; r < 32; ++r) {
          const size_t to = (size_t)__shfl((long long)mine, r) + d;
          if (!(key < __shfl(lim, r)) || !odd || wrow + r >= rows) continue;
          if (last)
            static_cast<T*>(a.out)[to] = from_f32<T>(__builtin_nanf(""));
          else
            a.part[to] = __builtin_nanf("");
        }
      }
    }
  }
  if (!last && kg == 0 && lh == 0 && wrow + l32 < rows) b.state(tok, head, seen ? m : -INFINITY, seen ? l : kNoKey);
}

template <typename T, int DH>
void part_at(const PartCall& a, int rows, hipStream_t s) {
  const dim3 blocks((unsigned)((int64_t)a.n_slots * a.n_kv * a.n_chunks));
  if (rows == 32)
    hipLaunchKernelGGL((quant_part_kernel<T, DH>), blocks, dim3(64 * kPartWaves), 0, s, a);
  else if (rows == 64)
    hipLaunchKernelGGL((quant_walk_kernel<T, DH, 2>), blocks, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((quant_walk_kernel<T, DH, 1>), blocks, dim3(256), 0, s, a);
}

}  // namespace

namespace {
// About the us of a call that shares its rows out to `tiles` row tiles and its keys to `chunks` chunks
// of `chunk`: a launch, and between the time of one workgroup and that of all of them on the chip, a
// little more than the longer; where there are chunks, the join and what it reads.  Either
// time is a fixed part and one for each 32 keys, with a part of each that grows with the head.
// The workgroups of fp32 have a CU each, so that what is over a full round counts half a round.
// Fitted, by least squares of the logarithms, to 11370 timings of 1086 calls of 1 to 512 sequences, 1
// to 4096 new tokens, 1 to 30000 keys, heads 8/1 of 256, 32/8 of 128, 8/2 of 64 and 4/2 of 192 (14 %
// off each), when the probabilities of few rows had one part in bf16.  With the present kernels what
// it chooses takes 4 % longer than the best of all in the mean and 14 % at the ninetieth hundredth, over
// the 3738 timings of 296 calls in profiles/quant_part_timings.txt; limits on the number of row tiles
// and of keys took over 10 % in the mean.
double part_time(bool fp32, int kind, double head, double tiles, double chunk, int chunks, double moved) {
  static const double of[2][3][8] = {
      {{0.836, 4.174, 0.136, 0.259, 0.051, 6.612, 0.102, 0.302},
       {1.194, 4.239, 0.196, 0.36, 1.317, 1.957, 0.082, 0.341},
       {0.934, 3.331, 0.396, 0.594, 0.81, 1.039, 0.091, 0.633}},
      {{0, 6.914, 0, 0.665, 0, 10.39, 0, 0.71},
       {0.188, 6.218, 0.25, 0.669, 0, 11.671, 0.041, 1.223},
       {0, 4.994, 0.381, 1.474, 0, 10.213, 0.127, 2.314}}};
  static const double join[2][2] = {{3.543, 0.173}, {2.818, 0.157}};  // us, us a MB
  const double* x = of[fp32][kind];
  const double w = head / 256, steps = chunk / 32;
  double n = tiles * chunks;
  if (fp32) {
    const double round = head < 128 ? 512 : 256;
    n = 0.5 * (n + round * ceil(n / round));
  }
  const double one = x[0] + x[1] * w + steps * (x[2] + x[3] * w);
  const double all = n / 256 * (x[4] + x[5] * w + steps * (x[6] + x[7] * w));
  return 3 + sqrt(one * one + all * all) + (chunks > 1 ? join[fp32][0] + join[fp32][1] * 1e-6 * moved * chunks : 0);
}
}  // namespace

// The rows of a workgroup and the chunks that part_time says are the fastest.  us by rows and, in
// brackets, chunks, the best of each, of calls captured into a graph, and what is taken:
//                                          32        64        128       taken
// 50 tokens on 866, heads 8/1 of 256       14.6 (7)  15.4 (7)  17.6 (7)  32 (7)
// 4 by 50 on 866, 8/1 of 256               18.7 (4)  20.1 (4)  22.5 (4)  64 (4)
// 64 by 1 to 61 on 300 to 866, 8/1 of 256  55.2 (1)  33.5 (1)  36.1 (1)  64 (1)
// 128 by 50 on 300 to 866, 8/1 of 256      134 (1)   62.9 (1)  52.6 (1)  128 (1)
// 500 on 8000, 8/1 of 256                  74.6 (2)  53.3 (8)  54.0 (8)  64 (6): 55.5
// 4096 on 28672, 8/1 of 256                1570 (1)  806 (1)   809 (2)   128 (2)
// 32 by 1 to 100 on 100 to 3000, 32/8/128  156 (1)   87.2 (1)  103 (3)   64 (1)
// 8 by 500 on 2000, 32/8 of 128            323 (1)   156 (1)   131 (1)   128 (1)
// fp32: 5 by 33 to 301 on 60 to 1301, 8/2/64 17.6 (1)  23.3 (4)  24.8 (4)  32 (1)
// fp32: 50 on 900, 8/1 of 256              16.8 (8)  21.7 (8)  27.3 (8)  32 (8)
// fp32: 4 by 200 on 1000, 8/1 of 256       36.7 (1)  44.8 (2)  45.3 (4)  32 (1)
// fp32: 64 by 50 on 866, 8/1 of 256        126 (1)   97.7 (1)  83.6 (1)  64 (1)
PartPlan plan_part(const fv_part_args& x, const fv_quant_pages& c, int max_keys) {
  static const int counts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32};
  PartPlan p{};
  const int64_t rows = (int64_t)x.n_q * (x.n_q_heads / c.n_kv_heads);
  double best = 0;
  for (int kind = 0; kind < 3; ++kind) {
    const int of = 32 << kind;
    const double shared = (double)rows / of + 0.5 * x.n_seqs;  // entries begin inside tiles
    const double tiles = (shared > x.n_seqs ? shared : x.n_seqs) * c.n_kv_heads;
    for (int count : counts) {
      const int64_t step = kind ? 32 : 32 * kPartWaves;  // with 32 rows, each wave as many keys
      const int64_t chunk = ((max_keys + count - 1) / count + step - 1) / step * step;
      const int64_t chunks = (max_keys + chunk - 1) / chunk;
      // not where the chip is full without, nor where the join's grid would have 2^32 threads
      if (count > 1 && (chunk < 128 || tiles * count > 768 || (int64_t)x.n_q * x.n_q_heads > 1 << 22)) break;
      const double us = part_time(c.dtype == FV_FP32, kind, c.head_dim, tiles, chunk < max_keys ? chunk : max_keys,
                                  (int)chunks, 8. * rows * c.n_kv_heads * c.head_dim);
      if (p.rows && us >= best) continue;
      best = us;
      p.rows = of;
      p.chunk = (int)chunk;
      p.n_chunks = (int)chunks;
    }
  }
  if (p.n_chunks > 1) p.work_bytes = (size_t)x.n_q * p.n_chunks * x.n_q_heads * (c.head_dim + 2) * 4;
  return p;
}

template <typename T>
void launch_quant_part(const fv_part_args& x, const fv_quant_pages& c, const PartPlan& p, hipStream_t s) {
  PartCall a{};
  const size_t layer = (size_t)x.layer * block_of(c.n_pages, c.n_kv_heads, 0, c.page_len, 0);
  a.q = x.q;
  a.k = static_cast<const unsigned char*>(c.k) + layer * kBlock * c.head_dim;
  a.v = static_cast<const unsigned char*>(c.v) + layer * kBlock * c.head_dim;
  a.k_scale = static_cast<const uint8_t*>(c.k_scale) + layer;
  a.v_scale = static_cast<const uint8_t*>(c.v_scale) + layer;
  a.out = x.out;
  a.cu_q = x.cu_q;
  a.seqs = x.seqs;
  a.table = c.table;
  a.len = c.len;
  a.part = static_cast<float*>(x.work);
  a.stat = a.part + (size_t)x.n_q * p.n_chunks * x.n_q_heads * c.head_dim;
  a.ldq = x.ldq;
  a.ldo = x.ldo;
  a.n_seqs = x.n_seqs;
  a.n_q = x.n_q;
  a.heads = x.n_q_heads;
  a.n_kv = c.n_kv_heads;
  a.group = x.n_q_heads / c.n_kv_heads;
  a.causal = x.causal;
  a.n_slots = (int)((int64_t)x.n_q * a.group / p.rows + x.n_seqs);
  a.page_len = c.page_len;
  a.n_pages = c.n_pages;
  a.max_seqs = c.max_seqs;
  a.max_pages = c.max_pages;
  a.chunk = p.chunk;
  a.n_chunks = p.n_chunks;
  a.per_page = (uint32_t)(((1ull << 31) + c.page_len / 16 - 1) / (c.page_len / 16));
  a.scale = x.scale * kLog2e;
  switch (c.head_dim) {
    case 64: part_at<T, 64>(a, p.rows, s); break;
    case 128: part_at<T, 128>(a, p.rows, s); break;
    case 192: part_at<T, 192>(a, p.rows, s); break;
    default: part_at<T, 256>(a, p.rows, s);
  }
  if (p.n_chunks > 1) {
    PagedCall j{};
    j.out = x.out;
    j.cu = x.cu_q;
    j.n_entries = x.n_seqs;
    j.part = a.part;
    j.stat = a.stat;
    j.ldo = x.ldo;
    j.n = x.n_q;
    j.heads = x.n_q_heads;
    j.n_chunks = p.n_chunks;
    launch_paged_join<T>(j, c.head_dim, s);
  }
}
template void launch_quant_part<bf16_t>(const fv_part_args&, const fv_quant_pages&, const PartPlan&, hipStream_t);
template void launch_quant_part<float>(const fv_part_args&, const fv_quant_pages&, const PartPlan&, hipStream_t);

}  // namespace fv
