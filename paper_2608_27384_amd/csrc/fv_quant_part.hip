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
// probabilities go in as three parts of bf16.
#include "fv_paged.h"
#include "fv_prompt.h"
#include "fv_quant.h"

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

constexpr int kPartWaves = 4;

// 32 rows a workgroup, whose waves share a chunk's keys out, straight from memory into registers,
// and join in LDS.
template <typename T, int DH>
__global__ __launch_bounds__(64 * kPartWaves, 1) void quant_part_kernel(PartCall a) {
  constexpr int SLABS = DH / 64, NK = DH / 16, ND = DH / 32, PITCH = DH + 4;
  constexpr int PARTS = sizeof(T) == 2 ? 1 : 3;
  __shared__ float sm[kPartWaves][32], sl[kPartWaves][32];
  __shared__ int seen_by[kPartWaves][32];
  __shared__ __attribute__((aligned(16))) float so[kPartWaves][32 * PITCH];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int l32 = lane & 31, lh = lane >> 5;
  // the heaviest tiles of a causal part, its last ones, go first
  int id = blockIdx.x;
  const int ch = id % a.n_chunks;
  id /= a.n_chunks;
  const int kh = id % a.n_kv, slot = a.n_slots - 1 - id / a.n_kv;
  int first;
  const int entry = prompt_of<32>(a, slot, &first);
  const int q0 = clamped(a.cu_q, entry, a.n_q), nq = max(0, clamped(a.cu_q, entry + 1, a.n_q) - q0);
  const int rows = nq * a.group, row0 = (slot - first) * 32;
  if (row0 < 0 || row0 >= rows) return;
  const int s = a.seqs[entry];
  const bool named = s >= 0 && s < a.max_seqs;
  const int nk = named ? min(max(a.len[s], 0), a.max_pages * a.page_len) : 0;
  // A row sees the keys [0, limit), which do not fall from one row to the next.
  auto limit = [&](int row) __attribute__((always_inline)) {
    return a.causal ? min(max(nk - nq + 1 + min(row, rows - 1) / a.group, 0), nk) : nk;
  };
  const int k0 = ch * a.chunk;
  const int k1 = min(ch == a.n_chunks - 1 ? nk : min(nk, k0 + a.chunk), limit(row0 + 31));
  const int steps = max(0, (k1 - k0 + 31) / 32);
  const int row = min(row0 + l32, rows - 1), tok = row / a.group, head = kh * a.group + row - tok * a.group;
  const bool here = row0 + l32 < rows;
  if (steps == 0 && a.n_chunks > 1) {  // of these keys no row sees any
    if (wave == 0 && lh == 0 && here) {
      const size_t at = ((size_t)(q0 + tok) * a.n_chunks + ch) * a.heads + head;
      a.stat[2 * at] = -INFINITY;
      a.stat[2 * at + 1] = named ? kNoKey : kNoEntry;
    }
    return;
  }
  if (!named) return;

  const int* table = a.table + (size_t)s * a.max_pages;
  const int lim = limit(row);
  const int whole = limit(row0);  // keys that every row of the tile sees
  u32x4 qf[NK][PARTS];
  {
    const T* q = static_cast<const T*>(a.q) + (size_t)(q0 + tok) * a.ldq + head * DH;
#pragma unroll
    for (int p = 0; p < NK; ++p) query8(q + 64 * (p / 4) + 32 * (p / 2 % 2) + 16 * lh + 8 * (p % 2), qf[p]);
  }
  f32x16 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) o[d] = zeros16();
  float m = -INFINITY, l = 0.f;  // l over the lane half's keys only
  bool unruly = false, seen = false;
  // the pool's block number of the 16 keys from `key` on, or -1
  auto block_at = [&](int key) __attribute__((always_inline)) {
    if (key >= k1) return -1;
    const int p = (int)__umulhi(key >> 3, a.per_page);
    const int page = p < a.max_pages ? table[p] : -1;
    return page < 0 || page >= a.n_pages ? -1 : page << 4 | (key - p * a.page_len) >> 4;
  };
  auto place = [&](int at) __attribute__((always_inline)) {
    return block_of(max(at, 0) >> 4, a.n_kv, kh, a.page_len, max(at, 0) & 15);
  };
  for (int i = wave; i < steps; i += kPartWaves) {
    const int key0 = k0 + 32 * i;
    const int at0 = __builtin_amdgcn_readfirstlane(block_at(key0));
    const int at1 = __builtin_amdgcn_readfirstlane(block_at(key0 + 16));
    const size_t p0 = place(at0), p1 = place(at1);
    const bool edge = key0 + 32 > whole || key0 + 32 > k1 || at0 < 0 || at1 < 0;
    const size_t mine = l32 < 16 ? p0 : p1;  // of the lane's key
    const unsigned char* kp = a.k + mine * (16 * DH) + 64 * (l32 & 15) + 16 * lh;
    const float ks = power_of(scale_exponent(a.k_scale[mine]));
    const float vs[2] = {power_of(scale_exponent(a.v_scale[p0])), power_of(scale_exponent(a.v_scale[p1]))};
    u32x4 kf[2 * SLABS];
#pragma unroll
    for (int x = 0; x < 2 * SLABS; ++x) kf[x] = *reinterpret_cast<const u32x4*>(kp + 1024 * (x / 2) + 32 * (x % 2));
    // values: of block c, the positions from 4 lh + 8 h on
    u32x2 vf[SLABS][2][2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const unsigned char* vp = a.v + (c ? p1 : p0) * (16 * DH) + 256 * lh + 16 * (l32 & 15) + 8 * (l32 >> 4);
#pragma unroll
      for (int x = 0; x < SLABS; ++x)
#pragma unroll
        for (int h = 0; h < 2; ++h) vf[x][c][h] = *reinterpret_cast<const u32x2*>(vp + 1024 * x + 512 * h);
    }
    f32x16 sc = zeros16();
#pragma unroll
    for (int p = 0; p < NK; ++p) {
      const u32x4 k = to_bf16x8(kf[p / 2][2 * (p % 2)], kf[p / 2][2 * (p % 2) + 1], ks);
#pragma unroll
      for (int x = 0; x < PARTS; ++x) sc = mma32(k, qf[p][x], sc, bf16_t{});
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
    u16x8 pf[2][PARTS];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      bf16_t at[PARTS];
      split<PARTS>(sc[r], at);
#pragma unroll
      for (int x = 0; x < PARTS; ++x) pf[r / 8][x][r % 8] = at[x];
    }
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const uint32_t lo = vf[d / 2][c][0][d % 2], hi = vf[d / 2][c][1][d % 2];
        const u32x4 v = u32x4{to_bf16<false>(lo, vs[c]), to_bf16<true>(lo, vs[c]), to_bf16<false>(hi, vs[c]),
                              to_bf16<true>(hi, vs[c])};
#pragma unroll
        for (int x = 0; x < PARTS; ++x) o[d] = mma32(v, __builtin_bit_cast(u32x4, pf[c][x]), o[d], bf16_t{});
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
  if (unruly) {  // NaN among the values at the edge: of the rows that see them
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    for (int i = wave; i < steps; i += kPartWaves) {
      const int from = k0 + 32 * i;
      for (int key = from; key < min(from + 32, k1); ++key) {
        const int at = __builtin_amdgcn_readfirstlane(block_at(key & ~15));
        if (at < 0 || (from + 32 <= whole && from + 32 <= k1)) continue;
        const unsigned char* vp = a.v + place(at) * (16 * DH) + 256 * (key % 16 / 4) + key % 4;
        for (int d = lane; d < DH; d += 64) {
          const bool odd = (vp[1024 * (d / 64) + 16 * (d % 16) + 4 * (d % 64 / 16)] & 127) == 127;
          if (!__any(odd)) continue;
          for (int r = 0; r < 32; ++r)
            if (key < __shfl(lim, r) && odd) mine[r * PITCH + d] = __builtin_nanf("");
        }
      }
    }
  }
  __syncthreads();
  for (int u = threadIdx.x; u < 32 * (DH / 4); u += 64 * kPartWaves) {
    const int r = u / (DH / 4), d = 4 * (u % (DH / 4));
    if (row0 + r >= rows) continue;
    f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kPartWaves; ++w) acc += *reinterpret_cast<const f32x4*>(so[w] + r * PITCH + d);
    const int t = (row0 + r) / a.group, h = kh * a.group + row0 + r - t * a.group;
    if (last)
      store4(static_cast<T*>(a.out) + (size_t)(q0 + t) * a.ldo + h * DH + d, acc[0], acc[1], acc[2], acc[3]);
    else
      *reinterpret_cast<f32x4*>(a.part + (((size_t)(q0 + t) * a.n_chunks + ch) * a.heads + h) * DH + d) = acc;
  }
  if (!last && wave == 0 && lh == 0 && here) {
    const size_t at = ((size_t)(q0 + tok) * a.n_chunks + ch) * a.heads + head;
    a.stat[2 * at] = any ? top : -INFINITY;
    a.stat[2 * at + 1] = any ? all : kNoKey;
  }
}

template <typename T, int DH>
void part_at(const PartCall& a, hipStream_t s) {
  const int64_t blocks = (int64_t)a.n_slots * a.n_kv * a.n_chunks;
  hipLaunchKernelGGL((quant_part_kernel<T, DH>), dim3((unsigned)blocks), dim3(64 * kPartWaves), 0, s, a);
}

}  // namespace

PartPlan plan_part(const fv_part_args& x, const fv_quant_pages& c, int max_keys) {
  PartPlan p{};
  const int group = x.n_q_heads / c.n_kv_heads;
  p.rows = 32;
  const int64_t cols = ((int64_t)x.n_q * group / p.rows + x.n_seqs) * c.n_kv_heads;
  const int least = kPartWaves * 64;
  int64_t chunk = ((int64_t)max_keys * cols + 1023) / 1024;
  chunk = (chunk + 31) / 32 * 32;
  if (chunk < least) chunk = least;
  int64_t chunks = (max_keys + chunk - 1) / chunk;
  // the join's grid, one of more than 2^32 threads otherwise
  if (chunks < 1 || (int64_t)x.n_q * x.n_q_heads > 1 << 22) chunks = 1;
  while (chunks > 1 && chunks * cols > 1 << 23) chunks /= 2;  // the last one is longer then
  p.chunk = (int)chunk;
  p.n_chunks = (int)chunks;
  if (chunks > 1) p.work_bytes = (size_t)x.n_q * chunks * x.n_q_heads * (c.head_dim + 2) * 4;
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
    case 64: part_at<T, 64>(a, s); break;
    case 128: part_at<T, 128>(a, s); break;
    case 192: part_at<T, 192>(a, s); break;
    default: part_at<T, 256>(a, s);
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
