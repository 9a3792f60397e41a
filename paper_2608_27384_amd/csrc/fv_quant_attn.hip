// Attention of one new token a sequence over the pages of a cache in 8 bits.
//
// Built as the attention over pages of the dtype is (fv_paged.hip): a sequence's keys in
// chunks, one workgroup each (per kv head and tile of 16 query heads), whose four waves walk
// their own tiles of 32 keys from memory straight into registers and join in LDS; a second
// kernel joins the chunks.  Memory bounds it: 192 sequences of 1 to 8191 keys, 32 query and 8 kv heads
// of 128, bf16, pages of 64: 272 us for 1.63 GB, 6.0 TB/s, as a plain read goes (6.2).  Small calls
// are a chain of trips to memory (sequence, table with the length, codes) and the join's launch:
// one sequence of 816 keys, 8 query heads and 1 kv head of 256, 8.5 us, 64 of 300 to 816 11.6.
//
// A lane's 16 bytes of a block are its matrix operands after a conversion to bf16, which is
// exact, the block's scale included: two codes an instruction, 4 cycles a wave.  Values lie in
// memory turned over (four positions of an element side by side), so nothing is permuted.
// Against codes that are bf16 numbers only the other operand limits the precision: fp32
// queries go in as three parts of bf16, 24 bits together, probabilities as two (16 bits) or,
// with fp32 results, three, all into fp32 sums.
#include "fv_paged.h"
#include "fv_quant.h"

namespace fv {
namespace {

template <typename T, int DH, bool STREAM>
__global__ __launch_bounds__(64 * kPagedWaves, 2) void quant_paged_kernel(PagedCall a) {
  constexpr int SLABS = DH / 64, KT = 32, NT = DH / 16;
  constexpr int QP = sizeof(T) == 2 ? 1 : 3, PP = sizeof(T) == 2 ? 2 : 3;  // parts of queries, of probabilities
  __shared__ float sm[kPagedWaves][16], sl[kPagedWaves][16];
  // fp32 queries of 256 elements are 96 registers in parts: they stay in LDS, where `so` comes later.
  // 64 sequences of 2000 to 4000 keys, 8/1 heads, 36.6 us, in registers 44.9; with shorter heads, whose
  // registers suffice, the same or a little more.
  constexpr bool PUT = sizeof(T) == 4 && DH == 256;
  __shared__ __attribute__((aligned(16))) float so[kPagedWaves][16][DH + 4];
  u32x4* const put = reinterpret_cast<u32x4*>(&so[0][0][0]);

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int l16 = lane & 15, lg = lane >> 4;
  int id = blockIdx.x;
  const int qt = id % a.q_tiles;
  id /= a.q_tiles;
  const int kh = id % a.n_kv;
  id /= a.n_kv;
  // each row begins one chunk further on (see paged_kernel)
  const int row = id / a.n_chunks, ch = (id + row) % a.n_chunks;
  const int s = a.seqs[row];
  if (s < 0 || s >= a.max_seqs) return;
  const int k0 = ch * a.chunk;
  const int* table = a.table + (size_t)s * a.max_pages;
  auto page_of = [&](int key) __attribute__((always_inline)) { return (int)__umulhi(key >> 3, a.per_page); };
  auto page_at = [&](int key) __attribute__((always_inline)) {
    const int p = page_of(key);
    return p < a.max_pages ? table[p] : -1;
  };
  // first key of the block that a lane looks up, past that of its wave's tile `base`
  int ahead = kPagedWaves * (lane / 2) * KT + 16 * (lane % 2);
  asm volatile("" : "+v"(ahead));
  int page = page_at(k0 + wave * KT + ahead);
  const int len = length_of(a, s);
  const int chunks = chunks_of(len, a.chunk, a.n_chunks);
  if (ch >= chunks && ch > 0) return;
  const int k1 = ch == a.n_chunks - 1 ? len : min(len, k0 + a.chunk);

  // queries: the head of column l16, zeros past the group
  const int head = qt * 16 + l16;
  u32x4 qf[2 * SLABS][QP];
  {
    const T* q = static_cast<const T*>(a.q) + (size_t)row * a.ldq + (kh * a.group + min(head, a.group - 1)) * DH;
#pragma unroll
    for (int b = 0; b < 2 * SLABS; ++b) {
      if (PUT && b % kPagedWaves != wave) continue;
      query8(q + 64 * (b / 2) + 16 * lg + 8 * (b % 2), qf[b]);
      if (head >= a.group)
#pragma unroll
        for (int i = 0; i < QP; ++i) qf[b][i] = u32x4{0, 0, 0, 0};
      if (PUT)
#pragma unroll
        for (int i = 0; i < QP; ++i) put[(b * QP + i) * 64 + lane] = qf[b][i];
    }
    if (PUT) __syncthreads();
  }

  f32x4 o[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;  // of the lane's query; l over the lane's keys only
  bool any = false;              // a key was seen

  const unsigned char* kp = static_cast<const unsigned char*>(a.k);
  const unsigned char* vp = static_cast<const unsigned char*>(a.v);
  const int tiles = (k1 - k0 + KT - 1) / KT;
  constexpr int GO = 32;  // tiles whose blocks the lanes look up at a time
  for (int base = wave; base < tiles; base += kPagedWaves * GO) {
    const int myKey = k0 + base * KT + ahead;
    if (base != wave) page = page_at(myKey);
    // block number in the pool, -1: no keys.  A layer has at most 2^20 pages of 1024 heads and
    // 16 blocks: 2^34, so the page and the block in it (as the row / 16 of its page)
    const int half = myKey >= k1 || page < 0 || page >= a.n_pages ? -1 : page << 4 | (myKey - page_of(myKey) * a.page_len) >> 4;
    auto block = [&](int at) __attribute__((always_inline)) {
      return block_of(max(at, 0) >> 4, a.n_kv, kh, a.page_len, max(at, 0) & 15);
    };
    // the scales' exponents, as the upper bits of the power
    const size_t mine = block(half);
    const int scales = (scale_exponent(a.k_scale[mine]) + 127) | (scale_exponent(a.v_scale[mine]) + 127) << 8;
    const int here = min(GO, (tiles - base + kPagedWaves - 1) / kPagedWaves);
    u32x4 kf[2][SLABS];
    auto load_keys = [&](int it) __attribute__((always_inline)) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const unsigned char* from = kp + block(__builtin_amdgcn_readlane(half, 2 * it + h)) * (16 * DH);
#pragma unroll
        for (int x = 0; x < SLABS; ++x)
          kf[h][x] = load_piece<STREAM>(reinterpret_cast<const u32x4*>(from + 1024 * x + 64 * l16 + 16 * lg));
      }
    };
    load_keys(0);
    for (int it = 0; it < here; ++it) {
      u32x4 vf[2][SLABS];
      int left[2];
      float ks[2], vs[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int at = __builtin_amdgcn_readlane(half, 2 * it + h), sc = __builtin_amdgcn_readlane(scales, 2 * it + h);
        left[h] = at < 0 ? 0 : min(16, k1 - (k0 + (base + kPagedWaves * it) * KT + 16 * h));
        ks[h] = __uint_as_float((uint32_t)(sc & 255) << 23);
        vs[h] = __uint_as_float((uint32_t)(sc >> 8) << 23);
        const unsigned char* from = vp + block(at) * (16 * DH);
#pragma unroll
        for (int x = 0; x < SLABS; ++x)
          vf[h][x] = load_piece<STREAM>(reinterpret_cast<const u32x4*>(from + 1024 * x + 16 * lane));
      }

      f32x4 sc[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        sc[h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int b = 0; b < 2 * SLABS; ++b) {
          const u32x4 k = to_bf16x8(kf[h][b / 2][2 * (b % 2)], kf[h][b / 2][2 * (b % 2) + 1], ks[h]);
#pragma unroll
          for (int i = 0; i < QP; ++i)
            sc[h] = mma64(k, PUT ? put[(b * QP + i) * 64 + lane] : qf[b][i], sc[h], bf16_t{});
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      if (it + 1 < here) load_keys(it + 1);  // while the softmax and the values are at work
      any = any || left[0] > 0 || left[1] > 0;
      if (left[0] != 16 || left[1] != 16) {  // keys that are not there: no weight, and values that hold nothing
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int n = min(max(left[h] - 4 * lg, 0), 4);  // of the lane's four
          const uint32_t keep = (uint32_t)((1ull << 8 * n) - 1);
#pragma unroll
          for (int x = 0; x < SLABS; ++x) vf[h][x] &= keep;
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (r >= n) sc[h][r] = -INFINITY;
        }
      }
      float top = -INFINITY;
#pragma unroll
      for (int h = 0; h < 2; ++h)
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
      u16x8 part[PP];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float p = __builtin_amdgcn_exp2f(sc[h][r] - ref);
          l += p;
          bf16_t at[PP];
          split<PP>(p, at);
#pragma unroll
          for (int i = 0; i < PP; ++i) part[i][4 * h + r] = at[i];
        }
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const uint32_t lo = vf[0][t / 4][t % 4], hi = vf[1][t / 4][t % 4];
        const u32x4 v = u32x4{to_bf16<false>(lo, vs[0]), to_bf16<true>(lo, vs[0]), to_bf16<false>(hi, vs[1]),
                              to_bf16<true>(hi, vs[1])};
#pragma unroll
        for (int i = 0; i < PP; ++i) o[t] = mma64(v, __builtin_bit_cast(u32x4, part[i]), o[t], bf16_t{});
      }
    }
  }

  // join the waves
  if (PUT) __syncthreads();
  l = sum_xor16_32(l);
  if (lg == 0) {
    sm[wave][l16] = m;
    // a sequence of keys that all score -inf has no softmax: NaN, as 0/0
    sl[wave][l16] = any && m == -INFINITY ? 0.f : l;
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) *reinterpret_cast<f32x4*>(&so[wave][l16][16 * t + 4 * lg]) = o[t];
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

template <typename T, int DH>
void quant_paged_at(const PagedCall& a, size_t bytes, hipStream_t s) {
  const int blocks = a.n * a.n_chunks * a.n_kv * a.q_tiles;
  hipLaunchKernelGGL((bytes > kStreamBytes ? quant_paged_kernel<T, DH, true> : quant_paged_kernel<T, DH, false>),
                     dim3(blocks), dim3(64 * kPagedWaves), 0, s, a);
}

}  // namespace

// Chunks' join is a launch of its own, and their workgroups more than the chip takes at once where
// there are many sequences.  One chunk where that costs more than the walk does; us of chunks and
// of one, bf16, lengths from a third of the longest on:
//   cols                  keys   440         700         1000         2040
//      1, 8/1 heads of 256     8.3 / 8.2   8.5 / 10.4   8.5 / 12.5   10.6 / 20.3
//      8, 32/8 of 128          7.4 / 6.3   7.8 / 7.9    7.7 / 9.3    10.3 / 15.1
//     64, 8/1 of 256           9.3 / 8.5  11.3 / 10.6  12.2 / 13.1   21.0 / 22.5
//    128, 8/2 of 64            8.0 / 5.7   8.6 / 7.0   9.5 / 8.1     14.6 / 13.2
//    256, 8/1 of 256          19.0 / 11.1 23.7 / 15.4  30.6 / 19.6   40.9 / 32.5
//   2048, 32/8 of 128         28.6 / 28.1 41.3 / 41.0  73.0 / 69.0  129   / 119
// and fp32, whose walk costs three times the products:
//      1, 8/1 of 256          10.3 / 12.0 10.3 / 15.7  10.5 / 18.6   12.6 / 31.3
//     64, 8/1 of 256          11.5 / 12.5 14.1 / 16.0  15.8 / 20.4   28.0 / 36.5
//    256, 8/1 of 256          25.7 / 16.0 32.2 / 20.3  42.8 / 24.6   56.3 / 40.7
//      2, 8/2 of 64            7.2 / 6.0   7.4 / 7.3    7.5 / 8.6     9.6 / 13.7
PagedPlan plan_quant(int n, int n_q_heads, int n_kv_heads, int head_dim, int max_keys, bool bf16) {
  PagedPlan p = plan_paged(n, n_q_heads, n_kv_heads, head_dim, max_keys, true);
  const int64_t cols = (int64_t)n * n_kv_heads * ((n_q_heads / n_kv_heads + 15) / 16);
  const int64_t few = bf16 ? 12 * cols : 0, least = bf16 || head_dim <= 128 ? 448 : 256;
  if (max_keys <= (cols >= 128 ? 2048 : few > least ? few : least)) {
    p.n_chunks = 1;
    p.work_bytes = 0;
  }
  return p;
}

template <typename T>
void launch_quant_paged(const fv_paged_args& x, const fv_quant_pages& c, const PagedPlan& p, hipStream_t s) {
  PagedCall a = paged_call(x, as_pages(c), p);
  const size_t layer = (size_t)x.layer * block_of(c.n_pages, c.n_kv_heads, 0, c.page_len, 0);
  a.k = static_cast<const unsigned char*>(c.k) + layer * kBlock * c.head_dim;
  a.v = static_cast<const unsigned char*>(c.v) + layer * kBlock * c.head_dim;
  a.k_scale = static_cast<const uint8_t*>(c.k_scale) + layer;
  a.v_scale = static_cast<const uint8_t*>(c.v_scale) + layer;
  // what the call may read: the keys and values planned for, which a layer's pages bound
  const size_t key = 2 * (size_t)c.n_kv_heads * c.head_dim;
  const size_t planned = (size_t)x.n * p.keys * key, pages = (size_t)c.n_pages * c.page_len * key;
  const size_t bytes = planned < pages ? planned : pages;
  switch (c.head_dim) {
    case 64: quant_paged_at<T, 64>(a, bytes, s); break;
    case 128: quant_paged_at<T, 128>(a, bytes, s); break;
    case 192: quant_paged_at<T, 192>(a, bytes, s); break;
    default: quant_paged_at<T, 256>(a, bytes, s);
  }
  launch_paged_join<T>(a, c.head_dim, s);
}
template void launch_quant_paged<bf16_t>(const fv_paged_args&, const fv_quant_pages&, const PagedPlan&, hipStream_t);
template void launch_quant_paged<float>(const fv_paged_args&, const fv_quant_pages&, const PagedPlan&, hipStream_t);

}  // namespace fv
