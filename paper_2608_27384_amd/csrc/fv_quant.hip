// The paged cache in 8 bits: rotary positions fused with the quantising append,
// and reading back.
#include "fv_quant.h"

namespace fv {
namespace {

struct QuantAppend {
  fv_rope_args a;
  fv_quant_pages c;
  double log2_theta;
};

// Eight elements in fp32.
__device__ __forceinline__ void load8(const bf16_t* p, float (&x)[8]) {
  const u32x4 v = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = __uint_as_float(v[e] << 16);
    x[2 * e + 1] = __uint_as_float(v[e] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const f32x4 v = load4_f32(p + 4 * h);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[4 * h + e] = v[e];
  }
}
// Turns eight pairs of a head.
__device__ __forceinline__ void turn8(const float* cs, const float* sn, float (&x)[8], float (&y)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float c = cs[e], s = sn[e], a = x[e], b = y[e];
    x[e] = a * c - b * s;
    y[e] = b * c + a * s;
  }
}

__device__ __forceinline__ float finite_size(float x) {
  const float a = fabsf(x);
  return a < INFINITY ? a : 0.f;
}
// Largest over the wave, the same in every lane (the lane exchanges of wave_sum).
template <int CTRL> __device__ __forceinline__ float dpp_max(float x) {
  return fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, false)));
}
__device__ __forceinline__ float wave_max(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
  x = dpp_max<0x128>(x);  // row_ror:8
  x = dpp_max<0x124>(x);  // row_ror:4
  x = dpp_max<0x4E>(x);   // quad_perm [2,3,0,1]
  x = dpp_max<0xB1>(x);   // quad_perm [1,0,3,2]
  return x;
}
// e of the scale 2^e that values up to `size` ask for: size <= 448 * 2^e = 1.75 * 2^(e + 8).
__device__ __forceinline__ int exponent_for(float size) {
  const uint32_t b = __float_as_uint(size);
  const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u);
  return min(max(e, kLeastScale - 127), kMostScale - 127);
}
// x * inv as e4m3, saturated (only a block at the largest scale has more than 448 of it);
// infinities and NaN as NaN.  The conversion rounds to nearest even, subnormal codes too.
__device__ __forceinline__ float within(float x, float inv) {
  return fabsf(x) < INFINITY ? __builtin_amdgcn_fmed3f(x * inv, -448.f, 448.f) : __builtin_nanf("");
}
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d, float inv) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(within(a, inv), within(b, inv), 0, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(within(c, inv), within(d, inv), w, true);
}
// Four codes times f <= 1, rounded again.
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float f) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a[0] * f, a[1] * f, 0, false);
  return __builtin_amdgcn_cvt_pk_fp8_f32(b[0] * f, b[1] * f, r, true);
}

// A run is the tokens of one block, which the caller lists side by side (or a token without a
// place).  A workgroup has the runs that begin among TT tokens of the list; the last may go on
// behind them, whose workgroup then leaves the first of its own alone.  A wave takes a run's keys
// or values of one head: it finds the largest size, which gives the scale, in registers, lays
// the block out in LDS over what it held, and stores it, whole or the pieces that changed.  So no
// two waves write one block, nothing is read twice, and the result does not depend on the order
// of anything.  Of the workgroups that have the same tokens (blockIdx.z) each takes its share of
// the runs' keys and values and of their queries, which go, a few pieces at a time, to the waves
// that are free.
// A workgroup's time is a chain of trips to memory (token, table, block's scale and codes), so
// all loads of a piece of work are issued before the first is used.  64 prompts of 300 to 816
// tokens, 8 query heads and 1 kv head of 256, bf16: 83 us for 368 MB, 4.4 TB/s, as large copies go
// (5.1); queries in a launch of their own beside it took 97 us.  64 single tokens: 6.3 us.
template <typename T, int DH, int TT>
__global__ __launch_bounds__(256) void quant_append_kernel(QuantAppend r) {
  constexpr int HALF = DH / 2, SLABS = DH / 64, ANG = TT + kBlock - 1, WAVES = 4;
  static_assert(TT + kBlock <= 64, "a token a lane");
  __shared__ __attribute__((aligned(16))) float cs[ANG][HALF], sn[ANG][HALF];
  __shared__ u32x4 image[WAVES][DH];                // blocks as they will be
  __shared__ int at[TT + kBlock];                   // positions, from the token before on
  __shared__ int run_tok[TT], run_rows[TT], n_runs;  // first token, which rows of the block
  __shared__ int taken;                              // pieces of queries
  __shared__ long long run_block[TT];               // of kv head 0, or -1

  const fv_rope_args& a = r.a;
  const fv_quant_pages& c = r.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int t0 = (blockIdx.y * gridDim.x + blockIdx.x) * TT, nt = min(TT, a.n - t0);
  if (nt <= 0) return;

  if (wave == 0) {  // lane l has token t0 - 1 + l
    const int i = t0 - 1 + lane;
    int s = -1, p = 0;
    if (lane < TT + kBlock && i >= 0 && i < a.n) {
      s = a.seqs[i];
      p = a.at[i];
      if (s >= c.max_seqs || p < 0 || p >= c.max_pages * c.page_len) s = -1;
      at[lane] = p;
    }
    const int s1 = __shfl_up(s, 1), p1 = __shfl_up(p, 1);
    const bool goes_on = lane > 0 && s >= 0 && s1 == s && p1 / kBlock == p / kBlock && p1 < p;
    const bool head = lane > 0 && lane <= nt && !goes_on;
    const uint64_t on = __ballot(goes_on), heads = __ballot(head);
    if (lane < TT) run_rows[lane] = 0;
    if (lane == 0) {
      n_runs = (int)__popcll(heads);
      taken = 0;
    }
    // A head's run ends before the first lane behind it that does not go on.
    const int x = (int)__popcll(heads & ((2ull << lane) - 1)) - 1;  // the run of the lane, if it has one
    if (head) {
      long long block = -1;
      if (s >= 0) {
        const int page = c.table[(size_t)s * c.max_pages + p / c.page_len];
        if (page >= 0 && page < c.n_pages)
          block = (long long)block_of(page, c.n_kv_heads, 0, c.page_len, p % c.page_len / kBlock);
      }
      run_tok[x] = lane - 1;
      run_block[x] = block;
    }
    const int first = 63 - __clzll(heads & ((2ull << lane) - 1));  // the last head up to the lane (-1: none)
    const uint64_t between = first < 0 ? 0 : ((2ull << lane) - 1) & ~((2ull << first) - 1);
    if (first >= 0 && (on & between) == between) atomicOr(&run_rows[x], s < 0 ? 1 : 1 << p % kBlock);
  }
  // the first token's angles, where there is one, while its place is looked up
  if (TT > 1) {
    __syncthreads();
    if (!n_runs) return;
  }
  const RopeAngles<DH> angles(a, r.log2_theta, 256);
  if (TT == 1) {
    angles.template form<true>(t0, 0, 1, cs, sn);
    __syncthreads();
    if (!n_runs) return;
  }
  const int first = run_tok[0], end = run_tok[n_runs - 1] + __popc(run_rows[n_runs - 1]);
  if (TT > 1 || end > 1) {
    angles.template form<true>(t0, TT == 1 ? 1 : first, end, cs, sn);
    __syncthreads();
  }

  const size_t layer = (size_t)a.layer * block_of(c.n_pages, c.n_kv_heads, 0, c.page_len, 0);
  unsigned char* mine = reinterpret_cast<unsigned char*>(image[wave]);
  // the workgroup's share of the keys and values, and further down of the queries
  const int part = blockIdx.z, parts = gridDim.z;
  const int all_items = n_runs * 2 * c.n_kv_heads, items = (part + 1) * all_items / parts;
  for (int item = part * all_items / parts + wave; item < items; item += WAVES) {
    const bool values = item & 1;
    const int g = (item >> 1) % c.n_kv_heads, run = (item >> 1) / c.n_kv_heads;
    const int tok = run_tok[run], rows = __builtin_amdgcn_readfirstlane(run_rows[run]), len = __popc(rows);
    const long long place = run_block[run];
    if (place < 0 && (values || !a.k_out)) continue;
    const bool anew = rows & 1;
    const size_t block = layer + (size_t)max(place, 0ll) + (size_t)g * (c.page_len / kBlock);
    u32x4* stored = static_cast<u32x4*>(values ? c.v : c.k) + block * DH;
    uint8_t* scale = static_cast<uint8_t*>(values ? c.v_scale : c.k_scale) + block;
    u32x4 old[SLABS];
    int e = kLeastScale - 127;
#pragma unroll
    for (int s = 0; s < SLABS; ++s) old[s] = u32x4{0, 0, 0, 0};
    if (place >= 0 && !anew) {
      e = scale_exponent(*scale);
#pragma unroll
      for (int s = 0; s < SLABS; ++s) old[s] = stored[64 * s + lane];
    }
    // the scale that `size` asks for; what the block holds at it, in the image
    auto begin = [&](float size) __attribute__((always_inline)) {
      const int now = max(e, exponent_for(wave_max(size)));
      if (now > e) {
        const float f = power_of(max(e - now, -126));
#pragma unroll
        for (int s = 0; s < SLABS; ++s)
#pragma unroll
          for (int x = 0; x < 4; ++x) old[s][x] = rescale4(old[s][x], f);
      }
#pragma unroll
      for (int s = 0; s < SLABS; ++s) image[wave][64 * s + lane] = old[s];
      __builtin_amdgcn_wave_barrier();
      const bool whole = anew || now > e;
      e = now;
      if (whole && lane == 0) *scale = (uint8_t)(now + 127);
      return whole;
    };
    bool whole;
    uint32_t touched;  // whether the lane's pieces change
    // Loads are for every lane, past the run's tokens of its last one: a load in a branch of its
    // own waits for its own trip to memory.
    if (!values) {
      constexpr int PIECES = DH / 16;
      float x[SLABS][8], y[SLABS][8];
      float size = 0.f;
#pragma unroll
      for (int j = 0; j < SLABS; ++j) {
        const int t = min((64 * j + lane) / PIECES, len - 1), i = 8 * ((64 * j + lane) % PIECES);
        const T* from = static_cast<const T*>(a.k) + (size_t)(t0 + tok + t) * a.ldk + g * DH + i;
        load8(from, x[j]);
        load8(from + HALF, y[j]);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < SLABS; ++j) {
        const int t = (64 * j + lane) / PIECES, i = 8 * ((64 * j + lane) % PIECES);
        if (t >= len) continue;
        turn8(&cs[tok + t][i], &sn[tok + t][i], x[j], y[j]);
        if (a.k_out) {
          T* out = static_cast<T*>(a.k_out) + (size_t)(t0 + tok + t) * a.ldk_out + g * DH + i;
          store8(out, x[j]);
          store8(out + HALF, y[j]);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) size = fmaxf(size, fmaxf(finite_size(x[j][k]), finite_size(y[j][k])));
      }
      if (place < 0) continue;
      whole = begin(size);
      const float inv = power_of(-e);
#pragma unroll
      for (int j = 0; j < SLABS; ++j) {
        const int t = (64 * j + lane) / PIECES, i = 8 * ((64 * j + lane) % PIECES);
        if (t >= len) continue;
        const int p = at[tok + t + 1] % kBlock;
        auto put = [&](int d, const float (&z)[8]) __attribute__((always_inline)) {
          *reinterpret_cast<u32x2*>(mine + d / 64 * 1024 + 64 * p + d % 64) =
              u32x2{encode4(z[0], z[1], z[2], z[3], inv), encode4(z[4], z[5], z[6], z[7], inv)};
        };
        put(i, x[j]);
        put(HALF + i, y[j]);
      }
      touched = rows >> lane / 4 & 1;
    } else {
      constexpr int PIECES = DH / 8, N = (4 * PIECES + 63) / 64;
      float x[N][4][8];
      float size = 0.f;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int u = min(64 * j + lane, 4 * PIECES - 1), p0 = 4 * (u / PIECES), i = 8 * (u % PIECES);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int row = t0 + tok + min(__popc(rows & ((1 << (p0 + t)) - 1)), len - 1);
          load8(static_cast<const T*>(a.v) + (size_t)row * a.ldv + g * DH + i, x[j][t]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int p0 = 4 * ((64 * j + lane) / PIECES);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const bool here = p0 < kBlock && (rows >> (p0 + t) & 1);
#pragma unroll
          for (int k = 0; k < 8; ++k) size = fmaxf(size, here ? finite_size(x[j][t][k]) : 0.f);
        }
      }
      whole = begin(size);
      const float inv = power_of(-e);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const int u = 64 * j + lane, p0 = 4 * (u / PIECES), i = 8 * (u % PIECES);
        const uint32_t here = p0 < kBlock ? rows >> p0 & 15 : 0;
        if (!here) continue;
        uint32_t keep = 0;  // bytes of the positions that are not the run's
#pragma unroll
        for (int t = 0; t < 4; ++t) keep |= here >> t & 1 ? 0u : 255u << 8 * t;
        unsigned char* to = mine + i / 64 * 1024 + 64 * p0 + i % 16 * 16 + i % 64 / 16 * 4;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          uint32_t* w = reinterpret_cast<uint32_t*>(to + 16 * k);
          uint32_t z = encode4(x[j][0][k], x[j][1][k], x[j][2][k], x[j][3][k], inv);
          if (keep) z = (z & ~keep) | (*w & keep);
          *w = z;
        }
      }
      touched = rows >> 4 * (lane / 16) & 15;
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (whole || touched) {
#pragma unroll
      for (int s = 0; s < SLABS; ++s) stored[64 * s + lane] = image[wave][64 * s + lane];
    }
    __builtin_amdgcn_wave_barrier();
  }

  // N pieces a lane, 16 N 64 elements a wave, at a time
  constexpr int PIECES = DH / 16, N = 2;
  const int pieces = (end - first) * a.n_q_heads * PIECES;
  const int from0 = part * pieces / parts, all = (part + 1) * pieces / parts;
  while (true) {
    int u0 = 0;
    if (lane == 0) u0 = from0 + atomicAdd(&taken, 64 * N);
    u0 = __builtin_amdgcn_readfirstlane(u0);
    if (u0 >= all) break;
    float x[N][8], y[N][8];
    int tok[N], at0[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int u = min(u0 + 64 * j + lane, all - 1), th = u / PIECES, t = th / a.n_q_heads;
      tok[j] = first + t;
      at0[j] = (th - t * a.n_q_heads) * DH + 8 * (u % PIECES);
      const T* from = static_cast<const T*>(a.q) + (size_t)(t0 + tok[j]) * a.ldq + at0[j];
      load8(from, x[j]);
      load8(from + HALF, y[j]);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int u = u0 + 64 * j + lane, i = 8 * (u % PIECES);
      if (u >= all) continue;
      turn8(&cs[tok[j]][i], &sn[tok[j]][i], x[j], y[j]);
      T* out = static_cast<T*>(a.q_out) + (size_t)(t0 + tok[j]) * a.ldq_out + at0[j];
      store8(out, x[j]);
      store8(out + HALF, y[j]);
    }
  }
}

// Reading back.  Block (b, entry, layer): the positions 16 b .. 16 b + 15 of a sequence, one
// wave the keys, one the values.  Rows go out whole, 128 bytes or more side by side; a
// lane's four positions of values are turned over in LDS.  Bounded by HBM: 64 sequences of 300 to
// 816 tokens in 18 layers, 1 kv head of 256, to bf16: 179 us for 995 MB, 5.5 TB/s; one of 560 5.1
// us, the trip to the table, the length and the codes.
template <typename T, int DH, bool STREAM>
__global__ __launch_bounds__(128) void quant_gather_kernel(fv_quant_pages c, const int* seqs, int n, int ld,
                                                           T* k_out, T* v_out) {
  constexpr int SLABS = DH / 64, VE = 16 / (int)sizeof(T);  // elements of a store
  constexpr int LANES = 64 / VE, STEPS = kBlock * LANES / 64;  // lanes of a row's slab, stores of a slab
  constexpr int PITCH = 72;
  typedef typename std::conditional<VE == 8, u32x2, uint32_t>::type Codes;
  __shared__ __attribute__((aligned(16))) unsigned char turned[SLABS][kBlock * PITCH];
  const int lane = threadIdx.x & 63, l = blockIdx.z, b = blockIdx.x;
  const bool values = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  T* const out = values ? v_out : k_out;
  for (int i = blockIdx.y; i < n; i += gridDim.y) {
    const int s = seqs[i];
    if (s < 0 || s >= c.max_seqs) continue;
    const int rows = min(min(c.len[s], c.max_pages * c.page_len), ld) - b * kBlock;
    if (rows <= 0) continue;
    const int page = c.table[(size_t)s * c.max_pages + b * kBlock / c.page_len];
    if (page < 0 || page >= c.n_pages) continue;
    const size_t block0 = (size_t)l * block_of(c.n_pages, c.n_kv_heads, 0, c.page_len, 0) +
                          block_of(page, c.n_kv_heads, 0, c.page_len, b * kBlock % c.page_len / kBlock);
    T* to = out + (((size_t)l * n + i) * ld + (size_t)b * kBlock) * c.n_kv_heads * DH;
    for (int g = 0; g < c.n_kv_heads; ++g, to += DH) {
      const size_t block = block0 + (size_t)g * (c.page_len / kBlock);
      const unsigned char* from = static_cast<const unsigned char*>(values ? c.v : c.k) + block * kBlock * DH;
      const float scale = power_of(scale_exponent(static_cast<const uint8_t*>(values ? c.v_scale : c.k_scale)[block]));
      Codes x[SLABS][STEPS];
      if (values) {
        u32x4 w[SLABS];
#pragma unroll
        for (int d = 0; d < SLABS; ++d)
          w[d] = load_piece<STREAM>(reinterpret_cast<const u32x4*>(from + 1024 * d + 16 * lane));
#pragma unroll
        for (int d = 0; d < SLABS; ++d)
#pragma unroll
          for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int t = 0; t < 4; ++t)
              turned[d][(4 * (lane / 16) + t) * PITCH + 16 * q + lane % 16] = (unsigned char)(w[d][q] >> 8 * t);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int d = 0; d < SLABS; ++d)
#pragma unroll
          for (int j = 0; j < STEPS; ++j)
            x[d][j] = *reinterpret_cast<const Codes*>(
                &turned[d][(64 / LANES * j + lane / LANES) * PITCH + lane % LANES * VE]);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      } else {
#pragma unroll
        for (int d = 0; d < SLABS; ++d)
#pragma unroll
          for (int j = 0; j < STEPS; ++j)
            x[d][j] = load_piece<STREAM>(reinterpret_cast<const Codes*>(from + 1024 * d + (64 * j + lane) * VE));
      }
#pragma unroll
      for (int j = 0; j < STEPS; ++j) {
        const int row = 64 / LANES * j + lane / LANES;
        if (row >= rows) continue;
        T* p = to + (size_t)row * c.n_kv_heads * DH + lane % LANES * VE;
#pragma unroll
        for (int d = 0; d < SLABS; ++d) {
          u32x4 y;
          if constexpr (VE == 8) {
            y = to_bf16x8(x[d][j][0], x[d][j][1], scale);
          } else {
            const uint32_t lo = to_bf16<false>(x[d][j], scale), hi = to_bf16<true>(x[d][j], scale);
            y = u32x4{lo << 16, lo & 0xffff0000u, hi << 16, hi & 0xffff0000u};
          }
          store_piece<STREAM>(reinterpret_cast<u32x4*>(p + 64 * d), y);
        }
      }
    }
  }
}

template <typename T, int DH, int TT>
void append_runs(const QuantAppend& r, int parts, hipStream_t s) {
  const unsigned n = (r.a.n + TT - 1) / TT, wide = n < 1 << 20 ? n : 1 << 20;
  hipLaunchKernelGGL((quant_append_kernel<T, DH, TT>), dim3(wide, (n + wide - 1) / wide, parts), dim3(256), 0, s, r);
}
template <typename T, int DH>
void append_at(const QuantAppend& r, hipStream_t s) {
  const QuantShare x = quant_share(r.a.n, r.c.n_kv_heads);
  switch (x.tokens) {
    case 1: return append_runs<T, DH, 1>(r, x.parts, s);
    case 4: return append_runs<T, DH, 4>(r, x.parts, s);
    default: return append_runs<T, DH, 8>(r, x.parts, s);
  }
}

template <typename T, int DH>
void gather_at(const fv_quant_pages& c, const int* seqs, int n, int ld, void* k_out, void* v_out, hipStream_t s) {
  const int holds = c.max_pages * c.page_len;
  const int blocks = ((ld < holds ? ld : holds) + kBlock - 1) / kBlock;
  // read in a byte an element, written in the dtype
  const size_t moved = 2 * (size_t)c.n_layers * n * blocks * kBlock * c.n_kv_heads * DH * (1 + sizeof(T));
  hipLaunchKernelGGL((moved > kStreamBytes ? quant_gather_kernel<T, DH, true> : quant_gather_kernel<T, DH, false>),
                     dim3(blocks, n < 65535 ? n : 65535, c.n_layers), dim3(128), 0, s, c, seqs, n, ld,
                     static_cast<T*>(k_out), static_cast<T*>(v_out));
}

}  // namespace

// A list of many tokens is as a rule prompts, whose runs are up to 16 long: workgroups of few tokens
// are then mostly ones that find no run of their own.  One of few is as a rule a token a sequence,
// each a run.  Where the tokens do not fill the chip, several workgroups have the same ones and
// share their blocks and queries out, or a workgroup's waves take many blocks one after another.
// us by parts, bf16 (in brackets: what is taken):
//                                         1 token          4 tokens               8 tokens
//   parts                                 1    4    8      1    2    4    8       1    2    4    8
//   64 single tokens, 8/1 heads of 256   (6.3)             9.0  6.7  6.6
//   64 single tokens, 32/8 of 128       10.9  5.7 (5.9)   31.1 17.9 10.9  7.5
//   500 single tokens, 32/8 of 128      13.8 14.5 20.6    33.3 19.8 13.8 (12.3)
//   a prompt of 400, 8/1 of 256         12.9              10.1  9.0 (9.2)
//   a prompt of 816, 8/1 of 256         21.5              11.3 (10.4) 14.1
//   2 prompts of 816, 32/8 of 128       58.3 68.9 91.0    27.0 24.6 25.1 27.9    22.3 17.2 (16.4) 17.3
//   4 prompts of 816, 8/1 of 256        55.7              25.1 26.2 35.1         (14.3) 17.6 21.1 29.9
//   8 prompts of 816, 32/8 of 128                         73.1 72.7 76.1 95.6    (42.4) 41.5 43.0 51.4
QuantShare quant_share(int n, int n_kv_heads) {
  QuantShare x;
  x.tokens = n < 128 ? 1 : n < 1024 ? 4 : 8;
  const int fill = n_kv_heads < 3 ? 256 * (n_kv_heads + 1) : 1024, most = n_kv_heads * x.tokens;
  x.parts = fill / ((n + x.tokens - 1) / x.tokens);
  if (x.parts > most) x.parts = most;
  if (x.parts < 1) x.parts = 1;
  return x;
}

template <typename T>
void launch_quant_append(const fv_rope_args& a, const fv_quant_pages& c, hipStream_t s) {
  const QuantAppend r{a, c, log2((double)a.theta)};
  switch (a.head_dim) {
    case 64: return append_at<T, 64>(r, s);
    case 128: return append_at<T, 128>(r, s);
    case 192: return append_at<T, 192>(r, s);
    default: return append_at<T, 256>(r, s);
  }
}
template void launch_quant_append<bf16_t>(const fv_rope_args&, const fv_quant_pages&, hipStream_t);
template void launch_quant_append<float>(const fv_rope_args&, const fv_quant_pages&, hipStream_t);

template <typename T>
void launch_quant_gather(const fv_quant_pages& c, const int* seqs, int n, int ld, void* k_out, void* v_out,
                         hipStream_t s) {
  switch (c.head_dim) {
    case 64: return gather_at<T, 64>(c, seqs, n, ld, k_out, v_out, s);
    case 128: return gather_at<T, 128>(c, seqs, n, ld, k_out, v_out, s);
    case 192: return gather_at<T, 192>(c, seqs, n, ld, k_out, v_out, s);
    default: return gather_at<T, 256>(c, seqs, n, ld, k_out, v_out, s);
  }
}
template void launch_quant_gather<bf16_t>(const fv_quant_pages&, const int*, int, int, void*, void*, hipStream_t);
template void launch_quant_gather<float>(const fv_quant_pages&, const int*, int, int, void*, void*, hipStream_t);

}  // namespace fv
