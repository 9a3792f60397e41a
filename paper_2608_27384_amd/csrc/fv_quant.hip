// The paged cache in 8 bits: rotary positions fused with the quantising append,
// and reading back.
#include "fv_quant.h"

namespace fv {
namespace {

constexpr int kWaves = kRopeThreads / 64;

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
// Eight pairs of a head, of which p holds the first halves.
template <int HALF, typename T>
__device__ __forceinline__ void turn8(const T* p, const float* cs, const float* sn, float (&x)[8], float (&y)[8]) {
  load8(p, x);
  load8(p + HALF, y);
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
// Largest over the wave, the same in every lane.
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int y = 1; y < 64; y <<= 1) x = fmaxf(x, __shfl_xor(x, y));
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

// A workgroup has TT tokens of the list: their queries, and the keys and values of the runs
// that begin among them.  A run is the tokens of one block, which the caller lists side by
// side; it may go on behind the workgroup's tokens, whose workgroup then leaves the first of
// its own alone.  A wave takes a run's keys or values of one head: it finds the largest size,
// which gives the scale, in registers, lays the block out in LDS over what it held, and
// stores it, whole or the pieces that changed.  So no two waves write one block, nothing is
// read twice, and the result does not depend on the order of anything.
template <typename T, int DH, int TT>
__global__ __launch_bounds__(kRopeThreads) void quant_append_kernel(QuantAppend r) {
  constexpr int HALF = DH / 2, SLABS = DH / 64, ANG = TT + kBlock - 1;
  __shared__ __attribute__((aligned(16))) float cs[ANG][HALF], sn[ANG][HALF];
  __shared__ u32x4 image[kWaves][DH];               // blocks as they will be
  __shared__ int seq[TT + kBlock], at[TT + kBlock];  // of the tokens from the one before on; seq -1: no place
  __shared__ int run_tok[TT], run_rows[TT], n_runs;  // first token, which rows of the block
  __shared__ long long run_block[TT];                // of kv head 0, or -1

  const fv_rope_args& a = r.a;
  const fv_quant_pages& c = r.c;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int t0 = blockIdx.x * TT, nt = min(TT, a.n - t0);

  const int near = min(TT + kBlock, a.n - t0 + 1);
  if (tid < near) {
    const int i = t0 - 1 + tid;
    int s = -1, p = 0;
    if (i >= 0) {
      s = a.seqs[i];
      p = a.at[i];
      if (s >= c.max_seqs || p < 0 || p >= c.max_pages * c.page_len) s = -1;
    }
    seq[tid] = s;
    at[tid] = p;
  }
  const RopeAngles<DH> angles(a, r.log2_theta);
  angles.form(t0, 0, nt, cs, sn);
  __syncthreads();
  if (wave == 0) {
    const int i = lane + 1;
    bool head = false;
    int s = -1, p = 0;
    if (lane < nt) {
      s = seq[i];
      p = at[i];
      head = s < 0 ? a.k_out != nullptr : seq[lane] != s || at[lane] / kBlock != p / kBlock || at[lane] >= p;
    }
    const uint64_t m = __ballot(head);
    if (head) {
      long long block = -1;
      int rows = 1 << p % kBlock;
      if (s >= 0) {
        const int page = c.table[(size_t)s * c.max_pages + p / c.page_len];
        if (page >= 0 && page < c.n_pages)
          block = (long long)block_of(page, c.n_kv_heads, 0, c.page_len, p % c.page_len / kBlock);
        for (int j = i + 1; j < near && seq[j] == s && at[j] / kBlock == p / kBlock && at[j] > at[j - 1]; ++j)
          rows |= 1 << at[j] % kBlock;
      }
      const int x = __popcll(m & ((1ull << lane) - 1));
      run_tok[x] = lane;
      run_rows[x] = s < 0 ? 1 : rows;
      run_block[x] = block;
    }
    if (lane == 0) n_runs = (int)__popcll(m);
  }
  __syncthreads();
  const int runs = n_runs;
  if (runs) {
    const int end = run_tok[runs - 1] + __popc(run_rows[runs - 1]);
    if (end > nt) {
      angles.form(t0, nt, end, cs, sn);
      __syncthreads();
    }
  }

  const size_t layer = (size_t)a.layer * block_of(c.n_pages, c.n_kv_heads, 0, c.page_len, 0);
  unsigned char* mine = reinterpret_cast<unsigned char*>(image[wave]);
  for (int item = wave; item < runs * 2 * c.n_kv_heads; item += kWaves) {
    const bool values = item & 1;
    const int g = (item >> 1) % c.n_kv_heads, run = (item >> 1) / c.n_kv_heads;
    const int tok = run_tok[run], rows = __builtin_amdgcn_readfirstlane(run_rows[run]), len = __popc(rows);
    const long long place = run_block[run];
    if (values && place < 0) continue;
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
    // the scale that `size` asks for; what the block holds at it, in the image; 2^-e
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
    if (!values) {
      constexpr int PIECES = DH / 16;
      float x[SLABS][8], y[SLABS][8];
      float size = 0.f;
#pragma unroll
      for (int j = 0; j < SLABS; ++j) {
        const int t = (64 * j + lane) / PIECES, i = 8 * ((64 * j + lane) % PIECES);
        if (t >= len) continue;
        const size_t row = t0 + tok + t;
        turn8<HALF>(static_cast<const T*>(a.k) + row * a.ldk + g * DH + i, &cs[tok + t][i], &sn[tok + t][i], x[j], y[j]);
        if (a.k_out) {
          T* out = static_cast<T*>(a.k_out) + row * a.ldk_out + g * DH + i;
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
        const int u = 64 * j + lane, p0 = 4 * (u / PIECES), i = 8 * (u % PIECES);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
          for (int k = 0; k < 8; ++k) x[j][t][k] = 0.f;
          if (p0 >= kBlock || !(rows >> (p0 + t) & 1)) continue;
          const size_t row = t0 + tok + __popc(rows & ((1 << (p0 + t)) - 1));
          load8(static_cast<const T*>(a.v) + row * a.ldv + g * DH + i, x[j][t]);
#pragma unroll
          for (int k = 0; k < 8; ++k) size = fmaxf(size, finite_size(x[j][t][k]));
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

  // the queries, from the last threads on: the first waves have the runs
  constexpr int PIECES = DH / 16;
  for (int u = kRopeThreads - 1 - tid; u < nt * a.n_q_heads * PIECES; u += kRopeThreads) {
    const int i = 8 * (u % PIECES), th = u / PIECES, t = th / a.n_q_heads, h = th - t * a.n_q_heads;
    const size_t row = t0 + t;
    float x[8], y[8];
    turn8<HALF>(static_cast<const T*>(a.q) + row * a.ldq + h * DH + i, &cs[t][i], &sn[t][i], x, y);
    T* out = static_cast<T*>(a.q_out) + row * a.ldq_out + h * DH + i;
    store8(out, x);
    store8(out + HALF, y);
  }
}

// Reading back.  Block (b, entry, layer): the positions 16 b .. 16 b + 15 of a sequence, one
// wave the keys, one the values.  Rows go out whole, 128 bytes or more side by side; a
// lane's four positions of values are turned over in LDS.
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

template <typename T, int DH>
void append_at(const QuantAppend& r, hipStream_t s) {
  if (quant_tokens(r.a.n) == 1)
    hipLaunchKernelGGL((quant_append_kernel<T, DH, 1>), dim3(r.a.n), dim3(kRopeThreads), 0, s, r);
  else
    hipLaunchKernelGGL((quant_append_kernel<T, DH, 16>), dim3((r.a.n + 15) / 16), dim3(kRopeThreads), 0, s, r);
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

// One token a workgroup where there are few and the time is one trip to memory; sixteen
// share the exponentials of the angles, and a prompt's block is then the work of one.
int quant_tokens(int n) { return n < 2048 ? 1 : 16; }

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
