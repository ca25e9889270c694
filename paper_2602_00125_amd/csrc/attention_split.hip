// Attention of a few queries against many keys, gfx950: a token of each sequence
// against its cache, short chunks. There are too few blocks of 128 queries to
// fill the chip, and the keys' bytes are what counts. The queries of all heads of
// a key head are columns side by side, 32 to a block, so that each key is read
// once for all of them; the keys are shared by `splits` blocks and within a block
// by its waves, each with LDS buffers of its own and no barrier between them: a
// wave's next tile is in flight while it works on one. The waves' results are
// joined in LDS, the blocks' by join_kernel, in order. Bound: HBM (16 tokens
// against 8192 keys, 32 over 8 heads of 128: 107 us bf16 = 5.0 TB/s; against
// 4096 keys in fp32 110 us = 4.9 TB/s, on the fp32 matrix instructions; against
// ragged caches of 8192 keys at most, 0.34 GB in use, bf16: 73 to 79 us = 4.3 to
// 4.6 TB/s, 4 of them the join).
#include <hip/hip_runtime.h>

#include "attention.hpp"
#include "attention_tile.hpp"

namespace mt {
namespace attn {

// What a wave multiplies tiles with: 32 own tokens, one a lane
template <bool BF, int DP>
struct Own {
  using T = Tile<BF, DP>;
  u32x4 f[T::NF];
  // row: the lane's token in global memory (not read unless ok)
  template <bool VEC>
  __device__ __forceinline__ void load(const char* row, bool ok, int D, int lane) {
    const int h = lane >> 5;
#pragma unroll
    for (int s = 0; s < T::NF; ++s) {
      const int d = (2 * s + h) * T::EPC;
      f[s] = u32x4{0, 0, 0, 0};
      if constexpr (VEC) {
        if (ok && d < D) f[s] = *(const u32x4*)(row + d * T::ES);
      } else if (ok) {
        if constexpr (BF) {
          u16x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (d + e < D) v[e] = ((const unsigned short*)row)[d + e];
          f[s] = __builtin_bit_cast(u32x4, v);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (d + e < D) f[s][e] = ((const unsigned*)row)[d + e];
        }
      }
    }
  }
  // sum over d of the lane's part of own . other
  __device__ __forceinline__ float dot(const Own& b) const {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < T::NF; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (BF) {
          s = fmaf(__uint_as_float(f[i][e] << 16), __uint_as_float(b.f[i][e] << 16), s);
          s = fmaf(__uint_as_float(f[i][e] & 0xffff0000u), __uint_as_float(b.f[i][e] & 0xffff0000u), s);
        } else {
          s = fmaf(__uint_as_float(f[i][e]), __uint_as_float(b.f[i][e]), s);
        }
      }
    return s;
  }
};

// C[r][n] = sum_d tile[r0 + r][d] own[n][d], r in 0..31 (r0 a multiple of 32).
template <bool BF, int DP>
__device__ __forceinline__ f32x16 dot(const char* S, int r0, const Own<BF, DP>& own, int lane) {
  using T = Tile<BF, DP>;
  const int r = tile_row(lane), h = lane >> 5;
  const char* row = S + (r0 + r) * T::RB;
  const int x = T::swz(r);
  f32x16 c = {};
#pragma unroll
  for (int s = 0; s < T::NF; ++s) {
    const u32x4 a = *(const u32x4*)(row + (((2 * s + h) ^ x) * 16)), b = own.f[s];
    if constexpr (BF) {
      c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
    }
  }
  return c;
}

// acc[d][n] += sum_r tile[r0 + r][d] c[r][n], r in 0..31.
template <bool BF, int DP>
__device__ __forceinline__ void accum(const char* S, int r0, const f32x16& c, f32x16 (&acc)[DP / 32], int lane) {
  using T = Tile<BF, DP>;
  const int h = lane >> 5;
  if constexpr (BF) {
    // ds_read_b64_tr_b16: lane s of a 16-lane group addresses four columns of
    // row s / 4; lane i receives the rows' column 4 p(i / 4) + i % 4, where
    // p swaps the middle two of four column groups (the order of tile_row)
    const int s = lane & 15, g = (lane >> 4) & 1;
    const int pc = ((s & 1) << 1) | ((s >> 1) & 1);
    const int rl = 8 * h + (s >> 2);
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      u32x4 b;
#pragma unroll
      for (int e = 0; e < 4; ++e) b[e] = pack_bf16(c[8 * kk + 2 * e], c[8 * kk + 2 * e + 1]);
      const char* base = S + (r0 + 16 * kk) * T::RB + 8 * (pc & 1);
#pragma unroll
      for (int db = 0; db < T::ND; ++db) {
        const int ch = 4 * db + 2 * g + (pc >> 1);
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_s16x4*)(const void*)(base + rl * T::RB + ((ch ^ T::swz(rl)) * 16)));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_s16x4*)(const void*)(base + (rl + 4) * T::RB + ((ch ^ T::swz(rl + 4)) * 16)));
        u32x4 a;
        const u32x2 l2 = __builtin_bit_cast(u32x2, lo), h2 = __builtin_bit_cast(u32x2, hi);
        a[0] = l2[0]; a[1] = l2[1]; a[2] = h2[0]; a[3] = h2[1];
        acc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b),
                                                          acc[db], 0, 0, 0);
      }
    }
  } else {
    const int d = tile_row(lane);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int r = 16 * (i >> 3) + 8 * h + (i & 7);
      const char* row = S + (r0 + r) * T::RB + 4 * (d & 3);
#pragma unroll
      for (int db = 0; db < T::ND; ++db) {
        const float a = *(const float*)(row + (((8 * db + (d >> 2)) ^ T::swz(r)) * 16));
        acc[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, c[i], acc[db], 0, 0, 0);
      }
    }
  }
}

// The running softmax of a wave's 32 queries.
template <int DP>
struct Softmax {
  float m = -kInf, l = 0.f;  // maximum (log2 units; may lag) and this half's sum
  // S (scaled by c in here) of N x 32 stream keys becomes P; acc is rescaled
  // when the maximum has grown enough.
  template <int N>
  __device__ __forceinline__ void step(f32x16 (&S)[N], float c, f32x16 (&acc)[DP / 32]) {
    float t = -kInf;
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) t = fmaxf(t, S[n][i]);
    t = max_halves(t) * c;
    // The result is the same for any m that keeps the terms in range, so m
    // follows the maximum only once it lags by 2^8.
    if (__any(t > m + 8.f)) {
      const float nm = fmaxf(t, m);
      const float f = nm == -kInf ? 1.f : __builtin_amdgcn_exp2f(m - nm);
      m = nm;
      l *= f;
#pragma unroll
      for (int db = 0; db < DP / 32; ++db) acc[db] *= f;
    }
    const float off = m == -kInf ? 0.f : m;
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        S[n][i] = __builtin_amdgcn_exp2f(fmaf(S[n][i], c, -off));
        l += S[n][i];
      }
  }
};

template <bool BF, int DP>
struct SplitGeom {
  static constexpr int HALF = 32 * Tile<BF, DP>::RB;  // 32 keys, or their values
  // Two tiles in flight where they fit; wide fp32 heads work long enough on
  // either half of one to load the other meanwhile.
  static constexpr int NBUF = HALF > 8192 ? 1 : 2;
  static constexpr int NW = 4;
  static constexpr int PITCH = DP + 4;  // floats a column in the join
};
template <bool BF, int DP, bool VEC>
__global__ __launch_bounds__(256, 1) void split_kernel(const AttnParams p) {
  using T = Tile<BF, DP>;
  using Gm = SplitGeom<BF, DP>;
  constexpr int NW = Gm::NW, NBUF = Gm::NBUF;
  constexpr int LOADS = VEC ? Loader<BF, DP, 32, 1, VEC>::JB : 0;  // in flight from fetching half a tile
  __shared__ __align__(1024) char lds[NW][NBUF][2][Gm::HALF];
  __shared__ float stat[2][NW][32];
  static_assert(NW * 32 * Gm::PITCH * 4 <= (int)sizeof(lds), "the join fits the tiles' LDS");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int cols = p.G * p.TQ, ncb = (cols + 31) >> 5;
  // the blocks of one head on one XCD
  const int w = work_item(p.B * p.HK * ncb * p.splits);
  if (w < 0) return;
  const int split = w % p.splits, cb = w / p.splits % ncb, bh = w / p.splits / ncb;
  const int hk = bh % p.HK, b = bh / p.HK;
  const Span sp = span_of(p, b);
  const int c = cb * 32 + (lane & 31);
  const bool ok = c < cols;
  const int g = ok ? c / p.TQ : 0, qi = ok ? c - g * p.TQ : 0, hq = hk * p.G + g;
  const int lim = ok ? visible(p, sp, qi) : 0;
  int kend = lim;  // of any column
#pragma unroll
  for (int o = 1; o < 32; o *= 2) {
    const int x = __shfl_xor(kend, o, 64);
    kend = x > kend ? x : kend;
  }
  // this block's share of the tiles, an equal number a split
  const int tiles = (kend + 31) >> 5, t_end = (int)((int64_t)tiles * (split + 1) / p.splits);
  const int t_first = __builtin_amdgcn_readfirstlane((int)((int64_t)tiles * split / p.splits) + wave);
  const int t_last = __builtin_amdgcn_readfirstlane(t_end);

  Own<BF, DP> q;
  q.template load<VEC>(row_of(p.q, b, qi, hq, T::ES), ok, p.D, lane);
  Loader<BF, DP, 32, 1, VEC> lk, lv;
  lk.init(0, lane, p.k.st, p.D);
  lv.init(0, lane, p.v.st, p.D);
  const char* kbase = row_of(p.k, b, 0, hk, T::ES);
  const char* vbase = row_of(p.v, b, 0, hk, T::ES);
  auto fetch_k = [&](int t, int buf) {
    lk.load(kbase + (int64_t)32 * t * p.k.st * T::ES, sp.len - 32 * t, lds[wave][buf][0]);
  };
  auto fetch_v = [&](int t, int buf) {
    lv.load(vbase + (int64_t)32 * t * p.v.st * T::ES, sp.len - 32 * t, lds[wave][buf][1]);
  };
  // this wave's LDS reads are done (before their bytes are loaded over)
  auto reads_done = [] { __asm__ __volatile__("s_waitcnt lgkmcnt(0)" ::: "memory"); };
  // all its loads but the last N are done
  auto loads_done = [](auto n) {
    gemm::wait_vmcnt<decltype(n)::value>();
    __asm__ __volatile__("" ::: "memory");
  };
  using std::integral_constant;
  f32x16 acc[T::ND] = {};
  Softmax<DP> sm;
  if (t_first < t_last) {
    fetch_k(t_first, 0);
    fetch_v(t_first, 0);
  }
  for (int t = t_first, buf = 0; t < t_last; t += NW, buf ^= NBUF - 1) {
    const bool more = t + NW < t_last;
    if (NBUF == 2) {
      reads_done();
      if (more) {
        fetch_k(t + NW, buf ^ 1);
        fetch_v(t + NW, buf ^ 1);
        loads_done(integral_constant<int, 2 * LOADS>{});
      } else {
        loads_done(integral_constant<int, 0>{});
      }
    } else {
      loads_done(integral_constant<int, LOADS>{});
    }
    f32x16 S[1] = {dot<BF, DP>(lds[wave][buf][0], 0, q, lane)};
    if (NBUF == 1 && more) {
      reads_done();
      fetch_k(t + NW, 0);
    }
    const int lm = lim - 32 * t - 8 * (lane >> 5);
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (16 * (i >> 3) + (i & 7) >= lm) S[0][i] = -kInf;
    sm.step(S, p.scale_log2, acc);
    if (NBUF == 1) {
      if (more) loads_done(integral_constant<int, LOADS>{});
      else loads_done(integral_constant<int, 0>{});
    }
    accum<BF, DP>(lds[wave][buf][1], 0, S[0], acc, lane);
    if (NBUF == 1 && more) {
      reads_done();
      fetch_v(t + NW, 0);
    }
  }
  // The waves' results meet: m, l, and acc by column.
  __syncthreads();
  float* join = (float*)&lds[0][0][0][0];
  const float l = sum_halves(sm.l);
  if (lane < 32) {
    stat[0][wave][lane] = sm.m;
    stat[1][wave][lane] = l;
  }
  {
    float* row = join + (wave * 32 + (lane & 31)) * Gm::PITCH + 8 * (lane >> 5);
#pragma unroll
    for (int db = 0; db < T::ND; ++db)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *(f32x4*)(row + 32 * db + 16 * (i >> 3) + (i & 7)) = f32x4{acc[db][i], acc[db][i + 1], acc[db][i + 2], acc[db][i + 3]};
  }
  __syncthreads();
  constexpr int TPC = NW * 2;  // threads a column
  const int col = threadIdx.x / TPC, part = threadIdx.x % TPC, cc = cb * 32 + col;
  if (cc >= cols) return;
  const int64_t row = ((int64_t)b * p.HQ + hk * p.G + cc / p.TQ) * p.TQ + cc % p.TQ;
  float M = -kInf, L = 0.f, f[NW];
#pragma unroll
  for (int i = 0; i < NW; ++i) M = fmaxf(M, stat[0][i][col]);
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    f[i] = stat[0][i][col] == -kInf ? 0.f : __builtin_amdgcn_exp2f(stat[0][i][col] - M);
    L += f[i] * stat[1][i][col];
  }
  auto sum = [&](int d) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NW; ++i) s += f[i] * join[(i * 32 + col) * Gm::PITCH + d];
    return s;
  };
  if (p.splits > 1) {
    float* out = p.part + (row * p.splits + split) * (p.D + 2);
    for (int d = part; d < p.D; d += TPC) out[d] = sum(d);
    if (part == 0) {
      out[p.D] = M;
      out[p.D + 1] = L;
    }
    return;
  }
  const float inv = 1.f / L;
  char* dst = row_of(p.o, b, cc % p.TQ, hk * p.G + cc / p.TQ, T::ES);
  for (int d = part; d < p.D; d += TPC) {
    const float v = L == 0.f ? 0.f : sum(d) * inv;
    if constexpr (BF) ((__bf16*)dst)[d] = (__bf16)v;
    else ((float*)dst)[d] = v;
  }
  if (p.lse && part == 0) p.lse[row] = L == 0.f ? -kInf : (M + __builtin_amdgcn_logf(L)) * kLn2;
}

// The splits' results of one row, a block each: o = sum of f_s acc_s over sum
// of f_s l_s with f_s = 2^(m_s - max m). Wave w adds the splits w, w + 4, ..;
// the waves' sums are added in order.
template <bool BF>
__global__ __launch_bounds__(256) void join_kernel(const AttnParams p) {
  __shared__ float sums[4][kAttnMaxD];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row = blockIdx.x;
  const float* part = p.part + row * p.splits * (p.D + 2);
  // lane s holds split s's statistics (at most 64 splits)
  const bool in = lane < p.splits;
  const float m = in ? part[lane * (p.D + 2) + p.D] : -kInf, l = in ? part[lane * (p.D + 2) + p.D + 1] : 0.f;
  float M = m;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) M = fmaxf(M, __shfl_xor(M, o, 64));
  const float f = m == -kInf ? 0.f : __builtin_amdgcn_exp2f(m - M);
  float L = f * l, a = 0.f, a2 = 0.f;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) L += __shfl_xor(L, o, 64);
  const bool d0 = lane < p.D, d1 = lane + 64 < p.D;
#pragma unroll 4
  for (int s = wave; s < p.splits; s += 4) {
    const float* x = part + s * (p.D + 2);
    const float fs = __shfl(f, s, 64);
    a += fs * (d0 ? x[lane] : 0.f);
    a2 += fs * (d1 ? x[lane + 64] : 0.f);
  }
  sums[wave][lane] = a;
  sums[wave][lane + 64] = a2;
  __syncthreads();
  const int d = threadIdx.x;
  if (d < p.D) {
    const int64_t bh = row / p.TQ;
    char* dst = row_of(p.o, (int)(bh / p.HQ), row - bh * p.TQ, (int)(bh % p.HQ), BF ? 2 : 4);
    const float v = L == 0.f ? 0.f : ((sums[0][d] + sums[1][d]) + (sums[2][d] + sums[3][d])) * (1.f / L);
    if constexpr (BF) ((__bf16*)dst)[d] = (__bf16)v;
    else ((float*)dst)[d] = v;
  }
  if (p.lse && d == 0) p.lse[row] = L == 0.f ? -kInf : (M + __builtin_amdgcn_logf(L)) * kLn2;
}

}  // namespace attn

hipError_t attn_fwd_split(const AttnParams& p, bool bf16, bool vec, hipStream_t stream) {
  const int64_t items = (int64_t)p.B * p.HK * (((int64_t)p.G * p.TQ + 31) / 32) * p.splits;
  const hipError_t e = attn_by_width(p.D, [&](auto dp) {
    constexpr int DP = decltype(dp)::value;
    const dim3 grid = attn_grid(items);
    if (bf16 && vec) attn::split_kernel<true, DP, true><<<grid, 256, 0, stream>>>(p);
    else if (bf16) attn::split_kernel<true, DP, false><<<grid, 256, 0, stream>>>(p);
    else if (vec) attn::split_kernel<false, DP, true><<<grid, 256, 0, stream>>>(p);
    else attn::split_kernel<false, DP, false><<<grid, 256, 0, stream>>>(p);
    return hipGetLastError();
  });
  if (e != hipSuccess || p.splits == 1) return e;
  const dim3 grid((unsigned)((int64_t)p.B * p.HQ * p.TQ));
  if (bf16) attn::join_kernel<true><<<grid, 256, 0, stream>>>(p);
  else attn::join_kernel<false><<<grid, 256, 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace mt
