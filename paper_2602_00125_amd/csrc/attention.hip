// Attention and its gradient, gfx950, one pass over the data each.
//
//   S = scale q k^T over the visible keys, lse = log sum exp S, P = exp(S - lse)
//   o = P v
//   delta = sum_d do o, dP = do v^T, dS = P (dP - delta)
//   dq = scale dS k, dk = scale dS^T q, dv = P^T do
//
// The scores are never stored: the forward keeps a running maximum and sum,
// the backward computes P anew from lse. The same scheme serves all three
// kernels. A wave owns 32 tokens (queries; keys in the dk / dv pass), one a
// lane of each half-wave, whose vectors sit in registers as the right operand
// of the MFMAs. Tiles of the other tokens stream through LDS. A product
// stream x own comes out with the wave's token in the lane and 16 of 32 stream
// tokens in registers (f32x16), so softmax statistics are one value a lane and
// P goes back into the next product from the registers it is in:
//   dot:   C[r][n]  = sum_d tile[r][d] own[n][d]     (S, dP)
//   accum: A[d][n] += sum_r tile[r][d] C[r][n]       (o, dq; dk, dv)
// The MFMA's C holds row 8 (i / 4) + 4 h + i % 4 in register i of lane half h.
// The rows of the left operand are handed to it in an order that makes this
// row 16 (i / 8) + 8 h + i % 8 of the tile (tile_row): eight consecutive stream
// tokens a half, which is what the next product's right operand wants (no
// exchange between lanes), and eight consecutive d of a result row, written by
// 16-byte stores.
//
// Sums, statistics and accumulators are fp32. With bf16 inputs P and dS are
// rounded to bf16 (nearest even) for the second product: the matrix cores'
// operand type, an error of 2^-8 of a term where the output is rounded to
// bf16 as well. The row sum of P is taken before the rounding.
//
// Each result is summed by one block in a fixed order: no atomics. dq and
// dk / dv take a pass each, and both compute S and dP (7 products in place of
// 5): adding dq across the blocks of one pass would take atomics, or partial
// sums of 4 bytes a d for every 128 keys, which cost more than the products.
#include <hip/hip_runtime.h>

#include <type_traits>
#include <utility>

#include "attention.hpp"
#include "gemm_dma.hpp"

namespace mt {
namespace attn {

using gemm::dma16;
using gemm::dma4;
using gemm::kOOB;
using gemm::kRsrcWord3;
using gemm::lds_byte_addr;
using gemm::uniform_ptr;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kInf = __builtin_inff();

// f(0), f(1), .. f(N - 1) with constant arguments.
template <typename F, int... I>
__device__ __forceinline__ void unroll_seq(F f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void unroll(F f) {
  unroll_seq(f, std::make_integer_sequence<int, N>{});
}

// All loads and LDS accesses of this wave done, then every wave's.
__device__ __forceinline__ void wait_all_barrier() {
  __asm__ __volatile__("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// The stream row a lane hands to the MFMA as row lane & 31 (see the top).
__device__ __forceinline__ int tile_row(int lane) {
  const int m = lane & 31;
  return 16 * (m >> 4) + 8 * ((m >> 2) & 1) + 4 * ((m >> 3) & 1) + (m & 3);
}

// Maximum / sum over the two lanes (n, n + 32) that share an own token.
__device__ __forceinline__ u32x2 halves(float v) {
  return __builtin_bit_cast(
      u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false));
}
__device__ __forceinline__ float max_halves(float v) {
  const u32x2 s = halves(v);
  return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float sum_halves(float v) {
  const u32x2 s = halves(v);
  return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

__device__ __forceinline__ unsigned pack_bf16(float a, float b) {
  bf16x2 v;
  v[0] = (__bf16)a;
  v[1] = (__bf16)b;
  return __builtin_bit_cast(unsigned, v);
}

__device__ __forceinline__ float ld_elem(const char* p, int64_t i, bool bf) {
  return bf ? __uint_as_float((unsigned)((const unsigned short*)p)[i] << 16) : ((const float*)p)[i];
}

typedef __attribute__((address_space(3))) const u32x4 lds_u32x4;
__device__ __forceinline__ u32x4 lds_read16(uint32_t at) { return *(lds_u32x4*)(uintptr_t)at; }
__device__ __forceinline__ u32x2 lds_read_tr(uint32_t at) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)at));
}

// A tile of stream tokens in LDS, rows of RB bytes in 16-byte chunks whose
// index is XORed with a function of the row, so that both kinds of reads hit
// distinct banks: `dot` reads one chunk of 16 rows that differ modulo 16,
// `accum` four consecutive rows x four chunks (bf16, ds_read_b64_tr_b16) or
// two rows 8 apart (fp32, 4-byte reads).
template <bool BF, int DP>
struct Tile {
  static constexpr int ES = BF ? 2 : 4;
  static constexpr int RB = DP <= 64 ? 64 * ES : 128 * ES;
  static constexpr int EPC = 16 / ES;
  static constexpr int ND = DP / 32;
  static constexpr int NF = DP * ES / 32;  // 16-byte own fragments a lane
  static __device__ __forceinline__ int swz(int r) {
    if constexpr (!BF) return r & 15;
    else if constexpr (RB == 256) return ((r & 3) << 2) | ((r >> 2) & 3);
    else return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
  }
};

// What a wave multiplies tiles with: 32 own tokens, one a lane, in registers
template <bool BF, int DP>
struct Own {
  using T = Tile<BF, DP>;
  u32x4 f[T::NF];
  __device__ __forceinline__ u32x4 frag(int s) const { return f[s]; }
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

// or as rows of a tile in LDS (from row n0 of it, a multiple of 32).
template <bool BF, int DP>
struct OwnTile {
  using T = Tile<BF, DP>;
  uint32_t at;  // the lane's row; chunk bits as in Left
  __device__ __forceinline__ OwnTile(const char* tile, int n0, int lane) {
    const int r = lane & 31;
    at = lds_byte_addr(tile) + (n0 + r) * T::RB + (((lane >> 5) ^ T::swz(r)) * 16);
  }
  __device__ __forceinline__ u32x4 frag(int s) const { return lds_read16(at ^ (32 * s)); }
};

// A lane's left operands from a bf16 tile: for `dot`, 16-byte chunks of the
// tile's rows (in the order of tile_row); for `accum`, 16 rows x 32 columns
// transposed. Places in the tile as byte offsets whose chunk bits (from bit 4
// on, below the rows') a step changes by XOR alone: one instruction a read, and
// no address kept from one read to another.
template <bool BF, int DP>
struct Left {
  using T = Tile<BF, DP>;
  uint32_t row, lo, hi;
  __device__ __forceinline__ explicit Left(int lane) {
    const int r = tile_row(lane), h = lane >> 5;
    row = r * T::RB + ((h ^ T::swz(r)) * 16);
    // ds_read_b64_tr_b16: lane s of a 16-lane group addresses four columns of
    // row s / 4; lane i receives the rows' column 4 p(i / 4) + i % 4, where
    // p swaps the middle two of four column groups (the order of tile_row)
    const int s = lane & 15, g = (lane >> 4) & 1;
    const int pc = ((s & 1) << 1) | ((s >> 1) & 1);
    const int rl = 8 * h + (s >> 2), c = 2 * g + (pc >> 1);
    lo = rl * T::RB + ((c ^ T::swz(rl)) * 16) + 8 * (pc & 1);
    hi = (rl + 4) * T::RB + ((c ^ T::swz(rl + 4)) * 16) + 8 * (pc & 1);
  }
  // at + off: LDS address of a tile's row (off, a constant, and the row's place
  // multiples of 32 rows); chunks 2 s + h of the 32 rows from there
  __device__ __forceinline__ u32x4 rows(uint32_t at, int off, int s) const { return lds_read16(((at + row) ^ (32 * s)) + off); }
  // rows 16 kk .. + 15 and columns 32 db .. + 31 from there
  __device__ __forceinline__ u32x4 cols(uint32_t at, int off, int kk, int db) const {
    const u32x2 a = lds_read_tr(((at + lo) ^ (64 * db)) + 16 * kk * T::RB + off);
    const u32x2 b = lds_read_tr(((at + hi) ^ (64 * db)) + 16 * kk * T::RB + off);
    return u32x4{a[0], a[1], b[0], b[1]};
  }
};

__device__ __forceinline__ f32x16 mfma_bf16(const u32x4& a, const u32x4& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// C[r][n] = sum_d tile[r0 + r][d] own[n][d], r in 0..31 (r0 a multiple of 32).
template <bool BF, int DP, typename O>
__device__ __forceinline__ f32x16 dot(const char* S, int r0, const O& own, int lane) {
  using T = Tile<BF, DP>;
  const int r = tile_row(lane), h = lane >> 5;
  const char* row = S + (r0 + r) * T::RB;
  const int x = T::swz(r);
  f32x16 c = {};
#pragma unroll
  for (int s = 0; s < T::NF; ++s) {
    const u32x4 a = *(const u32x4*)(row + (((2 * s + h) ^ x) * 16)), b = own.frag(s);
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

// Stream tokens into a tile of ROWS rows by NW waves: straight into LDS where
// 16-byte loads are allowed, by element through registers elsewhere. Rows from
// `left` on and columns from D on are zero.
template <bool BF, int DP, int ROWS, int NW, bool VEC>
struct Loader {
  using T = Tile<BF, DP>;
  static constexpr int JB = ROWS * T::RB / 1024 / NW;
  static_assert(ROWS * T::RB % (1024 * NW) == 0, "whole instructions for every wave");
  uint32_t off[JB];
  int wave, lane, D;
  int64_t st;
  __device__ __forceinline__ int row(int j) const { return (1024 * (wave + NW * j) + 16 * lane) / T::RB; }
  __device__ __forceinline__ int col(int j) const {
    const int byte = 1024 * (wave + NW * j) + 16 * lane;
    return (((byte % T::RB) / 16) ^ T::swz(byte / T::RB)) * T::EPC;
  }
  __device__ __forceinline__ void init(int wave_, int lane_, int64_t st_, int D_) {
    wave = wave_;
    lane = lane_;
    D = D_;
    st = st_;
    if constexpr (VEC) {
#pragma unroll
      for (int j = 0; j < JB; ++j) off[j] = col(j) < D ? (uint32_t)((row(j) * (uint32_t)st + col(j)) * T::ES) : kOOB;
    }
  }
  // base: the tile's first token in global memory
  __device__ __forceinline__ void load(const char* base, int left, char* tile) const {
    if constexpr (VEC) {
      const __amdgpu_buffer_rsrc_t r =
          __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(uniform_ptr(base)), (short)0, 0x7fffffff, kRsrcWord3);
      const uint32_t lds0 = lds_byte_addr(tile);
#pragma unroll
      for (int j = 0; j < JB; ++j) dma16(r, row(j) < left ? off[j] : kOOB, lds0 + 1024 * (wave + NW * j));
    } else {
      for (int j = 0; j < JB; ++j) {
        const int rr = row(j), d = col(j);
        u32x4 v = {0, 0, 0, 0};
        if (rr < left) {
          const char* src = base + (rr * st + d) * T::ES;
          if constexpr (BF) {
            u16x8 w = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (d + e < D) w[e] = ((const unsigned short*)src)[e];
            v = __builtin_bit_cast(u32x4, w);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (d + e < D) v[e] = ((const unsigned*)src)[e];
          }
        }
        *(u32x4*)(tile + 1024 * (wave + NW * j) + 16 * lane) = v;
      }
    }
  }
};

// Result rows: acc[d][n] x mul (or zero) to token n's row (not written unless ok).
template <bool BF, int DP, bool VEC>
__device__ __forceinline__ void store_rows(char* row, bool ok, int D, const f32x16 (&acc)[DP / 32], float mul, bool zero,
                                           bool add, int lane) {
  if (!ok) return;
  const int h = lane >> 5;
#pragma unroll
  for (int db = 0; db < DP / 32; ++db)
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      const int d = 32 * db + 16 * kk + 8 * h;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = zero ? 0.f : acc[db][8 * kk + e] * mul;
      if constexpr (VEC && BF) {
        if (d < D) {
          u32x4* dst = (u32x4*)(row + d * 2);
          if (add) {
            const u32x4 old = *dst;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              v[2 * e] += __uint_as_float(old[e] << 16);
              v[2 * e + 1] += __uint_as_float(old[e] & 0xffff0000u);
            }
          }
          u32x4 w;
#pragma unroll
          for (int e = 0; e < 4; ++e) w[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
          *dst = w;
        }
      } else if constexpr (VEC) {
#pragma unroll
        for (int q = 0; q < 2; ++q)
          if (d + 4 * q < D) {
            f32x4* dst = (f32x4*)(row + (d + 4 * q) * 4);
            f32x4 w = {v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
            if (add) w += *dst;
            *dst = w;
          }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (d + e < D) {
            const float w = add ? v[e] + ld_elem(row, d + e, BF) : v[e];
            if constexpr (BF) ((__bf16*)row)[d + e] = (__bf16)w;
            else ((float*)row)[d + e] = w;
          }
      }
    }
}

// Work item of this block: eight runs of consecutive items, one an XCD (blocks
// go to the XCDs in turn), so that the blocks that read one head's keys share
// an L2. -1: none.
__device__ __forceinline__ int work_item(int total) {
  const int per = (total + 7) >> 3;
  const int w = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
  return (int)(blockIdx.x >> 3) < per && w < total ? w : -1;
}

// Keys of a batch element, and the key position of its query 0.
struct Span {
  int len;
  int64_t start;
};
__device__ __forceinline__ Span span_of(const AttnParams& p, int b) {
  Span s;
  s.len = p.TK;
  if (p.kv_len) {
    const int n = p.kv_len[b];
    s.len = n < 0 ? 0 : n < p.TK ? n : p.TK;
  }
  s.start = p.q_start ? (int64_t)p.q_start[b] : (int64_t)p.TK - p.TQ;
  return s;
}
// How many keys query i sees (the first ones).
__device__ __forceinline__ int visible(const AttnParams& p, const Span& s, int i) {
  if (!p.causal) return s.len;
  const int64_t n = s.start + i + 1;
  return n <= 0 ? 0 : n < s.len ? (int)n : s.len;
}

__device__ __forceinline__ char* row_of(const HeadView& v, int b, int64_t t, int h, int es) {
  return (char*)v.p + (b * v.sb + t * v.st + h * v.sh) * es;
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

// ---------------------------------------------------------------- forward
// A block holds 128 queries of one head (32 a wave) and walks the keys they
// see in tiles of BK, each tile's loads in flight while the one before is
// worked on.
template <bool BF, int DP, bool VEC>
__global__ __launch_bounds__(256, 2) void fwd_kernel(const AttnParams p) {
  using T = Tile<BF, DP>;
  constexpr int BK = BF ? 64 : 32, N = BK / 32, BYTES = BK * T::RB;
  __shared__ __align__(1024) char lds[2][2][BYTES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nqb = (p.TQ + 127) >> 7;
  const int w = work_item(p.B * p.HQ * nqb);
  if (w < 0) return;
  // a key head's query heads together; the blocks that see most keys first
  const int g = w % p.G, qb = nqb - 1 - (w / p.G) % nqb, bh = w / p.G / nqb;
  const int hk = bh % p.HK, b = bh / p.HK, hq = hk * p.G + g;
  const Span sp = span_of(p, b);
  const int q0 = qb * 128 + wave * 32, qi = q0 + (lane & 31);
  const bool ok = qi < p.TQ;
  const int lim = ok ? visible(p, sp, qi) : 0;
  const int last = qb * 128 + 127 < p.TQ ? qb * 128 + 127 : p.TQ - 1;
  const int kend = visible(p, sp, last);  // of the whole block
  const int kall = visible(p, sp, qb * 128) / BK * BK;  // tiles that all its queries see whole
  const int wlast = q0 + 31 < p.TQ ? q0 + 31 : p.TQ - 1;
  const int wmax = q0 < p.TQ ? visible(p, sp, wlast) : 0;  // of this wave

  Own<BF, DP> q;
  q.template load<VEC>(row_of(p.q, b, ok ? qi : 0, hq, T::ES), ok, p.D, lane);
  Loader<BF, DP, BK, 4, VEC> lk, lv;
  lk.init(wave, lane, p.k.st, p.D);
  lv.init(wave, lane, p.v.st, p.D);
  const char* kbase = row_of(p.k, b, 0, hk, T::ES);
  const char* vbase = row_of(p.v, b, 0, hk, T::ES);
  auto fetch = [&](int k0, int buf) {
    lk.load(kbase + (int64_t)k0 * p.k.st * T::ES, sp.len - k0, lds[buf][0]);
    lv.load(vbase + (int64_t)k0 * p.v.st * T::ES, sp.len - k0, lds[buf][1]);
  };
  f32x16 acc[T::ND] = {};
  Softmax<DP> sm;
  auto tile = [&](auto masked, int k0, int buf) {
    wait_all_barrier();
    if (k0 + BK < kend) fetch(k0 + BK, buf ^ 1);
    if (masked && k0 >= wmax) return;
    f32x16 S[N];
#pragma unroll
    for (int n = 0; n < N; ++n) S[n] = dot<BF, DP>(lds[buf][0], 32 * n, q, lane);
    if constexpr (masked) {
      const int lm = lim - k0 - 8 * (lane >> 5);
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (32 * n + 16 * (i >> 3) + (i & 7) >= lm) S[n][i] = -kInf;
    }
    sm.step(S, p.scale_log2, acc);
#pragma unroll
    for (int n = 0; n < N; ++n) accum<BF, DP>(lds[buf][1], 32 * n, S[n], acc, lane);
  };
  int k0 = 0, buf = 0;
  if (kend > 0) fetch(0, 0);
  for (; k0 < kall; k0 += BK, buf ^= 1) tile(std::false_type{}, k0, buf);
  for (; k0 < kend; k0 += BK, buf ^= 1) tile(std::true_type{}, k0, buf);
  const float l = sum_halves(sm.l);
  store_rows<BF, DP, VEC>(row_of(p.o, b, ok ? qi : 0, hq, T::ES), ok, p.D, acc, 1.f / l, l == 0.f, false, lane);
  if (p.lse && ok && lane < 32)
    p.lse[((int64_t)b * p.HQ + hq) * p.TQ + qi] = l == 0.f ? -kInf : (sm.m + __builtin_amdgcn_logf(l)) * kLn2;
}

// Few queries against many keys (a token of each sequence against its cache;
// short chunks): too few blocks of 128 queries to fill the chip, and the keys'
// bytes are what counts. The queries of all heads of a key head are columns
// side by side, 32 to a block, so that each key is read once for all of them;
// the keys are shared by `splits` blocks and within a block by its waves, each
// with LDS buffers of its own and no barrier between them: a wave's next tile
// is in flight while it works on one. The waves' results are joined in LDS,
// the blocks' by join_kernel, in order.
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

// --------------------------------------------------------------- backward
// dq: the forward's walk with two tiles' products before and one after the
// softmax. Also delta, which the dk / dv pass reads.
template <bool BF, int DP, bool VEC>
__global__ __launch_bounds__(256, 2) void dq_kernel(const AttnParams p) {
  using T = Tile<BF, DP>;
  constexpr int BK = BF ? 64 : 32, N = BK / 32, BYTES = BK * T::RB;
  __shared__ __align__(1024) char lds[2][2][BYTES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nqb = (p.TQ + 127) >> 7;
  const int w = work_item(p.B * p.HQ * nqb);
  if (w < 0) return;
  const int g = w % p.G, qb = nqb - 1 - (w / p.G) % nqb, bh = w / p.G / nqb;
  const int hk = bh % p.HK, b = bh / p.HK, hq = hk * p.G + g;
  const Span sp = span_of(p, b);
  const int q0 = qb * 128 + wave * 32, qi = q0 + (lane & 31);
  const bool ok = qi < p.TQ;
  const int lim = ok ? visible(p, sp, qi) : 0;
  const int last = qb * 128 + 127 < p.TQ ? qb * 128 + 127 : p.TQ - 1;
  const int kend = p.with_dq ? visible(p, sp, last) : 0, kall = visible(p, sp, qb * 128) / BK * BK;
  const int wlast = q0 + 31 < p.TQ ? q0 + 31 : p.TQ - 1;
  const int wmax = q0 < p.TQ ? visible(p, sp, wlast) : 0;

  Loader<BF, DP, BK, 4, VEC> lk, lv;
  lk.init(wave, lane, p.k.st, p.D);
  lv.init(wave, lane, p.v.st, p.D);
  const char* kbase = row_of(p.k, b, 0, hk, T::ES);
  const char* vbase = row_of(p.v, b, 0, hk, T::ES);
  auto fetch = [&](int k0, int buf) {
    lk.load(kbase + (int64_t)k0 * p.k.st * T::ES, sp.len - k0, lds[buf][0]);
    lv.load(vbase + (int64_t)k0 * p.v.st * T::ES, sp.len - k0, lds[buf][1]);
  };
  if (kend > 0) fetch(0, 0);
  Own<BF, DP> q, go;
  const int64_t qrow = ok ? qi : 0, stat = ((int64_t)b * p.HQ + hq) * p.TQ + qrow;
  go.template load<VEC>(row_of(p.dout, b, qrow, hq, T::ES), ok, p.D, lane);
  q.template load<VEC>(row_of(p.o, b, qrow, hq, T::ES), ok, p.D, lane);
  const float delta = sum_halves(go.dot(q));
  if (ok && lane < 32) {  // as the dk / dv pass adds them to its products
    p.delta[stat] = -p.lse[stat] / p.scale;
    p.delta[(int64_t)p.B * p.HQ * p.TQ + stat] = -delta;
  }
  if (!p.with_dq) return;
  q.template load<VEC>(row_of(p.q, b, qrow, hq, T::ES), ok, p.D, lane);
  // P = exp2(c S - lse2). A query that sees nothing has lse = -inf; all its
  // keys are masked.
  const float lse2 = ok ? p.lse[stat] * kLog2e : 0.f;

  f32x16 acc[T::ND] = {};
  auto tile = [&](auto masked, int k0, int buf) {
    wait_all_barrier();
    if (k0 + BK < kend) fetch(k0 + BK, buf ^ 1);
    if (masked && k0 >= wmax) return;
    const char *K = lds[buf][0], *V = lds[buf][1];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      f32x16 S = dot<BF, DP>(K, 32 * n, q, lane);
      const f32x16 dP = dot<BF, DP>(V, 32 * n, go, lane);
      const int lm = lim - k0 - 8 * (lane >> 5);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        S[i] = __builtin_amdgcn_exp2f(fmaf(S[i], p.scale_log2, -lse2)) * (dP[i] - delta);
        if (masked && 32 * n + 16 * (i >> 3) + (i & 7) >= lm) S[i] = 0.f;
      }
      accum<BF, DP>(K, 32 * n, S, acc, lane);
    }
  };
  int k0 = 0, buf = 0;
  for (; k0 < kall; k0 += BK, buf ^= 1) tile(std::false_type{}, k0, buf);
  for (; k0 < kend; k0 += BK, buf ^= 1) tile(std::true_type{}, k0, buf);
  store_rows<BF, DP, VEC>(row_of(p.dq, b, qrow, hq, T::ES), ok, p.D, acc, p.scale, false, p.accumulate, lane);
}

// dk and dv: a block holds 128 keys of one head, 32 a wave, and walks the
// queries that see them, over all query heads of the group. QS waves share the
// same keys, each with its 32 queries of every tile; their accumulators are
// added in LDS at the end. So a block fills a CU with two waves a SIMD, which a
// wave alone could not hide LDS's latency with (measured on 4 x 4096 x 32 heads
// of 128, bf16: 1.8 ms with one wave a SIMD, 1.1 with two), and few blocks take
// half as long. Two accumulators leave no room for both keys and values of wide
// bf16 heads in 256 registers: the values stay in LDS there. Wide fp32 heads
// take all registers of a SIMD for one wave.
template <bool BF, int DP, int KG, int QS, int SUB>
struct KvGeom {
  using T = Tile<BF, DP>;
  static constexpr bool VLDS = BF && DP > 64;
  static constexpr int NW = KG * QS, BQ = 32 * QS * SUB, BKV = 32 * KG;
  static constexpr int BYTES = BQ * T::RB;
  // waves a SIMD that its registers are for
  static constexpr int OCC = BF || DP <= 64 ? 2 : 1;
};
template <bool BF, int DP, bool VEC, int KG, int QS, int SUB>
__global__ __launch_bounds__((64 * KG * QS), (KvGeom<BF, DP, KG, QS, SUB>::OCC)) void dkv_kernel(const AttnParams p) {
  using T = Tile<BF, DP>;
  using Gm = KvGeom<BF, DP, KG, QS, SUB>;
  constexpr bool VLDS = Gm::VLDS;
  constexpr int BQ = Gm::BQ, NW = Gm::NW, BKV = Gm::BKV;
  __shared__ __align__(1024) char lds[2][2][Gm::BYTES];
  __shared__ __align__(1024) char vlds[VLDS ? BKV * T::RB : 16];
  __shared__ __align__(256) float stats[2][2][64];  // lse, delta of the tile's queries
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kg = wave % KG, qs = wave / KG;  // which 32 keys, which queries of a tile
  const int nkb = (p.TK + BKV - 1) / BKV;
  // As many heads of an XCD at a time as fill its 32 CUs (their queries share
  // the L2), the blocks that see most queries first
  const int heads = p.B * p.HK, per = heads >> 3;
  int kb, bh;
  if (heads & 7) {
    if ((int)blockIdx.x >= heads * nkb) return;
    kb = blockIdx.x / heads;
    bh = blockIdx.x - kb * heads;
  } else {
    const int i = blockIdx.x >> 3, some = (32 + nkb - 1) / nkb, most = some < per ? some : per;
    const int h0 = i / (most * nkb) * most, now = per - h0 < most ? per - h0 : most, r = i - h0 * nkb;
    kb = r / now;
    bh = (blockIdx.x & 7) * per + h0 + (r - kb * now);
  }
  const int hk = bh % p.HK, b = bh / p.HK;
  const Span sp = span_of(p, b);
  const int k0 = kb * BKV + kg * 32, kj = k0 + (lane & 31);
  const bool in = kj < p.TK, ok = kj < sp.len;
  const int krow = in ? kj : 0;
  // query tiles from the first that sees a key of the block; from q_all on
  // every query sees all of them, before wfirst none sees a key of the wave
  const bool any = kb * BKV < sp.len;
  auto first_for = [&](int key) {
    const int64_t i = p.causal ? (int64_t)key - sp.start : 0;
    return i < 0 ? 0 : i < p.TQ ? (int)i : p.TQ;
  };
  const int q_first = any ? first_for(kb * BKV) / BQ * BQ : p.TQ;
  const int tiles = (p.TQ - q_first + BQ - 1) / BQ;
  const int q_all = first_for(kb * BKV + BKV - 1), wfirst = first_for(k0);
  const bool wave_on = k0 < sp.len;
  const int see = first_for(kj);  // queries from here on see the lane's key

  Loader<BF, DP, BQ, NW, VEC> lq, lo;
  lq.init(wave, lane, p.q.st, p.D);
  lo.init(wave, lane, p.dout.st, p.D);
  auto fetch = [&](int it, int buf) {
    const int hq = hk * p.G + it / tiles, t0 = q_first + (tiles - 1 - it % tiles) * BQ;
    lq.load(row_of(p.q, b, t0, hq, T::ES), p.TQ - t0, lds[buf][0]);
    lo.load(row_of(p.dout, b, t0, hq, T::ES), p.TQ - t0, lds[buf][1]);
    if (wave < 2) {  // a 4-byte statistic a lane
      const float* s = p.delta + ((int64_t)wave * p.B * p.HQ + (int64_t)b * p.HQ + hq) * p.TQ + t0;
      const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<char*>(uniform_ptr((const char*)s)), (short)0, 0x7fffffff, kRsrcWord3);
      dma4(r, lane < BQ && lane < p.TQ - t0 ? 4u * lane : kOOB, lds_byte_addr(stats[buf][wave]));
    }
  };
  const int iters = tiles * p.G;
  if (iters > 0) fetch(0, 0);
  Own<BF, DP> k;
  k.template load<VEC>(row_of(p.k, b, krow, hk, T::ES), ok, p.D, lane);
  const auto v = [&] {
    if constexpr (VLDS) {
      Loader<BF, DP, BKV, NW, VEC> l;
      l.init(wave, lane, p.v.st, p.D);
      if (iters > 0) l.load(row_of(p.v, b, kb * BKV, hk, T::ES), sp.len - kb * BKV, vlds);
      return OwnTile<BF, DP>(vlds, 32 * kg, lane);
    } else {
      Own<BF, DP> o;
      o.template load<VEC>(row_of(p.v, b, krow, hk, T::ES), ok, p.D, lane);
      return o;
    }
  }();
  f32x16 ak[T::ND] = {}, av[T::ND] = {};
  const Left<BF, DP> left(lane);
  int it = 0, buf = 0;
  auto tile = [&](auto masked, int t0) {
    wait_all_barrier();
    if (it + 1 < iters) fetch(it + 1, buf ^ 1);
    const char *Q = lds[buf][0], *O = lds[buf][1];
    const float *lse = stats[buf][0] + 8 * (lane >> 5), *delta = stats[buf][1] + 8 * (lane >> 5);
    ++it;
    buf ^= 1;
    if (!wave_on || (masked && t0 + BQ <= wfirst)) return;
    const int from = see - t0 - 8 * (lane >> 5);
    if constexpr (BF) {
      // The MFMAs in order, each step's left operand read AHEAD steps before it,
      // and the softmax's arithmetic between them: P under the product for dP,
      // dS under the one for dv.
      constexpr int NF = T::NF, NA = 2 * T::ND, PER = 2 * NF + 2 * NA, STEPS = SUB * PER;
      constexpr int AHEAD = 4, VA = 3;
      const uint32_t Qr = lds_byte_addr(Q) + 32 * SUB * qs * T::RB;
      auto load = [&](int step) {
        const int i = step % PER, at = step / PER * 32 * T::RB, O = at + Gm::BYTES;
        if (i < NF) return left.rows(Qr, at, i);
        if (i < 2 * NF) return left.rows(Qr, O, i - NF);
        const int j = (i - 2 * NF) % NA;
        return left.cols(Qr, i < 2 * NF + NA ? O : at, j / T::ND, j % T::ND);
      };
      auto vt = v;
      if constexpr (VLDS) __asm__ __volatile__("" : "+v"(vt.at));  // its addresses are not kept across tiles
      u32x4 ring[AHEAD], vring[VA];
      f32x16 S, dP;
      u32x4 P[2], dS[2];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) ring[i] = load(i);
      __builtin_amdgcn_sched_barrier(0);
      unroll<STEPS>([&](auto step) {
        constexpr int i = step % PER;
        const int r0 = 32 * (step / PER + SUB * qs);
        const u32x4 a = ring[step % AHEAD];
        if (i == 0) {  // lse and delta come in as the products' first terms
#pragma unroll
          for (int x = 0; x < 16; ++x) S[x] = lse[r0 + 16 * (x >> 3) + (x & 7)];
        }
        if (i == NF - 2) {
#pragma unroll
          for (int x = 0; x < 16; ++x) dP[x] = delta[r0 + 16 * (x >> 3) + (x & 7)];
        }
        if (i < NF) {
          S = mfma_bf16(a, k.frag(i), S);
        } else if (i < 2 * NF) {
          dP = mfma_bf16(a, VLDS ? vring[(i - NF) % VA] : vt.frag(i - NF), dP);
        } else {
          const int j = (i - 2 * NF) % NA, kk = j / T::ND, db = j % T::ND;
          if (i < 2 * NF + NA) av[db] = mfma_bf16(a, P[kk], av[db]);
          else ak[db] = mfma_bf16(a, dS[kk], ak[db]);
        }
        if (step + AHEAD < STEPS) ring[step % AHEAD] = load(step + AHEAD);
        if constexpr (VLDS) {
          const int f = i + VA - NF;
          if (f >= 0 && f < NF) vring[f % VA] = vt.frag(f);
        }
        // pairs of elements: NF steps share the 8 of P, NA those of dS
        if (i >= NF && i < 2 * NF) {
#pragma unroll
          for (int e = (i - NF) * 8 / NF; e < (i - NF + 1) * 8 / NF; ++e) {
#pragma unroll
            for (int x = 2 * e; x < 2 * e + 2; ++x) {
              S[x] = __builtin_amdgcn_exp2f(S[x] * p.scale_log2);
              if (masked && r0 + 16 * (x >> 3) + (x & 7) < from) S[x] = 0.f;
            }
            P[e >> 2][e & 3] = pack_bf16(S[2 * e], S[2 * e + 1]);
          }
        } else if (i >= 2 * NF && i < 2 * NF + NA) {
#pragma unroll
          for (int e = (i - 2 * NF) * 8 / NA; e < (i - 2 * NF + 1) * 8 / NA; ++e) {
#pragma unroll
            for (int x = 2 * e; x < 2 * e + 2; ++x) dP[x] *= S[x];
            dS[e >> 2][e & 3] = pack_bf16(dP[2 * e], dP[2 * e + 1]);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      });
    } else {
#pragma unroll
      for (int n = 0; n < SUB; ++n) {
        const int r0 = 32 * (n + SUB * qs);
        f32x16 S = dot<BF, DP>(Q, r0, k, lane);
        f32x16 dP = dot<BF, DP>(O, r0, v, lane);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int r = r0 + 16 * (i >> 3) + (i & 7);
          S[i] = __builtin_amdgcn_exp2f((S[i] + lse[r]) * p.scale_log2);
          if (masked && r < from) S[i] = 0.f;
          dP[i] = S[i] * (dP[i] + delta[r]);
        }
        accum<BF, DP>(O, r0, S, av, lane);
        accum<BF, DP>(Q, r0, dP, ak, lane);
      }
    }
  };
  // from the last query on, so that the blocks of a head read the same tiles at
  // a time whatever their first query is
  for (int g = 0; g < p.G && iters > 0; ++g) {
    int t0 = q_first + (tiles - 1) * BQ;
    for (; t0 >= q_first && t0 >= q_all; t0 -= BQ) tile(std::false_type{}, t0);
    for (; t0 >= q_first; t0 -= BQ) tile(std::true_type{}, t0);
  }
  // the waves of the same keys meet, one accumulator at a time
  if constexpr (QS > 1) {
    constexpr int FL = 16 * T::ND * 64;  // floats of a wave's accumulator
    static_assert(QS == 2 && KG * FL * 4 <= (int)sizeof(lds), "the accumulators of a wave of each pair fit the tiles' LDS");
    auto meet = [&](f32x16 (&a)[T::ND]) {
      f32x4* mine = (f32x4*)&lds[0][0][0] + kg * (FL / 4) + lane;
      __syncthreads();
      if (qs == 1) {
#pragma unroll
        for (int db = 0; db < T::ND; ++db)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            mine[(4 * db + i) * 64] = f32x4{a[db][4 * i], a[db][4 * i + 1], a[db][4 * i + 2], a[db][4 * i + 3]};
      }
      __syncthreads();
      if (qs == 0) {
#pragma unroll
        for (int db = 0; db < T::ND; ++db)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const f32x4 x = mine[(4 * db + i) * 64];
#pragma unroll
            for (int e = 0; e < 4; ++e) a[db][4 * i + e] += x[e];
          }
      }
    };
    meet(ak);
    meet(av);
    if (qs) return;
  }
  // keys past the batch element's length take no part: zero
  if (p.dk.p)
    store_rows<BF, DP, VEC>(row_of(p.dk, b, krow, hk, T::ES), in && (ok || !p.accumulate), p.D, ak, p.scale, !ok,
                            p.accumulate, lane);
  if (p.dv.p)
    store_rows<BF, DP, VEC>(row_of(p.dv, b, krow, hk, T::ES), in && (ok || !p.accumulate), p.D, av, 1.f, !ok,
                            p.accumulate, lane);
}

}  // namespace attn

namespace {

template <typename F>
hipError_t by_width(int D, F f) {
  if (D <= 64) return f(std::integral_constant<int, 64>{});
  if (D <= 96) return f(std::integral_constant<int, 96>{});
  return f(std::integral_constant<int, 128>{});
}
// the grid of `items` work items (attn::work_item)
dim3 grid_of(int64_t items) { return dim3((unsigned)((items + 7) / 8 * 8)); }

#define MT_ATTN_LAUNCH(kernel, items)                                                               \
  by_width(p.D, [&](auto dp) {                                                                      \
    constexpr int DP = decltype(dp)::value;                                                         \
    const dim3 grid = grid_of(items);                                                               \
    if (bf16 && vec) attn::kernel<true, DP, true><<<grid, 256, 0, stream>>>(p);                     \
    else if (bf16) attn::kernel<true, DP, false><<<grid, 256, 0, stream>>>(p);                      \
    else if (vec) attn::kernel<false, DP, true><<<grid, 256, 0, stream>>>(p);                       \
    else attn::kernel<false, DP, false><<<grid, 256, 0, stream>>>(p);                               \
    return hipGetLastError();                                                                       \
  })

}  // namespace

hipError_t attn_fwd(const AttnParams& p, bool bf16, bool vec, hipStream_t stream) {
  return MT_ATTN_LAUNCH(fwd_kernel, (int64_t)p.B * p.HQ * ((p.TQ + 127) / 128));
}
hipError_t attn_fwd_split(const AttnParams& p, bool bf16, bool vec, hipStream_t stream) {
  const int64_t items = (int64_t)p.B * p.HK * (((int64_t)p.G * p.TQ + 31) / 32) * p.splits;
  const hipError_t e = by_width(p.D, [&](auto dp) {
    constexpr int DP = decltype(dp)::value;
    const dim3 grid = grid_of(items);
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
hipError_t attn_bwd_dq(const AttnParams& p, bool bf16, bool vec, hipStream_t stream) {
  return MT_ATTN_LAUNCH(dq_kernel, (int64_t)p.B * p.HQ * ((p.TQ + 127) / 128));
}
hipError_t attn_bwd_dkv(const AttnParams& p, bool bf16, bool vec, hipStream_t stream) {
  return by_width(p.D, [&](auto dp) {
    constexpr int DP = decltype(dp)::value;
    const int64_t heads = (int64_t)p.B * p.HK;
    if (bf16) {
      const dim3 grid = grid_of(heads * ((p.TK + 32 * 4 - 1) / (32 * 4)));
      constexpr int T = 64 * 4 * 2;
      if (vec) attn::dkv_kernel<true, DP, true, 4, 2, 1><<<grid, T, 0, stream>>>(p);
      else attn::dkv_kernel<true, DP, false, 4, 2, 1><<<grid, T, 0, stream>>>(p);
    } else {
      const dim3 grid = grid_of(heads * ((p.TK + 127) / 128));
      constexpr int QS = DP <= 64 ? 2 : 1;
      if (vec) attn::dkv_kernel<false, DP, true, 4, QS, 1><<<grid, 256 * QS, 0, stream>>>(p);
      else attn::dkv_kernel<false, DP, false, 4, QS, 1><<<grid, 256 * QS, 0, stream>>>(p);
    }
    return hipGetLastError();
  });
}

}  // namespace mt
