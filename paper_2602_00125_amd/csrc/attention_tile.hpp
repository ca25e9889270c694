// What the attention kernels share (attention.hip, attention_split.hip): tiles
// of tokens in LDS, their loads and reads, result rows, the order of work.
//
// A wave owns 32 tokens, one a lane of each half-wave; tiles of the other tokens
// stream through LDS. A product stream x own has the wave's token in the lane
// and 16 of 32 stream tokens in registers (f32x16): the MFMA's C holds row
// 8 (i / 4) + 4 h + i % 4 in register i of lane half h. The rows of the left
// operand are handed to it in an order that makes this row 16 (i / 8) + 8 h +
// i % 8 of the tile (tile_row): eight consecutive stream tokens a half, which is
// what the next product's right operand wants (no exchange between lanes), and
// eight consecutive d of a result row, written by 16-byte stores.
#pragma once
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

// The wave's LDS accesses and all its loads but the last N done, then every wave's.
template <int N>
__device__ __forceinline__ void wait_barrier() {
  __asm__ __volatile__("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}
// The same with no regard to loads.
__device__ __forceinline__ void wait_lds_barrier() { __asm__ __volatile__("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

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
      if (left >= ROWS) {  // the test of the rows would be two vector instructions a load
#pragma unroll
        for (int j = 0; j < JB; ++j) dma16(r, off[j], lds0 + 1024 * (wave + NW * j));
      } else {
#pragma unroll
        for (int j = 0; j < JB; ++j) dma16(r, row(j) < left ? off[j] : kOOB, lds0 + 1024 * (wave + NW * j));
      }
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

// Keys of a batch element that any query of the call sees (what the last one
// does: keys past them are not read, as those past the length), and the key
// position of its query 0.
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
  if (p.causal) {
    const int64_t n = s.start + p.TQ;
    s.len = n <= 0 ? 0 : n < s.len ? (int)n : s.len;
  }
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

}  // namespace attn

template <typename F>
hipError_t attn_by_width(int D, F f) {
  if (D <= 64) return f(std::integral_constant<int, 64>{});
  if (D <= 96) return f(std::integral_constant<int, 96>{});
  return f(std::integral_constant<int, 128>{});
}
// the grid of `items` work items (attn::work_item)
inline dim3 attn_grid(int64_t items) { return dim3((unsigned)((items + 7) / 8 * 8)); }

}  // namespace mt
