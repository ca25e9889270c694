// The norm of queries and keys for each head and the rotary rotation in one
// pass, with its gradient, gfx950. For a head's row x of D values:
//
//   r = (mean x^2 + eps)^(-1/2),  n = x r,  u = n w,  y = rotate(u)
//
// rotate turns pair i of the first R values by the angle whose cosine and
// sine the tables hold for the row's token: (a, b) -> (a c - b s, b c + a s),
// pairs side by side (2 i, 2 i + 1) or halves apart (i, i + R / 2); the rest
// passes. The gradient:
//
//   g = rotate^T dy,  dw = sum over rows of g n,  e = g w
//   dx = r (e - n mean(n e))
//
// x is read, y (dx) written; r is computed anew in the backward, nothing is
// kept. Bound: HBM (4 x 4096 tokens, 40 heads of 128, bf16, 0.34 GB from HBM: 77 us
// = 4.4 TB/s; the gradient of 8 x 1021, 32 heads of 64, fp32, 0.20 GB: 36 us and 4
// for dw = 5.0). A row is held by L lanes (a power of two), VEC values each, its
// sums taken across them; a group of lanes takes several heads of one token,
// whose row of the tables and weights it reads once. Rows that do not allow
// vectors go to a kernel of a wave a row, by element. A token a sequence costs
// the launch (64 x 40 heads of 128: 4 us of kernel, 6 a call).
//
// dw: each lane keeps the sums of its columns over the rows it meets, a block
// adds its groups' in order, and a second launch the blocks' in order.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "kernels.hpp"

namespace mt {
namespace headnorm {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <bool BF, int VEC>
__device__ __forceinline__ void load(const char* p, float (&v)[VEC]) {
  if constexpr (BF) {
    uint32_t u[VEC / 2];
    if constexpr (VEC == 8) {
      const u32x4 t = *(const u32x4*)p;
#pragma unroll
      for (int e = 0; e < 4; ++e) u[e] = t[e];
    } else {
      const u32x2 t = *(const u32x2*)p;
      u[0] = t[0];
      u[1] = t[1];
    }
#pragma unroll
    for (int e = 0; e < VEC / 2; ++e) {
      v[2 * e] = __uint_as_float(u[e] << 16);
      v[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int q = 0; q < VEC / 4; ++q) {
      const f32x4 t = ((const f32x4*)p)[q];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * q + e] = t[e];
    }
  }
}
template <bool BF, int VEC>
__device__ __forceinline__ void store(char* p, const float (&v)[VEC]) {
  if constexpr (BF) {
    uint32_t u[VEC / 2];
#pragma unroll
    for (int e = 0; e < VEC / 2; ++e) {
      bf16x2 t;
      t[0] = (__bf16)v[2 * e];
      t[1] = (__bf16)v[2 * e + 1];
      u[e] = __builtin_bit_cast(uint32_t, t);
    }
    if constexpr (VEC == 8) *(u32x4*)p = u32x4{u[0], u[1], u[2], u[3]};
    else *(u32x2*)p = u32x2{u[0], u[1]};
  } else {
#pragma unroll
    for (int q = 0; q < VEC / 4; ++q) ((f32x4*)p)[q] = f32x4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
  }
}
template <bool BF>
__device__ __forceinline__ float load1(const char* p, int64_t i) {
  if constexpr (BF) return __uint_as_float((unsigned)((const unsigned short*)p)[i] << 16);
  else return ((const float*)p)[i];
}
template <bool BF>
__device__ __forceinline__ void store1(char* p, int64_t i, float v) {
  if constexpr (BF) ((__bf16*)p)[i] = (__bf16)v;
  else ((float*)p)[i] = v;
}

// Where a head's row starts; heads 0 .. HQ-1 are the queries', then the keys'.
__device__ __forceinline__ char* row_of(const HeadView& q, const HeadView& k, int HQ, int64_t b, int64_t t, int head, int es) {
  const HeadView& v = head < HQ ? q : k;
  return (char*)v.p + (b * v.sb + t * v.st + (head < HQ ? head : head - HQ) * v.sh) * es;
}

// The value of the lane n places on, in turn within a row of 16 lanes (a vector
// instruction's own operand path; __shfl goes through LDS).
template <int N>
__device__ __forceinline__ float row16(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x120 + N, 0xf, 0xf, false));
}
__device__ __forceinline__ float group_sum(float v, int L) {
  if (L == 16) {
    v += row16<8>(v);
    v += row16<4>(v);
    v += row16<2>(v);
    return v + row16<1>(v);
  }
  for (int o = L >> 1; o; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// Cosines and sines of the pairs a lane's VEC values belong to: c, s[e] for
// value e (halves apart) or for pair e (side by side, VEC / 2 of them);
// identity past R.
template <int VEC>
struct Angles {
  float c[VEC], s[VEC];
  __device__ __forceinline__ void load(const HeadNormParams& p, int64_t b, int64_t t, int d0) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      c[e] = 1.f;
      s[e] = 0.f;
    }
    if (d0 >= p.R) return;
    const float* cr = p.cos + b * p.cos_sb + t * p.cos_st;
    const float* sr = p.sin + b * p.sin_sb + t * p.sin_st;
    const int half = p.R >> 1;
    if (p.interleaved) {
#pragma unroll
      for (int e = 0; e < VEC / 2; ++e)
        if (d0 + 2 * e < p.R) {
          c[e] = cr[d0 / 2 + e];
          s[e] = sr[d0 / 2 + e];
        }
    } else {
      const int i = d0 < half ? d0 : d0 - half;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        c[e] = cr[i + e];
        s[e] = d0 < half ? sr[i + e] : -sr[i + e];
      }
    }
  }
};
// v := rotate(v) (TRANSPOSED: by the negated angles). partner: the lane that
// holds the other halves of this lane's pairs.
template <int VEC, bool TRANSPOSED>
__device__ __forceinline__ void rotate(float (&v)[VEC], const Angles<VEC>& a, const HeadNormParams& p, int partner) {
  const float sg = TRANSPOSED ? -1.f : 1.f;
  if (p.interleaved) {
#pragma unroll
    for (int e = 0; e < VEC / 2; ++e) {
      const float x = v[2 * e], y = v[2 * e + 1], s = sg * a.s[e];
      v[2 * e] = x * a.c[e] - y * s;
      v[2 * e + 1] = y * a.c[e] + x * s;
    }
  } else if (p.L == 16 && p.R == 16 * VEC) {  // whole heads of 16 lanes: the other half is 8 lanes on
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = v[e] * a.c[e] - row16<8>(v[e]) * (sg * a.s[e]);
  } else {
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = v[e] * a.c[e] - __shfl(v[e], partner, 64) * (sg * a.s[e]);
  }
}

// What a group of L lanes works on: HPG heads of one token at a time.
struct Lanes {
  int l, d0, partner;
  bool on;
  template <int VEC>
  __device__ __forceinline__ void init(const HeadNormParams& p) {
    const int lane = threadIdx.x & 63;
    l = lane & (p.L - 1);
    d0 = l * VEC;
    on = d0 < p.D;
    const int half = p.R >> 1;
    partner = lane;
    if (d0 < half) partner = lane + half / VEC;
    else if (d0 < p.R) partner = lane - half / VEC;
  }
};

// A launch has fewer than 2^32 threads along x: more blocks go along y.
constexpr int64_t kMaxX = 1 << 23;
__device__ __forceinline__ int64_t block_index() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

template <bool XB, bool YB, int VEC, int HPG>
__global__ __launch_bounds__(256) void fwd_kernel(const HeadNormParams p) {
  Lanes ln;
  ln.init<VEC>(p);
  const int heads = p.HQ + p.HK, chunks = (heads + HPG - 1) / HPG;
  const int64_t unit = (block_index() * 256 + threadIdx.x) >> p.L_shift;
  const int64_t tok = unit / chunks;
  if (tok >= (int64_t)p.B * p.T) return;  // whole groups leave together
  const int h0 = (int)(unit - tok * chunks) * HPG;
  const int64_t b = tok / p.T, t = tok - b * p.T;
  float x[HPG][VEC];
#pragma unroll
  for (int i = 0; i < HPG; ++i) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) x[i][e] = 0.f;
    if (ln.on && h0 + i < heads)
      load<XB, VEC>(row_of(p.q, p.k, p.HQ, b, t, h0 + i, XB ? 2 : 4) + ln.d0 * (XB ? 2 : 4), x[i]);
  }
  Angles<VEC> a;
  a.load(p, b, t, ln.d0);
#pragma unroll
  for (int i = 0; i < HPG; ++i) {
    const int head = h0 + i;
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < VEC; ++e) ss = fmaf(x[i][e], x[i][e], ss);
    const float r = rsqrtf(group_sum(ss, p.L) * p.inv_D + p.eps);
    const float* w = head < p.HQ ? p.wq : p.wk;
    float wv[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) wv[e] = 1.f;
    if (w && ln.on && head < heads) load<false, VEC>((const char*)(w + ln.d0), wv);
#pragma unroll
    for (int e = 0; e < VEC; ++e) x[i][e] = x[i][e] * r * wv[e];
    rotate<VEC, false>(x[i], a, p, ln.partner);
    if (ln.on && head < heads)
      store<YB, VEC>(row_of(p.yq, p.yk, p.HQ, b, t, head, YB ? 2 : 4) + ln.d0 * (YB ? 2 : 4), x[i]);
  }
}

// The block's column sums of dw, one row of p.part a block: [2][D].
template <int VEC>
__device__ __forceinline__ void block_dw(const HeadNormParams& p, const Lanes& ln, const float (&dq)[VEC], const float (&dk)[VEC]) {
  __shared__ float sums[2 * 256 * VEC];  // [which][group][L * VEC]
  const int grp = threadIdx.x >> p.L_shift, groups = 256 >> p.L_shift, W = p.L * VEC;
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    sums[grp * W + ln.d0 + e] = dq[e];
    sums[256 * VEC + grp * W + ln.d0 + e] = dk[e];
  }
  __syncthreads();
  for (int c = threadIdx.x; c < 2 * p.D; c += 256) {
    const int which = c >= p.D, d = which ? c - p.D : c;
    float s = 0.f;
    for (int g = 0; g < groups; ++g) s += sums[which * 256 * VEC + g * W + d];
    p.part[(int64_t)blockIdx.x * 2 * p.D + c] = s;
  }
}

// XB: x is bf16; YB: dy and dx are bf16. Persistent blocks.
template <bool XB, bool YB, int VEC, int HPG>
__global__ __launch_bounds__(256) void bwd_kernel(const HeadNormParams p) {
  constexpr int XE = XB ? 2 : 4, YE = YB ? 2 : 4;
  Lanes ln;
  ln.init<VEC>(p);
  const int heads = p.HQ + p.HK, chunks = (heads + HPG - 1) / HPG;
  const int64_t units = (int64_t)p.B * p.T * chunks, step = (int64_t)gridDim.x * (256 >> p.L_shift);
  float wq[VEC], wk[VEC], sq[VEC], sk[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    wq[e] = wk[e] = 1.f;
    sq[e] = sk[e] = 0.f;
  }
  if (p.wq && ln.on) load<false, VEC>((const char*)(p.wq + ln.d0), wq);
  if (p.wk && ln.on) load<false, VEC>((const char*)(p.wk + ln.d0), wk);
  for (int64_t unit = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> p.L_shift; unit < units; unit += step) {
    const int64_t tok = unit / chunks;
    const int h0 = (int)(unit - tok * chunks) * HPG;
    const int64_t b = tok / p.T, t = tok - b * p.T;
    float x[HPG][VEC], g[HPG][VEC];
#pragma unroll
    for (int i = 0; i < HPG; ++i) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) x[i][e] = g[i][e] = 0.f;
      if (ln.on && h0 + i < heads) {
        load<XB, VEC>(row_of(p.q, p.k, p.HQ, b, t, h0 + i, XE) + ln.d0 * XE, x[i]);
        load<YB, VEC>(row_of(p.dyq, p.dyk, p.HQ, b, t, h0 + i, YE) + ln.d0 * YE, g[i]);
      }
    }
    Angles<VEC> a;
    a.load(p, b, t, ln.d0);
#pragma unroll
    for (int i = 0; i < HPG; ++i) {
      const int head = h0 + i;
      const bool isq = head < p.HQ;
      rotate<VEC, true>(g[i], a, p, ln.partner);
      float ss = 0.f, xe = 0.f;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        ss = fmaf(x[i][e], x[i][e], ss);
        xe = fmaf(x[i][e], g[i][e] * (isq ? wq[e] : wk[e]), xe);
      }
      ss = group_sum(ss, p.L);
      xe = group_sum(xe, p.L);
      const float r = rsqrtf(ss * p.inv_D + p.eps);
      const float mean = xe * r * p.inv_D;  // of n e
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float n = x[i][e] * r, gn = g[i][e] * n;
        if (isq) sq[e] += gn;
        else sk[e] += gn;
        x[i][e] = r * (g[i][e] * (isq ? wq[e] : wk[e]) - n * mean);
      }
      if (p.with_dx && ln.on && head < heads) {
        char* dst = row_of(p.yq, p.yk, p.HQ, b, t, head, YE) + ln.d0 * YE;
        if (p.accumulate) {
          float old[VEC];
          load<YB, VEC>(dst, old);
#pragma unroll
          for (int e = 0; e < VEC; ++e) x[i][e] += old[e];
        }
        store<YB, VEC>(dst, x[i]);
      }
    }
  }
  if (p.part) block_dw<VEC>(p, ln, sq, sk);
}

// By element, a wave a row. u(d) and its partner's are read again where the
// rotation needs them.
template <bool XB, bool YB>
struct Row {
  const char *x, *dy;
  const float *w, *cr, *sr;
  __device__ __forceinline__ float weight(int d) const { return w ? w[d] : 1.f; }
  // index, partner and angle of value d < R
  __device__ __forceinline__ void pair(const HeadNormParams& p, int d, int& other, float& c, float& s) const {
    const int half = p.R >> 1;
    const bool first = p.interleaved ? !(d & 1) : d < half;
    const int i = p.interleaved ? d >> 1 : first ? d : d - half;
    other = p.interleaved ? d ^ 1 : first ? d + half : d - half;
    c = cr[i];
    s = first ? -sr[i] : sr[i];
  }
  __device__ __forceinline__ float g(const HeadNormParams& p, int d) const {
    float v = load1<YB>(dy, d);
    if (d < p.R) {
      int o;
      float c, s;
      pair(p, d, o, c, s);
      v = v * c - load1<YB>(dy, o) * s;
    }
    return v;
  }
  __device__ __forceinline__ float y(const HeadNormParams& p, int d, float r) const {
    float v = load1<XB>(x, d) * r * weight(d);
    if (d < p.R) {
      int o;
      float c, s;
      pair(p, d, o, c, s);
      v = v * c + load1<XB>(x, o) * r * weight(o) * s;
    }
    return v;
  }
};
template <bool XB, bool YB>
__device__ __forceinline__ Row<XB, YB> elem_row(const HeadNormParams& p, int64_t b, int64_t t, int head, bool bwd) {
  Row<XB, YB> row;
  row.x = row_of(p.q, p.k, p.HQ, b, t, head, XB ? 2 : 4);
  row.dy = bwd ? row_of(p.dyq, p.dyk, p.HQ, b, t, head, YB ? 2 : 4) : nullptr;
  row.w = head < p.HQ ? p.wq : p.wk;
  row.cr = p.cos + b * p.cos_sb + t * p.cos_st;
  row.sr = p.sin + b * p.sin_sb + t * p.sin_st;
  return row;
}

template <bool XB, bool YB>
__global__ __launch_bounds__(256) void fwd_elem_kernel(const HeadNormParams p) {
  const int lane = threadIdx.x & 63, heads = p.HQ + p.HK;
  const int64_t unit = block_index() * 4 + (threadIdx.x >> 6);
  if (unit >= (int64_t)p.B * p.T * heads) return;
  const int64_t tok = unit / heads, b = tok / p.T, t = tok - b * p.T;
  const int head = (int)(unit - tok * heads);
  const Row<XB, YB> row = elem_row<XB, YB>(p, b, t, head, false);
  float ss = 0.f;
  for (int d = lane; d < p.D; d += 64) {
    const float v = load1<XB>(row.x, d);
    ss = fmaf(v, v, ss);
  }
  const float r = rsqrtf(group_sum(ss, 64) * p.inv_D + p.eps);
  char* dst = row_of(p.yq, p.yk, p.HQ, b, t, head, YB ? 2 : 4);
  for (int d = lane; d < p.D; d += 64) store1<YB>(dst, d, row.y(p, d, r));
}

template <bool XB, bool YB>
__global__ __launch_bounds__(256) void bwd_elem_kernel(const HeadNormParams p) {
  __shared__ float sums[4][2][kHeadNormMaxD];  // a wave's dw; lane l of it owns the columns l, l + 64, ..
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, heads = p.HQ + p.HK;
  for (int which = 0; which < 2; ++which)
    for (int d = lane; d < p.D; d += 64) sums[wave][which][d] = 0.f;
  const int64_t units = (int64_t)p.B * p.T * heads;
  for (int64_t unit = (int64_t)blockIdx.x * 4 + wave; unit < units; unit += (int64_t)gridDim.x * 4) {
    const int64_t tok = unit / heads, b = tok / p.T, t = tok - b * p.T;
    const int head = (int)(unit - tok * heads);
    const Row<XB, YB> row = elem_row<XB, YB>(p, b, t, head, true);
    float ss = 0.f, xe = 0.f;
    for (int d = lane; d < p.D; d += 64) {
      const float v = load1<XB>(row.x, d);
      ss = fmaf(v, v, ss);
      xe = fmaf(v, row.g(p, d) * row.weight(d), xe);
    }
    const float r = rsqrtf(group_sum(ss, 64) * p.inv_D + p.eps);
    const float mean = group_sum(xe, 64) * r * p.inv_D;
    char* dst = p.with_dx ? row_of(p.yq, p.yk, p.HQ, b, t, head, YB ? 2 : 4) : nullptr;
    for (int d = lane; d < p.D; d += 64) {
      const float n = load1<XB>(row.x, d) * r, g = row.g(p, d);
      sums[wave][head >= p.HQ][d] += g * n;
      if (dst) {
        const float dx = r * (g * row.weight(d) - n * mean);
        store1<YB>(dst, d, p.accumulate ? load1<YB>(dst, d) + dx : dx);
      }
    }
  }
  if (!p.part) return;
  __syncthreads();
  for (int c = threadIdx.x; c < 2 * p.D; c += 256) {
    const int which = c >= p.D, d = which ? c - p.D : c;
    p.part[(int64_t)blockIdx.x * 2 * p.D + c] = (sums[0][which][d] + sums[1][which][d]) + (sums[2][which][d] + sums[3][which][d]);
  }
}

// dwq, dwk (+)= the blocks' parts, in order within each of 64 interleaved
// shares, then over the shares. A block covers 16 of the 2 D columns; a thread
// keeps eight loads in flight (4 x 16 shares of 64 parts one by one: 20 us).
__global__ __launch_bounds__(1024) void finish_kernel(const float* part, int parts, int D, float* dwq, float* dwk, int add) {
  __shared__ float sums[64][17];
  const int c = blockIdx.x * 16 + (threadIdx.x & 15), share = threadIdx.x >> 4;
  float s = 0.f;
  if (c < 2 * D) {
#pragma unroll 8
    for (int i = share; i < parts; i += 64) s += part[(int64_t)i * 2 * D + c];
  }
  sums[share][threadIdx.x & 15] = s;
  __syncthreads();
  if (share || c >= 2 * D) return;
  s = 0.f;
#pragma unroll 16
  for (int i = 0; i < 64; ++i) s += sums[i][threadIdx.x];
  float* out = c < D ? dwq : dwk;
  if (!out) return;
  out += c < D ? c : c - D;
  *out = add ? *out + s : s;
}

}  // namespace headnorm

namespace {

template <typename F>
hipError_t by_types(bool x, bool y, F f) {
  if (x) return y ? f(std::true_type{}, std::true_type{}) : f(std::true_type{}, std::false_type{});
  return y ? f(std::false_type{}, std::true_type{}) : f(std::false_type{}, std::false_type{});
}

}  // namespace

hipError_t head_norm_fwd(const HeadNormParams& p, bool x_bf16, bool y_bf16, int vec, int hpg, hipStream_t stream) {
  return by_types(x_bf16, y_bf16, [&](auto xb, auto yb) {
    constexpr bool XB = decltype(xb)::value, YB = decltype(yb)::value;
    const int64_t tokens = (int64_t)p.B * p.T, heads = p.HQ + p.HK;
    const int64_t units = vec ? tokens * ((heads + hpg - 1) / hpg) : tokens * heads;
    const int64_t per = vec ? 256 >> p.L_shift : 4;
    const int64_t blocks = (units + per - 1) / per, x = blocks < headnorm::kMaxX ? blocks : headnorm::kMaxX;
    const dim3 grid((unsigned)x, (unsigned)((blocks + x - 1) / x));
    if (vec == 8 && hpg == 4) headnorm::fwd_kernel<XB, YB, 8, 4><<<grid, 256, 0, stream>>>(p);
    else if (vec == 8) headnorm::fwd_kernel<XB, YB, 8, 1><<<grid, 256, 0, stream>>>(p);
    else if (vec == 4 && hpg == 4) headnorm::fwd_kernel<XB, YB, 4, 4><<<grid, 256, 0, stream>>>(p);
    else if (vec == 4) headnorm::fwd_kernel<XB, YB, 4, 1><<<grid, 256, 0, stream>>>(p);
    else headnorm::fwd_elem_kernel<XB, YB><<<grid, 256, 0, stream>>>(p);
    return hipGetLastError();
  });
}

hipError_t head_norm_bwd(const HeadNormParams& p, bool x_bf16, bool y_bf16, int vec, int blocks, hipStream_t stream) {
  return by_types(x_bf16, y_bf16, [&](auto xb, auto yb) {
    constexpr bool XB = decltype(xb)::value, YB = decltype(yb)::value;
    const dim3 grid((unsigned)blocks);
    if (vec == 8) headnorm::bwd_kernel<XB, YB, 8, 2><<<grid, 256, 0, stream>>>(p);
    else if (vec == 4) headnorm::bwd_kernel<XB, YB, 4, 2><<<grid, 256, 0, stream>>>(p);
    else headnorm::bwd_elem_kernel<XB, YB><<<grid, 256, 0, stream>>>(p);
    return hipGetLastError();
  });
}

hipError_t head_norm_finish(const float* part, int parts, int D, float* dwq, float* dwk, bool add, hipStream_t stream) {
  headnorm::finish_kernel<<<dim3((unsigned)((2 * D + 15) / 16)), 1024, 0, stream>>>(part, parts, D, dwq, dwk, add);
  return hipGetLastError();
}

}  // namespace mt
