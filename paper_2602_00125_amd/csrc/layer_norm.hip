// Layer norm and its gradient, gfx950. For a row x of C values:
//
//   mu = mean x,  r = (mean (x - mu)^2 + eps)^(-1/2),  n = (x - mu) r,  y = n w + b
//   g = dy w,  dx = r (g - mean g - n mean(g n)),  dw = sum over rows of dy n,  db = of dy
//
// A row is read once and held in registers by L lanes (a power of two up to a
// wave, or whole waves), so that the variance is a mean of squared deviations and not a
// difference of large numbers, and the gradient needs no saved statistics: it
// takes them again from the row that it reads anyway.
//
// The mean is taken twice, of the values and of what is left of them. The first is
// off by some ulps of itself, which rows of small deviations would show (16384 times
// 12345.678 had an n of 0.5); the second by some ulps of the deviations. The second
// is a quotient: what the first leaves of like values has few digits, the sum and the
// quotient are exact, and a row of one value has deviations of 0. The pass costs up
// to 3% of the gradient's time and up to 8% of the forward's (43690 x 768 bf16).
//
// Bound: HBM (16384 x 1024 fp32 to bf16 18.9 us, 5.3 TB/s; gradient of 8192 x 8192
// fp32 169 us, 4.8 TB/s; bf16 gradients, half the bytes, by the vector instructions
// too: 32768 x 1024 49 us, 4.1).
//
// dw, db: a lane keeps the sums of its columns over the rows that it meets, a
// block adds its groups' in order, a second launch the blocks' in order, both in
// 64 bits (with 32 the sums of 3506 x 64 were off by 2.2e-7 of their norm). A lane
// meets kLayerNormLaneRows rows at most: more rows take several launches, whose parts
// the last one adds (of 4096 like rows a lane the sums were off by 4e-5).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "language.hpp"

namespace mt {
namespace layernorm {

using namespace vio;

// Sums over a row's lanes; rows of more than a wave (WIDE) meet in LDS, one
// buffer a sum, used again only after another sum's barrier.
template <bool WIDE, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], int L, int grp, float (*red)[16]) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = lanes_sum(v[i], WIDE ? 64 : L);
  if constexpr (WIDE) {
    const int wave = threadIdx.x >> 6, W = L >> 6, first = grp * W;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) red[i][wave] = v[i];
    __syncthreads();
#pragma unroll
    // 16 lanes read a wave's sum each (one after another: 2730 x 12288 bf16 37 us, this way 36)
    for (int i = 0; i < N; ++i) {
      const int w = threadIdx.x & 15;
      v[i] = lanes_sum(w < W ? red[i][first + w] : 0.f, 16);
    }
  }
}

// Group k of lane l: columns (l + k L) VEC and on. A row's last group, where it is
// not whole, is the row's last VEC values: those before `lo` belong to the group
// before it, take no part in sums and are written twice alike. (By element a
// wave would go through up to seven loads and stores for it: 32768 x 1023 bf16
// 54 us, this way 30.) hi: VEC, or C where a row has less. WHOLE: C is a multiple
// of VEC, and a group has all its columns or none (1024: 27 us as any, 26 whole).
template <int VEC, bool WHOLE>
struct Columns {
  int c, lo, hi;
  __device__ __forceinline__ Columns(int l, int k, const LayerNormParams& p) {
    const int first = (l + k * p.L) * VEC;
    c = WHOLE ? first : max(min(first, p.C - VEC), 0);
    lo = WHOLE ? (first < p.C ? 0 : VEC) : first - c;
    hi = WHOLE ? VEC : min(p.C, VEC);
  }
  __device__ __forceinline__ bool any() const { return lo < hi; }
  __device__ __forceinline__ bool has(int e) const { return WHOLE ? lo == 0 : e >= lo && e < hi; }
  template <bool BF>
  __device__ __forceinline__ void load(const void* p, int64_t row, bool on, float (&v)[VEC]) const {
    load_some<BF, VEC>(p, row + c, on && any() ? (WHOLE ? VEC : hi) : 0, 0.f, v);
  }
};

// The row's values less their mean, and less the mean of that. (contract(off): a
// mean is rounded before it is subtracted.)
template <bool WIDE, bool WHOLE, int NV, int VEC>
__device__ __forceinline__ void center(float (&x)[NV][VEC], const LayerNormParams& p, int l, int grp, float (*red)[16]) {
#pragma clang fp contract(off)
#pragma unroll
  for (int pass = 0; pass < 2; ++pass) {
    float s[1] = {0.f};
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const Columns<VEC, WHOLE> c(l, k, p);
#pragma unroll
      for (int e = 0; e < VEC; ++e) s[0] += c.has(e) ? x[k][e] : 0.f;
    }
    row_sums<WIDE, 1>(s, p.L, grp, red + pass);
    const float mean = pass ? s[0] / p.C_f : s[0] * p.inv_C;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int e = 0; e < VEC; ++e) x[k][e] -= mean;
  }
}

template <bool XB, bool YB, int VEC, int NV, bool WIDE, bool WHOLE>
__global__ __launch_bounds__(1024) void fwd_kernel(const LayerNormParams p) {
  __shared__ float red[3][16];
  const int grp = threadIdx.x / (unsigned)p.L, l = threadIdx.x - grp * p.L, rows = blockDim.x / (unsigned)p.L;
  float w[NV][VEC], b[NV][VEC];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const Columns<VEC, WHOLE> c(l, k, p);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      w[k][e] = 1.f;
      b[k][e] = 0.f;
    }
    if (p.w) c.template load<false>(p.w, 0, true, w[k]);
    if (p.b) c.template load<false>(p.b, 0, true, b[k]);
  }
  // all rows of a block go through the loop the same number of times
  for (int64_t m0 = (int64_t)blockIdx.x * rows; m0 < p.M; m0 += (int64_t)gridDim.x * rows) {
    const int64_t m = m0 + grp;
    const bool on = m < p.M;
    float x[NV][VEC], q[1] = {0.f};
#pragma unroll
    for (int k = 0; k < NV; ++k) Columns<VEC, WHOLE>(l, k, p).template load<XB>(p.x, m * p.ldx, on, x[k]);
    center<WIDE, WHOLE>(x, p, l, grp, red);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const Columns<VEC, WHOLE> c(l, k, p);
#pragma unroll
      for (int e = 0; e < VEC; ++e) q[0] = fmaf(c.has(e) ? x[k][e] : 0.f, x[k][e], q[0]);
    }
    row_sums<WIDE, 1>(q, p.L, grp, red + 2);
    const float r = 1.f / sqrtf(fmaf(q[0], p.inv_C, p.eps));
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const Columns<VEC, WHOLE> c(l, k, p);
#pragma unroll
      for (int e = 0; e < VEC; ++e) x[k][e] = fmaf(x[k][e] * r, w[k][e], b[k][e]);
      store_some<YB, VEC>(p.out, m * p.ldo + c.c, on && c.any() ? c.hi : 0, x[k]);
    }
  }
}

template <bool XB, bool YB, int VEC, int NV, bool WIDE, bool WHOLE>
__global__ __launch_bounds__(1024) void bwd_kernel(const LayerNormParams p) {
  __shared__ float red[5][16];
  __shared__ float cols[1024 * 16];  // [group][C], where a block has several groups
  const int grp = threadIdx.x / (unsigned)p.L, l = threadIdx.x - grp * p.L, rows = blockDim.x / (unsigned)p.L;
  float w[NV][VEC], dw[NV][VEC], db[NV][VEC];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      w[k][e] = 1.f;
      dw[k][e] = db[k][e] = 0.f;
    }
    if (p.w) Columns<VEC, WHOLE>(l, k, p).template load<false>(p.w, 0, true, w[k]);
  }
  for (int64_t m0 = (int64_t)blockIdx.x * rows; m0 < p.M; m0 += (int64_t)gridDim.x * rows) {
    const int64_t m = m0 + grp;
    const bool on = m < p.M;
    float x[NV][VEC], g[NV][VEC], t[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const Columns<VEC, WHOLE> c(l, k, p);
      c.template load<XB>(p.x, m * p.ldx, on, x[k]);
      c.template load<YB>(p.dy, m * p.ldd, on, g[k]);
    }
    center<WIDE, WHOLE>(x, p, l, grp, red);
    // squares of the deviations, sums of g and of g times the deviations
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const Columns<VEC, WHOLE> c(l, k, p);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float d = c.has(e) ? x[k][e] : 0.f;
        const float gw = g[k][e] * w[k][e];
        t[0] = fmaf(d, d, t[0]);
        t[1] += c.has(e) ? gw : 0.f;
        t[2] = fmaf(d, gw, t[2]);
      }
    }
    row_sums<WIDE, 3>(t, p.L, grp, red + 2);
    const float r = 1.f / sqrtf(fmaf(t[0], p.inv_C, p.eps));
    const float mg = t[1] / p.C_f, mgn = t[2] * (r * p.inv_C);  // the means of g and of g n
    if (!on) continue;  // no barrier below
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const Columns<VEC, WHOLE> c(l, k, p);
      float o[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float n = x[k][e] * r;
        dw[k][e] = fmaf(g[k][e], n, dw[k][e]);
        db[k][e] += g[k][e];
        o[e] = r * (fmaf(g[k][e], w[k][e], -mg) - n * mgn);
      }
      if (!p.out || !c.any()) continue;
      if (!p.accumulate) {
        store_some<YB, VEC>(p.out, m * p.ldo + c.c, c.hi, o);
        continue;
      }
      float old[VEC];
      load_some<YB, VEC>(p.out, m * p.ldo + c.c, c.hi, 0.f, old);
#pragma unroll
      for (int e = 0; e < VEC; ++e) o[e] += old[e];
      if (c.lo == 0) {
        store_some<YB, VEC>(p.out, m * p.ldo + c.c, c.hi, o);
      } else {  // once only: another lane adds to the others
#pragma unroll
        for (int e = 0; e < VEC; ++e)
          if (c.has(e)) store_one<YB>(p.out, m * p.ldo + c.c + e, o[e]);
      }
    }
  }
  if (!p.part) return;
  float* part = p.part + (int64_t)blockIdx.x * 2 * p.C;
#pragma unroll
  for (int which = 0; which < 2; ++which, part += p.C) {
    if (rows == 1) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const Columns<VEC, WHOLE> c(l, k, p);
#pragma unroll
        for (int e = 0; e < VEC; ++e)
          if (c.has(e)) part[c.c + e] = which ? db[k][e] : dw[k][e];
      }
      continue;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const Columns<VEC, WHOLE> c(l, k, p);
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (c.has(e)) cols[grp * p.C + c.c + e] = which ? db[k][e] : dw[k][e];
    }
    __syncthreads();
    for (int c = threadIdx.x; c < p.C; c += blockDim.x) {
      double s = 0.0;
      for (int i = 0; i < rows; ++i) s += cols[i * p.C + c];
      part[c] = (float)s;
    }
  }
}

// dw, db (+)= the blocks' parts, in order within each of 64 interleaved shares,
// then over the shares; a block covers 16 of the 2 C columns. from: added to that
// (or NULL); to: receives the sums in dw's and db's place.
__global__ __launch_bounds__(1024) void finish_kernel(const float* part, int parts, int C, const double* from, double* to, float* dw,
                                                      float* db, int add) {
  __shared__ double sums[64][17];
  const int c = blockIdx.x * 16 + (threadIdx.x & 15), share = threadIdx.x >> 4;
  double s = 0.0;
  if (c < 2 * C) {
#pragma unroll 8
    for (int i = share; i < parts; i += 64) s += part[(int64_t)i * 2 * C + c];
  }
  sums[share][threadIdx.x & 15] = s;
  __syncthreads();
  if (share || c >= 2 * C) return;
  s = from ? from[c] : 0.0;
#pragma unroll 16
  for (int i = 0; i < 64; ++i) s += sums[i][threadIdx.x];
  if (to) {
    to[c] = s;
    return;
  }
  float* out = c < C ? dw : db;
  if (!out) return;
  out += c < C ? c : c - C;
  *out = (float)(add ? *out + s : s);
}

template <typename F>
hipError_t by_types(bool x, bool y, F f) {
  if (x) return y ? f(std::true_type{}, std::true_type{}) : f(std::true_type{}, std::false_type{});
  return y ? f(std::false_type{}, std::true_type{}) : f(std::false_type{}, std::false_type{});
}

// f(groups of values a lane, lanes past a wave) for the forms that are built.
template <int VEC, typename F>
hipError_t by_form(int nv, bool wide, F f) {
  using One = std::integral_constant<int, 1>;
  using Two = std::integral_constant<int, 2>;
  using Most = std::integral_constant<int, 16 / VEC>;
  if (nv == 1) return wide ? f(One{}, std::true_type{}) : f(One{}, std::false_type{});
  if (nv == 2) return wide ? f(Two{}, std::true_type{}) : f(Two{}, std::false_type{});
  return wide ? f(Most{}, std::true_type{}) : f(Most{}, std::false_type{});
}

}  // namespace layernorm

hipError_t layer_norm_fwd(const LayerNormParams& p, bool x_bf16, bool y_bf16, int nv, int threads, int blocks,
                          hipStream_t stream) {
  return layernorm::by_types(x_bf16, y_bf16, [&](auto xb, auto yb) {
    constexpr bool XB = decltype(xb)::value, YB = decltype(yb)::value;
    constexpr int VEC = XB || YB ? 8 : 4;
    return layernorm::by_form<VEC>(nv, p.L > 64, [&](auto n, auto wide) {
      if (p.C % VEC == 0)
        layernorm::fwd_kernel<XB, YB, VEC, decltype(n)::value, decltype(wide)::value, true>
            <<<dim3((unsigned)blocks), threads, 0, stream>>>(p);
      else
        layernorm::fwd_kernel<XB, YB, VEC, decltype(n)::value, decltype(wide)::value, false>
            <<<dim3((unsigned)blocks), threads, 0, stream>>>(p);
      return hipGetLastError();
    });
  });
}

hipError_t layer_norm_bwd(const LayerNormParams& p, bool x_bf16, bool y_bf16, int nv, int threads, int blocks,
                          hipStream_t stream) {
  return layernorm::by_types(x_bf16, y_bf16, [&](auto xb, auto yb) {
    constexpr bool XB = decltype(xb)::value, YB = decltype(yb)::value;
    constexpr int VEC = XB || YB ? 8 : 4;
    return layernorm::by_form<VEC>(nv, p.L > 64, [&](auto n, auto wide) {
      if (p.C % VEC == 0)
        layernorm::bwd_kernel<XB, YB, VEC, decltype(n)::value, decltype(wide)::value, true>
            <<<dim3((unsigned)blocks), threads, 0, stream>>>(p);
      else
        layernorm::bwd_kernel<XB, YB, VEC, decltype(n)::value, decltype(wide)::value, false>
            <<<dim3((unsigned)blocks), threads, 0, stream>>>(p);
      return hipGetLastError();
    });
  });
}

hipError_t layer_norm_finish(const float* part, int parts, int C, const double* from, double* to, float* dw, float* db, bool add,
                             hipStream_t stream) {
  layernorm::finish_kernel<<<dim3((unsigned)((2 * C + 15) / 16)), 1024, 0, stream>>>(part, parts, C, from, to, dw, db, add);
  return hipGetLastError();
}

}  // namespace mt
