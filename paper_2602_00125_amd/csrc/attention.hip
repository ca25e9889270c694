// Attention and its gradient, gfx950, one pass over the data each.
//
//   S = scale q k^T over the visible keys, lse = log sum exp S, P = exp(S - lse)
//   o = P v
//   delta = sum_d do o, dP = do v^T, dS = P (dP - delta)
//   dq = scale dS k, dk = scale dS^T q, dv = P^T do
//
// The scores are never stored: the forward keeps a running maximum and sum, the
// backward computes P anew from lse. A wave owns 32 tokens (queries; keys in the
// dk / dv pass) whose vectors are the right operand of the MFMAs, and tiles of
// the other tokens stream through LDS (see attention_tile.hpp):
//   C[r][n]  = sum_d tile[r][d] own[n][d]     (S, dP)
//   A[d][n] += sum_r tile[r][d] C[r][n]       (o, dq; dk, dv)
// so that softmax statistics are one value a lane and P goes into the second
// product from the registers it is in.
//
// Bound: the matrix cores and the softmax's vector instructions, one after the
// other. A tile that every query sees whole takes, in bf16 at a width of 128,
//   forward: 32 MFMAs (32 cycles of a SIMD each), 136 vector instructions (4
//   cycles; the 32 exponentials among them 16): 1024 + 928 cycles;
//   dq: 48 and 167 (32 exponentials): 1536 + 1052; dk / dv: 32 and 95 (16): 1024 + 572.
// A wave's MFMAs are written down in order, each step's left operand read from
// LDS a few steps before it and a share of the softmax between them; left to
// itself the compiler reads each operand right before its MFMA once registers
// are short. Measured on causal 4 x 4096 tokens, 32 heads over 8 of 128, bf16,
// at a clock of 1.9 GHz: forward 529 to 567 us on different cards (1.04 PFLOP/s,
// matrix cores busy 54% of the cycles), dq 726 us (1.13, 62%), dk / dv 1062 us
// (1.04, 47%). So forward and dq take what their products and their vector
// instructions take in turn (a tile 1900 and 2470 cycles): the two waves of a
// SIMD hardly overlap them. dk / dv (2200 for 1596) is bound by neither. No LDS
// bank conflicts; a third buffer for the tiles changes nothing. 1 x 16384, 16
// heads over 4: forward 977 us (1.13).
//
// Registers: bf16 by vectors spills none. In fp32 dk / dv spills 6 vector
// registers at a width of 64 and 14 at 128, where it and dq also move 80 to 150
// registers a tile to and from accumulation registers, beside 192 and 144 MFMAs
// (2 x 1024, 16 heads over 4 of 128, causal: matrix cores busy 27 to 28%).
// The variants by element spill up to 97.
//
// fp32 values are split into three bf16 parts (PL planes: each what the ones
// before left, rounded to nearest even), tiles on their way into LDS, P and dS in
// registers; a product runs as six MFMAs and leaves out terms of together 2^-24
// of it, of either sign (parts cut off in place of rounded left out up to 2^-21,
// always of the product's sign; rounding costs 1 to 2% of the forward, and of
// gradients nothing at widths of 64 and 128, 3% at 96, 5% by element): 2.7 times
// the rate of the fp32 matrix instructions (4 x 1024 tokens, 16 heads of 64,
// causal, gradient: 375 -> 207 us, now 185). The split is exact for values of 2^-110 and more (below, bits under
// 2^-133 are lost). Parts of an infinity, or of a value that bf16 rounds to one,
// are NaN, so results next to one are NaN.
//
// Sums, statistics and accumulators are fp32. With bf16 inputs P and dS are
// rounded to bf16 (nearest even) for the second product: the matrix cores'
// operand type, an error of 2^-8 of a term where the output is rounded to bf16
// as well. The row sum of P is taken before the rounding.
//
// Each result is summed in a fixed order, by one block or by several whose shares
// another launch joins in order: no atomics. dq and dk / dv take a pass each, and
// both compute S and dP (7 products in place of 5): adding dq across the blocks
// of one pass would take atomics, or partial sums of 4 bytes a d for every 128
// keys, which cost more than the products.
#include <hip/hip_runtime.h>

#include "attention.hpp"
#include "attention_tile.hpp"

namespace mt {
namespace attn {

// An operand of one MFMA step: 8 bf16 values a lane, or the parts of 8 fp32 ones.
template <int PL>
struct Frag {
  u32x4 p[PL];
};

template <int PL>
__device__ __forceinline__ f32x16 mma(const Frag<PL>& a, const Frag<PL>& b, f32x16 c) {
  auto one = [&](int i, int j) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a.p[i]), __builtin_bit_cast(bf16x8, b.p[j]), c,
                                                0, 0, 0);
  };
  if constexpr (PL == 3) {  // the small terms first
    one(2, 0);
    one(0, 2);
    one(1, 1);
    one(1, 0);
    one(0, 1);
  }
  one(0, 0);
  return c;
}

// Words w of the fragments from two neighbouring values: rounded to bf16, or
// their three parts (each rounded from what the ones before left).
template <int PL>
__device__ __forceinline__ void put(Frag<PL>& f, int w, float a, float b) {
#pragma unroll
  for (int i = 0; i < PL; ++i) {
    const uint32_t u = pack_bf16(a, b);
    f.p[i][w] = u;
    a -= __uint_as_float(u << 16);
    b -= __uint_as_float(u & 0xffff0000u);
  }
}

// 8 values of a row from column d on, zeros from column D on.
template <int PL, bool VEC>
__device__ __forceinline__ void row8(const char* row, int d, int D, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = 0.f;
  if constexpr (VEC && PL == 1) {
    if (d < D) {
      const u32x4 u = *(const u32x4*)(row + 2 * d);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[2 * e] = __uint_as_float(u[e] << 16);
        v[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
      }
    }
  } else if constexpr (VEC) {
#pragma unroll
    for (int q = 0; q < 2; ++q)
      if (d + 4 * q < D) {
        const f32x4 t = *(const f32x4*)(row + 4 * (d + 4 * q));
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * q + e] = t[e];
      }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (d + e < D) v[e] = ld_elem(row, d + e, PL == 1);
  }
}

// A wave's 32 own tokens in registers, one a lane of each half.
template <int PL, int DP>
struct Own32 {
  static constexpr int NF = DP / 16;
  static constexpr bool REGS = true;
  Frag<PL> f[NF];
  // row: the lane's token in global memory (not read unless ok)
  template <bool VEC>
  __device__ __forceinline__ void load(const char* row, bool ok, int D, int lane) {
#pragma unroll
    for (int s = 0; s < NF; ++s) {
      const int d = (2 * s + (lane >> 5)) * 8;
      if constexpr (PL == 1 && VEC) {
        f[s].p[0] = u32x4{0, 0, 0, 0};
        if (ok && d < D) f[s].p[0] = *(const u32x4*)(row + 2 * d);
      } else {
        float v[8];
        row8<PL, VEC>(row, d, ok ? D : 0, v);
#pragma unroll
        for (int e = 0; e < 4; ++e) put<PL>(f[s], e, v[2 * e], v[2 * e + 1]);
      }
    }
  }
  __device__ __forceinline__ const Frag<PL>& frag(int s) const { return f[s]; }
  __device__ __forceinline__ void fresh() {}
};
// or as rows of a tile in LDS, from row n0 of it (a multiple of 32), plane by plane.
template <int PL, int DP, int PLANE>
struct OwnRows {
  using T = Tile<true, DP>;
  static constexpr bool REGS = false;
  uint32_t at;  // the lane's row; chunk bits as in Left
  __device__ __forceinline__ OwnRows(const char* tile, int n0, int lane) {
    const int r = lane & 31;
    at = lds_byte_addr(tile) + (n0 + r) * T::RB + (((lane >> 5) ^ T::swz(r)) * 16);
  }
  __device__ __forceinline__ Frag<PL> frag(int s) const {
    Frag<PL> f;
#pragma unroll
    for (int i = 0; i < PL; ++i) f.p[i] = lds_read16((at ^ (32 * s)) + i * PLANE);
    return f;
  }
  // the addresses of its reads are not kept across tiles
  __device__ __forceinline__ void fresh() { __asm__ __volatile__("" : "+v"(at)); }
};

// sum over d of a's row times b's, this lane half's part
template <int PL, int DP, bool VEC>
__device__ __forceinline__ float row_dot(const char* a, const char* b, bool ok, int D, int lane) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < DP / 16; ++i) {
    const int d = (2 * i + (lane >> 5)) * 8;
    float x[8], y[8];
    row8<PL, VEC>(a, d, ok ? D : 0, x);
    row8<PL, VEC>(b, d, ok ? D : 0, y);
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(x[e], y[e], s);
  }
  return s;
}

// Stream tokens into a tile of ROWS rows by NW waves; rows from `left` on and
// columns from D on are zero. bf16: straight into LDS by fetch (see Loader).
// fp32: fetch reads into registers, part(e) for e in 0 .. PARTS - 1 splits a pair
// of values a thread and writes finished chunks, each plane ROWS rows.
template <int PL, int DP, int ROWS, int NW, bool VEC>
struct Stream {
  using T = Tile<true, DP>;
  static constexpr int CHUNKS = T::RB / 16, JB = ROWS * CHUNKS / (64 * NW), PARTS = 4 * JB;
  static_assert(ROWS * CHUNKS % (64 * NW) == 0, "whole chunks for every thread");
  f32x4 v[JB][2];
  Frag<PL> f;
  uint32_t off[JB];  // bytes from the tile's first token; columns past D: out of range
  int tid, D;
  int64_t st;
  __device__ __forceinline__ int row(int j) const { return (tid + 64 * NW * j) / CHUNKS; }
  __device__ __forceinline__ int chunk(int j) const { return (tid + 64 * NW * j) % CHUNKS; }
  __device__ __forceinline__ void init(int wave, int lane, int64_t st_, int D_) {
    tid = 64 * wave + lane;
    st = st_;
    D = D_;
#pragma unroll
    for (int j = 0; j < JB; ++j) off[j] = 8 * chunk(j) < D ? (row(j) * (uint32_t)st + 8 * chunk(j)) * 4u : kOOB;
  }
  __device__ __forceinline__ void fetch(const char* base, int left, char*) {
    if constexpr (VEC) {
      const __amdgpu_buffer_rsrc_t r =
          __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(uniform_ptr(base)), (short)0, 0x7fffffff, kRsrcWord3);
#pragma unroll
      for (int j = 0; j < JB; ++j) {
        const uint32_t o = row(j) < left ? off[j] : kOOB;
        v[j][0] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, o, 0, 0));
        // the chunk's second half may lie past D on its own
        v[j][1] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                                r, 8 * chunk(j) + 4 < D ? o + 16 : kOOB, 0, 0));
      }
    } else {
#pragma unroll
      for (int j = 0; j < JB; ++j) {
        float x[8];
        row8<PL, VEC>(base + row(j) * st * 4, 8 * chunk(j), row(j) < left ? D : 0, x);
        v[j][0] = f32x4{x[0], x[1], x[2], x[3]};
        v[j][1] = f32x4{x[4], x[5], x[6], x[7]};
      }
    }
  }
  __device__ __forceinline__ void part(int e, char* tile) {
    const int j = e >> 2, w = e & 3;
    put<PL>(f, w, v[j][w >> 1][2 * (w & 1)], v[j][w >> 1][2 * (w & 1) + 1]);
    if (w < 3) return;
#pragma unroll
    for (int i = 0; i < PL; ++i)
      *(u32x4*)(tile + i * ROWS * T::RB + row(j) * T::RB + ((chunk(j) ^ T::swz(row(j))) * 16)) = f.p[i];
  }
  // parts of share i of n
  __device__ __forceinline__ void share(int i, int n, char* tile) {
#pragma unroll
    for (int e = i * PARTS / n; e < (i + 1) * PARTS / n; ++e) part(e, tile);
  }
};
template <int DP, int ROWS, int NW, bool VEC>
struct Stream<1, DP, ROWS, NW, VEC> {
  Loader<true, DP, ROWS, NW, VEC> l;
  __device__ __forceinline__ void init(int wave, int lane, int64_t st, int D) { l.init(wave, lane, st, D); }
  __device__ __forceinline__ void fetch(const char* base, int left, char* tile) { l.load(base, left, tile); }
  __device__ __forceinline__ void share(int, int, char*) {}
};

// A step's left operand: every plane's.
template <int PL, int DP, int PLANE>
struct Planes {
  const Left<true, DP> left;
  __device__ __forceinline__ explicit Planes(int lane) : left(lane) {}
  __device__ __forceinline__ Frag<PL> rows(uint32_t at, int off, int s) const {
    Frag<PL> f;
#pragma unroll
    for (int i = 0; i < PL; ++i) f.p[i] = left.rows(at, off + i * PLANE, s);
    return f;
  }
  __device__ __forceinline__ Frag<PL> cols(uint32_t at, int off, int kk, int db) const {
    Frag<PL> f;
#pragma unroll
    for (int i = 0; i < PL; ++i) f.p[i] = left.cols(at, off + i * PLANE, kk, db);
    return f;
  }
};

// What holds for both kernels that stream keys past 128 queries a block. KS = 2:
// two waves for each 32 queries, which take halves of every tile and meet at the
// end, for grids that would leave SIMDs with one wave.
template <int PL, int DP, int KS>
struct QGeom {
  using T = Tile<true, DP>;
  static constexpr int BK = PL == 1 ? 64 : 32, N = BK / 32;  // keys of a tile a wave takes, and in parts of 32
  static constexpr int BT = BK * KS, NW = 4 * KS;            // keys a tile
  static constexpr int PLANE = BT * T::RB, BYTES = PL * PLANE;
  static constexpr int NF = DP / 16, ND = DP / 32;
  static constexpr int AHEAD = PL == 1 ? 4 : 2;  // steps that operands are read ahead
  static constexpr bool TWO = PL == 1 || DP <= 64;  // registers (and LDS) for two waves a SIMD
  static constexpr int OCC = TWO ? 2 : 1;
  static_assert(KS == 1 || TWO, "two waves a SIMD");
};
// Where wave (qg, 1) leaves a f32x16 for (qg, 0): 16-byte places a lane.
__device__ __forceinline__ void leave(f32x4* at, const f32x16& a) {
#pragma unroll
  for (int i = 0; i < 4; ++i) at[64 * i] = f32x4{a[4 * i], a[4 * i + 1], a[4 * i + 2], a[4 * i + 3]};
}
// a = a f + what was left g
__device__ __forceinline__ void take(const f32x4* at, f32x16& a, float f, float g) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x4 x = at[64 * i];
#pragma unroll
    for (int e = 0; e < 4; ++e) a[4 * i + e] = a[4 * i + e] * f + x[e] * g;
  }
}

// Which queries a block holds: 128 of a head, or (paired) two such sets one
// after the other. The heads of a key head run on the same XCDs, whose L2 their
// keys share: 8 / gcd(groups, 8) XCDs take a set of groups between them, block
// by block, those that see most keys first.
struct QBlocks {
  int b, hq, hk, qb[2], n;
  __device__ __forceinline__ bool init(const AttnParams& p) {
    const int nqb = (p.TQ + 127) >> 7, rows = p.paired ? (nqb + 1) >> 1 : nqb;
    const int groups = p.B * p.HK, S = groups & 1 ? 8 : groups & 2 ? 4 : groups & 4 ? 2 : 1, sets = 8 / S;
    const int x = blockIdx.x & 7, t = (blockIdx.x >> 3) * S + x % S, per = groups / sets;
    if (t >= per * p.G * rows) return false;
    const int g = t % p.G, r = t / p.G % rows, bh = x / S * per + t / p.G / rows;
    hk = bh % p.HK;
    b = bh / p.HK;
    hq = hk * p.G + g;
    qb[0] = nqb - 1 - r;
    qb[1] = r;
    n = p.paired && r < nqb - 1 - r ? 2 : 1;
    return true;
  }
};
inline dim3 qblock_grid(const AttnParams& p) {
  const int nqb = (p.TQ + 127) >> 7, rows = p.paired ? (nqb + 1) >> 1 : nqb;
  const int groups = p.B * p.HK, S = groups & 1 ? 8 : groups & 2 ? 4 : groups & 4 ? 2 : 1, sets = 8 / S;
  return dim3((unsigned)(8 * ((groups / sets * p.G * rows + S - 1) / S)));
}

// The lane's query of a set, and the keys the set sees.
struct QSet {
  int qi, lim, kend, kall;
  bool ok, sees;  // the query exists; and sees a key
  Span sp;
  __device__ __forceinline__ QSet(const AttnParams& p, int b, int qb, int qg, int lane, int BT) {
    sp = span_of(p, b);
    qi = qb * 128 + qg * 32 + (lane & 31);
    ok = qi < p.TQ;
    lim = ok ? visible(p, sp, qi) : 0;
    sees = lim > 0;
    kend = __builtin_amdgcn_readfirstlane(visible(p, sp, qb * 128 + 127 < p.TQ ? qb * 128 + 127 : p.TQ - 1));
    // tiles that every query sees whole
    kall = __builtin_amdgcn_readfirstlane(visible(p, sp, qb * 128)) / BT * BT;
    if (!ok) qi = 0;
  }
};

// ---------------------------------------------------------------- forward
// Two tiles are worked on at a time: the product for tile t + 1's scores runs
// over tile t's exponentials, and the product of tile t's P and values over
// tile t + 1's maximum. Keys are fetched two tiles ahead, values one; in fp32
// three and two, into registers, and split under the products a tile later.
template <int PL, int DP, bool VEC, int KS>
__device__ __forceinline__ void fwd_set(const AttnParams& p, char (&lds)[2][2][QGeom<PL, DP, KS>::BYTES],  // keys, values
                                        const QBlocks& at, int qb) {
  using Gm = QGeom<PL, DP, KS>;
  constexpr int ES = PL == 1 ? 2 : 4, BK = Gm::BK, BT = Gm::BT, N = Gm::N, NF = Gm::NF, ND = Gm::ND, RB = Gm::T::RB;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int qg = wave & 3, ks = wave >> 2;
  const QSet set(p, at.b, qb, qg, lane, BT);
  const int kend = set.kend, kall = set.kall;
  Own32<PL, DP> q;
  q.template load<VEC>(row_of(p.q, at.b, set.qi, at.hq, ES), set.ok, p.D, lane);
  Stream<PL, DP, BT, Gm::NW, VEC> lk, lv;
  lk.init(wave, lane, p.k.st, p.D);
  lv.init(wave, lane, p.v.st, p.D);
  const char* kbase = row_of(p.k, at.b, 0, at.hk, ES);
  const char* vbase = row_of(p.v, at.b, 0, at.hk, ES);
  auto fetch_k = [&](int k0, int buf) { lk.fetch(kbase + (int64_t)k0 * p.k.st * ES, set.sp.len - k0, lds[0][buf]); };
  auto fetch_v = [&](int k0, int buf) { lv.fetch(vbase + (int64_t)k0 * p.v.st * ES, set.sp.len - k0, lds[1][buf]); };
  const Planes<PL, DP, Gm::PLANE> left(lane);
  const float c = p.scale_log2;
  f32x16 acc[ND] = {};
  float m = -kInf, off = 0.f, l0 = 0.f, l1 = 0.f;  // maximum (log2 units; may lag), the same finite, sums

  // The maximum of a tile's scores, this lane's half: m follows it only once it
  // lags by 2^8, since any m that keeps the terms in range gives the result.
  auto follow = [&](float t) {
    t = max_halves(t) * c;
    if (__any(t > m + 8.f)) {
      const float nm = fmaxf(t, m), f = nm == -kInf ? 1.f : __builtin_amdgcn_exp2f(m - nm);
      m = nm;
      off = m == -kInf ? 0.f : m;
      l0 *= f;
      l1 *= f;
#pragma unroll
      for (int db = 0; db < ND; ++db) acc[db] *= f;
    }
  };
  // element x of part n: masked where the lane's query does not see the key
  auto hide = [&](f32x16 (&S)[N], int n, int x, int lm) {
    if (32 * n + 16 * (x >> 3) + (x & 7) >= lm) S[n][x] = -kInf;
  };
  // pair e (8 a part) of P from S, into the next product's operand
  auto probability = [&](const f32x16 (&S)[N], Frag<PL> (&P)[N][2], int e) {
    const int n = e >> 3, x = 2 * (e & 7);
    const float a = __builtin_amdgcn_exp2f(fmaf(S[n][x], c, -off)), b = __builtin_amdgcn_exp2f(fmaf(S[n][x + 1], c, -off));
    l0 += a;
    l1 += b;
    put<PL>(P[n][(e & 7) >> 2], e & 3, a, b);
  };
  // Tile k0 (its scores in S) is finished, the scores of the next one begun in
  // X, masked or not; or there is none.
  auto tile = [&](auto next, auto masked, const f32x16 (&S)[N], f32x16 (&X)[N], int k0) {
    const int buf = k0 / BT & 1;
    if constexpr (PL == 1) wait_all_barrier();
    else wait_lds_barrier();  // fp32 loads in flight end in registers
    if (PL == 1 && k0 + 2 * BT < kend) fetch_k(k0 + 2 * BT, buf);
    if (PL == 1 && k0 + BT < kend) fetch_v(k0 + BT, buf ^ 1);
    constexpr int NS = next ? N * NF : 0, NV = N * 2 * ND, PAIRS = 8 * N;
    const uint32_t K = lds_byte_addr(lds[0][buf ^ 1]) + ks * BK * RB, V = lds_byte_addr(lds[1][buf]) + ks * BK * RB;
    Frag<PL> P[N][2], ring[Gm::AHEAD];
    auto load = [&](auto i) {
      if constexpr (i < NS) {
        return left.rows(K, i / NF * 32 * RB, i % NF);
      } else {
        constexpr int j = i - NS;
        return left.cols(V, j / (2 * ND) * 32 * RB, j % (2 * ND) / ND, j % ND);
      }
    };
    unroll<Gm::AHEAD>([&](auto i) { ring[i] = load(i); });
    if constexpr (!next) {
#pragma unroll
      for (int e = 0; e < PAIRS; ++e) probability(S, P, e);
    }
    float t = -kInf;
    const int lm = set.lim - k0 - BT - ks * BK - 8 * (lane >> 5);
    __builtin_amdgcn_sched_barrier(0);
    unroll<NS + NV>([&](auto i) {
      const Frag<PL> a = ring[i % Gm::AHEAD];
      if constexpr (i < NS) {
        constexpr int n = i / NF, s = i % NF;
        X[n] = mma<PL>(a, q.frag(s), s == 0 ? f32x16{} : X[n]);
      } else {
        constexpr int j = i - NS, n = j / (2 * ND), kk = j % (2 * ND) / ND, db = j % ND;
        acc[db] = mma<PL>(a, P[n][kk], acc[db]);
      }
      if constexpr (i + Gm::AHEAD < NS + NV) ring[i % Gm::AHEAD] = load(std::integral_constant<int, i + Gm::AHEAD>{});
      if constexpr (i < NS) {
#pragma unroll
        for (int e = i * PAIRS / NS; e < (i + 1) * PAIRS / NS; ++e) probability(S, P, e);
      } else if constexpr (next) {
        constexpr int j = i - NS;
#pragma unroll
        for (int e = j * 16 * N / NV; e < (j + 1) * 16 * N / NV; ++e) {
          if constexpr (masked) hide(X, e >> 4, e & 15, lm);
          t = fmaxf(t, X[e >> 4][e & 15]);
        }
      }
      // (past the last tile: what is there, into buffers that are not read)
      lk.share(i, NS + NV, lds[0][buf]);
      lv.share(i, NS + NV, lds[1][buf ^ 1]);
      __builtin_amdgcn_sched_barrier(0);
    });
    if constexpr (next) follow(t);
    if (PL == 3 && k0 + 3 * BT < kend) fetch_k(k0 + 3 * BT, 0);
    if (PL == 3 && k0 + 2 * BT < kend) fetch_v(k0 + 2 * BT, 0);
  };

  if (kend > 0) {
    using std::false_type;
    using std::true_type;
    fetch_k(0, 0);
    fetch_v(0, 0);
    lk.share(0, 1, lds[0][0]);
    if (BT < kend) fetch_k(BT, 1);
    wait_all_barrier();
    f32x16 S[N], X[N];
    {
      const uint32_t K = lds_byte_addr(lds[0][0]) + ks * BK * RB;
      float t = -kInf;
      const int lm = set.lim - ks * BK - 8 * (lane >> 5);
#pragma unroll
      for (int n = 0; n < N; ++n) {
        S[n] = f32x16{};
#pragma unroll
        for (int s = 0; s < NF; ++s) S[n] = mma<PL>(left.rows(K, n * 32 * RB, s), q.frag(s), S[n]);
        for (int x = 0; x < 16; ++x) hide(S, n, x, lm);
#pragma unroll
        for (int x = 0; x < 16; ++x) t = fmaxf(t, S[n][x]);
      }
      follow(t);
    }
    lv.share(0, 1, lds[1][0]);
    lk.share(0, 1, lds[0][1]);
    if (PL == 3 && 2 * BT < kend) fetch_k(2 * BT, 0);
    if (PL == 3 && BT < kend) fetch_v(BT, 0);
    int k0 = 0;
    // two at a time: the scores change places without a copy
    for (; k0 + 3 * BT <= kall; k0 += 2 * BT) {
      tile(true_type{}, false_type{}, S, X, k0);
      tile(true_type{}, false_type{}, X, S, k0 + BT);
    }
    for (; k0 + BT < kend; k0 += BT) {
      tile(true_type{}, true_type{}, S, X, k0);
#pragma unroll
      for (int n = 0; n < N; ++n) S[n] = X[n];
    }
    tile(false_type{}, false_type{}, S, X, k0);
  }
  float l = sum_halves(l0 + l1);
  if constexpr (KS == 2) {
    static_assert(4 * 64 * 4 * (16 * ND + 2) <= (int)sizeof(lds), "a wave's results of each pair fit the tiles' LDS");
    f32x4* mine = (f32x4*)&lds[0][0][0] + qg * (4 * ND * 64) + lane;
    float* stat = (float*)&lds[0][0][0] + 4 * 16 * ND * 64 + qg * 128 + lane;
    __syncthreads();
    if (ks) {
      stat[0] = m;
      stat[64] = l;
#pragma unroll
      for (int db = 0; db < ND; ++db) leave(mine + 256 * db, acc[db]);
    }
    __syncthreads();
    if (ks) return;
    const float m2 = stat[0], top = fmaxf(m, m2);
    const float f = m == -kInf ? 0.f : __builtin_amdgcn_exp2f(m - top), g = m2 == -kInf ? 0.f : __builtin_amdgcn_exp2f(m2 - top);
    l = l * f + stat[64] * g;
    m = top;
#pragma unroll
    for (int db = 0; db < ND; ++db) take(mine + 256 * db, acc[db], f, g);
  }
  store_rows<PL == 1, DP, VEC>(row_of(p.o, at.b, set.qi, at.hq, ES), set.ok, p.D, acc, 1.f / l, l == 0.f, false, lane);
  if (p.lse && set.ok && lane < 32)
    p.lse[((int64_t)at.b * p.HQ + at.hq) * p.TQ + set.qi] = l == 0.f ? -kInf : (m + __builtin_amdgcn_logf(l)) * kLn2;
}
template <int PL, int DP, bool VEC, int KS>
__global__ __launch_bounds__((256 * KS), (QGeom<PL, DP, KS>::OCC)) void fwd_kernel(const AttnParams p) {
  __shared__ __align__(1024) char lds[2][2][QGeom<PL, DP, KS>::BYTES];
  QBlocks at;
  if (!at.init(p)) return;
  fwd_set<PL, DP, VEC, KS>(p, lds, at, at.qb[0]);
  if constexpr (KS == 2) {
    if (at.n < 2) return;
    wait_all_barrier();  // the first set's tiles and results are read
    fwd_set<PL, DP, VEC, KS>(p, lds, at, at.qb[1]);
  }
}

// --------------------------------------------------------------- backward
// dq, and for the dk / dv pass the statistics as it adds them to its products.
// Of a tile's parts of 32 keys the products for S and dP come first, P under the
// one for dP, dS under the next part's; then the products with the keys.
template <int PL, int DP, bool VEC, int KS>
__device__ __forceinline__ void dq_set(const AttnParams& p, char (&lds)[2][2][QGeom<PL, DP, KS>::BYTES],  // buffer: keys, values
                                       const QBlocks& at, int qb) {
  using Gm = QGeom<PL, DP, KS>;
  constexpr int ES = PL == 1 ? 2 : 4, BK = Gm::BK, BT = Gm::BT, N = Gm::N, NF = Gm::NF, ND = Gm::ND, RB = Gm::T::RB;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int qg = wave & 3, ks = wave >> 2;
  const QSet set(p, at.b, qb, qg, lane, BT);
  const int kend = p.with_dq ? set.kend : 0, kall = set.kall;
  Stream<PL, DP, BT, Gm::NW, VEC> lk, lv;
  lk.init(wave, lane, p.k.st, p.D);
  lv.init(wave, lane, p.v.st, p.D);
  const char* kbase = row_of(p.k, at.b, 0, at.hk, ES);
  const char* vbase = row_of(p.v, at.b, 0, at.hk, ES);
  auto fetch = [&](int k0, int buf) {
    lk.fetch(kbase + (int64_t)k0 * p.k.st * ES, set.sp.len - k0, lds[buf][0]);
    lv.fetch(vbase + (int64_t)k0 * p.v.st * ES, set.sp.len - k0, lds[buf][1]);
  };
  if (kend > 0) fetch(0, 0);
  const char* gorow = row_of(p.dout, at.b, set.qi, at.hq, ES);
  const int64_t stat = ((int64_t)at.b * p.HQ + at.hq) * p.TQ + set.qi;
  // A query that sees nothing counts as zeros, whatever it holds
  const float delta = sum_halves(row_dot<PL, DP, VEC>(gorow, row_of(p.o, at.b, set.qi, at.hq, ES), set.sees, p.D, lane));
  // P = exp2(c S - lse2); where a query sees nothing lse = -inf, and all its
  // keys are masked.
  const float lse = set.ok ? p.lse[stat] : 0.f, lse2 = lse * kLog2e;
  if (set.ok && lane < 32 && ks == 0) {
    p.delta[stat] = -lse / p.scale;
    p.delta[(int64_t)p.B * p.HQ * p.TQ + stat] = -delta;
  }
  if (!p.with_dq) return;
  Own32<PL, DP> q, go;
  q.template load<VEC>(row_of(p.q, at.b, set.qi, at.hq, ES), set.sees, p.D, lane);
  go.template load<VEC>(gorow, set.sees, p.D, lane);
  if (kend > 0) {
    lk.share(0, 1, lds[0][0]);
    lv.share(0, 1, lds[0][1]);
    if (PL == 3 && BT < kend) fetch(BT, 0);
  }
  const Planes<PL, DP, Gm::PLANE> left(lane);
  const float c = p.scale_log2;
  f32x16 acc[ND] = {};
  auto tile = [&](auto masked, int k0) {
    const int buf = k0 / BT & 1;
    if constexpr (PL == 1) wait_all_barrier();
    else wait_lds_barrier();  // fp32 loads in flight end in registers
    if (PL == 1 && k0 + BT < kend) fetch(k0 + BT, buf ^ 1);
    constexpr int NS = N * 2 * NF, NA = N * 2 * ND;
    const uint32_t K = lds_byte_addr(lds[buf][0]) + ks * BK * RB;
    auto load = [&](auto i) {
      if constexpr (i < NS) {
        constexpr int n = i / (2 * NF), r = i % (2 * NF);
        return left.rows(K, n * 32 * RB + r / NF * Gm::BYTES, r % NF);
      } else {
        constexpr int j = i - NS;
        return left.cols(K, j / (2 * ND) * 32 * RB, j % (2 * ND) / ND, j % ND);
      }
    };
    Frag<PL> ring[Gm::AHEAD], dS[N][2];
    f32x16 S[N], dP[N];
    const int lm = set.lim - k0 - ks * BK - 8 * (lane >> 5);
    auto probability = [&](int n, int x) {
      S[n][x] = __builtin_amdgcn_exp2f(fmaf(S[n][x], c, -lse2));
      if (masked && 32 * n + 16 * (x >> 3) + (x & 7) >= lm) S[n][x] = 0.f;
    };
    auto gradient = [&](int n, int e) {  // pair e of 8
      const int x = 2 * e;
      put<PL>(dS[n][e >> 2], e & 3, S[n][x] * (dP[n][x] - delta), S[n][x + 1] * (dP[n][x + 1] - delta));
    };
    unroll<Gm::AHEAD>([&](auto i) { ring[i] = load(i); });
    __builtin_amdgcn_sched_barrier(0);
    unroll<NS + NA>([&](auto i) {
      if constexpr (N == 1 && i == NS) {
#pragma unroll
        for (int e = 0; e < 8; ++e) gradient(0, e);
      }
      const Frag<PL> a = ring[i % Gm::AHEAD];
      constexpr int n = i / (2 * NF), r = i % (2 * NF), s = r % NF, j = i - NS;
      if constexpr (i >= NS) {
        acc[j % ND] = mma<PL>(a, dS[j / (2 * ND)][j % (2 * ND) / ND], acc[j % ND]);
      } else if constexpr (r < NF) {
        S[n] = mma<PL>(a, q.frag(s), s == 0 ? f32x16{} : S[n]);
      } else {
        dP[n] = mma<PL>(a, go.frag(s), s == 0 ? f32x16{} : dP[n]);
      }
      if constexpr (i + Gm::AHEAD < NS + NA) ring[i % Gm::AHEAD] = load(std::integral_constant<int, i + Gm::AHEAD>{});
      if constexpr (i < NS && r >= NF) {
#pragma unroll
        for (int x = s * 16 / NF; x < (s + 1) * 16 / NF; ++x) probability(n, x);
      } else if constexpr (i < NS && n > 0) {
#pragma unroll
        for (int e = s * 8 / NF; e < (s + 1) * 8 / NF; ++e) gradient(n - 1, e);
      } else if constexpr (N > 1 && i >= NS && j < 2 * ND) {
#pragma unroll
        for (int e = j * 8 / (2 * ND); e < (j + 1) * 8 / (2 * ND); ++e) gradient(N - 1, e);
      }
      lk.share(i, NS + NA, lds[buf ^ 1][0]);
      lv.share(i, NS + NA, lds[buf ^ 1][1]);
      __builtin_amdgcn_sched_barrier(0);
    });
    if (PL == 3 && k0 + 2 * BT < kend) fetch(k0 + 2 * BT, 0);
  };
  int k0 = 0;
  for (; k0 < kall; k0 += BT) tile(std::false_type{}, k0);
  for (; k0 < kend; k0 += BT) tile(std::true_type{}, k0);
  if constexpr (KS == 2) {
    static_assert(4 * 64 * 4 * 16 * ND <= (int)sizeof(lds), "a wave's results of each pair fit the tiles' LDS");
    f32x4* mine = (f32x4*)&lds[0][0][0] + qg * (4 * ND * 64) + lane;
    __syncthreads();
    if (ks) {
#pragma unroll
      for (int db = 0; db < ND; ++db) leave(mine + 256 * db, acc[db]);
    }
    __syncthreads();
    if (ks) return;
#pragma unroll
    for (int db = 0; db < ND; ++db) take(mine + 256 * db, acc[db], 1.f, 1.f);
  }
  store_rows<PL == 1, DP, VEC>(row_of(p.dq, at.b, set.qi, at.hq, ES), set.ok, p.D, acc, p.scale, false, p.accumulate, lane);
}

template <int PL, int DP, bool VEC, int KS>
__global__ __launch_bounds__((256 * KS), (QGeom<PL, DP, KS>::OCC)) void dq_kernel(const AttnParams p) {
  __shared__ __align__(1024) char lds[2][2][QGeom<PL, DP, KS>::BYTES];
  QBlocks at;
  if (!at.init(p)) return;
  dq_set<PL, DP, VEC, KS>(p, lds, at, at.qb[0]);
  if constexpr (KS == 2) {
    if (at.n < 2) return;
    wait_all_barrier();
    dq_set<PL, DP, VEC, KS>(p, lds, at, at.qb[1]);
  }
}

// dk and dv: a block holds 32 KG = 128 keys of one head and walks the queries
// that see them, over all query heads of the group. QS waves share the same 32
// keys, each with its 32 queries of every tile; their accumulators are added in
// LDS at the end. So a block fills a CU with two waves a SIMD (measured on 4 x
// 4096 x 32 heads of 128, bf16: 1.8 ms with one, 1.05 with two; 1.19 with 256
// keys a block or blocks of four waves). Grids that leave CUs without a block
// hold 64 keys a block in bf16 (6 x 777 ragged, 4 heads of 96: 41 us against 59
// with 128). Two accumulators leave no room for both keys and values in 256
// registers, so the values stay in LDS, but for bf16 heads of up to 96, which
// have the room (2 x 4096, 16 heads over 4 of 96, causal, gradient: 490 us against
// 503); wide fp32 heads take all registers of a SIMD for one wave, their LDS
// being full. Few blocks (few key heads, short sequences) share out a key's query
// tiles, and dkv_join_kernel adds the shares' sums in order (1 x 2048, 8 heads over
// 1 of 128, gradient: bf16 251 -> 86 us, fp32 2327 -> 365).
template <int PL, int DP, int KG>
struct KvGeom {
  using T = Tile<true, DP>;
  static constexpr int OCC = PL == 1 || DP <= 64 ? 2 : 1, QS = 4 * OCC / KG;
  static constexpr int NW = KG * QS, BQ = 32 * QS, BKV = 32 * KG;
  static constexpr bool VLDS = PL == 1 ? DP > 96 : DP <= 64;
  static constexpr int PLANE = BQ * T::RB, BYTES = PL * PLANE, VPLANE = BKV * T::RB;
  static constexpr int AHEAD = PL == 1 ? 4 : 2, VAHEAD = PL == 1 ? 3 : 1;
};
template <int PL, int DP, bool VEC, int KG>
__global__ __launch_bounds__((64 * KvGeom<PL, DP, KG>::NW), (KvGeom<PL, DP, KG>::OCC)) void dkv_kernel(const AttnParams p) {
  using Gm = KvGeom<PL, DP, KG>;
  constexpr int ES = PL == 1 ? 2 : 4, BQ = Gm::BQ, NW = Gm::NW, QS = Gm::QS, BKV = Gm::BKV, RB = Gm::T::RB;
  constexpr int NF = DP / 16, ND = DP / 32, NA = 2 * ND, AHEAD = Gm::AHEAD, VA = Gm::VAHEAD;
  constexpr bool VLDS = Gm::VLDS;
  __shared__ __align__(1024) char lds[2][2][Gm::BYTES];  // buffer: queries, output gradients
  __shared__ __align__(1024) char vlds[VLDS ? PL * Gm::VPLANE : 16];
  __shared__ __align__(256) float stats[2][2][BQ < 64 ? 64 : BQ];  // -lse / scale, -delta of the tile's queries
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kg = wave % KG, qs = wave / KG;  // which 32 keys, which queries of a tile
  const int nkb = (p.TK + BKV - 1) / BKV;
  // As many heads of an XCD at a time as fill its 32 CUs (their queries share
  // the L2), the blocks that see most queries first
  const int heads = p.B * p.HK, per = heads >> 3;
  int kb, bh, share = 0;
  if (p.splits > 1) {
    const int r = blockIdx.x / p.splits;
    share = blockIdx.x - r * p.splits;
    kb = r / heads;
    bh = r - kb * heads;
  } else if (heads & 7) {
    if ((int)blockIdx.x >= heads * nkb) return;
    kb = blockIdx.x / heads;
    bh = blockIdx.x - kb * heads;
  } else {
    const int i = blockIdx.x >> 3, few = (32 + nkb - 1) / nkb, most = few < per ? few : per;
    const int h0 = i / (most * nkb) * most, now = per - h0 < most ? per - h0 : most, r = i - h0 * nkb;
    kb = r / now;
    bh = (blockIdx.x & 7) * per + h0 + (r - kb * now);
  }
  const int hk = bh % p.HK, b = bh / p.HK;
  const Span sp = span_of(p, b);
  const int k0 = kb * BKV + kg * 32, kj = k0 + (lane & 31);
  const bool in = kj < p.TK, ok = kj < sp.len;
  const int krow = in ? kj : 0;
  // query tiles from the first that sees a key of the block, counted from the
  // first that sees a key at all (the ones before it are not read: P = 0 would
  // not keep their infinities and NaN out of the sums); from q_all on every
  // query sees all of them, before wfirst none sees a key of the wave
  const bool any = kb * BKV < sp.len;
  auto first_for = [&](int key) {
    const int64_t i = p.causal ? (int64_t)key - sp.start : 0;
    return i < 0 ? 0 : i < p.TQ ? (int)i : p.TQ;
  };
  const int q0 = first_for(0), q_first = any ? q0 + (first_for(kb * BKV) - q0) / BQ * BQ : p.TQ;
  const int tiles = (p.TQ - q_first + BQ - 1) / BQ;
  const int q_all = first_for(kb * BKV + BKV - 1), wfirst = first_for(k0);
  const bool wave_on = k0 < sp.len;
  const int see = first_for(kj);  // queries from here on see the lane's key

  Stream<PL, DP, BQ, NW, VEC> lq, lo;
  lq.init(wave, lane, p.q.st, p.D);
  lo.init(wave, lane, p.dout.st, p.D);
  // the block's share of the tiles of all heads
  const int all = tiles * p.G, begin = (int)((int64_t)all * share / p.splits);
  const int end = (int)((int64_t)all * (share + 1) / p.splits);
  const bool some = begin < end;
  auto fetch = [&](int it, int buf) {  // past the last: zeros, without a read
    const int hq = hk * p.G + it / tiles, t0 = q_first + (tiles - 1 - it % tiles) * BQ, n = it < end ? p.TQ - t0 : 0;
    lq.fetch(row_of(p.q, b, t0, hq, ES), n, lds[buf][0]);
    lo.fetch(row_of(p.dout, b, t0, hq, ES), n, lds[buf][1]);
  };
  auto fetch_stats = [&](int it, int buf) {
    const int hq = hk * p.G + it / tiles, t0 = q_first + (tiles - 1 - it % tiles) * BQ;
    if (wave < 2 * ((BQ + 63) / 64)) {  // a 4-byte statistic a lane
      const int which = wave & 1, q = 64 * (wave >> 1) + lane;
      const float* s = p.delta + ((int64_t)which * p.B * p.HQ + (int64_t)b * p.HQ + hq) * p.TQ + t0;
      const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<char*>(uniform_ptr((const char*)s)), (short)0, 0x7fffffff, kRsrcWord3);
      dma4(r, q < BQ && q < p.TQ - t0 ? 4u * q : kOOB, lds_byte_addr(stats[buf][which]) + 256 * (wave >> 1));
    }
  };
  if (some) {
    fetch(begin, 0);
    fetch_stats(begin, 0);
  }
  Own32<PL, DP> k;
  k.template load<VEC>(row_of(p.k, b, krow, hk, ES), ok, p.D, lane);
  auto v = [&] {
    if constexpr (VLDS) {
      Stream<PL, DP, BKV, NW, VEC> l;
      l.init(wave, lane, p.v.st, p.D);
      if (some) {
        l.fetch(row_of(p.v, b, kb * BKV, hk, ES), sp.len - kb * BKV, vlds);
        l.share(0, 1, vlds);
      }
      return OwnRows<PL, DP, Gm::VPLANE>(vlds, 32 * kg, lane);
    } else {
      Own32<PL, DP> o;
      o.template load<VEC>(row_of(p.v, b, krow, hk, ES), ok, p.D, lane);
      return o;
    }
  }();
  if (some) {
    lq.share(0, 1, lds[0][0]);
    lo.share(0, 1, lds[0][1]);
    if (PL == 3) fetch(begin + 1, 1);
  }
  const Planes<PL, DP, Gm::PLANE> left(lane);
  f32x16 ak[ND] = {}, av[ND] = {};
  int it = begin, buf = 0;
  auto tile = [&](auto masked, int t0) {
    // in fp32 the statistics go to LDS before the last tile's loads, which may
    // be in flight still
    if constexpr (PL == 1 || !VEC) wait_all_barrier();
    else wait_barrier<2 * decltype(lq)::JB + 2 * decltype(lo)::JB>();
    const int now = buf;
    if (it + 1 < end) {
      if constexpr (PL == 1) fetch(it + 1, now ^ 1);
      fetch_stats(it + 1, now ^ 1);
    }
    buf ^= 1;
    const int r0 = 32 * qs;
    if (wave_on && !(masked && t0 + r0 + 32 <= wfirst)) {
      const float *lse = stats[now][0] + r0 + 8 * (lane >> 5), *delta = stats[now][1] + r0 + 8 * (lane >> 5);
      const int from = see - t0 - r0 - 8 * (lane >> 5);
      const uint32_t Q = lds_byte_addr(lds[now][0]) + r0 * RB;
      constexpr int STEPS = 2 * NF + 2 * NA;
      auto load = [&](auto i) {
        if constexpr (i < 2 * NF) {
          return left.rows(Q, i / NF * Gm::BYTES, i % NF);
        } else {
          constexpr int j = (i - 2 * NF) % NA;
          return left.cols(Q, i < 2 * NF + NA ? Gm::BYTES : 0, j / ND, j % ND);
        }
      };
      v.fresh();
      Frag<PL> ring[AHEAD], vring[VA], P[2], dS[2];
      f32x16 S, dP;
      unroll<AHEAD>([&](auto i) { ring[i] = load(i); });
      __builtin_amdgcn_sched_barrier(0);
      // P under the product for dP, dS under the one for dv
      unroll<STEPS>([&](auto i) {
        const Frag<PL> a = ring[i % AHEAD];
        if constexpr (i == 0) {  // lse and delta come in as the products' first terms
#pragma unroll
          for (int x = 0; x < 16; ++x) S[x] = lse[16 * (x >> 3) + (x & 7)];
        }
        if constexpr (i == NF - 2) {
#pragma unroll
          for (int x = 0; x < 16; ++x) dP[x] = delta[16 * (x >> 3) + (x & 7)];
        }
        if constexpr (i < NF) {
          S = mma<PL>(a, k.frag(i), S);
        } else if constexpr (i < 2 * NF) {
          if constexpr (VLDS) dP = mma<PL>(a, vring[(i - NF) % VA], dP);
          else dP = mma<PL>(a, v.frag(i - NF), dP);
        } else {
          constexpr int j = (i - 2 * NF) % NA, kk = j / ND, db = j % ND;
          if constexpr (i < 2 * NF + NA) av[db] = mma<PL>(a, P[kk], av[db]);
          else ak[db] = mma<PL>(a, dS[kk], ak[db]);
        }
        if constexpr (i + AHEAD < STEPS) ring[i % AHEAD] = load(std::integral_constant<int, i + AHEAD>{});
        if constexpr (VLDS) {
          constexpr int f = i + VA - NF;
          if constexpr (f >= 0 && f < NF) vring[f % VA] = v.frag(f);
        }
        // pairs of elements: NF steps share the 8 of P, NA those of dS
        if constexpr (i >= NF && i < 2 * NF) {
#pragma unroll
          for (int e = (i - NF) * 8 / NF; e < (i - NF + 1) * 8 / NF; ++e) {
#pragma unroll
            for (int x = 2 * e; x < 2 * e + 2; ++x) {
              S[x] = __builtin_amdgcn_exp2f(S[x] * p.scale_log2);
              if (masked && 16 * (x >> 3) + (x & 7) < from) S[x] = 0.f;
            }
            put<PL>(P[e >> 2], e & 3, S[2 * e], S[2 * e + 1]);
          }
        } else if constexpr (i >= 2 * NF && i < 2 * NF + NA) {
#pragma unroll
          for (int e = (i - 2 * NF) * 8 / NA; e < (i - 2 * NF + 1) * 8 / NA; ++e)
            put<PL>(dS[e >> 2], e & 3, dP[2 * e] * S[2 * e], dP[2 * e + 1] * S[2 * e + 1]);
        }
        // (past the last tile: what is there, into a buffer that is not read)
        lq.share(i, STEPS, lds[now ^ 1][0]);
        lo.share(i, STEPS, lds[now ^ 1][1]);
        __builtin_amdgcn_sched_barrier(0);
      });
    } else {
      lq.share(0, 1, lds[now ^ 1][0]);
      lo.share(0, 1, lds[now ^ 1][1]);
    }
    if (PL == 3) fetch(it + 2, now);
    ++it;
  };
  // from the last query on, so that the blocks of a head read the same tiles at
  // a time whatever their first query is
  for (int t0 = some ? q_first + (tiles - 1 - begin % tiles) * BQ : 0; it < end; t0 = q_first + (tiles - 1) * BQ) {
    for (; it < end && t0 >= q_first && t0 >= q_all; t0 -= BQ) tile(std::false_type{}, t0);
    for (; it < end && t0 >= q_first; t0 -= BQ) tile(std::true_type{}, t0);
  }
  // the waves of the same keys meet, one accumulator at a time
  if constexpr (QS > 1) {
    constexpr int FL = 16 * ND * 64;  // floats of a wave's accumulator
    static_assert((QS - 1) * KG * FL * 4 <= (int)sizeof(lds), "the accumulators fit the tiles' LDS");
    auto meet = [&](f32x16 (&a)[ND]) {
      auto at = [&](int w) { return (f32x4*)&lds[0][0][0] + ((w - 1) * KG + kg) * (FL / 4) + lane; };
      __syncthreads();
      if (qs) {
#pragma unroll
        for (int db = 0; db < ND; ++db) leave(at(qs) + 256 * db, a[db]);
      }
      __syncthreads();
      if (qs == 0) {
#pragma unroll
        for (int w = 1; w < QS; ++w)
#pragma unroll
          for (int db = 0; db < ND; ++db) take(at(w) + 256 * db, a[db], 1.f, 1.f);
      }
    };
    meet(ak);
    meet(av);
    if (qs) return;
  }
  if (p.splits > 1) {
    auto row = [&](int which) {
      return (char*)(p.part + (((int64_t)(2 * share + which) * heads + bh) * p.TK + krow) * p.D);
    };
    store_rows<false, DP, VEC>(row(0), in, p.D, ak, p.scale, !ok, false, lane);
    store_rows<false, DP, VEC>(row(1), in, p.D, av, 1.f, !ok, false, lane);
    return;
  }
  // keys past the batch element's length or the last query's take no part: zero
  const bool write = in && (ok || !p.accumulate);
  if (p.dk.p) store_rows<PL == 1, DP, VEC>(row_of(p.dk, b, krow, hk, ES), write, p.D, ak, p.scale, !ok, p.accumulate, lane);
  if (p.dv.p) store_rows<PL == 1, DP, VEC>(row_of(p.dv, b, krow, hk, ES), write, p.D, av, 1.f, !ok, p.accumulate, lane);
}

// dk and dv from the shares of the tiles, added in order: W values a thread.
template <bool BF, int W>
__global__ __launch_bounds__(256) void dkv_join_kernel(const AttnParams p) {
  const int chunks = p.D / W;
  const int64_t rows = (int64_t)p.B * p.HK * p.TK, unit = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (unit >= 2 * rows * chunks) return;
  const int64_t r = unit / chunks;
  const int d = (int)(unit - r * chunks) * W, which = r >= rows;
  const int64_t row = which ? r - rows : r;
  const int bh = (int)(row / p.TK), key = (int)(row - (int64_t)bh * p.TK), b = bh / p.HK;
  const HeadView& out = which ? p.dv : p.dk;
  if (!out.p || (p.accumulate && key >= span_of(p, b).len)) return;
  float v[W] = {};
#pragma unroll 4
  for (int s = 0; s < p.splits; ++s) {
    const float* src = p.part + ((int64_t)(2 * s + which) * rows + row) * p.D + d;
#pragma unroll
    for (int e = 0; e < W; ++e) v[e] += src[e];
  }
  char* dst = row_of(out, b, key, bh - b * p.HK, BF ? 2 : 4);
#pragma unroll
  for (int e = 0; e < W; ++e) {
    if (p.accumulate) v[e] += ld_elem(dst, d + e, BF);
    if constexpr (BF) ((__bf16*)dst)[d + e] = (__bf16)v[e];
    else ((float*)dst)[d + e] = v[e];
  }
}

}  // namespace attn

namespace {

// launch(bf16 or fp32 parts, width, vectors or elements)
template <typename F>
hipError_t attn_launch(const AttnParams& p, bool bf16, bool vec, F launch) {
  return attn_by_width(p.D, [&](auto dp) {
    using std::integral_constant;
    if (bf16 && vec) launch(integral_constant<int, 1>{}, dp, std::true_type{});
    else if (bf16) launch(integral_constant<int, 1>{}, dp, std::false_type{});
    else if (vec) launch(integral_constant<int, 3>{}, dp, std::true_type{});
    else launch(integral_constant<int, 3>{}, dp, std::false_type{});
    return hipGetLastError();
  });
}

// Blocks of 128 queries: one a CU has two waves for each 32 queries (8 x 509
// queries, 383 keys, 8 heads of 64, fp32 forward: 21.5 us against 25.6 with one),
// and so have two a CU of causal attention, as pairs of a long and a short one:
// side by side the long ones would meet on some CUs (4 x 1024, 16 heads of 64,
// causal, fp32 gradient: 186 us against 208). Pairs that are more than the CUs
// would take a second round of blocks, and without a causal edge there is
// nothing to even out (6 x 777 ragged in pairs: gradient 96 us against 67).
template <typename F>
hipError_t attn_queries(AttnParams p, bool bf16, bool vec, F launch) {
  const int64_t sets = (p.TQ + 127) / 128, items = (int64_t)p.B * p.HQ * sets;
  const int64_t pairs = (int64_t)p.B * p.HQ * ((sets + 1) / 2);
  return attn_launch(p, bf16, vec, [&](auto pl, auto dp, auto v) {
    if constexpr (attn::QGeom<decltype(pl)::value, decltype(dp)::value, 1>::TWO) {
      p.paired = p.causal && items > 256 && pairs <= 256;
      if (items <= 256 || p.paired) {
        launch(pl, dp, v, std::integral_constant<int, 2>{}, attn::qblock_grid(p), p);
        return;
      }
    }
    launch(pl, dp, v, std::integral_constant<int, 1>{}, attn::qblock_grid(p), p);
  });
}

}  // namespace

hipError_t attn_fwd(const AttnParams& params, bool bf16, bool vec, hipStream_t stream) {
  return attn_queries(params, bf16, vec, [&](auto pl, auto dp, auto v, auto ks, dim3 grid, const AttnParams& p) {
    constexpr int KS = decltype(ks)::value;
    attn::fwd_kernel<decltype(pl)::value, decltype(dp)::value, decltype(v)::value, KS><<<grid, 256 * KS, 0, stream>>>(p);
  });
}
hipError_t attn_bwd_dq(const AttnParams& params, bool bf16, bool vec, hipStream_t stream) {
  return attn_queries(params, bf16, vec, [&](auto pl, auto dp, auto v, auto ks, dim3 grid, const AttnParams& p) {
    constexpr int KS = decltype(ks)::value;
    attn::dq_kernel<decltype(pl)::value, decltype(dp)::value, decltype(v)::value, KS><<<grid, 256 * KS, 0, stream>>>(p);
  });
}
hipError_t attn_bwd_dkv(const AttnParams& p, bool bf16, bool vec, hipStream_t stream) {
  const int keys = attn_kv_block(p, bf16);
  const int64_t items = (int64_t)p.B * p.HK * ((p.TK + keys - 1) / keys);
  const dim3 grid = p.splits > 1 ? dim3((unsigned)(items * p.splits)) : attn_grid(items);
  const hipError_t e = attn_launch(p, bf16, vec, [&](auto pl, auto dp, auto v) {
    constexpr int PL = decltype(pl)::value, DP = decltype(dp)::value;
    constexpr bool V = decltype(v)::value;
    if constexpr (PL == 1) {
      if (keys == 64) {
        attn::dkv_kernel<PL, DP, V, 2><<<grid, 512, 0, stream>>>(p);
        return;
      }
    }
    attn::dkv_kernel<PL, DP, V, 4><<<grid, 64 * attn::KvGeom<PL, DP, 4>::NW, 0, stream>>>(p);
  });
  if (e != hipSuccess || p.splits == 1) return e;
  const int w = vec ? 4 : 1;
  const int64_t units = 2 * (int64_t)p.B * p.HK * p.TK * (p.D / w);
  const dim3 join((unsigned)((units + 255) / 256));
  if (bf16 && vec) attn::dkv_join_kernel<true, 4><<<join, 256, 0, stream>>>(p);
  else if (bf16) attn::dkv_join_kernel<true, 1><<<join, 256, 0, stream>>>(p);
  else if (vec) attn::dkv_join_kernel<false, 4><<<join, 256, 0, stream>>>(p);
  else attn::dkv_join_kernel<false, 1><<<join, 256, 0, stream>>>(p);
  return hipGetLastError();
}

}  // namespace mt
