// Attention over packed caches with 8 or 16 query rows of a (layer, KV head)
// slice to an item: decoded tokens (the g heads of one to a few positions).
// Codes 16-byte aligned, scale rows whole.
//
// Such a call's floor is reading the codes once: 12 values a ns from memory,
// some 40 a clock and SM, at which a value may cost three instructions a lane and
// no more; it costs 2.6.
// A warp works by itself on 32 tokens at a time, from a ring of its own in shared
// memory (cp.async).  Products are warp-level MMAs of fp16 with the tokens and
// channels as the 16 rows and the query rows as the 8 columns, S^T = K Q^T and
// O^T = V^T P^T: one for 256 values, where the other way round (query rows as the
// 16 rows) takes one for 128.
//
// Codes become fp16 operands in registers.  A word w holds eight channels' codes.
// (w & 0x000f000f) | 0x3c003c00 is the pair of fp16 numbers 1 + u / 2^10 of the
// channels 0 and 4, (w & 0x00f000f0) | 0x2c002c00 the pair (64 + u) / 2^10 of 1 and
// 5, w >> 8 gives those of 2, 6 and 3, 7 (Q is laid out the same way); one fma with
// (s, -c s), s the fp16 number of the scale byte, makes (u - 8) s / 2^10 of each:
// exact, since s has four significant bits, 1032 / 2^10 s eleven and the result
// eight, and nothing passes 65504; but a byte below 32 would want bits below 2^-24.
// A warp that meets one (a vote a tile) takes (64 + u) / 2^7 for all, which holds every
// scale and wants two more shifts a word.  For V a pair is one channel of two
// tokens, from the two tokens' words after two byte permutations.
//
// Queries enter as q 2^k, k of the row such that the largest is near 2^14: a bf16
// number whole, an fp32 number as two fp16 terms (off by 2^-22 of it at most), or by
// 2^-39 of the row's largest where that is more.  Weights are exp2(s - m) with m 11
// below the largest score so far, raised when a score is 4 above that: at most 2^15,
// in one fp16 term for bf16 (off by 2^-11 of it at most, the output's own rounding by
// 2^-8) and two for fp32 (2^-22), or by 2^-36 of the row's largest where that is more.
// The MMA takes an fp16 number below 2^-14, a value of 2^-10 here (2^-13 in tiles with
// small scales), as one of that size when it lines its products up, so sums of such values
// are as exact as sums of values of that size.  Measured, fp32, 3,000 tokens, in the
// 2-norm: 7e-7 down to scales of 2^-14, 2.2e-6 at 2^-17, 1.6e-5 at 2^-23.
//
// bf16, 32 query on 8 KV heads of 128 channels: 131,071 tokens 39 us (3.7 TB/s with start
// and merge, 8), 64 caches of up to 8,192 tokens 73 (3.9 TB/s).  Bound by latency: 665
// instructions to a warp's tile, K products, softmax and V products one after the
// other, in 11 warps an SM; 57 and 60 % of the issue slots, 52 and 51 % of the memory's
// rate.  With scale bytes by shuffles and a multiply before every weight 77.6, with four
// blocks an SM and 128 registers 75.5.  16 rows (248 registers, two blocks an SM) over
// 131,071 tokens 51; 64 channels, 8 caches to 16,000 21.
#include <string.h>

#include <type_traits>

#include "packed.cuh"
#include "sm103.cuh"

namespace ckv {
namespace pk {
namespace {

using at::Item;
using at::Seg;
using at::Span;
using at::Tiles;
using at::Traj;
using sm103::fast_exp2;
using sm103::smem_addr;

constexpr int NW = 4;
constexpr int WT = 32;  // tokens of a warp,
constexpr int TT = NW * WT;  // of a tile
constexpr float kLazy = 4.0f, kLift = 11.0f;
// Weights are exp2 of the fused s scale - m; the largest passes 2^15 by half a step
// of its score then, 1/4 up to here, and not fp16's range.
constexpr float kFar = 4194304.0f;

template <int D, int QT>
struct Smem {
  static constexpr int kRow = D / 2;            // bytes of codes
  static constexpr int kStage = 2 * WT * kRow;  // K and V
  static constexpr int NST = D == 128 ? 3 : 6;
  union {
    alignas(128) uint8_t ring[NW][NST][kStage];
    float o[NW][8 * QT][D + 4];
  };
  uint32_t sc[NW][2][2][WT];  // scale bytes of a tile's tokens, of K and V, of two tiles by turns
  float2 ml[NW][8 * QT];
  unsigned nan[NW][8 * QT];
};

// Where a row's bytes stand in its tile: rows that a fragment reads together lie
// in different banks.  Row t at t kRow, with these bits turned over.
template <int D>
__device__ __forceinline__ uint32_t k_turn(int t) {
  return D == 128 ? 0 : (t >> 3 & 1) << 6;
}
template <int D>
__device__ __forceinline__ uint32_t v_turn(int t) {
  return D == 128 ? (t >> 4 & 1) << 6 | (t >> 3 & 1) << 5 : (t >> 3 & 3) << 5;
}

template <int N>
__device__ __forceinline__ void lds(uint32_t a, uint32_t (&w)[N]) {
  if constexpr (N == 4)
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(a) : "memory");
  else if constexpr (N == 2)
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(a) : "memory");
  else
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[0]) : "r"(a) : "memory");
}

__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, "
      "%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// d = a b
__device__ __forceinline__ void mma_first(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, "
      "%10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

__device__ __forceinline__ uint32_t bits(__half2 x) { return *reinterpret_cast<const uint32_t *>(&x); }
__device__ __forceinline__ __half2 half2_of(uint32_t x) { return *reinterpret_cast<const __half2 *>(&x); }

// A pair of scales, as the fp16 numbers of their bytes, and what the offsets of
// the codes take away again.
template <bool SMALL>
struct Sc {
  __half2 s, low, high;
};
// from the two bytes at bits 7 .. 14 and 23 .. 30
template <bool SMALL>
__device__ __forceinline__ Sc<SMALL> scales_of(uint32_t x) {
  Sc<SMALL> r;
  r.s = half2_of(x);
  if (SMALL) r.low = r.high = __hmul2(r.s, __float2half2_rn(-0.5625f));
  else r.low = __hmul2(r.s, __float2half2_rn(-1.0078125f)), r.high = __hmul2(r.s, __float2half2_rn(-0.0703125f));
  return r;
}
// (x & mask) | number
__device__ __forceinline__ __half2 number_of(uint32_t x, uint32_t mask, uint32_t number) {
  uint32_t y;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(y) : "r"(x), "r"(mask), "r"(number));
  return half2_of(y);
}
// pair P of a word's four
template <int P, bool SMALL>
__device__ __forceinline__ uint32_t values_of(uint32_t w, const Sc<SMALL> &s) {
  if (SMALL) {
    const uint32_t x = P == 0 ? w << 4 : P == 1 ? w : P == 2 ? w >> 4 : w >> 8;
    return bits(__hfma2(number_of(x, 0x00f000f0u, 0x38003800u), s.s, s.low));
  }
  const uint32_t x = P < 2 ? w : w >> 8;
  if (P % 2 == 0) return bits(__hfma2(number_of(x, 0x000f000fu, 0x3c003c00u), s.s, s.low));
  return bits(__hfma2(number_of(x, 0x00f000f0u, 0x2c002c00u), s.s, s.high));
}

// x = hi + lo as fp16 terms.
__device__ __forceinline__ void split2(float x, float y, uint32_t &hi, uint32_t &lo) {
  const __half2 h = __floats2half2_rn(x, y);
  hi = bits(h);
  lo = bits(__floats2half2_rn(x - __low2float(h), y - __high2float(h)));
}

// Bit g: byte g of a token's scale bytes is NaN.
template <int D>
__device__ __forceinline__ unsigned nan_groups(uint32_t w) {
  unsigned m = 0;
#pragma unroll
  for (int g = 0; g < D / kGroup; ++g) m |= ((w >> (8 * g) & 0xffu) >= kNanScale ? 1u : 0u) << g;
  return m;
}

template <typename T, int D, int QT>
__global__ void __launch_bounds__(NW * 32, QT == 2 ? 2 : 3) attend_packed_rows(const __grid_constant__ Launch P) {
  using S = Smem<D, QT>;
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int RI = 8 * QT, KW = D / 32, VW = D / 64, KS = D / 16, MT = D / 16, NST = S::NST;
  extern __shared__ __align__(128) uint8_t raw[];
  S &sm = *reinterpret_cast<S *>(raw);
  const at::Launch &L = P.L;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, r = lane / 4, c = lane % 4;
  at::pdl_start_next();
  const Item it = at::decode_item(L, blockIdx.x);
  const Seg &sg = L.seg[it.s];
  const Scales &sc = P.sc[it.s];
  const Traj &tj = L.t[it.s];

  const int r0 = it.rt * RI, rows = min(RI, sg.R - r0);
  // what the rows see: row r in lane r
  Span mine = {0, 0x7fffffff, 0};
  int lo = 0x7fffffff, hi = 0, se = 0;
  if (lane < rows) {
    mine = at::row_span(sg.pos, sg.S, tj.qpos[(r0 + lane) / L.g], L.window, L.sinks);
    if (mine.lo < mine.hi) lo = mine.lo, hi = mine.hi;
    se = mine.se;
  }
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) {
    lo = min(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = max(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    se = max(se, __shfl_xor_sync(0xffffffffu, se, o));
  }
  lo = __shfl_sync(0xffffffffu, lo, 0), hi = __shfl_sync(0xffffffffu, hi, 0), se = __shfl_sync(0xffffffffu, se, 0);
  // tokens that all rows see
  int all_lo = lane < rows ? mine.lo : 0, all_hi = lane < rows ? mine.hi : 0x7fffffff;
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) {
    all_lo = max(all_lo, __shfl_xor_sync(0xffffffffu, all_lo, o));
    all_hi = min(all_hi, __shfl_xor_sync(0xffffffffu, all_hi, o));
  }
  all_lo = __shfl_sync(0xffffffffu, all_lo, 0), all_hi = __shfl_sync(0xffffffffu, all_hi, 0);
  const Tiles tl = at::make_tiles(lo, hi, se, TT);
  const int j0 = at::chunk_tile(tl, it.c, it.n), j1 = at::chunk_tile(tl, it.c + 1, it.n);

  const int64_t base = it.l * sg.sl + it.kvh * sg.sh, sbase = it.l * sc.gl + it.kvh * sc.gh;
  const uint8_t *kb = static_cast<const uint8_t *>(sg.k) + base, *ksb = sc.k + sbase;
  const int64_t dv = static_cast<const uint8_t *>(sg.v) - static_cast<const uint8_t *>(sg.k);
  const int64_t dvs = sc.v - sc.k, step = 32 / KW * sg.st, tile_step = TT * sg.st, scale_step = TT * sc.gt;
  const uint32_t ring = smem_addr(sm.ring[warp]);
  // where the lane's copies go in a stage (16 bytes of row lane / KW, further ones 512 bytes on)
  const uint32_t to_k = (lane / KW * S::kRow + 16 * (lane % KW)) ^ k_turn<D>(lane / KW);
  const uint32_t to_v = WT * S::kRow + ((lane / KW * S::kRow + 16 * (lane % KW)) ^ v_turn<D>(lane / KW));
  // The chunk is one or two pieces of consecutive tokens (sinks, then the window);
  // the warp's tokens of a piece's tiles begin at `at` and end with the piece.
  struct Cursor {
    int at, end;
    const uint8_t *k, *s;  // the lane's rows of codes and scales there
  };
  auto cursor = [&](int j, int last) {  // tiles j .. last - 1 are of one piece
    Cursor x;
    x.at = at::tile_start(tl, j, TT) + WT * warp;
    x.end = at::tile_end(tl, last - 1, TT);
    x.k = kb + (int64_t)(x.at + lane / KW) * sg.st + 16 * (lane % KW);
    x.s = ksb + (int64_t)(x.at + lane) * sc.gt;
    return x;
  };
  // copies of the next tile into its stage: tokens behind the piece's end as its last one's
  auto load = [&](Cursor &x, uint32_t dst) {
    if (x.at < x.end) {
      auto copy = [&](int i, const uint8_t *src) {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + to_k + 512 * i), "l"(src) : "memory");
        // stages are 128-byte aligned: the turn of the row's bits above the lane's own
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(((dst + to_v) ^ v_turn<D>(32 / KW * i)) + 512 * i), "l"(src + dv)
                     : "memory");
      };
      if (x.at + WT <= x.end) {
        const uint8_t *src = x.k;
#pragma unroll
        for (int i = 0; i < KW; ++i, src += step) copy(i, src);
      } else {
#pragma unroll
        for (int i = 0; i < KW; ++i) {
          const int t = (i * 32 + lane) / KW;
          copy(i, x.k + (int64_t)(min(x.at + t, x.end - 1) - x.at - lane / KW) * sg.st);
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    x.at += TT, x.k += tile_step;
  };
  // a token's scale bytes, of K and V, in its lane; none: zeros
  auto load_scales = [&](Cursor &x, uint32_t &k, uint32_t &v) {
    using W = typename std::conditional<D == 128, uint32_t, uint16_t>::type;
    k = v = 0;
    if (x.at + lane < x.end) {
      k = __ldg(reinterpret_cast<const W *>(x.s));
      v = __ldg(reinterpret_cast<const W *>(x.s + dvs));
    }
    x.at += TT, x.s += scale_step;
  };
  // the first piece's begin, before anything else is read
  int j = j0, last = j0 < tl.nA ? min(tl.nA, j1) : j1;
  Cursor in = j < last ? cursor(j, last) : Cursor{0, 0, kb, ksb}, sc_in = in;
#pragma unroll
  for (int s = 0; s < NST - 1; ++s) load(in, ring + s * S::kStage);
  uint32_t ksc, vsc;
  load_scales(sc_in, ksc, vsc);

  // Q^T as the B operand: lane (r, c) holds query row r's channels of its K words
  uint32_t q[QT][KS][2], ql[QT][F32 ? KS : 1][2];
  float back[QT][2];  // what makes scores of products, of the rows 2 c and 2 c + 1
  Span sp[QT][2];
#pragma unroll
  for (int n = 0; n < QT; ++n) {
    const int row = r0 + 8 * n + r;
    float f[KW][8], top = 0.0f;
    if (8 * n + r < rows) {
      const T *src = static_cast<const T *>(tj.q) + at::row_index(L, tj, it.l, it.kvh, row) * D + 8 * KW * c;
#pragma unroll
      for (int x = 0; x < KW; ++x) {
        if constexpr (F32) {
          const float4 a = reinterpret_cast<const float4 *>(src)[2 * x], b = reinterpret_cast<const float4 *>(src)[2 * x + 1];
          f[x][0] = a.x, f[x][1] = a.y, f[x][2] = a.z, f[x][3] = a.w, f[x][4] = b.x, f[x][5] = b.y, f[x][6] = b.z, f[x][7] = b.w;
        } else {
          const uint4 w = reinterpret_cast<const uint4 *>(src)[x];
          const uint32_t y[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int i = 0; i < 4; ++i)
            f[x][2 * i] = __uint_as_float(y[i] << 16), f[x][2 * i + 1] = __uint_as_float(y[i] & 0xffff0000u);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) top = isfinite(f[x][i]) ? fmaxf(top, fabsf(f[x][i])) : top;
      }
    } else {
#pragma unroll
      for (int x = 0; x < KW; ++x)
#pragma unroll
        for (int i = 0; i < 8; ++i) f[x][i] = 0.0f;
    }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    // 100: smaller rows' scores are as good as zero
    const int k = min(14 + 127 - (int)(__float_as_uint(top) >> 23), 100);
    const float up = __uint_as_float((uint32_t)(127 + k) << 23);
#pragma unroll
    for (int x = 0; x < KW; ++x) {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[x][i] *= up;
#pragma unroll
      for (int i = 0; i < 4; ++i) {  // pair i: k-step 2 x + i / 2, register i % 2
        uint32_t h, l;
        split2(f[x][i], f[x][i + 4], h, l);
        q[n][2 * x + i / 2][i % 2] = h;
        // an infinite number is its first term: with the rest, inf - inf, scores of -inf would be NaN
        if constexpr (F32)
          ql[n][2 * x + i / 2][i % 2] = (isinf(f[x][i]) ? 0u : l & 0xffffu) | (isinf(f[x][i + 4]) ? 0u : l & 0xffff0000u);
      }
    }
    // 16 / 2^k, and the softmax scale (which no score overflows by but that of a scale of 2^13 and more)
    const float b = fmaxf(fminf(__uint_as_float((uint32_t)(131 - k) << 23) * L.scale_log2, 3.402823466e38f), 1.175494351e-38f);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      back[n][e] = __shfl_sync(0xffffffffu, b, 4 * (2 * c + e));
      const int w = 8 * n + 2 * c + e;
      sp[n][e] = {__shfl_sync(0xffffffffu, mine.lo, w), __shfl_sync(0xffffffffu, mine.hi, w),
                  __shfl_sync(0xffffffffu, mine.se, w)};
    }
  }

  float o[QT][MT][4];
  float m[QT][2], over[QT][2], lsum[QT][2];  // the reference that weights are relative to, the score that raises it
  unsigned gone[QT][2];  // groups of channels that are NaN
#pragma unroll
  for (int n = 0; n < QT; ++n) {
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[n][t][i] = 0.0f;
#pragma unroll
    for (int e = 0; e < 2; ++e) m[n][e] = over[n][e] = -INFINITY, lsum[n][e] = 0.0f, gone[n][e] = 0;
  }
  // the lane's tokens of a tile: as rows of K's fragments tk + 4 i + 2 h (i: MMA,
  // h: rows 0 .. 7 or 8 .. 15); as k of V's 8 c + 4 i + 2 h and the next one.  Row r
  // of the scores is then k = r of the weights.
  const int tk = 8 * (r >> 1) + (r & 1);
  const uint32_t gk = D == 128 ? c : c >> 1, gv = D == 128 ? r >> 1 : r >> 2;  // the lane's groups
  const uint32_t ksel = gk << 12 | gk << 4 | 0x0404, vsel = (4 + gv) << 12 | gv << 4;
  // where the lane reads in a stage: K's rows tk + 2 h, and V's 8 c + t (i: 4 rows on, whose bits are turned alike)
  uint32_t from_k[2], from_v[4];
#pragma unroll
  for (int h = 0; h < 2; ++h) from_k[h] = ((tk + 2 * h) * S::kRow + 4 * KW * c) ^ k_turn<D>(tk);
#pragma unroll
  for (int t = 0; t < 4; ++t) from_v[t] = WT * S::kRow + (((8 * c + t) * S::kRow + 4 * VW * r) ^ v_turn<D>(8 * c));
  const uint32_t scales = smem_addr(sm.sc[warp]);
  bool far = false;  // a reference so large that products are rounded before they are compared with it
  // a tile in stage `stage`, its scale bytes at `sc_at`; bad: groups of the lane's token whose values are NaN
  auto tile = [&](auto is_small, int a, int e, uint32_t stage, uint32_t sc_at, unsigned bad) {
    constexpr bool SMALL = decltype(is_small)::value;
    const bool whole = all_lo <= a && a + WT <= min(all_hi, e);
    float s[QT][2][4];
    uint32_t w[2][2][KW];
    Sc<SMALL> f[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        lds<KW>(stage + from_k[h] + 4 * S::kRow * i, w[i][h]);
        uint32_t b[1];
        lds<1>(sc_at + 4 * tk + 16 * i + 8 * h, b);
        f[i][h] = scales_of<SMALL>(__byte_perm(b[0], 0, ksel) >> 1);
      }
    }
#pragma unroll
    for (int x = 0; x < KW; ++x)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t a0[4] = {values_of<0, SMALL>(w[i][0][x], f[i][0]), values_of<0, SMALL>(w[i][1][x], f[i][1]),
                                values_of<1, SMALL>(w[i][0][x], f[i][0]), values_of<1, SMALL>(w[i][1][x], f[i][1])};
        const uint32_t a1[4] = {values_of<2, SMALL>(w[i][0][x], f[i][0]), values_of<2, SMALL>(w[i][1][x], f[i][1]),
                                values_of<3, SMALL>(w[i][0][x], f[i][0]), values_of<3, SMALL>(w[i][1][x], f[i][1])};
#pragma unroll
        for (int n = 0; n < QT; ++n) {
          if constexpr (F32) {
            if (x == 0) mma_first(s[n][i], a0, ql[n][0][0], ql[n][0][1]);
            else mma(s[n][i], a0, ql[n][2 * x][0], ql[n][2 * x][1]);
            mma(s[n][i], a1, ql[n][2 * x + 1][0], ql[n][2 * x + 1][1]);
          }
          if (x == 0 && !F32) mma_first(s[n][i], a0, q[n][0][0], q[n][0][1]);
          else mma(s[n][i], a0, q[n][2 * x][0], q[n][2 * x][1]);
          mma(s[n][i], a1, q[n][2 * x + 1][0], q[n][2 * x + 1][1]);
        }
      }
    if constexpr (SMALL) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const unsigned b = __shfl_sync(0xffffffffu, bad, tk + 2 * i);
#pragma unroll
        for (int n = 0; n < QT; ++n)
#pragma unroll
          for (int x = 0; x < 2; ++x)
            if (at::sees(sp[n][x], a + tk + 2 * i)) gone[n][x] |= b;
      }
    }
    uint32_t p[QT][2][2], pl[QT][F32 ? 2 : 1][2];
#pragma unroll
    for (int n = 0; n < QT; ++n) {
      if (!whole) {
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float &y = s[n][i >> 1][2 * (i & 1) + x];
            const int tok = a + tk + 2 * i;
            y = tok < e && at::sees(sp[n][x], tok) ? y : -INFINITY;
          }
      }
      float top[2], by[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        by[x] = SMALL ? back[n][x] * 0.125f : back[n][x];
        top[x] = __fmul_rn(fmaxf(fmaxf(s[n][0][x], s[n][0][2 + x]), fmaxf(s[n][1][x], s[n][1][2 + x])), by[x]);
      }
      if (__any_sync(0xffffffffu, top[0] > over[n][0] || top[1] > over[n][1])) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) top[x] = fmaxf(top[x], __shfl_xor_sync(0xffffffffu, top[x], d));
          if (top[x] > over[n][x]) {
            const float r2 = top[x] - kLift, f2 = m[n][x] == -INFINITY ? 0.0f : exp2f(m[n][x] - r2);
            lsum[n][x] *= f2;
#pragma unroll
            for (int t = 0; t < MT; ++t) o[n][t][x] *= f2, o[n][t][2 + x] *= f2;
            m[n][x] = r2;
            over[n][x] = top[x] + kLazy;
          }
        }
        far = far || __any_sync(0xffffffffu, fabsf(top[0]) > kFar || fabsf(top[1]) > kFar);
      }
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const float ref = m[n][x] == -INFINITY ? 0.0f : m[n][x];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float &y = s[n][i >> 1][2 * (i & 1) + x];
          y = fast_exp2(far ? __fmul_rn(y, by[x]) - ref : fmaf(y, by[x], -ref));
          lsum[n][x] += y;
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t hi2, lo2;
          split2(s[n][i][2 * h], s[n][i][2 * h + 1], hi2, lo2);
          p[n][i][h] = transposed(hi2);
          if constexpr (F32) pl[n][i][h] = transposed(lo2);
        }
    }
    // values of this tile are 8 times the others': the sums meanwhile too (weights of 1 / 8 would end at 2^-33)
    auto times = [&](float f) {
#pragma unroll
      for (int n = 0; n < QT; ++n)
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
          for (int x = 0; x < 4; ++x) o[n][t][x] *= f;
    };
    if (SMALL) times(8.0f);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint32_t w[4][VW], b[4];
      Sc<SMALL> f[2];
#pragma unroll
      for (int t = 0; t < 4; ++t) lds<VW>(stage + from_v[t] + 4 * S::kRow * i, w[t]);
      lds<4>(sc_at + 4 * WT + 32 * c + 16 * i, b);
#pragma unroll
      for (int h = 0; h < 2; ++h)
        f[h] = scales_of<SMALL>(__byte_perm(b[2 * h], b[2 * h + 1], vsel) >> 1 & 0x7f807f80u);
      // of each word the halves of two tokens side by side: y[h][word][half]
      uint32_t y[2][VW][2];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int x = 0; x < VW; ++x) {
          y[h][x][0] = __byte_perm(w[2 * h][x], w[2 * h + 1][x], 0x5410);
          y[h][x][1] = __byte_perm(w[2 * h][x], w[2 * h + 1][x], 0x7632);
        }
      auto step = [&](int t, const uint32_t (&av)[4]) {
#pragma unroll
        for (int n = 0; n < QT; ++n) {
          if constexpr (F32) mma(o[n][t], av, pl[n][i][0], pl[n][i][1]);
          mma(o[n][t], av, p[n][i][0], p[n][i][1]);
        }
      };
      // m-tile t: rows r and r + 8 are channels t of the lane's first and second
      // word (128 channels), or t of the halves of its one word (64)
#pragma unroll
      for (int u = 0; u < MT / 4; ++u) {
        auto part = [&](int h, int second) { return VW == 2 ? y[h][second % VW][u] : y[h][0][second]; };
        const uint32_t a0[4] = {values_of<0, SMALL>(part(0, 0), f[0]), values_of<0, SMALL>(part(0, 1), f[0]),
                                values_of<0, SMALL>(part(1, 0), f[1]), values_of<0, SMALL>(part(1, 1), f[1])};
        step(4 * u, a0);
        const uint32_t a1[4] = {values_of<1, SMALL>(part(0, 0), f[0]), values_of<1, SMALL>(part(0, 1), f[0]),
                                values_of<1, SMALL>(part(1, 0), f[1]), values_of<1, SMALL>(part(1, 1), f[1])};
        step(4 * u + 1, a1);
        const uint32_t a2[4] = {values_of<2, SMALL>(part(0, 0), f[0]), values_of<2, SMALL>(part(0, 1), f[0]),
                                values_of<2, SMALL>(part(1, 0), f[1]), values_of<2, SMALL>(part(1, 1), f[1])};
        step(4 * u + 2, a2);
        const uint32_t a3[4] = {values_of<3, SMALL>(part(0, 0), f[0]), values_of<3, SMALL>(part(0, 1), f[0]),
                                values_of<3, SMALL>(part(1, 0), f[1]), values_of<3, SMALL>(part(1, 1), f[1])};
        step(4 * u + 3, a3);
      }
    }
    if (SMALL) times(0.125f);
  };
  // a byte from 1 to 31
  auto small = [](uint32_t x) { return (((x & 0x7f7f7f7fu) + 0x7f7f7f7fu) | x) & ~(x | x << 1 | x << 2) & 0x80808080u; };
  while (j < last) {
    int a = at::tile_start(tl, j, TT) + WT * warp, st = 0;
    const int e = at::tile_end(tl, last - 1, TT);
    for (; j < last; ++j, a += TT) {
      uint32_t kn, vn;
      load_scales(sc_in, kn, vn);
      unsigned bad = 0;
      bool any_small = false;
      const uint32_t sc_at = scales + (j & 1) * (8 * WT);
      if (a < e) {
        const uint32_t nan = vsc & ((vsc & 0x7f7f7f7fu) + 0x08080808u) & 0x80808080u;  // a byte from 0xf8 on
        any_small = __any_sync(0xffffffffu, small(ksc) | small(vsc) | nan);
        if (any_small) {  // NaN scales of values stand as zeros
          bad = nan_groups<D>(vsc);
#pragma unroll
          for (int g = 0; g < D / kGroup; ++g)
            if (bad >> g & 1) vsc &= ~(0xffu << (8 * g));
        }
        asm volatile("st.shared.b32 [%0], %1;" ::"r"(sc_at + 4 * lane), "r"(ksc) : "memory");
        asm volatile("st.shared.b32 [%0], %1;" ::"r"(sc_at + 4 * WT + 4 * lane), "r"(vsc) : "memory");
      }
      asm volatile("cp.async.wait_group %0;" ::"n"(NST - 2) : "memory");
      // every lane's copies of this stage and its scale bytes are there, and its reads of the last one are done
      __syncwarp();
      load(in, ring + (st == 0 ? NST - 1 : st - 1) * S::kStage);
      const uint32_t stage = ring + st * S::kStage;
      st = st + 1 == NST ? 0 : st + 1;
      if (a < e) {
        if (any_small) tile(std::true_type{}, a, e, stage, sc_at, bad);
        else tile(std::false_type{}, a, e, stage, sc_at, 0u);
      }
      ksc = kn, vsc = vn;
    }
    last = j1;
    if (j < last) {  // the window behind the sinks
      asm volatile("cp.async.wait_all;" ::: "memory");
      __syncwarp();
      in = sc_in = cursor(j, last);
#pragma unroll
      for (int s = 0; s < NST - 1; ++s) load(in, ring + s * S::kStage);
      load_scales(sc_in, ksc, vsc);
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
  for (int n = 0; n < QT; ++n)
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) {
        lsum[n][x] += __shfl_xor_sync(0xffffffffu, lsum[n][x], d);
        gone[n][x] |= __shfl_xor_sync(0xffffffffu, gone[n][x], d);
      }
  __syncthreads();  // the rings are done with
#pragma unroll
  for (int n = 0; n < QT; ++n)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int w = 8 * n + 2 * c + x;
      float *dst = &sm.o[warp][w][8 * VW * r];
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        dst[t] = o[n][t][x] * 16.0f;
        dst[MT + t] = o[n][t][2 + x] * 16.0f;
      }
      if (r == 0) {
        sm.ml[warp][w] = make_float2(m[n][x], lsum[n][x]);
        sm.nan[warp][w] = gone[n][x];
      }
    }
  __syncthreads();
  for (int w = warp; w < rows; w += NW) {
    float mr = -INFINITY, lr = 0.0f, x[D / 32], f[NW];
    unsigned nan = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) mr = fmaxf(mr, sm.ml[i][w].x), nan |= sm.nan[i][w];
    const float ref = mr == -INFINITY ? 0.0f : mr;
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      f[i] = exp2f(sm.ml[i][w].x - ref);
      lr = fmaf(sm.ml[i][w].y, f[i], lr);
    }
#pragma unroll
    for (int g = 0; g < D / 32; ++g) {  // channel lane + 32 g: group g
      x[g] = 0.0f;
#pragma unroll
      for (int i = 0; i < NW; ++i) x[g] = fmaf(sm.o[i][w][lane + 32 * g], f[i], x[g]);
      if (nan >> g & 1) x[g] = __int_as_float(0x7fffffff);
    }
    at::write_row_warp<T, D>(L, sg, it, r0 + w, x, mr, lr);
  }
  at::pdl_chain();
}

template <typename T, int D, int QT>
cudaError_t launch(const Launch &P, cudaStream_t s, bool early) {
  constexpr int smem = (int)sizeof(Smem<D, QT>);
  const cudaError_t e =
      cudaFuncSetAttribute(attend_packed_rows<T, D, QT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  return at::launch_after(attend_packed_rows<T, D, QT>, P.L.item_off[P.L.n_seg], NW * 32, smem, s, early, P);
}

}  // namespace

cudaError_t launch_rows(const Launch &P, cudaStream_t s, bool early) {
  if (P.L.dtype == COMMITKV_F32) return P.L.d == 128 ? launch<float, 128, 1>(P, s, early) : launch<float, 64, 1>(P, s, early);
  if (P.L.rows_per_item == 8)
    return P.L.d == 128 ? launch<__nv_bfloat16, 128, 1>(P, s, early) : launch<__nv_bfloat16, 64, 1>(P, s, early);
  return P.L.d == 128 ? launch<__nv_bfloat16, 128, 2>(P, s, early) : launch<__nv_bfloat16, 64, 2>(P, s, early);
}

}  // namespace pk
}  // namespace ckv
