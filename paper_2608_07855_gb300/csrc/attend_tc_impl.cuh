// Attention on the tensor cores (bf16): the kernel of full-width caches
// (attend_tc.cu) and of packed ones (packed_tc.cu).
//
// A CTA of 384 threads per SM takes items of up to 256 query rows, two tiles of
// 128, over 128-token tiles of K and V:
//   warp 0      TMA: K and V tiles through one ring of stages
//   warp 1      the MMAs: S_b = Q_b K^T and O_b += P_b V (tcgen05, fp32 in TMEM)
//   warp 3      the plan of the next item (what its rows see) and its Q rows,
//               which lie apart in memory (heads of one position side by side)
//   warps 4-11  two softmax groups of 128 threads, a thread per row
// With two row tiles a group has one each and both take every K and V tile:
// while one group works on its scores the tensor cores run the other's
// products.  With one row tile the groups take alternate token tiles of it and
// join their sums at the end of the item.
// Per tile a thread reads its 128 scores from TMEM once, keeps a running
// maximum that is only raised when it falls behind by 2^8 (O is rescaled
// then), and puts the weights back over the scores as bf16 for P V.  Weights
// are rounded to bf16 because the product with bf16 values takes one type: an
// error of 2^-9 of each weight on average, that of the output's own rounding.
// Sums of weights are fp32 and not rounded.
// Packed caches have eight more warps (12-19) in the place of warp 0: they read
// codes and write the values, which are bf16 numbers, into the same stages.
// TMEM: S/P of group b at column 128 b, O of group b at 256 + D b.
#pragma once

#include <cudaTypedefs.h>
#include <string.h>

#include "attend_tc.cuh"
#include "packed.cuh"

namespace ckv {
namespace at {
namespace {

constexpr int BT = 128;  // tokens of a tile
constexpr int kMaxQ = 32;  // trajectories whose Q tiles TMA copies: what the launch parameters have room for

struct TcParams {
  static constexpr bool kPacked = false;
  Launch L;
  CUtensorMap k[kMaxSeg], v[kMaxSeg];  // [M][H][S][d], box 64 x 128 x 1 x 1
  CUtensorMap q[kMaxQ];                // [M H][W][g][d], box 64 x g x 128 / g x 1: a row tile
  int32_t has_q;                       // the q maps are there: at most kMaxQ trajectories, g divides 128
};

struct PackedParams {
  static constexpr bool kPacked = true;
  Launch L;
  pk::Scales sc[kMaxTraj];
  CUtensorMap q[kMaxQ];
  int32_t has_q;
};

static_assert(sizeof(TcParams) <= 32764 && sizeof(PackedParams) <= 32764, "kernel parameters");

template <int D>
struct Smem {
  static constexpr int kTile = BT * D * 2;
  static constexpr int NST = D == 128 ? 4 : 8;
  alignas(1024) uint8_t q[2][kTile];
  alignas(1024) uint8_t kv[NST][kTile];
  Span span[2][2 * BM];
  Plan plan[2];
  float4 stage[8][RowsOut::kStage];
  int3 first[8];  // what the rows of a softmax warp see of the first item
  float2 pub[BM];  // one row tile: group 1's (m, l)
  alignas(16) uint4 next;  // answer to the request for another item
  uint64_t ask, next_full, plan_full[2], plan_empty[2], q_full, q_empty, kv_full[NST], kv_empty[NST], s_full[2], p_full[2], o_full[2],
      o_empty[2], pub_full, pub_empty, drain;
  uint32_t tmem;
  int flags[kFlags];
};

__device__ __forceinline__ void tma4(void *dst, const CUtensorMap *m, int x, int tok, int h, int l, uint64_t *bar,
                                     uint64_t pol) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0], [%1, {%2, %3, %4, %5}], [%6], %7;" ::"r"(smem_addr(dst)),
      "l"(reinterpret_cast<uint64_t>(m)), "r"(x), "r"(tok), "r"(h), "r"(l), "r"(smem_addr(bar)), "l"(pol)
      : "memory");
}

// A Q row tile's 64 channels from x: all heads of the positions from w.
__device__ __forceinline__ void tma_q(void *dst, const CUtensorMap *m, int x, int w, int slice, uint64_t *bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(
          smem_addr(dst)),
      "l"(reinterpret_cast<uint64_t>(m)), "r"(x), "r"(0), "r"(w), "r"(slice), "r"(smem_addr(bar))
      : "memory");
}

constexpr uint32_t kHalf = BT * 128;  // one 64-channel half of a tile

__device__ __forceinline__ uint64_t desc_kmajor(const uint8_t *tile, int ks) {
  return smem_desc(smem_addr(tile) + (ks >> 2) * kHalf + (ks & 3) * 32, 16, 1024, kSwizzle128B);
}
__device__ __forceinline__ uint64_t desc_v(const uint8_t *tile, int ks) {
  return smem_desc(smem_addr(tile) + ks * 2048, kHalf, 1024, kSwizzle128B);
}

// Columns of tile j that are worked on: a multiple of 32.
__device__ __forceinline__ int tile_cols(const Tiles &t, int j) {
  return (tile_end(t, j, BT) - tile_start(t, j, BT) + 31) & ~31;
}

// A warp copies 32 rows (lane r has row r's address; none: zeros) into rows
// row0 .. of a Q tile, D / 8 lanes to a row.
template <int D>
__device__ __forceinline__ void copy_q(uint8_t *tile, int row0, const __nv_bfloat16 *src, int lane) {
  constexpr int LR = D / 8, RW = 32 / LR;  // lanes a row, rows a step
  const int part = lane % LR;
#pragma unroll
  for (int k = 0; k < 32 / RW; ++k) {
    const int r = k * RW + lane / LR;
    const uint64_t p = __shfl_sync(0xffffffffu, reinterpret_cast<uint64_t>(src), r);
    uint8_t *dst = tile + (part >> 3) * kHalf + sw128_offset(row0 + r, part & 7);
    if (!p) *reinterpret_cast<uint4 *>(dst) = make_uint4(0, 0, 0, 0);
    else asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_addr(dst)), "l"(p + 16 * part) : "memory");
  }
}
__device__ __forceinline__ void copy_q_done() {
  asm volatile("cp.async.wait_all;" ::: "memory");
  fence_proxy_async();
}

// The scores of a tile become weights relative to the row's reference maximum
// m (base 2), which is raised where a score is above it by more than kLazy;
// the row's sums are rescaled then.  The scores of this tile came after the
// products of the last one, so O is stable.
template <int D>
__device__ __forceinline__ void raise_max(uint32_t o_col, float top, float &m, float &lsum) {
  const bool raise = top > m + kLazy;           // false while both are -inf
  const bool fix = raise && m != -INFINITY;     // -inf: the row's sums are still zero
  if (__any_sync(0xffffffffu, fix)) {
    const float f = fix ? exp2f(m - top) : 1.0f;
    lsum *= f;
#pragma unroll 1
    for (int c0 = 0; c0 < D; c0 += 32) {
      uint32_t r[32];
      tmem_ld32(o_col + c0, r);
      tmem_wait_ld();
#pragma unroll
      for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * f);
      tmem_st32(o_col + c0, r);
    }
  }
  if (raise) m = top;
}

// Weights of 32 columns, as bf16 pairs, and their sum.
__device__ __forceinline__ void weigh32(const float *x, float2 scale2, float2 neg2, float2 (&ps)[2], uint32_t (&p)[16]) {
#pragma unroll
  for (int i = 0; i < 32; i += 2) {
    const float2 t = ffma2(make_float2(x[i], x[i + 1]), scale2, neg2);
    const float2 e = make_float2(fast_exp2(t.x), fast_exp2(t.y));
    ps[(i >> 1) & 1] = fadd2(ps[(i >> 1) & 1], e);
    const __nv_bfloat162 h = __floats2bfloat162_rn(e.x, e.y);
    p[i >> 1] = *reinterpret_cast<const uint32_t *>(&h);
  }
}

__device__ __forceinline__ float max32(const float *x, float m) {
  float mx[4] = {m, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
  for (int i = 0; i < 32; i += 8)
#pragma unroll
    for (int k = 0; k < 4; ++k) mx[k] = fmax3(mx[k], x[i + 2 * k], x[i + 2 * k + 1]);
  return fmaxf(fmax3(mx[0], mx[1], mx[2]), mx[3]);
}

// A tile that every row of the warp sees whole.
template <int D>
__device__ __forceinline__ void soft_full(uint32_t s_col, uint32_t o_col, float scale, float &m, float &lsum) {
  float x[BT];
#pragma unroll
  for (int c = 0; c < 4; ++c) tmem_ld32f(s_col + 32 * c, &x[32 * c]);
  tmem_wait_ld();
  float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
  for (int i = 0; i < BT; i += 8)
#pragma unroll
    for (int k = 0; k < 4; ++k) mx[k] = fmax3(mx[k], x[i + 2 * k], x[i + 2 * k + 1]);
  raise_max<D>(o_col, __fmul_rn(fmaxf(fmax3(mx[0], mx[1], mx[2]), mx[3]), scale), m, lsum);
  const float neg = m == -INFINITY ? 0.0f : -m;
  const float2 scale2 = make_float2(scale, scale), neg2 = make_float2(neg, neg);
  float2 ps[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    uint32_t p[16];
    weigh32(&x[32 * c], scale2, neg2, ps, p);
    tmem_st16(s_col + 16 * c, p);
  }
  tmem_wait_st();
  const float2 a = fadd2(ps[0], ps[1]);
  lsum += a.x + a.y;
}

// The same with half the registers: 64 scores at a time, the second half read twice
// (its weights go where scores of the first half were).
template <int D>
__device__ __forceinline__ void soft_halves(uint32_t s_col, uint32_t o_col, float scale, float &m, float &lsum) {
  float x[64], top = -INFINITY;
#pragma unroll
  for (int h = 1; h >= 0; --h) {
    tmem_ld32f(s_col + 64 * h, x);
    tmem_ld32f(s_col + 64 * h + 32, x + 32);
    tmem_wait_ld();
    top = max32(x + 32, max32(x, top));
  }
  raise_max<D>(o_col, __fmul_rn(top, scale), m, lsum);
  const float neg = m == -INFINITY ? 0.0f : -m;
  const float2 scale2 = make_float2(scale, scale), neg2 = make_float2(neg, neg);
  float2 ps[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (h) {
      tmem_ld32f(s_col + 64, x);
      tmem_ld32f(s_col + 96, x + 32);
      tmem_wait_ld();
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      uint32_t p[16];
      weigh32(x + 32 * c, scale2, neg2, ps, p);
      tmem_st16(s_col + 32 * h + 16 * c, p);
    }
  }
  tmem_wait_st();
  const float2 a = fadd2(ps[0], ps[1]);
  lsum += a.x + a.y;
}

// A tile that ends early or that some rows see in part: 32 columns at a time,
// read twice.
template <int D>
__device__ __forceinline__ void soft_masked(uint32_t s_col, uint32_t o_col, float scale, const Span &sp, int t0, int t1,
                                            float &m, float &lsum) {
  const int nc = (t1 - t0 + 31) >> 5, a = t0 - sp.lo, end = min(sp.hi, t1) - sp.lo, se = min(sp.se, t1) - t0;
  const unsigned len = end > 0 ? (unsigned)end : 0u;
  float x[32], top = -INFINITY;
  auto load = [&](int c) {
    tmem_ld32f(s_col + 32 * c, x);
    tmem_wait_ld();
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i] = (unsigned)(a + 32 * c + i) < len || 32 * c + i < se ? x[i] : -INFINITY;
  };
#pragma unroll 1
  for (int c = 0; c < nc; ++c) {
    load(c);
    top = max32(x, top);
  }
  raise_max<D>(o_col, __fmul_rn(top, scale), m, lsum);
  const float neg = m == -INFINITY ? 0.0f : -m;
  const float2 scale2 = make_float2(scale, scale), neg2 = make_float2(neg, neg);
  float2 ps[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
#pragma unroll 1
  for (int c = 0; c < nc; ++c) {
    uint32_t p[16];
    load(c);
    weigh32(x, scale2, neg2, ps, p);
    tmem_st16(s_col + 16 * c, p);
  }
  tmem_wait_st();
  const float2 b = fadd2(ps[0], ps[1]);
  lsum += b.x + b.y;
}

// Where K and V of tile j of an item's nt stand among the item's 2 nt tiles in
// the ring, for packed caches and items of one row tile: in the order in which the
// MMAs take them, K0 K1 V0 K2 V1 .., so that a tile is written as soon as the one
// four places before it is done with.
__device__ __forceinline__ int k_place(int j) { return max(2 * j - 1, 0); }
__device__ __forceinline__ int v_place(int j, int nt) { return min(2 * j + 2, 2 * nt - 1); }

// A warp of the eight that write the values of a packed cache, K and V tile after
// tile into the ring.  A lane has one token's 32 channels of a group, 16 bytes of
// codes and a scale byte, D / 64 times a tile; eight lanes write eight rows' 16
// bytes of one place, which lie in different banks.  What is written was read a
// tile ahead of K and of V: nothing else hides the loads' latency.  V's channels are
// left as the codes' pairs (paired_place); the results are put in order on their way
// out.  32 positions and 4 heads to one over 36,896 tokens, 12 layers of 8 KV heads of
// 128 channels: 306 us, of 222 without the writing (its shared-memory traffic and issue
// slots are what the MMAs and the softmax wait for); with four warps, which left the
// softmax its registers, 354.
template <int D>
__device__ __forceinline__ void write_values(const PackedParams &P, Smem<D> &sm, int pw, int lane) {
  constexpr int NST = Smem<D>::NST, UN = D / 64;
  const Launch &L = P.L;
  volatile int *flags = sm.flags;
  const int grp = D == 128 ? lane >> 3 : (lane >> 3) & 1;
  const int row0 = 16 * pw + (lane & 7) + (D == 128 ? 0 : 8 * (lane >> 4));
  constexpr int kStep = 8;  // rows between a lane's
  // where its first row begins in a tile (a step further: 128 kStep bytes)
  const uint32_t at = (grp >> 1) * kHalf + sw128_offset(row0, (grp & 1) * 4);
  uint32_t g = 0;  // tiles written
  for (int n = 0;; ++n) {
    if (!wait_warp(&sm.plan_full[n & 1], (n >> 1) & 1, flags)) break;
    const Plan pl = sm.plan[n & 1];
    if (pl.rows == 0) break;
    __syncwarp();
    if (lane == 0) mbar_arrive(&sm.plan_empty[n & 1]);
    const Item it = pl.it;
    const Seg &sg = L.seg[it.s];
    const pk::Scales &sc = P.sc[it.s];
    const int64_t base = it.l * sg.sl + it.kvh * sg.sh + 16 * grp, gbase = it.l * sc.gl + it.kvh * sc.gh + grp;
    const uint8_t *kc = static_cast<const uint8_t *>(sg.k) + base, *ks = sc.k + gbase;
    const int64_t dv = static_cast<const uint8_t *>(sg.v) - static_cast<const uint8_t *>(sg.k), dvs = sc.v - sc.k;
    const int j_ask = max(pl.j1 - kAsk, pl.j0);
    if (pl.j0 == pl.j1 && pw == 0 && lane == 0) mbar_arrive(&sm.ask);  // no tiles
    uint4 w[2][UN];
    unsigned s[2][UN];
    auto read = [&](int a, int e, int kv, int i) {
      const int t = a + row0 + kStep * i;
      const int64_t tok = min(t, e - 1);
      w[kv][i] = __ldg(reinterpret_cast<const uint4 *>(kc + tok * sg.st + (kv ? dv : 0)));
      s[kv][i] = t < e ? __ldg(ks + tok * sc.gt + (kv ? dvs : 0)) : 0;
    };
    if (pl.j0 < pl.j1) {
      const int a = tile_start(pl.tl, pl.j0, BT), e = tile_end(pl.tl, pl.j0, BT);
#pragma unroll
      for (int i = 0; i < UN; ++i) read(a, e, 0, i), read(a, e, 1, i);
    }
    bool ok = true;
    const int ahead = pl.rows > BM || pl.j0 == pl.j1 ? 0 : 1;  // K of this many tiles before V: k_place and v_place
    for (int j = pl.j0 - ahead; j < pl.j1 && ok; ++j) {
      if (j == j_ask && pw == 0 && lane == 0) mbar_arrive(&sm.ask);
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        const int here = kv ? j : j + ahead;
        if (here < pl.j0 || here >= pl.j1) continue;
        const int jn = min(here + 1, pl.j1 - 1);  // the last tile is read once more, and not written
        const int a = tile_start(pl.tl, jn, BT), e = tile_end(pl.tl, jn, BT);
        const int st = g % NST;
        if (ok && g >= NST && !wait_warp(&sm.kv_empty[st], (g / NST - 1) & 1, flags)) ok = false;
        if (!ok) break;
        const uint32_t dst = smem_addr(sm.kv[st]) + at;
#pragma unroll
        for (int i = 0; i < UN; ++i) {
          const uint32_t y[4] = {w[kv][i].x, w[kv][i].y, w[kv][i].z, w[kv][i].w};
          const pk::BfScale f = pk::bf_scale(s[kv][i]);
          read(a, e, kv, i);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            uint32_t x[4];
            if (kv) pk::values8_paired(y[k], f, x);
            else pk::values8(y[k], f, x);
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"((dst ^ (k << 4)) + 128 * kStep * i), "r"(x[0]), "r"(x[1]),
                         "r"(x[2]), "r"(x[3])
                         : "memory");
          }
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.kv_full[st]);
        ++g;
      }
    }
    if (!ok) break;
  }
}

template <int D, typename Params>
__global__ void __launch_bounds__(Params::kPacked ? 640 : 384, 1) attend_tc(const __grid_constant__ Params P, WsHeader *hdr) {
  using S = Smem<D>;
  constexpr int NST = S::NST;
  constexpr bool PACKED = Params::kPacked;
  extern __shared__ uint8_t smem_raw[];
  S &sm = *reinterpret_cast<S *>(smem_raw + ((0u - smem_addr(smem_raw)) & 1023u));
  const Launch &L = P.L;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
  volatile int *flags = sm.flags;

  pdl_start_next();
  if (threadIdx.x == 0) {
    sm.flags[kAbort] = sm.flags[kRedoing] = 0;
    for (int b = 0; b < 2; ++b) {
      mbar_init(&sm.plan_full[b], 1);
      mbar_init(&sm.plan_empty[b], PACKED ? 17 : 10);  // TMA or eight warps that write values, MMA, eight softmax warps
      mbar_init(&sm.s_full[b], 1);
      mbar_init(&sm.p_full[b], 4);
      mbar_init(&sm.o_full[b], 1);
      mbar_init(&sm.o_empty[b], 4);
    }
    mbar_init(&sm.ask, 1);
    mbar_init(&sm.next_full, 1);
    mbar_init(&sm.q_full, 1);
    mbar_init(&sm.q_empty, 1);
    for (int s = 0; s < NST; ++s) {
      mbar_init(&sm.kv_full[s], PACKED ? 8 : 1);
      mbar_init(&sm.kv_empty[s], 1);
    }
    mbar_init(&sm.drain, 1);
    mbar_init(&sm.pub_full, 4);
    mbar_init(&sm.pub_empty, 4);
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(&sm.tmem, 512);
    tmem_relinquish();
  }
  if (warp >= 4 && warp < 12) {  // the first item's rows, a thread each (later ones are planned ahead by one warp)
    const Item it = decode_item(L, blockIdx.x);
    const Seg &sg = L.seg[it.s];
    const int i = threadIdx.x - 128, r = it.rt * L.rows_per_item + i;
    int3 u = make_int3(0x7fffffff, 0, 0);
    const int32_t *qpos = nullptr;
    copy_q<D>(sm.q[i / BM], (i % BM) & ~31, i < L.rows_per_item ? row_query<__nv_bfloat16>(L, sg, it, r, D, qpos) : nullptr, lane);
    sm.span[0][i] = row_sees(L, sg, qpos, u);
    u = join_warp(u);
    if (lane == 0) sm.first[warp - 4] = u;
    copy_q_done();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tm = sm.tmem;

  // registers: 104 + 2 x 200 a thread of each group of four warps = 3 x 168
  // (packed: 48 + 2 x 128 + 2 x 88 = 5 x 96)
  if (PACKED && warp >= 12) {
    regs_dec<88>();
    if constexpr (PACKED) write_values<D>(P, sm, warp - 12, lane);
  } else if (warp < 4) {
    regs_dec<PACKED ? 48 : 104>();
    if (!PACKED && warp == 0 && lane == 0) {
      // ------------------------------------------------------------ TMA
      if constexpr (!PACKED) {
      const uint64_t pol = policy_evict_normal();
      uint32_t g = 0;  // tiles copied
      bool ok = true;
      auto load = [&](const CUtensorMap *m, int tok, const Item &it) {
        const int s = g % NST;
        if (g >= NST && !wait(&sm.kv_empty[s], (g / NST - 1) & 1, flags)) return false;
        mbar_expect_tx(&sm.kv_full[s], S::kTile);
#pragma unroll
        for (int x = 0; x < D / 64; ++x) tma4(sm.kv[s] + x * kHalf, m, 64 * x, tok, it.kvh, it.l, &sm.kv_full[s], pol);
        ++g;
        return true;
      };
      for (int n = 0; ok; ++n) {
        if (!wait(&sm.plan_full[n & 1], (n >> 1) & 1, flags)) break;
        const Plan pl = sm.plan[n & 1];
        if (pl.rows == 0) break;
        mbar_arrive(&sm.plan_empty[n & 1]);
        const Item it = pl.it;
        const int j_ask = max(pl.j1 - kAsk, pl.j0);
        for (int j = pl.j0; j < max(pl.j1, pl.j0 + 1) && ok; ++j) {
          if (j == j_ask) mbar_arrive(&sm.ask);
          if (j == pl.j1) break;  // no tiles
          const int tok = tile_start(pl.tl, j, BT);
          ok = load(&P.k[it.s], tok, it) && load(&P.v[it.s], tok, it);
        }
      }
      if (flags[kAbort])  // let the copies already issued land before the CTA leaves
        for (uint32_t u = g > NST ? g - NST : 0; u < g; ++u) mbar_wait_drain(&sm.kv_full[u % NST], (u / NST) & 1, kWait);
      }
    } else if (warp == 1) {
      // ------------------------------------------------------------ MMAs
      // The whole warp keeps step and one elected lane issues: in code that a
      // single lane runs, an MMA took 100 cycles to issue.
      uint32_t g = 0, np[2] = {0, 0}, uses[2] = {0, 0};  // earlier items: tiles, tiles of each group, items that filled O_b
      bool ok = true;
      auto kv_wait = [&](uint32_t u) { return wait_warp(&sm.kv_full[u % NST], (u / NST) & 1, flags); };
      // descriptors of stage 0 and of Q: a stage, k-step or row tile further adds to the address field
      const uint64_t k0 = desc_kmajor(sm.kv[0], 0), v0 = desc_v(sm.kv[0], 0), q0 = desc_kmajor(sm.q[0], 0);
      constexpr uint64_t kStep = S::kTile >> 4;
      // by one lane: S_b = Q K^T with K tile u
      auto qk = [&](int qt, int b, uint32_t u, int cols) {
        const uint32_t idesc = idesc_bf16_f32(BM, 0, 0, 0) | ((uint32_t)(cols >> 3) << 17);
        const uint64_t ka = k0 + (u % NST) * kStep, qa = q0 + qt * kStep;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
          const uint64_t at = ((ks >> 2) * kHalf + (ks & 3) * 32) >> 4;
          mma_bf16(tm + BT * b, qa + at, ka + at, idesc, ks > 0);
        }
        mma_commit(&sm.s_full[b]);
      };
      // by one lane: O_b (+)= P_b V with V tile u
      auto pv = [&](int b, uint32_t u, int cols, bool first) {
        constexpr uint32_t idesc = idesc_bf16_f32(BM, D, 0, 1);
        const uint64_t va = v0 + (u % NST) * kStep;
#pragma unroll
        for (int ks = 0; ks < BT / 16; ++ks)
          if (16 * ks < cols)
            mma_bf16_ts(tm + 256 + D * b, tm + BT * b + 8 * ks, va + ks * (2048 >> 4), idesc, !first || ks > 0);
      };
      // weights of group b's i-th tile of this item are there, and O_b may be written
      auto p_wait = [&](int b, int i) {
        return (i > 0 || uses[b] == 0 || wait_warp(&sm.o_empty[b], (uses[b] - 1) & 1, flags)) &&
               wait_warp(&sm.p_full[b], (np[b] + i) & 1, flags);
      };
      for (int n = 0; ok; ++n) {
        if (!wait_warp(&sm.plan_full[n & 1], (n >> 1) & 1, flags)) break;
        const Plan pl = sm.plan[n & 1];
        if (pl.rows == 0) break;
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.plan_empty[n & 1]);
        if (!wait_warp(&sm.q_full, n & 1, flags)) break;
        const int nt = pl.j1 - pl.j0;
        if (nt == 0 && lane == 0) mbar_arrive(&sm.q_empty);  // else behind the last Q K^T
        if (pl.rows > BM) {
          // two row tiles: tile j's Q K^T right behind tile j - 1's P V, group by group
          if (nt > 0 && (ok = kv_wait(2 * g))) {
            tc_fence_after();
            if (elect_one()) {
              const int cols = tile_cols(pl.tl, pl.j0);
              qk(0, 0, 2 * g, cols);
              qk(1, 1, 2 * g, cols);
              mma_commit(&sm.kv_empty[2 * g % NST]);
              if (nt == 1) mma_commit(&sm.q_empty);
            }
            __syncwarp();
          }
          for (int j = 1; j <= nt && ok; ++j) {
            const uint32_t uk = 2 * (g + j), uv = uk - 1;
            const int cv = tile_cols(pl.tl, pl.j0 + j - 1), ck = j < nt ? tile_cols(pl.tl, pl.j0 + j) : 0;
            if (!(ok = kv_wait(uv) && (j == nt || kv_wait(uk)))) break;
#pragma unroll
            for (int b = 0; b < 2; ++b) {
              if (!p_wait(b, j - 1)) {
                ok = false;
                break;
              }
              tc_fence_after();
              if (elect_one()) {
                pv(b, uv, cv, j == 1);
                if (b) mma_commit(&sm.kv_empty[uv % NST]);
                if (j < nt) {
                  qk(b, b, uk, ck);
                  if (b) mma_commit(&sm.kv_empty[uk % NST]);
                  if (b && j + 1 == nt) mma_commit(&sm.q_empty);
                } else {
                  mma_commit(&sm.o_full[b]);
                }
              }
              __syncwarp();
            }
          }
          np[0] += nt, np[1] += nt;
          uses[0] += nt > 0, uses[1] += nt > 0;
        } else {
          // one row tile, the groups take alternate token tiles
          for (int j = 0; j < nt + 2 && ok && nt > 0; ++j) {
            const uint32_t uk = 2 * g + (PACKED ? k_place(j) : 2 * j), uv = 2 * g + (PACKED ? v_place(j - 2, nt) : 2 * j - 3);
            const int b = j & 1, i = (j - 2) >> 1;
            if (j >= 2) {
              ok = (uint32_t)(j - 2) >= (uint32_t)nt || (kv_wait(uv) && p_wait(b, i));
              if (!ok) break;
              tc_fence_after();
              if (j - 2 < nt && elect_one()) {
                pv(b, uv, tile_cols(pl.tl, pl.j0 + j - 2), i == 0);
                mma_commit(&sm.kv_empty[uv % NST]);
                if (j >= nt) mma_commit(&sm.o_full[b]);
              }
              __syncwarp();
            }
            if (j < nt) {
              if (!(ok = kv_wait(uk))) break;
              tc_fence_after();
              if (elect_one()) {
                qk(0, b, uk, tile_cols(pl.tl, pl.j0 + j));
                mma_commit(&sm.kv_empty[uk % NST]);
                if (j + 1 == nt) mma_commit(&sm.q_empty);
              }
              __syncwarp();
            }
          }
          np[0] += (nt + 1) / 2, np[1] += nt / 2;
          uses[0] += nt > 0, uses[1] += nt > 1;
        }
        g += nt;
      }
      if (__any_sync(0xffffffffu, flags[kAbort] != 0)) {
        if (elect_one()) {
          mma_commit(&sm.drain);  // every MMA issued by this thread has completed
          mbar_wait_drain(&sm.drain, 0, kWait);
        }
        __syncwarp();
      }
    } else if (warp == 3) {
      // ------------------------------------------------------------ plans and Q rows
      int item = blockIdx.x;
      int q_last = -1;  // the last item whose Q TMA copied
      for (int n = 0;; ++n) {
        const int buf = n & 1;
        if (n >= 2 && !wait_warp(&sm.plan_empty[buf], ((n >> 1) - 1) & 1, flags)) break;
        if (n > 0) {
          if (!wait_warp(&sm.ask, (n - 1) & 1, flags)) break;
          if (lane == 0) ask_next(&sm.next, &sm.next_full);
          if (!wait_warp(&sm.next_full, (n - 1) & 1, flags)) {
            if (lane == 0) mbar_wait_drain(&sm.next_full, (n - 1) & 1, kWait);  // it lands before the block's memory goes
            break;
          }
          item = read_next(&sm.next);
          __syncwarp();
        }
        if (item < 0) {
          if (lane == 0) {
            sm.plan[buf].rows = 0;
            mbar_arrive(&sm.plan_full[buf]);
          }
          break;
        }
        const Item it = decode_item(L, item);
        const Seg &sg = L.seg[it.s];
        const int r0 = it.rt * L.rows_per_item, rows = min(L.rows_per_item, sg.R - r0);
        int3 u = make_int3(0x7fffffff, 0, 0);
        if (n == 0) {
          if (lane < 8) u = sm.first[lane];
        } else {
          rows_see<__nv_bfloat16, D, 2 * BM>(L, sg, it, r0, rows, sm.span[buf], u);
        }
        u = join_warp(u);
        if (lane == 0) {
          const Tiles tl = make_tiles(u.x, u.y, u.z, BT);
          sm.plan[buf] = {tl, chunk_tile(tl, it.c, it.n), chunk_tile(tl, it.c + 1, it.n), rows, it};
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.plan_full[buf]);
        if (n > 0 && !wait_warp(&sm.q_empty, (n - 1) & 1, flags)) break;
        if (n > 0 && P.has_q && sg.t >= 0) {
          // between two items nothing else hides this copy: TMA, where it can
          if (lane == 0) {
            const int nq = rows > BM ? 2 : 1;
            mbar_expect_tx(&sm.q_full, nq * S::kTile);
            for (int i = 0; i < nq; ++i)
              for (int x = 0; x < D / 64; ++x)
                tma_q(sm.q[i] + x * kHalf, &P.q[sg.t], 64 * x, (r0 + i * BM) / L.g, it.l * L.H + it.kvh, &sm.q_full);
          }
          q_last = n;
          __syncwarp();
          continue;
        }
        if (n > 0) {
#pragma unroll 1
          for (int i = 0; i < rows; i += 32) {
            const int32_t *qpos;
            copy_q<D>(sm.q[i / BM], i % BM, i + lane < rows ? row_query<__nv_bfloat16>(L, sg, it, r0 + i + lane, D, qpos) : nullptr, lane);
          }
          copy_q_done();
          __syncwarp();
        }
        if (lane == 0) mbar_arrive(&sm.q_full);
      }
      // left early: what is under way lands before the block's memory goes
      if (flags[kAbort] && q_last >= 0 && lane == 0) mbar_wait_drain(&sm.q_full, q_last & 1, kWait);
    }
  } else {
    // ------------------------------------------------------------ softmax
    regs_inc<PACKED ? 128 : 200>();
    const int hb = (warp - 4) >> 2, wq = warp & 3, row = wq * 32 + lane;
    const uint32_t lanes = (uint32_t)(wq * 32) << 16;
    const uint32_t s_col = tm + lanes + BT * hb, o_col = tm + lanes + 256 + D * hb;
    uint32_t ns = 0, uses = 0, npub = 0;  // score tiles, items that filled O_hb, joined items
    bool ok = true;
    for (int n = 0; ok; ++n) {
      if (!wait_warp(&sm.plan_full[n & 1], (n >> 1) & 1, flags)) break;
      const Plan pl = sm.plan[n & 1];
      if (pl.rows == 0) break;
      const Tiles tl = pl.tl;
      const bool two = pl.rows > BM;
      const int lrow = two ? hb * BM + row : row;  // row of the item
      const Span sp = sm.span[n & 1][lrow];
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.plan_empty[n & 1]);
      const Item it = pl.it;
      const Seg &sg = L.seg[it.s];
      const bool warp_rows = lrow - lane < pl.rows;  // the warp has a row of the item
      float m_used = -INFINITY, lsum = 0.0f;
      const int step = two ? 1 : 2, first = pl.j0 + (two ? 0 : hb);
      for (int j = first; j < pl.j1; j += step) {
        if (!wait_warp(&sm.s_full[hb], ns & 1, flags)) {
          ok = false;
          break;
        }
        ++ns;
        tc_fence_after();
        if (!warp_rows) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&sm.p_full[hb]);
          continue;
        }
        const int t0 = tile_start(tl, j, BT), t1 = tile_end(tl, j, BT);
        if (__all_sync(0xffffffffu, sp.lo <= t0 && t0 + BT <= min(sp.hi, t1)))
          if constexpr (PACKED) soft_halves<D>(s_col, o_col, L.scale_log2, m_used, lsum);
          else soft_full<D>(s_col, o_col, L.scale_log2, m_used, lsum);
        else
          soft_masked<D>(s_col, o_col, L.scale_log2, sp, t0, t1, m_used, lsum);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.p_full[hb]);
      }
      if (!ok) break;
      // ---------------------------------------------------------- results
      const bool mine = first < pl.j1, other = !two && pl.j0 + 1 < pl.j1;  // O_hb / O_1 of a joined item was filled
      if (mine && !wait_warp(&sm.o_full[hb], uses & 1, flags)) break;
      if (mine) ++uses;
      tc_fence_after();
      float f0 = 1.0f, f1 = 0.0f, m = m_used;
      if (!two) {
        if (hb == 1) {
          if (npub > 0 && !wait_warp(&sm.pub_empty, (npub - 1) & 1, flags)) break;
          ++npub;
          sm.pub[row] = make_float2(m_used, lsum);
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&sm.pub_full);
          continue;  // group 0 reads O_1
        }
        if (!wait_warp(&sm.pub_full, npub & 1, flags)) break;
        ++npub;
        tc_fence_after();
        const float2 o1 = sm.pub[row];
        m = fmaxf(m_used, o1.x);
        const float ref = m == -INFINITY ? 0.0f : m;
        f0 = exp2f(m_used - ref), f1 = exp2f(o1.x - ref);
        lsum = fmaf(lsum, f0, o1.y * f1);
      }
      const int r = it.rt * L.rows_per_item + lrow;
      const bool valid = lrow < pl.rows;
      float *pdst = nullptr, *ldst = nullptr;
      __nv_bfloat16 *dst = nullptr;
      if (valid && it.split) {
        pdst = L.po + part_index(L, sg, it, r) * D;
        L.pml[part_index(L, sg, it, r)] = make_float2(m, lsum);
      } else if (valid) {
        int rr = r;
        const Traj &t = L.t[traj_of_row(L, sg, rr)];
        const int64_t orow = row_index(L, t, it.l, it.kvh, rr);
        dst = static_cast<__nv_bfloat16 *>(t.out) + orow * D;
        if (t.lse) ldst = t.lse + orow;
      }
      if (ldst) *ldst = lse_of(m, lsum);
      const float inv = norm_of(lsum);
      const float g0 = dst ? f0 * inv : f0, g1 = dst ? f1 * inv : f1;
      float chk = 0.0f;
      if (warp_rows) {
        // 64 bytes of every row at a time through shared memory, so that four
        // lanes store them side by side, in few steps: both groups and all SMs
        // come here at the same time, with the tensor cores idle.
        RowsOut rows_out(smem_addr(sm.stage[warp - 4]),
                         pdst ? reinterpret_cast<uint64_t>(pdst) : reinterpret_cast<uint64_t>(dst), lane);
#pragma unroll 1
        for (int c0 = 0; c0 < D; c0 += 32) {
          float y[32];
#pragma unroll
          for (int i = 0; i < 32; ++i) y[i] = 0.0f;
#pragma unroll 1
          for (int k = 0; k < (mine ? 1 + other : 0); ++k) {
            float z[32];
            const float gk = k ? g1 : g0;
            tmem_ld32f(o_col + D * k + c0, z);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; ++i) y[i] = fmaf(z[i], gk, y[i]);
          }
          float ck[4] = {chk, 0.0f, 0.0f, 0.0f};  // NaN if any is not finite
#pragma unroll
          for (int i = 0; i < 32; ++i) ck[i & 3] = fmaf(y[i], 0.0f, ck[i & 3]);
          chk = (ck[0] + ck[1]) + (ck[2] + ck[3]);
          uint32_t w[32];
          if (it.split) {
#pragma unroll
            for (int i = 0; i < 32; ++i) w[i] = __float_as_uint(y[PACKED ? pk::paired_place(i) : i]);
            rows_out.put(w);
            rows_out.put(w + 16);
          } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int a = PACKED ? pk::paired_place(2 * i) : 2 * i, b = PACKED ? pk::paired_place(2 * i + 1) : 2 * i + 1;
              const __nv_bfloat162 h = __floats2bfloat162_rn(y[a], y[b]);
              w[i] = *reinterpret_cast<const uint32_t *>(&h);
            }
            rows_out.put(w);
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (mine) mbar_arrive(&sm.o_empty[hb]);
        if (other) mbar_arrive(&sm.o_empty[1]);
        if (!two) mbar_arrive(&sm.pub_empty);
      }
      unsigned bad = __ballot_sync(0xffffffffu, valid && ((chk != 0.0f && isfinite(lsum)) || is_far(m)));
      const bool redo = bad != 0;
      if (redo) redoing(flags, 1);
      while (bad) {  // a masked value that is not finite met a weight of zero, or the scores are very large
        const int b = __ffs(bad) - 1;
        bad &= bad - 1;
        const Span one = {__shfl_sync(0xffffffffu, sp.lo, b), __shfl_sync(0xffffffffu, sp.hi, b),
                          __shfl_sync(0xffffffffu, sp.se, b)};
        float mb = __shfl_sync(0xffffffffu, m, b), lb = __shfl_sync(0xffffffffu, lsum, b);
        const int32_t *qpos;
        const void *qb = row_query<__nv_bfloat16>(L, sg, it, r - lane + b, D, qpos);
        const bool far = is_far(mb);
        if constexpr (PACKED) {
          if (far) mb = pk::redo_max<D>(L, sg, P.sc[it.s], it.l, it.kvh, qb, one, pl.tl, BT, pl.j0, pl.j1);
        } else {
          if (far) mb = redo_max<__nv_bfloat16, D>(L, sg, it.l, it.kvh, qb, one, pl.tl, BT, pl.j0, pl.j1);
        }
        float o[D / 32] = {}, l2 = NAN;
        if (!isnan(mb)) {  // else the row is NaN
          const float ref = mb == -INFINITY ? 0.0f : mb;
          if constexpr (PACKED)
            l2 = pk::redo_row<D>(L, sg, P.sc[it.s], it.l, it.kvh, qb, one, pl.tl, BT, pl.j0, pl.j1, ref, o, far, !is_far(mb));
          else
            l2 = redo_row<__nv_bfloat16, D>(L, sg, it.l, it.kvh, qb, one, pl.tl, BT, pl.j0, pl.j1, ref, o, far, !is_far(mb));
        }
        __syncwarp();
        write_row_warp<__nv_bfloat16, D>(L, sg, it, r - lane + b, o, mb, far ? l2 : lb);
      }
      if (redo) redoing(flags, -1);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) tmem_dealloc(tm, 512);
  if (threadIdx.x == 0 && sm.flags[kAbort]) record_error(hdr, COMMITKV_ERR_TIMEOUT, 30);
  pdl_wait();
}

// ------------------------------------------------------------------ host
PFN_cuTensorMapEncodeTiled_v12000 encode_fn() {
  static const PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
    void *p = nullptr;
    cudaDriverEntryPointQueryResult q;
    const bool ok = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) ==
                        cudaSuccess &&
                    q == cudaDriverEntryPointSuccess;
    return ok ? reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p) : nullptr;
  }();
  return fn;
}

bool map_q(CUtensorMap *m, const Launch &L, const Traj &t) {
  auto enc = encode_fn();
  if (!enc) return false;
  const cuuint64_t d2 = (cuuint64_t)L.d * 2;
  const cuuint64_t dims[4] = {(cuuint64_t)L.d, (cuuint64_t)L.g, (cuuint64_t)t.W, (cuuint64_t)L.M * L.H};
  const cuuint64_t strides[3] = {t.W * d2, d2, (cuuint64_t)L.g * t.W * d2};
  const cuuint32_t box[4] = {64, (cuuint32_t)L.g, (cuuint32_t)(BM / L.g), 1}, es[4] = {1, 1, 1, 1};
  return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(t.q), dims, strides, box, es,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace
}  // namespace at
}  // namespace ckv
