// Attention over packed caches on the CUDA cores: any alignment and stride.
//
// One block of 256 threads per item; tiles of 64 tokens, whose values are
// written to shared memory as fp32 (exactly, from codes and scale).  Thread
// (ty, tx) of a 16 x 16 grid has row ty: its scores against four tokens (tx
// + 16 j) of a tile, then D / 16 channels of its sums, so a row's running max
// and sum live in registers of the 16 lanes that share it.  Bound by fp32 FMAs
// and the shared-memory reads that feed them; the kernel for what the others
// cannot read: one token over 131,071, bf16, 32 query on 8 KV heads of 128 channels,
// 714 us (aligned, on the tensor cores, 39).
//
// The only values of V that are not finite are 32 channels of a NaN scale.  They
// stand as zeros in the tile, so that a masked token's cannot reach a row, and
// the rows that see such a token note the group.
#include <string.h>

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
using sm103::ffma2;

constexpr int TT = 64;   // tokens per tile
constexpr int NT = 256;  // threads
constexpr int BM = 16;   // rows of an item

template <int D>
struct Smem {
  static constexpr int KP = D + 4;  // rows 16 bytes apart in the banks
  float q[BM][KP];
  union {  // the weights take the place of the keys
    float k[TT][KP];
    float p[BM][TT + 4];
  };
  float v[TT][D];
  uint8_t nan[TT];     // groups of a token's values that are NaN
  unsigned any_nan;
  unsigned row_nan[BM];
  const void *qrow[BM];
  int lo[BM], hi[BM], se[BM];
  int u_lo, u_hi, u_se;
};

template <typename T, int D>
__global__ void __launch_bounds__(NT, 2) attend_packed_simt(const __grid_constant__ Launch P) {
  constexpr int CH = D / 16, GR = D / kGroup;
  extern __shared__ __align__(16) uint8_t raw[];
  Smem<D> &sm = *reinterpret_cast<Smem<D> *>(raw);
  const at::Launch &L = P.L;
  const int tid = threadIdx.x, ty = tid / 16, tx = tid % 16;
  at::pdl_start_next();
  const Item it = at::decode_item(L, blockIdx.x);
  const Seg &sg = L.seg[it.s];
  const Scales &sc = P.sc[it.s];
  const int r0 = it.rt * BM;
  if (tid == 0) sm.u_lo = 0x7fffffff, sm.u_hi = 0, sm.u_se = 0;
  __syncthreads();
  for (int r = tid; r < BM; r += NT) {
    Span sp = {0, 0, 0};
    int rr = r0 + r;
    sm.qrow[r] = nullptr;
    sm.row_nan[r] = 0;
    if (rr < sg.R) {
      const Traj &t = L.t[sg.t];
      sm.qrow[r] = static_cast<const T *>(t.q) + at::row_index(L, t, it.l, it.kvh, rr) * D;
      sp = at::row_span(sg.pos, sg.S, t.qpos[rr / L.g], L.window, L.sinks);
      if (sp.lo < sp.hi) {
        atomicMin(&sm.u_lo, sp.lo);
        atomicMax(&sm.u_hi, sp.hi);
      }
      atomicMax(&sm.u_se, sp.se);
    }
    sm.lo[r] = sp.lo, sm.hi[r] = sp.hi, sm.se[r] = sp.se;
  }
  __syncthreads();
#pragma unroll 4
  for (int e = tid; e < BM * D; e += NT) {
    const T *q = static_cast<const T *>(sm.qrow[e / D]);
    sm.q[e / D][e % D] = q ? to_f32(q[e % D]) : 0.0f;
  }
  const Tiles tl = at::make_tiles(sm.u_lo, sm.u_hi, sm.u_se, TT);
  const int j0 = at::chunk_tile(tl, it.c, it.n), j1 = at::chunk_tile(tl, it.c + 1, it.n);
  const int64_t base = it.l * sg.sl + it.kvh * sg.sh, sbase = it.l * sc.gl + it.kvh * sc.gh;
  const uint8_t *kb = static_cast<const uint8_t *>(sg.k) + base, *vb = static_cast<const uint8_t *>(sg.v) + base;
  const uint8_t *ksb = sc.k + sbase, *vsb = sc.v + sbase;
  const Span sp = {sm.lo[ty], sm.hi[ty], sm.se[ty]};
  float m = -INFINITY, lsum = 0.0f;
  float2 o[CH / 2];
#pragma unroll
  for (int c = 0; c < CH / 2; ++c) o[c] = make_float2(0.0f, 0.0f);
  for (int j = j0; j < j1; ++j) {
    const int a = at::tile_start(tl, j, TT), n = at::tile_end(tl, j, TT) - a;
    __syncthreads();
    if (tid < TT) sm.nan[tid] = 0;
    if (tid == 0) sm.any_nan = 0;
    __syncthreads();
#pragma unroll 4
    for (int e = tid; e < TT * D / 4; e += NT) {
      const int i = e / (D / 4), c = 4 * (e % (D / 4));
      float4 x[2] = {make_float4(0.0f, 0.0f, 0.0f, 0.0f), make_float4(0.0f, 0.0f, 0.0f, 0.0f)};
      if (i < n) {
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          const int64_t tok = a + i;
          const uint8_t *w = (kv ? vb : kb) + tok * sg.st + c / 2;
          float sigma = sigma_of((kv ? vsb : ksb)[tok * sc.gt + c / kGroup]);
          if (kv && isnan(sigma)) {
            if (c % kGroup == 0) {
              atomicOr(reinterpret_cast<unsigned *>(&sm.nan[i & ~3]), 1u << (8 * (i & 3) + c / kGroup));
              atomicOr(&sm.any_nan, 1u);
            }
            sigma = 0.0f;
          }
          const unsigned w0 = w[0], w1 = w[1];
          x[kv] = make_float4((float)((int)(w0 & 15) - 8) * sigma, (float)((int)(w0 >> 4) - 8) * sigma,
                              (float)((int)(w1 & 15) - 8) * sigma, (float)((int)(w1 >> 4) - 8) * sigma);
        }
      }
      *reinterpret_cast<float4 *>(&sm.k[i][c]) = x[0];
      *reinterpret_cast<float4 *>(&sm.v[i][c]) = x[1];
    }
    __syncthreads();
    if (sm.any_nan) {
      for (int e = tid; e < BM * TT; e += NT) {
        const int r = e / TT, i = e % TT;
        const Span s1 = {sm.lo[r], sm.hi[r], sm.se[r]};
        if (i < n && sm.nan[i] && at::sees(s1, a + i)) atomicOr(&sm.row_nan[r], (unsigned)sm.nan[i]);
      }
    }
    float2 s2[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) s2[t] = make_float2(0.0f, 0.0f);
#pragma unroll 4
    for (int c = 0; c < D; c += 4) {
      const float4 q4 = *reinterpret_cast<const float4 *>(&sm.q[ty][c]);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const float4 k4 = *reinterpret_cast<const float4 *>(&sm.k[tx + 16 * t][c]);
        s2[t] = ffma2(make_float2(q4.x, q4.y), make_float2(k4.x, k4.y), s2[t]);
        s2[t] = ffma2(make_float2(q4.z, q4.w), make_float2(k4.z, k4.w), s2[t]);
      }
    }
    __syncthreads();  // the keys have been read
    float s[4], mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int tok = tx + 16 * t;
      s[t] = tok < n && at::sees(sp, a + tok) ? __fmul_rn(s2[t].x + s2[t].y, L.scale_log2) : -INFINITY;
      mx = fmaxf(mx, s[t]);
    }
#pragma unroll
    for (int w = 8; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
    const float mn = fmaxf(m, mx), ref = mn == -INFINITY ? 0.0f : mn;
    const float f = exp2f(m - ref);
    float ps = 0.0f;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const float p = exp2f(s[t] - ref);
      ps += p;
      sm.p[ty][tx + 16 * t] = p;
    }
#pragma unroll
    for (int w = 8; w > 0; w >>= 1) ps += __shfl_xor_sync(0xffffffffu, ps, w);
    lsum = fmaf(lsum, f, ps);
    m = mn;
#pragma unroll
    for (int c = 0; c < CH / 2; ++c) o[c].x *= f, o[c].y *= f;
    __syncwarp();  // a row's weights are written and read by the same half warp
#pragma unroll 2
    for (int t = 0; t < TT; t += 4) {
      const float4 p4 = *reinterpret_cast<const float4 *>(&sm.p[ty][t]);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float p = u == 0 ? p4.x : u == 1 ? p4.y : u == 2 ? p4.z : p4.w;
#pragma unroll
        for (int c = 0; c < CH / 4; ++c) {
          const float4 x = *reinterpret_cast<const float4 *>(&sm.v[t + u][64 * c + 4 * tx]);
          o[2 * c] = ffma2(make_float2(p, p), make_float2(x.x, x.y), o[2 * c]);
          o[2 * c + 1] = ffma2(make_float2(p, p), make_float2(x.z, x.w), o[2 * c + 1]);
        }
      }
    }
  }
  // the rows' sums through shared memory, then a warp per row
  __syncthreads();
  float(*so)[Smem<D>::KP] = sm.q;
  float *sml = &sm.p[0][0];
#pragma unroll
  for (int c = 0; c < CH / 4; ++c)
    *reinterpret_cast<float4 *>(&so[ty][64 * c + 4 * tx]) =
        make_float4(o[2 * c].x, o[2 * c].y, o[2 * c + 1].x, o[2 * c + 1].y);
  if (tx == 0) sml[2 * ty] = m, sml[2 * ty + 1] = lsum;
  __syncthreads();
  for (int r = tid / 32; r < BM && r0 + r < sg.R; r += NT / 32) {
    float x[D / 32];
#pragma unroll
    for (int c = 0; c < GR; ++c)  // channel tid % 32 + 32 c: group c
      x[c] = sm.row_nan[r] >> c & 1 ? __int_as_float(0x7fffffff) : so[r][tid % 32 + 32 * c];
    at::write_row_warp<T, D>(L, sg, it, r0 + r, x, sml[2 * r], sml[2 * r + 1]);
  }
  at::pdl_chain();
}

template <typename T, int D>
cudaError_t launch(const Launch &P, cudaStream_t s, bool early) {
  const int smem = (int)sizeof(Smem<D>);
  const cudaError_t e =
      cudaFuncSetAttribute(attend_packed_simt<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  return at::launch_after(attend_packed_simt<T, D>, P.L.item_off[P.L.n_seg], NT, smem, s, early, P);
}

template <typename T>
cudaError_t launch_t(const Launch &P, cudaStream_t s, bool early) {
  return P.L.d == 128 ? launch<T, 128>(P, s, early) : launch<T, 64>(P, s, early);
}

}  // namespace

cudaError_t launch_simt(const Launch &P, cudaStream_t s, bool early) {
  return P.L.dtype == COMMITKV_BF16 ? launch_t<__nv_bfloat16>(P, s, early) : launch_t<float>(P, s, early);
}

}  // namespace pk
}  // namespace ckv
