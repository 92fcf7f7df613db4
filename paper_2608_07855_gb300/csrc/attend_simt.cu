// Attention on the CUDA cores: caches, queries or outputs that the tensor-core
// kernels cannot read or write (pointers or strides that are not 16-byte
// aligned).
//
// One block of 256 threads per item; tiles of 64 tokens.  Thread (ty, tx) of a
// 16 x 16 grid owns TM rows: their scores against four tokens (tx + 16 j) of a
// tile, then D / 16 channels of their sums, so a row's running max and sum
// live in registers of the 16 lanes that share it.  Q, K, V and the weights go
// through shared memory as fp32.  Bound by fp32 FMAs (taken in packed pairs)
// and the shared-memory reads that feed them.
#include <string.h>

#include "attend.cuh"
#include "sm103.cuh"

namespace ckv {
namespace at {
namespace {

using sm103::ffma2;

constexpr int TT = 64;   // tokens per tile
constexpr int NT = 256;  // threads

template <int D, int TM>
struct Smem {
  static constexpr int BM = 16 * TM;
  static constexpr int KP = D + 4;  // rows 16 bytes apart in the banks
  float q[BM][KP];
  union {  // the weights take the place of the keys: two blocks of 64 rows fit an SM
    float k[TT][KP];
    float p[BM][TT + 4];
  };
  float v[TT][D];
  const void *qrow[BM];
  int lo[BM], hi[BM], se[BM];
  int u_lo, u_hi, u_se;
};

// Row i of a tile of K and V, channels 4 c .. 4 c + 3, as fp32.
template <typename T>
__device__ __forceinline__ void copy4(float *dst, const T *src, bool in, bool wide) {
  if constexpr (sizeof(T) == 4) {
    if (wide) {
      const int n = in ? 16 : 0;
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(sm103::smem_addr(dst)), "l"(src), "r"(n)
                   : "memory");
      return;
    }
  }
  float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (in) x = make_float4(to_f32(src[0]), to_f32(src[1]), to_f32(src[2]), to_f32(src[3]));
  *reinterpret_cast<float4 *>(dst) = x;
}

template <typename T, int D, int TM>
__global__ void __launch_bounds__(NT, 2) attend_simt(const __grid_constant__ Launch L) {
  constexpr int BM = 16 * TM, CH = D / 16;
  extern __shared__ __align__(16) uint8_t raw[];
  Smem<D, TM> &sm = *reinterpret_cast<Smem<D, TM> *>(raw);
  const int tid = threadIdx.x, ty = tid / 16, tx = tid % 16;
  pdl_start_next();
  const Item it = decode_item(L, blockIdx.x);
  const Seg &sg = L.seg[it.s];
  const int r0 = it.rt * BM;
  if (tid == 0) sm.u_lo = 0x7fffffff, sm.u_hi = 0, sm.u_se = 0;
  __syncthreads();
  for (int r = tid; r < BM; r += NT) {
    Span sp = {0, 0, 0};
    int rr = r0 + r;
    sm.qrow[r] = nullptr;
    if (rr < sg.R) {
      const Traj &t = L.t[traj_of_row(L, sg, rr)];
      sm.qrow[r] = static_cast<const T *>(t.q) + row_index(L, t, it.l, it.kvh, rr) * D;
      sp = row_span(sg.pos, sg.S, t.qpos[rr / L.g], L.window, L.sinks);
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
  const Tiles tl = make_tiles(sm.u_lo, sm.u_hi, sm.u_se, TT);
  const int j0 = chunk_tile(tl, it.c, it.n), j1 = chunk_tile(tl, it.c + 1, it.n);
  const T *kb = static_cast<const T *>(sg.k) + (int64_t)it.l * sg.sl + (int64_t)it.kvh * sg.sh;
  const T *vb = static_cast<const T *>(sg.v) + (int64_t)it.l * sg.sl + (int64_t)it.kvh * sg.sh;
  const bool wide = (((uintptr_t)kb | (uintptr_t)vb | (uintptr_t)(sg.st * 4)) & 15) == 0;
  Span sp[TM];
  float m[TM], lsum[TM];
  float2 o[TM][CH / 2];
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int r = ty * TM + i;
    sp[i] = {sm.lo[r], sm.hi[r], sm.se[r]};
    m[i] = -INFINITY;
    lsum[i] = 0.0f;
#pragma unroll
    for (int c = 0; c < CH / 2; ++c) o[i][c] = make_float2(0.0f, 0.0f);
  }
  for (int j = j0; j < j1; ++j) {
    const int a = tile_start(tl, j, TT), n = tile_end(tl, j, TT) - a;
    __syncthreads();
#pragma unroll 4
    for (int e = tid; e < TT * D / 4; e += NT) {
      const int i = e / (D / 4), c = 4 * (e % (D / 4));
      const int64_t at = (int64_t)(i < n ? a + i : 0) * sg.st + c;
      copy4(&sm.k[i][c], kb + at, i < n, wide);
      copy4(&sm.v[i][c], vb + at, i < n, wide);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    float2 s2[TM][4];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int c = 0; c < 4; ++c) s2[i][c] = make_float2(0.0f, 0.0f);
#pragma unroll 4
    for (int c = 0; c < D; c += 4) {
      float4 q4[TM], k4[4];
#pragma unroll
      for (int i = 0; i < TM; ++i) q4[i] = *reinterpret_cast<const float4 *>(&sm.q[ty * TM + i][c]);
#pragma unroll
      for (int t = 0; t < 4; ++t) k4[t] = *reinterpret_cast<const float4 *>(&sm.k[tx + 16 * t][c]);
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          s2[i][t] = ffma2(make_float2(q4[i].x, q4[i].y), make_float2(k4[t].x, k4[t].y), s2[i][t]);
          s2[i][t] = ffma2(make_float2(q4[i].z, q4[i].w), make_float2(k4[t].z, k4[t].w), s2[i][t]);
        }
    }
    __syncthreads();  // the keys have been read
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      float s[4], mx = -INFINITY;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int tok = tx + 16 * t;
        s[t] = tok < n && sees(sp[i], a + tok) ? __fmul_rn(s2[i][t].x + s2[i][t].y, L.scale_log2) : -INFINITY;
        mx = fmaxf(mx, s[t]);
      }
#pragma unroll
      for (int w = 8; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
      const float mn = fmaxf(m[i], mx), ref = mn == -INFINITY ? 0.0f : mn;
      const float f = exp2f(m[i] - ref);
      float ps = 0.0f;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const float p = exp2f(s[t] - ref);
        ps += p;
        sm.p[ty * TM + i][tx + 16 * t] = p;
      }
#pragma unroll
      for (int w = 8; w > 0; w >>= 1) ps += __shfl_xor_sync(0xffffffffu, ps, w);
      lsum[i] = fmaf(lsum[i], f, ps);
      m[i] = mn;
#pragma unroll
      for (int c = 0; c < CH / 2; ++c) o[i][c].x *= f, o[i][c].y *= f;
    }
    __syncwarp();  // a row's weights are written and read by the same half warp
#pragma unroll 2
    for (int t = 0; t < TT; t += 4) {
      float4 p4[TM];
#pragma unroll
      for (int i = 0; i < TM; ++i) p4[i] = *reinterpret_cast<const float4 *>(&sm.p[ty * TM + i][t]);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        float2 v2[CH / 2];
#pragma unroll
        for (int c = 0; c < CH / 4; ++c) {
          const float4 x = *reinterpret_cast<const float4 *>(&sm.v[t + u][64 * c + 4 * tx]);
          v2[2 * c] = make_float2(x.x, x.y);
          v2[2 * c + 1] = make_float2(x.z, x.w);
        }
#pragma unroll
        for (int i = 0; i < TM; ++i) {
          const float p = u == 0 ? p4[i].x : u == 1 ? p4[i].y : u == 2 ? p4[i].z : p4[i].w;
#pragma unroll
          for (int c = 0; c < CH / 2; ++c) o[i][c] = ffma2(make_float2(p, p), v2[c], o[i][c]);
        }
      }
    }
  }
  // the rows' sums through shared memory, then a warp per row
  __syncthreads();
  float(*so)[Smem<D, TM>::KP] = sm.q;
  float *sml = &sm.p[0][0];
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int r = ty * TM + i;
#pragma unroll
    for (int c = 0; c < CH / 4; ++c)
      *reinterpret_cast<float4 *>(&so[r][64 * c + 4 * tx]) =
          make_float4(o[i][2 * c].x, o[i][2 * c].y, o[i][2 * c + 1].x, o[i][2 * c + 1].y);
    if (tx == 0) sml[2 * r] = m[i], sml[2 * r + 1] = lsum[i];
  }
  __syncthreads();
  for (int r = tid / 32; r < BM && r0 + r < sg.R; r += NT / 32) {
    float x[D / 32];
    bool fine = true;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      x[c] = so[r][tid % 32 + 32 * c];
      fine = fine && isfinite(x[c]);
    }
    const float mr = sml[2 * r], lr = sml[2 * r + 1];
    if (!__all_sync(0xffffffffu, fine) && isfinite(lr)) {
      const Span one = {sm.lo[r], sm.hi[r], sm.se[r]};
      redo_row<T, D>(L, sg, it.l, it.kvh, sm.qrow[r], one, tl, TT, j0, j1, mr == -INFINITY ? 0.0f : mr, x, false,
                     false);
    }
    write_row_warp<T, D>(L, sg, it, r0 + r, x, mr, lr);
  }
  pdl_chain();
}

template <typename T, int D, int TM>
cudaError_t launch(const Launch &L, cudaStream_t s, bool early) {
  const int smem = (int)sizeof(Smem<D, TM>);
  const cudaError_t e = cudaFuncSetAttribute(attend_simt<T, D, TM>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  return launch_after(attend_simt<T, D, TM>, L.item_off[L.n_seg], NT, smem, s, early, L);
}

template <typename T>
cudaError_t launch_t(const Launch &L, cudaStream_t s, bool early) {
  if (L.rows_per_item == 16) return L.d == 128 ? launch<T, 128, 1>(L, s, early) : launch<T, 64, 1>(L, s, early);
  return L.d == 128 ? launch<T, 128, 4>(L, s, early) : launch<T, 64, 4>(L, s, early);
}

}  // namespace

cudaError_t launch_simt(const Launch &L, cudaStream_t s, bool early) {
  return L.dtype == COMMITKV_BF16 ? launch_t<__nv_bfloat16>(L, s, early) : launch_t<float>(L, s, early);
}

}  // namespace at
}  // namespace ckv
