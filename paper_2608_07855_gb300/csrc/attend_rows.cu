// Attention with 16 query rows of a (layer, KV head) slice to an item: decoded
// tokens (the g heads of one to a few positions).  16-byte aligned caches.
//
// Such a call is bound by reading K and V once, so the kernel is built around
// the loads: a block of four warps per item, two blocks on an SM, each warp
// with a ring of its own of three stages of K and V (8 KB), copied with
// 16-byte cp.async and never waiting for another warp: up to 128 KB an SM are
// under way.  16 rows are what one warp-level MMA takes, so mma.sync does the
// products from registers (the scores' fragments are the weights' operand as
// they stand); a tcgen05 tile has 128 rows, and with its round trip through
// tensor memory 4 rows over 64 caches of up to 8,192 tokens took 245 us against
// 191 to 200 here (95 to 99 % of the copy rate).
// bf16: the weights are split in two bf16 terms (2^-17 of each is lost): the
// second product per tile is free, and the output is as exact as with fp32
// weights.  fp32: every operand is split in two tf32 terms, three products
// (2^-21 of a factor is lost, the order of fp32's own rounding in a sum of
// 128); on the CUDA cores such calls were bound by FMAs and shared memory (8
// caches of up to 6,000 tokens: 74 us, 34 here).
// Tiles of 4 WT tokens, WT to a warp; the warps' sums are joined at the end.
#include <string.h>

#include "attend.cuh"
#include "sm103.cuh"

namespace ckv {
namespace at {
namespace {

using sm103::fast_exp2;
using sm103::smem_addr;

constexpr int NW = 4;
constexpr int NST = 3;
constexpr float kLazy = 8.0f;

template <typename T, int D>
struct Smem {
  static constexpr int kRow = D * (int)sizeof(T);
  static constexpr int WT = 4096 / kRow;  // tokens of a warp: 4 KB of K and of V
  static constexpr int TT = NW * WT;               // of a tile
  union {
    alignas(128) uint8_t ring[NW][NST][2][WT * kRow];
    float o[NW][16][D + 4];
  };
  float2 ml[NW][16];
};

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(a)
               : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(a)
               : "memory");
}
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, "
      "%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void mma1688(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, "
      "%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// x = hi + lo: hi rounded to tf32's 10 fraction bits, lo the exact rest, of
// which the MMA reads the first 10 as well: 2^-21 of x is lost at most.  (An
// infinite x gives NaN; see the end of the kernel.)
__device__ __forceinline__ void split_tf32(float x, uint32_t &hi, uint32_t &lo) {
  hi = (__float_as_uint(x) + 0x1000u) & 0xffffe000u;
  lo = __float_as_uint(x - __uint_as_float(hi));
}
__device__ __forceinline__ float lds32(uint32_t a) {
  float x;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(a) : "memory");
  return x;
}

// Two weights as bf16 pairs hi + lo.
__device__ __forceinline__ void split2(float x, float y, uint32_t &hi, uint32_t &lo) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
  const __nv_bfloat162 l = __floats2bfloat162_rn(x - __low2float(h), y - __high2float(h));
  hi = *reinterpret_cast<const uint32_t *>(&h);
  lo = *reinterpret_cast<const uint32_t *>(&l);
}

template <typename T, int D>
__global__ void __launch_bounds__(NW * 32, 2) attend_rows(const __grid_constant__ Launch L) {
  using S = Smem<T, D>;
  constexpr int WT = S::WT, TT = S::TT;
  constexpr bool F32 = sizeof(T) == 4;
  extern __shared__ __align__(128) uint8_t raw[];
  S &sm = *reinterpret_cast<S *>(raw);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  pdl_start_next();
  const Item it = decode_item(L, blockIdx.x);
  const Seg &sg = L.seg[it.s];

  const int r0 = it.rt * 16, rows = min(16, sg.R - r0);
  // what the rows see: row r in lane r
  Span mine = {0, 0x7fffffff, 0};
  int lo = 0x7fffffff, hi = 0, se = 0;
  uint64_t qp = 0;  // the row's query
  if (lane < rows) {
    int rr = r0 + lane;
    const Traj &t = L.t[traj_of_row(L, sg, rr)];
    qp = reinterpret_cast<uint64_t>(static_cast<const T *>(t.q) + row_index(L, t, it.l, it.kvh, rr) * D);
    mine = row_span(sg.pos, sg.S, t.qpos[rr / L.g], L.window, L.sinks);
    if (mine.lo < mine.hi) lo = mine.lo, hi = mine.hi;
    se = mine.se;
  }
  // Q as the A operand: lane holds rows lane / 4 and + 8; bf16 channels 2 (lane
  // % 4) + {0, 1, 8, 9} of each k-step of 16, fp32 channels lane % 4 + {0, 4} of
  // each of 8
  uint32_t q[D / (F32 ? 8 : 16)][4];
  Span sp[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = lane / 4 + 8 * h;
    sp[h] = {__shfl_sync(0xffffffffu, mine.lo, r), __shfl_sync(0xffffffffu, mine.hi, r),
             __shfl_sync(0xffffffffu, mine.se, r)};
    const uint32_t *p = reinterpret_cast<const uint32_t *>(__shfl_sync(0xffffffffu, qp, r));
#pragma unroll
    for (int k = 0; k < D / (F32 ? 8 : 16); ++k) {
      q[k][h] = p ? p[8 * k + lane % 4] : 0;
      q[k][2 + h] = p ? p[8 * k + 4 + lane % 4] : 0;
    }
  }
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) {
    lo = min(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = max(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    se = max(se, __shfl_xor_sync(0xffffffffu, se, o));
  }
  lo = __shfl_sync(0xffffffffu, lo, 0), hi = __shfl_sync(0xffffffffu, hi, 0), se = __shfl_sync(0xffffffffu, se, 0);
  const Tiles tl = make_tiles(lo, hi, se, TT);
  const int j0 = chunk_tile(tl, it.c, it.n), j1 = chunk_tile(tl, it.c + 1, it.n);

  // copies of tile j into its stage: tokens behind the tile's end as zeros
  constexpr int CH = S::kRow / 16;  // 16-byte pieces of a row
  const T *kb = static_cast<const T *>(sg.k) + (int64_t)it.l * sg.sl + (int64_t)it.kvh * sg.sh;
  const int64_t dv = reinterpret_cast<const uint8_t *>(sg.v) - reinterpret_cast<const uint8_t *>(sg.k);
  const uint32_t ring = smem_addr(sm.ring[warp]);
  constexpr uint32_t kStage = 2 * WT * S::kRow;
  auto load = [&](int j, int st) {
    if (j < j1) {
      const int a = tile_start(tl, j, TT) + WT * warp, e = tile_end(tl, j, TT);
#pragma unroll
      for (int i = 0; i < WT * CH / 32; ++i) {
        const int x = i * 32 + lane, r = x / CH, c = x % CH;
        const bool in = a + r < e;
        const uint8_t *src = reinterpret_cast<const uint8_t *>(kb + (int64_t)(in ? a + r : 0) * sg.st) + 16 * c;
        // pieces swapped by row, so that a fragment's rows lie in different banks
        const uint32_t dst = ring + st * kStage + r * S::kRow, kx = (c ^ (r & 7)) << 4, vx = F32 ? (c ^ (r & 6)) << 4 : kx;
        const int n = in ? 16 : 0;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + kx), "l"(src), "r"(n) : "memory");
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + WT * S::kRow + vx), "l"(src + dv), "r"(n)
                     : "memory");
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int s = 0; s < NST - 1; ++s) load(j0 + s, s);

  float o[D / 8][4];
#pragma unroll
  for (int n = 0; n < D / 8; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) o[n][i] = 0.0f;
  float m[2] = {-INFINITY, -INFINITY}, lsum[2] = {0.0f, 0.0f};
  for (int j = j0, st = 0; j < j1; ++j) {
    asm volatile("cp.async.wait_group %0;" ::"n"(NST - 2) : "memory");
    __syncwarp();  // every lane's copies of this stage are there, and its reads of the last one are done
    load(j + NST - 1, st == 0 ? NST - 1 : st - 1);
    const uint32_t ks = ring + st * kStage, vs = ks + WT * S::kRow;
    st = st + 1 == NST ? 0 : st + 1;
    constexpr int NT = WT / 8;  // groups of eight tokens
    float s[NT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[t][i] = 0.0f;
    if constexpr (F32) {
      // K row lane / 4 of each group, channels lane % 4 + {0, 4} of each k-step
      const int kr = lane / 4;
#pragma unroll
      for (int k0 = 0; k0 < D / 8; k0 += 2) {
        // the MMA's sums are cut off, not rounded: chains of two k-steps, joined in
        // fp32 (error of the outputs 4.5e-7 against 8e-7 with four, 3.6e-7 with one;
        // 167, 160 and 177 us for 16 caches of up to 8,192 tokens)
        float d[NT][4];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) d[t][i] = 0.0f;
#pragma unroll
        for (int k = k0; k < k0 + 2; ++k) {
          uint32_t ah[4], al[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) split_tf32(__uint_as_float(q[k][i]), ah[i], al[i]);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            uint32_t bh[2], bl[2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
              split_tf32(lds32(ks + (kr + 8 * t) * S::kRow + (((2 * k + i) ^ kr) << 4) + 4 * (lane % 4)), bh[i], bl[i]);
            mma1688(d[t], al, bh[0], bh[1]);
            mma1688(d[t], ah, bl[0], bl[1]);
            mma1688(d[t], ah, bh[0], bh[1]);
          }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[t][i] += d[t][i];
      }
    } else {
      // of 16 tokens K rows lane % 8 (+ 8: the second eight), 16-byte pieces 2 k and 2 k + 1
      const int kr = lane % 8 + (lane / 16) * 8, kc = (lane / 8) % 2;
#pragma unroll
      for (int k = 0; k < D / 16; ++k)
#pragma unroll
        for (int u = 0; u < NT / 2; ++u) {
          uint32_t b[4];
          ldsm4(b, ks + (16 * u + kr) * S::kRow + (((2 * k + kc) ^ (kr & 7)) << 4));
          mma16816(s[2 * u], q[k], b[0], b[1]);
          mma16816(s[2 * u + 1], q[k], b[2], b[3]);
        }
    }
    const int a = tile_start(tl, j, TT) + WT * warp, e = tile_end(tl, j, TT);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bool whole = a + WT <= e && sp[h].lo <= a && a + WT <= sp[h].hi;
      float top = -INFINITY;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float &x = s[t][2 * h + i];
          const int tok = a + 8 * t + 2 * (lane % 4) + i;
          if (!whole) x = tok < e && sees(sp[h], tok) ? x : -INFINITY;
          top = fmaxf(top, x);
        }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = __fmul_rn(fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2)), L.scale_log2);
      const bool raise = top > m[h] + kLazy;
      if (__any_sync(0xffffffffu, raise)) {
        const float f = raise ? (m[h] == -INFINITY ? 0.0f : exp2f(m[h] - top)) : 1.0f;
        lsum[h] *= f;
#pragma unroll
        for (int n = 0; n < D / 8; ++n) o[n][2 * h] *= f, o[n][2 * h + 1] *= f;
        if (raise) m[h] = top;
      }
      const float neg = m[h] == -INFINITY ? 0.0f : -m[h];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float &x = s[t][2 * h + i];
          x = fast_exp2(fmaf(x, L.scale_log2, neg));
          lsum[h] += x;
        }
    }
    if constexpr (F32) {
      // tokens 2 (lane % 4) and + 1 of a group as the k slots lane % 4 and + 4:
      // the scores' own layout; a tile's sums by themselves, as above
      uint32_t ah[NT][4], al[NT][4];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) split_tf32(s[t][2 * (i & 1) + (i >> 1)], ah[t][i], al[t][i]);
#pragma unroll
      for (int n = 0; n < D / 8; ++n) {
        float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const int vr = 8 * t + 2 * (lane % 4);
          uint32_t bh[2], bl[2];
#pragma unroll
          for (int i = 0; i < 2; ++i)
            split_tf32(lds32(vs + (vr + i) * S::kRow + (((2 * n + lane / 16) ^ (vr & 6)) << 4) + 4 * (lane / 4 % 4)),
                       bh[i], bl[i]);
          mma1688(d, al[t], bh[0], bh[1]);
          mma1688(d, ah[t], bl[0], bl[1]);
          mma1688(d, ah[t], bh[0], bh[1]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) o[n][i] += d[i];
      }
    } else {
      // V: tokens as the k dimension, two groups of eight channels at a time
      const int vr = lane % 16, vc = lane / 16;
#pragma unroll
      for (int u = 0; u < NT / 2; ++u) {
        uint32_t hi4[4], lo4[4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          split2(s[2 * u][2 * h], s[2 * u][2 * h + 1], hi4[h], lo4[h]);
          split2(s[2 * u + 1][2 * h], s[2 * u + 1][2 * h + 1], hi4[2 + h], lo4[2 + h]);
        }
#pragma unroll
        for (int n = 0; n < D / 16; ++n) {
          uint32_t b[4];
          ldsm4t(b, vs + (16 * u + vr) * S::kRow + (((2 * n + vc) ^ (vr & 7)) << 4));
          mma16816(o[2 * n], hi4, b[0], b[1]);
          mma16816(o[2 * n + 1], hi4, b[2], b[3]);
          mma16816(o[2 * n], lo4, b[0], b[1]);
          mma16816(o[2 * n + 1], lo4, b[2], b[3]);
        }
      }
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    lsum[h] += __shfl_xor_sync(0xffffffffu, lsum[h], 1);
    lsum[h] += __shfl_xor_sync(0xffffffffu, lsum[h], 2);
  }
  __syncthreads();  // the rings are done with
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = lane / 4 + 8 * h;
#pragma unroll
    for (int n = 0; n < D / 8; ++n)
      *reinterpret_cast<float2 *>(&sm.o[warp][r][8 * n + 2 * (lane % 4)]) = make_float2(o[n][2 * h], o[n][2 * h + 1]);
    if (lane % 4 == 0) sm.ml[warp][r] = make_float2(m[h], lsum[h]);
  }
  __syncthreads();
  for (int r = warp; r < rows; r += NW) {
    float mr = -INFINITY, lr = 0.0f, x[D / 32], w[NW];
#pragma unroll
    for (int i = 0; i < NW; ++i) mr = fmaxf(mr, sm.ml[i][r].x);
    const float ref = mr == -INFINITY ? 0.0f : mr;
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      w[i] = exp2f(sm.ml[i][r].x - ref);
      lr = fmaf(sm.ml[i][r].y, w[i], lr);
    }
    bool fine = true;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      x[c] = 0.0f;
#pragma unroll
      for (int i = 0; i < NW; ++i) x[c] = fmaf(sm.o[i][r][lane + 32 * c], w[i], x[c]);
      fine = fine && isfinite(x[c]);
    }
    const bool far = is_far(mr);
    if (far || !__all_sync(0xffffffffu, fine)) {
      const Span one = {__shfl_sync(0xffffffffu, mine.lo, r), __shfl_sync(0xffffffffu, mine.hi, r),
                        __shfl_sync(0xffffffffu, mine.se, r)};
      const void *qrow = reinterpret_cast<const void *>(__shfl_sync(0xffffffffu, qp, r));
      // a visible infinite key, whose score may be -inf, is NaN in the split products of fp32
      const bool anew = far || (F32 && !isfinite(lr));  // the maximum and the sum as well
      bool redo = isfinite(lr);
      if (anew) {
        const float top = redo_max<T, D>(L, sg, it.l, it.kvh, qrow, one, tl, TT, j0, j1);
        redo = !isnan(top);
        if (redo) mr = top;
        else lr = NAN;
      }
      if (redo) {
        const float l2 =
            redo_row<T, D>(L, sg, it.l, it.kvh, qrow, one, tl, TT, j0, j1, mr == -INFINITY ? 0.0f : mr, x, anew,
                           !is_far(mr));
        if (anew) lr = l2;
      }
    }
    write_row_warp<T, D>(L, sg, it, r0 + r, x, mr, lr);
  }
  pdl_chain();
}

template <typename T, int D>
cudaError_t launch(const Launch &L, cudaStream_t s, bool early) {
  constexpr int smem = (int)sizeof(Smem<T, D>);
  const cudaError_t e = cudaFuncSetAttribute(attend_rows<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  return launch_after(attend_rows<T, D>, L.item_off[L.n_seg], NW * 32, smem, s, early, L);
}

}  // namespace

cudaError_t launch_rows(const Launch &L, cudaStream_t s, bool early) {
  if (L.dtype == COMMITKV_BF16)
    return L.d == 128 ? launch<__nv_bfloat16, 128>(L, s, early) : launch<__nv_bfloat16, 64>(L, s, early);
  return L.d == 128 ? launch<float, 128>(L, s, early) : launch<float, 64>(L, s, early);
}

}  // namespace at
}  // namespace ckv
