// Packed caches (4-bit codes, a scale byte to 32 channels): what the kernels on
// them share.  The format is in include/commitkv.h.
#pragma once

#include <cuda_fp16.h>

#include "attend.cuh"

namespace ckv {
namespace pk {

constexpr int kGroup = 32;        // channels of a scale
constexpr int kNanScale = 0xf8;   // scale bytes from here on are NaN
constexpr float kUnit = 0.015625f;  // 2^-6: sigma over the fp16 number of the byte

// One trajectory's codes and scales; strides in bytes.
struct Cache {
  uint8_t *k, *v;
  int64_t sl, sh, st;
  uint8_t *ks, *vs;
  int64_t gl, gh, gt;
};

inline Cache to_dev(const commitkv_packed &x) {
  return {x.k, x.v, x.stride_layer, x.stride_head, x.stride_tok, x.k_scale, x.v_scale, x.scale_layer, x.scale_head, x.scale_tok};
}

// A segment's scale bytes, beside its codes; strides in bytes.
struct Scales {
  const uint8_t *k, *v;
  int64_t gl, gh, gt;
};

__device__ __forceinline__ float sigma_of(unsigned b) {
  if (b >= kNanScale) return __int_as_float(0x7fffffff);
  return __half2float(__ushort_as_half((unsigned short)(b << 7))) * kUnit;
}

// Values as bf16 numbers: (x & 0x000f000f) | 0x43004300 are the numbers 128 + u of two
// codes, one fma with (s, -136 s) makes them (u - 8) s: exact (136 s has eight
// significant bits).
struct BfScale {
  __nv_bfloat162 s, off;
};
__device__ __forceinline__ BfScale bf_scale(unsigned b) {
  // from 8 on the byte's exponent and mantissa are bf16's, 106 higher; below, steps of 2^-23
  uint32_t x = b * 16 + (106u << 7);
  if (b < 8) x = __float_as_uint((float)b * 1.1920928955078125e-7f) >> 16;
  if (b >= kNanScale) x = 0x7fff;
  x = __byte_perm(x, x, 0x1010);
  BfScale r;
  r.s = *reinterpret_cast<const __nv_bfloat162 *>(&x);
  r.off = __hmul2(r.s, __float2bfloat162_rn(-136.0f));
  return r;
}
__device__ __forceinline__ uint32_t bf_pair(uint32_t x, const BfScale &s) {
  uint32_t y;
  asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(y) : "r"(x), "r"(0x000f000fu), "r"(0x43004300u));
  const __nv_bfloat162 v = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&y), s.s, s.off);
  return *reinterpret_cast<const uint32_t *>(&v);
}
// A word's eight values in their order.
__device__ __forceinline__ void values8(uint32_t w, const BfScale &s, uint32_t (&x)[4]) {
  const uint32_t h = w >> 4;
  x[0] = bf_pair(__byte_perm(w, h, 0x4400), s);
  x[1] = bf_pair(__byte_perm(w, h, 0x5511), s);
  x[2] = bf_pair(__byte_perm(w, h, 0x6622), s);
  x[3] = bf_pair(__byte_perm(w, h, 0x7733), s);
}
// The same in the order 0, 4, 1, 5, 2, 6, 3, 7.
__device__ __forceinline__ void values8_paired(uint32_t w, const BfScale &s, uint32_t (&x)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = bf_pair(w >> (4 * i), s);
}
__device__ __forceinline__ constexpr int paired_place(int c) { return (c & ~7) + 2 * (c & 3) + (c >> 2 & 1); }

// Score of a token against a query, both read by one thread.
template <int D>
__device__ __forceinline__ float score_of(const __nv_bfloat16 *q, const uint8_t *codes, const uint8_t *scales) {
  float dot = 0.0f;
#pragma unroll 1
  for (int g = 0; g < D / kGroup; ++g) {
    const float sigma = sigma_of(scales[g]);
#pragma unroll 8
    for (int i = 0; i < kGroup; ++i)
      dot = fmaf(to_f32(q[kGroup * g + i]), (float)((int)(codes[16 * g + i / 2] >> (4 * (i & 1)) & 15) - 8) * sigma, dot);
  }
  return dot;
}

// at::redo_row and at::redo_max on packed caches.
template <int D>
__device__ __noinline__ float redo_row(const at::Launch &L, const at::Seg &sg, const Scales &sc, int l, int kvh,
                                       const void *qrow, at::Span sp, at::Tiles tl, int tile, int j0, int j1, float m,
                                       float *o, bool want_sum, bool fused) {
  const int lane = threadIdx.x & 31;
  const __nv_bfloat16 *q = static_cast<const __nv_bfloat16 *>(qrow);
  const int64_t base = (int64_t)l * sg.sl + (int64_t)kvh * sg.sh, gbase = (int64_t)l * sc.gl + (int64_t)kvh * sc.gh;
  const uint8_t *k = static_cast<const uint8_t *>(sg.k) + base, *v = static_cast<const uint8_t *>(sg.v) + base;
  float lsum = 0.0f;
  bool gone = false;
#pragma unroll
  for (int c = 0; c < D / 32; ++c) o[c] = 0.0f;
  for (int j = j0; j < j1; ++j) {
    const int a = at::tile_start(tl, j, tile), e = at::tile_end(tl, j, tile);
    for (int i0 = a; i0 < e; i0 += 32) {
      const int i = i0 + lane;
      const bool in = i < e && at::sees(sp, i);
      float p = 0.0f;
      if (in) {
        const float s = score_of<D>(q, k + (int64_t)i * sg.st, sc.k + gbase + (int64_t)i * sc.gt);
        p = exp2f(fused ? fmaf(s, L.scale_log2, -m) : __fmul_rn(s, L.scale_log2) - m);
      }
      lsum += p;
      if (gone) continue;
      const unsigned seen = __ballot_sync(0xffffffffu, in);
#pragma unroll 4
      for (int u = 0; u < 32; ++u) {
        const float pu = __shfl_sync(0xffffffffu, p, u);
        if (!(seen >> u & 1)) continue;
        const uint8_t *row = v + (int64_t)(i0 + u) * sg.st, *sr = sc.v + gbase + (int64_t)(i0 + u) * sc.gt;
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
          o[c] = fmaf(pu, (float)((int)(row[16 * c + lane / 2] >> (4 * (lane & 1)) & 15) - 8) * sigma_of(sr[c]), o[c]);
      }
    }
    bool done = true;  // NaN in every channel stays
#pragma unroll
    for (int c = 0; c < D / 32; ++c) done = done && isnan(o[c]);
    gone = __all_sync(0xffffffffu, done);
    if (gone && !want_sum) break;
  }
  return warp_sum(lsum);
}
template <int D>
__device__ __noinline__ float redo_max(const at::Launch &L, const at::Seg &sg, const Scales &sc, int l, int kvh,
                                       const void *qrow, at::Span sp, at::Tiles tl, int tile, int j0, int j1) {
  const uint8_t *k = static_cast<const uint8_t *>(sg.k) + (int64_t)l * sg.sl + (int64_t)kvh * sg.sh;
  const uint8_t *ks = sc.k + (int64_t)l * sc.gl + (int64_t)kvh * sc.gh;
  float top = -INFINITY;
  bool bad = false;
  for (int j = j0; j < j1; ++j) {
    const int e = at::tile_end(tl, j, tile);
    for (int i = at::tile_start(tl, j, tile) + (threadIdx.x & 31); i < e; i += 32) {
      if (!at::sees(sp, i)) continue;
      const float s =
          __fmul_rn(score_of<D>(static_cast<const __nv_bfloat16 *>(qrow), k + (int64_t)i * sg.st, ks + (int64_t)i * sc.gt),
                    L.scale_log2);
      bad = bad || isnan(s) || s == INFINITY;
      top = fmaxf(top, s);
    }
    if (__any_sync(0xffffffffu, bad)) return NAN;
  }
  return warp_max(top);
}

// Whether the fast kernels can read a cache: codes 16 bytes, scale rows whole.
inline bool wide(const Cache &c, int d) {
  const uintptr_t codes = (uintptr_t)c.k | (uintptr_t)c.v | (uintptr_t)(c.sl | c.sh | c.st);
  const uintptr_t scales = (uintptr_t)c.ks | (uintptr_t)c.vs | (uintptr_t)(c.gl | c.gh | c.gt);
  return codes % 16 == 0 && scales % (d / kGroup) == 0;
}

// An attention call's work: the launch description of full-width caches, whose
// segments' k, v, sl, sh and st are the codes' (bytes), and the scales beside it.
struct Launch {
  at::Launch L;
  Scales sc[kMaxTraj];
};
static_assert(sizeof(Launch) <= 32764, "kernel parameters");

// CUDA cores: any alignment; 16 rows per item.
cudaError_t launch_simt(const Launch &P, cudaStream_t s, bool early);
// Wide caches, queries 16-byte aligned; 8 rows per item, or 16 (bf16).
cudaError_t launch_rows(const Launch &P, cudaStream_t s, bool early);
// Wide caches of a bf16 shape, queries and outputs 16-byte aligned; 256 rows per item.
cudaError_t launch_tc(const Launch &P, WsHeader *hdr, cudaStream_t s, bool early);

// Fills the full-width rows from the codes: launch for `n` caches.
cudaError_t launch_read(const commitkv_shape *s, int n, const commitkv_packed *c, const commitkv_rows *r,
                        const uint8_t *layers, int n_layers, cudaStream_t stream);

commitkv_status check_caches(const commitkv_shape *s, int n, const commitkv_packed *x, bool positions, bool queries);

}  // namespace pk
}  // namespace ckv
