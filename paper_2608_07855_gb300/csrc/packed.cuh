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

__device__ __forceinline__ float sigma_of(unsigned b) {
  if (b >= kNanScale) return __int_as_float(0x7fffffff);
  return __half2float(__ushort_as_half((unsigned short)(b << 7))) * kUnit;
}

// Whether the fast kernels can read a cache: codes 16 bytes, scale rows whole.
inline bool wide(const Cache &c, int d) {
  const uintptr_t codes = (uintptr_t)c.k | (uintptr_t)c.v | (uintptr_t)(c.sl | c.sh | c.st);
  const uintptr_t scales = (uintptr_t)c.ks | (uintptr_t)c.vs | (uintptr_t)(c.gl | c.gh | c.gt);
  return codes % 16 == 0 && scales % (d / kGroup) == 0;
}

// An attention call's work: the launch description of full-width caches, whose
// segments' k, v, sl, sh and st are the codes' (bytes), and the scales beside it.
struct Scales {
  const uint8_t *k, *v;
  int64_t gl, gh, gt;
};
struct Launch {
  at::Launch L;
  Scales sc[kMaxTraj];
};
static_assert(sizeof(Launch) <= 32764, "kernel parameters");

// CUDA cores: any alignment.  Rows per item: 16 or 64.
cudaError_t launch_simt(const Launch &P, cudaStream_t s, bool early);
// Wide caches, queries 16-byte aligned; 8 rows per item, or 16 (bf16).
cudaError_t launch_rows(const Launch &P, cudaStream_t s, bool early);

// Fills the full-width rows from the codes: launch for `n` caches.
cudaError_t launch_read(const commitkv_shape *s, int n, const commitkv_packed *c, const commitkv_rows *r,
                        const uint8_t *layers, int n_layers, cudaStream_t stream);

commitkv_status check_caches(const commitkv_shape *s, int n, const commitkv_packed *x, bool positions, bool queries);

}  // namespace pk
}  // namespace ckv
