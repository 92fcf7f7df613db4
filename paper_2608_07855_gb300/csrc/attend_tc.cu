// Attention on the tensor cores (bf16, 16-byte aligned caches): the kernel's
// launch.  K and V tiles come by TMA.
#include "attend_tc_impl.cuh"

namespace ckv {
namespace at {
namespace {

bool map_kv(CUtensorMap *m, const void *base, const Launch &L, const Seg &sg) {
  auto enc = encode_fn();
  if (!enc) return false;
  const cuuint64_t dims[4] = {(cuuint64_t)L.d, (cuuint64_t)sg.S, (cuuint64_t)L.H, (cuuint64_t)L.M};
  const cuuint64_t strides[3] = {(cuuint64_t)sg.st * 2, (cuuint64_t)sg.sh * 2, (cuuint64_t)sg.sl * 2};
  const cuuint32_t box[4] = {64, BT, 1, 1}, es[4] = {1, 1, 1, 1};
  return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(base), dims, strides, box, es,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D>
cudaError_t launch(const TcParams &P, WsHeader *hdr, cudaStream_t s, bool early) {
  const int smem = (int)sizeof(Smem<D>) + 1024;
  const cudaError_t e = cudaFuncSetAttribute(attend_tc<D, TcParams>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  return launch_after(attend_tc<D, TcParams>, P.L.item_off[P.L.n_seg], 384, smem, s, early, P, hdr);
}

}  // namespace

cudaError_t launch_tc(const Launch &L, WsHeader *hdr, cudaStream_t s, bool early) {
  static thread_local TcParams P;
  P.L = L;
  P.has_q = L.n_traj <= kMaxQ && L.g <= BM && BM % L.g == 0;
  bool used[kMaxSeg] = {};
  for (int k = 0; k < L.n_seg; ++k) used[L.order[k]] = L.item_off[k] < L.item_off[k + 1];
  for (int i = 0; i < L.n_seg; ++i) {
    const Seg &sg = L.seg[i];
    if (!used[i]) continue;
    if (P.has_q && sg.t >= 0 && !map_q(&P.q[sg.t], L, L.t[sg.t])) return cudaErrorInvalidValue;
    if (sg.S == 0) continue;
    if (!map_kv(&P.k[i], sg.k, L, sg) || !map_kv(&P.v[i], sg.v, L, sg)) return cudaErrorInvalidValue;
  }
  return L.d == 128 ? launch<128>(P, hdr, s, early) : launch<64>(P, hdr, s, early);
}

}  // namespace at
}  // namespace ckv
