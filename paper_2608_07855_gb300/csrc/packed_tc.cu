// Attention over packed caches on the tensor cores (bf16, many rows): the
// kernel's launch.  Codes are read and their values written to shared memory by
// eight warps of each block, for every row tile again.
#include "attend_tc_impl.cuh"

namespace ckv {
namespace at {
namespace {

template <int D>
cudaError_t launch(const PackedParams &P, WsHeader *hdr, cudaStream_t s, bool early) {
  const int smem = (int)sizeof(Smem<D>) + 1024;
  const cudaError_t e =
      cudaFuncSetAttribute(attend_tc<D, PackedParams>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  return launch_after(attend_tc<D, PackedParams>, P.L.item_off[P.L.n_seg], 640, smem, s, early, P, hdr);
}

}  // namespace
}  // namespace at

namespace pk {

cudaError_t launch_tc(const Launch &X, WsHeader *hdr, cudaStream_t s, bool early) {
  static thread_local at::PackedParams P;
  const at::Launch &L = X.L;
  P.L = L;
  memcpy(P.sc, X.sc, sizeof P.sc);
  P.has_q = L.n_traj <= at::kMaxQ && L.g <= at::BM && at::BM % L.g == 0;
  for (int k = 0; k < L.n_seg && P.has_q; ++k) {
    const int t = L.order[k];
    if (L.item_off[k] < L.item_off[k + 1] && !at::map_q(&P.q[t], L, L.t[t])) return cudaErrorInvalidValue;
  }
  return L.d == 128 ? at::launch<128>(P, hdr, s, early) : at::launch<64>(P, hdr, s, early);
}

}  // namespace pk
}  // namespace ckv
