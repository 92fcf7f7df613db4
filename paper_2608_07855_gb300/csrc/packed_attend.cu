// Attention over packed caches: entry points and the division of their work.
#include <math.h>
#include <string.h>

#include <algorithm>

#include "packed.cuh"

namespace ckv {
namespace pk {
namespace {

using at::kAlign;

// The same trajectories as the full-width calls' checks and sizes see them.
void as_trajs(const commitkv_shape *s, int n, const commitkv_packed *x, commitkv_traj *tr) {
  memset(tr, 0, n * sizeof *tr);
  for (int t = 0; t < n; ++t) {
    tr[t].k = x[t].k, tr[t].v = x[t].v;
    tr[t].stride_tok = s->head_dim;
    tr[t].pos = x[t].pos;
    tr[t].S = x[t].S;
    tr[t].q = x[t].q, tr[t].q_pos = x[t].q_pos;
    tr[t].W = x[t].W;
  }
}

commitkv_status check_call(const commitkv_shape *s, int n, const commitkv_packed *x, commitkv_traj *tr, bool queries) {
  commitkv_status st = check_shape(s);
  if (st) return st;
  if ((st = check_caches(s, n, x, true, queries))) return st;
  as_trajs(s, n, x, tr);
  return at::check_args(s, n, tr, nullptr, queries);
}

size_t compact_bytes(int n, const commitkv_packed *x) {
  size_t b = 0;
  for (int t = 0; t < n; ++t) b += at::align_up((size_t)x[t].S);
  return b;
}

// Many rows: the trajectories' values in full width, a layer of all of them, K
// before V, each [H][S][d] dense.
bool many(const commitkv_shape *s, const commitkv_packed &x) { return (int64_t)(s->q_heads / s->kv_heads) * x.W > 16; }
size_t full_bytes(const commitkv_shape *s, const commitkv_packed &x) {  // K or V
  return at::align_up((size_t)s->kv_heads * x.S * s->head_dim * (s->dtype == COMMITKV_BF16 ? 2 : 4));
}
size_t back_bytes(const commitkv_shape *s, int n, const commitkv_packed *x) {
  size_t b = 0;
  for (int t = 0; t < n; ++t)
    if (many(s, x[t])) b += 2 * full_bytes(s, x[t]);
  return b;
}

// Attention of the trajectories of more than 16 rows, layer by layer: the layer's
// values into the workspace, behind what the full-width call takes of it, then
// that call.
commitkv_status attend_many(const commitkv_shape *s, int n, const commitkv_packed *x, const uint8_t *mask, int32_t window,
                            int32_t sinks, void *const *out, float *const *lse_out, const bool *back, void *workspace,
                            size_t attention, cudaStream_t stream) {
  commitkv_packed c[kMaxTraj];
  commitkv_rows rows[kMaxTraj];
  commitkv_traj tr[kMaxTraj] = {};
  int32_t ids[kMaxTraj];
  int m = 0;
  char *at = static_cast<char *>(workspace) + attention;
  commitkv_shape one = *s;
  one.layers = 1;
  for (int t = 0; t < n; ++t) {
    if (!back[t]) continue;
    ids[m] = t;
    c[m] = x[t];
    rows[m] = {at, at + full_bytes(s, x[t]), 0, (int64_t)x[t].S * s->head_dim, s->head_dim, 0, x[t].S};
    at += 2 * full_bytes(s, x[t]);
    tr[m].k = rows[m].k, tr[m].v = rows[m].v;
    tr[m].stride_layer = rows[m].stride_head * s->kv_heads;
    tr[m].stride_head = rows[m].stride_head, tr[m].stride_tok = s->head_dim;
    tr[m].pos = x[t].pos, tr[m].S = x[t].S;
    tr[m].q_pos = x[t].q_pos, tr[m].W = x[t].W;
    ++m;
  }
  for (int l = 0; l < s->layers && m > 0; ++l) {
    if (mask && !mask[l]) continue;
    void *o[kMaxTraj];
    float *lse[kMaxTraj];
    const uint8_t layer = (uint8_t)l;
    for (int i = 0; i < m; ++i) {
      const commitkv_packed &y = x[ids[i]];
      const int64_t r = (int64_t)l * s->q_heads * y.W, eb = s->dtype == COMMITKV_BF16 ? 2 : 4;
      tr[i].q = static_cast<const char *>(y.q) + r * s->head_dim * eb;
      o[i] = static_cast<char *>(out[ids[i]]) + r * s->head_dim * eb;
      lse[i] = lse_out && lse_out[ids[i]] ? lse_out[ids[i]] + r : nullptr;
    }
    if (launch_read(s, m, c, rows, &layer, 1, stream) != cudaSuccess) return COMMITKV_ERR_CUDA;
    const commitkv_status st =
        at::attend(&one, m, tr, nullptr, nullptr, window, sinks, o, lse, workspace, attention, stream);
    if (st) return st;
  }
  return COMMITKV_OK;
}

// What trajectories of more than 16 rows take, of a call together: the kernel of
// 8- or 16-row items, which reads the codes again for every one of them, the
// kernel of row tiles on the codes, which writes their values to shared memory
// again for every 256 rows, or the values read back once.  Estimated times in us,
// fits to calls of these kinds (bf16, 8 KV heads of 128 channels, 4 query heads to one;
// 8 queries over 4,000 tokens 14.7, 18.9 and 20.9, 16 over 16,000 31, 27 and 39, 64
// over 16,000 93, 37 and 52, 256 over 16,000 307, 90 and 91, 1,024 over 16,000 1,101,
// 278 and 233, 31 of 12 layers over 32,768 896, 279 and 803; fp32, 4 KV heads, 100
// over 4,000 47 and, read back, 47, 300 over 4,000 93 and 85).
enum Many { kManyRows, kManyTiles, kManyBack };
Many many_path(const commitkv_shape *s, int n, const commitkv_packed *x, void *const *out, int n_layers, int window,
               int sinks, const at::Forced &f, int sms) {
  const bool bf16 = s->dtype == COMMITKV_BF16, wide128 = s->head_dim == 128;
  const double slices = (double)n_layers * s->kv_heads, full = s->head_dim * (bf16 ? 2 : 4);
  double rows = 10.0, tiles = 15.0, back = 22.0 + 4.0 * n_layers;
  bool fast = !f.cuda_cores && !f.full, aligned = true;
  for (int t = 0; t < n; ++t) {
    if (!many(s, x[t])) continue;
    const int64_t R = (int64_t)(s->q_heads / s->kv_heads) * x[t].W;
    fast = fast && wide(to_dev(x[t]), s->head_dim) && (uintptr_t)x[t].q % 16 == 0;
    aligned = aligned && (uintptr_t)out[t] % 16 == 0;
    const int64_t seen = std::min<int64_t>(x[t].S, window ? (int64_t)window + sinks + x[t].W : x[t].S);
    rows += 1e-6 * slices * seen *
            (bf16 ? at::cdiv(R, 16) * (wide128 ? 38.0 : 27.0) : at::cdiv(R, 8) * (wide128 ? 34.0 : 21.0));
    if (bf16) {
      const double tile = slices * at::cdiv(R, 256) * at::cdiv(seen, 128) / sms;
      tiles += tile * (R <= 128 ? (wide128 ? 1.6 : 1.2) : (wide128 ? 2.4 : 1.7));
      back += tile * (wide128 ? 1.75 : 1.3);
    } else {
      back += slices * at::cdiv(R, 128) * at::cdiv(seen, 64) / sms * (wide128 ? 2.7 : 1.8);
    }
    back += slices * x[t].S * (s->head_dim * 1.0625 + 4 * full) / 6.5e6;
  }
  const bool can_tile = bf16 && aligned;
  if (!fast) return kManyBack;
  if (f.tiles) return can_tile ? kManyTiles : kManyBack;
  if (rows <= back && (!can_tile || rows <= tiles)) return kManyRows;
  return can_tile && tiles <= back ? kManyTiles : kManyBack;
}

// Times of items, by which work is divided: those of the CUDA cores and of the row
// tiles from calls of one path (1,507 us and 306 for the cases at their kernels), of 8
// and 16 rows a tile of a block with the SM's others at work.
enum { kSimt16, kRows8, kRows16, kTc, kPaths };
constexpr at::PathInfo kPath[kPaths] = {
    {16, 64, 2, 1.0, 11.5}, {8, 128, 3, 2.0, 1.7}, {16, 128, 2, 2.0, 1.9}, {256, 128, 1, 2.0, 1.7}};

}  // namespace
}  // namespace pk
}  // namespace ckv

using namespace ckv;

extern "C" {

size_t commitkv_packed_workspace_size(const commitkv_shape *shape, int32_t n_traj, const commitkv_packed *trajs) {
  commitkv_traj tr[kMaxTraj];
  if (pk::check_call(shape, n_traj, trajs, tr, false) != COMMITKV_OK) return 0;
  return at::kAlign + std::max(at::partial_bytes(shape, at::partial_rows(shape, n_traj, tr, nullptr)) +
                                   pk::back_bytes(shape, n_traj, trajs),
                               pk::compact_bytes(n_traj, trajs));
}

commitkv_status commitkv_packed_attention(const commitkv_shape *shape, int32_t n_traj, const commitkv_packed *trajs,
                                          const uint8_t *layer_mask, int32_t window, int32_t sinks, void *const *out,
                                          float *const *lse_out, void *workspace, size_t workspace_bytes,
                                          cudaStream_t stream) {
  using namespace at;
  commitkv_traj tr[kMaxTraj];
  commitkv_status st = pk::check_call(shape, n_traj, trajs, tr, true);
  if (st) return st;
  if (window < 0 || sinks < 0 || !out) return COMMITKV_ERR_INVALID_ARG;
  for (int t = 0; t < n_traj; ++t)
    if (trajs[t].W > 0 && !out[t]) return COMMITKV_ERR_INVALID_ARG;
  const size_t attention = kAlign + partial_bytes(shape, partial_rows(shape, n_traj, tr, nullptr));
  if (!workspace || (uintptr_t)workspace % kAlign || workspace_bytes < attention + pk::back_bytes(shape, n_traj, trajs))
    return COMMITKV_ERR_WORKSPACE;

  static thread_local pk::Launch P;
  memset(&P, 0, sizeof P);
  Launch &L = P.L;
  L.M = shape->layers;
  L.H = shape->kv_heads;
  L.Hq = shape->q_heads;
  L.g = shape->q_heads / shape->kv_heads;
  L.d = shape->head_dim;
  L.dtype = shape->dtype;
  const float scale = shape->softmax_scale > 0.0f ? shape->softmax_scale : 1.0f / sqrtf((float)shape->head_dim);
  L.scale_log2 = scale * 1.4426950408889634f;
  L.window = window;
  L.sinks = sinks;
  for (int l = 0; l < shape->layers; ++l)
    if (!layer_mask || layer_mask[l]) L.layer_ids[L.n_layers++] = (uint8_t)l;
  L.n_traj = L.n_seg = n_traj;
  int64_t queries = 0;
  for (int t = 0; t < n_traj; ++t) queries += trajs[t].W;
  if (L.n_layers == 0 || queries == 0) return COMMITKV_OK;
  const int64_t slices = (int64_t)L.n_layers * L.H;
  bool big = false, back[kMaxTraj];
  int path[kMaxTraj];
  const Forced forced = forced_paths();
  const int sms = sm_count();
  if (sms < 1) return COMMITKV_ERR_CUDA;
  const pk::Many many = pk::many_path(shape, n_traj, trajs, out, L.n_layers, window, sinks, forced, sms);
  for (int t = 0; t < n_traj; ++t) {
    const commitkv_packed &x = trajs[t];
    const pk::Cache c = pk::to_dev(x);
    L.t[t] = {x.q, x.q_pos, out[t], lse_out ? lse_out[t] : nullptr, x.W, 0};
    Seg &sg = L.seg[t];
    sg.k = c.k, sg.v = c.v;
    sg.sl = c.sl, sg.sh = c.sh, sg.st = c.st;
    P.sc[t] = {c.ks, c.vs, c.gl, c.gh, c.gt};
    sg.pos = x.pos;
    sg.S = x.S;
    sg.t = t;
    back[t] = pk::many(shape, x) && many == pk::kManyBack;
    sg.R = back[t] ? 0 : L.g * x.W;
    big = big || back[t];
    const bool fast = !forced.cuda_cores && pk::wide(c, L.d) && (uintptr_t)x.q % 16 == 0;
    path[t] = sg.R > 16 && many == pk::kManyTiles ? pk::kTc : !fast ? pk::kSimt16 : sg.R <= 8 || L.dtype == COMMITKV_F32 ? pk::kRows8 : pk::kRows16;
  }
  for (int s = 0; s < n_traj; ++s) L.order[s] = (uint8_t)s;
  std::sort(L.order, L.order + n_traj,
            [&](int a, int b) { return L.seg[a].S != L.seg[b].S ? L.seg[a].S > L.seg[b].S : a < b; });
  int64_t split_left[2] = {kMaxSplitSmall, kMaxSplit};
  for (int p = 0; p < pk::kPaths; ++p) {
    const PathInfo &pi = pk::kPath[p];
    int64_t &left = split_left[pi.rows > 16];
    Divide v;
    int ids[kMaxTraj];
    v.n = 0;
    for (int k = 0; k < n_traj; ++k) {
      const int s = L.order[k];
      Seg &sg = L.seg[s];
      if (path[s] != p) continue;
      sg.nrt = (int32_t)cdiv(sg.R, pi.rows);
      v.base[v.n] = slices * sg.nrt;
      v.rows[v.n] = slices * sg.R;
      v.tiles[v.n] = sg.R > 0 ? cdiv(std::min<int64_t>(sg.S, most_seen(L, sg, pi.rows)), pi.tile) : 0;
      ids[v.n++] = s;
    }
    if (v.n == 0) continue;
    const Division dv = divide(v, pi, (int64_t)sms * pi.resident, left, slices, false);
    int64_t items = 0;
    for (int i = 0; i < v.n; ++i) {
      Seg &sg = L.seg[ids[i]];
      const bool rest = dv.rest >= 0 && v.base[i] > 0 && v.tiles[i] > 0;
      sg.nchunk = (int32_t)(rest ? dv.chunks : std::max<int64_t>(1, cdiv(v.tiles[i], dv.len)));
      sg.nsplit = (int32_t)(rest ? dv.rest : sg.nchunk > 1 ? sg.nrt : 0);
      left -= slices * sg.nsplit * sg.nchunk;
      sg.Rs = std::min(sg.R, sg.nsplit * pi.rows);
      items += slices * ((sg.nrt - sg.nsplit) + (int64_t)sg.nsplit * sg.nchunk);
      if (items > (1 << 30)) return COMMITKV_ERR_UNSUPPORTED;
    }
  }
  int64_t parts = 0;
  bool merge = false;
  for (int s = 0; s < n_traj; ++s) {
    Seg &sg = L.seg[s];
    sg.part = parts;
    parts += slices * sg.nchunk * sg.Rs;
    L.out_off[s + 1] = L.out_off[s] + sg.Rs * L.H;
    merge = merge || sg.Rs > 0;
  }
  if (kAlign + partial_bytes(shape, parts) > workspace_bytes) return COMMITKV_ERR_WORKSPACE;  // partial_rows bounds it
  char *base = static_cast<char *>(workspace) + kAlign;
  L.po = reinterpret_cast<float *>(base);
  L.pml = reinterpret_cast<float2 *>(base + align_up((size_t)parts * L.d * 4));
  cudaError_t e = cudaSuccess;
  bool launched = false;
  for (int p = 0; p < pk::kPaths && e == cudaSuccess; ++p) {
    int32_t items = 0;
    for (int k = 0; k < n_traj; ++k) {
      const int s = L.order[k];
      const Seg &sg = L.seg[s];
      L.item_off[k] = items;
      if (path[s] == p) items += (int32_t)(slices * (sg.nrt - sg.nsplit + sg.nsplit * sg.nchunk));
    }
    L.item_off[n_traj] = items;
    if (items == 0) continue;
    L.rows_per_item = pk::kPath[p].rows;
    e = p == pk::kTc       ? pk::launch_tc(P, static_cast<WsHeader *>(workspace), stream, launched)
        : p == pk::kSimt16 ? pk::launch_simt(P, stream, launched)
                           : pk::launch_rows(P, stream, launched);
    launched = true;
  }
  if (e == cudaSuccess && merge) e = launch_combine(L, stream);
  if (e == cudaSuccess)
    return big ? pk::attend_many(shape, n_traj, trajs, layer_mask, window, sinks, out, lse_out, back, workspace, attention, stream)
               : COMMITKV_OK;
  cudaGetLastError();
  return COMMITKV_ERR_CUDA;
}

}  // extern "C"
