// Attention over resident caches: entry points, work division, and the merge
// of partial results.
#include <math.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>

#include "attend.cuh"

namespace ckv {
namespace at {
namespace {

constexpr size_t kAlign = 256;
size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Items that share rows with others (split tokens), at most, of all kernels of
// a call that take up to 16 rows and of all others: bounds the partial
// results.  Small row tiles are cheap to merge and come from calls whose time
// is the reading of the cache, which wants many blocks.
constexpr int64_t kMaxSplitSmall = 2048;  // up to 16 rows an item
constexpr int64_t kMaxSplit = 768;

// ------------------------------------------------------------------ merge
// o = sum 2^(m_i - m) o_i / sum 2^(m_i - m) l_i over a row's partial results,
// those of the prefix first.  NW warps to a row take kBatch parts each at a
// time (no more registers than the call has parts, so that rows are in flight
// together too), all loads of a batch in flight together: the call's time here is
// latency (3.5 us for 16 parts of 32 rows).  A part
// whose sum of weights is zero takes part like any other: it is zero, or NaN
// where a token of score -inf has a value that is not finite.
template <typename T, int D, int NW, int kBatch>
__global__ void __launch_bounds__(128) combine(const __grid_constant__ Launch L) {
  constexpr int C = D / 32;  // channels of a lane: C lane ..
  __shared__ float so[NW > 1 ? NW : 1][D];
  __shared__ float2 sml[NW];
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  const int64_t w = NW == 1 ? (int64_t)blockIdx.x * 4 + warp : blockIdx.x;
  const int per = L.out_off[L.n_traj];
  const int li = (int)(w / per);
  if (li >= L.n_layers) return;
  int x = (int)(w % per), a = 0, b = L.n_traj;
  while (b - a > 1) {
    const int m = (a + b) >> 1;
    if (x >= L.out_off[m]) a = m;
    else b = m;
  }
  x -= L.out_off[a];
  const Traj &t = L.t[a];
  const Seg &own = L.seg[a + L.prefix], &pre = L.seg[0];
  const int R = own.Rs, kvh = x / R, r = x % R, l = L.layer_ids[li], slice = li * L.H + kvh;
  const int64_t first = own.part + (int64_t)slice * own.nchunk * own.Rs + r;
  const int64_t pfirst = pre.part + (int64_t)slice * pre.nchunk * pre.Rs + t.row0 + r;
  const int np = L.prefix ? pre.nchunk : 0, n = np + own.nchunk;
  pdl_wait();  // the parts are written
  float m = -INFINITY, lsum = 0.0f, o[C];
#pragma unroll
  for (int c = 0; c < C; ++c) o[c] = 0.0f;
  for (int p0 = NW == 1 ? 0 : warp; p0 < n; p0 += kBatch * NW) {
    float2 ml[kBatch];
    float y[kBatch][C];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int p = p0 + i * NW;
      ml[i] = make_float2(-INFINITY, 0.0f);
#pragma unroll
      for (int c = 0; c < C; ++c) y[i][c] = 0.0f;
      if (p < n) {
        const int64_t row = p < np ? pfirst + (int64_t)p * pre.Rs : first + (int64_t)(p - np) * own.Rs;
        ml[i] = L.pml[row];
        const float *src = L.po + row * D + C * lane;
        if constexpr (C == 4) {
          const float4 v = *reinterpret_cast<const float4 *>(src);
          y[i][0] = v.x, y[i][1] = v.y, y[i][2] = v.z, y[i][3] = v.w;
        } else {
          const float2 v = *reinterpret_cast<const float2 *>(src);
          y[i][0] = v.x, y[i][1] = v.y;
        }
      }
    }
    float mn = m;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) mn = fmaxf(mn, ml[i].x);
    const float ref = mn == -INFINITY ? 0.0f : mn, f = exp2f(m - ref);
    m = mn;
    lsum *= f;
#pragma unroll
    for (int c = 0; c < C; ++c) o[c] *= f;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const float wt = exp2f(ml[i].x - ref);
      lsum = fmaf(ml[i].y, wt, lsum);
#pragma unroll
      for (int c = 0; c < C; ++c) o[c] = fmaf(y[i][c], wt, o[c]);
    }
  }
  if constexpr (NW > 1) {
#pragma unroll
    for (int c = 0; c < C; ++c) so[warp][C * lane + c] = o[c];
    if (lane == 0) sml[warp] = make_float2(m, lsum);
    __syncthreads();
    if (warp) return;
#pragma unroll
    for (int i = 0; i < NW; ++i) m = fmaxf(m, sml[i].x);
    const float ref = m == -INFINITY ? 0.0f : m;
    lsum = 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c) o[c] = 0.0f;
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      const float wt = exp2f(sml[i].x - ref);
      lsum = fmaf(sml[i].y, wt, lsum);
#pragma unroll
      for (int c = 0; c < C; ++c) o[c] = fmaf(so[i][C * lane + c], wt, o[c]);
    }
  }
  const int64_t row = row_index(L, t, l, kvh, r);
  const float inv = norm_of(lsum);
  T *dst = static_cast<T *>(t.out) + row * D + C * lane;
#pragma unroll
  for (int c = 0; c < C; ++c) dst[c] = from_f32<T>(o[c] * inv);
  if (t.lse && lane == 0) t.lse[row] = lse_of(m, lsum);
}

template <typename T, int D>
cudaError_t launch_combine_td(const Launch &L, cudaStream_t s) {
  const int64_t rows = (int64_t)L.out_off[L.n_traj] * L.n_layers;
  int parts = 1;
  for (int t = 0; t < L.n_traj; ++t)
    parts = std::max(parts, L.seg[t + L.prefix].nchunk + (L.prefix ? L.seg[0].nchunk : 0));
  if (parts <= 2) return launch_after(combine<T, D, 1, 2>, (unsigned)cdiv(rows, 4), 128, 0, s, true, L);
  if (parts <= 8) return launch_after(combine<T, D, 1, 8>, (unsigned)cdiv(rows, 4), 128, 0, s, true, L);
  return launch_after(combine<T, D, 4, 8>, (unsigned)rows, 128, 0, s, true, L);
}

}  // namespace

cudaError_t launch_combine(const Launch &L, cudaStream_t s) {
  if (L.out_off[L.n_traj] == 0 || L.n_layers == 0) return cudaSuccess;
  if (L.dtype == COMMITKV_BF16)
    return L.d == 128 ? launch_combine_td<__nv_bfloat16, 128>(L, s) : launch_combine_td<__nv_bfloat16, 64>(L, s);
  return L.d == 128 ? launch_combine_td<float, 128>(L, s) : launch_combine_td<float, 64>(L, s);
}

namespace {

// ------------------------------------------------------------------ host
int64_t rows_of(const commitkv_shape *s, const commitkv_traj &x) { return (int64_t)(s->q_heads / s->kv_heads) * x.W; }

commitkv_status check_args(const commitkv_shape *s, int n, const commitkv_traj *tr, const commitkv_traj *prefix,
                           bool need_q) {
  commitkv_status st = check_shape(s);
  if (st) return st;
  if ((st = check_trajs(s, n, tr, need_q))) return st;
  if (prefix) {
    commitkv_traj p = *prefix;  // its queries and pages are not read
    p.W = p.P = 0;
    if ((st = check_trajs(s, 1, &p, false))) return st;
  }
  int64_t rows = 0;  // of one (layer, KV head): indices of a slice are 32-bit
  for (int t = 0; t < n; ++t) rows += rows_of(s, tr[t]);
  return rows * s->kv_heads > (1 << 28) ? COMMITKV_ERR_INVALID_ARG : COMMITKV_OK;
}

// Partial rows that a call can need; monotone in S, W and n_traj.
int64_t partial_rows(const commitkv_shape *s, int n, const commitkv_traj *tr, const commitkv_traj *prefix) {
  int64_t all = 0, most = 0;
  for (int t = 0; t < n; ++t) {
    all += rows_of(s, tr[t]);
    most = std::max(most, rows_of(s, tr[t]));
  }
  if (prefix) most = all;
  const int64_t split = kMaxSplitSmall * std::min<int64_t>(most, 16) + kMaxSplit * std::min<int64_t>(most, 256);
  return split + (prefix ? 2 * all * s->kv_heads * s->layers : 0);
}

size_t partial_bytes(const commitkv_shape *s, int64_t rows) {
  return align_up((size_t)rows * s->head_dim * 4) + align_up((size_t)rows * 8);
}

int sm_count() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return 0;
  return n;
}

// How the row tiles of a path's segments are divided: estimated time in us of
// `slots` concurrent items.  An item costs `fixed` tiles besides its own, a
// call with partial results another kernel (kMergeUs) and their rows'
// writing and reading back.  Estimates for this card at its clocks, which weigh
// chunk lengths against one another.  To take tile_us and fixed again: event
// times of calls of as many whole items as there are slots (152 slices of 256
// rows, say) at two lengths; the slope is a tile, the rest is fixed, the launch
// included.  Last so, for 128 channels: 256 rows of bf16 1.8 us, 128 of fp32 3.3,
// 16 of bf16 1.4 and of fp32 1.9, on the CUDA cores 11.5 and 17; kPath's values
// are of earlier calls.  Measured: a three-prompt batch of 84 row tiles of
// 9 token tiles, 64 channels, 49 us in two chunks each, 28 whole; one token over
// 4 caches of 4,096 tokens 15 us in chunks, 46 whole.
constexpr double kMergeUs = 3.5, kMergeRowUs = 0.25e-3, kBytesPerUs = 6.5e6;
struct PathInfo {
  int rows, tile;        // of an item, tokens of a tile
  int resident;          // items at a time on an SM
  double fixed, tile_us;
};
struct Divide {  // segments in the order of their items
  int64_t base[kMaxSeg];   // slices x row tiles
  int64_t tiles[kMaxSeg];  // of a row tile, at most
  int64_t rows[kMaxSeg];   // of all slices
  int n;
};
struct Division {
  int64_t len;  // every row tile in chunks of `len` tiles,
  int64_t rest, chunks;  // or, where rest >= 0, the last `rest` row tiles alone, in `chunks`
};
// When the last item ends, in tiles, where slots take items in their order as
// they get free: slots that get free at the same time are kept together.  (The
// work and half an item in its place: 8 prompts behind 32,768 tokens 788 us,
// 703 so; 5 of up to 200 rows over 16,000 134 and 119; 40 agents with 40 rows
// each behind 5,000 142 and 122.  Items of up to 16 rows share the memory's rate
// instead, so their sum is what counts.)
double last_end(const Divide &v, int64_t len, double fixed, int64_t slots) {
  double at[kMaxSeg + 2];  // ascending; a segment leaves one kind of slots more at most
  int64_t n[kMaxSeg + 2];
  int k = 1;
  at[0] = 0.0, n[0] = slots;
  for (int s = 0; s < v.n; ++s) {
    const int64_t c = std::max<int64_t>(1, cdiv(v.tiles[s], len));
    const double item = (double)v.tiles[s] / c + fixed;
    int64_t left = v.base[s] * c;
    const int64_t rounds = left / slots - 1;  // of every slot
    if (rounds > 0) {
      left -= rounds * slots;
      for (int i = 0; i < k; ++i) at[i] += rounds * item;
    }
    while (left > 0) {
      const int64_t m = std::min(left, n[0]);
      const double end = at[0] + item;
      left -= m;
      n[0] -= m;
      if (n[0] == 0) {
        --k;
        for (int i = 0; i < k; ++i) at[i] = at[i + 1], n[i] = n[i + 1];
      }
      int i = k;  // behind all that end before
      while (i > 0 && at[i - 1] > end) --i;
      if (i > 0 && at[i - 1] == end) {
        n[i - 1] += m;
        continue;
      }
      for (int j = k; j > i; --j) at[j] = at[j - 1], n[j] = n[j - 1];
      at[i] = end, n[i] = m;
      ++k;
    }
  }
  return at[k - 1];
}

Division divide(const Divide &v, const PathInfo &pi, int64_t slots, int64_t most_items, int64_t slices, bool prefix) {
  int64_t longest = 1, kinds = 0, kind = 0;
  for (int s = 0; s < v.n; ++s) {
    longest = std::max(longest, v.tiles[s]);
    if (v.base[s] > 0 && v.tiles[s] > 0) ++kinds, kind = s;
  }
  Division best = {longest, -1, 0};
  double best_t = INFINITY;
  for (int64_t k = 1, len = 0; k <= longest; ++k) {  // chunks of the longest cache
    if (len == cdiv(longest, k)) continue;
    len = cdiv(longest, k);
    int64_t items = 0, split = 0, parts = 0;
    double work = 0;
    for (int s = 0; s < v.n; ++s) {
      const int64_t c = std::max<int64_t>(1, cdiv(v.tiles[s], len));
      items += v.base[s] * c;
      if (c > 1) split += v.base[s] * c;
      if (c > 1 || prefix) parts += v.rows[s] * c;
      work += (double)v.base[s] * (v.tiles[s] + c * pi.fixed);
    }
    if (split > most_items) break;
    const double one = len + pi.fixed;
    double t = items <= slots ? one : kinds == 1 ? cdiv(items, slots) * one
               : pi.rows > 16     ? last_end(v, len, pi.fixed, slots)
                                  : work / slots + 0.5 * one;
    t = t * pi.tile_us + parts * kMergeRowUs + (split > 0 && !prefix ? kMergeUs : 0.0);
    if (t < best_t * 0.98) best_t = t, best.len = len;  // fewer chunks unless more are clearly better
  }
  // one segment that fills some waves: only what is left of the last one is cut
  const int64_t total = kinds == 1 && !prefix ? v.base[kind] : 0, waves = total / slots;
  if (waves > 0) {
    const int64_t rest = total / slices - waves * slots / slices;
    for (int64_t n = 2; rest > 0 && rest * slices * n <= most_items && n <= v.tiles[kind]; ++n) {
      const double t = (waves * (v.tiles[kind] + pi.fixed) +
                        cdiv(rest * slices * n, slots) * ((double)v.tiles[kind] / n + pi.fixed)) * pi.tile_us +
                       kMergeUs + rest * slices * pi.rows * n * kMergeRowUs;
      if (t < best_t * 0.98) best_t = t, best.rest = rest, best.chunks = n;
    }
  }
  return best;
}

enum { kSimt16, kSimt64, kTc, kTcF32, kRows, kPaths };
constexpr PathInfo kPath[kPaths] = {
    {16, 64, 2, 1.0, 2.5}, {64, 64, 2, 1.0, 17.0}, {256, 128, 1, 2.0, 1.6}, {128, 64, 1, 3.0, 2.7}, {16, 64, 2, 2.0, 1.4}};

// For tests and diagnosis, read in every call: COMMITKV_SCORING=simt takes the
// CUDA cores where a call could have the tensor cores (attention as well as
// scoring), COMMITKV_ATTENTION=tiles the kernels of row tiles however few rows
// there are.
struct Forced {
  bool cuda_cores, tiles;
};
Forced forced_paths() {
  const char *s = getenv("COMMITKV_SCORING"), *a = getenv("COMMITKV_ATTENTION");
  return {s && s[0] == 's', a && a[0] == 't'};
}

// Tensor cores where 16-byte copies can read the cache and the rows' queries
// and outputs: up to 16 rows the kernel of 16-row items, others those of row
// tiles (but see few_rows); TMA, which bf16 tiles take, also wants distinct
// heads and layers.
int path_of(const Launch &L, const Seg &sg, const Forced &f) {
  const int cuda_cores = sg.R <= 16 ? kSimt16 : kSimt64;
  if (f.cuda_cores) return cuda_cores;
  const int eb = L.dtype == COMMITKV_BF16 ? 2 : 4;
  uintptr_t bits = (uintptr_t)sg.k | (uintptr_t)sg.v | (uintptr_t)((sg.sl | sg.sh | sg.st) * eb);
  for (int t = sg.t < 0 ? 0 : sg.t; t < (sg.t < 0 ? L.n_traj : sg.t + 1); ++t)
    bits |= L.t[t].W ? (uintptr_t)L.t[t].q | (uintptr_t)L.t[t].out : 0;
  if (bits % 16) return cuda_cores;
  if (sg.R <= 16 && !f.tiles) return kRows;
  if (eb == 4) return kTcF32;
  if (sg.S > 0 && (sg.sh == 0 || sg.sl == 0 || std::max(sg.sl, std::max(sg.sh, sg.st)) >= (1ll << 39))) return kRows;
  return kTc;
}

// Tokens of a cache that a row tile needs, estimated: with a window its rows see
// `window` + `sinks` tokens each, their positions' span more.  No more than that
// where a trajectory's queries are consecutive, or lie behind all of a shared
// prefix (every window then ends at the prefix's end); queries in another order
// may need up to all S, which the kernels find for themselves.
int64_t most_seen(const Launch &L, const Seg &sg, int rows) {
  return L.window ? (int64_t)L.window + L.sinks + std::min(rows, sg.R) / L.g : sg.S;
}

// What of a path's costs goes by the type.
PathInfo path_info(const Launch &L, int p) {
  PathInfo pi = kPath[p];
  if (p == kRows) {
    pi.tile = rows_tile(L);
    if (L.dtype == COMMITKV_F32) pi.tile_us = 2.3;
  }
  if (p == kTcF32 && L.d == 64) pi.tile_us = 1.8;
  return pi;
}

// Whether the segments of more than 16 rows go to the kernel of 16-row items as
// well: it reads K and V again for every 16 rows, but has half the others'
// start and end.  Estimates in us; measured there and here, bf16, 32 query on 8
// KV heads of 128 channels (the constants here: fits to these calls, each run
// both ways, with COMMITKV_ATTENTION=tiles and without): 8 queries over 1,000 tokens 17.4 and 11.4, over
// 16,000 26.0 and 23.4, 16 over 4,000 18.5 and 17.1, 100 over 500 21.2 and
// 15.3, 8 agents behind 16,000 31.8 and 27.2; 5 over 16 caches to 16,000 127
// and 161, 12 over 16 to 1,000 23 and 31, 32 over 32,768 44 and 120.  fp32, 16
// on 4: 16 over 6,000 25 and 32, 32 over 2,000 21 and 25, 64 over 3,000 26 and
// 58, 8 over 8 caches to 4,000 42 and 47, 16 agents behind 4,000 25 and 30 (taken
// for the other way); 4 on 2: 40 over 1,000 19 and 15.
bool few_rows(const Launch &L, const int *path, int64_t slices, int sms) {
  const bool bf16 = L.dtype == COMMITKV_BF16;
  const PathInfo few_pi = path_info(L, kRows), many_pi = path_info(L, bf16 ? kTc : kTcF32);
  const double few_us = bf16 ? 1.25 : 2.3;
  double few = 0.0, many = bf16 ? 15.0 : 18.0, tiles = 0.0, bytes = 0.0, start = bf16 ? 7.0 : 9.0;
  for (int s = 0; s < L.n_seg; ++s) {
    const Seg &sg = L.seg[s];
    if (path[s] == kRows && sg.R > 0) start = 0.0;  // launched anyway
    if (path[s] != kTc && path[s] != kTcF32) continue;
    const int64_t seen = std::min<int64_t>(sg.S, most_seen(L, sg, many_pi.rows));
    few += few_us * slices * cdiv(sg.R, 16) * (cdiv(seen, few_pi.tile) + 1) / (2.0 * sms);
    tiles += (double)slices * cdiv(sg.R, many_pi.rows) * (cdiv(seen, many_pi.tile) + (bf16 ? 0 : 3));
    bytes += (double)slices * seen * L.d * (bf16 ? 4 : 8);
  }
  return start + few < many + std::max(bytes / kBytesPerUs, many_pi.tile_us * tiles / sms);
}

commitkv_status attend(const commitkv_shape *shape, int32_t n_traj, const commitkv_traj *trajs,
                       const commitkv_traj *prefix, const uint8_t *layer_mask, int32_t window, int32_t sinks,
                       void *const *out, float *const *lse_out, void *workspace, size_t workspace_bytes,
                       cudaStream_t stream) {
  commitkv_status st = check_args(shape, n_traj, trajs, prefix, true);
  if (st) return st;
  if (window < 0 || sinks < 0 || !out) return COMMITKV_ERR_INVALID_ARG;
  for (int t = 0; t < n_traj; ++t)
    if (trajs[t].W > 0 && !out[t]) return COMMITKV_ERR_INVALID_ARG;
  if (!workspace || (uintptr_t)workspace % kAlign ||
      workspace_bytes < kAlign + partial_bytes(shape, partial_rows(shape, n_traj, trajs, prefix)))
    return COMMITKV_ERR_WORKSPACE;
  if (prefix && prefix->S == 0) prefix = nullptr;

  static thread_local Launch L;
  memset(&L, 0, sizeof L);
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
  L.n_traj = n_traj;
  L.prefix = prefix ? 1 : 0;
  L.n_seg = n_traj + L.prefix;
  int64_t all = 0;
  for (int t = 0; t < n_traj; ++t) {
    const commitkv_traj &x = trajs[t];
    L.t[t] = {x.q, x.q_pos, out[t], lse_out ? lse_out[t] : nullptr, x.W, (int32_t)all};
    all += rows_of(shape, x);
  }
  if (all == 0 || L.n_layers == 0) return COMMITKV_OK;
  int64_t most = prefix ? all : 0;
  for (int s = 0; s < L.n_seg; ++s) {
    const bool shared = prefix && s == 0;
    const commitkv_traj &x = shared ? *prefix : trajs[s - L.prefix];
    Seg &sg = L.seg[s];
    sg.k = x.k;
    sg.v = x.v;
    sg.sl = x.stride_layer;
    sg.sh = x.stride_head;
    sg.st = x.stride_tok;
    sg.pos = x.pos;
    sg.S = x.S;
    sg.t = shared ? -1 : s - L.prefix;
    sg.R = (int32_t)(shared ? all : rows_of(shape, x));
    most = std::max<int64_t>(most, sg.R);
  }
  const int sms = sm_count();
  if (sms < 1) return COMMITKV_ERR_CUDA;
  // which kernel takes each segment's rows, and how its tokens are divided
  int path[kMaxSeg];
  int64_t parts = 0;
  bool merge = false;
  const int64_t slices = (int64_t)L.n_layers * L.H;
  const Forced forced = forced_paths();
  for (int s = 0; s < L.n_seg; ++s) path[s] = path_of(L, L.seg[s], forced);
  if (!forced.tiles && few_rows(L, path, slices, sms))
    for (int s = 0; s < L.n_seg; ++s) path[s] = path[s] == kTc || path[s] == kTcF32 ? kRows : path[s];
  double rows_us = 0.0;  // time of the decode kernel, which reads its caches at the memory's rate
  for (int s = 0; s < L.n_seg; ++s) {
    const Seg &sg = L.seg[s];
    if (path[s] == kRows && sg.R > 0)
      rows_us += (double)slices * std::min<int64_t>(sg.S, most_seen(L, sg, 16)) * L.d *
                 (L.dtype == COMMITKV_BF16 ? 4 : 8) / kBytesPerUs;
  }
  for (int s = 0; s < L.n_seg; ++s) L.order[s] = (uint8_t)s;
  std::sort(L.order, L.order + L.n_seg,
            [&](int a, int b) { return L.seg[a].S != L.seg[b].S ? L.seg[a].S > L.seg[b].S : a < b; });
  int64_t split_left[2] = {kMaxSplitSmall, kMaxSplit};
  for (int p = 0; p < kPaths; ++p) {
    const PathInfo pi = path_info(L, p);
    int64_t &left = split_left[pi.rows > 16];
    Divide v;
    int ids[kMaxSeg];
    v.n = 0;
    for (int k = 0; k < L.n_seg; ++k) {
      const int s = L.order[k];
      Seg &sg = L.seg[s];
      if (path[s] != p) continue;
      sg.nrt = (int32_t)cdiv(sg.R, pi.rows);
      v.base[v.n] = slices * sg.nrt;
      v.rows[v.n] = slices * sg.R;
      // a cache without queries has no items, however long
      v.tiles[v.n] = sg.R > 0 ? cdiv(std::min<int64_t>(sg.S, most_seen(L, sg, pi.rows)), pi.tile) : 0;
      ids[v.n++] = s;
    }
    if (v.n == 0) continue;
    int64_t slots = (int64_t)sms * pi.resident;
    // A prefix on the tensor cores beside decoded caches, which run at the same
    // time: as few blocks as finish with them, the others' SMs read the caches
    // (64 agents behind a 16K prefix, 2,048 tokens each at most: 99 us with the
    // prefix on all SMs first, 78 so).
    if ((p == kTc || p == kTcF32) && v.n == 1 && rows_us > 0.0)
      slots = std::min(slots, std::max<int64_t>(
                                  1, (int64_t)(v.base[0] * v.tiles[0] / std::max(1.0, rows_us / pi.tile_us - 2 * pi.fixed))));
    const Division dv = divide(v, pi, slots, left, slices, prefix != nullptr);
    int64_t items = 0;
    for (int i = 0; i < v.n; ++i) {
      Seg &sg = L.seg[ids[i]];
      const bool rest = dv.rest >= 0 && v.base[i] > 0 && v.tiles[i] > 0;
      sg.nchunk = (int32_t)(rest ? dv.chunks : std::max<int64_t>(1, cdiv(v.tiles[i], dv.len)));
      sg.nsplit = (int32_t)(rest ? dv.rest : sg.nchunk > 1 ? sg.nrt : 0);
      left -= slices * sg.nsplit * sg.nchunk;
      if (prefix) sg.nsplit = sg.nrt;  // two caches: all results are partial
      sg.Rs = std::min(sg.R, sg.nsplit * pi.rows);
      items += slices * ((sg.nrt - sg.nsplit) + (int64_t)sg.nsplit * sg.nchunk);
      if (items > (1 << 30)) return COMMITKV_ERR_UNSUPPORTED;
    }
  }
  for (int s = 0; s < L.n_seg; ++s) {
    Seg &sg = L.seg[s];
    sg.part = parts;
    parts += (int64_t)L.n_layers * L.H * sg.nchunk * sg.Rs;
    if (sg.t >= 0) L.out_off[sg.t + 1] = L.out_off[sg.t] + sg.Rs * L.H;
    merge = merge || sg.Rs > 0;
  }
  if (kAlign + partial_bytes(shape, parts) > workspace_bytes) return COMMITKV_ERR_WORKSPACE;  // partial_rows bounds it
  char *base = static_cast<char *>(workspace) + kAlign;
  L.po = reinterpret_cast<float *>(base);
  L.pml = reinterpret_cast<float2 *>(base + align_up((size_t)parts * L.d * 4));
  cudaError_t e = cudaSuccess;
  bool launched = false;
  for (int p = 0; p < kPaths && e == cudaSuccess; ++p) {
    int32_t items = 0;
    for (int k = 0; k < L.n_seg; ++k) {
      const int s = L.order[k];
      const Seg &sg = L.seg[s];
      L.item_off[k] = items;
      if (path[s] == p) items += L.n_layers * L.H * (sg.nrt - sg.nsplit + sg.nsplit * sg.nchunk);
    }
    L.item_off[L.n_seg] = items;
    if (items == 0) continue;
    L.rows_per_item = kPath[p].rows;
    WsHeader *hdr = static_cast<WsHeader *>(workspace);
    e = p == kRows    ? launch_rows(L, stream, launched)
        : p == kTc    ? launch_tc(L, hdr, stream, launched)
        : p == kTcF32 ? launch_tc_f32(L, hdr, stream, launched)
                      : launch_simt(L, stream, launched);
    launched = true;
  }
  if (e == cudaSuccess && merge) e = launch_combine(L, stream);
  if (e == cudaSuccess) return COMMITKV_OK;
  cudaGetLastError();
  return COMMITKV_ERR_CUDA;
}

}  // namespace
}  // namespace at
}  // namespace ckv

using namespace ckv;

extern "C" {

size_t commitkv_attention_workspace_size(const commitkv_shape *shape, int32_t n_traj, const commitkv_traj *trajs,
                                         const commitkv_traj *prefix) {
  if (at::check_args(shape, n_traj, trajs, prefix, false) != COMMITKV_OK) return 0;
  return at::kAlign + at::partial_bytes(shape, at::partial_rows(shape, n_traj, trajs, prefix));
}

commitkv_status commitkv_window_attention(const commitkv_shape *shape, int32_t n_traj, const commitkv_traj *trajs,
                                          const uint8_t *layer_mask, int32_t window, int32_t sinks, void *const *out,
                                          float *const *lse_out, void *workspace, size_t workspace_bytes,
                                          cudaStream_t stream) {
  return at::attend(shape, n_traj, trajs, nullptr, layer_mask, window, sinks, out, lse_out, workspace, workspace_bytes,
                    stream);
}

commitkv_status commitkv_prefix_attention(const commitkv_shape *shape, int32_t n_traj, const commitkv_traj *trajs,
                                          const commitkv_traj *prefix, const uint8_t *layer_mask, int32_t window,
                                          int32_t sinks, void *const *out, float *const *lse_out, void *workspace,
                                          size_t workspace_bytes, cudaStream_t stream) {
  if (!prefix) return COMMITKV_ERR_INVALID_ARG;
  return at::attend(shape, n_traj, trajs, prefix, layer_mask, window, sinks, out, lse_out, workspace, workspace_bytes,
                    stream);
}

}  // extern "C"
