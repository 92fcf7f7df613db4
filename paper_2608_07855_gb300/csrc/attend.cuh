// Attention of new tokens over resident caches (commitkv_window_attention,
// commitkv_prefix_attention): launch description and what its kernels share.
//
// A segment is one cache (a trajectory's own, or the prefix that all of them
// share) with the query rows that attend to it.  The rows of a (layer, KV
// head) slice of a segment are numbered position by position, the g query
// heads of a position side by side: row r of a trajectory is position r / g,
// head kvh g + r % g, so the rows of a tile see nearly the same tokens; the
// prefix's rows are those of all trajectories, one after another.  A row sees
// the tokens [0, se) and [lo, hi) of a cache: positions increase, so both the
// causal end and the window are found by search.
//
// A work item is (segment, layer, KV head, row tile, chunk).  The tokens that
// a row tile needs, [0, max se) and [min lo, max hi), are only known on the
// device: its tiles are shared out evenly among the tile's chunks there.
// Results of a row that has one item go to the outputs, else partial results
// to the workspace, merged by combine.
#pragma once

#include "ckv_internal.cuh"

namespace ckv {
namespace at {

constexpr int kMaxSeg = kMaxTraj + 1;
constexpr float kLn2 = 0.6931471805599453f;

struct Seg {
  const void *k, *v;
  int64_t sl, sh, st;  // strides in elements
  const int32_t *pos;
  int64_t part;  // first partial row
  int32_t S;
  int32_t R;        // rows of a (layer, KV head) slice
  int32_t t;        // trajectory, -1: the shared prefix
  int32_t nrt;      // row tiles
  int32_t nsplit;   // the first nsplit of them have partial results, of nchunk items each; the others one item
  int32_t nchunk;
  int32_t Rs;       // rows of the first nsplit tiles
};

struct Traj {
  const void *q;
  const int32_t *qpos;
  void *out;
  float *lse;
  int32_t W;
  int32_t row0;  // its first row in the prefix segment
};

struct Launch {
  Seg seg[kMaxSeg];
  Traj t[kMaxTraj];
  int32_t item_off[kMaxSeg + 1];  // first item of the segment at each place of the order
  uint8_t order[kMaxSeg];         // segments, the longest first, so that what starts last ends soon
  int32_t out_off[kMaxTraj + 1];  // rows of a (selected) layer that combine merges, prefix per trajectory
  int32_t n_seg, n_traj, prefix;  // prefix: segment 0 is shared
  int32_t M, H, Hq, g, d, dtype, n_layers;
  int32_t window, sinks;
  int32_t rows_per_item;
  float scale_log2;
  float *po;      // partial sums [rows][d], not normalised
  float2 *pml;    // their reference max (base 2) and sum of weights
  uint8_t layer_ids[kMaxLayers];
};

// The kernels of a call overlap where they can (programmatic launches): each
// lets the next one start once all of its own blocks have, the kernels of the
// segments do not depend on one another, and the merge waits for all of them:
// the last block of a kernel that started early ends after the kernel ahead of
// it (every block: those that are done would keep their places from the rest).
__device__ __forceinline__ void pdl_start_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

__device__ __forceinline__ void pdl_chain() {
  if (blockIdx.x == gridDim.x - 1) pdl_wait();
}

// Launches a kernel; `early`: it may start before the call's last kernel ends.
template <typename... A>
cudaError_t launch_after(void (*kernel)(A...), unsigned blocks, unsigned threads, size_t smem, cudaStream_t s, bool early,
                         const A &...args) {
  cudaLaunchConfig_t c = {};
  c.gridDim = dim3(blocks);
  c.blockDim = dim3(threads);
  c.dynamicSmemBytes = smem;
  c.stream = s;
  cudaLaunchAttribute a = {};
  a.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  a.val.programmaticStreamSerializationAllowed = 1;
  c.attrs = &a;
  c.numAttrs = early ? 1 : 0;
  void *p[] = {const_cast<void *>(static_cast<const void *>(&args))...};
  ++launch_count();
  return cudaLaunchKernelExC(&c, reinterpret_cast<const void *>(kernel), p);
}

// CUDA cores: any layout and type.  Rows per item: 16 or 64.
cudaError_t launch_simt(const Launch &L, cudaStream_t s, bool early);
// 16 rows per item, caches and queries 16-byte aligned; tiles of rows_tile tokens.
cudaError_t launch_rows(const Launch &L, cudaStream_t s, bool early);
inline int rows_tile(const Launch &L) { return 16384 / (L.d * (L.dtype == COMMITKV_BF16 ? 2 : 4)); }
// Tensor cores: bf16, caches and queries 16-byte aligned.  256 rows per item.
cudaError_t launch_tc(const Launch &L, WsHeader *hdr, cudaStream_t s, bool early);
// Tensor cores: fp32, caches, queries and outputs 16-byte aligned.  128 rows per item.
cudaError_t launch_tc_f32(const Launch &L, WsHeader *hdr, cudaStream_t s, bool early);
cudaError_t launch_combine(const Launch &L, cudaStream_t s);

struct Item {
  int s, li, l, kvh, rt, c;
  int n;       // chunks of its row tile
  bool split;  // results are partial
};

__device__ __forceinline__ Item decode_item(const Launch &L, int item) {
  Item it;
  int a = 0, b = L.n_seg;  // the last place that starts at or before the item
  while (b - a > 1) {
    const int m = (a + b) >> 1;
    if (item >= L.item_off[m]) a = m;
    else b = m;
  }
  it.s = L.order[a];
  const Seg &sg = L.seg[it.s];
  // the later rows of a prompt see more: they come first
  int x = item - L.item_off[a], rt = sg.nrt - 1;
  const int slices = L.H * L.n_layers, whole = slices * (sg.nrt - sg.nsplit);
  it.split = x >= whole;
  it.c = 0;
  it.n = 1;
  if (it.split) {
    x -= whole;
    it.n = sg.nchunk;
    it.c = x % sg.nchunk;
    x /= sg.nchunk;
    rt = sg.nsplit - 1;
  }
  it.rt = rt - x / slices;
  x %= slices;
  it.kvh = x % L.H;
  it.li = x / L.H;
  it.l = L.layer_ids[it.li];
  return it;
}

// Trajectory and row within it of row r of a segment.  The launch description
// is read by the constant cache, one address at a time, so the lanes' searches
// are kept short: with as many queries everywhere the first guess is right.
__device__ __forceinline__ int traj_of_row(const Launch &L, const Seg &sg, int &r) {
  if (sg.t >= 0) return sg.t;
  int a = (int)((int64_t)r * L.n_traj / sg.R), b = a + 1;
  if (r < L.t[a].row0) b = a, a = 0;
  else if (b < L.n_traj && r >= L.t[b].row0) a = b, b = L.n_traj;
  while (b - a > 1) {
    const int m = (a + b) >> 1;
    if (r >= L.t[m].row0) a = m;
    else b = m;
  }
  r -= L.t[a].row0;
  return a;
}

// Row (l, h, w) of a [M][Hq][W] array.
__device__ __forceinline__ int64_t row_index(const Launch &L, const Traj &t, int l, int kvh, int r) {
  return ((int64_t)l * L.Hq + kvh * L.g + r % L.g) * t.W + r / L.g;
}

__device__ __forceinline__ int64_t part_index(const Launch &L, const Seg &sg, const Item &it, int r) {
  return sg.part + ((int64_t)(it.li * L.H + it.kvh) * sg.nchunk + it.c) * sg.Rs + r;
}

// First index of [a, b) whose position is above x (b: none).
__device__ __forceinline__ int first_above(const int32_t *pos, int a, int b, int64_t x) {
  while (a < b) {
    const int m = a + ((b - a) >> 1);
    if ((int64_t)pos[m] > x) b = m;
    else a = m + 1;
  }
  return a;
}

struct Span {
  int lo, hi, se;  // a row sees [0, se) and [lo, hi), se <= lo
};

__device__ __forceinline__ bool sees(const Span &s, int i) { return i < s.se || (i >= s.lo && i < s.hi); }

// What a query at position p sees of a cache.  Positions increase by one or
// more, so a window holds at most `window` tokens and the sinks are at most
// the first `sinks`: without gaps (the latest tokens, or a cache before its
// first checkpoint) the first guess is right and costs a round trip or two
// instead of a search.
__device__ __forceinline__ Span row_span(const int32_t *pos, int S, int p, int window, int sinks) {
  Span r = {0, 0, 0};
  if (S == 0) return r;
  const int64_t back = (int64_t)pos[S - 1] - p;  // >= the number of tokens after p
  if (back <= 0) r.hi = S;
  else {
    const int64_t gss = (int64_t)S - back;  // the end if they have no gaps, else before it
    if (gss >= 1 && pos[gss - 1] == p) r.hi = (int)gss;
    else r.hi = first_above(pos, gss > 0 ? (int)gss : 0, S, p);
  }
  if (window == 0) return r;
  const int64_t edge = (int64_t)p - window;  // positions above it are inside
  const int least = r.hi > window ? r.hi - window : 0;
  r.lo = least;
  if (least < r.hi && (int64_t)pos[least] <= edge) r.lo = first_above(pos, least + 1, r.hi, edge);
  const int most = sinks < r.lo ? sinks : r.lo;
  r.se = most;
  if (most > 0 && pos[most - 1] >= sinks) r.se = first_above(pos, 0, most, (int64_t)sinks - 1);
  return r;
}

// The tokens of a row tile, cut into tiles of `tile`: [0, se), then [lo, hi).
struct Tiles {
  int lo, hi, se, nA, n;  // nA tiles of sinks, n in all
};

__device__ __forceinline__ Tiles make_tiles(int lo, int hi, int se, int tile) {
  Tiles t;
  if (hi <= lo) lo = 0, hi = se, se = 0;  // sinks alone
  else if (se >= lo) hi = max(hi, se), lo = se = 0;  // one piece
  t.lo = lo, t.hi = hi, t.se = se;
  t.nA = (se + tile - 1) / tile;
  t.n = t.nA + (hi - lo + tile - 1) / tile;
  return t;
}
__device__ __forceinline__ int tile_start(const Tiles &t, int j, int tile) {
  return j < t.nA ? j * tile : t.lo + (j - t.nA) * tile;
}
__device__ __forceinline__ int tile_end(const Tiles &t, int j, int tile) {
  const int e = tile_start(t, j, tile) + tile, lim = j < t.nA ? t.se : t.hi;
  return e < lim ? e : lim;
}
// Tiles [chunk_tile(c), chunk_tile(c + 1)) are chunk c's of n (n^2 fits 32 bits).
__device__ __forceinline__ int chunk_tile(const Tiles &t, int c, int n) {
  return t.n / n * c + t.n % n * c / n;
}

// Score of a token against a query, both read by one thread, 16 bytes at a
// time where they can be.
template <typename T, int D>
__device__ __forceinline__ float score_of(const T *q, const T *ki) {
  constexpr int E = 16 / sizeof(T);
  float dot = 0.0f;
  if ((((uintptr_t)q | (uintptr_t)ki) & 15) == 0) {
#pragma unroll 4
    for (int c = 0; c < D; c += E) {
      const uint4 a = *reinterpret_cast<const uint4 *>(q + c), b = *reinterpret_cast<const uint4 *>(ki + c);
      const T *x = reinterpret_cast<const T *>(&a), *y = reinterpret_cast<const T *>(&b);
#pragma unroll
      for (int e = 0; e < E; ++e) dot = fmaf(to_f32(x[e]), to_f32(y[e]), dot);
    }
  } else {
#pragma unroll 16
    for (int c = 0; c < D; ++c) dot = fmaf(to_f32(q[c]), to_f32(ki[c]), dot);
  }
  return dot;
}

// The tile kernels take a weight as exp2 of the fused s scale - m, where m is the
// rounded product for the largest s: up to half a step of m apart, the same
// factor in all weights of the row (the product is __fmul_rn, so that no
// difference of two references is fused with it).  Beyond |m| = 2^26 (half a step of 2) it
// could pass the exponent's range, so such a row is done over with the product
// rounded as m was.
constexpr float kFar = 67108864.0f;
__device__ __forceinline__ bool is_far(float m) { return fabsf(m) > kFar && fabsf(m) < INFINITY; }

// sum of exp2(s - m) v and of exp2(s - m) over the visible tokens of tiles
// [j0, j1) for one row, by the 32 lanes of a warp: o[k] is channel lane + 32 k.
// A masked token's values have no part in it.  The tile kernels multiply masked
// tokens by weights of zero, which is wrong where a masked value is infinite or
// NaN, so they redo a row whose sums are not finite this way (its m and l never
// see masked tokens).  32 tokens at a time, a lane each for the scores.  Once the
// row is NaN in every channel its values are not read any more; the sum of its
// weights, where the caller wants it, is of all visible tokens all the same.
// `fused`: the weights are as the caller's own and other parts' sums have them,
// with the fused product (see is_far), not the one that m is.
template <typename T, int D>
__device__ __noinline__ float redo_row(const Launch &L, const Seg &sg, int l, int kvh, const void *qrow, Span sp,
                                       Tiles tl, int tile, int j0, int j1, float m, float *o, bool want_sum, bool fused) {
  const int lane = threadIdx.x & 31;
  const T *q = static_cast<const T *>(qrow);
  const T *k = static_cast<const T *>(sg.k) + (int64_t)l * sg.sl + (int64_t)kvh * sg.sh;
  const T *v = static_cast<const T *>(sg.v) + (int64_t)l * sg.sl + (int64_t)kvh * sg.sh;
  float lsum = 0.0f;
  bool gone = false;
#pragma unroll
  for (int c = 0; c < D / 32; ++c) o[c] = 0.0f;
  for (int j = j0; j < j1; ++j) {
    const int a = tile_start(tl, j, tile), e = tile_end(tl, j, tile);
    for (int i0 = a; i0 < e; i0 += 32) {
      const int i = i0 + lane;
      const bool in = i < e && sees(sp, i);
      float p = 0.0f;
      if (in) {
        const float s = score_of<T, D>(q, k + (int64_t)i * sg.st);
        p = exp2f(fused ? fmaf(s, L.scale_log2, -m) : __fmul_rn(s, L.scale_log2) - m);
      }
      lsum += p;
      if (gone) continue;
      const unsigned seen = __ballot_sync(0xffffffffu, in);
#pragma unroll 8
      for (int u = 0; u < 32; ++u) {
        const float pu = __shfl_sync(0xffffffffu, p, u);
        if (!(seen >> u & 1)) continue;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) o[c] = fmaf(pu, to_f32(v[(int64_t)(i0 + u) * sg.st + lane + 32 * c]), o[c]);
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

// The largest visible score of a row in base 2, NaN if one is NaN or +inf.
template <typename T, int D>
__device__ __noinline__ float redo_max(const Launch &L, const Seg &sg, int l, int kvh, const void *qrow, Span sp,
                                       Tiles tl, int tile, int j0, int j1) {
  const T *k = static_cast<const T *>(sg.k) + (int64_t)l * sg.sl + (int64_t)kvh * sg.sh;
  float top = -INFINITY;
  bool bad = false;
  for (int j = j0; j < j1; ++j) {
    const int e = tile_end(tl, j, tile);
    for (int i = tile_start(tl, j, tile) + (threadIdx.x & 31); i < e; i += 32) {
      if (!sees(sp, i)) continue;
      const float s = __fmul_rn(score_of<T, D>(static_cast<const T *>(qrow), k + (int64_t)i * sg.st), L.scale_log2);
      bad = bad || isnan(s) || s == INFINITY;
      top = fmaxf(top, s);
    }
    if (__any_sync(0xffffffffu, bad)) return NAN;
  }
  return warp_max(top);
}

template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16(x); }

// Log-sum-exp of a row from its reference max (base 2) and sum; -inf where it saw nothing.
__device__ __forceinline__ float lse_of(float m, float l) { return fmaf(m, kLn2, logf(l)); }
// What its sums are multiplied by: 0 for a row that saw nothing.
__device__ __forceinline__ float norm_of(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }

// Writes one row's sums (relative to m, base 2; channel lane + 32 k in o[k])
// as a warp: a partial result, or the outputs.
template <typename T, int D>
__device__ __forceinline__ void write_row_warp(const Launch &L, const Seg &sg, const Item &it, int r, const float *o,
                                               float m, float l) {
  const int lane = threadIdx.x & 31;
  if (it.split) {
    const int64_t pr = part_index(L, sg, it, r);
#pragma unroll
    for (int c = 0; c < D / 32; ++c) L.po[pr * D + lane + 32 * c] = o[c];
    if (lane == 0) L.pml[pr] = make_float2(m, l);
  } else {
    const Traj &t = L.t[traj_of_row(L, sg, r)];
    const int64_t row = row_index(L, t, it.l, it.kvh, r);
    const float inv = norm_of(l);
    T *dst = static_cast<T *>(t.out) + row * D;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) dst[lane + 32 * c] = from_f32<T>(o[c] * inv);
    if (t.lse && lane == 0) t.lse[row] = lse_of(m, l);
  }
}

}  // namespace at
}  // namespace ckv
