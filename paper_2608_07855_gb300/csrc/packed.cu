// Packed caches: writing rows as codes and scales, reading them back, and the
// gather of a checkpoint.
//
// All three move bytes.  A thread has 32 channels where codes move whole (write,
// gather: 16 bytes of codes and their scale byte), and 8 where full-width rows are
// written (read: 16 bytes of bf16), so that stores are whole lines.
#include <string.h>

#include <algorithm>

#include "packed.cuh"

namespace ckv {
namespace pk {
namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;  // rows of a thread that reads codes, loads in flight together

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct Rows {
  Cache c;
  void *k, *v;
  int64_t sl, sh, st;  // in elements
  int32_t first, count;
  int32_t blocks;  // of a slice
};

struct CopyLaunch {
  Rows r[kMaxTraj];
  int32_t off[kMaxTraj + 1];  // first block of a trajectory
  int32_t n_traj, H;
  uint8_t layer_ids[kMaxLayers];
};
static_assert(sizeof(CopyLaunch) <= 32764, "kernel parameters");

// A block's rows: tokens i0 .. of one (layer, KV head) of a trajectory, a head
// after the other for the same tokens, so that rows that lie side by side in a
// token-by-token layout are taken at the same time.  The thread's first row and
// its channels' place in it; a step further is RB rows.
template <int D, int CH, int UN>
struct Place {
  static constexpr int TR = D / CH, RB = kThreads / TR;  // threads of a row, rows of a step
  const Rows &r;
  int i, c;  // row, first channel
  int64_t code, scale, elem;
  __device__ __forceinline__ Place(const CopyLaunch &L, const Rows &r_, int b) : r(r_) {
    const int l = L.layer_ids[b / L.H / r.blocks], h = b % L.H, i0 = b / L.H % r.blocks * (RB * UN);
    i = i0 + (int)threadIdx.x / TR;
    c = threadIdx.x % TR * CH;
    const int64_t tok = (int64_t)r.first + i;
    code = l * r.c.sl + h * r.c.sh + tok * r.c.st + c / 2;
    scale = l * r.c.gl + h * r.c.gh + tok * r.c.gt + c / kGroup;
    elem = l * r.sl + h * r.sh + i * r.st + c;
  }
};
__device__ __forceinline__ int traj_of_block(const CopyLaunch &L) {
  int t = 0, e = L.n_traj;
  while (e - t > 1) {
    const int m = (t + e) >> 1;
    if ((int)blockIdx.x >= L.off[m]) t = m;
    else e = m;
  }
  return t;
}

// 32 channels of a row, as they are in memory.
template <typename T>
struct Group {
  static constexpr int kWords = 8 * sizeof(T);
  uint32_t w[kWords];
  __device__ __forceinline__ float get(int i) const {
    if (sizeof(T) == 4) return __uint_as_float(w[i]);
    return __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  }
};
template <typename T, bool VEC>
__device__ __forceinline__ Group<T> load_group(const T *src) {
  Group<T> x;
  if (VEC) {
#pragma unroll
    for (int k = 0; k < x.kWords / 4; ++k) {
      const uint4 v = reinterpret_cast<const uint4 *>(src)[k];
      x.w[4 * k] = v.x, x.w[4 * k + 1] = v.y, x.w[4 * k + 2] = v.z, x.w[4 * k + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < x.kWords; ++i) {
      if (sizeof(T) == 4) x.w[i] = reinterpret_cast<const uint32_t *>(src)[i];
      else
        x.w[i] = reinterpret_cast<const uint16_t *>(src)[2 * i] |
                 (uint32_t)reinterpret_cast<const uint16_t *>(src)[2 * i + 1] << 16;
    }
  }
  return x;
}
// The largest magnitude, as an fp32 number's bits (from 0x7f800000 on: not finite).
template <typename T>
__device__ __forceinline__ uint32_t top_of(const Group<T> &x) {
  constexpr uint32_t abs = sizeof(T) == 4 ? 0x7fffffffu : 0x7fff7fffu;
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < x.kWords; i += 2) {
    if (sizeof(T) == 4) m = max(max(m, x.w[i] & abs), x.w[i + 1] & abs);
    else m = __vimax3_u16x2(m, x.w[i] & abs, x.w[i + 1] & abs);
  }
  return sizeof(T) == 4 ? m : max(m << 16, m & 0xffff0000u);
}

// sigma's byte for a largest magnitude a (finite): the one nearest to a / 7, of
// two the even.  An estimate rounded down, then one exact comparison: the middle
// between two neighbours has five significant bits, seven times it eight.
__device__ __forceinline__ unsigned scale_byte(float a) {
  const unsigned b =
      min(__half_as_ushort(__float2half_rz(__fmul_rn(__fmul_rn(a, 1.0f / 7.0f), 1.0f / kUnit))) >> 7, kNanScale - 1);
  const float mid = __half2float(__ushort_as_half((unsigned short)((b << 7) | 64u))) * (7.0f * kUnit);
  return b + (b < kNanScale - 1 && (a > mid || (a == mid && (b & 1))) ? 1u : 0u);
}

// The code of x for sigma > 0, inv near its inverse, whatever x.  The product can
// only be on the wrong side of a middle by rounding; the remainder is exact (a
// multiple of x's last place, no larger than x) and says on which side x is, or
// that it is a tie.
__device__ __forceinline__ unsigned code_of(float x, float sigma, float inv) {
  const float a = fabsf(x);
  float n = fminf(rintf(a * inv), 8.0f);
  const float r = fmaf(-n, sigma, a), t = 2.0f * fabsf(r);
  if (t > sigma || (t == sigma && ((int)n & 1))) n += r > 0.0f ? 1.0f : -1.0f;
  const int i = min((int)n, 7);
  return 8 + (x < 0.0f ? -i : i);
}

// The scale byte of 32 channels, and their codes.  x / sigma lies between x low and
// x high, the neighbours of 1 / sigma; both products rounded to whole numbers (by
// adding 3 2^22, one rounding) agree unless a middle lies between them, as it does
// for a tie.  A bf16 number there is the middle itself (its distance to a middle is
// 0 or 2^-8 of it and more), so the even one of the two is right; an fp32 number
// is looked at again.
template <typename T>
__device__ __forceinline__ unsigned encode(const Group<T> &x, uint32_t (&codes)[4]) {
  const unsigned top = top_of(x), b = top < 0x7f800000u ? scale_byte(__uint_as_float(top)) : 0;
  if (b == 0) {
    codes[0] = codes[1] = codes[2] = codes[3] = 0x88888888u;
    return top < 0x7f800000u ? 0 : 0xff;  // infinite or NaN
  }
  const float sigma = __half2float(__ushort_as_half((unsigned short)(b << 7))) * kUnit;
  float inv;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(sigma));
  const float e = fmaf(-sigma, inv, 1.0f);  // 0: exact
  const float low = e < 0.0f ? __uint_as_float(__float_as_uint(inv) - 1) : inv;
  const float high = e > 0.0f ? __uint_as_float(__float_as_uint(inv) + 1) : inv;
  bool again = b < 8 || b == kNanScale - 1;  // x may be more than 7.5 sigma
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 8 * k + 7; i >= 8 * k; --i) {
      // the bits of 3 2^22 + n: even as n is, and the digits of their sum need no masks
      const int n = __float_as_int(fmaf(x.get(i), low, 12582912.0f)), d = __float_as_int(fmaf(x.get(i), high, 12582912.0f)) - n;
      if (sizeof(T) == 4) again = again || d != 0;
      w = w * 16 + (sizeof(T) == 4 ? n : n + (n & 1) * d);
    }
    codes[k] = w + (0x88888888u - 0x11111111u * 0x4b400000u);  // every digit is 8 + n
  }
  if (again) {
#pragma unroll
    for (int k = 0; k < 4; ++k) codes[k] = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) codes[i / 8] |= code_of(x.get(i), sigma, inv) << (4 * (i % 8));
  }
  return b;
}

template <bool VEC>
__device__ __forceinline__ void store_codes(uint8_t *dst, const uint32_t (&codes)[4]) {
  if (VEC) *reinterpret_cast<uint4 *>(dst) = make_uint4(codes[0], codes[1], codes[2], codes[3]);
  else
#pragma unroll
    for (int i = 0; i < 16; ++i) dst[i] = (uint8_t)(codes[i / 4] >> (8 * (i % 4)));
}

// Write: bound by reading the rows (2.5 bytes a value of bf16 with its codes; 4.5 of
// fp32); a lane's loads of K's and V's rows are both issued first.  4,096 bf16 tokens of
// 36 layers, 8 KV heads of 128 channels: 117 us, 6.4 TB/s; its 11 instructions a value
// keep three of four issue slots busy.  fp32 256 us, 5.3 TB/s.
template <typename T, int D, bool VEC>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 4 : 2) write_kernel(const __grid_constant__ CopyLaunch L) {
  const int t = traj_of_block(L);
  const Rows &r = L.r[t];
  const Place<D, kGroup, 1> p(L, r, blockIdx.x - L.off[t]);
  if (p.i >= r.count) return;
  Group<T> x[2];
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) x[kv] = load_group<T, VEC>(static_cast<const T *>(kv ? r.v : r.k) + p.elem);
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    uint32_t w[4];
    (kv ? r.c.vs : r.c.ks)[p.scale] = (uint8_t)encode(x[kv], w);
    store_codes<VEC>((kv ? r.c.v : r.c.k) + p.code, w);
  }
}

// Read: bound by writing the rows: 36,896 tokens of 12 layers 340 us, 4,096 of 36 layers
// 112, the copy rate; fp32 267, 5.1 TB/s.
template <typename T, int D, bool VEC>
__global__ void __launch_bounds__(kThreads) read_kernel(const __grid_constant__ CopyLaunch L) {
  const int t = traj_of_block(L);
  const Rows &r = L.r[t];
  const Place<D, 8, kUnroll> p(L, r, blockIdx.x - L.off[t]);
  uint32_t w[2][kUnroll];
  uint8_t s[2][kUnroll];
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    const uint8_t *codes = (kv ? r.c.v : r.c.k) + p.code, *scales = (kv ? r.c.vs : r.c.ks) + p.scale;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u, codes += p.RB * r.c.st, scales += p.RB * r.c.gt) {
      if (p.i + u * p.RB >= r.count) continue;
      s[kv][u] = *scales;
      if (VEC) {
        w[kv][u] = *reinterpret_cast<const uint32_t *>(codes);
      } else {
        w[kv][u] = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[kv][u] |= (uint32_t)codes[i] << (8 * i);
      }
    }
  }
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    T *dst = static_cast<T *>(kv ? r.v : r.k) + p.elem;
#pragma unroll
    for (int u = 0; u < kUnroll; ++u, dst += p.RB * r.st) {
      if (p.i + u * p.RB >= r.count) continue;
      uint32_t x[4];
      values8(w[kv][u], bf_scale(s[kv][u]), x);
      if constexpr (VEC && sizeof(T) == 2) {
        *reinterpret_cast<uint4 *>(dst) = make_uint4(x[0], x[1], x[2], x[3]);
      } else if constexpr (VEC) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
          reinterpret_cast<uint4 *>(dst)[i] =
              make_uint4(x[2 * i] << 16, x[2 * i] & 0xffff0000u, x[2 * i + 1] << 16, x[2 * i + 1] & 0xffff0000u);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          dst[i] = at::from_f32<T>(__uint_as_float(i % 2 ? x[i / 2] & 0xffff0000u : x[i / 2] << 16));
      }
    }
  }
}

// ------------------------------------------------------------------ checkpoint
struct GatherLaunch {
  Cache src[kMaxTraj], dst[kMaxTraj];
  const int32_t *idx[kMaxTraj];
  const int32_t *pos[kMaxTraj];
  int32_t *pos_out[kMaxTraj];
  const int32_t *n_idx;
  int32_t H, group_bits;  // 1 << group_bits groups of 32 channels in a row
};
static_assert(sizeof(GatherLaunch) <= 32764, "kernel parameters");

// 32 channels: codes and scale byte.  Retained rows lie apart, and a row of 128 channels
// is half a line: 64 bytes are asked for, where a load by itself brings the row beside
// it too (384 MB of 36,896 tokens' rows and scale bytes instead of 600).
struct Unit {
  uint4 codes;
  uint8_t scale;
};
template <bool VEC>
__device__ __forceinline__ Unit load_unit(const uint8_t *codes, const uint8_t *scale) {
  Unit x;
  if (VEC) {
    asm volatile("ld.global.L2::64B.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(x.codes.x), "=r"(x.codes.y), "=r"(x.codes.z), "=r"(x.codes.w)
                 : "l"(codes)
                 : "memory");
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = codes[4 * i] | codes[4 * i + 1] << 8 | codes[4 * i + 2] << 16 | (uint32_t)codes[4 * i + 3] << 24;
    x.codes = make_uint4(w[0], w[1], w[2], w[3]);
  }
  x.scale = *scale;
  return x;
}
template <bool VEC>
__device__ __forceinline__ void store_unit(uint8_t *codes, uint8_t *scale, const Unit &x) {
  if (VEC) {
    *reinterpret_cast<uint4 *>(codes) = x.codes;
  } else {
    const uint32_t w[4] = {x.codes.x, x.codes.y, x.codes.z, x.codes.w};
#pragma unroll
    for (int i = 0; i < 16; ++i) codes[i] = (uint8_t)(w[i / 4] >> (8 * (i % 4)));
  }
  *scale = x.scale;
}

// Into other caches: blockIdx.y = 2 (l H + h) + (V), a thread kUnroll units, whose indices
// are read together, then their rows.  Bound by memory: 36,896 tokens of 36 layers, 8 KV
// heads of 128 channels to 8,192, 100 us (660 MB: 6.6 TB/s; with a division for every row
// and lines of 128 bytes 143).
template <bool VEC>
__global__ void __launch_bounds__(kThreads) gather_kernel(const __grid_constant__ GatherLaunch L) {
  const int t = blockIdx.z, kv = blockIdx.y & 1, l = (blockIdx.y >> 1) / L.H, h = (blockIdx.y >> 1) % L.H;
  const Cache &s = L.src[t], &d = L.dst[t];
  const int n = L.n_idx[t], gb = L.group_bits, g = threadIdx.x & ((1 << gb) - 1);
  const int32_t *idx = L.idx[t];
  const int64_t sc = l * s.sl + h * s.sh, sg = l * s.gl + h * s.gh, dc = l * d.sl + h * d.sh, dg = l * d.gl + h * d.gh;
  const uint8_t *codes = (kv ? s.v : s.k) + sc + 16 * g, *scales = (kv ? s.vs : s.ks) + sg + g;
  uint8_t *to = (kv ? d.v : d.k) + dc + 16 * g, *to_scales = (kv ? d.vs : d.ks) + dg + g;
  const unsigned step = kThreads >> gb, row0 = blockIdx.x * (kUnroll * step) + (threadIdx.x >> gb);
  Unit x[kUnroll];
  int i[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) i[u] = row0 + u * step < (unsigned)n ? idx[row0 + u * step] : -1;
#pragma unroll
  for (int u = 0; u < kUnroll; ++u)
    if (i[u] >= 0) x[u] = load_unit<VEC>(codes + i[u] * s.st, scales + i[u] * s.gt);
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    if (i[u] < 0) continue;
    const int64_t row = row0 + u * step;
    store_unit<VEC>(to + row * d.st, to_scales + row * d.gt, x[u]);
    if (blockIdx.y == 0 && g == 0 && L.pos_out[t]) L.pos_out[t][row] = L.pos[t][i[u]];
  }
}

// In place: a block per slice, chunk by chunk; a chunk's rows are all read
// before any is written, and later chunks' sources lie behind all that was
// written (I_j increases, I_j >= j).  36,896 tokens of 36 layers, 8 KV heads of 128 channels
// to 8,192: 143 us, where the kernel above takes 100: bound by the latency of two dependent
// loads and a barrier a chunk, with all of a slice in one block.
template <bool VEC>
__global__ void __launch_bounds__(kThreads) gather_in_place_kernel(const __grid_constant__ GatherLaunch L) {
  const int t = blockIdx.z, kv = blockIdx.y & 1, l = (blockIdx.y >> 1) / L.H, h = (blockIdx.y >> 1) % L.H;
  const Cache &s = L.src[t];
  const int n = L.n_idx[t], gb = L.group_bits, rows = kThreads * kUnroll >> gb;
  const int32_t *idx = L.idx[t];
  uint8_t *codes = (kv ? s.v : s.k) + l * s.sl + h * s.sh, *scales = (kv ? s.vs : s.ks) + l * s.gl + h * s.gh;
  for (int j0 = 0; j0 < n; j0 += rows) {
    Unit x[kUnroll];
    int row[kUnroll];
    bool move[kUnroll];
    const int g = threadIdx.x & ((1 << gb) - 1);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      row[u] = j0 + ((u * kThreads + (int)threadIdx.x) >> gb);
      move[u] = false;
      if (row[u] >= n) continue;
      const int i = idx[row[u]];
      if ((move[u] = i != row[u])) x[u] = load_unit<VEC>(codes + i * s.st + 16 * g, scales + i * s.gt + g);
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (move[u]) store_unit<VEC>(codes + row[u] * s.st + 16 * g, scales + row[u] * s.gt + g, x[u]);
  }
}

__global__ void __launch_bounds__(kThreads) positions_in_place_kernel(const __grid_constant__ GatherLaunch L) {
  const int t = blockIdx.x, n = L.n_idx[t];
  const int32_t *idx = L.idx[t];
  int32_t *pos = L.pos_out[t];
  for (int j0 = 0; j0 < n; j0 += kThreads) {
    const int j = j0 + threadIdx.x;
    int v = 0;
    if (j < n) v = pos[idx[j]];
    __syncthreads();
    if (j < n) pos[j] = v;
  }
}

// ------------------------------------------------------------------ host
// Rows are written through these strides: no two layers or heads in one place.
bool distinct(const commitkv_shape *s, int64_t layer, int64_t head) {
  return (s->layers == 1 || layer > 0) && (s->kv_heads == 1 || head > 0);
}
bool writable(const commitkv_shape *s, const commitkv_packed &x) {
  return distinct(s, x.stride_layer, x.stride_head) && distinct(s, x.scale_layer, x.scale_head);
}

commitkv_status check_rows(const commitkv_shape *s, int n, const commitkv_packed *x, const commitkv_rows *r, bool write) {
  commitkv_status st = check_shape(s);
  if (st) return st;
  if ((st = check_caches(s, n, x, false, false))) return st;
  if (!r) return COMMITKV_ERR_INVALID_ARG;
  for (int t = 0; t < n; ++t) {
    if (r[t].first < 0 || r[t].count < 0 || r[t].first > x[t].S - r[t].count) return COMMITKV_ERR_INVALID_ARG;
    if (r[t].count == 0) continue;
    if (!r[t].k || !r[t].v) return COMMITKV_ERR_INVALID_ARG;
    if (write ? !writable(s, x[t])
              : (s->layers > 1 && r[t].stride_layer == 0) || (s->kv_heads > 1 && r[t].stride_head == 0) ||
                    (r[t].count > 1 && r[t].stride_tok == 0))
      return COMMITKV_ERR_INVALID_ARG;
    if (r[t].count > (1 << 30)) return COMMITKV_ERR_UNSUPPORTED;  // row numbers and a block's more are 32-bit
  }
  return COMMITKV_OK;
}

template <typename T, int D>
void launch_copy(const CopyLaunch &L, bool write, bool vec, cudaStream_t s) {
  const int blocks = L.off[L.n_traj];
  if (write) {
    if (vec) write_kernel<T, D, true><<<blocks, kThreads, 0, s>>>(L);
    else write_kernel<T, D, false><<<blocks, kThreads, 0, s>>>(L);
  } else {
    if (vec) read_kernel<T, D, true><<<blocks, kThreads, 0, s>>>(L);
    else read_kernel<T, D, false><<<blocks, kThreads, 0, s>>>(L);
  }
}

// layers: the layer of each of n_layers; the cache's and the rows' strides both go by it.
commitkv_status copy(const commitkv_shape *s, int n, const commitkv_packed *x, const commitkv_rows *r, const uint8_t *layers,
                     int n_layers, bool write, cudaStream_t stream) {
  static thread_local CopyLaunch L;
  memset(&L, 0, sizeof L);
  L.n_traj = n;
  L.H = s->kv_heads;
  memcpy(L.layer_ids, layers, n_layers);
  const int eb = s->dtype == COMMITKV_BF16 ? 2 : 4,
            per = kThreads * (write ? kGroup : 8 * kUnroll) / s->head_dim;  // rows of a block
  uintptr_t wide_bits = 0, code_bits = 0;  // of the rows, of the codes
  int64_t blocks = 0;
  for (int t = 0; t < n; ++t) {
    Rows &d = L.r[t];
    d.c = to_dev(x[t]);
    d.k = r[t].k, d.v = r[t].v;
    d.sl = r[t].stride_layer, d.sh = r[t].stride_head, d.st = r[t].stride_tok;
    d.first = r[t].first, d.count = r[t].count;
    d.blocks = (int32_t)cdiv(r[t].count, per);
    L.off[t] = (int32_t)blocks;
    blocks += (int64_t)n_layers * s->kv_heads * d.blocks;
    if (blocks >= (1ll << 31)) return COMMITKV_ERR_UNSUPPORTED;
    if (r[t].count == 0) continue;
    wide_bits |= (uintptr_t)d.k | (uintptr_t)d.v | (uintptr_t)((d.sl | d.sh | d.st) * eb);
    code_bits |= (uintptr_t)d.c.k | (uintptr_t)d.c.v | (uintptr_t)(d.c.sl | d.c.sh | d.c.st);
  }
  L.off[n] = (int32_t)blocks;
  if (blocks == 0) return COMMITKV_OK;
  const bool vec = wide_bits % 16 == 0 && code_bits % (write ? 16 : 4) == 0;
  if (s->dtype == COMMITKV_BF16) {
    if (s->head_dim == 128) launch_copy<__nv_bfloat16, 128>(L, write, vec, stream);
    else launch_copy<__nv_bfloat16, 64>(L, write, vec, stream);
  } else {
    if (s->head_dim == 128) launch_copy<float, 128>(L, write, vec, stream);
    else launch_copy<float, 64>(L, write, vec, stream);
  }
  ++launch_count();
  return cudaGetLastError() == cudaSuccess ? COMMITKV_OK : COMMITKV_ERR_CUDA;
}

commitkv_status copy_rows(const commitkv_shape *s, int32_t n, const commitkv_packed *x, const commitkv_rows *r,
                          const uint8_t *mask, bool write, cudaStream_t stream) {
  const commitkv_status st = check_rows(s, n, x, r, write);
  if (st) return st;
  uint8_t ids[kMaxLayers];
  int m = 0;
  for (int l = 0; l < s->layers; ++l)
    if (!mask || mask[l]) ids[m++] = (uint8_t)l;
  return copy(s, n, x, r, ids, m, write, stream);
}

}  // namespace

cudaError_t launch_read(const commitkv_shape *s, int n, const commitkv_packed *c, const commitkv_rows *r,
                        const uint8_t *layers, int n_layers, cudaStream_t stream) {
  return copy(s, n, c, r, layers, n_layers, false, stream) == COMMITKV_OK ? cudaSuccess : cudaErrorUnknown;
}

commitkv_status check_caches(const commitkv_shape *s, int n, const commitkv_packed *x, bool positions, bool queries) {
  if (n < 1 || n > kMaxTraj || !x) return COMMITKV_ERR_INVALID_ARG;
  for (int t = 0; t < n; ++t) {
    const commitkv_packed &c = x[t];
    if (c.S < 0 || c.W < 0 || c.P < 0) return COMMITKV_ERR_INVALID_ARG;
    if (c.S > 0 && (!c.k || !c.v || !c.k_scale || !c.v_scale || (positions && !c.pos))) return COMMITKV_ERR_INVALID_ARG;
    if (queries && c.W > 0 && (!c.q || !c.q_pos)) return COMMITKV_ERR_INVALID_ARG;
    if (c.stride_tok < s->head_dim / 2 || c.stride_head < 0 || c.stride_layer < 0 || c.scale_tok < s->head_dim / kGroup ||
        c.scale_head < 0 || c.scale_layer < 0)
      return COMMITKV_ERR_INVALID_ARG;
    if ((int64_t)(s->q_heads / s->kv_heads) * c.W > (1 << 24)) return COMMITKV_ERR_INVALID_ARG;
  }
  return COMMITKV_OK;
}

}  // namespace pk
}  // namespace ckv

using namespace ckv;

extern "C" {

commitkv_status commitkv_packed_write(const commitkv_shape *shape, int32_t n_traj, const commitkv_packed *caches,
                                      const commitkv_rows *rows, const uint8_t *layer_mask, cudaStream_t stream) {
  return pk::copy_rows(shape, n_traj, caches, rows, layer_mask, true, stream);
}

commitkv_status commitkv_packed_read(const commitkv_shape *shape, int32_t n_traj, const commitkv_packed *caches,
                                     const commitkv_rows *rows, const uint8_t *layer_mask, cudaStream_t stream) {
  return pk::copy_rows(shape, n_traj, caches, rows, layer_mask, false, stream);
}

commitkv_status commitkv_packed_compact(const commitkv_shape *shape, int32_t n_traj, const commitkv_packed *cache,
                                        const uint8_t *const *retired, const int32_t *const *pending,
                                        const int32_t *n_pending, const float *const *pending_priority,
                                        const float *const *fill_score, int32_t budget_B, int32_t pending_tokens_BN,
                                        int32_t pending_cap_pages, int32_t *const *idx_out, int32_t *n_idx_out,
                                        const commitkv_packed *dst, void *workspace, size_t workspace_bytes,
                                        cudaStream_t stream) {
  commitkv_status st = check_shape(shape);
  if (st) return st;
  if ((st = pk::check_caches(shape, n_traj, cache, true, false))) return st;
  commitkv_traj tr[kMaxTraj] = {};  // what the selection reads of a trajectory
  for (int t = 0; t < n_traj; ++t) {
    const commitkv_packed &x = cache[t];
    tr[t].k = x.k, tr[t].v = x.v;
    tr[t].stride_tok = shape->head_dim;
    tr[t].pos = x.pos;
    tr[t].S = x.S;
    tr[t].page_start = x.page_start, tr[t].page_len = x.page_len;
    tr[t].P = x.P;
  }
  if ((st = check_compact_args(shape, n_traj, tr, retired, pending, n_pending, pending_priority, fill_score, budget_B,
                               pending_tokens_BN, pending_cap_pages, idx_out, n_idx_out)))
    return st;
  if (dst && (st = pk::check_caches(shape, n_traj, dst, false, false))) return st;
  for (int t = 0; t < n_traj; ++t) {
    const commitkv_packed &to = dst ? dst[t] : cache[t];
    const int32_t most = std::min(budget_B, cache[t].S);
    if (most > 0 && (to.S < most || !pk::writable(shape, to))) return COMMITKV_ERR_INVALID_ARG;
  }
  if (!workspace || (uintptr_t)workspace % 256) return COMMITKV_ERR_WORKSPACE;
  size_t need = 256;
  for (int t = 0; t < n_traj; ++t) need += ((size_t)cache[t].S + 255) / 256 * 256;
  if (workspace_bytes < need) return COMMITKV_ERR_WORKSPACE;

  static thread_local CompactLaunch C;
  static thread_local pk::GatherLaunch G;
  memset(&C, 0, sizeof C);
  memset(&G, 0, sizeof G);
  C.n_traj = n_traj;
  C.M = shape->layers;
  C.H = shape->kv_heads;
  C.d = shape->head_dim;
  C.elem_bytes = 1;
  uint8_t *cls = static_cast<uint8_t *>(workspace) + 256;
  bool vec = true;
  int32_t most = 0;
  for (int t = 0; t < n_traj; ++t) {
    const commitkv_packed &x = cache[t];
    C.t[t].S = x.S, C.t[t].P = x.P, C.t[t].ps = x.page_start, C.t[t].pl = x.page_len, C.t[t].pos = x.pos;
    C.retired[t] = retired[t];
    C.n_pending[t] = n_pending[t];
    C.pending[t] = n_pending[t] ? pending[t] : nullptr;
    C.prio[t] = n_pending[t] ? pending_priority[t] : nullptr;
    C.fill[t] = fill_score[t];
    C.cls[t] = cls;
    cls += ((size_t)x.S + 255) / 256 * 256;
    C.idx[t] = idx_out[t];
    G.src[t] = pk::to_dev(x);
    G.dst[t] = dst ? pk::to_dev(dst[t]) : G.src[t];
    G.idx[t] = idx_out[t];
    G.pos[t] = x.pos;
    G.pos_out[t] = dst ? dst[t].pos : x.pos;
    most = std::max(most, std::min(budget_B, x.S));
    for (const pk::Cache *c : {&G.src[t], &G.dst[t]})
      if (x.S > 0)
        vec = vec && ((uintptr_t)c->k | (uintptr_t)c->v | (uintptr_t)(c->sl | c->sh | c->st)) % 16 == 0;
  }
  C.n_idx = n_idx_out;
  C.B = budget_B;
  C.B_N = pending_tokens_BN;
  C.cap = pending_cap_pages;
  G.n_idx = n_idx_out;
  G.H = shape->kv_heads;
  G.group_bits = shape->head_dim == 128 ? 2 : 1;
  const int64_t slices = 2ll * shape->layers * shape->kv_heads;
  if (slices > 65535) return COMMITKV_ERR_UNSUPPORTED;
  cudaError_t e = launch_compact(C, static_cast<WsHeader *>(workspace), stream);  // no outputs: the selection alone
  if (e == cudaSuccess && most > 0) {
    if (dst) {
      const dim3 grid((unsigned)pk::cdiv((int64_t)most << G.group_bits, pk::kThreads * pk::kUnroll), (unsigned)slices, n_traj);
      if (vec) pk::gather_kernel<true><<<grid, pk::kThreads, 0, stream>>>(G);
      else pk::gather_kernel<false><<<grid, pk::kThreads, 0, stream>>>(G);
      ++launch_count();
    } else {
      const dim3 grid(1, (unsigned)slices, n_traj);
      if (vec) pk::gather_in_place_kernel<true><<<grid, pk::kThreads, 0, stream>>>(G);
      else pk::gather_in_place_kernel<false><<<grid, pk::kThreads, 0, stream>>>(G);
      e = cudaGetLastError();
      if (e == cudaSuccess) pk::positions_in_place_kernel<<<n_traj, pk::kThreads, 0, stream>>>(G);
      launch_count() += 2;
    }
    if (e == cudaSuccess) e = cudaGetLastError();
  }
  return e == cudaSuccess ? COMMITKV_OK : COMMITKV_ERR_CUDA;
}

}  // extern "C"
