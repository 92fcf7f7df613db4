// Attention of many rows of fp32 caches (16-byte aligned) on the tensor cores.
//
// Every fp32 operand is a sum of three bf16 terms, each the rounded rest of the
// ones before (2^-25 of it is lost), and a product the six products of terms
// whose places add up to at most two (the others are below 2^-24): six bf16
// MMAs at 1,969 TFLOP/s (measured) against fp32's 80.  The MMA's sums are cut off, not
// rounded, so P V of a tile is a sum by itself and the running O is kept in
// fp32 registers.
//
// A CTA of 384 or 512 threads per SM takes items of up to 128 query rows over
// 64-token tiles:
//   warp 1      the MMAs: S = Q K^T of a tile, then P V of the one before
//   warp 3      the plan of the next item
//   warps 4-7   softmax, a thread per row: scores from TMEM, the weights' terms
//               back over them, O += D (the tile's P V) in registers
//   warps 8-    the split: K, V and Q from memory to registers, their terms to
//               shared memory in the MMA's layout; the next tile's K while the
//               MMAs run this one's.  Eight warps for 128 channels, whose splits
//               the MMAs waited for with four (six prompts of 300 rows over up to
//               9,000 tokens: 628 and 512 us), four for 64, where the softmax is
//               what they wait for (1,000 rows over 9,000: 403, with eight 407).
//               128 channels spill 80 bytes a thread and reload 200 (128 registers
//               a thread at launch).  One piece of code for K and V: the roles'
//               loops have to fit the instruction cache together (split apart,
//               1,507 against 1,025 us for 4,000 rows of 16 heads, 8,000 tokens)
// Shared memory holds one tile (Q, K and V of three terms: 192 KB), so a tile's
// K is split while the P V before it runs, its V while its own Q K^T does.
// TMEM: scores and weights of tile t at column 96 (t & 1) (the scores in the
// last 64 of 96 columns, a chunk's terms over those already read), D at 192 + D
// (t & 1).
#include <string.h>

#include "attend_tc.cuh"

namespace ckv {
namespace at {
namespace {

constexpr int BT = 64;  // tokens of a tile
constexpr int NT = 3;   // terms

template <int D>
struct Smem {
  static constexpr int SW = D == 128 ? 8 : 4;  // splitting warps
  static constexpr uint32_t kQ = BM * D * 2, kKV = BT * D * 2;
  alignas(1024) uint8_t q[NT][kQ];
  alignas(1024) uint8_t k[NT][kKV];
  alignas(1024) uint8_t v[NT][kKV];
  Span span[2][BM];
  Plan plan[2];
  float4 stage[4][RowsOut::kStage];
  int3 first[4];
  alignas(16) uint4 next;
  uint64_t ask, next_full, plan_full[2], plan_empty[2], q_full, q_empty, k_full, k_empty, v_full, v_empty, s_full[2], p_full[2],
      d_full[2], d_empty[2], drain;
  uint32_t tmem;
  int flags[kFlags];
};

// Takes a term off two values: their bf16 roundings, the exact rests stay.
__device__ __forceinline__ uint32_t take_term(float &x, float &y) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
  x -= __low2float(h);
  y -= __high2float(h);
  return *reinterpret_cast<const uint32_t *>(&h);
}

// Four channels each (4 c ..) of N rows of an operand of ROWS rows: their terms
// into the three tiles, all N side by side, since a value's terms depend on
// one another.
template <int ROWS, int N>
__device__ __forceinline__ void put_terms(uint32_t tile, uint32_t term_bytes, const int (&r)[N], const int (&c)[N],
                                          float4 (&x)[N]) {
  uint32_t at[N];
#pragma unroll
  for (int i = 0; i < N; ++i)
    at[i] = tile + (c[i] >> 4) * (ROWS * 128) + sw128_offset(r[i], (c[i] >> 1) & 7) + (c[i] & 1) * 8;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    uint32_t a[N], b[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      a[i] = take_term(x[i].x, x[i].y);
      b[i] = take_term(x[i].z, x[i].w);
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
      asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at[i] + t * term_bytes), "r"(a[i]), "r"(b[i]) : "memory");
  }
}

// The c-th of the six products of terms, growing in size: which term of A and
// of B.
__device__ __forceinline__ int term_a(int c) { return c == 1 ? 2 : c == 2 || c == 4 ? 1 : 0; }
__device__ __forceinline__ int term_b(int c) { return c == 0 ? 2 : c == 2 || c == 3 ? 1 : 0; }

template <int D>
__global__ void __launch_bounds__((8 + Smem<D>::SW) * 32, 1) attend_tc_f32(const __grid_constant__ Launch L, WsHeader *hdr) {
  using S = Smem<D>;
  extern __shared__ uint8_t smem_raw[];
  S &sm = *reinterpret_cast<S *>(smem_raw + ((0u - smem_addr(smem_raw)) & 1023u));
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
  volatile int *flags = sm.flags;

  pdl_start_next();
  if (threadIdx.x == 0) {
    sm.flags[kAbort] = sm.flags[kRedoing] = 0;
    for (int b = 0; b < 2; ++b) {
      mbar_init(&sm.plan_full[b], 1);
      mbar_init(&sm.plan_empty[b], 5 + S::SW);  // MMA, four softmax and the splitting warps
      mbar_init(&sm.s_full[b], 1);
      mbar_init(&sm.p_full[b], 4);
      mbar_init(&sm.d_full[b], 1);
      mbar_init(&sm.d_empty[b], 4);
    }
    mbar_init(&sm.ask, 1);
    mbar_init(&sm.next_full, 1);
    mbar_init(&sm.q_full, S::SW);
    mbar_init(&sm.q_empty, 1);
    mbar_init(&sm.k_full, S::SW);
    mbar_init(&sm.k_empty, 1);
    mbar_init(&sm.v_full, S::SW);
    mbar_init(&sm.v_empty, 1);
    mbar_init(&sm.drain, 1);
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(&sm.tmem, 512);
    tmem_relinquish();
  }
  if (warp >= 4 && warp < 8) {  // the first item's rows, a thread each
    const Item it = decode_item(L, blockIdx.x);
    const Seg &sg = L.seg[it.s];
    const int i = threadIdx.x - 128;
    const int32_t *qpos = nullptr;
    row_query<float>(L, sg, it, it.rt * BM + i, D, qpos);
    int3 u = make_int3(0x7fffffff, 0, 0);
    sm.span[0][i] = row_sees(L, sg, qpos, u);
    u = join_warp(u);
    if (lane == 0) sm.first[warp - 4] = u;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tm = sm.tmem;

  // registers a thread of each group of four warps: 80 + 224 + 200 = 3 x 168, or
  // 80 + 224 + 2 x 104 = 4 x 128
  if (warp < 4) {
    regs_dec<80>();
    if (warp == 1) {
      // ------------------------------------------------------------ MMAs
      // descriptors of the first terms; a term further adds to the address field
      const uint64_t q0 = smem_desc(smem_addr(sm.q[0]), 16, 1024, kSwizzle128B),
                     k0 = smem_desc(smem_addr(sm.k[0]), 16, 1024, kSwizzle128B),
                     v0 = smem_desc(smem_addr(sm.v[0]), BT * 128, 1024, kSwizzle128B);
      uint32_t t = 0;  // tiles of earlier items
      bool ok = true;
      for (int n = 0; ok; ++n) {
        if (!wait_warp(&sm.plan_full[n & 1], (n >> 1) & 1, flags)) break;
        const int nt = sm.plan[n & 1].j1 - sm.plan[n & 1].j0, rows = sm.plan[n & 1].rows;
        if (rows == 0) break;
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.plan_empty[n & 1]);
        if (!wait_warp(&sm.q_full, n & 1, flags)) break;
        if (nt == 0 && lane == 0) mbar_arrive(&sm.q_empty);
        for (int j = 0; j <= nt && nt > 0; ++j) {
          if (j < nt) {
            const uint32_t T = t + j, b = T & 1;
            if (!(ok = wait_warp(&sm.k_full, T & 1, flags))) break;
            tc_fence_after();
            if (elect_one()) {
              constexpr uint32_t idesc = idesc_bf16_f32(BM, BT, 0, 0);
#pragma unroll
              for (int c = 0; c < 6; ++c) {
                const uint64_t qa = q0 + term_a(c) * (S::kQ >> 4), ka = k0 + term_b(c) * (S::kKV >> 4);
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)
                  mma_bf16(tm + 96 * b + 32, qa + (((ks >> 2) * (BM * 128) + (ks & 3) * 32) >> 4),
                           ka + (((ks >> 2) * (BT * 128) + (ks & 3) * 32) >> 4), idesc, c > 0 || ks > 0);
              }
              mma_commit(&sm.s_full[b]);
              mma_commit(&sm.k_empty);
              if (j + 1 == nt) mma_commit(&sm.q_empty);
            }
            __syncwarp();
          }
          if (j > 0) {
            const uint32_t T = t + j - 1, b = T & 1, u = T >> 1;
            ok = wait_warp(&sm.v_full, T & 1, flags) &&
                 (u == 0 || wait_warp(&sm.d_empty[b], (u - 1) & 1, flags)) &&
                 wait_warp(&sm.p_full[b], u & 1, flags);
            if (!ok) break;
            tc_fence_after();
            if (elect_one()) {
              constexpr uint32_t idesc = idesc_bf16_f32(BM, D, 0, 1);
#pragma unroll
              for (int c = 0; c < 6; ++c) {
                const uint64_t va = v0 + term_b(c) * (S::kKV >> 4);
                const uint32_t pa = tm + 96 * b + 16 * term_a(c);
#pragma unroll
                for (int ks = 0; ks < BT / 16; ++ks)
                  mma_bf16_ts(tm + 192 + D * b, pa + 48 * (ks >> 1) + 8 * (ks & 1), va + (ks * 2048 >> 4), idesc,
                              c > 0 || ks > 0);
              }
              mma_commit(&sm.d_full[b]);
              mma_commit(&sm.v_empty);
            }
            __syncwarp();
          }
        }
        t += nt;
      }
      if (__any_sync(0xffffffffu, flags[kAbort] != 0)) {
        if (elect_one()) {
          mma_commit(&sm.drain);  // every MMA issued by this thread has completed
          mbar_wait_drain(&sm.drain, 0, kWait);
        }
        __syncwarp();
      }
    } else if (warp == 3) {
      // ------------------------------------------------------------ plans
      int item = blockIdx.x;
      for (int n = 0;; ++n) {
        const int buf = n & 1;
        if (n >= 2 && !wait_warp(&sm.plan_empty[buf], ((n >> 1) - 1) & 1, flags)) break;
        if (n > 0) {
          if (!wait_warp(&sm.ask, (n - 1) & 1, flags)) break;
          if (lane == 0) ask_next(&sm.next, &sm.next_full);
          if (!wait_warp(&sm.next_full, (n - 1) & 1, flags)) {
            if (lane == 0) mbar_wait_drain(&sm.next_full, (n - 1) & 1, kWait);  // it lands before the block's memory goes
            break;
          }
          item = read_next(&sm.next);
          __syncwarp();
        }
        if (item < 0) {
          if (lane == 0) {
            sm.plan[buf].rows = 0;
            mbar_arrive(&sm.plan_full[buf]);
          }
          break;
        }
        const Item it = decode_item(L, item);
        const Seg &sg = L.seg[it.s];
        const int r0 = it.rt * BM, rows = min(BM, sg.R - r0);
        int3 u = make_int3(0x7fffffff, 0, 0);
        if (n == 0) {
          if (lane < 4) u = sm.first[lane];
        } else {
          rows_see<float, D, BM>(L, sg, it, r0, rows, sm.span[buf], u);
        }
        u = join_warp(u);
        if (lane == 0) {
          const Tiles tl = make_tiles(u.x, u.y, u.z, BT);
          sm.plan[buf] = {tl, chunk_tile(tl, it.c, it.n), chunk_tile(tl, it.c + 1, it.n), rows, it};
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.plan_full[buf]);
      }
    }
  } else if (warp < 8) {
    // ------------------------------------------------------------ softmax
    regs_inc<224>();
    const int wq = warp & 3, row = wq * 32 + lane;
    const uint32_t lanes = (uint32_t)(wq * 32) << 16;
    uint32_t t = 0;
    bool ok = true;
    for (int n = 0; ok; ++n) {
      if (!wait_warp(&sm.plan_full[n & 1], (n >> 1) & 1, flags)) break;
      const Plan pl = sm.plan[n & 1];
      if (pl.rows == 0) break;
      const Span sp = sm.span[n & 1][row];
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.plan_empty[n & 1]);
      const int nt = pl.j1 - pl.j0;
      float2 o[D / 2];
      float m = -INFINITY, lsum = 0.0f;
#pragma unroll
      for (int c = 0; c < D / 2; ++c) o[c] = make_float2(0.0f, 0.0f);
      auto take = [&](uint32_t T) {  // O += the P V of tile T
        const uint32_t b = T & 1;
        if (!wait_warp(&sm.d_full[b], (T >> 1) & 1, flags)) return false;
        tc_fence_after();
#pragma unroll
        for (int c0 = 0; c0 < D; c0 += 32) {
          float y[32];
          tmem_ld32f(tm + lanes + 192 + D * b + c0, y);
          tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < 16; ++i) o[c0 / 2 + i] = fadd2(o[c0 / 2 + i], make_float2(y[2 * i], y[2 * i + 1]));
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.d_empty[b]);
        return true;
      };
      for (int j = 0; j < nt; ++j) {
        const uint32_t T = t + j, b = T & 1, col = tm + lanes + 96 * b;
        if (!(ok = wait_warp(&sm.s_full[b], (T >> 1) & 1, flags))) break;
        tc_fence_after();
        const int t0 = tile_start(pl.tl, pl.j0 + j, BT), t1 = tile_end(pl.tl, pl.j0 + j, BT);
        const int a = t0 - sp.lo, end = min(sp.hi, t1) - sp.lo, se = min(sp.se, t1) - t0;
        const unsigned len = end > 0 ? (unsigned)end : 0u;
        const bool all = __all_sync(0xffffffffu, sp.lo <= t0 && t0 + BT <= min(sp.hi, t1));
        float x[32], top = -INFINITY;
        auto load = [&](int c) {
          tmem_ld32f(col + 32 + 32 * c, x);
          tmem_wait_ld();
          if (!all) {
#pragma unroll
            for (int i = 0; i < 32; ++i) x[i] = (unsigned)(a + 32 * c + i) < len || 32 * c + i < se ? x[i] : -INFINITY;
          }
        };
#pragma unroll 1
        for (int c = 0; c < BT / 32; ++c) {
          load(c);
#pragma unroll
          for (int i = 0; i < 32; i += 2) top = fmax3(top, x[i], x[i + 1]);
        }
        top = __fmul_rn(top, L.scale_log2);
        const bool raise = top > m + kLazy;  // false while both are -inf
        const float f = raise && m != -INFINITY ? exp2f(m - top) : 1.0f;
        if (raise) m = top;
        const float neg = m == -INFINITY ? 0.0f : -m;
        float ps[2] = {0.0f, 0.0f};
#pragma unroll 1
        for (int c = 0; c < BT / 32; ++c) {
          load(c);
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            x[i] = fast_exp2(fmaf(x[i], L.scale_log2, neg));
            ps[i & 1] += x[i];
          }
#pragma unroll
          for (int k = 0; k < NT; ++k) {
            uint32_t p[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) p[i] = take_term(x[2 * i], x[2 * i + 1]);
            tmem_st16(col + 48 * c + 16 * k, p);
          }
        }
        tmem_wait_st();
        lsum = fmaf(lsum, f, ps[0] + ps[1]);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.p_full[b]);
        if (j > 0 && !(ok = take(T - 1))) break;
        if (__any_sync(0xffffffffu, f != 1.0f)) {  // those sums were relative to the old maximum
#pragma unroll
          for (int c = 0; c < D / 2; ++c) o[c].x *= f, o[c].y *= f;
        }
      }
      if (!ok) break;
      if (nt > 0 && !(ok = take(t + nt - 1))) break;
      t += nt;
      // ---------------------------------------------------------- results
      const Item it = pl.it;
      const Seg &sg = L.seg[it.s];
      const int r = it.rt * BM + row;
      uint64_t dst = 0;
      float g = 1.0f;
      if (row < pl.rows) {
        if (it.split) {
          const int64_t pr = part_index(L, sg, it, r);
          dst = reinterpret_cast<uint64_t>(L.po + pr * D);
          L.pml[pr] = make_float2(m, lsum);
        } else {
          int rr = r;
          const Traj &tr = L.t[traj_of_row(L, sg, rr)];
          const int64_t orow = row_index(L, tr, it.l, it.kvh, rr);
          dst = reinterpret_cast<uint64_t>(static_cast<float *>(tr.out) + orow * D);
          g = norm_of(lsum);
          if (tr.lse) tr.lse[orow] = lse_of(m, lsum);
        }
      }
      float ck[4] = {0.0f, 0.0f, 0.0f, 0.0f};  // NaN if any is not finite
      RowsOut rows_out(smem_addr(sm.stage[warp - 4]), dst, lane);
#pragma unroll
      for (int c0 = 0; c0 < D; c0 += 16) {
        uint32_t w[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float y = (i & 1 ? o[(c0 + i) / 2].y : o[(c0 + i) / 2].x) * g;
          ck[i & 3] = fmaf(y, 0.0f, ck[i & 3]);
          w[i] = __float_as_uint(y);
        }
        rows_out.put(w);
      }
      const float chk = (ck[0] + ck[1]) + (ck[2] + ck[3]);
      // A value that is not finite: masked ones met a weight of zero, and an
      // infinite key's terms are NaN though its score may be -inf.  Or very
      // large scores.
      unsigned bad = __ballot_sync(0xffffffffu, row < pl.rows && (chk != 0.0f || !isfinite(lsum) || is_far(m)));
      const bool redo = bad != 0;
      if (redo) redoing(flags, 1);
      while (bad) {
        const int k = __ffs(bad) - 1;
        bad &= bad - 1;
        const Span one = {__shfl_sync(0xffffffffu, sp.lo, k), __shfl_sync(0xffffffffu, sp.hi, k),
                          __shfl_sync(0xffffffffu, sp.se, k)};
        float mk = __shfl_sync(0xffffffffu, m, k), lk = __shfl_sync(0xffffffffu, lsum, k);
        const int32_t *qpos;
        const float *qk = row_query<float>(L, sg, it, r - lane + k, D, qpos);
        const bool anew = !isfinite(lk) || is_far(mk);  // the maximum and the sum as well
        if (anew) mk = redo_max<float, D>(L, sg, it.l, it.kvh, qk, one, pl.tl, BT, pl.j0, pl.j1);
        float ok_[D / 32] = {}, l2 = NAN;
        if (!isnan(mk))  // else the row is NaN
          l2 = redo_row<float, D>(L, sg, it.l, it.kvh, qk, one, pl.tl, BT, pl.j0, pl.j1, mk == -INFINITY ? 0.0f : mk, ok_,
                                  anew, !is_far(mk));
        __syncwarp();
        write_row_warp<float, D>(L, sg, it, r - lane + k, ok_, mk, anew ? l2 : lk);
      }
      if (redo) redoing(flags, -1);
    }
  } else {
    // ------------------------------------------------------------ split
    if constexpr (S::SW == 8) regs_dec<104>();
    else regs_inc<200>();
    constexpr int C4 = D / 4, NL = BT * C4 / (32 * S::SW);  // 16-byte pieces of a row, of a tile for each thread
    const int tid = threadIdx.x - 256;
    uint32_t t = 0;
    bool ok = true;
    for (int n = 0; ok; ++n) {
      if (!wait_warp(&sm.plan_full[n & 1], (n >> 1) & 1, flags)) break;
      const Plan pl = sm.plan[n & 1];
      if (pl.rows == 0) break;
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.plan_empty[n & 1]);
      const Item it = pl.it;
      const Seg &sg = L.seg[it.s];
      const int nt = pl.j1 - pl.j0;
      const float *kb = static_cast<const float *>(sg.k) + (int64_t)it.l * sg.sl + (int64_t)it.kvh * sg.sh;
      const float *vb = static_cast<const float *>(sg.v) + (int64_t)it.l * sg.sl + (int64_t)it.kvh * sg.sh;
      // pieces in the order K 0, K 1, V 0, K 2, V 1 ..: the i-th is of tile i / 2
      // (V: of the one before), which is what the MMAs take next
      float4 x[NL];
      auto fetch = [&](int i) {
        const bool is_v = i > 0 && (i & 1) == 0;
        const int j = i == 0 ? 0 : is_v ? i / 2 - 1 : (i + 1) / 2;
        const int t0 = j < nt ? tile_start(pl.tl, pl.j0 + j, BT) : 0, t1 = j < nt ? tile_end(pl.tl, pl.j0 + j, BT) : 0;
        const float *base = is_v ? vb : kb;
#pragma unroll
        for (int k = 0; k < NL; ++k) {
          const int e = k * 32 * S::SW + tid, r = e / C4, c = e % C4;
          x[k] = t0 + r < t1 ? *reinterpret_cast<const float4 *>(base + (int64_t)(t0 + r) * sg.st + 4 * c)
                             : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
      };
      fetch(0);
      if (n > 0 && !(ok = wait_warp(&sm.q_empty, (n - 1) & 1, flags))) break;
      {
        // Q: QR rows a warp, D / 4 lanes to a row
        constexpr int RW = 32 / C4 > 0 ? 32 / C4 : 1, QR = BM / S::SW;
        const int32_t *qpos;
        const int r32 = (warp - 8) * QR;
        const uint64_t src =
            lane < QR && r32 + lane < pl.rows
                ? reinterpret_cast<uint64_t>(row_query<float>(L, sg, it, it.rt * BM + r32 + lane, D, qpos))
                : 0;
#pragma unroll 1
        for (int k0 = 0; k0 < QR / RW; k0 += 4) {
          int r[4], c[4];
          float4 x[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            r[i] = r32 + (k0 + i) * RW + lane / C4, c[i] = lane % C4;
            const uint64_t p = __shfl_sync(0xffffffffu, src, r[i] - r32);
            x[i] = p ? reinterpret_cast<const float4 *>(p)[c[i]] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          }
          put_terms<BM>(smem_addr(sm.q[0]), S::kQ, r, c, x);
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.q_full);
      }
#pragma unroll 1
      for (int i = 0; i <= 2 * nt; ++i) {
        if (i == max(2 * (nt - kAsk), 0) && warp == 8 && lane == 0) mbar_arrive(&sm.ask);
        if (nt == 0) break;
        const bool is_v = i > 0 && (i & 1) == 0;
        const int j = i == 0 ? 0 : is_v ? i / 2 - 1 : (i + 1) / 2;
        if (j < nt) {
          const uint32_t T = t + j;
          ok = T == 0 || wait_warp(is_v ? &sm.v_empty : &sm.k_empty, (T - 1) & 1, flags);
          if (!ok) break;
          const uint32_t tile = smem_addr(is_v ? sm.v[0] : sm.k[0]);
#pragma unroll
          for (int k0 = 0; k0 < NL; k0 += 4) {
            int r[4], c[4];
            float4 y[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const int e = (k0 + k) * 32 * S::SW + tid;
              r[k] = e / C4, c[k] = e % C4, y[k] = x[k0 + k];
            }
            put_terms<BT>(tile, S::kKV, r, c, y);
          }
          fence_proxy_async();
          __syncwarp();
          if (lane == 0) mbar_arrive(is_v ? &sm.v_full : &sm.k_full);
        }
        fetch(i + 1);
      }
      t += nt;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) tmem_dealloc(tm, 512);
  if (threadIdx.x == 0 && sm.flags[kAbort]) record_error(hdr, COMMITKV_ERR_TIMEOUT, 31);
  pdl_wait();
}

template <int D>
cudaError_t launch(const Launch &L, WsHeader *hdr, cudaStream_t s, bool early) {
  constexpr int smem = (int)sizeof(Smem<D>) + 1024;
  static_assert(smem <= 232448, "shared memory");
  const cudaError_t e = cudaFuncSetAttribute(attend_tc_f32<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  return launch_after(attend_tc_f32<D>, L.item_off[L.n_seg], (8 + Smem<D>::SW) * 32, smem, s, early, L, hdr);
}

}  // namespace

cudaError_t launch_tc_f32(const Launch &L, WsHeader *hdr, cudaStream_t s, bool early) {
  return L.d == 128 ? launch<128>(L, hdr, s, early) : launch<64>(L, hdr, s, early);
}

}  // namespace at
}  // namespace ckv
