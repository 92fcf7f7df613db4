// What the tensor-core attention kernels of row tiles share: waits, the items
// handed out by the hardware, plans, and results on their way out.
#pragma once

#include "attend.cuh"
#include "sm103.cuh"

namespace ckv {
namespace at {

using namespace ckv::sm103;

constexpr int BM = 128;  // rows of a tile
constexpr uint64_t kWait = 4000000000ull;
constexpr float kLazy = 8.0f;

// A block's flags: set when a wait ran out, and how many of its warps are at
// rows that redo_row takes.  Those go through the whole cache a row at a time
// (bounded, but 4.9 s for 38,912 rows over 131,072 tokens that all need it,
// bf16, 128 channels), so waits do not run out meanwhile.
enum { kAbort, kRedoing, kFlags };

// Waits for the phase with the given parity; parks the thread before it first
// reads the clock.
__device__ __forceinline__ bool wait(uint64_t *bar, uint32_t parity, volatile int *flags) {
#pragma unroll 1
  for (int i = 0; i < 4; ++i)
    if (mbar_try_wait_sleep(bar, parity, 20000)) return true;
  uint64_t t0 = now_ns();
#pragma unroll 1
  while (!mbar_try_wait_sleep(bar, parity, 20000)) {
    if (flags[kAbort]) return false;
    if (flags[kRedoing]) t0 = now_ns();
    else if (now_ns() - t0 > kWait) {
      flags[kAbort] = 1;
      return false;
    }
  }
  return true;
}

// A warp enters (1) and leaves (-1) such rows.
__device__ __forceinline__ void redoing(volatile int *flags, int change) {
  if ((threadIdx.x & 31) == 0) atomicAdd_block(const_cast<int *>(flags) + kRedoing, change);
}

struct Plan {
  Tiles tl;
  int j0, j1;
  int rows;  // of the item; 0: no more items
  Item it;
};

// One block is launched per item, and one that is done with its own takes the
// next block's that has not started (PTX clusterlaunchcontrol), so items are
// handed out as SMs get free while a block keeps its tensor memory, its
// barriers and the pipeline across items.  It asks kAsk tiles before its end:
// long enough for the next item's plan, and not at the start, where the blocks
// with the longest items would take the last ones too (20 prompts of up to 300
// rows over up to 9,000 tokens: 301 us asking at the start, 274 so; 3 tiles or 9
// are within 1 % of 6).  The warp that plans asks, told by the warp that copies.
constexpr int kAsk = 6;
__device__ __forceinline__ void ask_next(uint4 *answer, uint64_t *bar) {
  fence_proxy_async();  // the last answer has been read
  mbar_expect_tx(bar, 16);
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(
                   smem_addr(answer)),
               "r"(smem_addr(bar))
               : "memory");
}
__device__ __forceinline__ int read_next(const uint4 *answer) {
  int x;
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b128 a;\n\t"
      "ld.shared.b128 a, [%1];\n\t"
      "mov.s32 %0, -1;\n\t"
      "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, a;\n\t"
      "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %0, a;\n\t}"
      : "=r"(x)
      : "r"(smem_addr(answer))
      : "memory");
  return x;
}

// One lane of a converged warp, always the same.
__device__ __forceinline__ bool elect_one() {
  uint32_t e;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(e));
  return e != 0;
}

__device__ __forceinline__ bool wait_warp(uint64_t *bar, uint32_t parity, volatile int *flags) {
  return __all_sync(0xffffffffu, wait(bar, parity, flags));
}

// Row r of an item: its query, and what it sees.  Behind the last row: zeros
// as queries, nothing to mask.
template <typename T>
__device__ __forceinline__ const T *row_query(const Launch &L, const Seg &sg, const Item &it, int r, int d,
                                              const int32_t *&qpos) {
  if (r >= sg.R) return nullptr;
  const Traj &t = L.t[traj_of_row(L, sg, r)];
  qpos = t.qpos + r / L.g;
  return static_cast<const T *>(t.q) + row_index(L, t, it.l, it.kvh, r) * d;
}
__device__ __forceinline__ Span row_sees(const Launch &L, const Seg &sg, const int32_t *qpos, int3 &u) {
  Span sp = {0, 0x7fffffff, 0};
  if (qpos) {
    sp = row_span(sg.pos, sg.S, *qpos, L.window, L.sinks);
    if (sp.lo < sp.hi) u.x = min(u.x, sp.lo), u.y = max(u.y, sp.hi);
    u.z = max(u.z, sp.se);
  }
  return sp;
}
// What `rows` rows from r0 see, by a warp: a lane for each position, since the
// rows of its g query heads see the same tokens, and gaps in the positions cost
// a search for each.  The rest of the N rows has nothing to mask.
template <typename T, int D, int N>
__device__ __forceinline__ void rows_see(const Launch &L, const Seg &sg, const Item &it, int r0, int rows, Span *span,
                                         int3 &u) {
  const int lane = threadIdx.x & 31, p0 = r0 / L.g, end = (r0 + rows - 1) / L.g;
#pragma unroll 1
  for (int p = p0 + lane; p <= end; p += 32) {
    const int a = max(r0, p * L.g), b = min(r0 + rows, (p + 1) * L.g);
    const int32_t *qpos = nullptr;
    row_query<T>(L, sg, it, a, D, qpos);
    const Span sp = row_sees(L, sg, qpos, u);
#pragma unroll 1
    for (int r = a; r < b; ++r) span[r - r0] = sp;
  }
#pragma unroll 1
  for (int i = rows + lane; i < N; i += 32) span[i] = {0, 0x7fffffff, 0};
}
// The union of what the rows of a warp see: (least lo, largest hi, largest se).
__device__ __forceinline__ int3 join_warp(int3 u) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    u.x = min(u.x, __shfl_xor_sync(0xffffffffu, u.x, o));
    u.y = max(u.y, __shfl_xor_sync(0xffffffffu, u.y, o));
    u.z = max(u.z, __shfl_xor_sync(0xffffffffu, u.z, o));
  }
  return u;
}

// A warp's 32 rows on their way out, 64 bytes of every row at a time: through
// shared memory, so that four lanes store a row's piece side by side.
struct RowsOut {
  static constexpr int kStage = 32 * 5;  // 16-byte words: 64 bytes of each row, 16 apart
  uint32_t stage;
  uint64_t to[4];  // where this lane's 16 bytes of rows lane / 4 + 8 k go
  int lane;
  // `row`: where this lane's row goes, 0: nowhere
  __device__ __forceinline__ RowsOut(uint32_t stage, uint64_t row, int lane) : stage(stage), lane(lane) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      to[k] = __shfl_sync(0xffffffffu, row, 8 * k + lane / 4);
      if (to[k]) to[k] += 16 * (lane % 4);
    }
  }
  __device__ __forceinline__ void put(const uint32_t *w) {  // 16 words of this lane's row
    __syncwarp();                                           // the last piece has been read
#pragma unroll
    for (int k = 0; k < 4; ++k)
      asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(stage + lane * 80 + 16 * k), "r"(w[4 * k]),
                   "r"(w[4 * k + 1]), "r"(w[4 * k + 2]), "r"(w[4 * k + 3])
                   : "memory");
    __syncwarp();
    uint4 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(v[k].x), "=r"(v[k].y), "=r"(v[k].z), "=r"(v[k].w)
                   : "r"(stage + (8 * k + lane / 4) * 80 + 16 * (lane % 4))
                   : "memory");
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (to[k]) {
        asm volatile("st.global.v4.b32 [%0], {%1, %2, %3, %4};" ::"l"(to[k]), "r"(v[k].x), "r"(v[k].y), "r"(v[k].z),
                     "r"(v[k].w)
                     : "memory");
        to[k] += 64;
      }
  }
};

}  // namespace at
}  // namespace ckv
