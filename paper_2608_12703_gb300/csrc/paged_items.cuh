// Attention over a paged cache: who works on what, and the end of an item, where
// the results of several warps and blocks are joined.  Shared by the kernels
// over 16-bit, 32-bit and 8-bit caches, whose inner loops differ.
#pragma once

#include "kernels.h"
#include "paged.cuh"

namespace asrspec {
namespace {

struct AttendArgs {
  PagedView c;
  PagedRows r;
  char* out;     // [B][R][H][D]
  float* lse;    // [B][R][H] or null
  int* tickets;  // [MAX_WORKERS] zero between calls: partial results delivered of the item that a warp begins
  float* ws;     // partial results: 2 a warp, [TR] max, [TR] sum, [TR][D] output
  int max_workers;
};
constexpr int MAX_WORKERS = 4096;

// ---------------------------------------------------------------------------
// The end of an item.  Every warp leaves its (max, sum, output) in shared
// memory, [TR] max, [TR] sum, [TR][D] output; `regions` of them are combined by
// a warp, or by the block where all its warps worked on the item.  This code
// runs once an item, mostly from a cold instruction cache: its loops stay
// rolled, and the round trips to L2 are overlapped by asynchronous copies.
// ---------------------------------------------------------------------------
// A kernel's shape: head dimension, rows of a tile, warps of a block (one block
// an SM), and steps of K and V (8 KB) that a warp has in flight or in use.
template <int D_, int TR_, int WARPS_, int STAGES_>
struct Shape {
  static constexpr int D = D_, TR = TR_, WARPS = WARPS_, STAGES = STAGES_;
  static constexpr int PART = TR * (D + 2);   // floats of a result
  // A warp's shared memory: the ring of its loads (16-bit types), then, the ring
  // drained, its result and room to fetch others' partial results into.
  static constexpr int RING = STAGES * 8192;
  static constexpr int REGION = (RING ? RING : 3 * PART * 4) / 4;   // floats
};

__device__ __forceinline__ void copy16(float* smem, const float* gmem) {   // by L2: another SM wrote it
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(smem)), "l"(gmem) : "memory");
}

struct Acc {   // four columns of a row
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  __device__ __forceinline__ void add(float pm, float pl, float4 po) {
    const float mx = fmaxf(m, pm), z = mx == -INFINITY ? 0.f : mx, f0 = ex2(m - z), f1 = ex2(pm - z);
    m = mx;
    // the products' rounding is written out: a warp and a block must join alike, whichever comes last
    l = fmaf(pl, f1, __fmul_rn(l, f0));
    o = make_float4(fmaf(po.x, f1, __fmul_rn(o.x, f0)), fmaf(po.y, f1, __fmul_rn(o.y, f0)),
                    fmaf(po.z, f1, __fmul_rn(o.z, f0)), fmaf(po.w, f1, __fmul_rn(o.w, f0)));
  }
};

template <typename T, int D>
__device__ __forceinline__ void put_row(const AttendArgs& a, int b, int kvh, int m, int col, const Acc& x) {
  const int row = (int)a.r.groups.div((uint32_t)m), hq = kvh * a.r.group + m - row * a.r.group;
  const size_t at = ((size_t)b * a.r.max_rows + row) * a.r.heads + hq;
  const float inv = x.l > 0.f ? __fdividef(1.f, x.l) : 0.f;
  if (a.lse && col == 0) a.lse[at] = (x.m + __log2f(x.l)) * LN2;
  T* out = reinterpret_cast<T*>(a.out) + at * D + col;
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4*>(out) = make_float4(x.o.x * inv, x.o.y * inv, x.o.z * inv, x.o.w * inv);
  } else {
    *reinterpret_cast<uint2*>(out) =
        make_uint2(Mma16<T>::pack(x.o.x * inv, x.o.y * inv), Mma16<T>::pack(x.o.z * inv, x.o.w * inv));
  }
}

template <typename T, typename C, bool BLOCK>
__device__ __noinline__ void finish_item(const AttendArgs& a, const WorkPlan& plan, float* sm, int regions, int b, int kvh,
                                         int tile, int rows, int u0, int u1, int worker, bool begins, bool whole, int share) {
  constexpr int D = C::D, TR = C::TR, WARPS = C::WARPS, PART = C::PART, C4 = D / 4;
  // partial results there is room for; more parts than that are joined in runs
  constexpr int ROOM = (BLOCK ? WARPS : 1) * C::REGION / PART;
  __shared__ int s_last;
  const int tid = BLOCK ? threadIdx.x : threadIdx.x & 31, nt = BLOCK ? WARPS * 32 : 32;
  const int nr = min(TR, rows - tile * TR);
  auto sync = [] {
    if (BLOCK) __syncthreads();
    else __syncwarp();
  };
  float* part = a.ws + (size_t)(2 * worker + (begins ? 1 : 0)) * PART;
  int n = regions, stride = C::REGION;   // what is added up: first the warps' results, then, by the last to come, the parts
  int p0 = 0, parts = 0, n0 = 0, n1 = 0, c0 = 0, c1 = 0, wf = 0;
  bool final = whole;
  Acc carry[(TR * C4 + (BLOCK ? WARPS * 32 : 32) - 1) / (BLOCK ? WARPS * 32 : 32)];   // from run to run
#pragma unroll 1
  for (;;) {
    sync();
    int e = 0;
#pragma unroll 1
    for (int x = tid; x < nr * C4; x += nt, ++e) {
      const int in = x / C4, col = (x - in * C4) * 4;
      Acc acc;
      if (p0 > 0) acc = carry[e];
#pragma unroll 1
      for (int w = 0; w < n; ++w) {
        const float* p = sm + w * stride;
        acc.add(p[in], p[TR + in], *reinterpret_cast<const float4*>(p + 2 * TR + in * D + col));
      }
      if (final) {
        put_row<T, D>(a, b, kvh, tile * TR + in, col, acc);
      } else if (parts == 0) {
        __stcg(reinterpret_cast<float4*>(part + 2 * TR + in * D + col), acc.o);
        if (col == 0) {
          __stcg(part + in, acc.m);
          __stcg(part + TR + in, acc.l);
        }
      } else {
        carry[e] = acc;
      }
    }
    if (final) {
      sync();   // the next item's results go to the same shared memory
      return;
    }
    if (parts == 0) {
      __threadfence();
      // The parts of the item, in key order: single warps wf .., then blocks c0
      // .. c1 whose warps all work on it, then single warps again.
      // Or, of a shared item, `share` blocks.
      if (share > 0) {
        c0 = u0, n1 = parts = share;
        wf = c0 * WARPS;
      } else {
        wf = plan.owner(u0);
        const int wl = plan.owner(u1 - 1);
        const bool from_first = wf % WARPS == 0 && plan.start(wf) == u0;
        const bool to_last = (wl % WARPS == WARPS - 1 || wl == plan.workers - 1) && plan.start(wl + 1) == u1;
        c0 = wf / WARPS + (from_first ? 0 : 1), c1 = wl / WARPS - (to_last ? 0 : 1);
        n0 = c0 <= c1 ? c0 * WARPS - wf : wl - wf + 1;
        n1 = c0 <= c1 ? c1 - c0 + 1 : 0;
        parts = n0 + n1 + (c0 <= c1 ? max(0, wl + 1 - (c1 + 1) * WARPS) : 0);
      }
      sync();
      int last = 0;
      if (tid == 0) {
        last = atomicAdd(a.tickets + wf, 1) == parts - 1;
        if (last) {
          a.tickets[wf] = 0;   // all have come: as the next call needs it
          __threadfence();
        }
        if (BLOCK) s_last = last;
      }
      if (BLOCK) {
        __syncthreads();
        last = s_last;
      } else {
        last = __shfl_sync(0xffffffffu, last, 0);
      }
      if (!last) return;
    } else {
      p0 += ROOM;
      sync();
    }
    n = min(ROOM, parts - p0), stride = PART;
    final = p0 + ROOM >= parts;
    const int used = 2 * TR + nr * D;   // floats of a part
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
      const int p = p0 + i;
      const int w = p < n0 ? wf + p : p < n0 + n1 ? (c0 + p - n0) * WARPS : (c1 + 1) * WARPS + p - n0 - n1;
      const float* src = a.ws + (size_t)(2 * w + (p == 0 ? 1 : 0)) * PART;
#pragma unroll 1
      for (int x = tid * 4; x < used; x += nt * 4) copy16(sm + i * PART + x, src + x);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  }
}

// Rows without keys: zeros, and -inf for the log-sum-exp.
template <typename T, int D>
__device__ __forceinline__ void clear_rows(const AttendArgs& a, const PlanMem& mem) {
  for (int b = blockIdx.x; b < a.c.batch; b += gridDim.x) {
    const int2 n = mem.lens[b];
    const int from = n.x + (a.r.causal ? n.y : 0) == 0 ? 0 : n.y;
    const size_t heads0 = ((size_t)b * a.r.max_rows + from) * a.r.heads, count = (size_t)(a.r.max_rows - from) * a.r.heads;
    uint4* o = reinterpret_cast<uint4*>(a.out + heads0 * D * sizeof(T));
    for (size_t i = threadIdx.x; i < count * (D * sizeof(T) / 16); i += blockDim.x) o[i] = make_uint4(0, 0, 0, 0);
    if (a.lse)
      for (size_t i = threadIdx.x; i < count; i += blockDim.x) a.lse[heads0 + i] = -INFINITY;
  }
}

// Who works on what.  Every end of an item costs its warps a few steps' time
// (pipeline fill, the way through shared memory), and every item that several
// blocks work on a way through L2 and a join besides; whole items cost balance
// instead.  So, by the lengths at hand and in steps:
//   WARP    a warp takes whole items;
//   BLOCK   a block takes whole items, its warps each a part of the steps;
//   SHARE   few items: all blocks, each item's number by its length;
//   SPLIT   equal runs of steps for all warps, items split wherever a run ends.
// Whole items are dealt longest sequence first, to and fro over the takers.
// Measured, us a call: 64 sequences of up to 448 slots, 20 heads: WARP 30, SPLIT
// 47; 32 of up to 1500, 12 heads: BLOCK 28, SPLIT 38; one of 230, 20 heads:
// BLOCK 10, SPLIT 14; one of 100001, 20 heads: SHARE 97, SPLIT 119; two of 1 and
// 35129, 16 heads: SHARE 60, with equal numbers of blocks 113.
enum Deal { DEAL_WARP, DEAL_BLOCK, DEAL_SHARE, DEAL_SPLIT };
constexpr int DEAL_SORT_MAX = 224;   // sequences that a block ranks, one a thread of all warps but the first
constexpr float END_COST = 4.f, SHARE_COST = 5.f, SPLIT_COST = 16.f;   // steps

struct DealMem {
  int *order, *pre;   // [B] sequences by falling length, [B + 1] items before each (SHARE: blocks)
  int items;
};
// SHARE: blocks of an item of `steps` out of `units`.  Their sum is no more than
// there are, and no item has more than shorten it: the join takes an eighth of
// a step a block.
__device__ __forceinline__ int blocks_of(int steps, int units, int items, int blocks, int warps) {
  const int most = 1 + (int)sqrtf(8.f * steps / warps);
  return min(min(steps, most), 1 + (int)((long long)(blocks - items) * steps / units));
}
constexpr size_t deal_bytes(int B) { return B <= DEAL_SORT_MAX ? ((size_t)B * 12 + 4 + 16 + 15) / 16 * 16 : 0; }

// The lengths, the units' prefix sums and the deal, the same in every block.
template <typename C, int KS>
__device__ __forceinline__ Deal make_plan(const AttendArgs& a, unsigned char* smem, WorkPlan& plan, PlanMem& mem, DealMem& dm) {
  constexpr int TR = C::TR, WARPS = C::WARPS;
  __shared__ int s_long, s_items;
  const int B = a.c.batch, tid = threadIdx.x, lane = tid & 31;
  const bool sort = B <= DEAL_SORT_MAX;
  mem.lens = reinterpret_cast<int2*>(smem);
  mem.pre = reinterpret_cast<int*>(mem.lens + B);
  int* steps = reinterpret_cast<int*>(smem + plan_bytes(B));   // [B], filled up to whole vectors
  dm.order = steps + (B + 3) / 4 * 4;
  dm.pre = dm.order + B;
  auto work = [&](int b) { return seq_work<KS, TR>(a.r, mem.lens[b].x, mem.lens[b].y); };
  for (int b = tid; b < B; b += blockDim.x) {
    paged_lens(a.c, a.r, b, mem.lens[b].x, mem.lens[b].y);
    const SeqWork s = work(b);
    mem.pre[b + 1] = a.c.kv_heads * s.tiles * s.steps;
    if (sort) steps[b] = s.steps;
  }
  if (sort && tid < 4 && B + tid < (B + 3) / 4 * 4) steps[B + tid] = -1;
  __syncthreads();
  if (tid < 32) {
    int base = 0, most = 0, items = 0;
    for (int b0 = 0; b0 < B; b0 += 32) {
      int x = 0;
      if (b0 + lane < B) {
        x = mem.pre[b0 + lane + 1];
        const SeqWork s = work(b0 + lane);
        most = max(most, s.steps);
        items += s.steps ? a.c.kv_heads * s.tiles : 0;
      }
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
      }
      if (b0 + lane < B) mem.pre[b0 + lane + 1] = base + x;
      base += __shfl_sync(0xffffffffu, x, 31);
    }
    most = __reduce_max_sync(0xffffffffu, most);
    items = __reduce_add_sync(0xffffffffu, items);
    if (lane == 0) mem.pre[0] = 0, s_long = most, s_items = items;
  } else if (sort && tid - 32 < B) {
    const int b = tid - 32, mine = steps[b];
    int rank = 0;
    for (int x = 0; x < B; x += 4) {
      const int4 y = *reinterpret_cast<const int4*>(steps + x);
      rank += (y.x > mine || (y.x == mine && x < b)) + (y.y > mine || (y.y == mine && x + 1 < b)) +
              (y.z > mine || (y.z == mine && x + 2 < b)) + (y.w > mine || (y.w == mine && x + 3 < b));
    }
    dm.order[rank] = b;
  }
  __syncthreads();
  plan.units = mem.pre[B];
  plan.workers = max(1, min(plan.units, a.max_workers));
  plan.share = plan.units / plan.workers;
  plan.more = plan.units - plan.share * plan.workers;
  dm.items = s_items;
  if (!sort) return DEAL_SPLIT;
  const float u = (float)plan.units, n = (float)s_items, longest = (float)s_long;
  const float warps = (float)a.max_workers, blocks = warps / WARPS;
  const float by_warp = fmaxf(longest + END_COST, n <= warps ? 0.f : 1.1f * (u + END_COST * n) / warps);
  const float by_block = fmaxf(longest / WARPS + END_COST + 1.f,
                               n <= blocks ? 0.f : 1.1f * (u / WARPS + (END_COST + 1.f) * n) / blocks);
  const int grid = a.max_workers / WARPS;
  const float by_share = dm.items > 0 && 2 * dm.items <= grid
                             ? longest / (WARPS * blocks_of(s_long, plan.units, dm.items, grid, WARPS)) + END_COST + 1.f + SHARE_COST
                             : 1e30f;
  const float split = u / warps + END_COST + SPLIT_COST;
  const float least = fminf(fminf(by_warp, by_block), fminf(by_share, split));
  const Deal deal = least == split ? DEAL_SPLIT : least == by_warp ? DEAL_WARP : least == by_block ? DEAL_BLOCK : DEAL_SHARE;
  if (deal == DEAL_SPLIT) return deal;
  if (tid < 32) {
    int base = 0;
    for (int b0 = 0; b0 < B; b0 += 32) {
      int x = 0;
      if (b0 + lane < B) {
        const SeqWork s = work(dm.order[b0 + lane]);
        x = s.steps ? a.c.kv_heads * s.tiles : 0;
        if (x && deal == DEAL_SHARE) x *= blocks_of(s.steps, plan.units, dm.items, grid, WARPS);
      }
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
      }
      if (b0 + lane < B) dm.pre[b0 + lane + 1] = base + x;
      base += __shfl_sync(0xffffffffu, x, 31);
    }
    if (lane == 0) dm.pre[0] = 0;
  }
  __syncthreads();
  return deal;
}

// What the two kernels below share: the plan, the walk over a warp's items and
// their ends.  `item` computes steps [s0, s0 + n) of one item and leaves the
// result in the warp's shared memory.
template <typename T, typename C, int KS, typename F>
__device__ __forceinline__ void attend_items(const AttendArgs& a, F item) {
  constexpr int REGION = C::REGION, D = C::D, TR = C::TR, WARPS = C::WARPS;
  const PagedView& c = a.c;
  const PagedRows& r = a.r;
  extern __shared__ __align__(16) unsigned char smem[];
  WorkPlan plan;
  PlanMem mem;
  DealMem dm;
  const Deal deal = make_plan<C, KS>(a, smem, plan, mem, dm);
  clear_rows<T, D>(a, mem);
  if (plan.units == 0) return;
  float* sm = reinterpret_cast<float*>(smem + plan_bytes(c.batch) + deal_bytes(c.batch));
  const int warp = threadIdx.x >> 5, w0 = blockIdx.x * WARPS, worker = w0 + warp;

  // SPLIT: this warp's run of units [u, u_end), the block's [block0, block1)
  const int w1 = min(w0 + WARPS, plan.workers), block0 = plan.start(min(w0, plan.workers)), block1 = plan.start(w1);
  int u = worker < plan.workers ? plan.start(worker) : block1;
  const int u_end = worker < plan.workers ? plan.start(worker + 1) : block1;
  if (deal == DEAL_SPLIT && w0 >= plan.workers) return;
  // WARP, BLOCK: taker and takers; consecutive items go to different SMs
  const int takers = deal == DEAL_WARP ? a.max_workers : gridDim.x;
  const int taker = deal == DEAL_WARP ? warp * gridDim.x + blockIdx.x : blockIdx.x;
  const int shares = deal == DEAL_SHARE ? dm.pre[c.batch] : dm.items;   // what dm.pre counts
  int share = 0, place = 0;   // SHARE: blocks of an item, this one's place among them
  bool team = deal != DEAL_WARP;   // all warps of the block work on one item
  for (int round = 0, at = block0;;) {
    int b, it, u0 = 0, u1 = 0, s0, n, active = WARPS;
    SeqWork s;
    if (deal == DEAL_SPLIT) {
      b = work_find(mem.pre, c.batch, at);
      s = seq_work<KS, TR>(r, mem.lens[b].x, mem.lens[b].y);
      it = (at - mem.pre[b]) / s.steps;
      u0 = mem.pre[b] + it * s.steps, u1 = u0 + s.steps;
      if (team && block1 > u1) {   // uniform over the block, at its first item only
        team = false;
        if (worker >= plan.workers) return;
        if (u > block0) {
          at = u;
          continue;
        }
      }
      s0 = u - u0, n = min(u1, u_end) - u;
      active = w1 - w0;
    } else {
      const int k = round * takers + (round & 1 ? takers - 1 - taker : taker);
      if (k >= shares) return;
      ++round;
      const int rank = work_find(dm.pre, c.batch, k);
      b = dm.order[rank];
      it = k - dm.pre[rank];
      s = seq_work<KS, TR>(r, mem.lens[b].x, mem.lens[b].y);
      s0 = 0, n = s.steps;
      if (deal == DEAL_SHARE) {
        share = blocks_of(s.steps, plan.units, dm.items, gridDim.x, WARPS);
        place = it % share;
        it /= share;
        u0 = (int)blockIdx.x - place;
        s0 = (int)((long long)s.steps * place / share);
        n = (int)((long long)s.steps * (place + 1) / share) - s0;
      }
      if (team) {
        active = min(WARPS, n);
        const int w_0 = n * min(warp, active) / active, w_1 = n * min(warp + 1, active) / active;
        s0 += w_0;
        n = w_1 - w_0;
      }
    }
    const int kvh = it / s.tiles, tile = it - kvh * s.tiles;
    if (n > 0) item(s, b, kvh, tile, s0, n, sm + warp * REGION);
    if (team) {
      const bool whole = deal == DEAL_BLOCK || (share ? share == 1 : block0 == u0 && block1 == u1);
      finish_item<T, C, true>(a, plan, sm, active, b, kvh, tile, s.rows * r.group, u0, u1, w0, share ? place == 0 : block0 == u0,
                              whole, share);
      if (deal != DEAL_BLOCK) return;
    } else {
      finish_item<T, C, false>(a, plan, sm + warp * REGION, 1, b, kvh, tile, s.rows * r.group, u0, u1, worker, s0 == 0,
                                   n == s.steps, 0);
      at = u += n;
      if (deal == DEAL_SPLIT && u >= u_end) return;
    }
  }
}

inline int attend_grid() {
  const int most = MAX_WORKERS / 12, sms = paged_sm_count();
  return sms < most ? sms : most;
}

}  // namespace
}  // namespace asrspec
