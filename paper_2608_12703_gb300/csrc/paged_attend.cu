// Attention of a block of new rows over a paged K/V cache, with the append of
// the block's K/V.
//
//   o_r = sum_j p_rj v_j,  p_rj = exp(scale q_r k_j - lse_r),  lse_r = log sum_j exp(scale q_r k_j)
//
// over the slots j that row r sees: j <= kv_len + r (causal) or j < kv_len.
// A slot's K and V are read once for a tile of rows, so the operator is bound
// by the bytes of the cache; the layout follows from that:
//   * a warp works alone, with no block barrier in the key loop.  It keeps a
//     tile of rows (the block's rows times the query heads that share a K/V
//     head) as mma A fragments.  Steps of K and V come by bulk copies, one a
//     run of slots in a page, into a ring of the warp's own, two or three steps
//     ahead (16 to 24 KB a warp, 192 KB an SM), and from there 16 bytes a lane
//     into B fragments.  The contraction index of q k and the output index of
//     p v may be permuted freely, so the permutations are chosen for these
//     reads: of a key a lane takes d = 32 j + 8 c .. + 7 (c = lane mod 4), which
//     are the operand pairs of two k-steps; of a value row it takes d = 8 g ..
//     + 7 (g = lane / 4), one element for each of eight n-tiles, paired with
//     its neighbour key by byte permutes.  mma.sync, not tcgen05: a tile has 1
//     to 32 rows, and the tensor pipe is far from its limit;
//   * who works on what is chosen from the lengths (make_plan).  Warps of a
//     block that all work on one item combine in shared memory; where an item
//     has several such partial results they go through the workspace, and
//     whoever delivers the last one joins them, in key order, so results do
//     not depend on timing;
//   * committed slots are read from the pages and the block's own rows from
//     k_new / v_new; one warp also copies those to the pages (nobody uses a
//     page's slot that this launch writes).
// Measured (device time, inputs of one call in L2 where they fit): 48 sequences
// of up to 40000 slots, 32 query heads on 8 of 128, fp16: 587 - 625 us for 3.95
// GB, 6.3 - 6.7 TB/s, the copy rate; one of 100001 slots, 9 rows, 20 heads of
// 64, bf16: 97 us for 512 MB, 76 of them the key loop at 6.7 TB/s, the rest
// launch, plan, uneven ends and the join; 64 of up to 448 slots, 7 rows, 20
// heads: 30 us for 78 MB, of which 14 steps of 1.3 us in the longest warp and 9
// us launch, plan and end; one of 230 slots: 10 us, all of it latency.
// Scores, running maximum and sum, and the output accumulate in fp32.  p is
// rounded to the cache's 16-bit type for the second product (relative error at
// most 2^-8 for bf16 and 2^-11 for fp16 a weight, as that of the rounded
// output); the sum takes p before rounding, so that rounding does not reach lse,
// which has those of fp32 sums and of the hardware's exp2 and log2, some 2^-20.
// fp16 has 5 bits of exponent: there p is taken relative to the strongest key
// times 2^15, the top of the type's range, so that it keeps its precision down
// to 2^-29 and vanishes below 2^-40 only.  The maximum is subtracted before the
// scale is applied: the rounding of a large scaled maximum (scores past 2^31)
// would move every p by powers of two, out of the types' range or to 0.
#include <atomic>
#include <type_traits>

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

// The halves of a pair of 16-bit values that are infinite or NaN, as a mask.
template <typename T>
__device__ __forceinline__ uint32_t nonfinite_halves(uint32_t x) {
  constexpr uint32_t E = std::is_same<T, __half>::value ? 0x7c00u : 0x7f80u;
  return ((x & E) == E ? 0xffffu : 0u) | (((x >> 16) & E) == E ? 0xffff0000u : 0u);
}

// The strongest key's weight in the second product, 2^log2.
template <typename T> struct TopWeight { static constexpr float log2 = 0.f, inv = 1.f; };
template <> struct TopWeight<__half> { static constexpr float log2 = 15.f, inv = 1.f / 32768.f; };

template <typename T> struct Pair;
template <> struct Pair<__nv_bfloat16> {
  using type = __nv_bfloat162;
  static __device__ __forceinline__ type zero() { return __float2bfloat162_rn(0.f); }
  static __device__ __forceinline__ type add_zero(uint32_t x, type s) {
    return __hfma2(*reinterpret_cast<const type*>(&x), zero(), s);
  }
};
template <> struct Pair<__half> {
  using type = __half2;
  static __device__ __forceinline__ type zero() { return __float2half2_rn(0.f); }
  static __device__ __forceinline__ type add_zero(uint32_t x, type s) {
    return __hfma2(*reinterpret_cast<const type*>(&x), zero(), s);
  }
};

__device__ __forceinline__ uint32_t reg_of(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// A key of an edge step may be hidden from some of the tile's rows, and a hidden
// value takes part in the product with weight 0: an infinity or NaN there would
// reach rows that do not see it.  Such values are taken out of the fragments
// and added to the rows that do see them.
template <typename T, int D, int MT, int E>
__device__ __forceinline__ void guard_values(const Keys16<T, D>& ks, int step, const int (&lim)[MT][E],
                                             uint4 (&vf)[Keys16<T, D>::NG][4][D / 64], float (&O)[MT][D / 8][4]) {
  using K = Keys16<T, D>;
  // x * 0 is NaN for an infinity or NaN, and stays in the sum
  typename Pair<T>::type sum = Pair<T>::zero();
#pragma unroll
  for (int u = 0; u < K::NG; ++u)
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll
      for (int j = 0; j < K::NV; ++j) {
        const uint4& v = vf[u][w][j];
        sum = Pair<T>::add_zero(v.w, Pair<T>::add_zero(v.z, Pair<T>::add_zero(v.y, Pair<T>::add_zero(v.x, sum))));
      }
  if (!__any_sync(0xffffffffu, nonfinite_halves<T>(*reinterpret_cast<uint32_t*>(&sum)) != 0)) return;
#pragma unroll
  for (int u = 0; u < K::NG; ++u)
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll
      for (int j = 0; j < K::NV; ++j) {
        uint4& v = vf[u][w][j];
        v.x &= ~nonfinite_halves<T>(v.x), v.y &= ~nonfinite_halves<T>(v.y);
        v.z &= ~nonfinite_halves<T>(v.z), v.w &= ~nonfinite_halves<T>(v.w);
      }
  for (int key = step * K::KS; key < min((step + 1) * K::KS, ks.s.keys); ++key) {
    const int grp = key / PG_GROUP;
    const char* row = key >= ks.s.paged
                          ? ks.vn + (long long)(key - ks.s.paged) * ks.r.n_r
                          : ks.c.v + paged_offset(ks.c, paged_id(ks.c, ks.table_row, grp), grp) + ks.head_off +
                                (key % PG_GROUP) * ks.c.slot_stride;
#pragma unroll
    for (int d = 0; d < D / 8; ++d)
#pragma unroll
      for (int x = 0; x < 2; ++x) {   // the lane's output columns (see the n-tiles of the second product)
        const float v = to_f32(reinterpret_cast<const T*>(row)[(d / 8) * 64 + ks.t * 16 + x * 8 + d % 8]);
        if (isfinite(v)) continue;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int e = 0; e < E; ++e)
            if (key < lim[mt][e]) O[mt][d][2 * e + x] += v;
      }
  }
}

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

// MT m-tiles of 8 E rows: up to 8 rows use half of one (E = 1), the softmax of
// the other half is left out.
template <typename T, typename C, int MT, int E>
__global__ void __launch_bounds__(C::WARPS * 32, 1) attend16_kernel(AttendArgs a) {
  constexpr int D = C::D, KS = Cfg16<D>::KS, NG = KS / PG_GROUP, NC = D / 32, NV = D / 64, TR = C::TR, STAGES = C::STAGES;
  static_assert(TR == 8 * E * MT && KS * D * 4 == 8192, "");
  const PagedView& c = a.c;
  const PagedRows& r = a.r;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const float sc = r.scale * LOG2E;
  __shared__ __align__(8) uint64_t bars[C::WARPS][STAGES][2];   // K and V of a stage have landed
  uint64_t(*bar)[2] = bars[threadIdx.x >> 5];
  if (lane < 2 * STAGES) mbar_init(&bar[lane >> 1][lane & 1], 1);
  fence_mbar_init();
  __syncwarp();
  uint32_t phases = 0;   // a bit a stage
  bool gave_up = false;

  attend_items<T, C, KS>(a, [&](const SeqWork& s, int b, int kvh, int tile, int s0, int n, float* sm) {
    const long long new_off = b * r.n_b + kvh * r.n_h;
    Keys16<T, D> ks{c, r, s, c.table + b * c.table_stride, kvh * c.head_stride, r.k_new + new_off, r.v_new + new_off, g, t};
    constexpr int KB = KS * D * 2;   // bytes of a step's K, and of its V
    const uint32_t ring = smem_u32(sm);
    Groups<T, D> groups(ks, s0);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // results were written here before
    __syncwarp();
#pragma unroll
    for (int i = 0; i < STAGES; ++i) {
      if (i < n) {
        const int at = groups.at(i);
        ks.fetch(s0 + i, c.k, ks.kn, groups.off, at, ring + i * 2 * KB, &bar[i][0]);
        ks.fetch(s0 + i, c.v, ks.vn, groups.off, at, ring + i * 2 * KB + KB, &bar[i][1]);
      }
    }

    uint32_t qa[MT][NC * 2][4];
    int lim[MT][E];   // slots that the fragment's rows see
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int m = tile * TR + mt * 8 * E + e * 8 + g, row = m / r.group, hq = kvh * r.group + m - row * r.group;
        lim[mt][e] = min(s.keys, r.causal ? s.len + row + 1 : s.len);
#pragma unroll
        for (int j = 0; j < NC; ++j) {
          const uint4 x = ldg_if(row < s.rows, r.q + b * r.q_b + row * r.q_r + hq * r.q_h + j * 64 + t * 16);
          qa[mt][2 * j][e] = x.x;
          qa[mt][2 * j][2 + e] = x.y;
          qa[mt][2 * j + 1][e] = x.z;
          qa[mt][2 * j + 1][2 + e] = x.w;
          if (E == 1) qa[mt][2 * j][1] = qa[mt][2 * j][3] = qa[mt][2 * j + 1][1] = qa[mt][2 * j + 1][3] = 0;
        }
      }
    using W = TopWeight<T>;
    float O[MT][D / 8][4], m_run[MT][E], l_run[MT][E];   // the maximum before the scale; sum and output times the top weight
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
      for (int e = 0; e < E; ++e) m_run[mt][e] = -INFINITY, l_run[mt][e] = 0.f;
#pragma unroll
      for (int d = 0; d < D / 8; ++d) O[mt][d][0] = O[mt][d][1] = O[mt][d][2] = O[mt][d][3] = 0.f;
    }

    int stage = 0;
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
      const int step = s0 + i;
      const bool full = ks.full(step), more = i + STAGES < n;
      const uint32_t slot = ring + stage * 2 * KB, parity = phases >> stage & 1;
      uint64_t* landed = bar[stage];
      phases ^= 1u << stage;
      stage = stage + 1 == STAGES ? 0 : stage + 1;
      float S[MT][KS / 8][4];
      bar_wait(&landed[0], parity, c.status, gave_up);
      {
        const uint32_t at = slot + g * (D * 2) + t * 16;
#pragma unroll
        for (int kt = 0; kt < KS / 8; ++kt) {
          uint4 kf[NC];
#pragma unroll
          for (int j = 0; j < NC; ++j) kf[j] = lds16(at + kt * 8 * (D * 2) + j * 64);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            S[mt][kt][0] = S[mt][kt][1] = S[mt][kt][2] = S[mt][kt][3] = 0.f;
#pragma unroll
            for (int j = 0; j < NC; ++j) {
              Mma16<T>::mma(S[mt][kt], qa[mt][2 * j], kf[j].x, kf[j].y);
              Mma16<T>::mma(S[mt][kt], qa[mt][2 * j + 1], kf[j].z, kf[j].w);
            }
          }
        }
      }
      __syncwarp();   // all lanes have read the slot
      int at = 0;
      if (more) {
        at = groups.at(i + STAGES);
        ks.fetch(step + STAGES, c.k, ks.kn, groups.off, at, slot, &landed[0]);
      }
      if (!full) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int kt = 0; kt < KS / 8; ++kt)
#pragma unroll
            for (int x = 0; x < 2 * E; ++x)
              if (step * KS + kt * 8 + 2 * t + (x & 1) >= lim[mt][x >> 1]) S[mt][kt][x] = -INFINITY;
      }
      uint32_t pf[MT][KS / 8][E];
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        float mx[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
          float x = fmaxf(S[mt][0][2 * e], S[mt][0][2 * e + 1]);
#pragma unroll
          for (int kt = 1; kt < KS / 8; ++kt) x = fmaxf(x, fmaxf(S[mt][kt][2 * e], S[mt][kt][2 * e + 1]));
          x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
          x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
          mx[e] = fmaxf(m_run[mt][e], x);
        }
        if (__any_sync(0xffffffffu, mx[0] > m_run[mt][0] || mx[E - 1] > m_run[mt][E - 1])) {
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float f = mx[e] == -INFINITY ? 1.f : ex2((m_run[mt][e] - mx[e]) * sc);
            m_run[mt][e] = mx[e];
            l_run[mt][e] *= f;
#pragma unroll
            for (int d = 0; d < D / 8; ++d) {
              O[mt][d][2 * e] *= f;
              O[mt][d][2 * e + 1] *= f;
            }
          }
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float m = m_run[mt][e] == -INFINITY ? 0.f : m_run[mt][e];
#pragma unroll
          for (int kt = 0; kt < KS / 8; ++kt) {
            const float p0 = ex2(fmaf(S[mt][kt][2 * e] - m, sc, W::log2)), p1 = ex2(fmaf(S[mt][kt][2 * e + 1] - m, sc, W::log2));
            l_run[mt][e] += p0 + p1;
            pf[mt][kt][e] = Mma16<T>::pack(p0, p1);
          }
        }
      }
      bar_wait(&landed[1], parity, c.status, gave_up);
      uint4 vf[NG][4][NV];
      {
        const uint32_t at = slot + KB + 2 * t * (D * 2) + g * 16;
#pragma unroll
        for (int x = 0; x < NG; ++x)
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const int in = x * PG_GROUP + (w & 1) + (w >> 1) * 8;
#pragma unroll
            for (int j = 0; j < NV; ++j) vf[x][w][j] = lds16(at + in * (D * 2) + j * 128);
            if (!full && step * KS + in + 2 * t >= s.keys)   // past the end: whatever the slot held
#pragma unroll
              for (int j = 0; j < NV; ++j) vf[x][w][j] = make_uint4(0, 0, 0, 0);
          }
      }
      if (!full && s.keys > s.len) guard_values<T, D, MT, E>(ks, step, lim, vf, O);
#pragma unroll
      for (int x = 0; x < NG; ++x)
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int d = 0; d < 8; ++d) {   // n-tile d of half j: output column 64 j + 8 n + d
            const uint32_t sel = d & 1 ? 0x7632 : 0x5410;
            const uint32_t b0 = __byte_perm(reg_of(vf[x][0][j], d >> 1), reg_of(vf[x][1][j], d >> 1), sel);
            const uint32_t b1 = __byte_perm(reg_of(vf[x][2][j], d >> 1), reg_of(vf[x][3][j], d >> 1), sel);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
              const uint32_t pa[4] = {pf[mt][2 * x][0], E > 1 ? pf[mt][2 * x][E - 1] : 0u, pf[mt][2 * x + 1][0],
                                      E > 1 ? pf[mt][2 * x + 1][E - 1] : 0u};
              Mma16<T>::mma(O[mt][j * 8 + d], pa, b0, b1);
            }
          }
      __syncwarp();
      if (more) ks.fetch(step + STAGES, c.v, ks.vn, groups.off, at, slot + KB, &landed[1]);
    }
    if (tile == 0 && s.keys > s.paged && s0 <= s.paged / KS && s.paged / KS < s0 + n) append_rows(c, r, s, b, kvh, D * sizeof(T));

    // of row g (+ 8 e) a lane holds columns 64 j + 16 t .. + 15
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        float l = l_run[mt][e];
        l += __shfl_xor_sync(0xffffffffu, l, 1);
        l += __shfl_xor_sync(0xffffffffu, l, 2);
        m_run[mt][e] *= sc;
        if constexpr (W::log2 != 0.f) {
          l *= W::inv;
#pragma unroll
          for (int d = 0; d < D / 8; ++d) O[mt][d][2 * e] *= W::inv, O[mt][d][2 * e + 1] *= W::inv;
        }
        const int in = mt * 8 * E + e * 8 + g;
        if (t == 0) {
          sm[in] = m_run[mt][e];
          sm[TR + in] = l;
        }
        float* o = sm + 2 * TR + in * D;
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int d = 0; d < 8; d += 4)
              *reinterpret_cast<float4*>(o + j * 64 + t * 16 + x * 8 + d) =
                  make_float4(O[mt][j * 8 + d][2 * e + x], O[mt][j * 8 + d + 1][2 * e + x], O[mt][j * 8 + d + 2][2 * e + x],
                              O[mt][j * 8 + d + 3][2 * e + x]);
      }
  });
}

// fp32: plain fp32 products (no TF32), four rows a warp.  Eight lanes share a
// key (lane e of them takes the 16-byte chunks e, e + 8, ..), four keys at a
// time; each group of eight lanes keeps its own running maximum, sum and
// output over its keys, combined at the end of the item.
template <typename C>
__global__ void __launch_bounds__(C::WARPS * 32, 1) attend32_kernel(AttendArgs a) {
  constexpr int D = C::D, TR = C::TR, KS = D == 64 ? 16 : 8, IT = KS / 4, NC = D / 32;
  const PagedView& c = a.c;
  const PagedRows& r = a.r;
  const int lane = threadIdx.x & 31, kg = lane >> 3, e = lane & 7;
  const float sc = r.scale * LOG2E;

  attend_items<float, C, KS>(a, [&](const SeqWork& s, int b, int kvh, int tile, int s0, int n, float* sm) {
    const int* table_row = c.table + b * c.table_stride;
    float q[TR][NC * 4], O[TR][NC * 4], m_run[TR], l_run[TR];
    int lim[TR];
#pragma unroll
    for (int x = 0; x < TR; ++x) {
      const int m = tile * TR + x, row = m / r.group, hq = kvh * r.group + m - row * r.group;
      lim[x] = row < s.rows ? min(s.keys, r.causal ? s.len + row + 1 : s.len) : 0;
      m_run[x] = -INFINITY;
      l_run[x] = 0.f;
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        const float4 v = row < s.rows ? __ldg(reinterpret_cast<const float4*>(r.q + b * r.q_b + row * r.q_r +
                                                                              hq * r.q_h + (e + 8 * j) * 16))
                                      : make_float4(0.f, 0.f, 0.f, 0.f);
        q[x][4 * j] = v.x * sc, q[x][4 * j + 1] = v.y * sc, q[x][4 * j + 2] = v.z * sc, q[x][4 * j + 3] = v.w * sc;
        O[x][4 * j] = O[x][4 * j + 1] = O[x][4 * j + 2] = O[x][4 * j + 3] = 0.f;
      }
    }
    for (int i = 0; i < n; ++i) {
      const int step = s0 + i;
      const int first = step * KS;
      long long page = 0;
      if (first < s.paged) {
        const int grp = first / PG_GROUP;
        page = paged_offset(c, paged_id(c, table_row, grp), grp) + kvh * c.head_stride + (first % PG_GROUP) * c.slot_stride;
      }
      float4 kf[IT][NC], vf[IT][NC];
#pragma unroll
      for (int k = 0; k < IT; ++k) {
        const int key = first + 4 * k + kg;
        const bool in_page = key < s.paged;
        const long long at = (in_page ? page + (4 * k + kg) * c.slot_stride
                                      : b * r.n_b + kvh * r.n_h + (long long)(key - s.paged) * r.n_r) + e * 16;
        const char *kp = (in_page ? c.k : r.k_new) + at, *vp = (in_page ? c.v : r.v_new) + at;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
          const uint4 x = ldg_if(key < s.keys, kp + j * 128), y = ldg_if(key < s.keys, vp + j * 128);
          kf[k][j] = *reinterpret_cast<const float4*>(&x);
          vf[k][j] = *reinterpret_cast<const float4*>(&y);
        }
      }
#pragma unroll
      for (int x = 0; x < TR; ++x) {
        float S[IT], mx = m_run[x];
#pragma unroll
        for (int k = 0; k < IT; ++k) {
          float d = 0.f;
#pragma unroll
          for (int j = 0; j < NC; ++j)
            d += (q[x][4 * j] * kf[k][j].x + q[x][4 * j + 1] * kf[k][j].y) +
                 (q[x][4 * j + 2] * kf[k][j].z + q[x][4 * j + 3] * kf[k][j].w);
          d += __shfl_xor_sync(0xffffffffu, d, 1);
          d += __shfl_xor_sync(0xffffffffu, d, 2);
          d += __shfl_xor_sync(0xffffffffu, d, 4);
          S[k] = first + 4 * k + kg < lim[x] ? d : -INFINITY;
          mx = fmaxf(mx, S[k]);
        }
        const float m = mx == -INFINITY ? 0.f : mx, f = ex2(m_run[x] - m);
        m_run[x] = mx;
        l_run[x] *= f;
#pragma unroll
        for (int j = 0; j < NC * 4; ++j) O[x][j] *= f;
#pragma unroll
        for (int k = 0; k < IT; ++k) {
          const float p = ex2(S[k] - m);
          l_run[x] += p;
          if (first + 4 * k + kg >= lim[x]) continue;   // hidden: an infinity or NaN there must not reach the row
#pragma unroll
          for (int j = 0; j < NC; ++j) {
            O[x][4 * j] += p * vf[k][j].x;
            O[x][4 * j + 1] += p * vf[k][j].y;
            O[x][4 * j + 2] += p * vf[k][j].z;
            O[x][4 * j + 3] += p * vf[k][j].w;
          }
        }
      }
    }
    if (tile == 0 && s.keys > s.paged && s0 <= s.paged / KS && s.paged / KS < s0 + n) append_rows(c, r, s, b, kvh, D * sizeof(float));
#pragma unroll
    for (int x = 0; x < TR; ++x) {
      float mx = fmaxf(m_run[x], __shfl_xor_sync(0xffffffffu, m_run[x], 8));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
      const float f = mx == -INFINITY ? 0.f : ex2(m_run[x] - mx);
      float l = l_run[x] * f;
      l += __shfl_xor_sync(0xffffffffu, l, 8);
      l += __shfl_xor_sync(0xffffffffu, l, 16);
#pragma unroll
      for (int j = 0; j < NC * 4; ++j) {
        float o = O[x][j] * f;
        o += __shfl_xor_sync(0xffffffffu, o, 8);
        o += __shfl_xor_sync(0xffffffffu, o, 16);
        O[x][j] = o;
      }
      if (kg != 0) continue;
      if (e == 0) {
        sm[x] = mx;
        sm[TR + x] = l;
      }
      float4* o = reinterpret_cast<float4*>(sm + 2 * TR + x * D);
#pragma unroll
      for (int j = 0; j < NC; ++j) o[e + 8 * j] = make_float4(O[x][4 * j], O[x][4 * j + 1], O[x][4 * j + 2], O[x][4 * j + 3]);
    }
  });
}

// Rows up to 8, 16 and 32 a tile; 12 warps where their registers allow it (a
// warp's step is a chain of dependent instructions, which other warps fill).
using S64x8 = Shape<64, 8, 12, 2>;
using S64x16 = Shape<64, 16, 12, 2>;
using S64x32 = Shape<64, 32, 8, 3>;
using S128x8 = Shape<128, 8, 8, 3>;
using S128x16 = Shape<128, 16, 8, 3>;
using F64x4 = Shape<64, 4, 8, 0>;
using F128x4 = Shape<128, 4, 8, 0>;

int attend_grid() {
  const int most = MAX_WORKERS / 12, sms = paged_sm_count();
  return sms < most ? sms : most;
}

// What a call does with the shape that its type, head dimension and rows ask for.
template <typename F>
auto with_shape(int dtype, int dim, int m_rows, F f) {
  if (dtype == 0) return dim == 64 ? f(F64x4{}) : f(F128x4{});
  if (dim == 128) return m_rows <= 8 ? f(S128x8{}) : f(S128x16{});
  return m_rows <= 8 ? f(S64x8{}) : m_rows <= 16 ? f(S64x16{}) : f(S64x32{});
}

int64_t attend_ws_bytes(int dtype, int dim, int m_rows) {
  return with_shape(dtype, dim, m_rows, [](auto s) {
    return (int64_t)MAX_WORKERS * 4 + (int64_t)attend_grid() * s.WARPS * 2 * s.PART * 4;
  });
}

// One block an SM.  The shared memory above 48 KB that a kernel needs is asked for once a device.
template <auto kernel, typename C>
cudaError_t launch_attend(AttendArgs& a, cudaStream_t st) {
  constexpr size_t REGIONS = (size_t)C::WARPS * C::REGION * 4;
  static std::atomic<uint64_t> ready{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (!(ready.load(std::memory_order_acquire) & bit)) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             (int)(REGIONS + plan_bytes(PG_MAX_BATCH) + deal_bytes(DEAL_SORT_MAX)));
    if (e != cudaSuccess) return e;
    ready.fetch_or(bit, std::memory_order_release);
  }
  const int grid = attend_grid();
  a.max_workers = grid * C::WARPS;
  kernel<<<grid, C::WARPS * 32, REGIONS + plan_bytes(a.c.batch) + deal_bytes(a.c.batch), st>>>(a);
  return cudaGetLastError();
}

template <typename T, typename C>
cudaError_t launch_shape(AttendArgs& a, cudaStream_t st) {
  if constexpr (C::TR == 4) return launch_attend<attend32_kernel<C>, C>(a, st);
  else return launch_attend<attend16_kernel<T, C, C::TR == 32 ? 2 : 1, C::TR == 8 ? 1 : 2>, C>(a, st);
}

}  // namespace
}  // namespace asrspec

using namespace asrspec;

extern "C" {

int64_t asr_spec_paged_attend_ws(const asr_paged_cache* c, const asr_paged_rows* r) {
  PagedView v;
  PagedRows w;
  if (int rc = paged_view(c, &v)) return rc;
  if (int rc = paged_rows(c, r, &w)) return rc;
  return attend_ws_bytes(c->dtype, c->head_dim, w.max_rows * w.group);
}

int asr_spec_paged_attend(const asr_paged_cache* c, const asr_paged_rows* r, void* out, float* lse, void* ws,
                          int64_t ws_bytes, void* stream) {
  AttendArgs a{};
  if (int rc = paged_view(c, &a.c)) return rc;
  if (int rc = paged_rows(c, r, &a.r)) return rc;
  if (!out || !ws || ((uintptr_t)out | (uintptr_t)ws) % 16 || (uintptr_t)lse % 4) return ASR_E_INVAL;
  const int m_rows = a.r.max_rows * a.r.group;
  if (ws_bytes < attend_ws_bytes(c->dtype, c->head_dim, m_rows)) return ASR_E_CAPACITY;
  const int tr = with_shape(c->dtype, c->head_dim, m_rows, [](auto s) { return s.TR; });
  const long long tiles = ((long long)m_rows + tr - 1) / tr;
  if (tiles * c->kv_heads * c->batch * ((long long)a.c.max_slots / 8 + a.r.max_rows / 8 + 2) > 0x7fffffffll)
    return ASR_E_CAPACITY;   // 32-bit units
  a.out = static_cast<char*>(out);
  a.lse = lse;
  a.tickets = static_cast<int*>(ws);
  a.ws = reinterpret_cast<float*>(a.tickets + MAX_WORKERS);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = with_shape(c->dtype, c->head_dim, m_rows, [&](auto s) {
    using C = decltype(s);
    if constexpr (C::TR == 4) return launch_shape<float, C>(a, st);
    else return c->dtype == 1 ? launch_shape<__nv_bfloat16, C>(a, st) : launch_shape<__half, C>(a, st);
  });
  return e == cudaSuccess ? ASR_OK : ASR_E_CUDA;
}

}  // extern "C"
