// Attention of prompts over an 8-bit paged cache: many rows a sequence, so that
// the tensor cores and the exponentials bound it and not the cache's bytes.
//
// One block an SM.  An item is 256 rows of a sequence and K/V head (its rows
// times the query heads that share the head), as two tiles of 128; a block goes
// through its items without a break, each part of it at its own pace, in tiles of 128 keys:
//   * 3 warps turn codes into fp16 in 128-byte-swizzled shared memory, two
//     stages of K and of V, a tile's loads in flight while the one before is
//     converted; both row tiles use what they write;
//   * one warp issues tcgen05.mma: S = q K^T (128 x 128, fp32 in tensor
//     memory) and O += p V with p read from tensor memory: beside the scores for
//     heads of 64, in their place for heads of 128, whose outputs leave no more
//     room. The two row tiles alternate, so that one's products
//     run while the other's scores are being weighed, and scores run ahead;
//   * 4 warps a row tile, a thread a row, weigh the scores by the maximum and
//     the reference of the weights (as in the kernel for few rows) of the tiles
//     before.  Those move only where a weight would leave [.., 2^15] or p grow
//     past 2^4, which after the first tiles is rare; the output is then rescaled in place.
//     Heads of 64 see that while they weigh, and weigh such a tile again; heads
//     of 128, whose weights take the scores' place, look at the scores first.
//     A weight vanishes where it is below 2^-35 of the row's largest.
// Measured: 4 prompts of 2048 rows behind up to 1000 slots, 20 heads of 64, bf16:
// 166 us in a stream of such calls for 62 GFLOP (tensor cores 20 % busy), 19
// the append; of a block's 280000 cycles a weighing warp spends 52 - 59 % on
// weights, 11 - 16 % waiting for scores, 17 - 19 % between items.  Issue slots are
// half used: a warp a scheduler and row tile waits for its own results.
// Append and attention in such a stream, both sides in one run: 186 us, 198
// where one thread walks and issues the products instead of a warp of which one
// lane issues.  Before that step 199 us, 201 with two looks at the scores.
// 4 prompts of 2048 rows behind 0, 400, 700 and 1000 slots, heads of 128: 20 heads 237 us for 130 GFLOP, 32 on 8 K/V
// heads 321 us for 208.
// Tried on earlier forms only, a call each: two threads a row (32 % more
// instructions) 200.6 us against 200.2; both looks in one as straight code, which
// waited for its instructions, 224 against 199.
// Slots hidden from a row weigh 0, and V codes that are NaN are taken out on the
// way in: the rows that see such a slot are made NaN at the end.
#include <atomic>
#include <type_traits>

#include "kernels.h"
#include "paged8.cuh"

namespace asrspec {
namespace {

constexpr int BM = 128, BN = 128, THREADS = 512;   // rows and keys of a tile; warps: 8 weigh, 3 convert K, 3 V, 1 issues products

struct Prompt8Args {
  Paged8View p;
  PagedRows r;
  char* out;
  float* lse;
  int tiles, items;   // of 256 rows
  int *next, *done;   // zero between calls: items taken besides each block's first, blocks that are done
};

template <int D> struct Prompt8Mem {
  static constexpr int HB = D / 64, BLOCK = 16384;             // 64 columns of 128 rows
  static constexpr int Q = 0, K = 2 * HB * BLOCK, V = K + 2 * HB * BLOCK, LENS = V + 2 * HB * BLOCK, END = LENS + 8 * PG_MAX_BATCH;
  // one block an SM: each takes all of tensor memory
  static constexpr int BYTES = (END < 120 * 1024 ? 120 * 1024 : END) + 1024;
};

struct Prompt8Bars {   // s, p: a buffer of scores; pv, q: a row tile
  uint64_t q_full[2], k_full[2], k_free[2], v_full[2], v_free[2], sc_full[8], s_full[2], p_full[2], pv_done[2][4], item_full[4], begun[4], ended[4], drained;
};
struct GroupScales {   // of a tile's 8 groups
  float k[8], v[8], lv[8];
};

__device__ __forceinline__ uint64_t desc_mn(uint32_t addr) {   // as umma_desc_sw128, the contiguous axis not the contraction's
  return (umma_desc_sw128(addr) & ~(0x3fffull << 16)) | (uint64_t)(1024 >> 4) << 16;
}
__device__ __forceinline__ void umma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void umma_f16_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// 32 lanes, 32 columns; the caller waits.
__device__ __forceinline__ void tmem_ld32(uint32_t at, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,"
      "%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
        "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
        "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(at));
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_st16(uint32_t at, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(at),
               "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
               "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
               : "memory");
}
__device__ __forceinline__ void sts16(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ uint4 ld_if_l2(bool in, const char* p) {   // by L2; zero where not `in`
  uint4 v;
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %5, 0;\n\t"
      "mov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\tmov.b32 %3, 0;\n\t"
      "@p ld.global.cg.v4.u32 {%0,%1,%2,%3}, [%4];\n\t}"
      : "=&r"(v.x), "=&r"(v.y), "=&r"(v.z), "=&r"(v.w)
      : "l"(p), "r"((int)in)
      : "memory");
  return v;
}
// Pairs of floats in one operation.
__device__ __forceinline__ uint64_t two(float lo, float hi) {
  uint64_t x;
  asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(lo), "f"(hi));
  return x;
}
__device__ __forceinline__ float2 parts(uint64_t x) {
  float2 v;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(x));
  return v;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// A row's 128 scores, 32 at a time, the next ones on their way; f(q, s) for each.
// Not unrolled further: this code and the other row tile's share an instruction cache.
template <typename F>
__device__ __forceinline__ void for_scores(uint32_t at, bool full, int left, F f) {
  uint32_t s[2][32];
  tmem_ld32(at, s[0]);
#pragma unroll 1
  for (int q2 = 0; q2 < 2; ++q2) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int q = q2 * 2 + h;
      tmem_wait_ld();
      if (h == 0 || q2 == 0) tmem_ld32(at + (q + 1) * 32, s[h ^ 1]);
      if (!full)   // columns that the row does not see
#pragma unroll
        for (int i = 0; i < 32; ++i) s[h][i] = q * 32 + i < left ? s[h][i] : 0xff800000u;
      f(q, s[h]);
    }
  }
}

// First look at a tile's scores: the row's maximum, and log2 of the largest weight
// relative to the maximum mx.
__device__ __forceinline__ void look(uint32_t at, bool full, int left, const GroupScales& gs, float mx, float sc, float& most, float& top) {
  most = top = -INFINITY;
  for_scores(at, full, left, [&](int q, uint32_t (&s)[32]) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t* x = s + h * 16;
      float g = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
#pragma unroll
      for (int i = 2; i < 16; i += 2) g = max3(g, __uint_as_float(x[i]), __uint_as_float(x[i + 1]));
      g *= gs.k[q * 2 + h];
      most = fmaxf(most, g);
      top = fmaxf(top, (g - mx) * sc + gs.lv[q * 2 + h]);
    }
  });
}
// Second look: the weights, relative to the maximum, times 2^li and the groups'
// scales, take the scores' place.  With lf = li + log2 of a group's scale
//   w = 2^((S t - base) sc + lf),   l = sum over groups of 2^-lf sum w :
// lf is held at -60, below which fp16 has no weight but the sum still sees it.  Returns the sum.
__device__ __forceinline__ float weigh(uint32_t at, bool full, int left, const GroupScales& gs, float base, float sc, int li) {
  const uint64_t base2 = two(-base, -base), sc2 = two(sc, sc);
  float sum = 0.f;
  for_scores(at, full, left, [&](int q, uint32_t (&s)[32]) {
    uint32_t p[16];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float ks = gs.k[q * 2 + h], lf = fmaxf(gs.lv[q * 2 + h] + (float)li, -60.f);
      const uint64_t ks2 = two(ks, ks), lf2 = two(lf, lf);
      uint64_t sum2 = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int x = h * 16 + 2 * i;
        const float2 t = parts(fma2(fma2(two(__uint_as_float(s[x]), __uint_as_float(s[x + 1])), ks2, base2), sc2, lf2));
        const float w0 = ex2(t.x), w1 = ex2(t.y);
        sum2 = add2(sum2, two(w0, w1));
        p[h * 8 + i] = Mma16<__half>::pack(w0, w1);
      }
      const float2 part = parts(sum2);
      sum = fmaf(part.x + part.y, ex2(-lf), sum);
    }
    tmem_st16(at + q * 16, p);   // over scores that have been read: the next 32 lie past these 16 columns
  });
  return sum;
}

// Both looks at once, the weights to p_at: relative to the maximum and the reference of the tiles before, which the caller
// compares with what it finds.  ready(): p_at may be written.
template <typename F>
__device__ __forceinline__ float weigh_once(uint32_t at, uint32_t p_at, bool full, int left, const GroupScales& gs, float base, float sc,
                                            int li, float& most, float& top, F ready) {
  const uint64_t base2 = two(-base, -base), sc2 = two(sc, sc);
  float sum = 0.f;
  most = top = -INFINITY;
  for_scores(at, full, left, [&](int q, uint32_t (&s)[32]) {
    uint32_t p[16];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t* x = s + h * 16;
      float g = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
#pragma unroll
      for (int i = 2; i < 16; i += 2) g = max3(g, __uint_as_float(x[i]), __uint_as_float(x[i + 1]));
      const float ks = gs.k[q * 2 + h], lv = gs.lv[q * 2 + h], lf = fmaxf(lv + (float)li, -60.f);
      g *= ks;
      most = fmaxf(most, g);
      top = fmaxf(top, (g - base) * sc + lv);
      const uint64_t ks2 = two(ks, ks), lf2 = two(lf, lf);
      uint64_t sum2 = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 t = parts(fma2(fma2(two(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1])), ks2, base2), sc2, lf2));
        const float w0 = ex2(t.x), w1 = ex2(t.y);
        sum2 = add2(sum2, two(w0, w1));
        p[h * 8 + i] = Mma16<__half>::pack(w0, w1);
      }
      const float2 part = parts(sum2);
      sum = fmaf(part.x + part.y, ex2(-lf), sum);
    }
    if (q == 0) ready();
    tmem_st16(p_at + q * 16, p);
  });
  return sum;
}

// What a block works on.
struct Item {
  int b, kvh, m0, len, rows, keys;
  int n0, n1;   // key tiles of its two row tiles: up to what the last row sees
  __device__ __forceinline__ int n() const { return max(n0, n1); }
};
__device__ __forceinline__ int seen_by(const PagedRows& r, int len, int m) { return r.causal ? len + (int)r.groups.div(m) + 1 : len; }

// A block's items: the first by its number, each other one the next that no block has, in order of falling row tile (late
// rows see most).  One thread fetches them, an item ahead, into four slots; a slot is free when everyone has left its item.
// No warp waits for another one but by bar_wait: one whose wait has given up leaves at its next item, and those that stay must
// find out by waits that end too.
struct Items {
  const Prompt8Args& a;
  Prompt8Bars& bars;
  const int2* lens;
  int* slots;
  int4* nan_keys;   // [4][quads], of a slot's item: none yet
  int *any_nan, quads;
  // item number i; false where it has no work
  __device__ __forceinline__ bool set(int i, Item& it) const {
    const int per = a.p.c.kv_heads * a.p.c.batch, tile = i / per, in = i - tile * per;
    it.b = in / a.p.c.kv_heads, it.kvh = in - it.b * a.p.c.kv_heads;
    it.m0 = (a.tiles - 1 - tile) * 2 * BM;
    it.len = lens[it.b].x, it.rows = lens[it.b].y;
    it.keys = it.rows == 0 ? 0 : it.len + (a.r.causal ? it.rows : 0);
    const int m_rows = it.rows * a.r.group;
    it.n0 = it.m0 >= m_rows ? 0 : (seen_by(a.r, it.len, min(it.m0 + BM, m_rows) - 1) + BN - 1) / BN;
    it.n1 = it.m0 + BM >= m_rows ? 0 : (seen_by(a.r, it.len, min(it.m0 + 2 * BM, m_rows) - 1) + BN - 1) / BN;
    return it.n0 > 0;
  }
  // the block's item k, for a warp; false past the end
  __device__ __forceinline__ bool take(int k, Item& it, bool& gave_up) const {
    bar_wait(&bars.item_full[k & 3], k >> 2 & 1, a.p.c.status, gave_up);
    const int i = gave_up ? -1 : *reinterpret_cast<volatile int*>(slots + (k & 3));
    return __all_sync(0xffffffffu, i >= 0 && set(i, it));   // a whole warp: one answer where a wait has given up too
  }
  __device__ __forceinline__ void fetch(int k, bool& gave_up) const {   // one thread
    if (k >= 4) bar_wait(&bars.ended[k & 3], (k >> 2) - 1 & 1, a.p.c.status, gave_up);
    Item it;
    int i = k == 0 ? (int)blockIdx.x : (int)gridDim.x + atomicAdd(a.next, 1);
    while (i < a.items && !set(i, it)) i = (int)gridDim.x + atomicAdd(a.next, 1);
#pragma unroll 4
    for (int q = 0; q < quads; ++q) nan_keys[(k & 3) * quads + q] = make_int4(0x7fffffff, 0x7fffffff, 0x7fffffff, 0x7fffffff);
    any_nan[k & 3] = 0;
    slots[k & 3] = i < a.items ? i : -1;
    mbar_arrive(&bars.item_full[k & 3]);
  }
  __device__ __forceinline__ void leave(int k) const { mbar_arrive(&bars.ended[k & 3]); }
};
__device__ __forceinline__ bool elect_one() {
  uint32_t one;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
  return one != 0;
}
// One arrival a warp, after all its lanes: arrivals at one barrier go one by one.
__device__ __forceinline__ void warp_arrive(uint64_t* bar) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
}

template <typename T, int D>
__global__ void __launch_bounds__(THREADS, 1) prompt8_kernel(const Prompt8Args a) {
  using M = Prompt8Mem<D>;
  // Tensor memory, 512 columns: two buffers of scores, for heads of 64 the weights of each beside them, the outputs of both row
  // tiles.  Heads of 64 fill 512, heads of 128 too: no room for a third buffer of scores.
  constexpr int HB = M::HB, NS = 2;
  constexpr bool ONCE = D == 64;
  constexpr int P_COL = 2 * BN, O_COL = ONCE ? P_COL + BN : 2 * BN, P_STEP = ONCE ? BN / 2 : BN;
  static_assert(O_COL + 2 * D <= 512, "");
  extern __shared__ uint8_t raw[];
  __shared__ __align__(8) Prompt8Bars bars;
  __shared__ GroupScales scales[8];
  __shared__ __align__(16) int nan_key[4][D];   // by item: of a column of V the first key whose code is a NaN
  __shared__ int any_nan[4];
  __shared__ uint32_t s_tmem;
  __shared__ int s_items[4];
  const uint32_t smem = (smem_u32(raw) + 1023) / 1024 * 1024;
  int2* const lens = reinterpret_cast<int2*>(raw + (smem - smem_u32(raw)) + M::LENS);
  const PagedView& c = a.p.c;
  const PagedRows& r = a.r;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars.q_full[i], 4), mbar_init(&bars.k_full[i], 3), mbar_init(&bars.v_full[i], 3);
      mbar_init(&bars.k_free[i], 1), mbar_init(&bars.v_free[i], 1);
      mbar_init(&bars.s_full[i], 1), mbar_init(&bars.p_full[i], 4);
      for (int j = 0; j < 4; ++j) mbar_init(&bars.pv_done[i][j], 1);
    }
    for (int i = 0; i < 8; ++i) mbar_init(&bars.sc_full[i], 2);
    for (int i = 0; i < 4; ++i) mbar_init(&bars.item_full[i], 1), mbar_init(&bars.begun[i], 1), mbar_init(&bars.ended[i], 8 + 5 + 1);
    mbar_init(&bars.drained, 1);
    fence_mbar_init();
  }
  for (int b = tid; b < c.batch; b += THREADS) paged_lens(c, r, b, lens[b].x, lens[b].y);
  if (warp == 14) tmem_alloc(&s_tmem, 512), tmem_relinquish();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  bool gave_up = false;
  for (int b = blockIdx.x; b < c.batch; b += gridDim.x) {   // rows past a sequence's own, or without keys
    const int2 n = lens[b];
    const int from = n.x + (r.causal ? n.y : 0) == 0 ? 0 : n.y;
    const size_t heads0 = ((size_t)b * r.max_rows + from) * r.heads, count = (size_t)(r.max_rows - from) * r.heads;
    uint4* o = reinterpret_cast<uint4*>(a.out + heads0 * D * sizeof(T));
    for (size_t i = tid; i < count * (D * sizeof(T) / 16); i += THREADS) o[i] = make_uint4(0, 0, 0, 0);
    if (a.lse)
      for (size_t i = tid; i < count; i += THREADS) a.lse[heads0 + i] = -INFINITY;
  }
  const Items src{a, bars, lens, s_items, reinterpret_cast<int4*>(nan_key), any_nan, D / 4};
  pdl_wait();   // the append, and the call before, whose last block sets the counts back

  // 8 warps of 168 registers and 8 of 88: what the block was launched with, 16 of 128
  if (warp < 8) asm volatile("setmaxnreg.inc.sync.aligned.u32 168;");
  else asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
  if (warp < 8) {
    // ------------------------------------------------------------ the weights of a row
    const int x = warp >> 2, row_in = tid & 127;
    const uint32_t lanes = (uint32_t)(warp & 3) << 21, o_at = tmem + lanes + O_COL + x * D;
    int pairs = 0, tiles = 0, steps = 0;   // begun before this item: pairs of the block, its key tiles, this row tile's
    // q of an item, as fp16 rows in shared memory; returns the scale that its scores need.  The products with the q before are
    // done: the last scores have come.
    auto take_q = [&](const Item& it) {
      const int m = it.m0 + x * BM + row_in, row = (int)r.groups.div(m), hq = it.kvh * r.group + m - row * r.group;
      const bool mine = m < it.rows * r.group;
      const char* src = r.q + it.b * r.q_b + (long long)row * r.q_r + hq * r.q_h;
      const uint32_t dst = smem + M::Q + x * HB * M::BLOCK + row_in * 128;
      float sc = r.scale * LOG2E;
      uint4 v[D / 8];
#pragma unroll
      for (int i = 0; i < D / 8; ++i) v[i] = ldg_if(mine, src + i * 16);
      if constexpr (!std::is_same<T, __half>::value) {   // to fp16 by a power of two: see the kernel for few rows
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < D / 8; ++i)
#pragma unroll
          for (int y = 0; y < 4; ++y) most = max(most, max(reg_of(v[i], y) & 0x7fffu, reg_of(v[i], y) >> 16 & 0x7fffu));
        const int e = min(100, 14 - ((int)(most >> 7) - 127));
        const float f0 = pow2(e / 2), f1 = pow2(e - e / 2);
        sc = fmaxf(sc * pow2(-(e / 2)) * pow2(-(e - e / 2)), 1.17549435e-38f);
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
          uint32_t y[4];
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            const uint32_t w = reg_of(v[i], z);
            y[z] = Mma16<__half>::pack(__int_as_float(w << 16) * f0 * f1, __int_as_float(w & 0xffff0000u) * f0 * f1);
          }
          v[i] = make_uint4(y[0], y[1], y[2], y[3]);
        }
      }
#pragma unroll
      for (int i = 0; i < D / 8; ++i)
        sts16(dst + i / 8 * M::BLOCK + ((i % 8) ^ (row_in & 7)) * 16, nan_for_inf(v[i].x), nan_for_inf(v[i].y), nan_for_inf(v[i].z),
              nan_for_inf(v[i].w));
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      warp_arrive(&bars.q_full[x]);
      return sc;
    };
    Item it{};
    float next_sc = 0.f;
    bool more = true, idle = false;
    for (int k = -1; more; ++k) {   // before the first item one without rows
      const int nx = x ? it.n1 : it.n0, m = it.m0 + x * BM + row_in;
      const bool mine = m < it.rows * r.group;
      const int lim = mine ? min(it.keys, seen_by(r, it.len, m)) : 0, all_see = nx ? seen_by(r, it.len, it.m0 + x * BM) : 0;
      const float sc = next_sc;
      // A wait tells a phase only from the one before.  A row tile that sat out an item has seen none of its phases: it goes
      // on once the products have come to this item, when all of them have passed.
      if (nx > 0 && idle) bar_wait(&bars.begun[k & 3], k >> 2 & 1, c.status, gave_up);
      idle = nx == 0;
      float mx = -INFINITY, l = 0.f;   // the maximum, in units of the product; the sum of p
      int li = 126;                    // log2 of what weights are multiplied by
      Item next;
      more = src.take(k + 1, next, gave_up);
      if (more) {   // its rows of q come near
        const int nm = next.m0 + x * BM + row_in, nrow = (int)r.groups.div(nm), nhq = next.kvh * r.group + nm - nrow * r.group;
        if (nm < next.rows * r.group)
          asm volatile("prefetch.global.L2 [%0];" ::"l"(r.q + next.b * r.q_b + (long long)nrow * r.q_r + nhq * r.q_h));
      }
      for (int j = 0; j < nx; ++j) {
        const int pair = pairs + min(j, it.n0) + min(j, it.n1) + (x && j < it.n0), buf = pair % NS, tile = tiles + j;
        const uint32_t s_at = tmem + lanes + buf * BN;
        const GroupScales& gs = scales[tile & 7];
        bar_wait(&bars.sc_full[tile & 7], tile >> 3 & 1, c.status, gave_up);
        bar_wait(&bars.s_full[buf], pair / NS & 1, c.status, gave_up);
        __syncwarp();
        tc_fence_after();
        const bool full = (j + 1) * BN <= all_see;   // of every row that counts
        const int left = lim - j * BN;               // columns that this row sees
        // Once a tile's products have been added: a wait cannot tell a phase from the one after the next, but of four barriers
        // in turn the one of four tiles ago is known to have passed, since scores run ahead by fewer.
        auto added = [&](int t) {
          bar_wait(&bars.pv_done[x][(steps + t) & 3], (steps + t) >> 2 & 1, c.status, gave_up);
          __syncwarp();
          tc_fence_after();
        };
        auto rescale = [&](float f) {
#pragma unroll 1
          for (int q = 0; q < D / 32; ++q) {
            uint32_t o[32];
            tmem_ld32(o_at + q * 32, o);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
            tmem_st16(o_at + q * 32, o);
            tmem_st16(o_at + q * 32 + 16, o + 16);
          }
        };
        if constexpr (ONCE) {
          float most, top, sum, shift = 0.f;   // log2 of what the output so far is to be multiplied by
          bool moved = false;
#pragma unroll 1
          for (int pass = 0;; ++pass) {
            sum = weigh_once(s_at, tmem + lanes + P_COL + buf * P_STEP, full, left, gs, mx == -INFINITY ? 0.f : mx, sc, li, most, top, [&] {
              if (pass == 0 && j > 0) added(j - 1);
            });
            // The first tile brings the first maximum and, once the weights are relative to that, their size.  Later ones move
            // them only where a weight would leave fp16 or p grows past 2^4.  At most three passes.
            if (!__any_sync(0xffffffffu, (most - mx) * sc > 4.f || top + (float)li > 15.f || (j == 0 && top + (float)li < 4.f && li < 126)) ||
                pass == 4)
              break;
            moved = true;
            if (most > mx) {
              if (mx == -INFINITY) {
                top = -126.f;
                for (int u = 0; u < 8; ++u) top = fmaxf(top, gs.lv[u]);
              } else {
                const float grown = (most - mx) * sc;
                const int up = min((int)fminf(grown, 1000.f), 126 - li);
                top -= grown, shift += (float)up - grown;
                l *= ex2(-grown), li += up;
              }
              mx = most;
            }
            const int to = top > -1e4f ? max(-126, min(126, 11 - (int)ceilf(fminf(top, 1000.f)))) : li;
            if (to < li ? top + (float)li > 11.f : j == 0) shift += (float)(to - li), li = to;
            __syncwarp();
          }
          if (moved && j > 0) rescale(ex2(shift));
          l += sum;
        } else {
          float most, top;
          float grown = 0.f;
          int up = 0;
#pragma unroll 1
          for (bool again = false;; again = true) {   // the largest weight is relative to the maximum: where that grows, once more
            look(s_at, full, left, gs, mx, sc, most, top);
            if (again || !__any_sync(0xffffffffu, (most - mx) * sc > 4.f)) break;
            if (most > mx) {
              grown = mx == -INFINITY ? 0.f : (most - mx) * sc;
              up = min((int)fminf(grown, 1000.f), 126 - li);
              mx = most, l *= ex2(-grown), li += up;
            }
            __syncwarp();
          }
          if (__any_sync(0xffffffffu, grown > 0.f || top + (float)li > 15.f)) {
            const int e = top + (float)li > 11.f ? min((int)ceilf(top) + li - 11, li + 126) : 0;
            li -= e;
            if (j > 0) {   // the tile before has been added
              const float f = ex2((float)(up - e) - grown);
              added(j - 1);
              rescale(f);
            }
            __syncwarp();
          }
          l += weigh(s_at, full, left, gs, mx == -INFINITY ? 0.f : mx, sc, li);
        }
        tmem_wait_st();
        tc_fence_before();
        warp_arrive(&bars.p_full[buf]);
      }
      pairs += it.n0 + it.n1, tiles += it.n(), steps += nx;
      const Item was = it;
      it = next;
      if (more && (x ? it.n1 : it.n0) > 0) next_sc = take_q(it);
      if (k < 0) continue;
      // -------------------------------------------------------------- the rows' ends
      if (nx > 0) {
        bar_wait(&bars.pv_done[x][(steps - 1) & 3], (steps - 1) >> 2 & 1, c.status, gave_up);
        __syncwarp();
        tc_fence_after();
      }
      const int row = (int)r.groups.div(m), hq = was.kvh * r.group + m - row * r.group;
      const size_t at = ((size_t)was.b * r.max_rows + row) * r.heads + hq;
      T* out = reinterpret_cast<T*>(a.out) + at * D;
      const bool nans = *reinterpret_cast<volatile int*>(&any_nan[k & 3]) != 0;
      const float f = l != 0.f ? __fdividef(1.f, l) * pow2(-li) : 0.f;
#pragma unroll 1
      for (int q = 0; q < D / 32; ++q) {
        uint32_t o[32];
        if (nx > 0) {
          __syncwarp();
          tmem_ld32(o_at + q * 32, o);
          tmem_wait_ld();
        }
#pragma unroll
        for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
        if (nans)
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (nan_key[k & 3][q * 32 + i] < lim) o[i] = 0x7fffffffu;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t w[4];
#pragma unroll
          for (int y = 0; y < 4; ++y) w[y] = Mma16<T>::pack(__uint_as_float(o[i * 8 + 2 * y]), __uint_as_float(o[i * 8 + 2 * y + 1]));
          if (mine) *reinterpret_cast<uint4*>(out + q * 32 + i * 8) = make_uint4(w[0], w[1], w[2], w[3]);
        }
      }
      if (mine && a.lse) a.lse[at] = (mx * sc + __log2f(l)) * LN2;
      tc_fence_before();
      __syncwarp();
      if (lane == 0) src.leave(k);
    }
  } else if (warp < 14) {
    // ------------------------------------------------------------ codes to fp16
    // Of K or of V.  A warp takes every third of a tile's 8 groups; LK lanes a key, KI keys an instruction, IT instructions a
    // group.  Of every 32 groups of an item, four tiles, a lane looks up one: its place, its scale, the next round's page.
    constexpr int LK = D / 16, KI = 32 / LK, IT = PG_GROUP / KI, MINE = 3;
    const bool is_v = warp >= 11;
    const int w = is_v ? warp - 11 : warp - 8, col = lane % LK;
    const char* pages = (is_v ? c.v : c.k) + col * 16 + lane / LK * c.slot_stride;
    const float* scale_pages = is_v ? a.p.v_scale : a.p.k_scale;
    uint64_t *full = is_v ? bars.v_full : bars.k_full, *free = is_v ? bars.v_free : bars.k_free;
    const uint32_t stages = smem + (is_v ? M::V : M::K);
    const long long step = KI * c.slot_stride;
    Item it;
    int k = -1, j = 0, next_pid = 0;
    long long off = 0;
    float scale = 1.f;
    uint4 x[MINE][IT];
    bool more = true;
    auto take = [&] {   // the next item, and the one after it is fetched
      ++k;
      if (tid == 8 * 32) {
        if (k == 0) src.fetch(0, gave_up);
        if (k == 0 || more) src.fetch(k + 1, gave_up);
      }
      __syncwarp();
      more = src.take(k, it, gave_up);
      j = 0;
    };
    auto load = [&] {   // of tile j
      const int groups = (it.keys + PG_GROUP - 1) / PG_GROUP;
      if (j % 4 == 0) {
        const int grp = j * 8 + lane;
        auto page = [&](int g) { return g < groups ? __ldg(c.table + it.b * c.table_stride + c.groups.div((uint32_t)g)) : 0; };
        const int pid = paged_valid(c, j == 0 ? page(grp) : next_pid);
        off = paged_offset(c, pid, grp) + it.kvh * c.head_stride;
        scale = grp < groups ? __ldcg(scale_pages + a.p.scale_at(pid, it.kvh, grp)) : 1.f;
        next_pid = page(grp + 32);   // looked at when used
      }
      const bool whole = (j + 1) * BN <= it.keys;
#pragma unroll
      for (int g = 0; g < MINE; ++g) {
        const int in = w + 3 * g;
        const char* at = pages + __shfl_sync(0xffffffffu, off, (j % 4 * 8 + in) & 31);
        const int left = in >= 8 ? 0 : whole ? PG_GROUP : it.keys - j * BN - in * PG_GROUP;
#pragma unroll
        for (int i = 0; i < IT; ++i) x[g][i] = ld_if_l2(i * KI + lane / LK < left, at + i * step);
      }
    };
    take();
    if (more) load();
    for (int tile = 0; more; ++tile) {
      const int st = tile & 1;
      if (w == 0) {   // the tile's scales
        GroupScales& gs = scales[tile & 7];
        if (lane / 8 == j % 4) {
          if (is_v) gs.v[lane % 8] = scale, gs.lv[lane % 8] = fmaxf(__log2f(scale), -126.f);
          else gs.k[lane % 8] = fmaxf(scale, 1.17549435e-38f);   // times -inf, where a score is hidden, it must stay that
        }
        warp_arrive(&bars.sc_full[tile & 7]);
      }
      if (is_v) {
        const int slot = k & 3;
        uint32_t bad = 0;
#pragma unroll
        for (int g = 0; g < MINE; ++g)
#pragma unroll
          for (int i = 0; i < IT; ++i)
#pragma unroll
            for (int y = 0; y < 4; ++y) bad |= (reg_of(x[g][i], y) & 0x7f7f7f7fu) + 0x01010101u;
        if (bad & 0x80808080u) {
          any_nan[slot] = 1;
#pragma unroll
          for (int g = 0; g < MINE; ++g)
#pragma unroll
            for (int i = 0; i < IT; ++i) {
              uint4& v = x[g][i];
#pragma unroll 1
              for (int y = 0; y < 16; ++y)
                if (nan_codes(reg_of(v, y / 4)) >> (y % 4 * 8) & 1)
                  atomicMin(&nan_key[slot][col * 16 + y], j * BN + (w + 3 * g) * PG_GROUP + i * KI + lane / LK);
              v.x &= ~nan_codes(v.x), v.y &= ~nan_codes(v.y), v.z &= ~nan_codes(v.z), v.w &= ~nan_codes(v.w);
            }
        }
      }
      if (tile >= 2) bar_wait(&free[st], (tile >> 1) - 1 & 1, c.status, gave_up);
      const uint32_t dst = stages + st * HB * M::BLOCK + col / 4 * M::BLOCK + (w * PG_GROUP + lane / LK) * 128;
#pragma unroll
      for (int g = 0; g < MINE; ++g) {
        if (w + 3 * g >= 8) break;
#pragma unroll
        for (int i = 0; i < IT; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t c0 = reg_of(x[g][i], 2 * h), c1 = reg_of(x[g][i], 2 * h + 1);
            sts16(dst + (3 * g * PG_GROUP + i * KI) * 128 + (((col % 4 * 2 + h) ^ ((i * KI + lane / LK) & 7)) << 4), half2_of(c0),
                  half2_of(c0 >> 16), half2_of(c1), half2_of(c1 >> 16));
          }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      warp_arrive(&full[st]);
      if (++j >= it.n()) {
        if (warp != 8 && lane == 0) src.leave(k);
        take();
      }
      if (more) load();
    }
  } else if (warp == 14) {
    // ------------------------------------------------------------ products
    // The whole warp walks, one lane issues: 186 us against 198 where one thread does both (see above).
    const bool lead = elect_one();
    constexpr uint32_t F32 = 1u << 4, M128 = (uint32_t)(BM >> 4) << 24;   // accumulator type; fp16 operands are 0
    constexpr uint32_t id_s = F32 | M128 | (uint32_t)(BN >> 3) << 17, id_o = F32 | M128 | 8u << 17 | 1u << 16;   // V: contraction axis outermost
    const uint64_t qd = umma_desc_sw128(smem + M::Q), kd = umma_desc_sw128(smem + M::K), vd = desc_mn(smem + M::V);
    constexpr uint32_t STEP = HB * M::BLOCK / 16;    // between q's of row tiles, between stages, in a descriptor's units
    int pairs = 0, tiles = 0, qs0 = 0, qs1 = 0, pv0 = 0, pv1 = 0;   // pairs and key tiles before this item; of each row tile: q's, outputs begun
    Item it;
    for (int k = 0; src.take(k, it, gave_up); ++k) {
      const int n0 = __shfl_sync(0xffffffffu, it.n0, 0), n1 = __shfl_sync(0xffffffffu, it.n1, 0), n = n0 + n1;
      if (lead) mbar_arrive(&bars.begun[k & 3]);   // nothing of the items before is left to be issued
      // Scores run ahead of outputs within an item: the next one's q comes from threads that may wait for outputs.  Where weights
      // have a place of their own, by two pairs, a buffer being free once its scores are weighed; where they take the scores'
      // place, by one.  Pair i: key tile i / 2 of row tile i % 2, the last one of row tile 1; of row tile 0 alone i.
      constexpr int LAG = ONCE ? 2 : 1;
      for (int i = 0; i < n + LAG; ++i) {
        const int o = i - LAG, o_buf = (pairs + o) & 1;
        if (ONCE && o >= 0) bar_wait(&bars.p_full[o_buf], (pairs + o) >> 1 & 1, c.status, gave_up);
        if (i < n) {
          const int x = n1 == 0 ? 0 : i < 2 * n0 ? i & 1 : 1, j = n1 == 0 ? i : i >> 1, st = tiles + j & 1;
          if (j == 0) bar_wait(&bars.q_full[x], (x ? qs1++ : qs0++) & 1, c.status, gave_up);
          bar_wait(&bars.k_full[st], tiles + j >> 1 & 1, c.status, gave_up);
          tc_fence_after();
          const int buf = (pairs + i) & 1;
          if (lead) {
#pragma unroll
            for (int h = 0; h < HB; ++h)
#pragma unroll
              for (int y = 0; y < 4; ++y)
                umma_f16(tmem + buf * BN, qd + x * STEP + h * (M::BLOCK / 16) + y * 2, kd + st * STEP + h * (M::BLOCK / 16) + y * 2, id_s, h + y > 0);
            umma_commit(&bars.s_full[buf]);
            if (x == 1 || j >= n1) umma_commit(&bars.k_free[st]);
          }
          __syncwarp();
        }
        if (o >= 0) {
          const int x = n1 == 0 ? 0 : o < 2 * n0 ? o & 1 : 1, j = n1 == 0 ? o : o >> 1, st = tiles + j & 1;
          bar_wait(&bars.v_full[st], tiles + j >> 1 & 1, c.status, gave_up);
          if (!ONCE) bar_wait(&bars.p_full[o_buf], (pairs + o) >> 1 & 1, c.status, gave_up);
          tc_fence_after();
          const int pv = x ? pv1++ : pv0++;
          if (lead) {
#pragma unroll
            for (int h = 0; h < HB; ++h)
#pragma unroll
              for (int y = 0; y < BN / 16; ++y)
                umma_f16_ts(tmem + O_COL + x * D + h * 64, tmem + (ONCE ? P_COL : 0) + o_buf * P_STEP + y * 8, vd + st * STEP + h * (M::BLOCK / 16) + y * 128, id_o, j + y > 0);
            umma_commit(&bars.pv_done[x][pv & 3]);
            if (x == 1 || j >= n1) umma_commit(&bars.v_free[st]);
          }
          __syncwarp();
        }
      }
      pairs += n, tiles += max(n0, n1);
      if (lead) src.leave(k);
    }
    // Where a wait has given up products may still be on their way: they end before tensor and shared memory are let go.
    if (lead) umma_commit(&bars.drained);
    __syncwarp();
    bool late = false;
    bar_wait(&bars.drained, 0, c.status, late);
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 14) tmem_dealloc(tmem, 512);
  if (tid == 0 && atomicAdd(a.done, 1) == (int)gridDim.x - 1) *a.next = 0, *a.done = 0;   // as the next call needs them
}

template <typename T, int D>
cudaError_t launch_d(Prompt8Args& a, bool appended, cudaStream_t st) {
  constexpr auto kernel = prompt8_kernel<T, D>;
  static std::atomic<uint64_t> ready{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (!(ready.load(std::memory_order_acquire) & bit)) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Prompt8Mem<D>::BYTES);
    if (e != cudaSuccess) return e;
    ready.fetch_or(bit, std::memory_order_release);
  }
  const int sms = paged_sm_count(), grid = a.items < sms ? a.items : sms;
  return launch_ex(kernel, dim3((unsigned)grid), dim3(THREADS), Prompt8Mem<D>::BYTES, st, appended, 1, a);
}

}  // namespace

cudaError_t launch_prompt8(const Paged8View& c, const PagedRows& r, int dtype, void* out, float* lse, int* counts, bool appended,
                           cudaStream_t st) {
  const int tiles = (r.max_rows * r.group + 2 * BM - 1) / (2 * BM);
  const long long items = (long long)tiles * c.c.kv_heads * c.c.batch;
  if (items > 0x7fffffffll - 100000) return cudaErrorInvalidValue;
  Prompt8Args a{c, r, static_cast<char*>(out), lse, tiles, (int)items, counts, counts + 1};
  if (dtype == 1) return c.dim == 64 ? launch_d<__nv_bfloat16, 64>(a, appended, st) : launch_d<__nv_bfloat16, 128>(a, appended, st);
  return c.dim == 64 ? launch_d<__half, 64>(a, appended, st) : launch_d<__half, 128>(a, appended, st);
}

}  // namespace asrspec
