// Eviction from a paged K/V cache by accumulated attention weight.
//
// Per (sequence, K/V head) with more than `budget` slots in use, the budget
// slots of highest rank stay: protected slots first (one of the `recent`
// newest positions, or of the `first` oldest), all alike, then the others by
// score, a NaN lowest; equals by lowest slot.  A cached key carries its position in
// itself, so the slots' order is free: the j-th freed slot below the budget
// takes the j-th kept slot at or past it.  Sources and destinations are
// disjoint, so the moves run in any order over the whole GPU and move the
// fewest rows there are to move.
//
// One launch, a cluster of 1 to 8 blocks per (sequence, head), each on a
// contiguous part of the slots:
//   * the rank of the last kept slot by a radix search, 8 bits a pass over a
//     histogram (summed over the cluster through distributed shared memory);
//   * freed and kept slots listed in slot order, from exclusive counts over
//     warps and blocks;
//   * the moves, rows dealt out over the cluster: addresses first, for a batch
//     of rows at a time, then 16-byte chunks with several rows in flight a
//     thread.  Bound by the bytes of the moved rows where many move, by the
//     chain of passes where few do.
// Measured: 8 sequences of 30001 to 40000 slots, 8 heads of 128, fp16, cut to
// 16384: 133 us, of which 30 are search and lists and the rest 557 MB of moves;
// 64 of 200 to 448 slots, 20 heads of 64, bf16, cut to 256: 16 us.
#include <atomic>

#include "kernels.h"
#include "paged.cuh"

namespace asrspec {
namespace {

constexpr int EV_MAX_CLUSTER = 8;
// Slots whose rank a block keeps in shared memory; past them it is taken anew.
constexpr int EV_KEYS = 8192, EV_KEYS_LARGE = 40960;

struct EvictArgs {
  PagedView c;
  const int *len, *seen;
  const float* score;
  const int* pos;
  long long in_b, in_h, out_b, out_h;   // elements
  float* score_out;
  int *pos_out, *len_out;
  int in_cap, out_cap, budget, recent, first;
  int *holes, *srcs;                    // workspace: [B K][max_moves] each
  int max_moves, chunks, keys;          // 16-byte chunks of a row; ranks kept in shared memory
};

// Slots in use; a length out of range sets the status word and is left alone (-1).
__device__ __forceinline__ int evict_len(const EvictArgs& a, int b) {
  const int n = a.len[b];
  if (n < 0 || n > a.in_cap || n > a.c.max_slots || min(n, a.budget) > a.out_cap) {
    if (a.c.status) set_status(a.c.status, ST_CAPACITY);
    return -1;
  }
  return n;
}

// Rank of a slot as an unsigned key: larger stays.
__device__ __forceinline__ uint32_t rank_key(float score, int pos, int newest, int first) {
  if (pos >= newest || pos < first) return 0xffffffffu;
  return score != score ? 0u : ordered_bits(score + 0.f);   // -0 ranks as 0
}

__device__ __forceinline__ void st_cluster(int* at, int rank, int v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(dsmem_addr(at, rank)), "r"(v) : "memory");
}
__device__ __forceinline__ int ld_cluster(const int* at, int rank) {
  int v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(dsmem_addr(at, rank)) : "memory");
  return v;
}

template <int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) evict_kernel(EvictArgs a) {
  constexpr int WARPS = THREADS / 32;
  __shared__ int hist[4][256];
  __shared__ int s_hist[256], s_cut[4][3];   // the cluster's; a pass's bin, how many of it stay, how many it has
  __shared__ int2 s_warp[2][WARPS], s_rank[2][EV_MAX_CLUSTER];
  __shared__ long long s_to[THREADS], s_of[THREADS];
  extern __shared__ uint32_t s_key[];
  const int CL = gridDim.x, rank = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int n = evict_len(a, b);
  const size_t task = (size_t)b * a.c.kv_heads + h;
  const float* sc = a.score + b * a.in_b + h * a.in_h;
  const int* ps = a.pos + b * a.in_b + h * a.in_h;
  float* so = a.score_out + b * a.out_b + h * a.out_h;
  int* po = a.pos_out + b * a.out_b + h * a.out_h;
  if (h == 0 && rank == 0 && tid == 0) a.len_out[b] = n < 0 ? a.len[b] : min(n, a.budget);
  const int i0 = (int)((long long)max(n, 0) * rank / CL), i1 = (int)((long long)max(n, 0) * (rank + 1) / CL);
  if (n <= a.budget) {   // uniform over the cluster
    if (so != sc)
      for (int i = i0 + tid; i < i1; i += THREADS) so[i] = sc[i];
    if (po != ps)
      for (int i = i0 + tid; i < i1; i += THREADS) po[i] = ps[i];
    return;
  }
  auto sync = [&] {
    if (CL > 1) cluster_sync();
    else __syncthreads();
  };
  const int newest = a.seen[b] - a.recent;
  const int cached = min(i1 - i0, a.keys);
  auto key = [&](int i) { return i - i0 < cached ? s_key[i - i0] : rank_key(sc[i], ps[i], newest, a.first); };
  // Ranks to shared memory; scores and positions below the budget to the
  // outputs, where the moves then overwrite the freed slots.
  const bool copy_s = so != sc, copy_p = po != ps;
  const int ends = max(i0 + cached, copy_s || copy_p ? min(i1, a.budget) : 0);
  for (int i = i0 + tid; i < ends; i += THREADS * 8) {
    float x[8];
    int p[8];
#pragma unroll
    for (int y = 0; y < 8; ++y) {
      x[y] = __ldcg(sc + min(i + y * THREADS, ends - 1));
      p[y] = __ldcg(ps + min(i + y * THREADS, ends - 1));
    }
#pragma unroll
    for (int y = 0; y < 8; ++y) {
      const int at = i + y * THREADS;
      if (at >= ends) break;
      if (at - i0 < cached) s_key[at - i0] = rank_key(x[y], p[y], newest, a.first);
      if (copy_s && at < a.budget) so[at] = x[y];
      if (copy_p && at < a.budget) po[at] = p[y];
    }
  }
  for (int i = tid; i < 4 * 256; i += THREADS) hist[0][i] = 0;
  __syncthreads();

  // the key of the budget-th slot: fix 8 bits a pass from the top
  uint32_t prefix = 0;
  int need = a.budget;
#pragma unroll 1
  for (int pass = 0; pass < 4; ++pass) {
    const int shift = 24 - 8 * pass;
    const uint32_t mask = pass == 0 ? 0u : 0xffffffffu << (shift + 8);
#pragma unroll 4
    for (int base = i0 + warp * 32; base < i1; base += THREADS) {
      const uint32_t k = base + lane < i1 ? key(base + lane) : 0u;
      const bool in = base + lane < i1 && (k & mask) == prefix;
      const unsigned live = __ballot_sync(0xffffffffu, in);
      if (in) {   // equal digits of a warp are one addition: scores crowd in few bins
        const int digit = (k >> shift) & 255;
        const unsigned same = __match_any_sync(live, digit);
        if (lane == __ffs(same) - 1) atomicAdd(&hist[pass][digit], __popc(same));
      }
    }
    sync();
    if (CL > 1) {   // the cluster's histogram
      for (int bin = tid; bin < 256; bin += THREADS) {
        int x[EV_MAX_CLUSTER], sum = 0;
#pragma unroll
        for (int q = 0; q < EV_MAX_CLUSTER; ++q) x[q] = q < CL ? ld_cluster(&hist[pass][bin], q) : 0;
#pragma unroll
        for (int q = 0; q < EV_MAX_CLUSTER; ++q) sum += x[q];
        s_hist[bin] = sum;
      }
      __syncthreads();
    }
    if (warp == 0) {   // bins from the top, 8 a lane
      const int* bins = CL > 1 ? s_hist : hist[pass];
      int x[8], mine = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) mine += x[j] = bins[255 - (lane * 8 + j)];
      int inc = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
      }
      int before = inc - mine;
      if (before < need && need <= inc) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (before < need && need <= before + x[j]) {
            s_cut[pass][0] = 255 - (lane * 8 + j);
            s_cut[pass][1] = need - before;
            s_cut[pass][2] = x[j];
          }
          before += x[j];
        }
      }
    }
    __syncthreads();
    prefix |= (uint32_t)s_cut[pass][0] << shift;
    need = s_cut[pass][1];
    if (need == s_cut[pass][2]) {   // the whole bin stays (never all slots, so prefix > 0): cut just below it
      prefix -= 1;
      need = 0;
      break;
    }
  }

  // Slots above the key stay, and of those equal to it the first `need` in slot
  // order.  Warps and blocks count before they list; warp w has 32-slot rows
  // [w0, w1) of the block's part.
  const int per = ((i1 - i0 + 31) / 32 + WARPS - 1) / WARPS * 32;
  const int w0 = i0 + warp * per, w1 = min(i1, w0 + per);
  const unsigned below = (1u << lane) - 1;
  // exclusive counts over the cluster of two numbers of a warp, and the first one's sum
  auto before_warp = [&](int which, int2 count, int& total) {
    if (lane == 0) s_warp[which][warp] = count;
    __syncthreads();
    int2 x = make_int2(0, 0), all = x;
    for (int w = 0; w < WARPS; ++w) {
      const int2 y = s_warp[which][w];
      if (w < warp) x.x += y.x, x.y += y.y;
      all.x += y.x, all.y += y.y;
    }
    total = all.x;
    if (CL > 1) {
      if (tid < CL) {
        st_cluster(&s_rank[which][rank].x, tid, all.x);
        st_cluster(&s_rank[which][rank].y, tid, all.y);
      }
      cluster_sync();
      total = 0;
      for (int q = 0; q < CL; ++q) {
        const int2 y = s_rank[which][q];
        if (q < rank) x.x += y.x, x.y += y.y;
        total += y.x;
      }
    }
    return x;
  };
  int count = 0, total = 0, eq0 = 0, moves = 0;
  if (need > 0) {   // uniform over the cluster: some of the slots at the cut stay and some go
    for (int base = w0; base < w1; base += 32)
      count += __popc(__ballot_sync(0xffffffffu, base + lane < w1 && key(base + lane) == prefix));
    eq0 = before_warp(0, make_int2(count, 0), total).x;
  }
  // f(slot, kept, its place among the freed below the budget, its place among the kept past it)
  auto walk = [&](int hole, int src, auto f) {
    int eq = eq0;
#pragma unroll 4
    for (int base = w0; base < w1; base += 32) {
      const int i = base + lane;
      const uint32_t k = i < w1 ? key(i) : 0u;
      const unsigned e = __ballot_sync(0xffffffffu, i < w1 && k == prefix);
      const bool keep = i < w1 && (k > prefix || (k == prefix && eq + __popc(e & below) < need));
      const unsigned bh = __ballot_sync(0xffffffffu, i < w1 && !keep && i < a.budget);
      const unsigned bs = __ballot_sync(0xffffffffu, keep && i >= a.budget);
      f(i, keep, bh, bs, hole, src);
      eq += __popc(e);
      hole += __popc(bh);
      src += __popc(bs);
    }
    count = hole;
    total = src;
  };
  walk(0, 0, [](int, bool, unsigned, unsigned, int, int) {});
  const int2 at0 = before_warp(1, make_int2(count, total), moves);
  int *holes = a.holes + task * a.max_moves, *srcs = a.srcs + task * a.max_moves;
  walk(at0.x, at0.y, [&](int i, bool, unsigned bh, unsigned bs, int hole, int src) {
    if (bh >> lane & 1) __stcg(holes + hole + __popc(bh & below), i);
    if (bs >> lane & 1) __stcg(srcs + src + __popc(bs & below), i);
  });
  sync();

  // the moves: batches of THREADS rows, this block every CL-th batch
  const int* table = a.c.table + b * a.c.table_stride;
  const int in_row = tid % a.chunks, row0 = tid / a.chunks, rows = THREADS / a.chunks;
  for (int j0 = rank * THREADS; j0 < moves; j0 += CL * THREADS) {
    const int j = j0 + tid;
    if (j < moves) {
      const int to = __ldcg(holes + j), of = __ldcg(srcs + j);
      const int tp = __ldg(table + to / a.c.page_size), fp = __ldg(table + of / a.c.page_size);
      const bool ok = (unsigned)tp < (unsigned)a.c.n_pages && (unsigned)fp < (unsigned)a.c.n_pages;
      if (!ok && a.c.status) set_status(a.c.status, ST_BOUNDS);
      const long long head = h * a.c.head_stride;
      s_to[tid] = tp * a.c.page_stride + (to % a.c.page_size) * a.c.slot_stride + head;
      s_of[tid] = ok ? fp * a.c.page_stride + (of % a.c.page_size) * a.c.slot_stride + head : -1;
      if (ok) {   // else the slot keeps its own
        so[to] = sc[of];
        po[to] = ps[of];
      }
    }
    __syncthreads();
    const int m = min(THREADS, moves - j0);
    constexpr int U = 4;
    for (int x0 = row0; x0 < m; x0 += rows * U) {
      uint4 k[U], v[U];
#pragma unroll
      for (int y = 0; y < U; ++y) {
        const int x = x0 + y * rows;
        if (x < m && s_of[x] >= 0) {
          k[y] = ldg_stream(a.c.k + s_of[x] + in_row * 16);
          v[y] = ldg_stream(a.c.v + s_of[x] + in_row * 16);
        }
      }
#pragma unroll
      for (int y = 0; y < U; ++y) {
        const int x = x0 + y * rows;
        if (x < m && s_of[x] >= 0) {
          *reinterpret_cast<uint4*>(a.c.k + s_to[x] + in_row * 16) = k[y];
          *reinterpret_cast<uint4*>(a.c.v + s_to[x] + in_row * 16) = v[y];
        }
      }
    }
    __syncthreads();
  }
}

// The shared memory above 48 KB of the large blocks, asked for once a device.
cudaError_t allow_large_keys() {
  static std::atomic<uint64_t> ready{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (!(ready.load(std::memory_order_acquire) & bit)) {
    e = cudaFuncSetAttribute(evict_kernel<1024>, cudaFuncAttributeMaxDynamicSharedMemorySize, EV_KEYS_LARGE * 4);
    if (e != cudaSuccess) return e;
    ready.fetch_or(bit, std::memory_order_release);
  }
  return cudaSuccess;
}

}  // namespace
}  // namespace asrspec

using namespace asrspec;

extern "C" {

// Moves of one head: no more than the freed slots below the budget, nor than the slots past it.
static int64_t evict_max_moves(const asr_paged_scores* s, int32_t budget) {
  const int64_t past = (int64_t)s->slots - budget;
  return past < 1 ? 1 : past < budget ? past : budget;
}

int64_t asr_spec_paged_evict_ws(const asr_paged_cache* c, const asr_paged_scores* s, int32_t budget) {
  PagedView v;
  if (int rc = paged_view(c, &v)) return rc;
  if (!s || s->slots < 1 || budget < 1) return ASR_E_INVAL;
  return ((int64_t)c->batch * c->kv_heads * 2 * evict_max_moves(s, budget) + c->batch) * 4;
}

int asr_spec_paged_evict(const asr_paged_cache* c, const asr_paged_scores* s, const int32_t* len, const int32_t* seen,
                         int32_t budget, int32_t recent, int32_t first, int32_t* len_out, void* ws, int64_t ws_bytes,
                         void* stream) {
  EvictArgs a{};
  if (int rc = paged_view(c, &a.c)) return rc;
  if (!s || !s->score || !s->score_out || !s->pos || !s->pos_out || !len || !seen || !len_out || !ws) return ASR_E_INVAL;
  if (s->slots < 1 || s->slots_out < 1 || s->head_stride < s->slots || s->out_head_stride < s->slots_out ||
      s->batch_stride < 0 || s->out_batch_stride < 0 || budget < 1 || recent < 0 || first < 0)
    return ASR_E_INVAL;
  if (((uintptr_t)s->score | (uintptr_t)s->score_out | (uintptr_t)s->pos | (uintptr_t)s->pos_out | (uintptr_t)len |
       (uintptr_t)seen | (uintptr_t)len_out | (uintptr_t)ws) % 4)
    return ASR_E_INVAL;
  const int64_t moves = evict_max_moves(s, budget), tasks = (int64_t)c->batch * c->kv_heads;
  if (ws_bytes < (tasks * 2 * moves + c->batch) * 4) return ASR_E_CAPACITY;
  a.len = len;
  a.seen = seen;
  a.score = s->score;
  a.pos = s->pos;
  a.in_b = s->batch_stride;
  a.in_h = s->head_stride;
  a.out_b = s->out_batch_stride;
  a.out_h = s->out_head_stride;
  a.score_out = s->score_out;
  a.pos_out = s->pos_out;
  a.len_out = len_out;
  a.in_cap = s->slots;
  a.out_cap = s->slots_out;
  a.budget = budget;
  a.recent = recent;
  a.first = first;
  a.max_moves = (int)moves;
  a.holes = static_cast<int*>(ws);
  a.srcs = a.holes + tasks * moves;
  a.chunks = c->head_dim * (c->dtype == 0 ? 4 : 2) / 16;
  // Heads read len while others may be done: in place, the lengths go through the workspace.
  const bool in_place = len_out == len;
  if (in_place) a.len_out = a.srcs + tasks * moves;
  // A block takes 2048 slots of a head comfortably; more blocks share a head
  // while all of them together stay below four an SM.
  int cluster = 1;
  while (cluster < EV_MAX_CLUSTER && s->slots > 2048 * cluster && tasks * cluster * 2 <= 4 * paged_sm_count()) cluster *= 2;
  const int part = (s->slots + cluster - 1) / cluster;
  a.keys = part < EV_KEYS ? part : EV_KEYS;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const dim3 grid(cluster, c->kv_heads, c->batch);
  cudaError_t e;
  // Few slots a block: smaller blocks, so that more heads share an SM and hide one another's passes.
  // Many slots and no more blocks than SMs: large blocks, which have an SM's shared memory to themselves
  // (12 heads of up to 120000 slots: 189 us with blocks of 256, 63 with these).
  if (part > 4096 && tasks * cluster <= paged_sm_count()) {
    a.keys = part < EV_KEYS_LARGE ? part : EV_KEYS_LARGE;
    e = allow_large_keys();
    if (e == cudaSuccess) e = launch_ex(evict_kernel<1024>, grid, dim3(1024), a.keys * 4, st, false, cluster, a);
  } else if (part <= 512) e = launch_ex(evict_kernel<128>, grid, dim3(128), a.keys * 4, st, false, cluster, a);
  else e = launch_ex(evict_kernel<256>, grid, dim3(256), a.keys * 4, st, false, cluster, a);
  if (e == cudaSuccess && in_place) e = cudaMemcpyAsync(len_out, a.len_out, c->batch * 4, cudaMemcpyDeviceToDevice, st);
  return e == cudaSuccess ? ASR_OK : ASR_E_CUDA;
}

}  // extern "C"
