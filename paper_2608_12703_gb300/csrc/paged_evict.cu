// Eviction from a paged K/V cache by accumulated attention weight.
//
// Per (sequence, K/V head) with more than `budget` slots in use, the budget
// slots of highest rank stay: protected slots first (one of the `recent`
// newest positions, or of the `first` oldest), then by score, equal scores by
// lowest slot; a NaN score ranks lowest.  A cached key carries its position in
// itself, so the slots' order is free: the j-th freed slot below the budget
// takes the j-th kept slot at or past it.  Sources and destinations are
// disjoint, so the moves run in any order over the whole GPU and move the
// fewest rows there are to move.
//   * select: one block per (sequence, head) finds the rank of the last kept
//     slot by a radix search, 8 bits a pass over a histogram, then lists freed
//     and kept slots in slot order and writes the kept scores and positions;
//   * move: one 16-byte chunk a lane, rows of K and V from list to list.
#include "kernels.h"
#include "paged.cuh"

namespace asrspec {
namespace {

constexpr int EV_THREADS = 512;
constexpr int EV_WARPS = EV_THREADS / 32;

struct EvictArgs {
  PagedView c;
  const int *len, *seen;
  const float* score;
  const int* pos;
  long long in_b, in_h, out_b, out_h;   // elements
  float* score_out;
  int *pos_out, *len_out;
  int in_cap, out_cap, budget, recent, first;
  int *count, *holes, *srcs;            // workspace: [B K], [B K][max_moves] each
  int max_moves;
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

__global__ void __launch_bounds__(EV_THREADS) evict_select_kernel(EvictArgs a) {
  __shared__ int hist[256];
  __shared__ uint32_t s_prefix;
  __shared__ int s_need;
  __shared__ int s_cnt[3][EV_WARPS];
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int n = evict_len(a, b), task = b * a.c.kv_heads + h;
  const float* sc = a.score + b * a.in_b + h * a.in_h;
  const int* ps = a.pos + b * a.in_b + h * a.in_h;
  float* so = a.score_out + b * a.out_b + h * a.out_h;
  int* po = a.pos_out + b * a.out_b + h * a.out_h;
  pdl_launch();
  if (n <= a.budget) {
    if (so != sc)
      for (int i = tid; i < n; i += EV_THREADS) so[i] = sc[i];
    if (po != ps)
      for (int i = tid; i < n; i += EV_THREADS) po[i] = ps[i];
    if (tid == 0) a.count[task] = 0;
    return;
  }
  const int newest = a.seen[b] - a.recent;
  // the key of the budget-th slot: fix 8 bits a pass from the top
  uint32_t prefix = 0;
  int need = a.budget;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256; i += EV_THREADS) hist[i] = 0;
    __syncthreads();
    const uint32_t mask = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
    for (int i = tid; i < n; i += EV_THREADS) {
      const uint32_t k = rank_key(sc[i], ps[i], newest, a.first);
      if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & 255], 1);
    }
    __syncthreads();
    if (warp == 0) {   // bins from the top, 8 a lane
      int mine = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) mine += hist[255 - (lane * 8 + j)];
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
          const int bin = 255 - (lane * 8 + j), x = hist[bin];
          if (before < need && need <= before + x) {
            s_prefix = prefix | ((uint32_t)bin << shift);
            s_need = need - before;
          }
          before += x;
        }
      }
    }
    __syncthreads();
    prefix = s_prefix;
    need = s_need;
  }
  // in slot order: slots above the key stay, and the first `need` equal to it
  int *holes = a.holes + (size_t)task * a.max_moves, *srcs = a.srcs + (size_t)task * a.max_moves;
  int n_eq = 0, n_hole = 0, n_src = 0;
  for (int i0 = 0; i0 < n; i0 += EV_THREADS) {
    const int i = i0 + tid;
    const bool in = i < n;
    float x = 0.f;
    int p = 0;
    uint32_t k = 0;
    if (in) {
      x = sc[i];
      p = ps[i];
      k = rank_key(x, p, newest, a.first);
    }
    const unsigned below = (1u << lane) - 1;
    const unsigned beq = __ballot_sync(0xffffffffu, in && k == prefix);
    if (lane == 0) s_cnt[0][warp] = __popc(beq);
    __syncthreads();
    int eq = n_eq + __popc(beq & below);
    for (int w = 0; w < EV_WARPS; ++w) {
      if (w < warp) eq += s_cnt[0][w];
      n_eq += s_cnt[0][w];
    }
    const bool keep = in && (k > prefix || (k == prefix && eq < need));
    const bool hole = in && !keep && i < a.budget, src = keep && i >= a.budget;
    const unsigned bh = __ballot_sync(0xffffffffu, hole), bs = __ballot_sync(0xffffffffu, src);
    if (lane == 0) {
      s_cnt[1][warp] = __popc(bh);
      s_cnt[2][warp] = __popc(bs);
    }
    __syncthreads();
    int at_h = n_hole + __popc(bh & below), at_s = n_src + __popc(bs & below);
    for (int w = 0; w < EV_WARPS; ++w) {
      if (w < warp) {
        at_h += s_cnt[1][w];
        at_s += s_cnt[2][w];
      }
      n_hole += s_cnt[1][w];
      n_src += s_cnt[2][w];
    }
    if (hole) holes[at_h] = i;
    if (src) srcs[at_s] = i;
    if (keep && i < a.budget) {
      so[i] = x;
      po[i] = p;
    }
  }
  __syncthreads();
  for (int j = tid; j < n_hole; j += EV_THREADS) {
    const int to = holes[j], of = srcs[j];
    so[to] = sc[of];
    po[to] = ps[of];
  }
  if (tid == 0) a.count[task] = n_hole;
}

constexpr int EM_THREADS = 256;

__global__ void __launch_bounds__(EM_THREADS) evict_move_kernel(EvictArgs a, int chunks) {
  const int h = blockIdx.y, b = blockIdx.z, task = b * a.c.kv_heads + h;
  pdl_wait();
  if (h == 0 && blockIdx.x == 0 && threadIdx.x == 0) {
    const int n = evict_len(a, b);
    a.len_out[b] = n < 0 ? a.len[b] : min(n, a.budget);
  }
  const int n = a.count[task];
  const int* table = a.c.table + b * a.c.table_stride;
  const long long head = h * a.c.head_stride;
  const int per = EM_THREADS / chunks;   // rows a block moves at a time
  const int chunk = threadIdx.x % chunks;
  for (int j = blockIdx.x * per + threadIdx.x / chunks; j < n; j += gridDim.x * per) {
    const int to = a.holes[(size_t)task * a.max_moves + j], of = a.srcs[(size_t)task * a.max_moves + j];
    const int tp = table[to / a.c.page_size], fp = table[of / a.c.page_size];
    if ((unsigned)tp >= (unsigned)a.c.n_pages || (unsigned)fp >= (unsigned)a.c.n_pages) {
      if (a.c.status) set_status(a.c.status, ST_BOUNDS);
      continue;
    }
    const long long t = tp * a.c.page_stride + (to % a.c.page_size) * a.c.slot_stride + head + chunk * 16;
    const long long f = fp * a.c.page_stride + (of % a.c.page_size) * a.c.slot_stride + head + chunk * 16;
    const uint4 k = *reinterpret_cast<const uint4*>(a.c.k + f), v = *reinterpret_cast<const uint4*>(a.c.v + f);
    *reinterpret_cast<uint4*>(a.c.k + t) = k;
    *reinterpret_cast<uint4*>(a.c.v + t) = v;
  }
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
  return (int64_t)c->batch * c->kv_heads * (1 + 2 * evict_max_moves(s, budget)) * 4;
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
  if (ws_bytes < tasks * (1 + 2 * moves) * 4) return ASR_E_CAPACITY;
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
  a.count = static_cast<int*>(ws);
  a.holes = a.count + tasks;
  a.srcs = a.holes + tasks * moves;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = launch_ex(evict_select_kernel, dim3(c->kv_heads, c->batch), dim3(EV_THREADS), 0, st, false, 1, a);
  if (e != cudaSuccess) return ASR_E_CUDA;
  const int chunks = c->head_dim * (c->dtype == 0 ? 4 : 2) / 16, per = EM_THREADS / chunks;
  int64_t x = (moves + per - 1) / per;
  const int64_t most = (paged_sm_count() * 16 + tasks - 1) / tasks;
  if (x > most) x = most;
  e = launch_ex(evict_move_kernel, dim3((unsigned)x, c->kv_heads, c->batch), dim3(EM_THREADS), 0, st, true, 1, a, chunks);
  return e == cudaSuccess ? ASR_OK : ASR_E_CUDA;
}

}  // extern "C"
