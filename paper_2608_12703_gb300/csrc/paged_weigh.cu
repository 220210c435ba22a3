// The attention weight that each cached slot received from a block's committed
// rows, added to a running score per (sequence, K/V head, slot):
//
//   score'[j] = (j < kv_len ? score[j] : 0) + sum_r sum_h exp(scale q_rh k_j - lse_rh)
//
// over rows r < rows[b] that see slot j (j <= kv_len + r, or j < kv_len when
// not causal) and the query heads h of the K/V head.  It runs after the
// verification, when the number of committed rows is known, on the lse that
// the attention left: one pass over K, no join.  Bound by the bytes of K and
// of the scores; keys come from the pages into registers a step ahead, each warp a
// contiguous run of steps.  16-bit products are exact, fp32 ones fp32 (no TF32);
// all sums are fp32 in a fixed order, exp2 is the hardware's.
// Measured: 8 sequences of up to 40000 slots, 32 query heads on 8 of 128, bf16:
// 78 us for 506 MB, 96 % of the copy rate (four blocks of four warps an SM, 4 KB
// of K a warp in flight); 64 of up to 448 slots, 7 rows, 20 heads of 64: 11.6 us
// for 40 MB, launch and latency.
#include <type_traits>

#include "kernels.h"
#include "paged.cuh"

namespace asrspec {
namespace {

constexpr int PW_WARPS = 4;

struct WeighArgs {
  PagedView c;
  PagedRows r;
  const float *lse, *score;   // score may be null (zeros)
  float* out;
  long long lse_b, lse_r, score_b, score_h;   // elements
  int* pos;                   // or null; strides as score's
  const int* first_pos;
  int cap;
};

// A sequence without rows keeps its scores: its slots still take part.
template <int KS, int TR>
__device__ __forceinline__ SeqWork weigh_seq(const WeighArgs& a, int len, int rows) {
  SeqWork s = seq_work<KS, TR>(a.r, len, rows);
  s.paged = len + (a.r.causal ? rows : 0);
  if (s.paged > a.cap) {
    if (a.c.status) set_status(a.c.status, ST_CAPACITY);
    s.len = s.rows = s.paged = s.tiles = 0;
  }
  s.keys = s.paged;
  s.steps = (s.paged + KS - 1) / KS;
  return s;
}

// One lane's slot: its score before, and the end of it.
__device__ __forceinline__ float old_score(const WeighArgs& a, const SeqWork& s, int b, int kvh, int key) {
  return key < min(s.len, s.paged) && a.score ? __ldcg(a.score + b * a.score_b + kvh * a.score_h + key) : 0.f;
}
__device__ __forceinline__ void put_score(const WeighArgs& a, const SeqWork& s, int b, int kvh, int key, float v) {
  if (key >= s.paged) return;
  const long long at = b * a.score_b + kvh * a.score_h + key;
  a.out[at] = v;
  if (a.pos && key >= s.len) a.pos[at] = a.first_pos[b] + key - s.len;   // the slot of a new row
}

template <typename T, int D>
__global__ void __launch_bounds__(PW_WARPS * 32, 4) weigh16_kernel(WeighArgs a, int max_workers) {
  constexpr int KS = Cfg16<D>::KS, NG = KS / PG_GROUP, NC = D / 32, TR = 16;
  const PagedView& c = a.c;
  const PagedRows& r = a.r;
  PlanMem mem;
  const WorkPlan plan = work_plan(c, r, mem, max_workers, [&](int len, int rows) {
    return c.kv_heads * weigh_seq<KS, TR>(a, len, rows).steps;
  });
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int worker = (threadIdx.x >> 5) * gridDim.x + blockIdx.x;
  if (plan.units == 0 || worker >= plan.workers) return;
  int u = plan.start(worker);
  const int u_end = plan.start(worker + 1);
  const float sc = r.scale * LOG2E;

  while (u < u_end) {
    const int b = work_find(mem.pre, c.batch, u);
    const SeqWork s = weigh_seq<KS, TR>(a, mem.lens[b].x, mem.lens[b].y);
    const int rem = u - mem.pre[b], kvh = rem / s.steps, s0 = rem - kvh * s.steps;
    const int n = min(s.steps - s0, u_end - u);
    u += n;
    Keys16<T, D> ks{c, r, s, c.table + b * c.table_stride, kvh * c.head_stride, nullptr, nullptr, g, t};
    int pid[NG];
    long long off[NG];
    uint4 kf[KS / 8][NC];
    if (s.tiles) {
#pragma unroll
      for (int x = 0; x < NG; ++x) pid[x] = ks.id(s0, x);
      ks.offsets(s0, pid, off);
      ks.load_k(s0, off, kf);
      if (n > 1)
#pragma unroll
        for (int x = 0; x < NG; ++x) pid[x] = ks.id(s0 + 1, x);
    }
    uint32_t qa[NC * 2][4];
    float ls[2];
    int lim[2];
    auto rows_of = [&](int tile) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int m = tile * TR + e * 8 + g, row = m / r.group, hq = kvh * r.group + m - row * r.group;
        const bool in = row < s.rows;
        const float x = in ? a.lse[b * a.lse_b + row * a.lse_r + hq] : -INFINITY;
        lim[e] = x == -INFINITY ? 0 : r.causal ? s.len + row + 1 : s.paged;   // an empty row weighs nothing, whatever its scores
        ls[e] = x * LOG2E;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
          const uint4 v = in ? __ldg(reinterpret_cast<const uint4*>(r.q + b * r.q_b + row * r.q_r + hq * r.q_h +
                                                                    j * 64 + t * 16))
                             : make_uint4(0, 0, 0, 0);
          qa[2 * j][e] = v.x;
          qa[2 * j][2 + e] = v.y;
          qa[2 * j + 1][e] = v.z;
          qa[2 * j + 1][2 + e] = v.w;
        }
      }
    };
    if (s.tiles) rows_of(0);
    // Of a step's KS slots a lane ends with the sum of one, after the exchange below.
    constexpr int V = KS / 4;
    const int mine = ((g % V) >> 1) * 8 + 2 * t + (g & 1);
    float old = old_score(a, s, b, kvh, s0 * KS + mine);
    for (int i = 0; i < n; ++i) {
      const int step = s0 + i;
      float w[KS / 8][2];
#pragma unroll
      for (int kt = 0; kt < KS / 8; ++kt) w[kt][0] = w[kt][1] = 0.f;
      for (int tile = 0; tile < s.tiles; ++tile) {
        if (s.tiles > 1) rows_of(tile);
        float S[KS / 8][4];
#pragma unroll
        for (int kt = 0; kt < KS / 8; ++kt) {
          S[kt][0] = S[kt][1] = S[kt][2] = S[kt][3] = 0.f;
#pragma unroll
          for (int j = 0; j < NC; ++j) {
            Mma16<T>::mma(S[kt], qa[2 * j], kf[kt][j].x, kf[kt][j].y);
            Mma16<T>::mma(S[kt], qa[2 * j + 1], kf[kt][j].z, kf[kt][j].w);
          }
        }
#pragma unroll
        for (int kt = 0; kt < KS / 8; ++kt)
#pragma unroll
          for (int x = 0; x < 4; ++x)
            if (step * KS + kt * 8 + 2 * t + (x & 1) < lim[x >> 1]) w[kt][x & 1] += ex2(fmaf(S[kt][x], sc, -ls[x >> 1]));
      }
      if (s.tiles && i + 1 < n) {
        ks.offsets(step + 1, pid, off);
        ks.load_k(step + 1, off, kf);
        if (i + 2 < n)
#pragma unroll
          for (int x = 0; x < NG; ++x) pid[x] = ks.id(step + 2, x);
      }
      const float before = old;
      if (i + 1 < n) old = old_score(a, s, b, kvh, (step + 1) * KS + mine);
      // The eight lanes of a column hold the sums of their rows for V slots
      // each: every exchange halves the slots that a lane goes on with.
      float v[V];
#pragma unroll
      for (int x = 0; x < V; ++x) v[x] = w[x >> 1][x & 1];
      if (V == 8) {
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float give = g & 4 ? v[x] : v[x + V / 2], keep = g & 4 ? v[x + V / 2] : v[x];
          v[x] = keep + __shfl_xor_sync(0xffffffffu, give, 16);
        }
      } else {
#pragma unroll
        for (int x = 0; x < V; ++x) v[x] += __shfl_xor_sync(0xffffffffu, v[x], 16);
      }
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const float give = g & 2 ? v[x] : v[x + 2], keep = g & 2 ? v[x + 2] : v[x];
        v[x] = keep + __shfl_xor_sync(0xffffffffu, give, 8);
      }
      const float give = g & 1 ? v[0] : v[1], keep = g & 1 ? v[1] : v[0];
      const float sum = keep + __shfl_xor_sync(0xffffffffu, give, 4);
      if (g < V) put_score(a, s, b, kvh, step * KS + mine, before + sum);
    }
  }
}

// fp32 (no TF32): eight lanes share a key, four keys at a time; rows from L1.
template <int D>
__global__ void __launch_bounds__(PW_WARPS * 32) weigh32_kernel(WeighArgs a, int max_workers) {
  constexpr int KS = 16, IT = KS / 4, NC = D / 32;
  const PagedView& c = a.c;
  const PagedRows& r = a.r;
  PlanMem mem;
  const WorkPlan plan = work_plan(c, r, mem, max_workers, [&](int len, int rows) {
    return c.kv_heads * weigh_seq<KS, 1>(a, len, rows).steps;
  });
  const int lane = threadIdx.x & 31, kg = lane >> 3, e = lane & 7;
  const int worker = (threadIdx.x >> 5) * gridDim.x + blockIdx.x;
  if (plan.units == 0 || worker >= plan.workers) return;
  int u = plan.start(worker);
  const int u_end = plan.start(worker + 1);
  const float sc = r.scale * LOG2E;

  while (u < u_end) {
    const int b = work_find(mem.pre, c.batch, u);
    const SeqWork s = weigh_seq<KS, 1>(a, mem.lens[b].x, mem.lens[b].y);
    const int rem = u - mem.pre[b], kvh = rem / s.steps, step = rem - kvh * s.steps;
    ++u;
    const int grp = step;
    float4 kf[IT][NC];
    if (s.tiles) {
      const char* p = c.k + paged_offset(c, paged_id(c, c.table + b * c.table_stride, grp), grp) + kvh * c.head_stride +
                      kg * c.slot_stride + e * 16;
#pragma unroll
      for (int k = 0; k < IT; ++k)
#pragma unroll
        for (int j = 0; j < NC; ++j)
          kf[k][j] = step * KS + 4 * k + kg < s.paged
                         ? *reinterpret_cast<const float4*>(p + (long long)(4 * k) * c.slot_stride + j * 128)
                         : make_float4(0.f, 0.f, 0.f, 0.f);
    }
    float w[IT];
#pragma unroll
    for (int k = 0; k < IT; ++k) w[k] = 0.f;
    // Four rows at a time are independent chains of products and exchanges; one
    // or two rows would pay for four (one row, 128 wide: 20 us against 25).
    auto add_rows = [&](auto at_once, int m0) {
      constexpr int MR = decltype(at_once)::value;
      float d[MR][IT], ls[MR];
      int lim[MR];
#pragma unroll
      for (int x = 0; x < MR; ++x) {
        const int m = min(m0 + x, s.tiles - 1), row = (int)r.groups.div((uint32_t)m), hq = kvh * r.group + m - row * r.group;
        const float y = a.lse[b * a.lse_b + row * a.lse_r + hq];
        lim[x] = m0 + x < s.tiles && y != -INFINITY ? (r.causal ? s.len + row + 1 : s.paged) : 0;
        ls[x] = y * LOG2E;
#pragma unroll
        for (int k = 0; k < IT; ++k) d[x][k] = 0.f;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
          const float4 q =
              __ldg(reinterpret_cast<const float4*>(r.q + b * r.q_b + row * r.q_r + hq * r.q_h + (e + 8 * j) * 16));
#pragma unroll
          for (int k = 0; k < IT; ++k)
            d[x][k] += (q.x * kf[k][j].x + q.y * kf[k][j].y) + (q.z * kf[k][j].z + q.w * kf[k][j].w);
        }
      }
#pragma unroll
      for (int o = 1; o < 8; o <<= 1)
#pragma unroll
        for (int x = 0; x < MR; ++x)
#pragma unroll
          for (int k = 0; k < IT; ++k) d[x][k] += __shfl_xor_sync(0xffffffffu, d[x][k], o);
#pragma unroll
      for (int x = 0; x < MR; ++x)
#pragma unroll
        for (int k = 0; k < IT; ++k)
          if (step * KS + 4 * k + kg < lim[x]) w[k] += ex2(fmaf(d[x][k], sc, -ls[x]));
    };
    if (s.tiles > 2) {
      for (int m0 = 0; m0 < s.tiles; m0 += 4) add_rows(std::integral_constant<int, 4>{}, m0);
    } else {
      for (int m0 = 0; m0 < s.tiles; ++m0) add_rows(std::integral_constant<int, 1>{}, m0);
    }
#pragma unroll
    for (int k = 0; k < IT; ++k)
      if (e == k) {
        const int key = step * KS + 4 * k + kg;
        put_score(a, s, b, kvh, key, old_score(a, s, b, kvh, key) + w[k]);
      }
  }
}

}  // namespace
}  // namespace asrspec

using namespace asrspec;

extern "C" int asr_spec_paged_weigh(const asr_paged_cache* c, const asr_paged_rows* r, const asr_paged_scores* sc,
                                    const float* lse, int64_t lse_batch_stride, int64_t lse_row_stride, void* stream) {
  WeighArgs a{};
  if (int rc = paged_view(c, &a.c)) return rc;
  if (int rc = paged_rows(c, r, &a.r)) return rc;
  a.r.k_new = a.r.v_new = nullptr;   // the block's rows are in their pages
  if (!sc || !sc->score_out || !lse || sc->slots < 1 || sc->head_stride < sc->slots || sc->batch_stride < 0)
    return ASR_E_INVAL;
  if ((sc->pos != nullptr) != (sc->first_pos != nullptr)) return ASR_E_INVAL;
  if (((uintptr_t)sc->score | (uintptr_t)sc->score_out | (uintptr_t)sc->pos | (uintptr_t)sc->first_pos | (uintptr_t)lse) % 4)
    return ASR_E_INVAL;
  if ((long long)c->kv_heads * c->batch * (a.c.max_slots / PG_GROUP + 1) > 0x7fffffffll) return ASR_E_CAPACITY;   // 32-bit units
  a.lse = lse;
  a.lse_b = lse_batch_stride;
  a.lse_r = lse_row_stride;
  a.score = sc->score;
  a.out = sc->score_out;
  a.score_b = sc->batch_stride;
  a.score_h = sc->head_stride;
  a.pos = sc->pos;
  a.first_pos = sc->first_pos;
  a.cap = sc->slots;
  const int grid = paged_sm_count() * 4, workers = grid * PW_WARPS;
  const size_t smem = plan_bytes(c->batch);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const dim3 g(grid), b(PW_WARPS * 32);
  cudaError_t e;
  const bool wide = c->head_dim == 128;
  if (c->dtype == 0)
    e = wide ? launch_ex(weigh32_kernel<128>, g, b, smem, st, false, 1, a, workers)
             : launch_ex(weigh32_kernel<64>, g, b, smem, st, false, 1, a, workers);
  else if (c->dtype == 1)
    e = wide ? launch_ex(weigh16_kernel<__nv_bfloat16, 128>, g, b, smem, st, false, 1, a, workers)
             : launch_ex(weigh16_kernel<__nv_bfloat16, 64>, g, b, smem, st, false, 1, a, workers);
  else
    e = wide ? launch_ex(weigh16_kernel<__half, 128>, g, b, smem, st, false, 1, a, workers)
             : launch_ex(weigh16_kernel<__half, 64>, g, b, smem, st, false, 1, a, workers);
  return e == cudaSuccess ? ASR_OK : ASR_E_CUDA;
}
