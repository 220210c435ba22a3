// Verification of drafted tokens against the target's probabilities, from
// given random numbers (the sampled counterpart of the greedy longest-prefix
// acceptance).
//
//   p_i = softmax(target_i / T),  q_i = softmax(draft_i / T), or one at the drafted token
//   draft i is accepted while u_i q_i(x_i) < p_i(x_i), in order; n = accepted drafts
//   token = argmax_j w_j / e_j,  w = max(0, p_n - q_n) after a rejection, p_n after none
//
// e_j are given exponential variates: the argmax of w_j / e_j is a draw from w
// / sum w (of independent exponential clocks of rates w_j the first to ring is
// j with probability w_j / sum w), without a prefix sum over the vocabulary.
// So accepted drafts and token follow the target's distribution exactly.
//
// Two launches.  Statistics: every live row's (max, sum exp) in one pass, a
// row split over blocks so that one utterance fills the GPU too.  Decision:
// a cluster of 8 blocks per utterance; each combines the statistics, finds n
// and runs the race over an eighth of the vocabulary, and block 0 takes the
// best.  Bound by the bytes of the logits: rows past the first rejection are
// read as well (which rows those are is known only when all have been read).
// Everything is fp32; a maximum of (value, lowest index) keys does not depend
// on order, and the partial sums are combined in a fixed one.
#include "kernels.h"
#include "paged.cuh"

namespace asrspec {
namespace {

constexpr int AS_THREADS = 256;
constexpr int AS_CLUSTER = 8;
constexpr int AS_MAX_K = 31;
constexpr int AS_MAX_SPLIT = 32;

struct SampleArgs {
  const char *target, *draft_logits;         // draft_logits may be null
  long long t_b, t_r, d_b, d_r;              // bytes
  const int *draft, *lens;
  const float *u, *race;
  long long race_b;                          // elements
  float inv_t;
  int B, k, V, splits;
  int *accepted, *token, *step;
  float* prob;
  float2* part;                              // [B][2 k + 1][splits] (max, sum)
  int* status;
};

// Drafts of an utterance; -1 sits out.  A length or token out of range sets the status word and sits out.
__device__ __forceinline__ int live_drafts(const SampleArgs& a, int b) {
  const int n = a.lens ? a.lens[b] : a.k;
  if (n < -1 || n > a.k) {
    if (a.status) set_status(a.status, ST_BAD_LENS);
    return -1;
  }
  return n;
}

// logit -> finite or -inf: NaN counts as masked, +inf as the largest float
__device__ __forceinline__ float clean(float x) { return x != x ? -INFINITY : fminf(x, 3.4028234e38f); }

// exp((x - m) / T); 0 for a masked x or an empty row (m = -inf)
__device__ __forceinline__ float weight(float x, float m, float c) {
  return x == -INFINITY ? 0.f : exp2f((x - m) * c);
}

template <typename T> struct Vec16 {   // the values of 16 bytes
  static constexpr int N = 8;
  static __device__ __forceinline__ void get(const uint4& v, float* f) {
    const uint32_t r[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = r[i] & 0xffffu, hi = r[i] >> 16;
      const unsigned short a = (unsigned short)lo, b = (unsigned short)hi;
      f[2 * i] = to_f32(*reinterpret_cast<const T*>(&a));
      f[2 * i + 1] = to_f32(*reinterpret_cast<const T*>(&b));
    }
  }
};

template <> struct Vec16<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void get(const uint4& v, float* f) {
    f[0] = __uint_as_float(v.x), f[1] = __uint_as_float(v.y), f[2] = __uint_as_float(v.z), f[3] = __uint_as_float(v.w);
  }
};

template <typename T>
__global__ void __launch_bounds__(AS_THREADS) sample_stats_kernel(SampleArgs a) {
  constexpr int N = Vec16<T>::N, UN = 4;
  __shared__ float s_m[AS_THREADS / 32], s_l[AS_THREADS / 32];
  const int split = blockIdx.x, rr = blockIdx.y, b = blockIdx.z;
  const int n = live_drafts(a, b);
  pdl_launch();
  const bool is_draft = rr > a.k;
  const int row = is_draft ? rr - a.k - 1 : rr;
  if (n < 0 || row > n || (is_draft && row >= n)) return;
  const T* x = reinterpret_cast<const T*>(is_draft ? a.draft_logits + b * a.d_b + row * a.d_r : a.target + b * a.t_b + row * a.t_r);
  const float c = a.inv_t * LOG2E;
  // elements before the first 16-byte boundary, whole vectors, rest
  const int head = min(a.V, (int)(((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / sizeof(T)));
  const int nv = (a.V - head) / N, tail = head + nv * N;
  const int v0 = (int)((long long)nv * split / a.splits), v1 = (int)((long long)nv * (split + 1) / a.splits);
  const uint4* xv = reinterpret_cast<const uint4*>(x + head);
  float m = -INFINITY, l = 0.f;
  auto add = [&](const float* f, int cnt) {
    float mx = m;
    for (int i = 0; i < cnt; ++i) mx = fmaxf(mx, f[i]);
    if (mx == -INFINITY) return;
    if (mx > m) {
      l *= exp2f((m - mx) * c);
      m = mx;
    }
    for (int i = 0; i < cnt; ++i) l += weight(f[i], m, c);
  };
  for (int i = v0 + threadIdx.x; i < v1; i += AS_THREADS * UN) {
    uint4 v[UN];
    float f[UN * N];
#pragma unroll
    for (int j = 0; j < UN; ++j)
      if (i + j * AS_THREADS < v1) v[j] = ldg_stream(reinterpret_cast<const char*>(xv + i + j * AS_THREADS));
#pragma unroll
    for (int j = 0; j < UN; ++j) {
      if (i + j * AS_THREADS < v1) {
        Vec16<T>::get(v[j], f + j * N);
#pragma unroll
        for (int y = 0; y < N; ++y) f[j * N + y] = clean(f[j * N + y]);
      } else {
#pragma unroll
        for (int y = 0; y < N; ++y) f[j * N + y] = -INFINITY;
      }
    }
    float mx = m;
#pragma unroll
    for (int y = 0; y < UN * N; ++y) mx = fmaxf(mx, f[y]);
    if (mx == -INFINITY) continue;
    if (mx > m) {
      l *= exp2f((m - mx) * c);
      m = mx;
    }
#pragma unroll
    for (int y = 0; y < UN * N; ++y) l += weight(f[y], m, c);
  }
  if (split == 0 && threadIdx.x < 32) {   // the ragged ends
    const int lane = threadIdx.x;
    if (lane < head) {
      const float f = clean(to_f32(x[lane]));
      add(&f, 1);
    }
    if (tail + lane < a.V) {
      const float f = clean(to_f32(x[tail + lane]));
      add(&f, 1);
    }
  }
  auto combine = [&](float pm, float pl) {
    const float mx = fmaxf(m, pm);
    if (mx == -INFINITY) return;
    l = l * (m == -INFINITY ? 0.f : exp2f((m - mx) * c)) + pl * (pm == -INFINITY ? 0.f : exp2f((pm - mx) * c));
    m = mx;
  };
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float pm = __shfl_xor_sync(0xffffffffu, m, o), pl = __shfl_xor_sync(0xffffffffu, l, o);
    combine(pm, pl);
  }
  const int warp = threadIdx.x >> 5;
  if ((threadIdx.x & 31) == 0) {
    s_m[warp] = m;
    s_l[warp] = l;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < AS_THREADS / 32; ++w) combine(s_m[w], s_l[w]);
    a.part[((long long)b * (2 * a.k + 1) + rr) * a.splits + split] = make_float2(m, l);
  }
}

template <typename T>
__global__ void __launch_bounds__(AS_THREADS) sample_decide_kernel(SampleArgs a) {
  __shared__ float s_px[AS_MAX_K + 1], s_qx[AS_MAX_K + 1];   // p_i(x_i), q_i(x_i)
  __shared__ float s_pm[AS_MAX_K + 1], s_pl[AS_MAX_K + 1], s_qm[AS_MAX_K + 1], s_ql[AS_MAX_K + 1];
  __shared__ unsigned long long s_key[2][AS_THREADS / 32], s_best[2];
  __shared__ int s_bad;
  const int b = blockIdx.y, part = blockIdx.x, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int n_draft = live_drafts(a, b);
  const float c = a.inv_t * LOG2E;
  if (tid == 0) s_bad = 0;
  __syncthreads();
  for (int i = tid; i < n_draft; i += AS_THREADS) {
    const int x = a.draft[(long long)b * a.k + i];
    if (x < 0 || x >= a.V) s_bad = 1;
  }
  pdl_wait();
  __syncthreads();
  const bool out = n_draft < 0 || s_bad;   // uniform over the cluster
  if (s_bad && tid == 0 && part == 0 && a.status) set_status(a.status, ST_BAD_TOKEN);
  if (out) {
    if (part == 0) {
      if (tid == 0) {
        a.accepted[b] = 0;
        a.token[b] = -1;
        a.step[b] = 0;
      }
      for (int i = tid; i < a.k; i += AS_THREADS) a.prob[(long long)b * a.k + i] = 0.f;
    }
    return;
  }
  // a warp per row: combine its statistics, read the drafted token's probability
  for (int rr = warp; rr < 2 * a.k + 1; rr += AS_THREADS / 32) {
    const bool is_draft = rr > a.k;
    const int row = is_draft ? rr - a.k - 1 : rr;
    if (row > n_draft || (is_draft && (row >= n_draft || !a.draft_logits))) continue;
    float2 s = make_float2(-INFINITY, 0.f);
    if (lane < a.splits) s = a.part[((long long)b * (2 * a.k + 1) + rr) * a.splits + lane];
    const float m = warp_max(s.x);
    const float l = warp_sum(s.x == -INFINITY ? 0.f : s.y * exp2f((s.x - m) * c));
    if (lane == 0) {
      float px = 0.f;
      if (row < n_draft) {
        const int x = a.draft[(long long)b * a.k + row];
        const T* p = reinterpret_cast<const T*>(is_draft ? a.draft_logits + b * a.d_b + row * a.d_r
                                                         : a.target + b * a.t_b + row * a.t_r);
        px = l > 0.f ? weight(clean(to_f32(p[x])), m, c) / l : 0.f;
      }
      (is_draft ? s_qx : s_px)[row] = px;
      (is_draft ? s_qm : s_pm)[row] = m;
      (is_draft ? s_ql : s_pl)[row] = l;
    }
  }
  __syncthreads();
  // the first rejection (each warp finds it for itself)
  float px = 0.f, qx = 1.f;
  bool take = false;
  if (lane < n_draft) {
    px = s_px[lane];
    if (a.draft_logits) qx = s_qx[lane];
    take = a.u[(long long)b * a.k + lane] * qx < px;
  }
  const int n = __ffs(~__ballot_sync(0xffffffffu, take)) - 1;   // n_draft <= 31: lane n_draft never takes
  if (part == 0 && warp == 0 && lane < a.k)
    a.prob[(long long)b * a.k + lane] = lane < n_draft ? (px >= qx ? (px > 0.f ? 1.f : 0.f) : px / qx) : 0.f;
  // the race over this block's share of the vocabulary
  const bool rejected = n < n_draft;
  const T* pr = reinterpret_cast<const T*>(a.target + b * a.t_b + n * a.t_r);
  const T* qr = rejected && a.draft_logits ? reinterpret_cast<const T*>(a.draft_logits + b * a.d_b + n * a.d_r) : nullptr;
  const int gone = rejected && !a.draft_logits ? a.draft[(long long)b * a.k + n] : -1;
  const float pm = s_pm[n], pi = s_pl[n] > 0.f ? 1.f / s_pl[n] : 0.f;
  const float qm = qr ? s_qm[n] : 0.f, qi = qr && s_ql[n] > 0.f ? 1.f / s_ql[n] : 0.f;
  const float* e = a.race + b * a.race_b;
  const int v0 = (int)((long long)a.V * part / AS_CLUSTER), v1 = (int)((long long)a.V * (part + 1) / AS_CLUSTER);
  unsigned long long best = 0, best_p = 0;   // keys of positive values are above 2^63
#pragma unroll 4
  for (int j = v0 + tid; j < v1; j += AS_THREADS) {
    const float p = weight(clean(to_f32(pr[j])), pm, c) * pi;
    if (!(p > 0.f)) continue;
    const float ej = e[j];
    float w = p;
    if (qr) w = fmaxf(p - weight(clean(to_f32(qr[j])), qm, c) * qi, 0.f);
    if (j == gone) w = 0.f;
    const float vp = p / ej, vw = w / ej;
    if (vp > 0.f) {
      const unsigned long long x = argmax_key(vp, j);
      best_p = x > best_p ? x : best_p;
    }
    if (vw > 0.f) {
      const unsigned long long x = argmax_key(vw, j);
      best = x > best ? x : best;
    }
  }
  best = warp_max_u64(best);
  best_p = warp_max_u64(best_p);
  if (lane == 0) {
    s_key[0][warp] = best;
    s_key[1][warp] = best_p;
  }
  __syncthreads();
  if (tid < 2) {
    unsigned long long x = 0;
    for (int w = 0; w < AS_THREADS / 32; ++w) x = s_key[tid][w] > x ? s_key[tid][w] : x;
    s_best[tid] = x;
  }
  cluster_sync();
  if (part == 0 && warp == 0) {
    unsigned long long x = 0, y = 0;
    if (lane < AS_CLUSTER) {
      asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(x) : "r"(dsmem_addr(&s_best[0], lane)));
      asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(y) : "r"(dsmem_addr(&s_best[1], lane)));
    }
    x = warp_max_u64(x);
    y = warp_max_u64(y);
    if (lane == 0) {
      const unsigned long long k = x ? x : y;   // no residual left (p = q): draw from p
      a.accepted[b] = n;
      a.token[b] = k ? (int)argmax_index(k) : -1;
      a.step[b] = k ? n + 1 : 0;
    }
  }
  cluster_sync();   // s_best stays until block 0 has read it
}

int pick_splits(int rows, int V) {
  // A row is cut so that all rows together give each SM a few blocks, none below 2048 elements.
  int s = (8 * paged_sm_count() + rows - 1) / rows;
  const int most = V / 2048 < 1 ? 1 : V / 2048;
  if (s > most) s = most;
  return s < 1 ? 1 : s > AS_MAX_SPLIT ? AS_MAX_SPLIT : s;
}

}  // namespace
}  // namespace asrspec

using namespace asrspec;

extern "C" {

int64_t asr_spec_accept_sampled_ws(int32_t B, int32_t k) {
  if (B < 1 || B > 65535 || k < 0 || k > AS_MAX_K) return ASR_E_INVAL;
  return (int64_t)B * (2 * k + 1) * AS_MAX_SPLIT * sizeof(float2);
}

int asr_spec_accept_sampled(const asr_sampled_logits* x, const int32_t* draft, const int32_t* lens, const float* u,
                            const float* race, int64_t race_stride, float temperature, int32_t* accepted, int32_t* token,
                            int32_t* step, float* prob, int32_t* status, void* ws, int64_t ws_bytes, void* stream) {
  if (!x || !x->target || !race || !accepted || !token || !step || !ws) return ASR_E_INVAL;
  if (x->dtype < 0 || x->dtype > 2 || x->batch < 1 || x->batch > 65535 || x->k < 0 || x->k > AS_MAX_K || x->vocab < 1 ||
      x->vocab > (1 << 30))
    return ASR_E_INVAL;
  if (x->k > 0 && (!draft || !u || !prob)) return ASR_E_INVAL;
  if (!(temperature > 0.f) || !(1.f / temperature > 0.f) || !(1.f / temperature < 3e38f)) return ASR_E_INVAL;
  const int64_t es = x->dtype == 0 ? 4 : 2;
  if (x->target_row_stride < x->vocab || x->target_batch_stride < 0 || race_stride < x->vocab ||
      (x->draft_logits && (x->draft_row_stride < x->vocab || x->draft_batch_stride < 0)))
    return ASR_E_INVAL;
  if ((uintptr_t)x->target % es || (uintptr_t)x->draft_logits % es ||
      ((uintptr_t)draft | (uintptr_t)lens | (uintptr_t)u | (uintptr_t)race | (uintptr_t)accepted | (uintptr_t)token |
       (uintptr_t)step | (uintptr_t)prob | (uintptr_t)status) % 4 ||
      (uintptr_t)ws % 8)
    return ASR_E_INVAL;
  if (ws_bytes < asr_spec_accept_sampled_ws(x->batch, x->k)) return ASR_E_CAPACITY;
  SampleArgs a{};
  a.target = static_cast<const char*>(x->target);
  a.draft_logits = static_cast<const char*>(x->draft_logits);
  a.t_b = x->target_batch_stride * es;
  a.t_r = x->target_row_stride * es;
  a.d_b = x->draft_batch_stride * es;
  a.d_r = x->draft_row_stride * es;
  a.draft = draft;
  a.lens = lens;
  a.u = u;
  a.race = race;
  a.race_b = race_stride;
  a.inv_t = 1.f / temperature;
  a.B = x->batch;
  a.k = x->k;
  a.V = x->vocab;
  a.accepted = accepted;
  a.token = token;
  a.step = step;
  a.prob = prob;
  a.part = static_cast<float2*>(ws);
  a.status = status;
  const int rows = x->draft_logits ? 2 * x->k + 1 : x->k + 1;
  a.splits = pick_splits(rows * x->batch, x->vocab);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const dim3 g1(a.splits, rows, x->batch), g2(AS_CLUSTER, x->batch), blk(AS_THREADS);
  cudaError_t e;
  auto go = [&](auto stats, auto decide) {
    cudaError_t r = launch_ex(stats, g1, blk, 0, st, false, 1, a);
    return r != cudaSuccess ? r : launch_ex(decide, g2, blk, 0, st, true, AS_CLUSTER, a);
  };
  if (x->dtype == 0) e = go(sample_stats_kernel<float>, sample_decide_kernel<float>);
  else if (x->dtype == 1) e = go(sample_stats_kernel<__nv_bfloat16>, sample_decide_kernel<__nv_bfloat16>);
  else e = go(sample_stats_kernel<__half>, sample_decide_kernel<__half>);
  return e == cudaSuccess ? ASR_OK : ASR_E_CUDA;
}

}  // extern "C"
