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
// One launch, a cluster of blocks per utterance, each on its share of the
// vocabulary.  First every live row's (max, sum exp) in one pass; the blocks
// exchange them through distributed shared memory, and each finds n for itself
// and runs the race over its share; rank 0 takes the best.  Bound by the bytes
// of the logits: rows past the first rejection are read as well (which rows
// those are is known only when all have been read).  Everything is fp32; a
// maximum of (value, lowest index) keys does not depend on order, and the
// partial sums are combined in a fixed one.
// Measured: 64 utterances of 6 drafts with their logits, 51866 tokens, fp32: 38 us
// (173 MB; 32 of them up to the first rejection, the statistics' 159 MB at 5
// TB/s); one of 8 greedy drafts: 9.6 us, latency.
// Loads go straight to registers: through shared memory by asynchronous 16-byte
// copies the first took 65 us for 54, by bulk copies and a block barrier a chunk
// 63 for 43.
#include <atomic>

#include "kernels.h"
#include "paged.cuh"

namespace asrspec {
namespace {

constexpr int AS_MAX_K = 31;
constexpr int AS_ROWS = 2 * AS_MAX_K + 1;
// A residual p - q of no more than this part of p is the rounding of p and q:
// equal rows that are aligned differently add up in different orders, and their
// sums differ by some 2^-22.  It counts as 0, so that p = q leaves nothing to
// draw from; what a true residual of that size weighs is 2^-18 of the tokens at most.
constexpr float NO_RESIDUAL = 1.f / (1 << 18);

struct SampleArgs {
  const char *target, *draft_logits;         // draft_logits may be null
  long long t_b, t_r, d_b, d_r;              // bytes
  const int *draft, *lens;
  const float *u, *race;
  long long race_b;                          // elements
  float inv_t;
  int k, V;
  int *accepted, *token, *step;
  float* prob;
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
__device__ __forceinline__ float clean(float x) { return fminf(fmaxf(x, -INFINITY), 3.4028234e38f); }

// exp((x - m) / T) for finite m; 0 for a masked x
__device__ __forceinline__ float weight(float x, float m, float c) { return ex2((x - m) * c); }

// The values of 16 bytes, and their maximum (which passes over NaN).
template <typename T> struct Vec16;
template <> struct Vec16<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void get(const uint4& v, float* f) {
    f[0] = __uint_as_float(v.x), f[1] = __uint_as_float(v.y), f[2] = __uint_as_float(v.z), f[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ float top(const uint4& v) {
    return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
  }
};
template <> struct Vec16<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void get(const uint4& v, float* f) {
    const uint32_t r[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[2 * i] = __uint_as_float(r[i] << 16), f[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
  }
  static __device__ __forceinline__ float top(const uint4& v) {
    const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&v);
    const float2 f = __bfloat1622float2(__hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3])));
    return fmaxf(f.x, f.y);
  }
};
template <> struct Vec16<__half> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void get(const uint4& v, float* f) {
    const __half2* p = reinterpret_cast<const __half2*>(&v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 x = __half22float2(p[i]);
      f[2 * i] = x.x, f[2 * i + 1] = x.y;
    }
  }
  static __device__ __forceinline__ float top(const uint4& v) {
    const __half2* p = reinterpret_cast<const __half2*>(&v);
    const float2 f = __half22float2(__hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3])));
    return fmaxf(f.x, f.y);
  }
};

// Weights of two raw logits, two lanes an instruction where there is one: the
// saturation to [0, 1] turns the NaN of a NaN logit into 0 and the infinity of
// an infinite one into 1.
__device__ __forceinline__ uint64_t pair(float x) {
  const uint32_t b = __float_as_uint(x);
  return (uint64_t)b << 32 | b;
}
__device__ __forceinline__ float weight2(float x, float y, uint64_t minus_m, uint64_t c) {
  float d, e;
  asm("{\n\t.reg .b64 t;\n\tmov.b64 t, {%2, %3};\n\tadd.rn.f32x2 t, t, %4;\n\tmul.rn.f32x2 t, t, %5;\n\t"
      "mov.b64 {%0, %1}, t;\n\t}"
      : "=f"(d), "=f"(e)
      : "f"(x), "f"(y), "l"(minus_m), "l"(c));
  return __saturatef(ex2(d)) + __saturatef(ex2(e));
}

struct Stat {   // max and sum of weights relative to it
  float m = -INFINITY, l = 0.f;
  __device__ __forceinline__ void add(float pm, float pl, float c) {
    const float mx = fmaxf(m, pm);
    if (mx == -INFINITY) return;
    l = fmaf(pl, weight(pm, mx, c), __fmul_rn(l, weight(m, mx, c)));
    m = mx;
  }
};

// CL blocks a cluster, GROUPS rows at a time in a block, ROW threads on each.
template <typename T, int CL, int GROUPS, int ROW>
__global__ void __launch_bounds__(ROW * GROUPS, 1024 / (ROW * GROUPS)) accept_kernel(SampleArgs a) {
  constexpr int N = Vec16<T>::N, UN = (GROUPS == 1 || ROW == 32) && sizeof(T) == 4 ? 8 : 4;
  constexpr int THREADS = ROW * GROUPS, WARPS = THREADS / 32, ROW_WARPS = ROW / 32;
  __shared__ float2 s_warp[AS_ROWS][ROW_WARPS];          // a warp's part of a row
  __shared__ float2 s_part[AS_ROWS][CL];                 // every block's part of a row
  __shared__ float s_m[AS_ROWS], s_inv[AS_ROWS], s_x[AS_ROWS];   // the row's max, 1 / sum, its draft's logit, then probability
  __shared__ unsigned long long s_key[WARPS], s_best[2][CL];   // every block's best, of w and of the second race
  const int b = blockIdx.y, part = blockIdx.x, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int n_draft = live_drafts(a, b);
  const float c = fminf(a.inv_t * LOG2E, 3.4028234e38f);   // finite for the lowest temperatures, so that 0 c is 0
  int mine = 0;   // a lane's draft and its random number
  float u = 1.f;
  if (lane < n_draft) {
    mine = a.draft[(long long)b * a.k + lane];
    u = a.u[(long long)b * a.k + lane];
  }
  const bool bad = __any_sync(0xffffffffu, mine < 0 || mine >= a.V);
  if (n_draft < 0 || bad) {   // uniform over the cluster
    if (part == 0) {
      if (tid == 0) {
        if (bad && a.status) set_status(a.status, ST_BAD_TOKEN);
        a.accepted[b] = 0;
        a.token[b] = -1;
        a.step[b] = 0;
      }
      if (tid < a.k) a.prob[(long long)b * a.k + tid] = 0.f;
    }
    return;
  }
  cluster_arrive_relaxed();   // this block runs; whether the others do is waited for before anything is stored to them
  // rows: target 0 .. n_draft, then draft 0 .. n_draft - 1
  const int n_rows = n_draft + 1 + (a.draft_logits ? n_draft : 0);
  auto row_ptr = [&](int r) {
    return reinterpret_cast<const T*>(r > n_draft ? a.draft_logits + b * a.d_b + (r - n_draft - 1) * a.d_r
                                                  : a.target + b * a.t_b + r * a.t_r);
  };

  if (warp == 0 && lane < n_draft) {
    s_x[lane] = clean(to_f32(row_ptr(lane)[mine]));
    if (a.draft_logits) s_x[n_draft + 1 + lane] = clean(to_f32(row_ptr(n_draft + 1 + lane)[mine]));
  }

  const int rt = tid % ROW;
  for (int r = tid / ROW; r < n_rows; r += GROUPS) {
    const T* x = row_ptr(r);
    // elements before the first 16-byte boundary, whole vectors, rest
    const int head = min(a.V, (int)(((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / sizeof(T)));
    const int nv = (a.V - head) / N, tail = head + nv * N;
    const int v0 = (int)((long long)nv * part / CL), v1 = (int)((long long)nv * (part + 1) / CL);
    const char* xv = reinterpret_cast<const char*>(x + head);
    Stat s;
    for (int i = v0 + rt; i < v1; i += ROW * UN) {
      uint4 v[UN];
      float mx = s.m, l = 0.f;
#pragma unroll
      for (int j = 0; j < UN; ++j)
        if (i + j * ROW < v1) v[j] = ldg_stream(xv + (long long)(i + j * ROW) * 16);
#pragma unroll
      for (int j = 0; j < UN; ++j) {
        if (i + j * ROW >= v1) break;
        mx = fmaxf(mx, Vec16<T>::top(v[j]));
      }
      if (mx == -INFINITY) continue;
      mx = fminf(mx, 3.4028234e38f);
      const uint64_t minus_m = pair(-mx), cc = pair(c);
#pragma unroll
      for (int j = 0; j < UN; ++j) {
        if (i + j * ROW >= v1) break;
        float f[N];
        Vec16<T>::get(v[j], f);
#pragma unroll
        for (int y = 0; y < N; y += 2) l += weight2(f[y], f[y + 1], minus_m, cc);
      }
      s.l = fmaf(s.l, weight(s.m, mx, c), l);
      s.m = mx;
    }
    if (part == 0 && rt < 32) {   // the ragged ends
      if (lane < head) s.add(clean(to_f32(x[lane])), 1.f, c);
      if (tail + lane < a.V) s.add(clean(to_f32(x[tail + lane])), 1.f, c);
    }
    const float m = warp_max(s.m);
    const float l = m == -INFINITY ? 0.f : warp_sum(s.l * weight(s.m, m, c));
    if (lane == 0) s_warp[r][rt >> 5] = make_float2(m, l);
  }
  __syncthreads();
  cluster_wait();
  for (int x = tid; x < n_rows * CL; x += THREADS) {   // this block's part of every row to every block
    const int r = x / CL, to = x - r * CL;
    Stat s;
    for (int w = 0; w < ROW_WARPS; ++w) s.add(s_warp[r][w].x, s_warp[r][w].y, c);
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(dsmem_addr(&s_part[r][part], to)), "f"(s.m), "f"(s.l) : "memory");
  }
  cluster_sync();
  for (int r = warp; r < n_rows; r += WARPS) {
    const float2 x = lane < CL ? s_part[r][lane] : make_float2(-INFINITY, 0.f);
    const float m = warp_max(x.x), l = m == -INFINITY ? 0.f : warp_sum(x.y * weight(x.x, m, c));
    if (lane == 0) {
      const int i = r > n_draft ? r - n_draft - 1 : r;
      s_m[r] = l > 0.f ? m : 0.f;
      s_inv[r] = l > 0.f ? 1.f / l : 0.f;
      if (i < n_draft) s_x[r] = weight(s_x[r], s_m[r], c) * s_inv[r];
    }
  }
  __syncthreads();
  // the first rejection (each warp finds it for itself)
  float px = 0.f, qx = 1.f;
  bool take = false;
  if (lane < n_draft) {
    px = s_x[lane];
    if (a.draft_logits) qx = s_x[n_draft + 1 + lane];
    take = u * qx < px;
  }
  const int n = __ffs(~__ballot_sync(0xffffffffu, take)) - 1;   // n_draft <= 31: lane n_draft never takes
  if (part == 0 && warp == 0 && lane < a.k)
    a.prob[(long long)b * a.k + lane] = lane < n_draft ? (px >= qx ? (px > 0.f ? 1.f : 0.f) : px / qx) : 0.f;

  // the race over this block's share of the vocabulary
  const bool rejected = n < n_draft, minus = rejected && a.draft_logits;
  const T *pr = row_ptr(n), *qr = minus ? row_ptr(n_draft + 1 + n) : pr;
  const int gone = rejected && !a.draft_logits ? __shfl_sync(0xffffffffu, mine, n) : -1;
  const float pm = s_m[n], pi = s_inv[n];
  const float qm = minus ? s_m[n_draft + 1 + n] : 0.f, qi = minus ? s_inv[n_draft + 1 + n] : 0.f;
  const float* e = a.race + b * a.race_b;
  const int j0 = (int)((long long)a.V * part / CL), j1 = (int)((long long)a.V * (part + 1) / CL);
  // Of equal values the lowest index: a thread meets its indices in order.
  auto race = [&](bool residual, int second) {
    float best = 0.f;
    int at = 0;
    constexpr int RU = 8;
    for (int jj = j0 + tid; jj < j1; jj += THREADS * RU) {
      float p[RU], q[RU], ej[RU];
#pragma unroll
      for (int y = 0; y < RU; ++y) {
        const int j = min(jj + y * THREADS, j1 - 1);   // the share's last entry again: never better than itself
        p[y] = to_f32(pr[j]);
        ej[y] = __ldg(e + j);
        q[y] = minus ? to_f32(qr[j]) : -INFINITY;
      }
#pragma unroll
      for (int y = 0; y < RU; ++y) {
        const int j = min(jj + y * THREADS, j1 - 1);
        float w = weight(clean(p[y]), pm, c) * pi;
        if (residual) {
          const float rest = __fsub_rn(w, __fmul_rn(weight(clean(q[y]), qm, c), qi));
          w = j != gone && rest > w * NO_RESIDUAL ? rest : 0.f;
        }
        // A quotient is off by 2 ulp at most: as good as w itself.
        const float v = __fdividef(w, ej[y]);
        if (v > best) best = v, at = j;
      }
    }
    const unsigned long long key = warp_max_u64(best > 0.f ? argmax_key(best, at) : 0ull);
    if (lane == 0) s_key[warp] = key;
    __syncthreads();
    if (warp == 0) {
      const unsigned long long x = warp_max_u64(lane < WARPS ? s_key[lane] : 0ull);
      if (lane < CL) asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(dsmem_addr(&s_best[second][part], lane)), "l"(x) : "memory");
    }
    cluster_sync();
    return warp_max_u64(lane < CL ? s_best[second][lane] : 0ull);
  };
  unsigned long long best = race(rejected, 0);
  if (best == 0 && rejected) best = race(false, 1);   // no residual left (p = q): draw from p; uniform over the cluster
  if (part == 0 && tid == 0) {
    a.accepted[b] = n;
    a.token[b] = best ? (int)argmax_index(best) : -1;
    a.step[b] = best ? n + 1 : 0;
  }
}

template <typename T, int CL, int GROUPS, int ROW>
cudaError_t launch_accept(const SampleArgs& a, int B, cudaStream_t st) {
  constexpr auto kernel = accept_kernel<T, CL, GROUPS, ROW>;
  if constexpr (CL > 8) {   // clusters above 8 are asked for once a device
    static std::atomic<uint64_t> ready{0};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = 1ull << (dev & 63);
    if (!(ready.load(std::memory_order_acquire) & bit)) {
      e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
      if (e != cudaSuccess) return e;
      ready.fetch_or(bit, std::memory_order_release);
    }
  }
  return launch_ex(kernel, dim3(CL, B), dim3(ROW * GROUPS), 0, st, false, CL, a);
}

// Few utterances: wide clusters of large blocks shorten the chain of reads;
// then the largest blocks of which all fit the SMs at once (1024 threads an SM).
// A block's share of a short row keeps a warp busy, not a block: a row a warp.
// Measured, us (wide clusters below 16 utterances, 256 threads a row before): 15
// of 10 drafts, bf16, 33 -> 16; 25 of 6, fp32, 22 -> 19; 38 of 14 over 2217
// tokens, fp32, 33 -> 10.5.
template <typename T>
cudaError_t launch_accept_t(const SampleArgs& a, int B, cudaStream_t st) {
  const int sms = paged_sm_count();
  if (a.V <= 8192) return launch_accept<T, 4, 8, 32>(a, B, st);
  if (B <= 8) return launch_accept<T, 16, 4, 256>(a, B, st);
  if (B * 8 <= sms) return launch_accept<T, 8, 4, 256>(a, B, st);
  if (B * 4 <= sms) return launch_accept<T, 8, 2, 256>(a, B, st);
  return launch_accept<T, 8, 1, 256>(a, B, st);
}

}  // namespace
}  // namespace asrspec

using namespace asrspec;

extern "C" {

int asr_spec_accept_sampled(const asr_sampled_logits* x, const int32_t* draft, const int32_t* lens, const float* u,
                            const float* race, int64_t race_stride, float temperature, int32_t* accepted, int32_t* token,
                            int32_t* step, float* prob, int32_t* status, void* stream) {
  if (!x || !x->target || !race || !accepted || !token || !step) return ASR_E_INVAL;
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
       (uintptr_t)step | (uintptr_t)prob | (uintptr_t)status) % 4)
    return ASR_E_INVAL;
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
  a.k = x->k;
  a.V = x->vocab;
  a.accepted = accepted;
  a.token = token;
  a.step = step;
  a.prob = prob;
  a.status = status;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (x->dtype == 0) e = launch_accept_t<float>(a, x->batch, st);
  else if (x->dtype == 1) e = launch_accept_t<__nv_bfloat16>(a, x->batch, st);
  else e = launch_accept_t<__half>(a, x->batch, st);
  return e == cudaSuccess ? ASR_OK : ASR_E_CUDA;
}

}  // extern "C"
