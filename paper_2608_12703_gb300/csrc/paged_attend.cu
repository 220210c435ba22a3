// Attention of a block of new rows over a paged K/V cache, with the append of
// the block's K/V.
//
//   o_r = sum_j p_rj v_j,  p_rj = exp(scale q_r k_j - lse_r),  lse_r = log sum_j exp(scale q_r k_j)
//
// over the slots j that row r sees: j <= kv_len + r (causal) or j < kv_len.
// A slot's K and V are read once for a tile of rows, so the operator is bound
// by the bytes of the cache; the layout follows from that:
//   * a warp works alone: no shared memory, no block barrier in the key loop.
//     It keeps a tile of rows (the block's rows times the query heads that
//     share a K/V head) as mma A fragments and streams keys from the pages
//     straight into B fragments, 16 bytes a lane.  The contraction index of
//     q k and the output index of p v may be permuted freely, so the
//     permutations are chosen for the loads: of a key a lane takes d = 32 j +
//     8 c .. + 7 (c = lane mod 4), which are the operand pairs of two k-steps;
//     of a value row it takes d = 8 g .. + 7 (g = lane / 4), one element for
//     each of eight n-tiles, paired with its neighbour key by byte permutes;
//   * K of step i + 1 is requested as soon as the scores of step i are done,
//     V of step i + 1 as soon as its product is: one of the two is always in
//     flight, 8 KB a warp;
//   * equal shares whatever the lengths: the (sequence, head, tile, step) units
//     are dealt in contiguous runs over all resident warps (paged.cuh), and a
//     second kernel joins the items that more than one warp worked on, in key
//     order, so results do not depend on timing;
//   * steps below kv_len are read from the pages; the last ones take the
//     block's own rows from k_new / v_new, which the warp that holds them also
//     writes to the pages (other tiles read them from k_new, never from a page
//     written in the same launch).
// Scores, running maximum and sum, and the output accumulate in fp32.  p is
// rounded to the cache's 16-bit type for the second product (relative error at
// most 2^-8 for bf16 and 2^-11 for fp16 a weight, as that of the rounded
// output); the sum takes p before rounding, so lse is exact to fp32.
#include <type_traits>

#include "kernels.h"
#include "paged.cuh"

namespace asrspec {
namespace {

constexpr int PA_WARPS = 4;



struct AttendArgs {
  PagedView c;
  PagedRows r;
  char* out;     // [B][R][H][D]
  float* lse;    // [B][R][H] or null
  float* ws;     // partial results: 2 per warp, [TR] max, [TR] sum, [TR][D] output
  int max_workers, min_units;
};

// The halves of a pair of 16-bit values that are infinite or NaN, as a mask.
template <typename T>
__device__ __forceinline__ uint32_t nonfinite_halves(uint32_t x) {
  constexpr uint32_t E = std::is_same<T, __half>::value ? 0x7c00u : 0x7f80u;
  return ((x & E) == E ? 0xffffu : 0u) | (((x >> 16) & E) == E ? 0xffff0000u : 0u);
}

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
template <typename T, int D, int MT>
__device__ __forceinline__ void guard_values(const Keys16<T, D>& ks, int step, const int (&lim)[MT][2],
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
  for (int key = step * K::KS; key < min((step + 1) * K::KS, ks.keys); ++key) {
    const int grp = key / PG_GROUP;
    const char* row = ks.fresh && key >= ks.len
                          ? ks.vn + (long long)(key - ks.len) * ks.r.n_r
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
          for (int e = 0; e < 2; ++e)
            if (key < lim[mt][e]) O[mt][d][2 * e + x] += v;
      }
  }
}

template <typename T, int D, int MT, int MINB>
__global__ void __launch_bounds__(PA_WARPS * 32, MINB) attend16_kernel(AttendArgs a) {
  constexpr int KS = Cfg16<D>::KS, NG = KS / PG_GROUP, NC = D / 32, NV = D / 64, TR = 16 * MT;
  const PagedView& c = a.c;
  const PagedRows& r = a.r;
  PlanMem mem;
  const WorkPlan plan = work_plan(c, r, mem, a.max_workers, a.min_units, [&](int len, int rows) {
    const SeqWork s = seq_work<KS, TR>(r, len, rows);
    return (long long)c.kv_heads * s.tiles * s.steps;
  });
  pdl_launch();
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int worker = (threadIdx.x >> 5) * gridDim.x + blockIdx.x;   // few workers spread over the SMs
  if (worker >= plan.workers) return;
  long long u = work_start(plan, worker);
  const long long u_end = work_start(plan, worker + 1);
  const float sc = r.scale * LOG2E;

  while (u < u_end) {
    const int b = work_find(mem.pre, c.batch, u);
    const SeqWork s = seq_work<KS, TR>(r, mem.lens[b].x, mem.lens[b].y);
    const int rem = (int)(u - mem.pre[b]), item = rem / s.steps, s0 = rem - item * s.steps;
    const int n = (int)min((long long)(s.steps - s0), u_end - u);
    const int kvh = item / s.tiles, tile = item - kvh * s.tiles;
    u += n;

    const bool fresh = r.k_new != nullptr, append = fresh && tile == 0;
    const long long new_off = b * r.n_b + kvh * r.n_h;
    Keys16<T, D> ks{c, r, c.table + b * c.table_stride, kvh * c.head_stride, r.k_new + new_off, r.v_new + new_off,
                    s.len, s.keys, g, t, fresh};
    int pid[NG];
    long long off[NG];
    uint4 kf[KS / 8][NC], vf[NG][4][NV];
#pragma unroll
    for (int x = 0; x < NG; ++x) pid[x] = ks.id(s0, x);

    uint32_t qa[MT][NC * 2][4];
    int lim[MT][2];   // keys the fragment's rows see
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int m = tile * TR + mt * 16 + e * 8 + g, row = m / r.group, hq = kvh * r.group + m - row * r.group;
        lim[mt][e] = r.causal ? s.len + row + 1 : s.keys;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
          const uint4 x = row < s.rows ? __ldg(reinterpret_cast<const uint4*>(r.q + b * r.q_b + row * r.q_r +
                                                                              hq * r.q_h + j * 64 + t * 16))
                                       : make_uint4(0, 0, 0, 0);
          qa[mt][2 * j][e] = x.x;
          qa[mt][2 * j][2 + e] = x.y;
          qa[mt][2 * j + 1][e] = x.z;
          qa[mt][2 * j + 1][2 + e] = x.w;
        }
      }
    float O[MT][D / 8][4], m_run[MT][2], l_run[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      m_run[mt][0] = m_run[mt][1] = -INFINITY;
      l_run[mt][0] = l_run[mt][1] = 0.f;
#pragma unroll
      for (int d = 0; d < D / 8; ++d) O[mt][d][0] = O[mt][d][1] = O[mt][d][2] = O[mt][d][3] = 0.f;
    }

    // Step i's products and step i + 1's loads; i = -1 only loads.
#pragma unroll 1
    for (int i = -1; i < n; ++i) {
      const int step = s0 + i;
      const bool full = ks.full(step), more = i + 1 < n;
      float S[MT][KS / 8][4];
      if (i >= 0) {
        if (!full && append) ks.append_k(step, kf);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int kt = 0; kt < KS / 8; ++kt) {
            S[mt][kt][0] = S[mt][kt][1] = S[mt][kt][2] = S[mt][kt][3] = 0.f;
#pragma unroll
            for (int j = 0; j < NC; ++j) {
              Mma16<T>::mma(S[mt][kt], qa[mt][2 * j], kf[kt][j].x, kf[kt][j].y);
              Mma16<T>::mma(S[mt][kt], qa[mt][2 * j + 1], kf[kt][j].z, kf[kt][j].w);
            }
          }
      }
      if (more) {
        ks.offsets(step + 1, pid, off);
        ks.load_k(step + 1, off, kf);
        if (i + 2 < n)
#pragma unroll
          for (int x = 0; x < NG; ++x) pid[x] = ks.id(step + 2, x);
      }
      if (i >= 0) {
        if (!full) {
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int kt = 0; kt < KS / 8; ++kt)
#pragma unroll
              for (int x = 0; x < 4; ++x)
                if (step * KS + kt * 8 + 2 * t + (x & 1) >= min(lim[mt][x >> 1], s.keys)) S[mt][kt][x] = -INFINITY;
        }
        uint32_t pf[MT][KS / 8][2];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          float mx[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float x = fmaxf(S[mt][0][2 * e], S[mt][0][2 * e + 1]);
#pragma unroll
            for (int kt = 1; kt < KS / 8; ++kt) x = fmaxf(x, fmaxf(S[mt][kt][2 * e], S[mt][kt][2 * e + 1]));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
            mx[e] = fmaxf(m_run[mt][e], x * sc);
          }
          if (__any_sync(0xffffffffu, mx[0] > m_run[mt][0] || mx[1] > m_run[mt][1])) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float f = mx[e] == -INFINITY ? 1.f : ex2(m_run[mt][e] - mx[e]);
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
          for (int e = 0; e < 2; ++e) {
            const float m = m_run[mt][e] == -INFINITY ? 0.f : m_run[mt][e];
#pragma unroll
            for (int kt = 0; kt < KS / 8; ++kt) {
              const float p0 = ex2(fmaf(S[mt][kt][2 * e], sc, -m)), p1 = ex2(fmaf(S[mt][kt][2 * e + 1], sc, -m));
              l_run[mt][e] += p0 + p1;
              pf[mt][kt][e] = Mma16<T>::pack(p0, p1);
            }
          }
        }
        if (!full) {
          if (append) ks.append_v(step, vf);
          guard_values<T, D, MT>(ks, step, lim, vf, O);
        }
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
                const uint32_t pa[4] = {pf[mt][2 * x][0], pf[mt][2 * x][1], pf[mt][2 * x + 1][0], pf[mt][2 * x + 1][1]};
                Mma16<T>::mma(O[mt][j * 8 + d], pa, b0, b1);
              }
            }
      }
      if (more) ks.load_v(step + 1, off, vf);
    }

    // the item's result: of row g (+ 8 e) a lane holds columns 64 j + 16 t .. + 15
    const bool whole = n == s.steps;
    float* part = a.ws + (size_t)(2 * worker + (s0 == 0 ? 1 : 0)) * (TR * (D + 2));
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float l = l_run[mt][e];
        l += __shfl_xor_sync(0xffffffffu, l, 1);
        l += __shfl_xor_sync(0xffffffffu, l, 2);
        const int in = mt * 16 + e * 8 + g, m = tile * TR + in, row = m / r.group;
        if (row >= s.rows) continue;
        const int hq = kvh * r.group + m - row * r.group;
        if (whole) {
          const size_t at = ((size_t)b * r.max_rows + row) * r.heads + hq;
          const float inv = l > 0.f ? 1.f / l : 0.f;
          if (a.lse && t == 0) a.lse[at] = (m_run[mt][e] + log2f(l)) * LN2;
          uint32_t* o = reinterpret_cast<uint32_t*>(a.out + at * D * sizeof(T));
#pragma unroll
          for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const float* f[8];
#pragma unroll
              for (int d = 0; d < 8; ++d) f[d] = &O[mt][j * 8 + d][2 * e + x];
              uint4 w;
              w.x = Mma16<T>::pack(*f[0] * inv, *f[1] * inv);
              w.y = Mma16<T>::pack(*f[2] * inv, *f[3] * inv);
              w.z = Mma16<T>::pack(*f[4] * inv, *f[5] * inv);
              w.w = Mma16<T>::pack(*f[6] * inv, *f[7] * inv);
              *reinterpret_cast<uint4*>(o + (j * 64 + t * 16 + x * 8) / 2) = w;
            }
        } else {
          if (t == 0) {
            part[in] = m_run[mt][e];
            part[TR + in] = l;
          }
          float* o = part + 2 * TR + in * D;
#pragma unroll
          for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
              for (int d = 0; d < 8; d += 4)
                *reinterpret_cast<float4*>(o + j * 64 + t * 16 + x * 8 + d) =
                    make_float4(O[mt][j * 8 + d][2 * e + x], O[mt][j * 8 + d + 1][2 * e + x],
                                O[mt][j * 8 + d + 2][2 * e + x], O[mt][j * 8 + d + 3][2 * e + x]);
        }
      }
  }
}

// fp32: plain fp32 products (no TF32), four rows a warp.  Eight lanes share a
// key (lane e of them takes the 16-byte chunks e, e + 8, ..), four keys at a
// time; each group of eight lanes keeps its own running maximum, sum and
// output over its keys, combined at the end of the item.
template <int D>
__global__ void __launch_bounds__(PA_WARPS * 32) attend32_kernel(AttendArgs a) {
  constexpr int TR = 4, KS = D == 64 ? 16 : 8, IT = KS / 4, NC = D / 32;
  const PagedView& c = a.c;
  const PagedRows& r = a.r;
  PlanMem mem;
  const WorkPlan plan = work_plan(c, r, mem, a.max_workers, a.min_units, [&](int len, int rows) {
    const SeqWork s = seq_work<KS, TR>(r, len, rows);
    return (long long)c.kv_heads * s.tiles * s.steps;
  });
  pdl_launch();
  const int lane = threadIdx.x & 31, kg = lane >> 3, e = lane & 7;
  const int worker = (threadIdx.x >> 5) * gridDim.x + blockIdx.x;
  if (worker >= plan.workers) return;
  long long u = work_start(plan, worker);
  const long long u_end = work_start(plan, worker + 1);
  const float sc = r.scale * LOG2E;

  while (u < u_end) {
    const int b = work_find(mem.pre, c.batch, u);
    const SeqWork s = seq_work<KS, TR>(r, mem.lens[b].x, mem.lens[b].y);
    const int rem = (int)(u - mem.pre[b]), item = rem / s.steps, s0 = rem - item * s.steps;
    const int n = (int)min((long long)(s.steps - s0), u_end - u);
    const int kvh = item / s.tiles, tile = item - kvh * s.tiles;
    u += n;
    const int* table_row = c.table + b * c.table_stride;

    float q[TR][NC * 4], O[TR][NC * 4], m_run[TR], l_run[TR];
    int lim[TR];
#pragma unroll
    for (int x = 0; x < TR; ++x) {
      const int m = tile * TR + x, row = m / r.group, hq = kvh * r.group + m - row * r.group;
      lim[x] = row < s.rows ? (r.causal ? s.len + row + 1 : s.keys) : 0;
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
      const int key0 = (s0 + i) * KS;
      const int grp = key0 / PG_GROUP;
      const int pid = paged_id(c, table_row, grp);
      const bool pid_ok = pid != 0 || __ldg(table_row + c.groups.div((uint32_t)grp)) == 0;   // no stand-in
      const long long off =
          paged_offset(c, pid, grp) + kvh * c.head_stride + (long long)(key0 % PG_GROUP + kg) * c.slot_stride + e * 16;
      float4 kf[IT][NC], vf[IT][NC];
#pragma unroll
      for (int k = 0; k < IT; ++k) {
        const int key = key0 + 4 * k + kg;
        const bool fresh = r.k_new != nullptr && key >= s.len, in = key < s.keys;
        const char* kp = c.k + off + (long long)(4 * k) * c.slot_stride;
        const char* vp = c.v + off + (long long)(4 * k) * c.slot_stride;
        const long long no = b * r.n_b + (long long)(key - s.len) * r.n_r + kvh * r.n_h + e * 16;
        const char* ksrc = fresh ? r.k_new + no : kp;
        const char* vsrc = fresh ? r.v_new + no : vp;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
          kf[k][j] = in ? *reinterpret_cast<const float4*>(ksrc + j * 128) : make_float4(0.f, 0.f, 0.f, 0.f);
          vf[k][j] = in ? *reinterpret_cast<const float4*>(vsrc + j * 128) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
      }
      if (r.k_new != nullptr && tile == 0 && pid_ok && key0 + KS > s.len) {   // the step's new rows go to their page
#pragma unroll
        for (int k = 0; k < IT; ++k) {
          const int key = key0 + 4 * k + kg;
          if (key < s.len || key >= s.keys) continue;
#pragma unroll
          for (int j = 0; j < NC; ++j) {
            *reinterpret_cast<float4*>(c.k + off + (long long)(4 * k) * c.slot_stride + j * 128) = kf[k][j];
            *reinterpret_cast<float4*>(c.v + off + (long long)(4 * k) * c.slot_stride + j * 128) = vf[k][j];
          }
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
          S[k] = key0 + 4 * k + kg < min(lim[x], s.keys) ? d : -INFINITY;
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
          if (key0 + 4 * k + kg >= lim[x]) continue;   // hidden: an infinity or NaN there must not reach the row
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
    const bool whole = n == s.steps;
    float* part = a.ws + (size_t)(2 * worker + (s0 == 0 ? 1 : 0)) * (TR * (D + 2));
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
      const int m = tile * TR + x, row = m / r.group;
      if (row >= s.rows || kg != 0) continue;
      if (whole) {
        const size_t at = ((size_t)b * r.max_rows + row) * r.heads + kvh * r.group + m - row * r.group;
        const float inv = l > 0.f ? 1.f / l : 0.f;
        if (a.lse && e == 0) a.lse[at] = (mx + log2f(l)) * LN2;
        float4* o = reinterpret_cast<float4*>(a.out + at * D * sizeof(float));
#pragma unroll
        for (int j = 0; j < NC; ++j)
          o[e + 8 * j] = make_float4(O[x][4 * j] * inv, O[x][4 * j + 1] * inv, O[x][4 * j + 2] * inv, O[x][4 * j + 3] * inv);
      } else {
        if (e == 0) {
          part[x] = mx;
          part[TR + x] = l;
        }
        float4* o = reinterpret_cast<float4*>(part + 2 * TR + x * D);
#pragma unroll
        for (int j = 0; j < NC; ++j) o[e + 8 * j] = make_float4(O[x][4 * j], O[x][4 * j + 1], O[x][4 * j + 2], O[x][4 * j + 3]);
      }
    }
  }
}

// Joins the items that several warps worked on, in key order, and fills the
// rows that have no keys.  WPT warps share one (sequence, row, head): many
// partials and few rows with one long sequence, the reverse in a batch.
constexpr int PJ_WARPS = 8;

template <typename T, int D, int KS, int TR, int WPT>
__global__ void __launch_bounds__(PJ_WARPS * 32) join_kernel(AttendArgs a) {
  constexpr int LP = D / 4;            // lanes that hold one output row, 4 columns each
  constexpr int PP = 32 / LP * WPT;    // partials at a time
  __shared__ float s_m[PJ_WARPS], s_l[PJ_WARPS], s_o[PJ_WARPS][D];
  const PagedView& c = a.c;
  const PagedRows& r = a.r;
  PlanMem mem;
  const WorkPlan plan = work_plan(c, r, mem, a.max_workers, a.min_units, [&](int len, int rows) {
    const SeqWork s = seq_work<KS, TR>(r, len, rows);
    return (long long)c.kv_heads * s.tiles * s.steps;
  });
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const long long tasks = (long long)c.batch * r.max_rows * r.heads;
  const long long task = (long long)blockIdx.x * (PJ_WARPS / WPT) + warp / WPT;
  const bool live = task < tasks;
  pdl_wait();
  int wf = 0, wl = 0, in = 0;
  long long at = task;
  if (live) {
    const int hq = (int)(task % r.heads), row = (int)(task / r.heads % r.max_rows), b = (int)(task / r.heads / r.max_rows);
    const SeqWork s = seq_work<KS, TR>(r, mem.lens[b].x, mem.lens[b].y);
    if (row >= s.rows || s.keys == 0) {
      if (warp % WPT == 0) {
        if (a.lse && lane == 0) a.lse[at] = -INFINITY;
        T* o = reinterpret_cast<T*>(a.out) + at * D;
        for (int d = lane; d < D; d += 32) o[d] = T(0.f);
      }
    } else {
      const int kvh = hq / r.group, m = row * r.group + hq - kvh * r.group, tile = m / TR;
      in = m - tile * TR;
      const long long u0 = mem.pre[b] + (long long)(kvh * s.tiles + tile) * s.steps;
      wf = work_owner(plan, u0);
      wl = work_owner(plan, u0 + s.steps - 1);
    }
  }
  const bool join = live && wl > wf;
  if (WPT == 1 && !join) return;
  const int sub = lane / LP, col = (lane % LP) * 4;
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  if (join) {
#pragma unroll 4
    for (int w = wf + (warp % WPT) * (32 / LP) + sub; w <= wl; w += PP) {
      const float* part = a.ws + (size_t)(2 * w + (w == wf ? 1 : 0)) * (TR * (D + 2));
      const float pm = part[in], pl = part[TR + in];
      const float4 po = *reinterpret_cast<const float4*>(part + 2 * TR + in * D + col);
      const float mx = fmaxf(m, pm), z = mx == -INFINITY ? 0.f : mx, f0 = ex2(m - z), f1 = ex2(pm - z);
      m = mx;
      l = l * f0 + pl * f1;
      o.x = o.x * f0 + po.x * f1;
      o.y = o.y * f0 + po.y * f1;
      o.z = o.z * f0 + po.z * f1;
      o.w = o.w * f0 + po.w * f1;
    }
    if (LP < 32) {
      const float pm = __shfl_xor_sync(0xffffffffu, m, 16), pl = __shfl_xor_sync(0xffffffffu, l, 16);
      const float px = __shfl_xor_sync(0xffffffffu, o.x, 16), py = __shfl_xor_sync(0xffffffffu, o.y, 16);
      const float pz = __shfl_xor_sync(0xffffffffu, o.z, 16), pw = __shfl_xor_sync(0xffffffffu, o.w, 16);
      const float mx = fmaxf(m, pm), z = mx == -INFINITY ? 0.f : mx, f0 = ex2(m - z), f1 = ex2(pm - z);
      m = mx;
      l = l * f0 + pl * f1;
      o = make_float4(o.x * f0 + px * f1, o.y * f0 + py * f1, o.z * f0 + pz * f1, o.w * f0 + pw * f1);
    }
  }
  if (WPT > 1) {
    if (join && sub == 0) {
      if (lane == 0) {
        s_m[warp] = m;
        s_l[warp] = l;
      }
      *reinterpret_cast<float4*>(&s_o[warp][col]) = o;
    }
    __syncthreads();
    if (!join || warp % WPT != 0 || sub != 0) return;
    m = -INFINITY;
#pragma unroll
    for (int w = 0; w < WPT; ++w) m = fmaxf(m, s_m[warp + w]);
    l = 0.f;
    o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < WPT; ++w) {
      const float f = m == -INFINITY ? 0.f : ex2(s_m[warp + w] - m);
      const float4 po = *reinterpret_cast<const float4*>(&s_o[warp + w][col]);
      l += s_l[warp + w] * f;
      o = make_float4(o.x + po.x * f, o.y + po.y * f, o.z + po.z * f, o.w + po.w * f);
    }
  }
  if (sub != 0) return;
  const float inv = l > 0.f ? 1.f / l : 0.f;
  if (a.lse && lane == 0) a.lse[at] = (m + log2f(l)) * LN2;
  T* out = reinterpret_cast<T*>(a.out) + at * D + col;
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4*>(out) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
  } else {
    *reinterpret_cast<uint2*>(out) = make_uint2(Mma16<T>::pack(o.x * inv, o.y * inv), Mma16<T>::pack(o.z * inv, o.w * inv));
  }
}

struct Shape {   // of one call's kernels
  int tr, blocks_per_sm;
};
Shape attend_shape(int dtype, int dim, int m_rows) {
  if (dtype == 0) return {4, 2};
  if (dim == 128) return {16, 2};
  return m_rows > 16 ? Shape{32, 2} : Shape{16, 3};
}

template <typename T, int D, int KS, int TR>
cudaError_t launch_join(const AttendArgs& a, size_t smem, cudaStream_t st) {
  const long long tasks = (long long)a.c.batch * a.r.max_rows * a.r.heads;
  // Whole blocks join one row each while the rows alone do not fill the SMs.
  if (tasks < 152 * 2)
    return launch_ex(join_kernel<T, D, KS, TR, PJ_WARPS>, dim3((unsigned)tasks), dim3(PJ_WARPS * 32), smem, st, true, 1, a);
  return launch_ex(join_kernel<T, D, KS, TR, 1>, dim3((unsigned)((tasks + PJ_WARPS - 1) / PJ_WARPS)), dim3(PJ_WARPS * 32),
                   smem, st, true, 1, a);
}

template <typename T, int D, int MT, int MINB>
cudaError_t launch16(const AttendArgs& a, int grid, size_t smem, cudaStream_t st) {
  cudaError_t e = launch_ex(attend16_kernel<T, D, MT, MINB>, dim3(grid), dim3(PA_WARPS * 32), smem, st, false, 1, a);
  if (e != cudaSuccess) return e;
  return launch_join<T, D, Cfg16<D>::KS, 16 * MT>(a, smem, st);
}
template <int D>
cudaError_t launch32(const AttendArgs& a, int grid, size_t smem, cudaStream_t st) {
  cudaError_t e = launch_ex(attend32_kernel<D>, dim3(grid), dim3(PA_WARPS * 32), smem, st, false, 1, a);
  if (e != cudaSuccess) return e;
  return launch_join<float, D, D == 64 ? 16 : 8, 4>(a, smem, st);
}
template <typename T>
cudaError_t launch16_dim(const AttendArgs& a, int dim, int tr, int grid, size_t smem, cudaStream_t st) {
  if (dim == 128) return launch16<T, 128, 1, 2>(a, grid, smem, st);
  return tr == 32 ? launch16<T, 64, 2, 2>(a, grid, smem, st) : launch16<T, 64, 1, 3>(a, grid, smem, st);
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
  const Shape s = attend_shape(c->dtype, c->head_dim, w.max_rows * w.group);
  return (int64_t)paged_sm_count() * s.blocks_per_sm * PA_WARPS * 2 * s.tr * (c->head_dim + 2) * 4;
}

int asr_spec_paged_attend(const asr_paged_cache* c, const asr_paged_rows* r, void* out, float* lse, void* ws,
                          int64_t ws_bytes, void* stream) {
  AttendArgs a{};
  if (int rc = paged_view(c, &a.c)) return rc;
  if (int rc = paged_rows(c, r, &a.r)) return rc;
  if (!out || !ws || ((uintptr_t)out | (uintptr_t)ws) % 16 || (uintptr_t)lse % 4) return ASR_E_INVAL;
  const Shape s = attend_shape(c->dtype, c->head_dim, a.r.max_rows * a.r.group);
  const int grid = paged_sm_count() * s.blocks_per_sm;
  if (ws_bytes < (int64_t)grid * PA_WARPS * 2 * s.tr * (c->head_dim + 2) * 4) return ASR_E_CAPACITY;
  const long long tiles = ((long long)a.r.max_rows * a.r.group + s.tr - 1) / s.tr;
  if (tiles * c->kv_heads * ((long long)a.c.max_slots / 8 + 1) > 0x7fffffffll) return ASR_E_CAPACITY;   // 32-bit units a sequence
  if ((long long)c->batch * a.r.max_rows * a.r.heads > 0x7fffffffll) return ASR_E_CAPACITY;
  a.out = static_cast<char*>(out);
  a.lse = lse;
  a.ws = static_cast<float*>(ws);
  a.max_workers = grid * PA_WARPS;
  a.min_units = 1;
  const size_t smem = plan_bytes(c->batch);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (c->dtype == 0) e = c->head_dim == 64 ? launch32<64>(a, grid, smem, st) : launch32<128>(a, grid, smem, st);
  else if (c->dtype == 1) e = launch16_dim<__nv_bfloat16>(a, c->head_dim, s.tr, grid, smem, st);
  else e = launch16_dim<__half>(a, c->head_dim, s.tr, grid, smem, st);
  return e == cudaSuccess ? ASR_OK : ASR_E_CUDA;
}

}  // extern "C"
