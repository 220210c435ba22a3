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

#include "paged_items.cuh"

namespace asrspec {
namespace {

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
