// Attention of a block of rows over an 8-bit paged cache.
//
//   o_r = sum_j p_rj s_j v_j / l_r,  p_rj = exp(scale (q_r k_j) t_j - m_r),  l_r = sum_j p_rj
//
// with k_j, v_j the codes of slot j and t_j, s_j the scales of its group.  The
// work is dealt as over a 16-bit cache (paged_items.cuh): a warp keeps a tile
// of rows and walks steps of keys, 8 KB of K and V, that bulk copies bring to a
// ring of its own.  What differs:
//   * codes become fp16 on the way to the tensor cores, two an instruction and
//     exactly.  q is taken to fp16 too: fp16 rows as they are; bf16 rows by a power of two
//     that brings their largest element to [2^14, 2^15), which keeps all 8 bits of
//     elements down to 2^-31 of it (at most 2^100: below 2^-117 they lose bits);
//   * keys are the first index of both products (S^T = K q^T, O^T = V^T p^T), so
//     that 16 of them meet 8 rows in an instruction and no half of a tile is left
//     empty by blocks of up to 8 rows, which are most.  p^T changes
//     places between the products by movmatrix;
//   * a group of 16 slots is one tile of the first product and one k-step of
//     the second, so its scales are one factor of S^T and one of p.  p s_j is
//     rounded to fp16 relative to the row's largest so far (not p's: a group of
//     small scale and large weight would vanish beside one of large scale), the
//     reference a power of two, so that moving it is exact.
// New rows are appended by a kernel before, whose end this one's plan and q do
// not wait for (programmatic launch).  An append by the warps themselves took
// one launch less and longer everywhere: its chain of rows, scale, codes and
// copies lies before a warp's last steps (64 sequences 28 -> 33 us, one token 11 -> 13 us).
// Measured, device time with the append: 48 sequences of up to 80000 slots, 32
// query heads on 8 of 128, fp16: 624 us for 3.96 GB, 6.3 TB/s (of 6.75 copied);
// 64 of up to 448 slots, 7 rows, 20 heads of 64, bf16: 28 us for 41 MB, 3 of
// them the plan, 2 q and the first copies, 8 steps of 64 keys of 1.5 us in the
// longest warp, 2 the end; one of 230 slots, one row: 11 us, all of it latency.
// The conversion costs nothing that shows (codes taken as they are: 624 and 28
// us; converted by masks and shifts: 899 and 35), and neither scores a step ahead of
// the weights nor steps of 32 keys shorten the short case (31 and 32 us).
#include <atomic>

#include "paged8.cuh"
#include "paged_items.cuh"

namespace asrspec {
namespace {

struct Attend8Args : AttendArgs {
  Paged8View p;
};

__device__ __forceinline__ uint32_t transposed(uint32_t x) {   // of an 8 x 8 matrix of 16-bit values
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

template <int N> struct Bytes { uint32_t w[N / 4]; };
template <int N> __device__ __forceinline__ Bytes<N> lds_bytes(uint32_t at) {
  Bytes<N> v;
  if constexpr (N == 8) {
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.w[0]), "=r"(v.w[1]) : "r"(at) : "memory");
  } else {
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.w[0]), "=r"(v.w[1]), "=r"(v.w[2]), "=r"(v.w[3]) : "r"(at) : "memory");
  }
  return v;
}
template <int D> struct Cfg8 { static constexpr int KS = 4096 / D, NG = KS / PG_GROUP; };   // keys and groups of a step

// Where a run of steps lies: of every 32 groups a lane looks up one, page ids a
// round ahead of their use, scales as soon as the page is known.  Copies run
// ahead of the products, so the scales of the round before are kept.
template <int D>
struct Groups8 {
  static constexpr int NG = Cfg8<D>::NG, STEPS = 32 / NG;
  const Paged8View& p;
  const int* table_row;
  int kvh, grp0, groups, next_pid, round;
  long long off;
  float ks[2], vs[2];   // this round's, the one's before
  __device__ __forceinline__ int page(int r) const {
    const int grp = grp0 + r * 32 + (threadIdx.x & 31);
    return grp < groups ? __ldg(table_row + p.c.groups.div((uint32_t)grp)) : 0;   // looked at when used
  }
  __device__ __forceinline__ Groups8(const Paged8View& view, int b, int head, int keys, int s0)
      : p(view), table_row(view.c.table + b * view.c.table_stride), kvh(head), grp0(s0 * NG),
        groups((keys + PG_GROUP - 1) / PG_GROUP), next_pid(0), round(-1), off(0), ks{1.f, 1.f}, vs{1.f, 1.f} {
    next_pid = page(0);
  }
  // step i of the run: its first lane; `off` is this round's from here on
  __device__ __forceinline__ int at(int i) {
    if (i % STEPS == 0) {
      round = i / STEPS;
      const int grp = grp0 + round * 32 + (threadIdx.x & 31), pid = paged_valid(p.c, next_pid);
      off = paged_offset(p.c, pid, grp) + kvh * p.c.head_stride;
      ks[1] = ks[0], vs[1] = vs[0];
      if (grp < groups) {
        const long long at = p.scale_at(pid, kvh, grp);
        ks[0] = p.k_scale[at], vs[0] = p.v_scale[at];   // written by the append before
      } else {
        ks[0] = vs[0] = 1.f;
      }
      next_pid = page(round + 1);
    }
    return i % STEPS * NG;
  }
  __device__ __forceinline__ void scales(int i, float (&k)[NG], float (&v)[NG]) const {
    const bool now = i / STEPS == round;
    const float mk = now ? ks[0] : ks[1], mv = now ? vs[0] : vs[1];
#pragma unroll
    for (int u = 0; u < NG; ++u) {
      k[u] = __shfl_sync(0xffffffffu, mk, i % STEPS * NG + u);
      v[u] = __shfl_sync(0xffffffffu, mv, i % STEPS * NG + u);
    }
  }
};

// A step's codes of K (or V) into shared memory, rows of D in slot order,
// counted on `bar`; nothing is written past the end.  Lane at + u has the
// offset of the step's group u.  One copy where the step lies in one page and a
// head's slots are contiguous, a copy a group where the latter alone, else one a row.
template <int D>
__device__ __forceinline__ void fetch8(const PagedView& c, int step, int keys, const char* pages, long long off, int at, uint32_t dst,
                                       uint64_t* bar) {
  constexpr int KS = Cfg8<D>::KS, NG = Cfg8<D>::NG, GROUP_BYTES = PG_GROUP * D;
  const int lane = threadIdx.x & 31, rows = min(KS, keys - step * KS);
  if (c.slot_stride == D) {
    if (rows == KS && (int)c.groups.d % NG == 0) {   // a run's steps begin at multiples of NG groups
      if (lane == at) {
        mbar_arrive_expect_tx(bar, KS * D);
        bulk_copy(dst, pages + off, KS * D, bar);
      }
      return;
    }
    if (lane == at) mbar_arrive_expect_tx(bar, rows * D);
    __syncwarp();
    const int n = min(PG_GROUP, rows - (lane - at) * PG_GROUP);
    if ((unsigned)(lane - at) < NG && n > 0) bulk_copy(dst + (lane - at) * GROUP_BYTES, pages + off, n * D, bar);
    return;
  }
  if (lane == at) mbar_arrive_expect_tx(bar, rows * D);
  __syncwarp();
#pragma unroll
  for (int r0 = 0; r0 < KS; r0 += 32) {
    const int row = r0 + lane;
    const long long base = __shfl_sync(0xffffffffu, off, at + row / PG_GROUP);
    if (row < rows) bulk_copy(dst + row * D, pages + base + (row % PG_GROUP) * c.slot_stride, D, bar);
  }
}

// NT tiles of 8 rows.
template <typename T, typename C, int NT>
__global__ void __launch_bounds__(C::WARPS * 32, 1) attend8_kernel(const Attend8Args a) {
  constexpr int D = C::D, KS = Cfg8<D>::KS, NG = Cfg8<D>::NG, NJ = D / 64, MT = D / 16, VB = D / 8, TR = C::TR, STAGES = C::STAGES;
  static_assert(TR == 8 * NT && KS * D * 2 == 8192, "");
  const PagedView& c = a.c;
  const PagedRows& r = a.r;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  constexpr float TOP = 32768.f, MOST = 8.507059173e37f;   // the largest weight; 2^126
  __shared__ __align__(8) uint64_t bars[C::WARPS][STAGES][2];
  uint64_t(*bar)[2] = bars[threadIdx.x >> 5];
  if (lane < 2 * STAGES) mbar_init(&bar[lane >> 1][lane & 1], 1);
  fence_mbar_init();
  __syncwarp();
  uint32_t phases = 0;   // a bit a stage
  bool gave_up = false;

  attend_items<T, C, KS>(a, [&](const SeqWork& s, int b, int kvh, int tile, int s0, int n, float* sm) {
    constexpr int KB = KS * D;   // bytes of a step's K, and of its V
    const uint32_t ring = smem_u32(sm);
    // q, on its way before the pages are looked up and while the append still runs
    uint4 xq[NT][NJ][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int m = tile * TR + nt * 8 + g, row = (int)r.groups.div(m), hq = kvh * r.group + m - row * r.group;
      const char* src = r.q + b * r.q_b + row * r.q_r + hq * r.q_h + t * 32;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        xq[nt][j][0] = ldg_if(row < s.rows, src + j * 128);
        xq[nt][j][1] = ldg_if(row < s.rows, src + j * 128 + 16);
      }
    }
    pdl_wait();   // the append
    Groups8<D> groups(a.p, b, kvh, s.keys, s0);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // results were written here before
    __syncwarp();
#pragma unroll
    for (int i = 0; i < STAGES; ++i) {
      if (i < n) {
        const int at = groups.at(i);
        fetch8<D>(c, s0 + i, s.keys, c.k, groups.off, at, ring + i * 2 * KB, &bar[i][0]);
        fetch8<D>(c, s0 + i, s.keys, c.v, groups.off, at, ring + i * 2 * KB + KB, &bar[i][1]);
      }
    }

    // q as B fragments: of row g a lane takes d = 64 j + 16 t .. + 15, two registers a k-step
    uint32_t qb[NT][NJ][4][2];
    float sc[NT][2];      // of rows 2 t, 2 t + 1: the scale, in powers of two
    int lim[NT][2];       // slots that they see
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      uint4 (&x)[NJ][2] = xq[nt];
      int e = 0;
      if constexpr (sizeof(T) == 2 && !std::is_same<T, __half>::value) {
        uint32_t most = 0;   // the largest magnitude's bits
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t w = reg_of(x[j][h], i);
              most = max(most, max(w & 0x7fffu, w >> 16 & 0x7fffu));
            }
        most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
        // to [2^14, 2^15); infinities and NaN stay what they are here
        e = min(100, 14 - ((int)(most >> 7) - 127));
        const float f0 = pow2(e / 2), f1 = pow2(e - e / 2);
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t w = reg_of(x[j][h], i);
              y[i] = Mma16<__half>::pack(__int_as_float(w << 16) * f0 * f1, __int_as_float(w & 0xffff0000u) * f0 * f1);
            }
            x[j][h] = make_uint4(y[0], y[1], y[2], y[3]);
          }
      }
#pragma unroll
      for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          qb[nt][j][i][0] = nan_for_inf(reg_of(x[j][i / 2], i % 2 * 2));
          qb[nt][j][i][1] = nan_for_inf(reg_of(x[j][i / 2], i % 2 * 2 + 1));
        }
#pragma unroll
      for (int x2 = 0; x2 < 2; ++x2) {
        const int m2 = tile * TR + nt * 8 + 2 * t + x2, row2 = (int)r.groups.div(m2);
        lim[nt][x2] = min(s.keys, r.causal ? s.len + row2 + 1 : s.len);
        const int e2 = __shfl_sync(0xffffffffu, e, 8 * t + 4 * x2);
        sc[nt][x2] = fmaxf(r.scale * LOG2E * pow2(-(e2 / 2)) * pow2(-(e2 - e2 / 2)), 1.17549435e-38f);
      }
    }
    float O[NT][MT][4], m_run[NT][2], l_run[NT][2];
    // Weights of the second product: p s_j / ref <= 1.  `ref` is 2^d with the exact inverse 2^-d, first the smallest.
    float inv[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int x = 0; x < 2; ++x) m_run[nt][x] = -INFINITY, l_run[nt][x] = 0.f, inv[nt][x] = MOST;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) O[nt][mt][0] = O[nt][mt][1] = O[nt][mt][2] = O[nt][mt][3] = 0.f;
    }

    int stage = 0;
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
      const int step = s0 + i;
      const bool full = (step + 1) * KS <= min(s.len, s.keys), more = i + STAGES < n;
      const uint32_t slot = ring + stage * 2 * KB, parity = phases >> stage & 1;
      uint64_t* landed = bar[stage];
      phases ^= 1u << stage;
      stage = stage + 1 == STAGES ? 0 : stage + 1;
      float ks[NG], vs[NG];
      groups.scales(i, ks, vs);
      float S[NT][NG][4];
      bar_wait(&landed[0], parity, c.status, gave_up);
#pragma unroll
      for (int u = 0; u < NG; ++u) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) S[nt][u][0] = S[nt][u][1] = S[nt][u][2] = S[nt][u][3] = 0.f;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const uint32_t at = slot + (u * PG_GROUP + g) * D + j * 64 + t * 16;
          const uint4 k0 = lds16(at), k1 = lds16(at + 8 * D);
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const uint32_t w0 = reg_of(k0, x), w1 = reg_of(k1, x);
            const uint32_t ka[4] = {half2_of(w0), half2_of(w1), half2_of(w0 >> 16), half2_of(w1 >> 16)};
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) Mma16<__half>::mma(S[nt][u], ka, qb[nt][j][x][0], qb[nt][j][x][1]);
          }
        }
      }
      __syncwarp();   // all lanes have read the slot
      int at = 0;
      if (more) {
        at = groups.at(i + STAGES);
        fetch8<D>(c, step + STAGES, s.keys, c.k, groups.off, at, slot, &landed[0]);
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int u = 0; u < NG; ++u)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            S[nt][u][x] *= ks[u];
            if (!full && step * KS + u * PG_GROUP + g + (x >> 1) * 8 >= lim[nt][x & 1]) S[nt][u][x] = -INFINITY;
          }
      uint32_t pb[NT][NG][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float mx[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          mx[x] = fmaxf(S[nt][0][x], S[nt][0][x + 2]);
#pragma unroll
          for (int u = 1; u < NG; ++u) mx[x] = fmaxf(mx[x], fmaxf(S[nt][u][x], S[nt][u][x + 2]));
          mx[x] = fmaxf(mx[x], __shfl_xor_sync(0xffffffffu, mx[x], 4));
          mx[x] = fmaxf(mx[x], __shfl_xor_sync(0xffffffffu, mx[x], 8));
          mx[x] = fmaxf(mx[x], __shfl_xor_sync(0xffffffffu, mx[x], 16));
          mx[x] = fmaxf(mx[x], m_run[nt][x]);
        }
        if (__any_sync(0xffffffffu, mx[0] > m_run[nt][0] || mx[1] > m_run[nt][1])) {
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            // what was weighed before shrinks with the new maximum, and the reference with it, by whole powers of two; the
            // rest of the factor goes to the output
            if (mx[x] == m_run[nt][x]) continue;
            const float grown = m_run[nt][x] == -INFINITY ? 0.f : (mx[x] - m_run[nt][x]) * sc[nt][x];
            const int k = min((int)fminf(grown, 1000.f), 253 - (__float_as_int(inv[nt][x]) >> 23));   // inv stays <= 2^126
            const float f = ex2((float)k - grown);
            m_run[nt][x] = mx[x];
            l_run[nt][x] *= ex2(-grown);
            inv[nt][x] = __int_as_float(__float_as_int(inv[nt][x]) + (k << 23));
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) O[nt][mt][x] *= f, O[nt][mt][x + 2] *= f;
          }
        }
        float p[NG][4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const float m = m_run[nt][x & 1] == -INFINITY ? 0.f : m_run[nt][x & 1];
#pragma unroll
          for (int u = 0; u < NG; ++u) {
            p[u][x] = ex2((S[nt][u][x] - m) * sc[nt][x & 1]);
            l_run[nt][x & 1] += p[u][x];
          }
        }
        // One pass but at a first tile or a much larger scale, four at most; the bound is for scales that are infinite.
        for (int pass = 0;; ++pass) {
          float big[2] = {0.f, 0.f};
#pragma unroll
          for (int u = 0; u < NG; ++u) {
            float w[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const float f = vs[u] * inv[nt][x & 1];
              w[x] = p[u][x] * (f > MOST ? MOST : f);   // a scale that is no number shows
              big[x & 1] = fmaxf(big[x & 1], w[x]);
            }
            pb[nt][u][0] = Mma16<__half>::pack(w[0], w[1]);
            pb[nt][u][1] = Mma16<__half>::pack(w[2], w[3]);
          }
          if (!__any_sync(0xffffffffu, big[0] > TOP || big[1] > TOP) || pass == 4) break;
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            big[x] = fmaxf(big[x], __shfl_xor_sync(0xffffffffu, big[x], 4));
            big[x] = fmaxf(big[x], __shfl_xor_sync(0xffffffffu, big[x], 8));
            big[x] = fmaxf(big[x], __shfl_xor_sync(0xffffffffu, big[x], 16));
            if (big[x] <= TOP) continue;
            // 2^-k with big 2^-k in [TOP / 2, TOP]
            const float f = pow2(max(-126, 141 - (__float_as_int(big[x]) >> 23)));
            inv[nt][x] *= f;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) O[nt][mt][x] *= f, O[nt][mt][x + 2] *= f;
          }
        }
#pragma unroll
        for (int u = 0; u < NG; ++u) pb[nt][u][0] = transposed(pb[nt][u][0]), pb[nt][u][1] = transposed(pb[nt][u][1]);
      }
      bar_wait(&landed[1], parity, c.status, gave_up);
#pragma unroll
      for (int u = 0; u < NG; ++u) {
        const uint32_t vat = slot + KB + (u * PG_GROUP + 2 * t) * D + g * VB;
        Bytes<VB> v[4];   // keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const int in = (w & 1) + (w >> 1) * 8;
          v[w] = lds_bytes<VB>(vat + in * D);
          if (!full && step * KS + u * PG_GROUP + 2 * t + in >= s.keys)   // past the end: whatever the slot held
#pragma unroll
            for (int x = 0; x < VB / 4; ++x) v[w].w[x] = 0;
        }
        if (!full && s.keys > s.len) {
          // A key of this step may be hidden from some of the rows: a NaN of its value would reach them by a product with
          // weight 0.  Such codes are taken out, and NaN is added to the rows that do see them.
          uint32_t bad = 0;
#pragma unroll
          for (int w = 0; w < 4; ++w)
#pragma unroll
            for (int x = 0; x < VB / 4; ++x) bad |= nan_codes(v[w].w[x]);
          if (__any_sync(0xffffffffu, bad != 0)) {
            // rows that see the first `seen` keys: of a lane's column d the first NaN key of its four, then of the four lanes
#pragma unroll
            for (int x = 0; x < VB; ++x) {
              int first = 0x7fffffff;
#pragma unroll
              for (int w = 3; w >= 0; --w)
                if (nan_codes(v[w].w[x / 4]) >> (x % 4 * 8) & 1) first = step * KS + u * PG_GROUP + 2 * t + (w & 1) + (w >> 1) * 8;
              first = min(first, __shfl_xor_sync(0xffffffffu, first, 1));
              first = min(first, __shfl_xor_sync(0xffffffffu, first, 2));
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int y = 0; y < 2; ++y)
                  if (first < lim[nt][y]) O[nt][x / 2][(x & 1) * 2 + y] = __int_as_float(0x7fffffff);
            }
#pragma unroll
            for (int w = 0; w < 4; ++w)
#pragma unroll
              for (int x = 0; x < VB / 4; ++x) v[w].w[x] &= ~nan_codes(v[w].w[x]);
          }
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {   // of d rows g * VB + 2 mt, + 1
          const uint32_t sel = mt & 1 ? 0x7362 : 0x5140;
          const uint32_t lo = __byte_perm(v[0].w[mt / 2], v[1].w[mt / 2], sel), hi = __byte_perm(v[2].w[mt / 2], v[3].w[mt / 2], sel);
          const uint32_t va[4] = {half2_of(lo), half2_of(lo >> 16), half2_of(hi), half2_of(hi >> 16)};
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) Mma16<__half>::mma(O[nt][mt], va, pb[nt][u][0], pb[nt][u][1]);
        }
      }
      __syncwarp();
      if (more) fetch8<D>(c, step + STAGES, s.keys, c.v, groups.off, at, slot + KB, &landed[1]);
    }

    // of rows 2 t, 2 t + 1 (+ 8 nt) a lane holds columns g * VB .. + VB - 1
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float l = l_run[nt][x];
        l += __shfl_xor_sync(0xffffffffu, l, 4);
        l += __shfl_xor_sync(0xffffffffu, l, 8);
        l += __shfl_xor_sync(0xffffffffu, l, 16);
        const int in = nt * 8 + 2 * t + x;
        if (g == 0) {
          sm[in] = m_run[nt][x] * sc[nt][x];
          sm[TR + in] = l;
        }
        // inv is a power of two from 2^-126 to 2^126; where it is still the first one nothing has a weight
        const float f = __fdividef(1.f, inv[nt][x]);
        float* o = sm + 2 * TR + in * D + g * VB;
#pragma unroll
        for (int mt = 0; mt < MT; mt += 2)
          *reinterpret_cast<float4*>(o + 2 * mt) = make_float4(O[nt][mt][x] * f, O[nt][mt][x + 2] * f, O[nt][mt + 1][x] * f, O[nt][mt + 1][x + 2] * f);
      }
  });
  pdl_wait();   // blocks without work too end after the append
}

// Rows up to 8, 16 and 32 a tile, as over a 16-bit cache.
using S64x8 = Shape<64, 8, 12, 2>;
using S64x16 = Shape<64, 16, 12, 2>;
using S64x32 = Shape<64, 32, 8, 3>;
using S128x8 = Shape<128, 8, 8, 3>;
using S128x16 = Shape<128, 16, 8, 3>;

template <typename F>
auto with_shape(int dim, int m_rows, F f) {
  if (dim == 128) return m_rows <= 8 ? f(S128x8{}) : f(S128x16{});
  return m_rows <= 8 ? f(S64x8{}) : m_rows <= 16 ? f(S64x16{}) : f(S64x32{});
}

int64_t attend8_ws_bytes(int dim, int m_rows) {
  return with_shape(dim, m_rows, [](auto s) {
    return (int64_t)MAX_WORKERS * 4 + (int64_t)attend_grid() * s.WARPS * 2 * s.PART * 4;
  });
}

// One block an SM.  The shared memory above 48 KB that a kernel needs is asked for once a device.
template <typename T, typename C>
cudaError_t launch_attend8(Attend8Args& a, bool appended, cudaStream_t st) {
  constexpr auto kernel = attend8_kernel<T, C, C::TR / 8>;
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
  return launch_ex(kernel, dim3(grid), dim3(C::WARPS * 32), REGIONS + plan_bytes(a.c.batch) + deal_bytes(a.c.batch), st, appended, 1, a);
}

}  // namespace
}  // namespace asrspec

using namespace asrspec;

extern "C" {

int64_t asr_spec_paged8_attend_ws(const asr_paged8_cache* c, const asr_paged_rows* r, int32_t dtype) {
  Paged8View v;
  PagedRows w;
  if (int rc = paged8_view(c, &v)) return rc;
  if (dtype < 1) return ASR_E_INVAL;
  if (int rc = paged8_rows(c, r, dtype, &w)) return rc;
  return attend8_ws_bytes(c->head_dim, w.max_rows * w.group);
}

int asr_spec_paged8_attend(const asr_paged8_cache* c, const asr_paged_rows* r, int32_t dtype, void* out, float* lse,
                           void* ws, int64_t ws_bytes, void* stream) {
  Attend8Args a{};
  if (int rc = paged8_view(c, &a.p)) return rc;
  if (dtype < 1) return ASR_E_INVAL;
  if (int rc = paged8_rows(c, r, dtype, &a.r)) return rc;
  if (a.r.k_new)
    if (int rc = paged8_writable(c)) return rc;
  if (!out || !ws || ((uintptr_t)out | (uintptr_t)ws) % 16 || (uintptr_t)lse % 4) return ASR_E_INVAL;
  const int m_rows = a.r.max_rows * a.r.group;
  if (ws_bytes < attend8_ws_bytes(c->head_dim, m_rows)) return ASR_E_CAPACITY;
  const int tr = with_shape(c->head_dim, m_rows, [](auto s) { return s.TR; });
  const long long tiles = ((long long)m_rows + tr - 1) / tr;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  // The kernel for prompts takes 256 rows of a K/V head a block and does not share keys between blocks: it needs rows to fill its
  // tiles and items to fill the SMs.  Rows are those that a call has room for: a prompt among single rows takes all of them
  // there.  Measured for heads of 64 and sequences of one length (heads of 128 and uneven ones follow unmeasured), us a call, this kernel and that one: 20 heads of 64, 32 sequences of 448
  // slots, 64 rows 67 and 68, 96 rows 113 and 84, 256 rows 356 and 117; 40 items of 256 rows by 1000 slots 67 and 40; 8
  // items of 300 rows by 8000 slots 50 and 151, 6 of 256 by 100000 268 and 1608.
  const long long items = ((long long)m_rows + 255) / 256 * c->kv_heads * c->batch;
  const bool prompt = m_rows > 64 && 4 * items >= paged_sm_count();
  if (!prompt && tiles * c->kv_heads * c->batch * ((long long)a.p.c.max_slots / 32 + 2) > 0x7fffffffll) return ASR_E_CAPACITY;   // 32-bit units
  const bool appends = a.r.k_new != nullptr;
  if (appends && launch_append8(a.p, a.r, dtype, st) != cudaSuccess) return ASR_E_CUDA;
  a.r.k_new = a.r.v_new = nullptr;   // the rows are in the pages from here on
  if (prompt)
    return launch_prompt8(a.p, a.r, dtype, out, lse, static_cast<int*>(ws), appends, st) == cudaSuccess ? ASR_OK : ASR_E_CUDA;
  a.c = a.p.c;
  a.out = static_cast<char*>(out);
  a.lse = lse;
  a.tickets = static_cast<int*>(ws);
  a.ws = reinterpret_cast<float*>(a.tickets + MAX_WORKERS);
  const cudaError_t e = with_shape(c->head_dim, m_rows, [&](auto s) {
    using C = decltype(s);
    return dtype == 1 ? launch_attend8<__nv_bfloat16, C>(a, appends, st) : launch_attend8<__half, C>(a, appends, st);
  });
  return e == cudaSuccess ? ASR_OK : ASR_E_CUDA;
}

}  // extern "C"
