// Attention of prompts over an 8-bit paged cache: many rows a sequence, so that
// the tensor cores and the exponentials bound it and not the cache's bytes.
//
// A block takes 256 rows of a sequence and K/V head (its rows times the query
// heads that share the head), as two tiles of 128, and walks tiles of 128 keys:
//   * 4 warps turn codes into fp16 in 128-byte-swizzled shared memory, two
//     stages of K and of V, a tile's loads in flight while the one before is
//     converted; both row tiles use what they write;
//   * one thread issues tcgen05.mma: S = q K^T (128 x 128, fp32 in tensor
//     memory) and O += p V with p read from tensor memory, where it takes the
//     place of the scores.  The two row tiles alternate, so that one's products
//     run while the other's scores are being weighed;
//   * 4 warps a row tile, a thread a row, weigh the scores.  The first pass over them takes
//     each group's maximum, the second the exponentials.  Running maximum and
//     reference of the weights (as in the kernel for few rows) move only when
//     a weight would leave [.., 2^15] or a maximum grows by more than 2^4 in p, which
//     after the first tiles is rare; the output is then rescaled in place.
//     A weight vanishes where it is below 2^-35 of the row's largest.
// Slots hidden from a row weigh 0, and V codes that are NaN are taken out on the
// way in: the rows that see such a slot are made NaN at the end.
#include <atomic>
#include <type_traits>

#include "kernels.h"
#include "paged8.cuh"

namespace asrspec {
namespace {

constexpr int BM = 128, BN = 128, THREADS = 416;   // rows and keys of a tile; 8 warps weigh, 4 convert, 1 issues products

struct Prompt8Args {
  Paged8View p;
  PagedRows r;
  char* out;
  float* lse;
  int tiles;   // of 256 rows
};

template <int D> struct Prompt8Mem {
  static constexpr int HB = D / 64, BLOCK = 16384;             // 64 columns of 128 rows
  static constexpr int Q = 0, K = 2 * HB * BLOCK, V = K + 2 * HB * BLOCK, END = V + 2 * HB * BLOCK;
  // one block an SM: each takes all of tensor memory
  static constexpr int BYTES = (END < 120 * 1024 ? 120 * 1024 : END) + 1024;
};

struct Prompt8Bars {
  uint64_t q_full[2], k_full[2], k_free[2], v_full[2], v_free[2], sc_full[4], s_full[2], p_full[2], o_full[2];
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
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

template <typename T, int D>
__global__ void __launch_bounds__(THREADS, 1) prompt8_kernel(const Prompt8Args a) {
  using M = Prompt8Mem<D>;
  constexpr int HB = M::HB;
  extern __shared__ uint8_t raw[];
  __shared__ __align__(8) Prompt8Bars bars;
  __shared__ GroupScales scales[4];
  __shared__ int nan_key[D];      // of a column of V the first key whose code is a NaN
  __shared__ int s_len, s_rows, s_any_nan;
  __shared__ uint32_t s_tmem;
  const uint32_t smem = (smem_u32(raw) + 1023) / 1024 * 1024;
  const PagedView& c = a.p.c;
  const PagedRows& r = a.r;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int kvh = blockIdx.x % c.kv_heads, b = blockIdx.x / c.kv_heads % c.batch;
  const int m0 = (a.tiles - 1 - (int)(blockIdx.x / c.kv_heads / c.batch)) * 2 * BM;   // late rows, which see most, first

  if (tid == 0) {
    int len, rows;
    paged_lens(c, r, b, len, rows);
    s_len = len, s_rows = rows, s_any_nan = 0;
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars.q_full[i], BM), mbar_init(&bars.k_full[i], 128), mbar_init(&bars.v_full[i], 128);
      mbar_init(&bars.k_free[i], 1), mbar_init(&bars.v_free[i], 1), mbar_init(&bars.s_full[i], 1);
      mbar_init(&bars.p_full[i], BM), mbar_init(&bars.o_full[i], 1);
    }
    for (int i = 0; i < 4; ++i) mbar_init(&bars.sc_full[i], 128);
    fence_mbar_init();
  }
  if (tid < D) nan_key[tid] = 0x7fffffff;
  if (warp == 12) tmem_alloc(&s_tmem, 512), tmem_relinquish();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  const int len = s_len, rows = s_rows, keys = rows == 0 ? 0 : len + (r.causal ? rows : 0), m_rows = rows * r.group;
  // key tiles of each row tile: up to what its last row sees
  auto seen_by = [&](int m) { return r.causal ? len + (int)r.groups.div(m) + 1 : len; };
  auto tiles_of = [&](int x) {
    const int first = m0 + x * BM;
    return first >= m_rows ? 0 : (seen_by(min(first + BM, m_rows) - 1) + BN - 1) / BN;
  };
  const int n0 = tiles_of(0), n1 = tiles_of(1), n = max(n0, n1);
  bool gave_up = false;
  pdl_wait();   // the append

  if (warp < 8) {
    // ------------------------------------------------------------ the weights of a row
    const int x = warp >> 2, row_in = tid & 127, nx = x ? n1 : n0, m = m0 + x * BM + row_in;
    const int row = (int)r.groups.div(m), hq = kvh * r.group + m - row * r.group;
    const uint32_t lanes = (uint32_t)(warp & 3) << 21, s_at = tmem + lanes + x * BN, o_at = tmem + lanes + 2 * BN + x * D;
    const bool mine = m < m_rows;
    const int lim = mine ? min(keys, seen_by(m)) : 0, all_see = nx ? seen_by(m0 + x * BM) : 0;
    float sc = r.scale * LOG2E;
    if (nx > 0) {
      const char* src = r.q + b * r.q_b + (long long)row * r.q_r + hq * r.q_h;
      const uint32_t dst = smem + M::Q + x * HB * M::BLOCK + row_in * 128;
      float f0 = 1.f, f1 = 1.f;
      if constexpr (!std::is_same<T, __half>::value) {   // to fp16 by a power of two: see the kernel for few rows
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
          const uint4 v = ldg_if(mine, src + i * 16);
#pragma unroll
          for (int y = 0; y < 4; ++y) most = max(most, max(reg_of(v, y) & 0x7fffu, reg_of(v, y) >> 16 & 0x7fffu));
        }
        const int e = min(100, 14 - ((int)(most >> 7) - 127));
        f0 = pow2(e / 2), f1 = pow2(e - e / 2);
        sc = fmaxf(sc * pow2(-(e / 2)) * pow2(-(e - e / 2)), 1.17549435e-38f);
      }
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        uint4 v = ldg_if(mine, src + i * 16);
        if constexpr (!std::is_same<T, __half>::value) {
          uint32_t y[4];
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            const uint32_t w = reg_of(v, z);
            y[z] = Mma16<__half>::pack(__int_as_float(w << 16) * f0 * f1, __int_as_float(w & 0xffff0000u) * f0 * f1);
          }
          v = make_uint4(y[0], y[1], y[2], y[3]);
        }
        sts16(dst + i / 8 * M::BLOCK + ((i % 8) ^ (row_in & 7)) * 16, v.x, v.y, v.z, v.w);
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      mbar_arrive(&bars.q_full[x]);
    }
    float mx = -INFINITY, l = 0.f;   // the maximum, in units of the product; the sum of p
    int li = 126;                    // log2 of what weights are multiplied by
    for (int j = 0; j < nx; ++j) {
      const GroupScales& gs = scales[j & 3];
      bar_wait(&bars.sc_full[j & 3], j >> 2 & 1, c.status, gave_up);
      bar_wait(&bars.s_full[x], j & 1, c.status, gave_up);
      __syncwarp();
      tc_fence_after();
      const bool full = (j + 1) * BN <= all_see;   // of every row that counts
      const int left = lim - j * BN;               // columns that this row sees
      float gm[8];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t s[32];
        tmem_ld32(s_at + q * 32, s);
        tmem_wait_ld();
        if (!full)
#pragma unroll
          for (int i = 0; i < 32; ++i) s[i] = q * 32 + i < left ? s[i] : 0xff800000u;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float g0 = __uint_as_float(s[h * 16]), g1 = __uint_as_float(s[h * 16 + 1]);
#pragma unroll
          for (int i = 2; i < 16; i += 2) g0 = fmaxf(g0, __uint_as_float(s[h * 16 + i])), g1 = fmaxf(g1, __uint_as_float(s[h * 16 + i + 1]));
          gm[q * 2 + h] = fmaxf(g0, g1) * gs.k[q * 2 + h];
        }
      }
      float most = gm[0], top = -INFINITY;
#pragma unroll
      for (int u = 1; u < 8; ++u) most = fmaxf(most, gm[u]);
#pragma unroll
      for (int u = 0; u < 8; ++u) top = fmaxf(top, (gm[u] - mx) * sc + gs.lv[u]);
      if (__any_sync(0xffffffffu, (most - mx) * sc > 4.f || top + (float)li > 15.f)) {
        float grown = 0.f;
        int k = 0;
        if (most > mx) {
          grown = mx == -INFINITY ? 0.f : (most - mx) * sc;
          k = min((int)fminf(grown, 1000.f), 126 - li);
          mx = most, l *= ex2(-grown), li += k;
        }
        top = -INFINITY;
#pragma unroll
        for (int u = 0; u < 8; ++u) top = fmaxf(top, (gm[u] - mx) * sc + gs.lv[u]);
        const int e = top + (float)li > 11.f ? min((int)ceilf(top) + li - 11, li + 126) : 0;
        li -= e;
        if (j > 0) {   // the products before have been added up: the scores' came after them
          const float f = ex2((float)(k - e) - grown);
          __syncwarp();
#pragma unroll
          for (int q = 0; q < D / 32; ++q) {
            uint32_t o[32];
            tmem_ld32(o_at + q * 32, o);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
            tmem_st16(o_at + q * 32, o);
            tmem_st16(o_at + q * 32 + 16, o + 16);
          }
        }
      }
      const float base = mx == -INFINITY ? 0.f : mx, inv = pow2(li);
      const uint64_t base2 = two(-base, -base), sc2 = two(sc, sc);
      uint64_t sum2 = 0;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t s[32], p[16];
        tmem_ld32(s_at + q * 32, s);
        tmem_wait_ld();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float ks = gs.k[q * 2 + h], f = fminf(gs.v[q * 2 + h] * inv, 8.507059173e37f);
          const uint64_t ks2 = two(ks, ks), f2 = two(f, f);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int at = h * 16 + 2 * i;
            float2 t = parts(mul2(fma2(two(__uint_as_float(s[at]), __uint_as_float(s[at + 1])), ks2, base2), sc2));
            if (!full) t = make_float2(q * 32 + at < left ? t.x : -INFINITY, q * 32 + at + 1 < left ? t.y : -INFINITY);
            const uint64_t e2 = two(ex2(t.x), ex2(t.y));
            sum2 = add2(sum2, e2);
            const float2 w = parts(mul2(e2, f2));
            p[h * 8 + i] = Mma16<__half>::pack(w.x, w.y);
          }
        }
        tmem_st16(s_at + q * 16, p);   // over scores that have been read
      }
      const float2 sum = parts(sum2);
      l += sum.x + sum.y;
      tmem_wait_st();
      tc_fence_before();
      mbar_arrive(&bars.p_full[x]);
    }
    // ---------------------------------------------------------------- the row's end
    if (nx > 0) {
      bar_wait(&bars.o_full[x], 0, c.status, gave_up);
      __syncwarp();
      tc_fence_after();
    }
    const size_t at = ((size_t)b * r.max_rows + row) * r.heads + hq;
    T* out = reinterpret_cast<T*>(a.out) + at * D;
    const bool there = row < r.max_rows;
    const bool any_nan = *reinterpret_cast<volatile int*>(&s_any_nan) != 0;
    const float f = lim > 0 && l != 0.f ? __fdividef(1.f, l) * pow2(-li) : 0.f;
#pragma unroll
    for (int q = 0; q < D / 32; ++q) {
      uint32_t o[32];
      if (nx > 0) {
        __syncwarp();
        tmem_ld32(o_at + q * 32, o);
        tmem_wait_ld();
      }
#pragma unroll
      for (int i = 0; i < 32; ++i) o[i] = lim > 0 ? __float_as_uint(__uint_as_float(o[i]) * f) : 0u;
      if (any_nan)
#pragma unroll
        for (int i = 0; i < 32; ++i)
          if (nan_key[q * 32 + i] < lim) o[i] = 0x7fffffffu;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t w[4];
#pragma unroll
        for (int y = 0; y < 4; ++y) w[y] = Mma16<T>::pack(__uint_as_float(o[i * 8 + 2 * y]), __uint_as_float(o[i * 8 + 2 * y + 1]));
        if (there) *reinterpret_cast<uint4*>(out + q * 32 + i * 8) = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
    if (there && a.lse) a.lse[at] = lim > 0 ? (mx * sc + __log2f(l)) * LN2 : -INFINITY;
    tc_fence_before();
  } else if (warp < 12) {
    // ------------------------------------------------------------ codes to fp16
    constexpr int LK = D / 16, KI = 32 / LK, IT = 32 / KI;   // lanes a key, keys an instruction, instructions of a warp's 32 keys
    const int w = warp - 8, key0 = w * 32 + lane / LK, col = lane % LK, groups = (keys + PG_GROUP - 1) / PG_GROUP;
    const int* table_row = c.table + b * c.table_stride;
    const long long head = kvh * c.head_stride + col * 16;
    uint4 kc[IT], vc[IT];
    int pid[2];
    long long off[2];
    float ks = 1.f, vs = 1.f;
    auto look_up = [&](int j) {
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const int grp = j * 8 + w * 2 + g;
        pid[g] = grp < groups ? __ldg(table_row + c.groups.div((uint32_t)grp)) : 0;   // looked at when used
      }
    };
    auto place = [&](int j) {   // pages of tile j, as looked up; its scales, a group a lane
      const int g0 = j * 8 + w * 2;
#pragma unroll
      for (int g = 0; g < 2; ++g) off[g] = paged_offset(c, pid[g] = paged_valid(c, pid[g]), g0 + g) + head;
      ks = vs = 1.f;
      if (lane < 2 && g0 + lane < groups) {
        const long long at = a.p.scale_at(lane ? pid[1] : pid[0], kvh, g0 + lane);
        ks = __ldcg(a.p.k_scale + at), vs = __ldcg(a.p.v_scale + at);
      }
    };
    auto load = [&](const char* pages, int j, uint4 (&x)[IT]) {
#pragma unroll
      for (int i = 0; i < IT; ++i) {
        const int in = i * KI + lane / LK;
        x[i] = ld_if_l2(j * BN + w * 32 + in < keys, pages + off[i * KI / PG_GROUP] + (in % PG_GROUP) * c.slot_stride);
      }
    };
    auto store = [&](uint32_t dst, const uint4 (&x)[IT]) {
#pragma unroll
      for (int i = 0; i < IT; ++i) {
        const int key = key0 + i * KI;
        const uint32_t at = dst + col / 4 * M::BLOCK + key * 128;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t c0 = reg_of(x[i], 2 * h), c1 = reg_of(x[i], 2 * h + 1);
          sts16(at + (((col % 4 * 2 + h) ^ (key & 7)) << 4), half2_of(c0), half2_of(c0 >> 16), half2_of(c1), half2_of(c1 >> 16));
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    };
    if (n > 0) {
      look_up(0);
      place(0);
      load(c.k, 0, kc);
      load(c.v, 0, vc);
      look_up(1);
    }
    for (int j = 0; j < n; ++j) {
      const int st = j & 1;
      if (lane < 2) {
        GroupScales& gs = scales[j & 3];
        gs.k[w * 2 + lane] = ks, gs.v[w * 2 + lane] = vs;
        gs.lv[w * 2 + lane] = fmaxf(__log2f(vs), -126.f);
      }
      mbar_arrive(&bars.sc_full[j & 3]);
      if (j >= 2) bar_wait(&bars.k_free[st], (j >> 1) - 1 & 1, c.status, gave_up);
      store(smem + M::K + st * HB * M::BLOCK, kc);
      mbar_arrive(&bars.k_full[st]);
      const bool more = j + 1 < n;
      if (more) {
        place(j + 1);
        load(c.k, j + 1, kc);
      }
      uint32_t bad = 0;
#pragma unroll
      for (int i = 0; i < IT; ++i) bad |= nan_codes(vc[i].x) | nan_codes(vc[i].y) | nan_codes(vc[i].z) | nan_codes(vc[i].w);
      if (bad) {
        s_any_nan = 1;
#pragma unroll 1
        for (int i = 0; i < IT; ++i) {
          uint4 v = make_uint4(0, 0, 0, 0);
#pragma unroll
          for (int y = 0; y < IT; ++y)
            if (y == i) v = vc[y];
#pragma unroll 1
          for (int y = 0; y < 16; ++y)
            if (nan_codes(reg_of(v, y / 4)) >> (y % 4 * 8) & 1) atomicMin(&nan_key[col * 16 + y], j * BN + key0 + i * KI);
        }
#pragma unroll
        for (int i = 0; i < IT; ++i) {
          vc[i].x &= ~nan_codes(vc[i].x), vc[i].y &= ~nan_codes(vc[i].y);
          vc[i].z &= ~nan_codes(vc[i].z), vc[i].w &= ~nan_codes(vc[i].w);
        }
      }
      if (j >= 2) bar_wait(&bars.v_free[st], (j >> 1) - 1 & 1, c.status, gave_up);
      store(smem + M::V + st * HB * M::BLOCK, vc);
      mbar_arrive(&bars.v_full[st]);
      if (more) {
        load(c.v, j + 1, vc);
        look_up(j + 2);
      }
    }
  } else if (lane == 0) {
    // ------------------------------------------------------------ products
    constexpr uint32_t F32 = 1u << 4, M128 = (uint32_t)(BM >> 4) << 24;   // accumulator type; fp16 operands are 0
    constexpr uint32_t id_s = F32 | M128 | (uint32_t)(BN >> 3) << 17, id_o = F32 | M128 | 8u << 17 | 1u << 16;   // V: contraction axis outermost
    auto scores = [&](int x, int j) {
      const uint32_t q = smem + M::Q + x * HB * M::BLOCK, k = smem + M::K + (j & 1) * HB * M::BLOCK;
#pragma unroll
      for (int h = 0; h < HB; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          umma_f16(tmem + x * BN, umma_desc_sw128(q + h * M::BLOCK + i * 32), umma_desc_sw128(k + h * M::BLOCK + i * 32), id_s, h + i > 0);
      umma_commit(&bars.s_full[x]);
    };
    if (n > 0) bar_wait(&bars.k_full[0], 0, c.status, gave_up);
    for (int x = 0; x < 2; ++x)
      if ((x ? n1 : n0) > 0) {
        bar_wait(&bars.q_full[x], 0, c.status, gave_up);
        tc_fence_after();
        scores(x, 0);
      }
    if (n > 0) umma_commit(&bars.k_free[0]);
    for (int j = 0; j < n; ++j) {
      bar_wait(&bars.v_full[j & 1], j >> 1 & 1, c.status, gave_up);
      if (j + 1 < n) bar_wait(&bars.k_full[j + 1 & 1], (j + 1) >> 1 & 1, c.status, gave_up);
      for (int x = 0; x < 2; ++x) {
        const int nx = x ? n1 : n0;
        if (j < nx) {
          bar_wait(&bars.p_full[x], j & 1, c.status, gave_up);
          tc_fence_after();
          const uint32_t v = smem + M::V + (j & 1) * HB * M::BLOCK;
#pragma unroll
          for (int h = 0; h < HB; ++h)
#pragma unroll
            for (int i = 0; i < BN / 16; ++i)
              umma_f16_ts(tmem + 2 * BN + x * D + h * 64, tmem + x * BN + i * 8, desc_mn(v + h * M::BLOCK + i * 2048), id_o, j + i > 0);
          if (j + 1 == nx) umma_commit(&bars.o_full[x]);
        }
        if (x) umma_commit(&bars.v_free[j & 1]);
        if (j + 1 < nx) scores(x, j + 1);
        if (x && j + 1 < n) umma_commit(&bars.k_free[j + 1 & 1]);
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 12) tmem_dealloc(tmem, 512);
}

template <typename T, int D>
cudaError_t launch_d(const Prompt8Args& a, bool appended, cudaStream_t st) {
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
  const long long blocks = (long long)a.tiles * a.p.c.kv_heads * a.p.c.batch;
  return launch_ex(kernel, dim3((unsigned)blocks), dim3(THREADS), Prompt8Mem<D>::BYTES, st, appended, 1, a);
}

}  // namespace

cudaError_t launch_prompt8(const Paged8View& c, const PagedRows& r, int dtype, void* out, float* lse, bool appended, cudaStream_t st) {
  Prompt8Args a{c, r, static_cast<char*>(out), lse, (r.max_rows * r.group + 2 * BM - 1) / (2 * BM)};
  if ((long long)a.tiles * c.c.kv_heads * c.c.batch > 0x7fffffffll) return cudaErrorInvalidValue;
  if (dtype == 1) return c.dim == 64 ? launch_d<__nv_bfloat16, 64>(a, appended, st) : launch_d<__nv_bfloat16, 128>(a, appended, st);
  return c.dim == 64 ? launch_d<__half, 64>(a, appended, st) : launch_d<__half, 128>(a, appended, st);
}

}  // namespace asrspec
