// Shared parts of the operators over a paged K/V cache: fast division, page
// rows, the distribution of (sequence, head, key step) work over warps, and
// the register fragments in which a warp reads keys.
#pragma once

#include <cuda_fp16.h>

#include "common.cuh"

namespace asrspec {

constexpr int PG_GROUP = 16;         // page sizes are multiples of this many slots
constexpr int PG_MAX_BATCH = 1024;   // sequences of one call (their prefix sums sit in shared memory)
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// n / d for 0 <= n < 2^31 by one multiply and shift (mul = ceil(2^(31 + bits) / d), bits = ceil(log2 d)).
struct FastDiv {
  uint32_t d, mul, shift;
  __device__ __forceinline__ uint32_t div(uint32_t n) const {
    return d == 1 ? n : (uint32_t)(((uint64_t)n * mul) >> shift);
  }
};
inline FastDiv make_fastdiv(uint32_t d) {
  FastDiv f{d, 0, 0};
  if (d > 1) {
    uint32_t bits = 0;
    while ((1ull << bits) < d) ++bits;
    f.shift = 31 + bits;
    f.mul = (uint32_t)(((1ull << f.shift) + d - 1) / d);
  }
  return f;
}

// A paged cache as the kernels see it.  Strides in bytes.
struct PagedView {
  char *k, *v;
  long long page_stride, head_stride, slot_stride;
  const int* table;
  long long table_stride;
  int n_pages, page_size, max_slots, kv_heads, batch;
  FastDiv groups;   // 16-slot groups per page
  int* status;
};

// The rows of one call.  Strides in bytes.
struct PagedRows {
  const char* q;
  long long q_b, q_r, q_h;
  const char *k_new, *v_new;
  long long n_b, n_r, n_h;
  const int *kv_len, *rows;
  int max_rows, heads, group, causal;
  float scale;
};

// Committed slots and rows of one sequence.  Values out of range set the
// status word and leave the sequence without rows.
__device__ __forceinline__ void paged_lens(const PagedView& c, const PagedRows& r, int b, int& len, int& rows) {
  len = r.kv_len[b];
  rows = r.rows ? r.rows[b] : r.max_rows;
  int bad = 0;
  if (rows < 0 || rows > r.max_rows) bad |= ST_BAD_LENS;
  if (len < 0 || len > c.max_slots || (!bad && r.causal && len + rows > c.max_slots)) bad |= ST_CAPACITY;
  if (bad) {
    if (c.status) set_status(c.status, bad);
    len = rows = 0;
  }
}

// The page of a sequence's 16-slot group `grp`.  An id out of range sets the
// status word and page 0 stands in, so that reads stay in the pool.
__device__ __forceinline__ int paged_id(const PagedView& c, const int* table_row, int grp) {
  int pid = __ldg(table_row + c.groups.div((uint32_t)grp));
  if ((unsigned)pid >= (unsigned)c.n_pages) {
    if (c.status) set_status(c.status, ST_BOUNDS);
    pid = 0;
  }
  return pid;
}
// Byte offset of a group's slot 0 in the pool.
__device__ __forceinline__ long long paged_offset(const PagedView& c, int pid, int grp) {
  const int in_page = grp - (int)(c.groups.div((uint32_t)grp) * c.groups.d);
  return (long long)pid * c.page_stride + (long long)(in_page * PG_GROUP) * c.slot_stride;
}

// 2^x by the hardware's approximation (2 ulp; 0 below 2^-126).
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ uint4 ldg_stream(const char* p) {   // read once: no L1 line
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}

// ---------------------------------------------------------------------------
// Work distribution.  The units of a call are key steps in the order
// (sequence, item, step), an item being what one warp keeps in registers (a
// K/V head and a tile of rows).  U units are dealt to W warps in contiguous
// runs, warp w taking [w U / W, (w + 1) U / W): equal shares whatever the
// lengths, at most two items of a warp are shared with others.
// ---------------------------------------------------------------------------
struct WorkPlan {
  long long units;   // U
  int workers;       // W in use
};
__device__ __forceinline__ long long work_start(const WorkPlan& p, long long w) { return w * p.units / p.workers; }
// the warp whose run holds unit u
__device__ __forceinline__ int work_owner(const WorkPlan& p, long long u) {
  return (int)(((u + 1) * p.workers - 1) / p.units);
}

// The block's copy of the call's lengths and the prefix sums of the sequences'
// units, so that later look-ups stay on chip: shared memory of plan_bytes(B).
struct PlanMem {
  long long* pre;   // [B + 1]
  int2* lens;       // [B] committed slots, rows
};
inline size_t plan_bytes(int B) { return (2 * (size_t)B + 1) * sizeof(long long); }

// Every thread of the block calls it.  units(len, rows): a sequence's units;
// fewer units than min_units are not dealt to a warp of their own.
template <typename F>
__device__ __forceinline__ WorkPlan work_plan(const PagedView& c, const PagedRows& r, PlanMem& mem, int max_workers,
                                              int min_units, F units) {
  extern __shared__ __align__(16) long long plan_smem[];
  const int B = c.batch, lane = threadIdx.x & 31;
  mem.pre = plan_smem;
  mem.lens = reinterpret_cast<int2*>(plan_smem + B + 1);
  for (int b = threadIdx.x; b < B; b += blockDim.x) {
    int2 n;
    paged_lens(c, r, b, n.x, n.y);
    mem.lens[b] = n;
    mem.pre[b + 1] = units(n.x, n.y);
  }
  __syncthreads();
  if (threadIdx.x < 32) {
    long long base = 0;
    for (int b0 = 0; b0 < B; b0 += 32) {
      long long x = b0 + lane < B ? mem.pre[b0 + lane + 1] : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
      }
      if (b0 + lane < B) mem.pre[b0 + lane + 1] = base + x;
      base += __shfl_sync(0xffffffffu, x, 31);
    }
    if (lane == 0) mem.pre[0] = 0;
  }
  __syncthreads();
  WorkPlan p;
  p.units = mem.pre[B];
  const long long w = (p.units + min_units - 1) / min_units;
  p.workers = (int)(w < 1 ? 1 : w < max_workers ? w : max_workers);
  return p;
}
// the sequence that holds unit u: pre[b] <= u < pre[b + 1]
__device__ __forceinline__ int work_find(const long long* pre, int B, long long u) {
  int lo = 0, hi = B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (pre[mid] <= u) lo = mid;
    else hi = mid;
  }
  return lo;
}

// ---------------------------------------------------------------------------
// 16-bit types on mma.sync m16n8k16 (fp32 accumulate)
// ---------------------------------------------------------------------------
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(float v) { return v; }

template <typename T> struct Mma16;
template <> struct Mma16<__nv_bfloat16> {
  static __device__ __forceinline__ void mma(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
  }
};
template <> struct Mma16<__half> {
  static __device__ __forceinline__ void mma(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
  }
};

template <int D> struct Cfg16 { static constexpr int KS = D == 64 ? 32 : 16; };   // keys a step

// one sequence's share of the work
struct SeqWork {
  int len, rows, keys, steps, tiles;
};
template <int KS, int TR>
__device__ __forceinline__ SeqWork seq_work(const PagedRows& r, int len, int rows) {
  SeqWork s;
  s.len = len;
  s.rows = rows;
  s.keys = s.rows ? s.len + (r.causal ? s.rows : 0) : 0;
  s.steps = (s.keys + KS - 1) / KS;
  s.tiles = (s.rows * r.group + TR - 1) / TR;
  return s;
}

// The step's fragments of one head.  Full steps lie below kv_len; the others
// pick each key's source and zero what is past the end.
template <typename T, int D>
struct Keys16 {
  static constexpr int KS = Cfg16<D>::KS, NG = KS / PG_GROUP, NC = D / 32, NV = D / 64;
  const PagedView& c;
  const PagedRows& r;
  const int* table_row;
  long long head_off;
  const char *kn, *vn;   // this sequence's and head's new rows
  int len, keys, g, t;
  bool fresh;            // slots from len on are read from them

  __device__ __forceinline__ int id(int step, int u) const {   // page of group u of a step, fetched ahead
    const int grp = step * NG + u;
    return grp * PG_GROUP < keys ? paged_id(c, table_row, grp) : 0;
  }
  __device__ __forceinline__ bool full(int step) const { return (step + 1) * KS <= len; }
  __device__ __forceinline__ void offsets(int step, const int* pid, long long* off) const {
#pragma unroll
    for (int u = 0; u < NG; ++u) off[u] = paged_offset(c, pid[u], step * NG + u) + head_off;
  }

  // K: kf[key tile][16-byte chunk], lane's key 8 w + g of a group
  __device__ __forceinline__ void load_k(int step, const long long* off, uint4 (&kf)[KS / 8][NC]) const {
    const int lane_off = g * (int)c.slot_stride + t * 16, row8 = 8 * (int)c.slot_stride;
    if (full(step)) {
#pragma unroll
      for (int u = 0; u < NG; ++u) {
        const char* p = c.k + off[u] + lane_off;
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
          for (int j = 0; j < NC; ++j) kf[u * 2 + w][j] = ldg_stream(p + w * row8 + j * 64);
      }
    } else {
#pragma unroll
      for (int u = 0; u < NG; ++u)
#pragma unroll
        for (int w = 0; w < 2; ++w)
          edge<NC, 64>(c.k + off[u] + lane_off + w * row8, kn + t * 16, step * KS + u * PG_GROUP + w * 8 + g, kf[u * 2 + w]);
    }
  }
  // V: vf[group][which of the lane's four keys 2t, 2t+1, 2t+8, 2t+9][64-wide half]
  __device__ __forceinline__ void load_v(int step, const long long* off, uint4 (&vf)[NG][4][NV]) const {
    const int slot = (int)c.slot_stride, lane_off = 2 * t * slot + g * 16;
#pragma unroll
    for (int u = 0; u < NG; ++u) {
      const char* p = c.v + off[u] + lane_off;
      if (full(step)) {
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
          for (int j = 0; j < NV; ++j) vf[u][w][j] = ldg_stream(p + ((w & 1) + (w >> 1) * 8) * slot + j * 128);
      } else {
#pragma unroll
        for (int w = 0; w < 4; ++w)
          edge<NV, 128>(p + ((w & 1) + (w >> 1) * 8) * slot, vn + g * 16,
                        step * KS + u * PG_GROUP + 2 * t + (w & 1) + (w >> 1) * 8, vf[u][w]);
      }
    }
  }
  // One key of an edge step: from its page, or from the block's rows; zero past the end.
  template <int N, int STRIDE>
  __device__ __forceinline__ void edge(const char* page, const char* fresh_rows, int key, uint4 (&f)[N]) const {
    const char* src = fresh && key >= len ? fresh_rows + (long long)(key - len) * r.n_r : page;
#pragma unroll
    for (int j = 0; j < N; ++j) f[j] = make_uint4(0, 0, 0, 0);
    if (key < keys) {
#pragma unroll
      for (int j = 0; j < N; ++j) f[j] = *reinterpret_cast<const uint4*>(src + j * STRIDE);
    }
  }
  // Write the new rows of an edge step to their pages, from the fragments that
  // the step is about to use.  A bad page id is reported by id(); nothing goes there.
  __device__ __forceinline__ void append_k(int step, const uint4 (&kf)[KS / 8][NC]) const {
#pragma unroll
    for (int u = 0; u < NG; ++u)
#pragma unroll
      for (int w = 0; w < 2; ++w) append<NC, 64>(c.k, step, u, w * 8 + g, t * 16, kf[u * 2 + w]);
  }
  __device__ __forceinline__ void append_v(int step, const uint4 (&vf)[NG][4][NV]) const {
#pragma unroll
    for (int u = 0; u < NG; ++u)
#pragma unroll
      for (int w = 0; w < 4; ++w) append<NV, 128>(c.v, step, u, 2 * t + (w & 1) + (w >> 1) * 8, g * 16, vf[u][w]);
  }
  template <int N, int STRIDE>
  __device__ __forceinline__ void append(char* pages, int step, int u, int in, int byte, const uint4 (&f)[N]) const {
    const int key = step * KS + u * PG_GROUP + in, grp = step * NG + u;
    if (key < len || key >= keys) return;
    const int pid = __ldg(table_row + c.groups.div((uint32_t)grp));
    if ((unsigned)pid >= (unsigned)c.n_pages) return;
    char* p = pages + paged_offset(c, pid, grp) + head_off + in * c.slot_stride + byte;
#pragma unroll
    for (int j = 0; j < N; ++j) *reinterpret_cast<uint4*>(p + j * STRIDE) = f[j];
  }
};

// ---- Host: argument checks shared by the entry points ------------------------
int paged_view(const asr_paged_cache* c, PagedView* v);
int paged_rows(const asr_paged_cache* c, const asr_paged_rows* r, PagedRows* v);
int paged_sm_count();

}  // namespace asrspec
