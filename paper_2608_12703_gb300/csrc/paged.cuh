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
  FastDiv groups;   // by `group`
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
__device__ __forceinline__ int paged_valid(const PagedView& c, int pid) {
  if ((unsigned)pid < (unsigned)c.n_pages) return pid;
  if (c.status) set_status(c.status, ST_BOUNDS);
  return 0;
}
__device__ __forceinline__ int paged_id(const PagedView& c, const int* table_row, int grp) {
  return paged_valid(c, __ldg(table_row + c.groups.div((uint32_t)grp)));
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

__device__ __forceinline__ uint4 ldg_if(bool in, const char* p) {   // zero where not `in`
  uint4 v;
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %5, 0;\n\t"
      "mov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\tmov.b32 %3, 0;\n\t"
      "@p ld.global.nc.v4.u32 {%0,%1,%2,%3}, [%4];\n\t}"
      : "=&r"(v.x), "=&r"(v.y), "=&r"(v.z), "=&r"(v.w)
      : "l"(p), "r"((int)in));
  return v;
}

// Global -> shared copy counted on an mbarrier; addresses and size multiples of 16 bytes.
__device__ __forceinline__ void bulk_copy(uint32_t smem, const char* p, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem), "l"(p),
               "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}
// Waits for a phase, at most about a second; then, and at once from there on,
// it gives up: the status word says so and the results are invalid.
__device__ __forceinline__ void bar_wait(uint64_t* bar, uint32_t parity, int* status, bool& gave_up) {
  if (mbar_try_wait(bar, parity) || gave_up) return;
  const long long t0 = clock64();
  while (!mbar_try_wait(bar, parity)) {
    if (clock64() - t0 > (1ll << 31)) {
      if (status) set_status(status, ST_WAIT_TIMEOUT);
      gave_up = true;
      return;
    }
  }
}
__device__ __forceinline__ uint4 lds16(uint32_t smem) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(smem) : "memory");
  return v;
}

// ---------------------------------------------------------------------------
// Work distribution.  The units of a call are key steps in the order
// (sequence, item, step), an item being what one warp keeps in registers (a
// K/V head and a tile of rows).  U units are dealt to W warps in contiguous
// runs of U / W or one more: equal shares whatever the lengths; at most two
// items of a warp are shared with other warps.  The warps of a block are
// neighbours.  U < 2^31 (checked on the host).
// ---------------------------------------------------------------------------
struct WorkPlan {
  int units, workers;   // U, W in use
  int share, more;      // every warp takes `share` units, the first `more` one more
  __device__ __forceinline__ int start(int w) const { return w * share + min(w, more); }
  __device__ __forceinline__ int owner(int u) const {   // the warp whose run holds unit u
    const unsigned edge = (unsigned)more * (share + 1);
    return (unsigned)u < edge ? (unsigned)u / (share + 1u) : more + ((unsigned)u - edge) / (unsigned)share;
  }
};

// The block's copy of the call's lengths and the prefix sums of the sequences'
// units, so that later look-ups stay on chip: shared memory of plan_bytes(B).
struct PlanMem {
  int2* lens;   // [B] committed slots, rows
  int* pre;     // [B + 1]
};
constexpr size_t plan_bytes(int B) { return ((size_t)B * 12 + 4 + 15) / 16 * 16; }

// Every thread of the block calls it.  units(len, rows): a sequence's units.
template <typename F>
__device__ __forceinline__ WorkPlan work_plan(const PagedView& c, const PagedRows& r, PlanMem& mem, int max_workers, F units) {
  extern __shared__ __align__(16) unsigned char plan_smem[];
  const int B = c.batch, lane = threadIdx.x & 31;
  mem.lens = reinterpret_cast<int2*>(plan_smem);
  mem.pre = reinterpret_cast<int*>(mem.lens + B);
  for (int b = threadIdx.x; b < B; b += blockDim.x) {
    int2 n;
    paged_lens(c, r, b, n.x, n.y);
    mem.lens[b] = n;
    mem.pre[b + 1] = units(n.x, n.y);
  }
  __syncthreads();
  if (threadIdx.x < 32) {
    int base = 0;
    for (int b0 = 0; b0 < B; b0 += 32) {
      int x = b0 + lane < B ? mem.pre[b0 + lane + 1] : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
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
  p.workers = max(1, min(p.units, max_workers));
  p.share = p.units / p.workers;
  p.more = p.units - p.share * p.workers;
  return p;
}
// the sequence that holds unit u, pre[b] <= u < pre[b + 1]; a warp's lanes search together
__device__ __forceinline__ int work_find(const int* pre, int B, int u) {
  const int lane = threadIdx.x & 31;
  int lo = 0;
  if (B > 32) {
    const int step = (B + 31) >> 5, at = lane * step;
    lo = (__popc(__ballot_sync(0xffffffffu, at < B && pre[at] <= u)) - 1) * step;
    B = min(B, lo + step);
  }
  return lo + __popc(__ballot_sync(0xffffffffu, lo + lane < B && pre[lo + lane] <= u)) - 1;
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

// One sequence's share of the work: its keys in steps of KS, first the slots in
// pages, then, where the block's own rows are passed, those rows (whose slots
// are the next ones).
struct SeqWork {
  int len, rows;       // committed slots, rows
  int paged, keys;     // keys in pages, all keys
  int steps, tiles;
};
template <int KS, int TR>
__device__ __forceinline__ SeqWork seq_work(const PagedRows& r, int len, int rows) {
  SeqWork s;
  s.len = len;
  s.rows = rows;
  const int fresh = r.k_new != nullptr ? rows : 0;
  s.paged = rows == 0 ? 0 : len + (r.causal ? rows - fresh : 0);
  s.keys = s.paged + fresh;
  s.steps = (s.keys + KS - 1) / KS;
  s.tiles = (rows * r.group + TR - 1) / TR;
  return s;
}

// A warp's reader of one head's keys and values, step by step.
template <typename T, int D>
struct Keys16 {
  static constexpr int KS = Cfg16<D>::KS, NG = KS / PG_GROUP, NC = D / 32, NV = D / 64, ROW = D * 2;
  const PagedView& c;
  const PagedRows& r;
  SeqWork s;
  const int* table_row;
  long long head_off;
  const char *kn, *vn;   // this sequence's and head's new rows
  int g, t;

  // all of a step's keys are committed, so every row sees them
  __device__ __forceinline__ bool full(int step) const { return (step + 1) * KS <= min(s.len, s.paged); }

  __device__ __forceinline__ int id(int step, int u) const {   // page of group u of a step, fetched ahead
    const int grp = step * NG + u;
    return grp * PG_GROUP < s.paged ? paged_id(c, table_row, grp) : 0;
  }
  __device__ __forceinline__ void offsets(int step, const int* pid, long long* off) const {
#pragma unroll
    for (int u = 0; u < NG; ++u) off[u] = paged_offset(c, pid[u], step * NG + u) + head_off;
  }

  // K from the pages into mma B fragments, kf[key tile][16-byte chunk]: a lane's
  // keys are 8 w + g of a group, zero past the end.
  __device__ __forceinline__ void load_k(int step, const long long* off, uint4 (&kf)[KS / 8][NC]) const {
    const int slot = (int)c.slot_stride, lane_off = g * slot + t * 16, left = s.paged - step * KS;
    if (full(step)) {
#pragma unroll
      for (int u = 0; u < NG; ++u) {
        const char* p = c.k + off[u] + lane_off;
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
          for (int j = 0; j < NC; ++j) kf[u * 2 + w][j] = ldg_stream(p + w * 8 * slot + j * 64);
      }
    } else {
#pragma unroll
      for (int u = 0; u < NG; ++u) {
        const char* p = c.k + off[u] + lane_off;
#pragma unroll
        for (int w = 0; w < 2; ++w)
#pragma unroll
          for (int j = 0; j < NC; ++j) kf[u * 2 + w][j] = ldg_if(u * PG_GROUP + w * 8 + g < left, p + w * 8 * slot + j * 64);
      }
    }
  }
  // A step's K (or V) by bulk copies into shared memory, rows of D in slot
  // order, counted on `bar`.  `off`: the lane's group's offset in the pool (see
  // Groups), the step's groups being lanes at, at + 1.  A copy a group where a
  // head's slots are contiguous, else one a row; the block's own rows one a
  // row.  Nothing is written past the end.
  __device__ __forceinline__ void fetch(int step, const char* pages, const char* fresh, long long off, int at, uint32_t dst,
                                        uint64_t* bar) const {
    const int lane = threadIdx.x & 31;
    const bool runs = c.slot_stride == ROW;
    if (runs && (step + 1) * KS <= s.paged) {
      long long o[NG];
#pragma unroll
      for (int u = 0; u < NG; ++u) o[u] = __shfl_sync(0xffffffffu, off, at + u);
      if (lane == 0) {
        mbar_arrive_expect_tx(bar, KS * ROW);
#pragma unroll
        for (int u = 0; u < NG; ++u) bulk_copy(dst + u * PG_GROUP * ROW, pages + o[u], PG_GROUP * ROW, bar);
      }
      return;
    }
    const int in_pages = min(KS, s.paged - step * KS), rows = min(KS, s.keys - step * KS);
    if (lane == at) mbar_arrive_expect_tx(bar, rows * ROW);
    if (runs && (unsigned)(lane - at) < NG) {
      const int n = min(PG_GROUP, in_pages - (lane - at) * PG_GROUP);
      if (n > 0) bulk_copy(dst + (lane - at) * PG_GROUP * ROW, pages + off, n * ROW, bar);
    }
    const int row0 = runs ? max(in_pages, 0) : 0, row = row0 + lane;
    const long long base = __shfl_sync(0xffffffffu, off, at + (NG > 1 && row >= PG_GROUP ? 1 : 0));
    if (row < rows)
      bulk_copy(dst + row * ROW,
                row < in_pages ? pages + base + (row % PG_GROUP) * c.slot_stride
                               : fresh + (long long)(step * KS + row - s.paged) * r.n_r,
                ROW, bar);
  }
};

// Where a run of steps lies in the pool: of every 32 groups a lane looks up one,
// the next 32's page ids a round ahead of their use.
template <typename T, int D>
struct Groups {
  static constexpr int NG = Keys16<T, D>::NG, STEPS = 32 / NG;
  const Keys16<T, D>& ks;
  int grp0, next_pid;
  long long off;
  __device__ __forceinline__ int page(int round) const {
    const int grp = grp0 + round * 32 + (threadIdx.x & 31);
    return grp * PG_GROUP < ks.s.paged ? __ldg(ks.table_row + ks.c.groups.div((uint32_t)grp)) : 0;   // looked at when used
  }
  __device__ __forceinline__ Groups(const Keys16<T, D>& k, int s0) : ks(k), grp0(s0 * NG), next_pid(0), off(0) { next_pid = page(0); }
  // step i of the run: its first lane; the offsets are this round's from here on
  __device__ __forceinline__ int at(int i) {
    if (i % STEPS == 0) {
      const int round = i / STEPS;
      off = paged_offset(ks.c, paged_valid(ks.c, next_pid), grp0 + round * 32 + (threadIdx.x & 31)) + ks.head_off;
      next_pid = page(round + 1);
    }
    return i % STEPS * NG;
  }
};

// A warp writes one head's new rows to their pages, 16 bytes a lane, K and V
// side by side.  A bad page id is reported and nothing goes there.
__device__ __forceinline__ void append_rows(const PagedView& c, const PagedRows& r, const SeqWork& s, int b, int kvh,
                                            int row_bytes) {
  const int lane = threadIdx.x & 31, chunks = row_bytes / 16;      // 8, 16 or 32 a row
  const bool is_v = (lane / (chunks < 16 ? chunks : 16)) & 1;
  const int* table_row = c.table + b * c.table_stride;
  const char* src0 = (is_v ? r.v_new : r.k_new) + b * r.n_b + kvh * r.n_h;
  char* dst0 = (is_v ? c.v : c.k) + kvh * c.head_stride;
  const int at_once = chunks < 16 ? 32 / (2 * chunks) : 1;
  for (int i = chunks < 16 ? lane / (2 * chunks) : 0; i < s.rows; i += at_once) {
    const int slot = s.len + i, page = slot / c.page_size;
    const int pid = __ldg(table_row + page);
    if ((unsigned)pid >= (unsigned)c.n_pages) {
      if (c.status) set_status(c.status, ST_BOUNDS);
      continue;
    }
    const char* src = src0 + (long long)i * r.n_r;
    char* dst = dst0 + pid * c.page_stride + (slot - page * c.page_size) * c.slot_stride;
    for (int x = lane % (chunks < 16 ? chunks : 16); x < chunks; x += 16)
      *reinterpret_cast<uint4*>(dst + x * 16) = __ldg(reinterpret_cast<const uint4*>(src + x * 16));
  }
}

// ---- Host: argument checks shared by the entry points ------------------------
int paged_view(const asr_paged_cache* c, PagedView* v);
int paged_rows(const asr_paged_cache* c, const asr_paged_rows* r, PagedRows* v);
int paged_sm_count();

}  // namespace asrspec
