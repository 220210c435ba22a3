// Who holds which pages of a cache: private pages for what a call is about to
// write (reserve), sequences that go on from others (fork), live pages to the
// front of the pool (compact).
//
// The state is a table of page ids and a count of holders a page; what is free
// is read off the counts, so which pages a call takes depends on the state
// alone: the j-th free page goes to the j-th need.  A plan decides and lists
// what has to be copied; a second kernel copies, over all arrays that the pages
// have a part in (K, V and scales of every layer).  The copies are bound by
// HBM (every byte read and written once), all else by launches and by the
// chain of dependent look-ups: the plan is one block where the pool has up to
// CHUNK pages, so that its steps are block barriers and not launches.
// Measured, device time: private pages for 256 sequences after a fork, 6 layers
// of 12 heads of 64, bf16: 46 us for 227 MB, 10 of them the plan; for 8 samples 13
// us, latency; 1024 sequences' rows of up to 2500 entries forked: 9 us, 8 the
// second kernel (three dependent look-ups, then 13 MB); 32 layers of 20 heads of 64 in 8
// bits compacted: 103 us for 590 MB, 5.7 TB/s.  Copies in pieces of a page
// whatever it holds took 70 us where 46 are needed; runs of neighbouring pieces
// a warp, to look job and array up less often, 10 % longer than tasks dealt in turn.
#include <cstring>

#include "kernels.h"
#include "paged.cuh"

namespace asrspec {
namespace {

constexpr int MAX_ARRAYS = 1024;
constexpr int PIECE = 256;                     // units of the heads that a warp copies together, where one has fewer
constexpr int PER = 8, CHUNK = 1024 * PER;     // pages that a thread and a block look at

struct PoolView {
  const int* table;
  long long table_stride;
  const int *held, *refs;
  int* table_out;
  long long out_stride;
  int *held_out, *refs_out;
  int n_pages, page_size, max_pages, batch;
  int* status;
};

// An array as the copy kernels read it, in units of 16 or 4 bytes.
struct PlanArray {
  char* base;
  long long page_stride, head_stride, row_stride;
  FastDiv row_units;               // by the units of a row
  int heads, rows, row_slots, unit;
  int runs;                        // a head's rows lie side by side
  int together;                    // heads of a task
  int first_task, pad;             // tasks of the arrays before it
};
struct PlanHead {
  int n, tasks, page_size, each;   // each: an array's tasks where all have as many, else 0
};

// A workspace, 16-byte parts in this order.
struct PoolMem {
  int* ctl;      // [8] blocks that are done (zero between calls), jobs, live, live pages below that
  int* count;    // [chunks] a chunk's free (compact: live) pages, then those before it
  int* list;     // [n_pages] reserve: free pages in order; compact: where pages below `live` are free
  int* src;      // [n_pages] reserve: holders of a page; compact: live pages at or past `live`
  int* low;      // [n_pages] reserve: lowest holder
  int4* job;     // [n_pages] source, destination, slots
  int* was;      // [batch] fork: pages held before,
  int* now;      // [batch] after,
  int* from;     // [batch] and the sequence whose row is staged, -1: its own
  int* rows;     // [batch][max_pages] fork: the rows
};
enum { C_DONE, C_JOBS, C_LIVE, C_BELOW };
size_t round16(size_t n) { return (n + 15) / 16 * 16; }
size_t pool_mem(const PoolView& p, void* at, PoolMem* m) {
  const size_t chunks = ((size_t)p.n_pages + CHUNK - 1) / CHUNK;
  char* x = static_cast<char*>(at);
  auto take = [&](auto*& to, size_t n) {
    to = reinterpret_cast<std::remove_reference_t<decltype(to)>>(x);
    x += round16(n * sizeof(*to));
  };
  take(m->ctl, 8);
  take(m->count, chunks);
  take(m->list, p.n_pages);
  take(m->src, p.n_pages);
  take(m->low, p.n_pages);
  take(m->job, p.n_pages);
  take(m->was, p.batch);
  take(m->now, p.batch);
  take(m->from, p.batch);
  take(m->rows, (size_t)p.batch * p.max_pages);
  return x - static_cast<char*>(at);
}

__device__ __forceinline__ void report(const PoolView& p, int bits) {
  if (p.status) set_status(p.status, bits);
}
__device__ __forceinline__ int held_of(const PoolView& p, int b) {
  const int n = p.held[b];
  if (n >= 0 && n <= p.max_pages) return n;
  report(p, ST_BAD_LENS);
  return 0;
}
__device__ __forceinline__ bool in_pool(const PoolView& p, int id) {
  if ((unsigned)id < (unsigned)p.n_pages) return true;
  report(p, ST_BOUNDS);
  return false;
}

// Sum of x over the block, `before` that over the threads before this one.
__device__ __forceinline__ int block_scan(int x, int& before, int* warps) {
  const int lane = threadIdx.x & 31, w = threadIdx.x / 32, n = blockDim.x / 32;
  int y = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int z = __shfl_up_sync(0xffffffffu, y, o);
    if (lane >= o) y += z;
  }
  __syncthreads();   // a scan before this one has been read
  if (lane == 31) warps[w] = y;
  __syncthreads();
  int s = lane < n ? warps[lane] : 0;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int z = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += z;
  }
  before = y - x + (w ? __shfl_sync(0xffffffffu, s, w - 1) : 0);
  return __shfl_sync(0xffffffffu, s, 31);
}

// Which of a thread's PER pages of a chunk are free (bit k: page first + k); pages past the end are neither.
struct Pages {
  int first, n, r[PER];
  __device__ __forceinline__ Pages(const PoolView& p, int chunk) {
    first = chunk * CHUNK + threadIdx.x * PER;
    n = max(0, min(PER, p.n_pages - first));
    if (n == PER && ((uintptr_t)p.refs & 15) == 0) {
#pragma unroll
      for (int k = 0; k < PER; k += 4) {
        const int4 v = *reinterpret_cast<const int4*>(p.refs + first + k);
        r[k] = v.x, r[k + 1] = v.y, r[k + 2] = v.z, r[k + 3] = v.w;
      }
    } else {
#pragma unroll
      for (int k = 0; k < PER; ++k) r[k] = k < n ? p.refs[first + k] : 0;
    }
  }
  // refs > 0: live, 0: free; a count below 0 is neither
  __device__ __forceinline__ unsigned live() const {
    unsigned m = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) m |= (k < n && r[k] > 0) << k;
    return m;
  }
  __device__ __forceinline__ unsigned free() const {
    unsigned m = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) m |= (k < n && r[k] == 0) << k;
    return m;
  }
};

// This block is the last of so many to come here; it sees what the others wrote.
__device__ __forceinline__ bool last_block(int* done, int blocks) {
  __shared__ int s_last;
  if (blocks > 1) __threadfence();
  __syncthreads();
  if (blocks == 1) return true;
  if (threadIdx.x == 0) {
    s_last = atomicAdd(done, 1) == blocks - 1;
    if (s_last) *done = 0;   // as the next call needs it
    __threadfence();
  }
  __syncthreads();
  return s_last;
}

// Each chunk's count becomes the sum of those before it; returns the sum of all.
__device__ __forceinline__ int scan_chunks(int* count, int chunks, int* warps) {
  int all = 0;
  for (int i0 = 0; i0 < chunks; i0 += blockDim.x) {
    const int i = i0 + threadIdx.x;
    const int x = i < chunks ? __ldcg(count + i) : 0;
    int before;
    const int sum = block_scan(x, before, warps);
    if (i < chunks) count[i] = all + before;
    all += sum;
  }
  __syncthreads();
  return all;
}

// ------------------------------------------------------------------- fork
struct Fork {
  int was, now, from;   // from == -1: its own entries
};
__device__ __forceinline__ Fork fork_of(const PoolView& p, const int* parent, const int* keep, int b) {
  const int from = parent ? parent[b] : b, was = held_of(p, b);
  if (from < -1 || from >= p.batch) {
    report(p, ST_BOUNDS);
    return {was, was, -1};
  }
  if (from < 0) return {was, 0, -1};
  int now = from == b ? was : held_of(p, from);
  if (keep) {
    const int k = keep[b];
    if (k < 0) {
      report(p, ST_BAD_LENS);
      return {was, was, -1};
    }
    now = min(now, (int)(((long long)k + p.page_size - 1) / p.page_size));
  }
  return {was, now, from == b ? -1 : from};
}

// Counts of holders to the output and, where the table is written in place, the
// rows that sequences take from others, before any is written.
__global__ void __launch_bounds__(256) fork_stage_kernel(const PoolView p, const int* parent, const int* keep, const PoolMem ws,
                                                         bool in_place) {
  pdl_launch();
  if (p.refs_out != p.refs)
    for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < p.n_pages; i += gridDim.x * blockDim.x) p.refs_out[i] = p.refs[i];
  if (!in_place) return;
  for (int b = blockIdx.x; b < p.batch; b += gridDim.x) {
    const Fork f = fork_of(p, parent, keep, b);
    if (f.from >= 0)
      for (int j = threadIdx.x; j < f.now; j += blockDim.x)
        ws.rows[(long long)b * p.max_pages + j] = p.table[f.from * p.table_stride + j];
    if (threadIdx.x == 0) ws.was[b] = f.was, ws.now[b] = f.now, ws.from[b] = f.from;
  }
}

// A block takes FORK_RUN entries of a sequence, FORK_PER a thread: most rows whole, so that the look-ups before the entries are
// paid once.
constexpr int FORK_PER = 8, FORK_RUN = 256 * FORK_PER;
__global__ void __launch_bounds__(256) fork_kernel(const PoolView p, const int* parent, const int* keep, const PoolMem ws,
                                                   bool in_place) {
  const int b = blockIdx.x;
  if (in_place) pdl_wait();
  const Fork f = in_place ? Fork{ws.was[b], ws.now[b], ws.from[b]} : fork_of(p, parent, keep, b);
  if (blockIdx.y == 0 && threadIdx.x == 0) p.held_out[b] = f.now;
  const int* own = p.table + b * p.table_stride;
  const int* next = f.from < 0 ? own : in_place ? ws.rows + (long long)b * p.max_pages : p.table + f.from * p.table_stride;
  const bool writes = p.table_out != p.table || f.from >= 0;
  for (int j0 = blockIdx.y * FORK_RUN; j0 < max(f.was, f.now); j0 += gridDim.y * FORK_RUN) {
    int old[FORK_PER], id[FORK_PER];
#pragma unroll
    for (int k = 0; k < FORK_PER; ++k) {
      const int j = j0 + k * 256 + threadIdx.x;
      old[k] = j < f.was ? own[j] : -1;
      id[k] = j < f.now ? f.from < 0 ? old[k] : next[j] : -1;
    }
#pragma unroll
    for (int k = 0; k < FORK_PER; ++k) {
      const int j = j0 + k * 256 + threadIdx.x;
      if (j < f.now && writes) p.table_out[b * p.out_stride + j] = id[k];
    }
    if (!in_place) pdl_wait();   // the counts are there
#pragma unroll
    for (int k = 0; k < FORK_PER; ++k) {
      const int j = j0 + k * 256 + threadIdx.x;
      const bool out = j < f.was && in_pool(p, old[k]), in = j < f.now && in_pool(p, id[k]);
      if (out && in && old[k] == id[k]) continue;
      if (out) atomicSub(p.refs_out + old[k], 1);
      if (in) atomicAdd(p.refs_out + id[k], 1);
    }
  }
  pdl_wait();   // every block ends after the kernel before it
}

// ---------------------------------------------------------------- reserve
// Pages that a sequence's rows touch: [x, y], y < x: none.
__device__ __forceinline__ int2 wanted(const PoolView& p, const int* lens, const int* rows, int b) {
  const int n = lens[b], r = rows[b], held = p.held[b];
  if (r == 0 && held >= 0 && held <= p.max_pages) return make_int2(0, -1);
  if (r < 0 || n < 0 || held < 0 || held > p.max_pages || n > (long long)held * p.page_size) {
    report(p, ST_BAD_LENS);
    return make_int2(0, -1);
  }
  if ((long long)n + r > (long long)p.max_pages * p.page_size) {
    report(p, ST_CAPACITY);
    return make_int2(0, -1);
  }
  return make_int2(n / p.page_size, (n + r - 1) / p.page_size);
}

struct ReserveMem {   // a sequence's first touched page, what it holds, its tail (see below), entries touched before it
  int first[PG_MAX_BATCH], held[PG_MAX_BATCH], keeps[PG_MAX_BATCH], before[PG_MAX_BATCH + 1], warps[32];
  int list[1024];   // the pages that the call takes, where they are no more than these
};
// Entry i of those touched, in order of sequence and slot: its sequence, page and id (-1: none held), and whether it
// needs another page.
struct Touched {
  int b, j, old;
  bool fresh;
};
__device__ __forceinline__ Touched touched(const PoolView& p, const ReserveMem& m, int i) {
  Touched t;
  int lo = 0, hi = p.batch;   // before[lo] <= i < before[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (m.before[mid] <= i) lo = mid;
    else hi = mid;
  }
  t.b = lo;
  const int at = i - m.before[lo];
  t.j = m.first[lo] + at;
  t.old = t.j < m.held[lo] ? p.table[lo * p.table_stride + t.j] : -1;
  if (t.j >= m.held[lo]) t.fresh = true;
  else t.fresh = !(at == 0 && m.keeps[lo]) && in_pool(p, t.old) && p.refs[t.old] > 1;
  return t;
}

// The first `counters` blocks count the free pages of their chunks, and the last of
// them to be done decides; the others copy the table entries that the call does not touch.
__global__ void __launch_bounds__(1024, 1) reserve_kernel(const PoolView p, const int* lens, const int* rows, int* counts, const PoolMem ws,
                                                       int counters) {
  extern __shared__ __align__(16) unsigned char smem[];
  ReserveMem& m = *reinterpret_cast<ReserveMem*>(smem);
  const int tid = threadIdx.x, chunks = (p.n_pages + CHUNK - 1) / CHUNK;
  pdl_launch();
  if ((int)blockIdx.x >= counters) {   // a warp a sequence
    for (int b = ((int)blockIdx.x - counters) * 32 + tid / 32; b < p.batch; b += ((int)gridDim.x - counters) * 32) {
      const int2 w = wanted(p, lens, rows, b);
      const int held = held_of(p, b);
      for (int j = tid & 31; j < held; j += 32)
        if (j < w.x || j > w.y) p.table_out[b * p.out_stride + j] = p.table[b * p.table_stride + j];
    }
    return;
  }
  // What the sequences touch.  A tail is a first touched page that others hold
  // too; if all who hold it are about to write there the lowest of them keeps it.
  // (Read by every counter: its loads overlap the counting.)
  const int b = tid;
  int2 w = make_int2(0, -1);
  int held = 0, was = 0, tail = -1, tail_refs = 0;
  if (b < p.batch) {
    w = wanted(p, lens, rows, b);
    held = held_of(p, b), was = p.held[b];
    if (w.x <= w.y && w.x < held) {
      const int id = p.table[b * p.table_stride + w.x];
      if ((unsigned)id < (unsigned)p.n_pages && (tail_refs = p.refs[id]) > 1) tail = id;
    }
  }
  unsigned free0 = 0;   // of this block's first chunk
  for (int c = blockIdx.x; c < chunks; c += counters) {
    const Pages g(p, c);
    if (p.refs_out != p.refs)
#pragma unroll
      for (int k = 0; k < PER; ++k)
        if (k < g.n) p.refs_out[g.first + k] = g.r[k];
    if (c == (int)blockIdx.x) free0 = g.free();
    int before;
    const int n = block_scan(__popc(g.free()), before, m.warps);
    if (tid == 0) ws.count[c] = n;
  }
  if (!last_block(ws.ctl + C_DONE, counters)) return;

  if (b < p.batch) m.first[b] = w.x, m.held[b] = held;
  if (tail >= 0) ws.src[tail] = 0, ws.low[tail] = p.batch;
  int before;
  const int total = block_scan(max(0, w.y - w.x + 1), before, m.warps);
  if (b < p.batch) m.before[b] = before;
  if (tid == 0) m.before[p.batch] = total;
  __syncthreads();
  if (tail >= 0) atomicAdd(ws.src + tail, 1), atomicMin(ws.low + tail, b);
  const int free = scan_chunks(ws.count, chunks, m.warps);
  if (b < p.batch) m.keeps[b] = tail >= 0 && __ldcg(ws.src + tail) == tail_refs && __ldcg(ws.low + tail) == b;
  __syncthreads();

  int need = 0, before0 = 0;
  Touched first{0, 0, -1, false};   // of the first round
  for (int i0 = 0; i0 < total; i0 += blockDim.x) {
    const int i = i0 + tid;
    Touched t{0, 0, -1, false};
    if (i < total) t = touched(p, m, i);
    need += block_scan(t.fresh, before, m.warps);
    if (i0 == 0) first = t, before0 = before;
  }
  const bool enough = need <= free;
  if (tid == 0) {
    if (!enough) report(p, ST_CAPACITY);
    counts[0] = enough ? need : 0;
    counts[1] = enough ? free - need : free;
    ws.ctl[C_JOBS] = enough ? need : 0;
  }
  if (b < p.batch) p.held_out[b] = enough && w.x <= w.y ? max(held, w.y + 1) : was;
  // the first `need` free pages
  int* const list = need <= 1024 ? m.list : ws.list;
  for (int c = 0; enough && c < chunks; ++c) {
    const int at = ws.count[c];
    if (at >= need) break;
    const unsigned bits = chunks == 1 ? free0 : Pages(p, c).free();
    block_scan(__popc(bits), before, m.warps);
    before += at;
#pragma unroll
    for (int k = 0; k < PER; ++k)
      if (bits >> k & 1) {
        if (before < need) list[before] = c * CHUNK + tid * PER + k;
        ++before;
      }
  }
  __syncthreads();
  int base = 0;
  for (int i0 = 0; i0 < total; i0 += blockDim.x) {
    const int i = i0 + tid;
    Touched t = first;
    int n = 0;
    before = before0;
    if (total > (int)blockDim.x) {   // several rounds: looked up again, before anything of this one is written
      t = Touched{0, 0, -1, false};
      if (i < total) t = touched(p, m, i);
      n = block_scan(t.fresh, before, m.warps);
    }
    if (i < total && !(t.fresh && enough)) {
      if (t.j < m.held[t.b]) p.table_out[t.b * p.out_stride + t.j] = t.old;
    } else if (i < total) {
      const int id = list[base + before];
      p.table_out[t.b * p.out_stride + t.j] = id;
      // the page of slot lens[b] is copied up to it; pages past it hold nothing
      ws.job[base + before] = make_int4(t.old, id, t.old >= 0 && t.j == m.first[t.b] ? lens[t.b] % p.page_size : 0, 0);
    }
    base += n;
  }
  __syncthreads();   // nobody reads the counts of holders any more, which may be refs_out
  for (int i = tid; enough && i < need; i += blockDim.x) {
    const int4 job = ws.job[i];
    if (job.x >= 0) atomicSub(p.refs_out + job.x, 1);
    atomicAdd(p.refs_out + job.y, 1);
  }
}

// ---------------------------------------------------------------- compact
// Lists of a chunk, from what is live before it, all in all and below that: the
// free pages below `live`, the live ones at or past it, and where the latter go
// by the former's places (-2 - j: the j-th of them).
__device__ __forceinline__ void compact_lists(const PoolView& p, const PoolMem& ws, int* where, const Pages& g, int before,
                                              int live, int below) {
  const unsigned bits = g.live();
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    if (k >= g.n) break;
    const int id = g.first + k;
    const bool on = bits >> k & 1;
    int to = on ? id : -1;
    if (on && id >= live) {
      ws.src[before - below] = id;
      to = -2 - (before - below);
    } else if (!on && id < live) {
      ws.list[id - before] = id;
    }
    where[id] = to;
    before += on;
  }
}
// One block: counts, and the lists besides.
__global__ void __launch_bounds__(1024) compact_one_kernel(const PoolView p, int* where, int* live_out, const PoolMem ws) {
  __shared__ int warps[32], s_below;
  pdl_launch();
  const Pages g(p, 0);
  int before;
  const int live = block_scan(__popc(g.live()), before, warps);
  // the thread that holds page `live` (or the first past the end) knows what is live below it
  if (live >= g.first && live < g.first + PER) s_below = before + __popc(g.live() & ((1u << (live - g.first)) - 1));
  if (live == CHUNK && threadIdx.x == 0) s_below = live;
  __syncthreads();
  compact_lists(p, ws, where, g, before, live, s_below);
  if (threadIdx.x == 0) ws.ctl[C_LIVE] = *live_out = live, ws.ctl[C_JOBS] = live - s_below;
}
__global__ void __launch_bounds__(1024) compact_count_kernel(const PoolView p, int* live_out, const PoolMem ws) {
  __shared__ int warps[32];
  const int chunks = (p.n_pages + CHUNK - 1) / CHUNK;
  pdl_launch();
  int before;
  for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
    const Pages g(p, c);
    const int n = block_scan(__popc(g.live()), before, warps);
    if (threadIdx.x == 0) ws.count[c] = n;
  }
  if (!last_block(ws.ctl + C_DONE, gridDim.x)) return;
  const int live = scan_chunks(ws.count, chunks, warps);
  int below = live;
  if (live < p.n_pages) {   // those below `live`: of the chunks before its own, and of its own
    const int c = live / CHUNK;
    const Pages g(p, c);
    const int left = max(0, min(PER, live - g.first));
    below = ws.count[c] + block_scan(__popc(g.live() & ((1u << left) - 1)), before, warps);
  }
  if (threadIdx.x == 0) ws.ctl[C_LIVE] = *live_out = live, ws.ctl[C_BELOW] = below, ws.ctl[C_JOBS] = live - below;
}
__global__ void __launch_bounds__(1024) compact_list_kernel(const PoolView p, int* where, const PoolMem ws) {
  __shared__ int warps[32];
  pdl_launch();
  pdl_wait();
  const int chunks = (p.n_pages + CHUNK - 1) / CHUNK, live = ws.ctl[C_LIVE], below = ws.ctl[C_BELOW];
  for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
    const Pages g(p, c);
    int before;
    block_scan(__popc(g.live()), before, warps);
    compact_lists(p, ws, where, g, ws.count[c] + before, live, below);
  }
}

// ------------------------------------------------------------------ copies
// A task is one head of an array's part in a page (some heads where they are
// small), up to the slots in use: what a page does not hold is neither read nor
// stepped over.  A warp takes a task, 8 units a lane at a time.
template <typename U>
__device__ __forceinline__ void copy_heads(const PlanArray& a, int head0, int src, int dst, int slots) {
  const int rows = min(a.rows, (slots + a.row_slots - 1) / a.row_slots), len = rows * (int)a.row_units.d, heads = min(a.together, a.heads - head0);
  const char* from = a.base + src * a.page_stride + head0 * a.head_stride;
  char* to = a.base + dst * a.page_stride + head0 * a.head_stride;
  const bool plain = heads == 1 && a.runs;
  for (int u0 = threadIdx.x & 31; u0 < heads * len; u0 += 256) {
    U x[8];
    long long off[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int u = u0 + k * 32;
      if (plain) {
        off[k] = (long long)u * (int)sizeof(U);
      } else {
        const int h = heads == 1 ? 0 : u / len, in = u - h * len, r = (int)a.row_units.div(in);
        off[k] = h * a.head_stride + r * a.row_stride + (in - r * (int)a.row_units.d) * (int)sizeof(U);
      }
      if (u < heads * len) x[k] = *reinterpret_cast<const U*>(from + off[k]);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (u0 + k * 32 < heads * len) *reinterpret_cast<U*>(to + off[k]) = x[k];
  }
}

// The array that holds a task: first_task rises from 0.
__device__ __forceinline__ int array_of(const PlanArray* arrays, int n, int task) {
  const int lane = threadIdx.x & 31;
  int lo = 0;
  if (n > 32) {
    const int step = (n + 31) >> 5, at = lane * step;
    lo = (__popc(__ballot_sync(0xffffffffu, at < n && __ldg(&arrays[at].first_task) <= task)) - 1) * step;
    n = min(n, lo + step);
  }
  return lo + __popc(__ballot_sync(0xffffffffu, lo + lane < n && __ldg(&arrays[min(lo + lane, n - 1)].first_task) <= task)) - 1;
}
// All tasks of all jobs; job(j): source, destination, slots.
template <typename F>
__device__ __forceinline__ void copy_jobs(const PlanHead* plan, int n_arrays, int jobs, F job) {
  const PlanArray* arrays = reinterpret_cast<const PlanArray*>(plan + 1);
  const PlanHead head = *plan;
  const long long tasks = (long long)jobs * head.tasks;
  for (long long t = (long long)blockIdx.x * 8 + threadIdx.x / 32; t < tasks; t += gridDim.x * 8ll) {
    const int j = (int)(t / head.tasks), task = (int)(t - (long long)j * head.tasks);
    const int3 now = job(j);
    if (now.z <= 0) continue;
    const PlanArray a = arrays[head.each ? task / head.each : array_of(arrays, n_arrays, task)];   // a copy: stores might alias it
    const int head0 = (task - a.first_task) * a.together;
    if (a.unit == 16) copy_heads<uint4>(a, head0, now.x, now.y, now.z);
    else copy_heads<uint32_t>(a, head0, now.x, now.y, now.z);
  }
}

__global__ void __launch_bounds__(256, 2) reserve_copy_kernel(const PlanHead* plan, int n_arrays, const PoolMem ws) {
  pdl_wait();
  copy_jobs(plan, n_arrays, ws.ctl[C_JOBS], [&](int j) {
    const int4 job = ws.job[j];
    return make_int3(job.x, job.y, job.z);
  });
}

// Copies, counts of holders, table entries and new ids.  The counts may be
// written in place: of a move one thread reads and writes both.
__global__ void __launch_bounds__(256, 2) compact_copy_kernel(const PoolView p, const PlanHead* plan, int n_arrays, int* where, const PoolMem ws) {
  pdl_wait();
  const int jobs = ws.ctl[C_JOBS], live = ws.ctl[C_LIVE];
  const int at = blockIdx.x * 256 + threadIdx.x, step = gridDim.x * 256;
  for (int i = at; i < p.n_pages; i += step) {
    const int r = p.refs[i];
    if (i >= live ? r <= 0 : r > 0) p.refs_out[i] = i < live ? r : 0;   // the others are a move's
  }
  for (int j = at; j < jobs; j += step) {
    const int src = ws.src[j], dst = ws.list[j], r = p.refs[src];
    p.refs_out[dst] = r;
    p.refs_out[src] = 0;
    where[src] = dst;
  }
  for (int b = blockIdx.x * 8 + threadIdx.x / 32; b < p.batch; b += gridDim.x * 8) {
    const int held = held_of(p, b);
    for (int j = threadIdx.x & 31; j < held; j += 32) {
      int id = p.table[b * p.table_stride + j];
      if (in_pool(p, id)) {
        id = __ldcg(where + id);   // a moved page's: as listed, or already its new id
        if (id < -1) id = ws.list[-2 - id];
      }
      p.table_out[b * p.out_stride + j] = id;
    }
  }
  if (!n_arrays) return;
  const int page = __ldg(&plan->page_size);
  copy_jobs(plan, n_arrays, jobs, [&](int j) { return make_int3(ws.src[j], ws.list[j], page); });
}

// ----------------------------------------------------------- host side
// table_out and refs_out may be their inputs themselves, with the same stride.
int pool_view(const asr_page_pool* c, bool with_held_out, PoolView* v) {
  if (!c || !c->page_table || !c->held || !c->refs || !c->table_out || !c->refs_out || (with_held_out && !c->held_out))
    return ASR_E_INVAL;
  if (c->batch < 1 || c->batch > PG_MAX_BATCH || c->n_pages < 1) return ASR_E_INVAL;
  if (c->n_pages > (1 << 30) || (long long)c->batch * c->max_pages > (1ll << 30)) return ASR_E_CAPACITY;   // 32-bit counts and steps
  if (c->page_size < PG_GROUP || c->page_size % PG_GROUP || c->page_size > (1 << 20)) return ASR_E_INVAL;
  if (c->max_pages < 1 || (long long)c->max_pages * c->page_size > (1ll << 30)) return ASR_E_INVAL;
  if (c->table_stride < c->max_pages || c->table_out_stride < c->max_pages) return ASR_E_INVAL;
  if (c->table_out == c->page_table && c->table_out_stride != c->table_stride) return ASR_E_INVAL;
  for (const void* x : {(const void*)c->page_table, (const void*)c->held, (const void*)c->refs, (const void*)c->table_out,
                        (const void*)c->held_out, (const void*)c->refs_out, (const void*)c->status})
    if ((uintptr_t)x % 4) return ASR_E_INVAL;
  *v = {c->page_table, c->table_stride, c->held, c->refs, c->table_out, c->table_out_stride, c->held_out, c->refs_out,
        c->n_pages, c->page_size, c->max_pages, c->batch, c->status};
  return ASR_OK;
}

int pool_args(const asr_page_pool* c, bool with_held_out, const void* plan, int n_arrays, void* ws, int64_t ws_bytes, PoolView* v,
              PoolMem* m) {
  if (int rc = pool_view(c, with_held_out, v)) return rc;
  if (n_arrays < 0 || n_arrays > MAX_ARRAYS || (n_arrays > 0 && !plan) || (uintptr_t)plan % 16) return ASR_E_INVAL;
  if (!ws || (uintptr_t)ws % 16) return ASR_E_INVAL;
  return ws_bytes < (int64_t)pool_mem(*v, ws, m) ? ASR_E_CAPACITY : ASR_OK;
}

unsigned chunk_blocks(const PoolView& p) {
  const int chunks = (p.n_pages + CHUNK - 1) / CHUNK, sms = paged_sm_count();
  return (unsigned)(chunks < sms ? chunks : sms);
}
// Blocks of 256 threads: a few rounds of the resident ones, no more than the work could fill.
unsigned copy_blocks(long long warps) {
  const long long most = 8ll * paged_sm_count(), want = (warps + 7) / 8;
  return (unsigned)(want < 1 ? 1 : want < most ? want : most);
}

}  // namespace
}  // namespace asrspec

using namespace asrspec;

extern "C" {

int64_t asr_spec_pool_plan_bytes(int32_t n) {
  if (n < 0 || n > MAX_ARRAYS) return ASR_E_INVAL;
  return (int64_t)(sizeof(PlanHead) + (size_t)n * sizeof(PlanArray));
}

int asr_spec_pool_plan(const asr_page_array* arrays, int32_t n, int32_t page_size, void* plan) {
  if (n < 0 || n > MAX_ARRAYS || (n && !arrays) || !plan || (uintptr_t)plan % 8) return ASR_E_INVAL;
  if (page_size < PG_GROUP || page_size % PG_GROUP || page_size > (1 << 20)) return ASR_E_INVAL;
  PlanHead head{n, 0, page_size, 0};
  PlanArray* out = reinterpret_cast<PlanArray*>(static_cast<PlanHead*>(plan) + 1);
  for (int i = 0; i < n; ++i) {
    const asr_page_array& a = arrays[i];
    if (!a.base || a.heads < 1 || a.rows < 1 || a.row_bytes < 4 || a.row_slots < 1) return ASR_E_INVAL;
    if ((long long)a.rows * a.row_slots != page_size) return ASR_E_INVAL;
    if (a.page_stride <= 0 || a.head_stride <= 0 || a.row_stride < a.row_bytes) return ASR_E_INVAL;
    for (int64_t s : {a.page_stride, a.head_stride, a.row_stride})
      if (s >= (1ll << 40)) return ASR_E_INVAL;
    const uint64_t all = (uint64_t)(uintptr_t)a.base | a.page_stride | a.head_stride | a.row_stride | (uint64_t)a.row_bytes;
    if (all % 4) return ASR_E_INVAL;
    const int unit = all % 16 ? 4 : 16;
    const long long per_head = (long long)a.rows * (a.row_bytes / unit);
    if (per_head * a.heads > 0x7fffffffll) return ASR_E_CAPACITY;
    PlanArray x{};
    x.base = static_cast<char*>(a.base);
    x.page_stride = a.page_stride, x.head_stride = a.head_stride, x.row_stride = a.row_stride;
    x.row_units = make_fastdiv(a.row_bytes / unit);
    x.heads = a.heads, x.rows = a.rows, x.row_slots = a.row_slots, x.unit = unit;
    x.runs = a.rows == 1 || a.row_stride == a.row_bytes;
    x.together = per_head >= PIECE ? 1 : (int)(PIECE / per_head);
    x.first_task = head.tasks;
    const int tasks = (a.heads + x.together - 1) / x.together;
    if ((long long)head.tasks + tasks > 0x7fffffffll) return ASR_E_CAPACITY;
    head.tasks += tasks;
    head.each = i == 0 || head.each == tasks ? tasks : -1;
    memcpy(out + i, &x, sizeof x);
  }
  if (head.each < 0) head.each = 0;
  memcpy(plan, &head, sizeof head);
  return ASR_OK;
}

int64_t asr_spec_pool_ws(const asr_page_pool* pool) {
  PoolView v;
  PoolMem m;
  if (int rc = pool_view(pool, false, &v)) return rc;
  return (int64_t)pool_mem(v, nullptr, &m);
}

int asr_spec_pool_reserve(const asr_page_pool* pool, const void* plan, int32_t n_arrays, const int32_t* lens,
                          const int32_t* rows, int32_t* counts, void* ws, int64_t ws_bytes, void* stream) {
  PoolView p;
  PoolMem m;
  if (int rc = pool_args(pool, true, plan, n_arrays, ws, ws_bytes, &p, &m)) return rc;
  if (!lens || !rows || !counts || ((uintptr_t)lens | (uintptr_t)rows | (uintptr_t)counts) % 4) return ASR_E_INVAL;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int counters = (int)chunk_blocks(p), copiers = p.table_out == p.table ? 0 : (p.batch + 31) / 32;
  cudaError_t e = launch_ex(reserve_kernel, dim3(counters + copiers), dim3(1024), sizeof(ReserveMem), st, false, 1, p, lens, rows, counts,
                            m, counters);
  if (e == cudaSuccess && n_arrays)   // a sequence has one page to copy at most; how many do is known on the device
    e = launch_ex(reserve_copy_kernel, dim3(copy_blocks((long long)p.batch * 1024)), dim3(256), 0, st, true, 1,
                  static_cast<const PlanHead*>(plan), (int)n_arrays, m);
  return e == cudaSuccess ? ASR_OK : ASR_E_CUDA;
}

int asr_spec_pool_fork(const asr_page_pool* pool, const int32_t* parent, const int32_t* keep, void* ws, int64_t ws_bytes,
                       void* stream) {
  PoolView p;
  PoolMem m;
  if (int rc = pool_args(pool, true, nullptr, 0, ws, ws_bytes, &p, &m)) return rc;
  if (((uintptr_t)parent | (uintptr_t)keep) % 4) return ASR_E_INVAL;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool in_place = p.table_out == p.table || p.held_out == p.held;
  const long long stage = in_place ? p.batch : 1, counts = p.refs_out == p.refs ? 1 : (p.n_pages + 255ll) / 256;
  const long long most = 8ll * paged_sm_count(), want = stage > counts ? stage : counts;
  cudaError_t e = launch_ex(fork_stage_kernel, dim3((unsigned)(want < most ? want : most)), dim3(256), 0, st, false, 1, p, parent, keep,
                            m, in_place);
  const int chunks = (p.max_pages + FORK_RUN - 1) / FORK_RUN;
  if (e == cudaSuccess)
    e = launch_ex(fork_kernel, dim3(p.batch, chunks < 64 ? chunks : 64), dim3(256), 0, st, true, 1, p, parent, keep, m, in_place);
  return e == cudaSuccess ? ASR_OK : ASR_E_CUDA;
}

int asr_spec_pool_compact(const asr_page_pool* pool, const void* plan, int32_t n_arrays, int32_t* where, int32_t* live,
                          void* ws, int64_t ws_bytes, void* stream) {
  PoolView p;
  PoolMem m;
  if (int rc = pool_args(pool, false, plan, n_arrays, ws, ws_bytes, &p, &m)) return rc;
  if (!where || !live || ((uintptr_t)where | (uintptr_t)live) % 4) return ASR_E_INVAL;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (p.n_pages <= CHUNK) {
    e = launch_ex(compact_one_kernel, dim3(1), dim3(1024), 0, st, false, 1, p, where, live, m);
  } else {
    e = launch_ex(compact_count_kernel, dim3(chunk_blocks(p)), dim3(1024), 0, st, false, 1, p, live, m);
    if (e == cudaSuccess) e = launch_ex(compact_list_kernel, dim3(chunk_blocks(p)), dim3(1024), 0, st, true, 1, p, where, m);
  }
  if (e == cudaSuccess)
    e = launch_ex(compact_copy_kernel, dim3(copy_blocks(n_arrays ? (long long)p.n_pages * 16 : p.n_pages / 32 + p.batch)), dim3(256), 0, st,
                  true, 1, p, static_cast<const PlanHead*>(plan), (int)n_arrays, where, m);
  return e == cudaSuccess ? ASR_OK : ASR_E_CUDA;
}

}  // extern "C"
