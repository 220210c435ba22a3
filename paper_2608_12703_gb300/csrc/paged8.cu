// The append to an 8-bit paged cache, and the argument checks of its operators.
//
//   a group of 16 slots and a head:  s = max(2^e, the group's own scale where it goes on),
//   e the least with |x| <= 448 2^e for the new rows' values;  code = rn(x / s)
//
// A warp takes one (sequence, K/V head, group), of K or of V.  Scales are
// powers of two: e4m3 has the same relative precision over its whole range, so nothing
// is lost against a scale of max / 448, the division is exact, and a group
// whose scale grows keeps its codes' values but for those that leave the type's
// normal range (below 2^-6 of the new scale).
// Measured: 4 x 2048 rows of 20 heads of 64, bf16: 19 us for 63 MB (9.3 at the
// copy rate), four waves of warps that wait for their rows once each (K and V by one warp: as long);
// rows of a decode step 2.5 to 5 us, latency.
#include "kernels.h"
#include "paged8.cuh"

namespace asrspec {
namespace {

// The bits of the least power of two, 2^-126 at least, by which amax divided is at most 448 = 1.75 * 2^8.
__device__ __forceinline__ float scale_for(float amax) {
  const int bits = __float_as_int(amax), e = (bits >> 23) - 8 + ((bits & 0x7fffff) > 0x600000);
  return __int_as_float(max(e, 1) << 23);
}

// 8 elements as they come, and as floats.
template <typename T> struct Eight {
  uint4 v[sizeof(T) / 2];
  __device__ __forceinline__ void load(const char* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) v[i] = __ldg(reinterpret_cast<const uint4*>(p) + i);
  }
  __device__ __forceinline__ float at(int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(reg_of(v[i / 4], i % 4));
    else {
      const uint16_t h = (uint16_t)(reg_of(v[0], i / 2) >> (i % 2 * 16));
      return to_f32(*reinterpret_cast<const T*>(&h));
    }
  }
};

// Lanes take 8 elements of a row: rows of a group in passes of 32 / (D / 8).
// Bound by HBM (new rows read, a quarter to half as many bytes of codes
// written) for prompts, by the chain lengths -> rows -> maximum -> codes for
// few rows; the rows' loads do not wait for the page's id.
template <typename T, int D>
__global__ void __launch_bounds__(256) append8_kernel(const Paged8View p, const PagedRows r, int max_groups, int tasks) {
  constexpr int CH = D / 8, AT_ONCE = 32 / CH, PASSES = PG_GROUP / AT_ONCE;
  pdl_launch();
  const int task = blockIdx.x * 8 + threadIdx.x / 32, lane = threadIdx.x & 31;
  if (task >= tasks) return;
  const bool is_v = task & 1;
  const int kvh = (task >> 1) % p.c.kv_heads, t2 = (task >> 1) / p.c.kv_heads, b = t2 / max_groups;
  int len, rows;
  paged_lens(p.c, r, b, len, rows);
  const int grp = len / PG_GROUP + t2 % max_groups, slot0 = grp * PG_GROUP;
  if (rows == 0 || slot0 >= len + rows) return;
  const int pid = __ldg(p.c.table + b * p.c.table_stride + p.c.groups.div((uint32_t)grp));
  const char* src = (is_v ? r.v_new : r.k_new) + b * r.n_b + kvh * r.n_h + lane % CH * (8 * (int)sizeof(T));
  Eight<T> x[PASSES];
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int row = slot0 + i * AT_ONCE + lane / CH - len;
    if (row >= 0 && row < rows) x[i].load(src + row * r.n_r);
  }
  if ((unsigned)pid >= (unsigned)p.c.n_pages) {
    if (p.c.status && lane == 0) set_status(p.c.status, ST_BOUNDS);
    return;
  }
  float* scale_at = (is_v ? p.v_scale : p.k_scale) + p.scale_at(pid, kvh, grp);
  const float own = slot0 < len ? *scale_at : 0.f;
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int row = slot0 + i * AT_ONCE + lane / CH - len;
    if (row < 0 || row >= rows) continue;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float a = fabsf(x[i].at(j));
      if (a <= 3.4028235e38f) amax = fmaxf(amax, a);
    }
  }
  const float s = fmaxf(scale_for(warp_max(amax)), own);
  const bool anew = slot0 < len && s != own;
  // powers of two from 2^-126 to 2^126 have an exact inverse; any other scale came from elsewhere
  const bool exact = (__float_as_int(s) & 0x807fffff) == 0 && s <= 8.507059173e37f;
  const float inv = exact ? __int_as_float((254 << 23) - __float_as_int(s)) : 1.f;
  char* codes = (is_v ? p.c.v : p.c.k) + paged_offset(p.c, pid, grp) + kvh * p.c.head_stride + lane % CH * 8;
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int at = i * AT_ONCE + lane / CH, row = slot0 + at - len;
    if (row >= rows || (row < 0 && !anew)) continue;
    uint2* to = reinterpret_cast<uint2*>(codes + at * p.c.slot_stride);
    float y[8];
    if (row < 0) {
      const uint2 c = *to;
      const uint32_t w[2] = {c.x, c.y};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float2 v = e4m3x2_value(w[j / 2] >> (j % 2 * 16));
        y[2 * j] = v.x * own;
        y[2 * j + 1] = v.y * own;
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        y[j] = x[i].at(j);
        if (!(fabsf(y[j]) <= 3.4028235e38f)) y[j] = __int_as_float(0x7fffffff);
      }
    }
    uint32_t c[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) c[j] = e4m3x2(y[2 * j] * inv, y[2 * j + 1] * inv);
    if (!exact)
#pragma unroll
      for (int j = 0; j < 4; ++j) c[j] = e4m3x2(y[2 * j] / s, y[2 * j + 1] / s);
    *to = make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
  }
  __syncwarp();   // every lane has read the group's own scale
  if (lane == 0 && s != own) *scale_at = s;
}

template <typename T>
cudaError_t launch_append_t(const Paged8View& c, const PagedRows& r, cudaStream_t st) {
  const int max_groups = (r.max_rows + PG_GROUP - 2) / PG_GROUP + 1;
  const long long tasks = 2ll * c.c.batch * max_groups * c.c.kv_heads;
  if (tasks > 0x7fffffffll - 8) return cudaErrorInvalidValue;
  const unsigned grid = (unsigned)((tasks + 7) / 8);
  return c.dim == 64 ? launch_ex(append8_kernel<T, 64>, dim3(grid), dim3(256), 0, st, false, 1, c, r, max_groups, (int)tasks)
                     : launch_ex(append8_kernel<T, 128>, dim3(grid), dim3(256), 0, st, false, 1, c, r, max_groups, (int)tasks);
}

}  // namespace

cudaError_t launch_append8(const Paged8View& c, const PagedRows& r, int dtype, cudaStream_t st) {
  if (dtype == 0) return launch_append_t<float>(c, r, st);
  return dtype == 1 ? launch_append_t<__nv_bfloat16>(c, r, st) : launch_append_t<__half>(c, r, st);
}

// The checks of paged_view, for elements of one byte.
int paged8_view(const asr_paged8_cache* c, Paged8View* v) {
  if (!c || !c->k_pages || !c->v_pages || !c->k_scale || !c->v_scale || !c->page_table) return ASR_E_INVAL;
  if (c->head_dim != 64 && c->head_dim != 128) return ASR_E_INVAL;
  if (c->batch < 1 || c->batch > PG_MAX_BATCH || c->kv_heads < 1 || c->kv_heads > 1024 || c->n_pages < 1)
    return ASR_E_INVAL;
  if (c->page_size < PG_GROUP || c->page_size % PG_GROUP || c->page_size > (1 << 20)) return ASR_E_INVAL;
  if (c->max_pages < 1 || (long long)c->max_pages * c->page_size > (1ll << 30)) return ASR_E_INVAL;
  if (c->table_stride < c->max_pages || (uintptr_t)c->page_table % 4 || (uintptr_t)c->status % 4) return ASR_E_INVAL;
  if (((uintptr_t)c->k_pages | (uintptr_t)c->v_pages) % 16 || ((uintptr_t)c->k_scale | (uintptr_t)c->v_scale) % 4)
    return ASR_E_INVAL;
  for (int64_t s : {c->page_stride, c->head_stride, c->slot_stride})
    if (s <= 0 || s % 16 || s >= (1ll << 40)) return ASR_E_INVAL;
  if (c->slot_stride < c->head_dim || c->slot_stride > (1 << 26)) return ASR_E_INVAL;   // 16 slots' offsets fit 32 bits
  for (int64_t s : {c->scale_page_stride, c->scale_head_stride})
    if (s < 0 || s >= (1ll << 40)) return ASR_E_INVAL;
  v->c.k = static_cast<char*>(c->k_pages);
  v->c.v = static_cast<char*>(c->v_pages);
  v->c.page_stride = c->page_stride;
  v->c.head_stride = c->head_stride;
  v->c.slot_stride = c->slot_stride;
  v->c.table = c->page_table;
  v->c.table_stride = c->table_stride;
  v->c.n_pages = c->n_pages;
  v->c.page_size = c->page_size;
  v->c.max_slots = c->max_pages * c->page_size;
  v->c.kv_heads = c->kv_heads;
  v->c.batch = c->batch;
  v->c.groups = make_fastdiv(c->page_size / PG_GROUP);
  v->c.status = c->status;
  v->k_scale = c->k_scale;
  v->v_scale = c->v_scale;
  v->s_page = c->scale_page_stride;
  v->s_head = c->scale_head_stride;
  v->dim = c->head_dim;
  return ASR_OK;
}

// Whether an element of one array of scales is `apart` elements behind another one of the same array, other than itself:
//   dp s_page + dh s_head + dg = apart,  |dp| < n_pages, |dh| < kv_heads, |dg| < groups of a page.
// For each dh only the multiples of s_page next to what is left can come near enough.
static bool scales_meet(const asr_paged8_cache* c, long long apart) {
  using Wide = __int128;
  const Wide groups = c->page_size / PG_GROUP, most = c->n_pages - 1, sp = most ? c->scale_page_stride : 0;
  const Wide sh = c->kv_heads > 1 ? c->scale_head_stride : 0;
  if (apart == 0 && most && sp < groups) return true;   // dh = 0: of one head's scales those of two pages
  for (int dh = apart ? 1 - c->kv_heads : 1; dh < c->kv_heads; ++dh) {
    const Wide left = apart - dh * sh;
    Wide at = sp ? left / sp : 0;   // rounded towards 0
    for (Wide dp : {at - 1, at, at + 1}) {
      dp = dp < -most ? -most : dp > most ? most : dp;
      const Wide off = left - dp * sp;
      if (off < groups && -off < groups) return true;
    }
  }
  return false;
}

// An append writes scales and codes by (page, head, group), each by a warp of its own: none may share memory with another's.
// Caches whose scales do (one scale broadcast over pages or heads, K's and V's in one array) can only be read.
int paged8_writable(const asr_paged8_cache* c) {
  if (c->k_pages == c->v_pages) return ASR_E_INVAL;
  const long long apart = (long long)((intptr_t)c->v_scale - (intptr_t)c->k_scale) / 4, groups = c->page_size / PG_GROUP;
  const __int128 head = c->kv_heads > 1 ? (__int128)(c->kv_heads - 1) * c->scale_head_stride + groups : groups;
  const __int128 all = c->n_pages > 1 ? (__int128)(c->n_pages - 1) * c->scale_page_stride + head : head;
  const bool nested = (c->kv_heads == 1 || c->scale_head_stride >= groups) && (c->n_pages == 1 || c->scale_page_stride >= head);
  if (nested && (apart >= all || -apart >= all)) return ASR_OK;   // as most caches are
  return apart == 0 || scales_meet(c, 0) || scales_meet(c, apart) ? ASR_E_INVAL : ASR_OK;
}

// paged_rows of a cache of the rows' type.
int paged8_rows(const asr_paged8_cache* c, const asr_paged_rows* r, int dtype, PagedRows* v) {
  if (dtype < 0 || dtype > 2) return ASR_E_INVAL;
  asr_paged_cache like{};
  like.kv_heads = c->kv_heads;
  like.dtype = dtype;
  return paged_rows(&like, r, v);
}

}  // namespace asrspec

using namespace asrspec;

extern "C" int asr_spec_paged8_append(const asr_paged8_cache* c, const asr_paged_rows* r, int32_t dtype, void* stream) {
  Paged8View v;
  PagedRows w;
  if (int rc = paged8_view(c, &v)) return rc;
  if (!r || !r->k_new || !r->v_new) return ASR_E_INVAL;
  if (int rc = paged8_writable(c)) return rc;
  asr_paged_rows rows = *r;   // the queries are not looked at: the new rows stand in for them
  rows.q = r->k_new;
  rows.q_batch_stride = rows.q_row_stride = rows.q_head_stride = 0;
  rows.heads = c->kv_heads;
  rows.causal = 1;
  rows.scale = 1.f;
  if (int rc = paged8_rows(c, &rows, dtype, &w)) return rc;
  return launch_append8(v, w, dtype, static_cast<cudaStream_t>(stream)) == cudaSuccess ? ASR_OK : ASR_E_CUDA;
}
