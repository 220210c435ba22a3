// Argument checks of the operators over a paged K/V cache (host).
#include <mutex>

#include "kernels.h"
#include "paged.cuh"

namespace asrspec {

int paged_sm_count() {
  constexpr int MAX_DEVICES = 64;
  static std::mutex mu;
  static int count[MAX_DEVICES] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= MAX_DEVICES) return 152;
  std::lock_guard<std::mutex> lock(mu);
  if (!count[dev] && cudaDeviceGetAttribute(&count[dev], cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    count[dev] = 152;
  return count[dev];
}

// 16-byte alignment of every address a kernel forms: bases and byte strides.
int paged_view(const asr_paged_cache* c, PagedView* v) {
  if (!c || !c->k_pages || !c->v_pages || !c->page_table) return ASR_E_INVAL;
  if (c->dtype < 0 || c->dtype > 2 || (c->head_dim != 64 && c->head_dim != 128)) return ASR_E_INVAL;
  if (c->batch < 1 || c->batch > PG_MAX_BATCH || c->kv_heads < 1 || c->kv_heads > 1024 || c->n_pages < 1)
    return ASR_E_INVAL;
  if (c->page_size < PG_GROUP || c->page_size % PG_GROUP || c->page_size > (1 << 20)) return ASR_E_INVAL;
  if (c->max_pages < 1 || (long long)c->max_pages * c->page_size > (1ll << 30)) return ASR_E_INVAL;
  if (c->table_stride < c->max_pages || (uintptr_t)c->page_table % 4 || (uintptr_t)c->status % 4) return ASR_E_INVAL;
  const long long es = c->dtype == 0 ? 4 : 2;
  if (((uintptr_t)c->k_pages | (uintptr_t)c->v_pages) % 16) return ASR_E_INVAL;
  if (c->page_stride < 0 || c->head_stride < 0 || c->slot_stride < 0 || (c->page_stride * es) % 16 ||
      (c->head_stride * es) % 16 || (c->slot_stride * es) % 16 || c->slot_stride < c->head_dim ||
      c->slot_stride * es > (1 << 26))   // 16 slots' offsets fit 32 bits
    return ASR_E_INVAL;
  v->k = static_cast<char*>(c->k_pages);
  v->v = static_cast<char*>(c->v_pages);
  v->page_stride = c->page_stride * es;
  v->head_stride = c->head_stride * es;
  v->slot_stride = c->slot_stride * es;
  v->table = c->page_table;
  v->table_stride = c->table_stride;
  v->n_pages = c->n_pages;
  v->page_size = c->page_size;
  v->max_slots = c->max_pages * c->page_size;
  v->kv_heads = c->kv_heads;
  v->batch = c->batch;
  v->groups = make_fastdiv(c->page_size / PG_GROUP);
  v->status = c->status;
  return ASR_OK;
}

int paged_rows(const asr_paged_cache* c, const asr_paged_rows* r, PagedRows* v) {
  if (!r || !r->q || !r->kv_len || (r->k_new == nullptr) != (r->v_new == nullptr)) return ASR_E_INVAL;
  if (r->max_rows < 1 || r->max_rows > 4096 || r->heads < 1 || r->heads > 4096 || r->heads % c->kv_heads)
    return ASR_E_INVAL;
  if (r->k_new && !r->causal) return ASR_E_INVAL;
  if (!(r->scale > 0.f) || r->scale > 1e30f) return ASR_E_INVAL;
  if (((uintptr_t)r->kv_len | (uintptr_t)r->rows) % 4) return ASR_E_INVAL;
  const long long es = c->dtype == 0 ? 4 : 2;
  const int64_t st[6] = {r->q_batch_stride, r->q_row_stride, r->q_head_stride,
                         r->new_batch_stride, r->new_row_stride, r->new_head_stride};
  for (int i = 0; i < (r->k_new ? 6 : 3); ++i)
    if (st[i] < 0 || (st[i] * es) % 16) return ASR_E_INVAL;
  if (r->k_new && r->new_row_stride * es > (1 << 26)) return ASR_E_INVAL;   // 16 rows' offsets fit 32 bits
  if (((uintptr_t)r->q | (uintptr_t)r->k_new | (uintptr_t)r->v_new) % 16) return ASR_E_INVAL;
  v->q = static_cast<const char*>(r->q);
  v->q_b = r->q_batch_stride * es;
  v->q_r = r->q_row_stride * es;
  v->q_h = r->q_head_stride * es;
  v->k_new = static_cast<const char*>(r->k_new);
  v->v_new = static_cast<const char*>(r->v_new);
  v->n_b = r->new_batch_stride * es;
  v->n_r = r->new_row_stride * es;
  v->n_h = r->new_head_stride * es;
  v->kv_len = r->kv_len;
  v->rows = r->rows;
  v->max_rows = r->max_rows;
  v->heads = r->heads;
  v->group = r->heads / c->kv_heads;
  v->groups = make_fastdiv(v->group);
  v->causal = r->causal != 0;
  v->scale = r->scale;
  return ASR_OK;
}

}  // namespace asrspec
