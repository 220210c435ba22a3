// Penalties for repeated tokens, biases and grammar masks on the logits of a
// block of rows.
//
//   x' = x > 0 ? x / repetition : x * repetition   (tokens seen),
//   x' - frequency c - presence (c > 0) + bias,  -inf where the mask says so
//
// with c the token's count after the prompt, the row's own drafts included.
// Bound by the logits, read and written once.  A block takes a run of the
// vocabulary and some or all rows of an utterance: it counts its part of the
// history in shared memory once, a thread keeps its tokens' counts and biases
// in registers and walks the rows, so the history is read by each run of the
// vocabulary instead of by each row, and between two rows only the draft that
// lies between them is looked at.
// Measured: 64 utterances, 1 to 7 rows of 51866 in fp32, histories of up to 448,
// bias and mask: 39 us for 176 MB, 4.5 TB/s (of 6.75 copied): what a block does before its
// first row is near half of its instructions, and 8 elements a thread, which halve
// that, leave fewer blocks to wait with (43 us); all first loads together
// 42 -> 39 us.  One utterance of 9 rows: 3.5 us.
#include "kernels.h"
#include "paged.cuh"

namespace asrspec {
namespace {

constexpr int THREADS = 256;

struct AdjustArgs {
  asr_logit_rules r;
  long long batch, row, out_batch, out_row;   // bytes
  int rows_each;                              // of a block
};

template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

template <int BYTES> struct Word;
template <> struct Word<2> { using type = uint16_t; };
template <> struct Word<4> { using type = uint32_t; };
template <> struct Word<8> { using type = uint2; };
template <> struct Word<16> { using type = uint4; };

// W elements an access, J accesses a thread and row: token base + (j * THREADS + thread) * W + w.
template <typename T, int W, int J>
__global__ void __launch_bounds__(THREADS, W * J >= 8 ? 4 : 6) adjust_kernel(const AdjustArgs a) {
  constexpr int RUN = THREADS * W * J;
  using Access = typename Word<W * sizeof(T)>::type;
  __shared__ int seen[RUN];   // 2 * count + (seen at all)
  const asr_logit_rules& r = a.r;
  const int tid = threadIdx.x, b = blockIdx.z, base = blockIdx.x * RUN;
  const bool reports = blockIdx.x == 0 && blockIdx.y == 0 && r.status;
  // All of the first loads go out together, before it is known how many tokens and rows there are to look at.
  const int n = r.lens ? __ldg(r.lens + b) : r.rows - 1, have = r.history_len ? __ldg(r.history_len + b) : r.history_max;
  const int prompt = r.prompt_len ? __ldg(r.prompt_len + b) : 0;
  const float rep = r.repetition ? __ldg(r.repetition + b) : r.repetition_all;
  const float freq = r.frequency ? __ldg(r.frequency + b) : r.frequency_all, pres = r.presence ? __ldg(r.presence + b) : r.presence_all;
  const int* history = r.history + b * r.history_stride;
  const int* draft = r.draft ? r.draft + (long long)b * (r.rows - 1) : nullptr;
  int early[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) early[i] = tid + i * THREADS < r.history_max ? __ldg(history + tid + i * THREADS) : 0;
  const int between = draft && tid < r.rows - 1 ? __ldg(draft + tid) : 0;
  const int row0 = blockIdx.y * a.rows_each;

  union Part {
    Access word;
    T x[W];
    __device__ Part() {}
  };
  // This thread's accesses: whole, beyond the end, or (one thread, where W does not divide the vocabulary) with a ragged one.
  const int tok0 = base + tid * W;
  bool whole[J], ragged = false;
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int tok = tok0 + j * THREADS * W;
    whole[j] = tok + W <= r.vocab;
    ragged |= W > 1 && tok < r.vocab && !whole[j];
  }
  const char* src = static_cast<const char*>(r.logits) + b * a.batch + row0 * a.row + tok0 * (long long)sizeof(T);
  char* dst = static_cast<char*>(r.out) + b * a.out_batch + row0 * a.out_row + tok0 * (long long)sizeof(T);
  const int* words = r.mask + (b * r.mask_batch_stride + row0 * r.mask_row_stride + tok0 / 32);   // 32 divides THREADS * W
  const int bit = tok0 % 32;
  // the next row is on its way while this one is worked on, the first two while the history is counted
  Part in[2][J];
  uint32_t allowed[2][J];
  auto load = [&](Part (&x)[J], uint32_t (&m)[J]) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      m[j] = r.mask && tok0 + j * THREADS * W < r.vocab ? (uint32_t)__ldg(words + j * (THREADS * W / 32)) >> bit : 0xffffffffu;
      if (whole[j]) x[j].word = *reinterpret_cast<const Access*>(src + j * (THREADS * W * (int)sizeof(T)));
    }
    if (ragged)
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int w = 0; w < W; ++w)
          if (!whole[j] && tok0 + j * THREADS * W + w < r.vocab) x[j].x[w] = reinterpret_cast<const T*>(src)[j * THREADS * W + w];
    src += a.row, words += r.mask_row_stride;
  };
  if (row0 < r.rows) load(in[0], allowed[0]);
  if (row0 + 1 < r.rows) load(in[1], allowed[1]);
  float bias[J][W];
#pragma unroll
  for (int j = 0; j < J; ++j)
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const int tok = base + (j * THREADS + tid) * W + w;
      bias[j][w] = r.bias && tok < r.vocab ? __ldg(r.bias + b * r.bias_stride + tok) : 0.f;
    }
  for (int i = tid; i < RUN; i += THREADS) seen[i] = 0;
  if (n < -1 || n >= r.rows || have < 0 || have > r.history_max || prompt < 0 || prompt > have) {
    if (reports && tid == 0) set_status(r.status, ST_BAD_LENS);
    return;
  }
  const int row1 = min(n + 1, row0 + a.rows_each);
  if (row0 >= row1 && !reports) return;
  __syncthreads();
  bool bad = false;
  auto note = [&](int tok, bool said) {
    bad |= (unsigned)tok >= (unsigned)r.vocab;
    const int at = tok - base;
    if ((unsigned)at >= (unsigned)RUN || tok >= r.vocab) return;
    atomicOr(seen + at, 1);
    if (said) atomicAdd(seen + at, 2);
  };
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (tid + i * THREADS < have) note(early[i], tid + i * THREADS >= prompt);
  for (int i = tid + 2 * THREADS; i < have; i += THREADS) note(__ldg(history + i), i >= prompt);
  if (draft && tid < (reports ? n : min(row0, n))) {
    if (tid < row0) note(between, true);
    bad |= (unsigned)between >= (unsigned)r.vocab;
  }
  if (reports && bad) set_status(r.status, ST_BAD_TOKEN);
  __syncthreads();
  if (row0 >= row1) return;
  int c[J][W];
#pragma unroll
  for (int j = 0; j < J; ++j)
#pragma unroll
    for (int w = 0; w < W; ++w) c[j][w] = seen[(j * THREADS + tid) * W + w];
  int any = 0;   // of this thread's tokens
#pragma unroll
  for (int j = 0; j < J; ++j)
#pragma unroll
    for (int w = 0; w < W; ++w) any |= c[j][w];
  auto work = [&](int row, Part (&x)[J], uint32_t (&m)[J]) {
    float v[J][W];
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int w = 0; w < W; ++w) v[j][w] = to_f32(x[j].x[w]);
    if (any)
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int w = 0; w < W; ++w)
          if (c[j][w]) {
            v[j][w] = v[j][w] > 0.f ? v[j][w] / rep : v[j][w] * rep;
            const int count = c[j][w] >> 1;
            if (count) v[j][w] = v[j][w] - freq * (float)count - pres;
          }
#pragma unroll
    for (int j = 0; j < J; ++j) {
#pragma unroll
      for (int w = 0; w < W; ++w) x[j].x[w] = from_f32<T>(m[j] >> w & 1 ? v[j][w] + bias[j][w] : -INFINITY);
      if (whole[j]) *reinterpret_cast<Access*>(dst + j * (THREADS * W * (int)sizeof(T))) = x[j].word;
    }
    if (ragged)
#pragma unroll
      for (int j = 0; j < J; ++j)
#pragma unroll
        for (int w = 0; w < W; ++w)
          if (!whole[j] && tok0 + j * THREADS * W + w < r.vocab) reinterpret_cast<T*>(dst)[j * THREADS * W + w] = x[j].x[w];
    dst += a.out_row;
    // the draft that the next row comes after
    if (draft && row + 1 < row1) {
      const int d = __ldg(draft + row);
      if ((unsigned)(d - base) < (unsigned)RUN && d < r.vocab)
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
          for (int w = 0; w < W; ++w)
            if (tok0 + j * THREADS * W + w == d) any = c[j][w] = (c[j][w] + 2) | 1;
    }
  };
  for (int row = row0; row < row1; row += 2) {
    work(row, in[0], allowed[0]);
    if (row + 1 >= row1) break;
    if (row + 2 < row1) load(in[0], allowed[0]);
    work(row + 1, in[1], allowed[1]);
    if (row + 3 < row1) load(in[1], allowed[1]);
  }
}

// Rows of an utterance are dealt to several blocks where there are few of them.
template <typename T, int W, int J>
cudaError_t launch_adjust(AdjustArgs& a, cudaStream_t st) {
  const int runs = (a.r.vocab + THREADS * W * J - 1) / (THREADS * W * J), rows = a.r.rows;
  const long long blocks = (long long)runs * a.r.batch, want = 4ll * paged_sm_count();
  int parts = (int)((want + blocks - 1) / blocks);
  if (parts > rows) parts = rows;
  a.rows_each = (rows + parts - 1) / parts;
  parts = (rows + a.rows_each - 1) / a.rows_each;
  adjust_kernel<T, W, J><<<dim3(runs, parts, a.r.batch), THREADS, 0, st>>>(a);
  return cudaGetLastError();
}

// Elements of an access by the rows' alignment; of a thread and row 4, or 8 of 16 bits
// where the call is large enough for every SM to have blocks all the same.
template <typename T, int W>
cudaError_t launch_width(AdjustArgs& a, cudaStream_t st) {
  const bool large = (long long)a.r.batch * a.r.rows * a.r.vocab >= 8ll * THREADS * 4 * paged_sm_count();
  if constexpr (sizeof(T) == 2) {
    if (W == 8 || large) return launch_adjust<T, W, 8 / W>(a, st);
  }
  if constexpr (W <= 4) return launch_adjust<T, W, 4 / W>(a, st);
  else return cudaErrorInvalidValue;   // 8 of 16 bits: above
}
template <typename T>
cudaError_t launch_type(AdjustArgs& a, cudaStream_t st) {
  const uintptr_t all = (uintptr_t)a.r.logits | (uintptr_t)a.r.out | a.batch | a.row | a.out_batch | a.out_row;
  const int most = 16 / (int)sizeof(T), w = all % 16 == 0 ? most : all % 8 == 0 ? most / 2 : all % 4 == 0 ? most / 4 : 1;
  if constexpr (sizeof(T) == 2)
    if (w == 8) return launch_width<T, 8>(a, st);
  return w == 4 ? launch_width<T, 4>(a, st) : w == 2 ? launch_width<T, 2>(a, st) : launch_width<T, 1>(a, st);
}

}  // namespace
}  // namespace asrspec

using namespace asrspec;

extern "C" int asr_spec_adjust_logits(const asr_logit_rules* r, void* stream) {
  if (!r || !r->logits || !r->out) return ASR_E_INVAL;
  if (r->batch < 1 || r->batch > 65535 || r->rows < 1 || r->rows > 32 || r->vocab < 1 || r->vocab > (1 << 30) || r->dtype < 0 || r->dtype > 2)
    return ASR_E_INVAL;
  const long long es = r->dtype == 0 ? 4 : 2;
  if (((uintptr_t)r->logits | (uintptr_t)r->out) % es) return ASR_E_INVAL;
  if (r->row_stride < r->vocab || r->out_row_stride < r->vocab || r->batch_stride < 0 || r->out_batch_stride < 0) return ASR_E_INVAL;
  if (r->batch > 1 && (r->batch_stride < r->vocab || r->out_batch_stride < r->vocab)) return ASR_E_INVAL;
  for (int64_t s : {r->batch_stride, r->row_stride, r->out_batch_stride, r->out_row_stride})
    if (s >= (1ll << 45)) return ASR_E_INVAL;
  if (r->out == r->logits && (r->out_batch_stride != r->batch_stride || r->out_row_stride != r->row_stride)) return ASR_E_INVAL;
  if (r->history_max < 0 || r->history_max > (1 << 30) || r->history_stride < r->history_max || (!r->history && r->history_max > 0)) return ASR_E_INVAL;
  if (r->bias_stride < 0 || r->mask_batch_stride < 0 || r->mask_row_stride < 0) return ASR_E_INVAL;
  for (const void* x : {(const void*)r->history, (const void*)r->history_len, (const void*)r->prompt_len, (const void*)r->draft,
                        (const void*)r->lens, (const void*)r->repetition, (const void*)r->frequency, (const void*)r->presence,
                        (const void*)r->bias, (const void*)r->mask, (const void*)r->status})
    if ((uintptr_t)x % 4) return ASR_E_INVAL;
  if (!(r->repetition_all > 0.f) || !(r->repetition_all <= 1e30f)) return ASR_E_INVAL;
  for (float x : {r->frequency_all, r->presence_all})
    if (!(x >= -1e30f && x <= 1e30f)) return ASR_E_INVAL;
  AdjustArgs a{*r, r->batch_stride * es, r->row_stride * es, r->out_batch_stride * es, r->out_row_stride * es, 0};
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = r->dtype == 0   ? launch_type<float>(a, st)
                        : r->dtype == 1 ? launch_type<__nv_bfloat16>(a, st)
                                        : launch_type<__half>(a, st);
  return e == cudaSuccess ? ASR_OK : ASR_E_CUDA;
}
