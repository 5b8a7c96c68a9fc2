// Entry points of the operators on paged caches and of the log probabilities: argument checks, then the launchers.
#include <algorithm>

#include "api_checks.cuh"
#include "paged.cuh"

using namespace lazy;

namespace {

constexpr int MAX_ROWS = 1 << 30;
constexpr long long MAX_COLUMNS = 1 << 30;  // rows of a sequence times query heads of a key/value head

// The pages as the kernels take them.
int take_pages(const lazy_pages *p, int dtype, PagedKV &kv) {
  if (!p || p->n_pages < 0 || p->page_size < 1 || p->table_pages < 0 || p->ld_table < p->table_pages) return LAZY_E_BADARG;
  if (p->page_stride < 0 || p->slot_stride < 0 || p->head_stride < 0) return LAZY_E_BADARG;
  if (!p->table || !p->len || !p->k || !p->v) return LAZY_E_BADARG;
  if (!co_rows_ok(p->k, p->page_stride, dtype) || !co_rows_ok(p->v, p->slot_stride, dtype) || !co_rows_ok(p->v, p->head_stride, dtype))
    return LAZY_E_BADARG;
  kv = {p->k, p->v, p->page_stride, p->slot_stride, p->head_stride, p->table, p->len, p->n_pages, p->page_size, p->table_pages, p->ld_table};
  return LAZY_OK;
}

}  // namespace

extern "C" {

int lazy_k_rope_table(void *stream, float *table, int32_t max_pos, int32_t head_dim, float theta) {
  if (max_pos < 0 || head_dim < 2 || head_dim % 2 || !(theta > 0.f)) return LAZY_E_BADARG;
  if ((long long)max_pos * (head_dim / 2) > 0x7fffff00LL) return LAZY_E_CAPACITY;
  if (max_pos == 0) return LAZY_OK;
  if (!table || ((uintptr_t)table & 7)) return LAZY_E_BADARG;
  return launch_rope_table((cudaStream_t)stream, table, max_pos, head_dim, theta);
}

int lazy_k_paged_append(void *stream, int32_t dtype, const void *q, int32_t ldq, const void *k, const void *v, int32_t ldkv,
                        const int32_t *pos, const float *rope_table, int32_t max_pos, const void *g_q, const void *g_k,
                        float eps, const int32_t *d_cu_q, int32_t n_rows, int32_t n_seqs, const lazy_pages *pages,
                        int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, void *q_out, int32_t ldq_out, void *k_out,
                        int32_t ldk_out) {
  if (bad_dtype(dtype) || n_rows < 0 || n_seqs < 0 || max_pos < 0 || !(eps >= 0.f)) return LAZY_E_BADARG;
  LAZY_TRY(check_heads(n_heads, n_kv_heads, head_dim));
  if (n_rows > MAX_ROWS || n_seqs > MAX_ROWS) return LAZY_E_CAPACITY;
  if (n_rows == 0) return LAZY_OK;
  if (n_seqs == 0 || (!d_cu_q && n_rows != n_seqs)) return LAZY_E_BADARG;
  const long long wq = (long long)n_heads * head_dim, wk = (long long)n_kv_heads * head_dim;
  if (bad_rows(q, ldq, wq, dtype) || bad_rows(k, ldkv, wk, dtype) || bad_rows(v, ldkv, wk, dtype) || bad_rows(q_out, ldq_out, wq, dtype) ||
      (k_out && bad_rows(k_out, ldk_out, wk, dtype)) || !pos || !rope_table || ((uintptr_t)rope_table & 15) || ((uintptr_t)g_q & 15) ||
      ((uintptr_t)g_k & 15))
    return LAZY_E_BADARG;
  AppendArgs a = {q, k, v, ldq, ldkv, pos, rope_table, max_pos, g_q, g_k, eps, d_cu_q, n_rows, n_seqs, {}, 0, n_heads, n_kv_heads,
                  head_dim, q_out, k_out, ldq_out, ldk_out};
  LAZY_TRY(take_pages(pages, dtype, a.kv));
  a.max_len = paged_capacity(a.kv);
  DevStatus *status = dev_status_ptr();
  if (!status) return LAZY_E_CUDA;
  return launch_paged_append((cudaStream_t)stream, dtype, a, status);
}

size_t lazy_k_attention_paged_scratch_floats(int32_t n_rows, int32_t n_seqs, int32_t max_q, int32_t max_kv, int32_t n_heads,
                                             int32_t n_kv_heads, int32_t head_dim) {
  if (n_rows < 0 || n_seqs < 0 || max_q < 0 || max_kv < 0 || check_heads(n_heads, n_kv_heads, head_dim) != LAZY_OK) return 0;
  // bounds may be any numbers: no call has more rows or sequences
  n_rows = std::min(n_rows, MAX_GRID_YZ);
  n_seqs = std::min(n_seqs, MAX_GRID_YZ);
  return attention_paged_scratch_floats(n_rows, n_seqs, max_q, max_kv, n_heads, n_kv_heads, head_dim);
}

int lazy_k_attention_paged(void *stream, int32_t dtype, const void *q, int32_t ldq, const int32_t *d_cu_q, int32_t n_rows,
                           int32_t n_seqs, int32_t max_q, const lazy_pages *pages, int32_t max_kv, int32_t n_heads,
                           int32_t n_kv_heads, int32_t head_dim, float *scratch, size_t scratch_floats, void *o) {
  if (bad_dtype(dtype) || n_rows < 0 || n_seqs < 0 || max_q < 0 || max_kv < 0) return LAZY_E_BADARG;
  LAZY_TRY(check_heads(n_heads, n_kv_heads, head_dim));
  if (n_rows > MAX_GRID_YZ || n_seqs > MAX_GRID_YZ) return LAZY_E_CAPACITY;
  if (n_rows == 0) return LAZY_OK;
  if (n_seqs == 0 || max_q == 0 || (!d_cu_q && n_rows != n_seqs)) return LAZY_E_BADARG;
  if (bad_rows(q, ldq, (long long)n_heads * head_dim, dtype) || !scratch || !o || ((uintptr_t)o & 15)) return LAZY_E_BADARG;
  PagedArgs a = {q, ldq, d_cu_q, n_rows, n_seqs, max_q, {}, max_kv, n_heads, n_kv_heads, head_dim, o};
  LAZY_TRY(take_pages(pages, dtype, a.kv));
  const int most = paged_capacity(a.kv);
  if (a.max_kv > most) a.max_kv = most;
  if (a.max_q > n_rows) a.max_q = n_rows;
  if ((long long)a.max_q * (n_heads / n_kv_heads) > MAX_COLUMNS) return LAZY_E_CAPACITY;
  if (scratch_floats < attention_paged_scratch_need(dtype, n_rows, n_seqs, a.max_q, a.max_kv, n_heads, n_kv_heads, head_dim))
    return LAZY_E_CAPACITY;
  DevStatus *status = dev_status_ptr();
  if (!status) return LAZY_E_CUDA;
  return launch_attention_paged((cudaStream_t)stream, dtype, a, scratch, status);
}

int lazy_k_token_logprobs(void *stream, int32_t dtype, const void *logits, int64_t ld, const int32_t *tokens, int32_t n_rows,
                          int32_t vocab, int32_t n_top, float *logprob, float *entropy, int32_t *rank, int32_t *top_id,
                          float *top_logprob) {
  if (bad_dtype(dtype) || n_rows < 0 || vocab < 1 || ld < vocab || n_top < 0 || n_top > LAZY_MAX_TOP || n_top > vocab) return LAZY_E_BADARG;
  if (vocab > (1 << 30) || n_rows > MAX_ROWS) return LAZY_E_CAPACITY;
  if (n_rows == 0) return LAZY_OK;
  if (!logits || ((uintptr_t)logits & (dtype == LAZY_F32 ? 3 : 1)) || (n_top > 0 && (!top_id || !top_logprob))) return LAZY_E_BADARG;
  if (!tokens && (logprob || rank)) return LAZY_E_BADARG;
  DevStatus *status = dev_status_ptr();
  if (!status) return LAZY_E_CUDA;
  const LogprobArgs a = {logits, ld, tokens, n_rows, vocab, n_top, logprob, entropy, rank, top_id, top_logprob};
  return launch_token_logprobs((cudaStream_t)stream, dtype, a, status);
}

}  // extern "C"
