// Entry points of the operators on bounded and shared caches: argument checks, then the launchers.
#include "api_checks.cuh"

using namespace lazy;

namespace {

constexpr long long MAX_KEYS = 0x7fffff00LL;  // that a row of the shared prefix's attention sees

}  // namespace

extern "C" {

size_t lazy_k_attention_mass_scratch_floats(int32_t n_seqs, int32_t n_total, int32_t max_len, int32_t n_heads,
                                            int32_t n_kv_heads, int32_t window) {
  if (n_seqs < 0 || n_total < 0 || max_len < 0 || n_heads < 1 || n_kv_heads < 0 || window < 0) return 0;
  if (n_kv_heads == 0) n_kv_heads = n_heads;
  if (n_heads % n_kv_heads) return 0;
  return attention_mass_scratch_floats(n_seqs, n_total, max_len, n_heads, n_kv_heads, window);
}

int lazy_k_attention_mass(void *stream, int32_t dtype, const void *q, int32_t ldq, const void *k, int32_t ldkv,
                          const int32_t *d_cu_seqlens, int32_t n_seqs, int32_t max_len, int32_t n_total,
                          int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t window, float *scratch,
                          size_t scratch_floats, float *mass) {
  if (bad_dtype(dtype) || n_seqs < 0 || max_len < 0 || n_total < 0 || window < 0) return LAZY_E_BADARG;
  LAZY_TRY(check_heads(n_heads, n_kv_heads, head_dim));
  if (n_seqs > MAX_GRID_YZ) return LAZY_E_CAPACITY;
  if (n_seqs == 0 || n_total == 0) return LAZY_OK;
  if (max_len < 1) return LAZY_E_BADARG;
  if (bad_rows(q, ldq, (long long)n_heads * head_dim, dtype) || bad_rows(k, ldkv, (long long)n_kv_heads * head_dim, dtype) ||
      !d_cu_seqlens || !scratch || !mass)
    return LAZY_E_BADARG;
  if (scratch_floats < attention_mass_scratch_need(n_seqs, n_total, max_len, n_heads, n_kv_heads, window))
    return LAZY_E_CAPACITY;
  DevStatus *status = dev_status_ptr();
  if (!status) return LAZY_E_CUDA;
  return launch_attention_mass((cudaStream_t)stream, dtype, q, ldq, k, ldkv, d_cu_seqlens, n_seqs, max_len, n_total,
                               n_heads, n_kv_heads, head_dim, window, scratch, mass, status);
}

size_t lazy_k_evict_scratch_ints(int32_t n_seqs, int32_t n_kv_heads, int32_t budget) {
  if (n_seqs < 0 || n_kv_heads < 1 || budget < 1) return 0;
  return evict_scratch_ints(n_seqs, n_kv_heads, budget);
}

int lazy_k_evict(void *stream, int32_t dtype, const void *k, const void *v, int32_t ldkv, const int32_t *pos,
                 const float *mass, const int32_t *d_cu_seqlens, int32_t n_seqs, int32_t max_len, int32_t n_total,
                 int32_t n_kv_heads, int32_t head_dim, int32_t budget, int32_t n_recent, int32_t *scratch,
                 size_t scratch_ints, void *kc, void *vc, float *cmass, int32_t *cpos, int32_t *clen, int32_t cap) {
  if (bad_dtype(dtype) || n_seqs < 0 || max_len < 0 || n_total < 0 || budget < 1 || n_recent < 0 ||
      n_recent > budget || cap < budget)
    return LAZY_E_BADARG;
  LAZY_TRY(check_heads(n_kv_heads, n_kv_heads, head_dim));
  if (n_seqs > MAX_GRID_YZ) return LAZY_E_CAPACITY;
  if (n_seqs == 0) return LAZY_OK;
  const long long width = (long long)n_kv_heads * head_dim;
  if (!d_cu_seqlens || !scratch || !clen) return LAZY_E_BADARG;
  if (n_total > 0 && (max_len < 1 || bad_rows(k, ldkv, width, dtype) || bad_rows(v, ldkv, width, dtype) ||
                      bad_rows(kc, width, width, dtype) || bad_rows(vc, width, width, dtype) || !pos || !mass || !cmass ||
                      !cpos))
    return LAZY_E_BADARG;
  if (scratch_ints < evict_scratch_ints(n_seqs, n_kv_heads, budget)) return LAZY_E_CAPACITY;
  DevStatus *status = dev_status_ptr();
  if (!status) return LAZY_E_CUDA;
  return launch_evict((cudaStream_t)stream, dtype, k, v, ldkv, pos, mass, d_cu_seqlens, n_seqs, max_len, n_total,
                      n_kv_heads, head_dim, budget, n_recent, scratch, kc, vc, cmass, cpos, clen, cap, status);
}

size_t lazy_k_evict_step_scratch_floats(int32_t n_seqs, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                                        int32_t budget) {
  if (n_seqs < 0 || budget < 1 || check_heads(n_heads, n_kv_heads, head_dim) != LAZY_OK) return 0;
  return evict_step_scratch_floats(n_seqs, n_heads, n_kv_heads, head_dim, budget);
}

int lazy_k_evict_step(void *stream, int32_t dtype, const void *q, int32_t ldq, const void *k_new, const void *v_new,
                      int32_t ld_new, const int32_t *pos_new, void *kc, void *vc, int32_t cap, const float *mass_in,
                      float *mass_out, const int32_t *pos_in, int32_t *pos_out, const int32_t *len_in,
                      int32_t *len_out, int32_t n_seqs, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                      int32_t budget, int32_t n_recent, float *scratch, size_t scratch_floats, void *o, int32_t *slot,
                      int32_t *gone) {
  if (bad_dtype(dtype) || n_seqs < 0 || budget < 1 || n_recent < 0 || n_recent >= budget || cap < budget)
    return LAZY_E_BADARG;
  LAZY_TRY(check_heads(n_heads, n_kv_heads, head_dim));
  if (n_seqs > MAX_GRID_YZ) return LAZY_E_CAPACITY;
  if (n_seqs == 0) return LAZY_OK;
  const long long width = (long long)n_kv_heads * head_dim;
  if (bad_rows(q, ldq, (long long)n_heads * head_dim, dtype) || bad_rows(k_new, ld_new, width, dtype) ||
      bad_rows(v_new, ld_new, width, dtype) || bad_rows(kc, width, width, dtype) || bad_rows(vc, width, width, dtype) ||
      !pos_new || !mass_in || !mass_out || !pos_in || !pos_out || !len_in || !len_out || !scratch || !o ||
      ((uintptr_t)o & 15) || !slot || !gone)
    return LAZY_E_BADARG;
  if (scratch_floats < evict_step_scratch_need(n_seqs, n_heads, n_kv_heads, head_dim, budget)) return LAZY_E_CAPACITY;
  DevStatus *status = dev_status_ptr();
  if (!status) return LAZY_E_CUDA;
  const EvictStepArgs a = {q, k_new, v_new, ldq, ld_new, pos_new, kc, vc, cap, mass_in, mass_out, pos_in, pos_out, len_in,
                           len_out, n_seqs, n_heads, n_kv_heads, head_dim, budget, n_recent, o, slot, gone};
  return launch_evict_step((cudaStream_t)stream, dtype, a, scratch, status);
}

size_t lazy_k_attention_prefix_scratch_floats(int32_t n_rows, int32_t n_seqs, int32_t max_q, int32_t n_pre,
                                              int32_t max_kv, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim) {
  if (n_rows < 0 || n_seqs < 0 || max_q < 0 || n_pre < 0 || max_kv < 0 || (long long)n_pre + max_kv > MAX_KEYS ||
      check_heads(n_heads, n_kv_heads, head_dim) != LAZY_OK)
    return 0;
  return attention_prefix_scratch_floats(n_rows, n_seqs, max_q, n_pre, max_kv, n_heads, n_kv_heads, head_dim);
}

int lazy_k_attention_prefix(void *stream, int32_t dtype, const void *q, int32_t ldq, const int32_t *d_cu_q,
                            int32_t n_rows, int32_t n_seqs, int32_t max_q, const void *k_pre, const void *v_pre,
                            int32_t ld_pre, int32_t n_pre, const void *k, const void *v, int32_t ldkv, int32_t kv_rows,
                            const int32_t *kv_idx, const int32_t *d_cu_kv, int32_t n_kv, int32_t max_kv,
                            int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, float *scratch,
                            size_t scratch_floats, void *o) {
  if (bad_dtype(dtype) || n_rows < 0 || n_seqs < 0 || max_q < 0 || n_pre < 0 || kv_rows < 0 || n_kv < 0 || max_kv < 0)
    return LAZY_E_BADARG;
  LAZY_TRY(check_heads(n_heads, n_kv_heads, head_dim));
  if (n_rows > MAX_GRID_YZ || n_seqs > MAX_GRID_YZ || (long long)n_pre + max_kv > MAX_KEYS) return LAZY_E_CAPACITY;
  if (n_rows == 0) return LAZY_OK;
  if (n_seqs == 0 || max_q == 0) return LAZY_E_BADARG;
  const long long width = (long long)n_kv_heads * head_dim;
  if (bad_rows(q, ldq, (long long)n_heads * head_dim, dtype) || !d_cu_q || !d_cu_kv || !scratch || !o ||
      ((uintptr_t)o & 15))
    return LAZY_E_BADARG;
  if (n_pre > 0 && (bad_rows(k_pre, ld_pre, width, dtype) || bad_rows(v_pre, ld_pre, width, dtype))) return LAZY_E_BADARG;
  if (n_kv > 0 && max_kv > 0 &&
      (!kv_idx || kv_rows < 1 || bad_rows(k, ldkv, width, dtype) || bad_rows(v, ldkv, width, dtype)))
    return LAZY_E_BADARG;
  if (scratch_floats < attention_prefix_scratch_need(n_rows, n_seqs, max_q, n_pre, max_kv, n_heads, n_kv_heads, head_dim))
    return LAZY_E_CAPACITY;
  DevStatus *status = dev_status_ptr();
  if (!status) return LAZY_E_CUDA;
  const PrefixArgs a = {q, ldq, d_cu_q, n_rows, n_seqs, max_q, k_pre, v_pre, ld_pre, n_pre, k, v, ldkv, kv_rows, kv_idx,
                        d_cu_kv, n_kv, max_kv, n_heads, n_kv_heads, head_dim, o};
  return launch_attention_prefix((cudaStream_t)stream, dtype, a, scratch, status);
}

int lazy_k_verify(void *stream, const float *p, int32_t ldp, const float *q, int32_t ldq, const int32_t *draft,
                  const int32_t *d_cu_draft, int32_t n_seqs, int32_t n_draft, int32_t max_draft, int32_t vocab,
                  const float *u_accept, const float *u_sample, int32_t *n_accept, int32_t *tokens) {
  if (n_seqs < 0 || n_draft < 0 || max_draft < 0 || max_draft == 0x7fffffff || vocab < 1 || ldp < vocab || (q && ldq < vocab))
    return LAZY_E_BADARG;
  if (n_seqs > (1 << 24) || vocab > (1 << 30) || (long long)n_draft + n_seqs > 0x7fffffff) return LAZY_E_CAPACITY;
  if (n_seqs == 0) return LAZY_OK;
  if (!p || !d_cu_draft || !u_sample || !n_accept || !tokens || (n_draft > 0 && (!draft || !u_accept))) return LAZY_E_BADARG;
  DevStatus *status = dev_status_ptr();
  if (!status) return LAZY_E_CUDA;
  return launch_verify((cudaStream_t)stream, p, ldp, q, ldq, draft, d_cu_draft, n_seqs, n_draft, max_draft, vocab,
                       u_accept, u_sample, n_accept, tokens, status);
}

}  // extern "C"
