// Attention of one or several new rows per sequence over a paged cache, softmax(q k / sqrt(dh)) v: row i of a sequence's T
// sees the first len - T + i + 1 of its tokens.
#include "attn_split.cuh"
#include "paged.cuh"

namespace lazy {

namespace {

// ---- general form: every type and head width, on CUDA cores; partial softmaxes of split key ranges, then their merge ----------

// Row r's sequence and how many tokens it sees (0: it belongs to none, or its tables do not fit).  By whole warps.
__device__ __forceinline__ int paged_row_sees(const PagedArgs &a, int r, bool report, DevStatus *status, int &s) {
  s = a.cu_q ? paged_find_seq(a.cu_q, a.n_seqs, r) : r;
  int start, rows, len;
  if (s < 0 || !paged_seq(a.kv, a.cu_q, s, a.n_rows, a.max_q, a.max_kv, report, status, start, rows, len) || rows == 0) return 0;
  if (r < start || r >= start + rows) {  // boundaries that do not ascend
    if (report) dev_fail(status, LAZY_E_BADARG, W_PAGED, s, r);
    return 0;
  }
  return len - rows + (r - start) + 1;
}

// grid (splits, n_heads, n_rows)
template <typename T>
__global__ void __launch_bounds__(AS_THREADS)
paged_partial_kernel(const PagedArgs a, int group, int per_split, float *__restrict__ part_o, float *__restrict__ part_ml,
                     DevStatus *status) {
  __shared__ AttnSplitSmem<T> sm;
  const int h = blockIdx.y, r = blockIdx.z, g = h / group;
  int s;
  const int n = paged_row_sees(a, r, blockIdx.x == 0 && h == 0 && threadIdx.x == 0, status, s);
  if (n == 0) return;
  const size_t part = ((size_t)r * gridDim.y + h) * gridDim.x + blockIdx.x;
  const int32_t *table = a.kv.table + (size_t)s * a.kv.ld_table;
  auto at = [&](int j) -> long long {
    const int nth = j / a.kv.page_size, page = table[nth];
    if (page < 0 || page >= a.kv.n_pages) {
      dev_fail(status, LAZY_E_BADARG, W_PAGED, s, page);
      return -1;
    }
    return (long long)page * a.kv.page_stride + (long long)(j - nth * a.kv.page_size) * a.kv.slot_stride + (long long)g * a.kv.head_stride;
  };
  attn_split_partial<T>(
      sm, (const T *)a.q + (size_t)r * a.ldq + (size_t)h * a.head_dim, a.head_dim, blockIdx.x * per_split,
      min(n, (int)blockIdx.x * per_split + per_split),
      [&](int j) -> const T * {
        const long long i = at(j);
        return i < 0 ? nullptr : (const T *)a.kv.k + i;
      },
      [&](int j) -> const T * {
        const long long i = at(j);
        return i < 0 ? nullptr : (const T *)a.kv.v + i;
      },
      part_o + part * a.head_dim, part_ml + part * 2, nullptr);
}

// grid (n_heads, n_rows)
template <typename T>
__global__ void __launch_bounds__(AS_THREADS)
paged_merge_kernel(const PagedArgs a, const float *__restrict__ part_o, const float *__restrict__ part_ml, int splits) {
  const int h = blockIdx.x, r = blockIdx.y;
  int s;
  if (paged_row_sees(a, r, false, nullptr, s) == 0) return;  // the row is left as it was
  const size_t rh = (size_t)r * gridDim.x + h;
  attn_split_merge<T>(part_o + rh * splits * a.head_dim, part_ml + rh * splits * 2, splits, a.head_dim, (T *)a.o + rh * a.head_dim,
                      nullptr);
}

template <typename T>
int paged_general(cudaStream_t st, const PagedArgs &a, float *scratch, DevStatus *status) {
  const long long rh = (long long)a.n_rows * a.n_heads;
  const int splits = attn_split_count(rh, a.max_kv);
  float *part_o = scratch, *part_ml = scratch + (size_t)rh * splits * a.head_dim;
  LAZY_TRY(co_launch(paged_partial_kernel<T>, dim3(splits, a.n_heads, a.n_rows), dim3(AS_THREADS), 0, st, 1, false, a,
                     a.n_heads / a.n_kv_heads, attn_split_keys(a.max_kv, splits), part_o, part_ml, status));
  return co_launch(paged_merge_kernel<T>, dim3(a.n_heads, a.n_rows), dim3(AS_THREADS), 0, st, 1, false, a, part_o, part_ml, splits);
}

}  // namespace

size_t attention_paged_scratch_need(int n_rows, int n_seqs, int max_q, int max_kv, int n_heads, int n_kv_heads, int head_dim) {
  const long long rh = (long long)n_rows * n_heads;
  return (size_t)rh * attn_split_count(rh, max_kv) * (head_dim + 2);
}
size_t attention_paged_scratch_floats(int n_rows, int n_seqs, int max_q, int max_kv, int n_heads, int n_kv_heads, int head_dim) {
  return attn_split_parts((long long)n_rows * n_heads, max_kv) * (head_dim + 2);
}

int launch_attention_paged(cudaStream_t st, int dtype, const PagedArgs &a, float *scratch, DevStatus *status) {
  if (a.n_rows == 0) return LAZY_OK;
  return dtype == LAZY_F32 ? paged_general<float>(st, a, scratch, status) : paged_general<bf16>(st, a, scratch, status);
}

}  // namespace lazy
