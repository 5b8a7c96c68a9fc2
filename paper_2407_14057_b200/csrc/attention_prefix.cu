// Attention of a batch of requests that share one prefix.  Every query row sees the whole prefix and the first part of
// its request's own key list (row i of T rows: keys j <= C - T + i of C), so the prefix part is one product of all
// rows with the prefix's keys: it is computed for the batch together and read once, not once per request.
#include "attn_split.cuh"

namespace lazy {

namespace {

__device__ __forceinline__ int px_seq_of_row(const int32_t *cu, int n_seqs, int r) {
  int lo = 0, hi = n_seqs;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cu[mid] <= r) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Own keys that row r sees, as a range of the key list: [*first, *first + return value).  Tables that do not fit
// their declared sizes are reported and give no keys.
__device__ __forceinline__ int px_own_keys(const PrefixArgs &a, int r, int *first, DevStatus *status) {
  const int s = px_seq_of_row(a.cu_q, a.n_seqs, r);
  const int q0 = a.cu_q[s], q1 = a.cu_q[s + 1], c0 = a.cu_kv[s], c1 = a.cu_kv[s + 1];
  *first = c0;
  if (r < q0 || r >= q1 || q1 - q0 > a.max_q || c0 < 0 || c1 < c0 || c1 > a.n_kv || c1 - c0 > a.max_kv) {
    dev_fail(status, LAZY_E_BADARG, W_PREFIX, r, s);
    return 0;
  }
  return max((c1 - c0) - (q1 - q0) + (r - q0) + 1, 0);
}

// ---- general form ---------------------------------------------------------------------------------------------
// grid (splits, n_heads, n_rows)
template <typename T>
__global__ void __launch_bounds__(AS_THREADS)
prefix_partial_kernel(const PrefixArgs a, int per_split, float *__restrict__ part_o, float *__restrict__ part_ml,
                      DevStatus *status) {
  __shared__ AttnSplitSmem sm;
  __shared__ int s_first, s_own;
  const int r = blockIdx.z, h = blockIdx.y, H = gridDim.y, g = h / (H / a.n_kv_heads);
  if (threadIdx.x == 0) s_own = px_own_keys(a, r, &s_first, status);
  __syncthreads();
  const int first = s_first, n = a.n_pre + s_own;
  const int k0 = blockIdx.x * per_split;
  const size_t part = ((size_t)r * H + h) * gridDim.x + blockIdx.x;
  const size_t col = (size_t)g * a.head_dim;
  auto row = [&](const void *pre, const void *own, int j) -> const T * {
    if (j < a.n_pre) return (const T *)pre + (size_t)j * a.ld_pre + col;
    const int i = a.kv_idx[first + (j - a.n_pre)];
    if (i < 0 || i >= a.kv_rows) {
      dev_fail(status, LAZY_E_BADARG, W_PREFIX, first + (j - a.n_pre), i);
      return nullptr;
    }
    return (const T *)own + (size_t)i * a.ldkv + col;
  };
  attn_split_partial<T>(sm, (const T *)a.q + (size_t)r * a.ldq + (size_t)h * a.head_dim, a.head_dim, k0,
                        min(n, k0 + per_split), [&](int j) { return row(a.k_pre, a.k, j); },
                        [&](int j) { return row(a.v_pre, a.v, j); }, part_o + part * a.head_dim, part_ml + part * 2,
                        nullptr);
}

// grid (n_heads, n_rows)
template <typename T>
__global__ void __launch_bounds__(AS_THREADS)
prefix_merge_kernel(const float *__restrict__ part_o, const float *__restrict__ part_ml, int n_splits, int head_dim,
                    T *__restrict__ o) {
  const size_t rh = (size_t)blockIdx.y * gridDim.x + blockIdx.x;
  attn_split_merge<T>(part_o + rh * n_splits * head_dim, part_ml + rh * n_splits * 2, n_splits, head_dim,
                      o + rh * head_dim, nullptr);
}

template <typename T>
int prefix_general(cudaStream_t st, const PrefixArgs &a, float *scratch, DevStatus *status) {
  const int keys = a.n_pre + a.max_kv;
  const int splits = attn_split_count((long long)a.n_rows * a.n_heads, keys);
  float *part_ml = scratch + (size_t)a.n_rows * a.n_heads * splits * a.head_dim;
  prefix_partial_kernel<T><<<dim3(splits, a.n_heads, a.n_rows), AS_THREADS, 0, st>>>(
      a, attn_split_keys(keys, splits), scratch, part_ml, status);
  LAZY_COUNT_LAUNCH();
  prefix_merge_kernel<T><<<dim3(a.n_heads, a.n_rows), AS_THREADS, 0, st>>>(scratch, part_ml, splits, a.head_dim, (T *)a.o);
  LAZY_COUNT_LAUNCH();
  return launch_ok();
}

}  // namespace

size_t attention_prefix_scratch_floats(int n_rows, int n_seqs, int max_q, int n_pre, int max_kv, int n_heads,
                                       int n_kv_heads, int head_dim) {
  (void)n_seqs, (void)max_q, (void)n_kv_heads;
  return (size_t)n_rows * n_heads * attn_split_count((long long)n_rows * n_heads, n_pre + max_kv) * (head_dim + 2);
}

int launch_attention_prefix(cudaStream_t st, int dtype, const PrefixArgs &a, float *scratch, DevStatus *status) {
  if (a.n_rows == 0) return LAZY_OK;
  return dtype == LAZY_F32 ? prefix_general<float>(st, a, scratch, status) : prefix_general<bf16>(st, a, scratch, status);
}

}  // namespace lazy
