// Accumulated attention weight of prompts: mass[g, j] = sum over the last `window` rows i >= j of a sequence (0 = all rows)
// and over the query heads h of key/value head g of softmax_j(q_i,h . k_j,g / sqrt(dh)).  window = 1 with a
// division by the heads is the Eq. 1 score.  No probability matrix is written: pass 1 leaves each (row, head)'s
// log-sum-exp, pass 2 forms the logits again, key-major, so that a thread owns a key and sums over the rows in registers.
// Each key's sum is taken by one thread group in a fixed order: no atomics, the same bits every time.
//
// A "lane" is one (row, head of the group) pair; lanes of a key/value head are numbered row-major, f = row * group +
// head.  lse[g][f] (log2 units) of all rows of the batch is the scratch between the passes.
#include "cache_ops.cuh"

namespace lazy {

namespace {

// ---- general form: CUDA cores, any storage type and head width -------------------------------------------------
// 64 x 64 tiles of logits, 256 threads with 4 x 4 each, the head taken 32 columns at a time through shared memory.
constexpr int MG_T = 64, MG_K = 32, MG_THREADS = 256;

template <typename T>
__device__ __forceinline__ void mg_load(const T *row, int c0, int head_dim, float *dst) {
  // eight threads per row, four columns each; a row that does not exist reads as zeros
  const int c = (threadIdx.x & 7) * 4;
#pragma unroll
  for (int i = 0; i < 4; ++i) dst[c + i] = row && c0 + c + i < head_dim ? Elem<T>::to_f(row[c0 + c + i]) : 0.f;
}

// grid (tiles of the stationary side, n_kv_heads, n_seqs).  PASS 1: stationary lanes, streamed keys.  PASS 2:
// stationary keys, streamed lanes.
template <typename T, int PASS>
__global__ void __launch_bounds__(MG_THREADS)
mass_general_kernel(const T *__restrict__ q, int ldq, const T *__restrict__ k, int ldkv,
                    const int32_t *__restrict__ cu, int max_len, int n_total, int group, int head_dim, int window,
                    float *lse, float *__restrict__ mass, DevStatus *status) {
  __shared__ float sa[MG_T][MG_K + 1], sb[MG_T][MG_K + 1];
  const int g = blockIdx.y, s = blockIdx.z;
  int start, n;
  if (!co_span(cu, s, n_total, max_len, status, W_MASS, start, n)) return;
  const int first = window > 0 ? max(n - window, 0) : 0;  // rows [first, n) accumulate
  const int n_lanes = (n - first) * group;
  const int n_a = PASS == 1 ? n_lanes : n, a0 = blockIdx.x * MG_T;
  if (a0 >= n_a) return;
  float *lse_g = lse + ((size_t)g * n_total + start + first) * group;  // lane f of this sequence at lse_g[f]
  const float scale = rsqrtf((float)head_dim) * CO_LOG2E;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  // keys [b_begin, b_end) or lanes [b_begin, b_end) that matter to this tile
  int b_begin = 0, b_end;
  if (PASS == 1) b_end = min(n, first + (min(a0 + MG_T, n_a) - 1) / group + 1);
  else {
    b_begin = max(a0 - first, 0) * group;  // the first lane whose row sees key a0
    b_end = n_lanes;
  }
  auto lane_row = [&](int f) -> const T * {
    return f < n_lanes ? q + (size_t)(start + first + f / group) * ldq + (size_t)(g * group + f % group) * head_dim : nullptr;
  };
  auto key_row = [&](int j) -> const T * { return j < n ? k + (size_t)(start + j) * ldkv + (size_t)g * head_dim : nullptr; };
  float m[4], l[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
  }
  for (int b0 = b_begin; b0 < b_end; b0 += MG_T) {
    float x[4][4] = {};
    for (int c0 = 0; c0 < head_dim; c0 += MG_K) {
      __syncthreads();
      for (int r = threadIdx.x >> 3; r < MG_T; r += MG_THREADS / 8) {
        mg_load<T>(PASS == 1 ? lane_row(a0 + r) : key_row(a0 + r), c0, head_dim, sa[r]);
        mg_load<T>(PASS == 1 ? key_row(b0 + r) : lane_row(b0 + r), c0, head_dim, sb[r]);
      }
      __syncthreads();
#pragma unroll 8
      for (int c = 0; c < MG_K; ++c) {
        float av[4], bv[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          av[i] = sa[ty * 4 + i][c];
          bv[i] = sb[tx + i * 16][c];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) x[i][j] = fmaf(av[i], bv[j], x[i][j]);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int a = a0 + ty * 4 + i;
      if (PASS == 1) {
        const int row = first + a / group;
        float mt = m[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int key = b0 + tx + j * 16;
          x[i][j] = key <= row && key < n && a < n_a ? x[i][j] * scale : -INFINITY;
          mt = fmaxf(mt, x[i][j]);
        }
        const float ref = mt == -INFINITY ? 0.f : mt;
        float sum = l[i] * exp2f(m[i] - ref);
#pragma unroll
        for (int j = 0; j < 4; ++j) sum += exp2f(x[i][j] - ref);
        m[i] = mt;
        l[i] = sum;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int f = b0 + tx + j * 16;
          if (f < n_lanes && first + f / group >= a) l[i] += exp2f(x[i][j] * scale - lse_g[f]);
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int a = a0 + ty * 4 + i;
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) {
      const float lo = __shfl_xor_sync(0xffffffffu, l[i], o);
      if (PASS == 1) {
        const float mo = __shfl_xor_sync(0xffffffffu, m[i], o);
        const float mt = fmaxf(m[i], mo), ref = mt == -INFINITY ? 0.f : mt;
        l[i] = l[i] * exp2f(m[i] - ref) + lo * exp2f(mo - ref);
        m[i] = mt;
      } else {
        l[i] += lo;
      }
    }
    if (tx == 0 && a < n_a) {
      if (PASS == 1) lse_g[a] = m[i] + log2f(l[i]);
      else mass[(size_t)g * n_total + start + a] = l[i];
    }
  }
}

template <typename T>
int mass_general(cudaStream_t st, const T *q, int ldq, const T *k, int ldkv, const int32_t *cu, int n_seqs, int max_len,
                 int n_total, int n_heads, int n_kv_heads, int head_dim, int window, float *lse, float *mass,
                 DevStatus *status) {
  const int group = n_heads / n_kv_heads;
  const int rows = window > 0 && window < max_len ? window : max_len;
  const long long tiles = ((long long)rows * group + MG_T - 1) / MG_T;
  if (tiles > 0x7fffffffLL) return LAZY_E_CAPACITY;
  mass_general_kernel<T, 1><<<dim3((unsigned)tiles, n_kv_heads, n_seqs), MG_THREADS, 0, st>>>(
      q, ldq, k, ldkv, cu, max_len, n_total, group, head_dim, window, lse, mass, status);
  LAZY_COUNT_LAUNCH();
  mass_general_kernel<T, 2><<<dim3(cdiv(max_len, MG_T), n_kv_heads, n_seqs), MG_THREADS, 0, st>>>(
      q, ldq, k, ldkv, cu, max_len, n_total, group, head_dim, window, lse, mass, status);
  LAZY_COUNT_LAUNCH();
  return launch_ok();
}

}  // namespace

size_t attention_mass_scratch_floats(int n_seqs, int n_total, int max_len, int n_heads, int n_kv_heads, int window) {
  (void)n_seqs, (void)max_len, (void)n_kv_heads, (void)window;
  return (size_t)n_total * n_heads;
}

int launch_attention_mass(cudaStream_t st, int dtype, const void *q, int ldq, const void *k, int ldkv,
                          const int32_t *cu, int n_seqs, int max_len, int n_total, int n_heads, int n_kv_heads,
                          int head_dim, int window, float *scratch, float *mass, DevStatus *status) {
  if (n_seqs == 0 || max_len == 0) return LAZY_OK;
  if (dtype == LAZY_F32)
    return mass_general<float>(st, (const float *)q, ldq, (const float *)k, ldkv, cu, n_seqs, max_len, n_total, n_heads,
                               n_kv_heads, head_dim, window, scratch, mass, status);
  return mass_general<bf16>(st, (const bf16 *)q, ldq, (const bf16 *)k, ldkv, cu, n_seqs, max_len, n_total, n_heads,
                            n_kv_heads, head_dim, window, scratch, mass, status);
}

}  // namespace lazy
