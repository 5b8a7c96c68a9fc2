// Eviction from a prompt's cache by accumulated attention weight: of every (sequence, key/value head) the newest
// n_recent rows stay, and of the older ones those with the largest weight, up to the budget; equal weights go
// to the lower row.  Heads choose for themselves, so slot t of two heads may hold different tokens.
//
// Two launches.  Select: one CTA per (sequence, head) finds the weight at the last kept rank by a radix select
// over order-preserving keys, held in shared memory, then walks the rows in order and writes each kept row's
// index, weight and position to its slot.  Gather: the whole grid copies the kept K and V rows, 16 bytes a
// thread (the part that is bound by memory: kept rows are read and written once).
#include "cache_ops.cuh"

namespace lazy {

namespace {

constexpr int ES_THREADS = 1024, ES_WARPS = ES_THREADS / 32;
constexpr int ES_BITS = 11, ES_BINS = 1 << ES_BITS;
constexpr int ES_KEYS = 49152;  // keys held in shared memory (192 KiB); longer sequences are read again per pass
constexpr int ES_SMEM = ES_KEYS * 4;

// Exclusive prefix sum over the CTA's threads of one value each; *total receives the sum.
__device__ __forceinline__ int block_exclusive(int v, int *warp_sums, int *total) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int up = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += up;
  }
  __syncthreads();  // warp_sums may still be read from the call before
  if (lane == 31) warp_sums[warp] = incl;
  __syncthreads();
  int w = lane < ES_WARPS ? warp_sums[lane] : 0;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int up = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w += up;
  }
  *total = __shfl_sync(0xffffffffu, w, ES_WARPS - 1);
  const int before = warp ? __shfl_sync(0xffffffffu, w, warp - 1) : 0;
  return before + incl - v;
}

// grid (n_kv_heads, n_seqs)
__global__ void __launch_bounds__(ES_THREADS)
evict_select_kernel(const float *__restrict__ mass, int n_total, const int32_t *__restrict__ pos,
                    const int32_t *__restrict__ cu, int max_len, int budget, int n_recent, int cap,
                    int32_t *__restrict__ idx, float *__restrict__ cmass, int32_t *__restrict__ cpos,
                    int32_t *__restrict__ clen, DevStatus *status) {
  extern __shared__ uint32_t es_keys[];
  __shared__ int hist[ES_BINS];
  __shared__ int warp_sums[ES_WARPS];
  __shared__ int s_bin, s_above;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int g = blockIdx.x, s = blockIdx.y, Hkv = gridDim.x;
  const size_t sg = (size_t)s * Hkv + g;
  int start, n;
  const bool ok = co_span(cu, s, n_total, max_len, status, W_EVICT, start, n);
  const int keep = ok ? min(n, budget) : 0;
  // what the copying kernel goes by (the heads' common length may be overwritten by a later step)
  if (threadIdx.x == 0) {
    idx[sg * (budget + 1) + budget] = keep;
    if (ok) clen[sg] = keep;
  }
  if (keep == 0) return;
  const float *m = mass + (size_t)g * n_total + start;
  const int old = n - min(n_recent, keep);  // rows that compete
  const int need = keep - (n - old);        // how many of them stay
  uint32_t bar = 0u;                        // keys above it stay; `ties` of those equal to it, lowest rows first
  int ties = 0;
  if (need == old) {
    ties = 0x7fffffff;  // all stay
  } else if (need == 0) {
    bar = 0xffffffffu;
  } else {
    const bool held = old <= ES_KEYS;
    if (held)
      for (int i = threadIdx.x; i < old; i += ES_THREADS) es_keys[i] = co_weight_key(m[i]);
    uint32_t prefix = 0u, mask = 0u;
    int left = need;
    for (int pass = 0; pass < 3; ++pass) {  // digits of 11, 11 and 10 bits from the top
      const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0), bins = pass == 2 ? 1024 : ES_BINS;
      for (int i = threadIdx.x; i < bins; i += ES_THREADS) hist[i] = 0;
      __syncthreads();
      for (int i = threadIdx.x; i < old; i += ES_THREADS) {
        const uint32_t key = held ? es_keys[i] : co_weight_key(m[i]);
        if ((key & mask) == prefix) atomicAdd(&hist[(key >> shift) & (bins - 1)], 1);
      }
      __syncthreads();
      // counts from the top: thread t owns the two bins at 2 t and 2 t + 1 counted downwards
      const int b0 = bins - 1 - 2 * (int)threadIdx.x, b1 = b0 - 1;
      const int c0 = b0 >= 0 ? hist[b0] : 0, c1 = b1 >= 0 ? hist[b1] : 0;
      int total;
      const int above = block_exclusive(c0 + c1, warp_sums, &total);
      if (c0 && above < left && left <= above + c0) {
        s_bin = b0;
        s_above = above;
      } else if (c1 && above + c0 < left && left <= above + c0 + c1) {
        s_bin = b1;
        s_above = above + c0;
      }
      __syncthreads();
      left -= s_above;
      prefix |= (uint32_t)s_bin << shift;
      mask |= (uint32_t)(bins - 1) << shift;
      __syncthreads();
    }
    bar = prefix;
    ties = left;
  }
  // ---- in row order: which rows stay, and where
  int placed = 0, tied = 0;
  for (int i0 = 0; i0 < n; i0 += ES_THREADS) {
    const int i = i0 + threadIdx.x;
    float w = 0.f;
    bool above = false, equal = false;
    if (i < n) {
      w = m[i];
      const uint32_t key = co_weight_key(w);
      above = i >= old || need == old || key > bar;
      equal = !above && key == bar && need > 0;
    }
    int total;
    const int mine = block_exclusive((above ? 1 : 0) | (equal ? 1 << 16 : 0), warp_sums, &total);
    const int ties_before = tied + (mine >> 16);
    const bool stays = above || (equal && ties_before < ties);
    if (stays) {
      const int slot = placed + (mine & 0xffff) + min(ties_before, ties) - min(tied, ties);
      idx[sg * (budget + 1) + slot] = start + i;
      cmass[sg * cap + slot] = w;
      cpos[sg * cap + slot] = pos[start + i];
    }
    placed += (total & 0xffff) + min(tied + (total >> 16), ties) - min(tied, ties);
    tied += total >> 16;
  }
}

// grid (slot groups, n_kv_heads, n_seqs); vecs 16-byte pieces per row
__global__ void __launch_bounds__(256)
evict_gather_kernel(const uint4 *__restrict__ k, const uint4 *__restrict__ v, long long ld, int vecs,
                    const int32_t *__restrict__ idx, int budget, uint4 *__restrict__ kc, uint4 *__restrict__ vc,
                    int cap, int per_block) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int g = blockIdx.y, s = blockIdx.z, Hkv = gridDim.y;
  const size_t sg = (size_t)s * Hkv + g;
  const int32_t *list = idx + sg * (budget + 1);
  const int keep = list[budget];
  const int first = blockIdx.x * per_block, last = min(first + per_block, keep);
  for (int i = threadIdx.x; i < (last - first) * vecs; i += blockDim.x) {
    const int slot = first + i / vecs, c = i % vecs;
    const size_t from = (size_t)list[slot] * ld + (size_t)g * vecs + c;
    const size_t to = (((size_t)s * cap + slot) * Hkv + g) * vecs + c;
    kc[to] = k[from];
    vc[to] = v[from];
  }
}

}  // namespace

size_t evict_scratch_ints(int n_seqs, int n_kv_heads, int budget) {
  return (size_t)n_seqs * n_kv_heads * ((size_t)budget + 1);
}

int launch_evict(cudaStream_t st, int dtype, const void *k, const void *v, int ldkv, const int32_t *pos,
                 const float *mass, const int32_t *cu, int n_seqs, int max_len, int n_total, int n_kv_heads,
                 int head_dim, int budget, int n_recent, int32_t *idx, void *kc, void *vc, float *cmass, int32_t *cpos,
                 int32_t *clen, int cap, DevStatus *status) {
  if (n_seqs == 0) return LAZY_OK;
  LAZY_TRY(co_allow_smem<evict_select_kernel>(ES_SMEM));
  const size_t smem = (size_t)(max_len < ES_KEYS ? max_len : ES_KEYS) * 4;
  LAZY_TRY(co_launch(evict_select_kernel, dim3(n_kv_heads, n_seqs), dim3(ES_THREADS), smem, st, 1, false, mass, n_total, pos,
                     cu, max_len, budget, n_recent, cap, idx, cmass, cpos, clen, status));
  const int most = budget < max_len ? budget : max_len;
  const int vecs = head_dim * elem_bytes(dtype) / 16;
  const int per_block = cdiv(2048, vecs);  // eight 16-byte pieces of K and of V per thread
  if (most == 0) return LAZY_OK;
  return co_launch(evict_gather_kernel, dim3(cdiv(most, per_block), n_kv_heads, n_seqs), dim3(256), 0, st, 1, true,
                   (const uint4 *)k, (const uint4 *)v, (long long)ldkv * elem_bytes(dtype) / 16, vecs,
                   (const int32_t *)idx, budget, (uint4 *)kc, (uint4 *)vc, cap, per_block);
}

}  // namespace lazy
