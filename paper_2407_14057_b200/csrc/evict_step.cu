// One token on a bounded cache.  Per (sequence, key/value head): while the cache holds fewer than `budget` tokens the new
// one is appended; then it takes the slot of the token with the least accumulated attention weight among those
// older than the newest n_recent positions (equal weights: the lowest slot).  The new token's query heads attend to
// what the cache then holds, and every slot's weight grows by what the group's heads gave it.
//
// The choice depends on the weights before the step alone, so it needs no attention result, and the caches are
// read once.  bytes: K and V rows of the held slots (the bound), 16 bytes of weight and position per slot.
#include "attn_split.cuh"

namespace lazy {

namespace {

__device__ __forceinline__ unsigned long long min_u64(unsigned long long a, unsigned long long b) { return a < b ? a : b; }

// What one slot weighs in the choice: the smallest value is evicted.  Protected slots come after all others.
__device__ __forceinline__ unsigned long long step_rank(float w, int pos, long long first_recent, int slot) {
  const uint32_t key = (long long)pos < first_recent ? co_weight_key(w) : 0xffffffffu;
  return ((unsigned long long)key << 32) | (uint32_t)slot;
}

// ---- general form: place, partial attention, merge, accumulate -----------------------------------------------

// grid (n_kv_heads, n_seqs): chooses the slot, writes the new row there and the slot's new weight (0) and position.
// held[s, g] = tokens after the step (0: the sequence is skipped).
template <typename T>
__global__ void __launch_bounds__(256)
step_place_kernel(const T *__restrict__ k_new, const T *__restrict__ v_new, int ld_new,
                  const int32_t *__restrict__ pos_new, T *__restrict__ kc, T *__restrict__ vc, int cap, int head_dim,
                  const float *mass_in, float *mass_out, const int32_t *pos_in, int32_t *pos_out,
                  const int32_t *len_in, int32_t *len_out, int budget, int n_recent, int32_t *__restrict__ held,
                  int32_t *__restrict__ slot_out, int32_t *__restrict__ gone_out, DevStatus *status) {
  __shared__ unsigned long long best_s[8];
  const int g = blockIdx.x, s = blockIdx.y, Hkv = gridDim.x;
  const size_t sg = (size_t)s * Hkv + g;
  const int len = len_in[sg];
  if (len < 0 || len > budget) {
    if (threadIdx.x == 0) {
      dev_fail(status, LAZY_E_CAPACITY, W_EVICT, (int)sg, len);
      held[sg] = 0;
      slot_out[sg] = gone_out[sg] = -1;
    }
    return;
  }
  const float *mi = mass_in + sg * cap;
  const int32_t *pi = pos_in + sg * cap;
  float *mo = mass_out + sg * cap;
  int32_t *po = pos_out + sg * cap;
  const int p_new = pos_new[s];
  const long long first_recent = (long long)p_new - n_recent;
  unsigned long long best = ~0ull;
  for (int j = threadIdx.x; j < len; j += blockDim.x) {
    const float w = mi[j];
    const int p = pi[j];
    best = min_u64(best, step_rank(w, p, first_recent, j));
    if (mo != mi) mo[j] = w;
    if (po != pi) po[j] = p;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) best = min_u64(best, __shfl_xor_sync(0xffffffffu, best, o));
  if ((threadIdx.x & 31) == 0) best_s[threadIdx.x >> 5] = best;
  __syncthreads();
  for (int w = 0; w < 8; ++w) best = min_u64(best, best_s[w]);
  const bool full = len >= budget;
  const int slot = full ? (int)(uint32_t)best : len;
  const int gone = full ? pi[slot] : -1;
  __syncthreads();  // every thread has read the slot's position before it is overwritten
  if (threadIdx.x == 0) {
    held[sg] = full ? len : len + 1;
    len_out[sg] = full ? len : len + 1;
    slot_out[sg] = slot;
    gone_out[sg] = gone;
    mo[slot] = 0.f;
    po[slot] = p_new;
  }
  const size_t row = (((size_t)s * cap + slot) * Hkv + g) * head_dim, from = (size_t)s * ld_new + (size_t)g * head_dim;
  for (int c = threadIdx.x; c < head_dim; c += blockDim.x) {
    kc[row + c] = k_new[from + c];
    vc[row + c] = v_new[from + c];
  }
}

// grid (splits, n_heads, n_seqs)
template <typename T>
__global__ void __launch_bounds__(AS_THREADS)
step_partial_kernel(const T *__restrict__ q, int ldq, const T *__restrict__ kc, const T *__restrict__ vc, int cap,
                    int head_dim, int group, const int32_t *__restrict__ held, int budget, int per_split,
                    float *__restrict__ part_o, float *__restrict__ part_ml, float *__restrict__ logits) {
  __shared__ AttnSplitSmem sm;
  const int h = blockIdx.y, s = blockIdx.z, H = gridDim.y, g = h / group, Hkv = H / group;
  const int n = held[(size_t)s * Hkv + g], k0 = blockIdx.x * per_split;
  const size_t sh = (size_t)s * H + h, part = sh * gridDim.x + blockIdx.x;
  const size_t base = ((size_t)s * cap * Hkv + g) * head_dim, ld = (size_t)Hkv * head_dim;
  attn_split_partial<T>(sm, q + (size_t)s * ldq + (size_t)h * head_dim, head_dim, k0, min(n, k0 + per_split),
                        [&](int j) { return kc + base + j * ld; }, [&](int j) { return vc + base + j * ld; },
                        part_o + part * head_dim, part_ml + part * 2, logits + sh * budget);
}

// grid (n_heads, n_seqs)
template <typename T>
__global__ void __launch_bounds__(AS_THREADS)
step_merge_kernel(const float *__restrict__ part_o, const float *__restrict__ part_ml, int n_splits, int head_dim,
                  T *__restrict__ o, float *__restrict__ stats) {
  const size_t sh = (size_t)blockIdx.y * gridDim.x + blockIdx.x;
  attn_split_merge<T>(part_o + sh * n_splits * head_dim, part_ml + sh * n_splits * 2, n_splits, head_dim,
                      o + sh * head_dim, stats + sh * 2);
}

// grid (slot groups, n_kv_heads, n_seqs)
__global__ void __launch_bounds__(256)
step_accumulate_kernel(const float *__restrict__ logits, const float *__restrict__ stats,
                       const int32_t *__restrict__ held, int group, int budget, int cap, float *mass) {
  const int g = blockIdx.y, s = blockIdx.z, Hkv = gridDim.y, H = Hkv * group;
  const int j = blockIdx.x * 256 + threadIdx.x;
  if (j >= held[(size_t)s * Hkv + g]) return;
  float w = 0.f;
  for (int i = 0; i < group; ++i) {
    const size_t sh = (size_t)s * H + g * group + i;
    w = fmaf(exp2f(logits[sh * budget + j] - stats[sh * 2]), stats[sh * 2 + 1], w);
  }
  mass[((size_t)s * Hkv + g) * cap + j] += w;
}

struct StepScratch {  // floats: partial outputs | partial (max, sum) | logits | merged (max, 1 / sum) | held (int32)
  size_t part_o, part_ml, logits, stats, held, total;
};
StepScratch step_scratch(int n_seqs, int n_heads, int n_kv_heads, int head_dim, int budget) {
  const size_t sh = (size_t)n_seqs * n_heads, splits = (size_t)attn_split_count((long long)sh, budget);
  StepScratch c;
  c.part_o = 0;
  c.part_ml = c.part_o + sh * splits * head_dim;
  c.logits = c.part_ml + sh * splits * 2;
  c.stats = c.logits + sh * budget;
  c.held = c.stats + sh * 2;
  c.total = c.held + (size_t)n_seqs * n_kv_heads;
  return c;
}

template <typename T>
int step_general(cudaStream_t st, const EvictStepArgs &a, float *scratch, DevStatus *status) {
  const StepScratch c = step_scratch(a.n_seqs, a.n_heads, a.n_kv_heads, a.head_dim, a.budget);
  int32_t *held = reinterpret_cast<int32_t *>(scratch + c.held);
  const int splits = attn_split_count((long long)a.n_seqs * a.n_heads, a.budget), group = a.n_heads / a.n_kv_heads;
  step_place_kernel<T><<<dim3(a.n_kv_heads, a.n_seqs), 256, 0, st>>>(
      (const T *)a.k_new, (const T *)a.v_new, a.ld_new, a.pos_new, (T *)a.kc, (T *)a.vc, a.cap, a.head_dim, a.mass_in,
      a.mass_out, a.pos_in, a.pos_out, a.len_in, a.len_out, a.budget, a.n_recent, held, a.slot, a.gone, status);
  LAZY_COUNT_LAUNCH();
  step_partial_kernel<T><<<dim3(splits, a.n_heads, a.n_seqs), AS_THREADS, 0, st>>>(
      (const T *)a.q, a.ldq, (const T *)a.kc, (const T *)a.vc, a.cap, a.head_dim, group, held, a.budget,
      attn_split_keys(a.budget, splits),      scratch + c.part_o, scratch + c.part_ml, scratch + c.logits);
  LAZY_COUNT_LAUNCH();
  step_merge_kernel<T><<<dim3(a.n_heads, a.n_seqs), AS_THREADS, 0, st>>>(
      scratch + c.part_o, scratch + c.part_ml, splits, a.head_dim, (T *)a.o, scratch + c.stats);
  LAZY_COUNT_LAUNCH();
  step_accumulate_kernel<<<dim3(cdiv(a.budget, 256), a.n_kv_heads, a.n_seqs), 256, 0, st>>>(
      scratch + c.logits, scratch + c.stats, held, group, a.budget, a.cap, a.mass_out);
  LAZY_COUNT_LAUNCH();
  return launch_ok();
}

}  // namespace

size_t evict_step_scratch_floats(int n_seqs, int n_heads, int n_kv_heads, int head_dim, int budget) {
  return step_scratch(n_seqs, n_heads, n_kv_heads, head_dim, budget).total;
}

int launch_evict_step(cudaStream_t st, int dtype, const EvictStepArgs &a, float *scratch, DevStatus *status) {
  if (a.n_seqs == 0) return LAZY_OK;
  return dtype == LAZY_F32 ? step_general<float>(st, a, scratch, status) : step_general<bf16>(st, a, scratch, status);
}

}  // namespace lazy
