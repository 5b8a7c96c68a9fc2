// One token on a bounded cache.  Per (sequence, key/value head): while the cache holds fewer than `budget` tokens the new
// one is appended; then it takes the slot of the token with the least accumulated attention weight among those
// older than the newest n_recent positions (equal weights: the lowest slot).  The new token's query heads attend to
// what the cache then holds, and every slot's weight grows by what the group's heads gave it.
//
// The choice depends on the weights before the step alone, so it needs no attention result, and the caches are
// read once.  bytes: K and V rows of the held slots (the bound), 16 bytes of weight and position per slot.
#include "attn_split.cuh"
#include "rows_mma.cuh"

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
  __shared__ AttnSplitSmem<T> sm;
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


// ---- one launch: bf16, head width up to 128, up to 16 query heads per key/value head ------------------------------
// A cluster of CTAs holds one (sequence, key/value head), each CTA a contiguous part of the slots, each warp every
// fourth group of 16 of them.  The first groups' rows are requested before anything else, the choice of the slot
// (a minimum over the part's weights, then over the cluster) runs underneath; the new token's row replaces the chosen slot's in
// shared memory when its group comes up.  The parts' maxima, sums and outputs meet in distributed shared memory, and
// every CTA adds the final weights of its own slots to their masses from the logits it kept (in shared memory, or in
// the scratch when a part is too long).  32 sequences of up to 2048 slots, 8 heads of 128 in groups of 4: 45 us for 232 MB, 5.2
// TB/s (the loop alone runs at the memory's rate); one sequence of 1024 slots, 32 heads: 11.3 us, the time of its steps one
// after the other: two rounds of loads, the choice, the exchange, the masses.
constexpr int SF_WARPS = 4, SF_THREADS = SF_WARPS * 32, SF_STAGES = 2, SF_CTAS = 3;
constexpr int SF_MAX_CLUSTER = 8, SF_LARGE_CLUSTER = 16;  // the second is beyond what every device has to offer: see step_cluster
// A part's logits stay in shared memory up to this size: with three CTAs on an SM, with two or one
constexpr int SF_LOGIT_BYTES = 8192, SF_LOGIT_BYTES_2 = 40960;
constexpr int SF_BATCH = 8;           // slots a thread has in flight in the loops over weights

template <int HD, int NT>
struct StepShared {
  float m[NT * 8], l[NT * 8];       // this CTA's maxima and sums, read by the cluster
  float wm[SF_WARPS][NT * 8], wl[SF_WARPS][NT * 8];
  float fm[NT * 8], finv[NT * 8];   // final
  unsigned long long best;
  unsigned long long wbest[SF_WARPS];
};
template <int HD, int NT>
constexpr int step_stage_bytes = SF_WARPS * SF_STAGES * RowsMma<HD, NT>::STAGE;

template <int HD, int NT, int MAX_CLUSTER>
__global__ void __launch_bounds__(SF_THREADS, SF_CTAS)
step_fused_kernel(const EvictStepArgs a, int group, int part_slots, int logits_in_smem, float *__restrict__ scratch,
                  DevStatus *status) {
  using Rows = RowsMma<HD, NT>;
  extern __shared__ __align__(128) uint8_t step_smem[];
  __shared__ StepShared<HD, NT> sh;
  const int rank = (int)co_cluster_rank(), csize = (int)co_cluster_size();
  const int sg = blockIdx.x / csize, s = sg / a.n_kv_heads, g = sg - s * a.n_kv_heads;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float *mi = a.mass_in + (size_t)sg * a.cap;
  const int32_t *pi = a.pos_in + (size_t)sg * a.cap;
  float *mo = a.mass_out + (size_t)sg * a.cap;
  int32_t *po = a.pos_out + (size_t)sg * a.cap;
  // The first batch of weights and positions of this CTA's slots is asked for before anything else: the rows would
  // hold it up, and it need not wait for the length (what lies behind it is not looked at).
  const int lo = rank * part_slots, behind = min(lo + part_slots, a.budget);
  int bp[SF_BATCH];
  float bw[SF_BATCH];
  auto fetch = [&](int j0, int end) {
#pragma unroll
    for (int i = 0; i < SF_BATCH; ++i) {
      const int j = j0 + i * SF_THREADS;
      bp[i] = j < end ? pi[j] : 0;
      bw[i] = j < end ? mi[j] : 0.f;
    }
  };
  fetch(lo + threadIdx.x, behind);
  const int p_new = a.pos_new[s];
  const int len = a.len_in[sg];
  bf16 *o = (bf16 *)a.o + ((size_t)s * a.n_heads + (size_t)g * group) * HD;
  if (len < 0 || len > a.budget) {  // the whole cluster alike
    if (rank == 0) {
      for (int i = threadIdx.x; i < group * HD; i += SF_THREADS) o[i] = __float2bfloat16_rn(0.f);
      if (threadIdx.x == 0) {
        dev_fail(status, LAZY_E_CAPACITY, W_EVICT, sg, len);
        a.slot[sg] = a.gone[sg] = -1;
      }
    }
    return;
  }
  const bool full = len >= a.budget;
  const int n = full ? len : len + 1;
  const int hi = max(min(behind, n), lo), end = min(hi, len);  // this CTA's slots: [lo, hi), [lo, end) of them held before
  const int groups = (hi - lo + RM_KEYS - 1) / RM_KEYS;
  const size_t ld = (size_t)a.n_kv_heads * HD;
  bf16 *kc = (bf16 *)a.kc + (size_t)s * a.cap * ld + (size_t)g * HD, *vc = (bf16 *)a.vc + (size_t)s * a.cap * ld + (size_t)g * HD;
  const uint32_t stages = smem_u32(step_smem) + warp * SF_STAGES * Rows::STAGE;
  Rows rows;
  auto request = [&](int i) {  // group warp + 4 i of this CTA
    const int j0 = lo + (warp + i * SF_WARPS) * RM_KEYS;
    if (j0 < hi)
      rows_load<HD>(stages + (i % SF_STAGES) * Rows::STAGE, [&](int r, const bf16 *&kr, const bf16 *&vr) {
        const int j = min(j0 + r, max(len - 1, 0));
        kr = kc + j * ld;
        vr = vc + j * ld;
        return j0 + r < len;  // the slot being appended holds nothing yet
      });
    rm_cp_commit();
  };
  // ---- the slot
  int slot = len;
  const bool look = full || po != pi;
  const long long first_recent = (long long)p_new - a.n_recent;
  unsigned long long best = ~0ull;
  auto take = [&](int j0) {
#pragma unroll
    for (int i = 0; i < SF_BATCH; ++i) {
      const int j = j0 + i * SF_THREADS;
      if (j < end) {
        best = min_u64(best, step_rank(bw[i], bp[i], first_recent, j));
        if (po != pi) po[j] = bp[i];
      }
    }
  };
#pragma unroll
  for (int i = 0; i < SF_STAGES - 1; ++i) request(i);
  rows.init([&](int c) -> const bf16 * {
    return c < group ? (const bf16 *)a.q + (size_t)s * a.ldq + (size_t)(g * group + c) * HD : nullptr;
  });
  if (look) {
    take(lo + threadIdx.x);
    for (int j0 = lo + threadIdx.x + SF_THREADS * SF_BATCH; j0 < end; j0 += SF_THREADS * SF_BATCH) {
      fetch(j0, end);
      take(j0);
    }
    if (full) {
#pragma unroll
      for (int k = 16; k > 0; k >>= 1) best = min_u64(best, __shfl_xor_sync(0xffffffffu, best, k));
      if (lane == 0) sh.wbest[warp] = best;
      __syncthreads();
      if (threadIdx.x == 0) {
        for (int w = 1; w < SF_WARPS; ++w) best = min_u64(best, sh.wbest[w]);
        sh.best = best;
      }
      if (csize > 1) {
        co_cluster_sync();
        best = *co_map_shared(&sh.best, lane & (csize - 1));  // csize is a power of two
#pragma unroll
        for (int k = MAX_CLUSTER / 2; k > 0; k >>= 1) best = min_u64(best, __shfl_xor_sync(0xffffffffu, best, k));
      } else {
        __syncthreads();
        best = sh.best;
      }
      slot = (int)(uint32_t)best;
    } else {
      __syncthreads();
    }
  }
  if (threadIdx.x == 0 && slot >= lo && slot < hi) {  // every thread of the CTA has read the old position
    a.slot[sg] = slot;
    a.gone[sg] = full ? pi[slot] : -1;
    po[slot] = p_new;
  }
  // ---- attention over this CTA's slots; logits [slot][columns of the group, an even number]
  const int lcols = (group + 1) & ~1;
  float *lg = logits_in_smem ? reinterpret_cast<float *>(step_smem + step_stage_bytes<HD, NT>)
                             : scratch + ((size_t)sg * csize + rank) * part_slots * lcols;
  for (int i = 0; warp + i * SF_WARPS < groups; ++i) {
    request(i + SF_STAGES - 1);
    rm_cp_wait<SF_STAGES - 1>();
    __syncwarp();
    const uint32_t stage = stages + (i % SF_STAGES) * Rows::STAGE;
    const int j0 = lo + (warp + i * SF_WARPS) * RM_KEYS;
    if (slot >= j0 && slot < j0 + RM_KEYS) {  // the new row: into the stage and the cache
      if ((lane & 15) < Rows::CHUNKS) {
        const int c = lane & 15, r = slot - j0;
        const bool is_v = lane >= 16;
        const bf16 *src = (const bf16 *)(is_v ? a.v_new : a.k_new) + (size_t)s * a.ld_new + (size_t)g * HD + c * 8;
        const uint4 x = *reinterpret_cast<const uint4 *>(src);
        const uint32_t dst = stage + (is_v ? Rows::HALF : 0) + Rows::at(r, c);
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
        *reinterpret_cast<uint4 *>((is_v ? vc : kc) + slot * ld + c * 8) = x;
      }
      __syncwarp();
    }
    int vis[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t) vis[t][0] = vis[t][1] = hi - j0;
    rows.template process<false>(stage, vis, 0xffffu, [&](int t, int r, float x0, float x1) {
      const int c = t * 8 + (lane & 3) * 2;
      if (c < lcols && j0 + r < hi) *reinterpret_cast<float2 *>(lg + (size_t)(j0 - lo + r) * lcols + c) = make_float2(x0, x1);
    });
    __syncwarp();  // the stage may be requested again
  }
  rm_cp_wait<0>();
  rows.finish();
  auto old_masses = [&](int j0) {
#pragma unroll
    for (int i = 0; i < SF_BATCH; ++i) {
      const int j = j0 + i * SF_THREADS;
      bw[i] = j < end ? mi[j] : 0.f;
    }
  };
  old_masses(lo + threadIdx.x);  // on their way during the exchange
  // ---- the CTA's part: warps' outputs against the common maximum, added in warp order
  if (lane < 4) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        sh.wm[warp][t * 8 + lane * 2 + i] = rows.m[t][i];
        sh.wl[warp][t * 8 + lane * 2 + i] = rows.l[t][i];
      }
  }
  __syncthreads();  // also: no warp reads its stages any more
  float *wo = reinterpret_cast<float *>(step_smem);  // [warp][column][HD]
  float *co = wo + SF_WARPS * NT * 8 * HD;           // [column][HD]: the CTA's outputs against its maxima, read by the cluster
  static_assert((SF_WARPS + 1) * NT * 8 * HD * 4 <= step_stage_bytes<HD, NT>, "the stages hold the outputs in the end");
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int c = t * 8 + (lane & 3) * 2 + i;
      float mx = sh.wm[0][c];
#pragma unroll
      for (int w = 1; w < SF_WARPS; ++w) mx = fmaxf(mx, sh.wm[w][c]);
      const float ref = mx == -INFINITY ? 0.f : mx;
      const float f = ex2_approx(rows.m[t][i] - ref) * WEIGHT_UNLIFT;
#pragma unroll
      for (int k = 0; k < HD / 16; ++k) {
        wo[((size_t)warp * NT * 8 + c) * HD + k * 16 + (lane >> 2)] = rows.o[t][k][i] * f;
        wo[((size_t)warp * NT * 8 + c) * HD + k * 16 + 8 + (lane >> 2)] = rows.o[t][k][2 + i] * f;
      }
      if (warp == 0 && lane < 4) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < SF_WARPS; ++w) sum += sh.wl[w][c] * ex2_approx(sh.wm[w][c] - ref);
        sh.m[c] = mx;
        sh.l[c] = sum;
      }
    }
  __syncthreads();
  for (int i = threadIdx.x; i < group * HD; i += SF_THREADS) {
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < SF_WARPS; ++w) sum += wo[(size_t)w * NT * 8 * HD + i];
    co[i] = sum;
  }
  if (csize > 1) co_cluster_sync();
  else __syncthreads();
  // ---- the final maxima and sums, the same in every thread that needs them; this CTA's share of the outputs.  All
  // reads of the other CTAs' memory are in flight together.
  auto gather = [&](int c, float &ref, float &inv, float *scale) {
    float rm[MAX_CLUSTER], rl[MAX_CLUSTER], mx = -INFINITY, sum = 0.f;
#pragma unroll
    for (int r = 0; r < MAX_CLUSTER; ++r) {
      rm[r] = r < csize ? *co_map_shared(&sh.m[c], r) : -INFINITY;
      rl[r] = r < csize ? *co_map_shared(&sh.l[c], r) : 0.f;
    }
#pragma unroll
    for (int r = 0; r < MAX_CLUSTER; ++r) mx = fmaxf(mx, rm[r]);
    ref = mx == -INFINITY ? 0.f : mx;
#pragma unroll
    for (int r = 0; r < MAX_CLUSTER; ++r) {
      scale[r] = ex2_approx(rm[r] - ref);
      sum += rl[r] * scale[r];
    }
    inv = 1.f / sum;
  };
  for (int i = rank * SF_THREADS + threadIdx.x; i < group * HD; i += csize * SF_THREADS) {
    float part[MAX_CLUSTER], scale[MAX_CLUSTER], ref, inv, sum = 0.f;
#pragma unroll
    for (int r = 0; r < MAX_CLUSTER; ++r) part[r] = r < csize ? *co_map_shared(co + i, r) : 0.f;
    gather(i / HD, ref, inv, scale);
#pragma unroll
    for (int r = 0; r < MAX_CLUSTER; ++r) sum += part[r] * scale[r];  // ranks that do not exist: 0 x 0
    o[i] = __float2bfloat16_rn(sum * inv);
  }
  if (threadIdx.x < group) {
    float scale[MAX_CLUSTER], ref, inv;
    gather(threadIdx.x, ref, inv, scale);
    sh.fm[threadIdx.x] = ref;
    sh.finv[threadIdx.x] = inv;
  }
  __syncthreads();
  if (csize > 1) co_cluster_arrive();  // the other CTAs' parts have been read
  // ---- the slots' masses
  for (int j0 = lo + threadIdx.x; j0 < hi; j0 += SF_THREADS * SF_BATCH) {
    float w[SF_BATCH];
    int j[SF_BATCH];
    if (j0 >= lo + SF_THREADS * SF_BATCH) old_masses(j0);
#pragma unroll
    for (int i = 0; i < SF_BATCH; ++i) {
      j[i] = min(j0 + i * SF_THREADS, hi - 1);
      w[i] = 0.f;
    }
#pragma unroll 2
    for (int c = 0; c < lcols; c += 2) {
      const float m0 = sh.fm[c], f0 = sh.finv[c], m1 = sh.fm[c + 1], f1 = sh.finv[c + 1];
#pragma unroll
      for (int i = 0; i < SF_BATCH; ++i) {
        const float2 x = *reinterpret_cast<const float2 *>(lg + (size_t)(j[i] - lo) * lcols + c);
        w[i] = fmaf(ex2_approx(x.x - m0), f0, w[i]);
        if (c + 1 < group) w[i] = fmaf(ex2_approx(x.y - m1), f1, w[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < SF_BATCH; ++i)
      if (j0 + i * SF_THREADS < hi) mo[j[i]] = (j[i] == slot ? 0.f : bw[i]) + w[i];
  }
  if (rank == 0 && threadIdx.x == 0) a.len_out[sg] = n;  // the cluster has read the old length long ago
  if (csize > 1) co_cluster_wait();                      // nobody leaves while its parts are being read
}

bool step_fused_eligible(int dtype, int head_dim, int group) {
  return dtype == LAZY_BF16 && head_dim <= 128 && group <= 16;
}

// CTAs per (sequence, head): the next power of two that still leaves every warp a group of 16 slots and room for
// all CTAs at once at three per SM.  A second wave costs more than it spreads: 32 sequences of 2048 slots on 8 heads
// take 47 us with one CTA each, 61 us with two, 63 us with four.  Sixteen to a cluster, where the heads are few and the lists
// long: a CTA's four warps get through 1000 slots in some 14 us, whatever is left idle beside it (8000 slots on 8 heads: 19.6 us
// with eight, 16.3 with sixteen; 16000 on one: 30.8 and 18.6; 2000 on eight: 9.5 and 9.6; 4000 on 16: 15.9 and 15.7).
int step_cluster(long long heads, int budget) {
  if (heads * SF_LARGE_CLUSTER <= co_cluster_ctas(SF_LARGE_CLUSTER, 2) && budget > SF_LARGE_CLUSTER * 2 * SF_WARPS * RM_KEYS)
    return SF_LARGE_CLUSTER;
  int c = 1;
  while (c < SF_MAX_CLUSTER && heads * c * 2 <= co_cluster_ctas(c * 2, SF_CTAS) && budget > c * SF_WARPS * RM_KEYS) c *= 2;
  return c;
}
int step_part_slots(int budget, int cluster) { return cdiv(cdiv(budget, RM_KEYS), cluster) * RM_KEYS; }

template <int HD, int NT, int MAX_CLUSTER>
int step_fused_launch(cudaStream_t st, const EvictStepArgs &a, int cluster, float *scratch, DevStatus *status) {
  const int group = a.n_heads / a.n_kv_heads, part = step_part_slots(a.budget, cluster);
  const long long heads = (long long)a.n_seqs * a.n_kv_heads, logit_bytes = (long long)part * ((group + 1) & ~1) * 4;
  const int in_smem = logit_bytes <= (heads * cluster <= 2LL * sm_count() ? SF_LOGIT_BYTES_2 : SF_LOGIT_BYTES);
  const int smem = step_stage_bytes<HD, NT> + (in_smem ? (int)logit_bytes : 0);
  LAZY_TRY((co_allow_smem<step_fused_kernel<HD, NT, MAX_CLUSTER>>(step_stage_bytes<HD, NT> + SF_LOGIT_BYTES_2, false,
                                                                 MAX_CLUSTER > SF_MAX_CLUSTER)));
  return co_launch(step_fused_kernel<HD, NT, MAX_CLUSTER>, dim3((unsigned)(heads * cluster)), dim3(SF_THREADS), smem, st, cluster,
                   false, a, group, part, in_smem, scratch, status);
}
template <int HD, int NT>
int step_fused(cudaStream_t st, const EvictStepArgs &a, float *scratch, DevStatus *status) {
  const int cluster = step_cluster((long long)a.n_seqs * a.n_kv_heads, a.budget);
  return cluster > SF_MAX_CLUSTER ? step_fused_launch<HD, NT, SF_LARGE_CLUSTER>(st, a, cluster, scratch, status)
                                  : step_fused_launch<HD, NT, SF_MAX_CLUSTER>(st, a, cluster, scratch, status);
}

}  // namespace

// What the call needs, or (`any`) as much as any smaller one does: of the general form's parts the most there can be.
static size_t step_scratch_floats(int n_seqs, int n_heads, int n_kv_heads, int head_dim, int budget, bool any) {
  size_t general = step_scratch(n_seqs, n_heads, n_kv_heads, head_dim, budget).total;
  if (any) {
    const size_t sh = (size_t)n_seqs * n_heads, splits = (size_t)attn_split_count((long long)sh, budget);
    general += (attn_split_parts((long long)sh, budget) - sh * splits) * (head_dim + 2);
  }
  // the one-launch form keeps at most every slot's logits, an even number of columns, parts rounded up to 16 slots; + 4: they
  // are read two at a time and start on a 16-byte boundary
  const size_t heads = (size_t)n_seqs * n_kv_heads, group = n_heads / n_kv_heads;
  const size_t fused = heads * ((size_t)budget + SF_LARGE_CLUSTER * RM_KEYS) * ((group + 1) & ~(size_t)1) + 4;
  return general > fused ? general : fused;
}
size_t evict_step_scratch_need(int n_seqs, int n_heads, int n_kv_heads, int head_dim, int budget) {
  return step_scratch_floats(n_seqs, n_heads, n_kv_heads, head_dim, budget, false);
}
size_t evict_step_scratch_floats(int n_seqs, int n_heads, int n_kv_heads, int head_dim, int budget) {
  return step_scratch_floats(n_seqs, n_heads, n_kv_heads, head_dim, budget, true);
}

int launch_evict_step(cudaStream_t st, int dtype, const EvictStepArgs &a, float *scratch, DevStatus *status) {
  if (a.n_seqs == 0) return LAZY_OK;
  const int group = a.n_heads / a.n_kv_heads;
  if (step_fused_eligible(dtype, a.head_dim, group)) {
    float *logits = reinterpret_cast<float *>(align_up((uintptr_t)scratch, 16));
    return co_head_dim(a.head_dim, [&](auto hd) {
      return group <= 8 ? step_fused<hd.value, 1>(st, a, logits, status) : step_fused<hd.value, 2>(st, a, logits, status);
    });
  }
  return dtype == LAZY_F32 ? step_general<float>(st, a, scratch, status) : step_general<bf16>(st, a, scratch, status);
}

}  // namespace lazy
