// Attention of single query rows over split key ranges on CUDA cores, for every storage type and head width: the
// form behind the tensor-core kernels of the bounded-cache step and of the shared prefix.  One CTA takes a range of
// keys of one (row, head), 128 at a time: a warp per key for the logits (lanes along the head), a thread per column for the weighted
// sum; the partial softmaxes (maximum in log2 units, sum, unnormalised output) are merged by a second kernel.
#pragma once
#include "cache_ops.cuh"

namespace lazy {

constexpr int AS_TILE = 128, AS_THREADS = 128, AS_MAX_HD = 256;

struct AttnSplitSmem {
  float q[AS_MAX_HD];
  float logit[AS_TILE];
};

// Key rows are given by key_k(j) / key_v(j): pointers to the head's part of key j's K and V row, or NULL for a
// key that is skipped.  Keys [k0, k1), AS_TILE at a time with a running maximum; logits (may be NULL) receives
// their logits in log2 units.  Call with all AS_THREADS threads.
template <typename T, typename KeyK, typename KeyV>
__device__ __forceinline__ void attn_split_partial(AttnSplitSmem &sm, const T *q, int head_dim, int k0, int k1,
                                                   KeyK key_k, KeyV key_v, float *part_o, float *part_ml,
                                                   float *logits) {
  constexpr int COLS = AS_MAX_HD / AS_THREADS;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float scale = rsqrtf((float)head_dim) * CO_LOG2E;
  for (int c = threadIdx.x; c < head_dim; c += AS_THREADS) sm.q[c] = Elem<T>::to_f(q[c]) * scale;
  float m = -INFINITY, l = 0.f, acc[COLS];
#pragma unroll
  for (int i = 0; i < COLS; ++i) acc[i] = 0.f;
  for (int t0 = k0; t0 < k1; t0 += AS_TILE) {
    const int cnt = min(AS_TILE, k1 - t0);
    __syncthreads();  // q is there; the logits of the tile before have been read
    for (int j = warp; j < cnt; j += AS_THREADS / 32) {
      const T *row = key_k(t0 + j);
      float dot = 0.f;
      if (row)
        for (int c = lane; c < head_dim; c += 32) dot = fmaf(sm.q[c], Elem<T>::to_f(row[c]), dot);
      dot = warp_sum(dot);
      if (lane == 0) {
        sm.logit[j] = row ? dot : -INFINITY;
        if (logits) logits[t0 + j] = sm.logit[j];
      }
    }
    __syncthreads();
    float mt = -INFINITY;
    for (int j = lane; j < cnt; j += 32) mt = fmaxf(mt, sm.logit[j]);
    mt = fmaxf(m, warp_max(mt));
    const float ref = mt == -INFINITY ? 0.f : mt;  // nothing seen so far: every weight is 2^-inf = 0
    const float alpha = exp2f(m - ref);
    m = mt;
    float lt = 0.f;
    for (int j = lane; j < cnt; j += 32) lt += exp2f(sm.logit[j] - ref);
    l = l * alpha + warp_sum(lt);
#pragma unroll
    for (int i = 0; i < COLS; ++i) {
      const int c = threadIdx.x + i * AS_THREADS;
      if (c >= head_dim) continue;
      float a = acc[i] * alpha;
      for (int j = 0; j < cnt; ++j) {
        const T *row = key_v(t0 + j);
        if (row) a = fmaf(exp2f(sm.logit[j] - ref), Elem<T>::to_f(row[c]), a);
      }
      acc[i] = a;
    }
  }
#pragma unroll
  for (int i = 0; i < COLS; ++i)
    if (threadIdx.x + i * AS_THREADS < head_dim) part_o[threadIdx.x + i * AS_THREADS] = acc[i];
  if (threadIdx.x == 0) {
    part_ml[0] = m;
    part_ml[1] = l;
  }
}

// Merges n parts of one (row, head): o = sum_i 2^(m_i - m) o_i / l, l = sum_i 2^(m_i - m) l_i.  A row with no keys
// gives zeros.  stats (may be NULL) receives (m, 1 / l).  Parts i lie at part_o + i * head_dim and part_ml + 2 i; parts with an
// empty sum are not read.
template <typename T>
__device__ __forceinline__ void attn_split_merge(const float *part_o, const float *part_ml, int n, int head_dim, T *o,
                                                 float *stats) {
  float m = -INFINITY;
  for (int i = 0; i < n; ++i)
    if (part_ml[2 * i + 1] > 0.f) m = fmaxf(m, part_ml[2 * i]);
  float l = 0.f;
  bool bad = false;
  for (int i = 0; i < n; ++i) {
    const float li = part_ml[2 * i + 1];
    if (li > 0.f) l = fmaf(exp2f(part_ml[2 * i] - m), li, l);
    bad |= li != li;  // a NaN logit: the row's answer is NaN, as the formula has it
  }
  const float inv = bad ? NAN : (l > 0.f ? 1.f / l : 0.f);
  for (int c = threadIdx.x; c < head_dim; c += blockDim.x) {
    float acc = 0.f;
    for (int i = 0; i < n; ++i)
      if (part_ml[2 * i + 1] > 0.f) acc = fmaf(exp2f(part_ml[2 * i] - m), part_o[(size_t)i * head_dim + c], acc);
    o[c] = Elem<T>::from_f(acc * inv);
  }
  if (stats && threadIdx.x == 0) {
    stats[0] = m;
    stats[1] = inv;
  }
}

// Key ranges per (row, head): enough CTAs for four on every SM, in whole tiles.
inline int attn_split_count(long long rows_heads, int n_keys) {
  const long long tiles = cdiv(n_keys > 0 ? n_keys : 1, AS_TILE);
  long long want = (4LL * 148 + rows_heads - 1) / (rows_heads > 0 ? rows_heads : 1);
  if (want < 1) want = 1;
  if (want > tiles) want = tiles;
  const long long per = (tiles + want - 1) / want;
  return (int)((tiles + per - 1) / per);
}
// Keys per range when n_keys are cut into `splits` ranges of whole tiles.
inline int attn_split_keys(int n_keys, int splits) {
  return cdiv(cdiv(n_keys > 0 ? n_keys : 1, AS_TILE), splits) * AS_TILE;
}

}  // namespace lazy
