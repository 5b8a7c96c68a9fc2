// Attention of single query rows over split key ranges on CUDA cores, for every storage type and head width: the
// form behind the tensor-core kernels of the bounded-cache step and of the shared prefix.  One CTA takes a range of
// keys of one (row, head), 128 at a time: a warp per eight keys for the logits (lanes along the head), a thread per four columns and
// every few keys for the weighted sum, eight rows in flight in either; the partial softmaxes (maximum in log2 units, sum, unnormalised output) are merged by a second kernel.
#pragma once
#include "cache_ops.cuh"

namespace lazy {

constexpr int AS_TILE = 128, AS_THREADS = 128, AS_MAX_HD = 256;
constexpr int AS_KEYS = 8;  // key rows that a warp (logits) or a thread (weighted sum) has in flight

template <typename T>
struct AttnSplitSmem {
  float q[AS_MAX_HD];
  float logit[AS_TILE];                // then the weights
  const T *k_row[AS_TILE], *v_row[AS_TILE];
  float4 sum[AS_THREADS];
  float l[AS_THREADS / 32];
};

__device__ __forceinline__ float4 as_load4(const float *p) { return *reinterpret_cast<const float4 *>(p); }
__device__ __forceinline__ float4 as_load4(const bf16 *p) {
  const uint2 u = *reinterpret_cast<const uint2 *>(p);
  float4 x;
  bf16x2_unpack(u.x, x.x, x.y);
  bf16x2_unpack(u.y, x.z, x.w);
  return x;
}

// Key rows are given by key_k(j) / key_v(j): pointers to the head's part of key j's K and V row, or NULL for a
// key that is skipped.  Keys [k0, k1), AS_TILE at a time with a running maximum; logits (may be NULL) receives
// their logits in log2 units.  Call with all AS_THREADS threads.
template <typename T, typename KeyK, typename KeyV>
__device__ __forceinline__ void attn_split_partial(AttnSplitSmem<T> &sm, const T *q, int head_dim, int k0, int k1,
                                                   KeyK key_k, KeyV key_v, float *part_o, float *part_ml,
                                                   float *logits) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float scale = rsqrtf((float)head_dim) * CO_LOG2E;
  for (int c = threadIdx.x; c < head_dim; c += AS_THREADS) sm.q[c] = Elem<T>::to_f(q[c]) * scale;
  // weighted sum: a thread has four columns of every `key_lanes`-th key
  const int quads = head_dim / 4, key_lanes = AS_THREADS / quads, quad = threadIdx.x % quads, key_lane = threadIdx.x / quads;
  float m = -INFINITY, l = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int t0 = k0; t0 < k1; t0 += AS_TILE) {
    const int cnt = min(AS_TILE, k1 - t0);
    if (t0 > k0) __syncthreads();  // the weights of the tile before have been used
    if ((int)threadIdx.x < cnt) {
      sm.k_row[threadIdx.x] = key_k(t0 + threadIdx.x);
      sm.v_row[threadIdx.x] = key_v(t0 + threadIdx.x);
    }
    __syncthreads();  // and q is there
    for (int j0 = warp * AS_KEYS; j0 < cnt; j0 += AS_THREADS / 32 * AS_KEYS) {
      float dot[AS_KEYS];
      const T *row[AS_KEYS];
#pragma unroll
      for (int i = 0; i < AS_KEYS; ++i) {
        row[i] = j0 + i < cnt ? sm.k_row[j0 + i] : nullptr;
        dot[i] = 0.f;
      }
      for (int c = lane * 4; c < head_dim; c += 128) {
        const float4 a = *reinterpret_cast<const float4 *>(sm.q + c);
        float4 x[AS_KEYS];
#pragma unroll
        for (int i = 0; i < AS_KEYS; ++i) x[i] = row[i] ? as_load4(row[i] + c) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int i = 0; i < AS_KEYS; ++i)
          dot[i] = fmaf(a.x, x[i].x, fmaf(a.y, x[i].y, fmaf(a.z, x[i].z, fmaf(a.w, x[i].w, dot[i]))));
      }
      float mine = -INFINITY;
#pragma unroll
      for (int i = 0; i < AS_KEYS; ++i) {
        const float d = warp_sum(dot[i]);
        if (lane == i && row[i]) mine = d;
      }
      if (lane < AS_KEYS && j0 + lane < cnt) {
        sm.logit[j0 + lane] = mine;
        if (logits) logits[t0 + j0 + lane] = mine;
      }
    }
    __syncthreads();
    float mt = -INFINITY;
    for (int j = lane; j < cnt; j += 32) mt = fmaxf(mt, sm.logit[j]);
    mt = fmaxf(m, warp_max(mt));
    const float ref = mt == -INFINITY ? 0.f : mt;  // nothing seen so far: every weight is 2^-inf = 0
    const float alpha = exp2f(m - ref);
    m = mt;
    l *= alpha;
    __syncthreads();  // every warp has the maximum: the logits become weights
    if ((int)threadIdx.x < cnt) {
      const float p = exp2f(sm.logit[threadIdx.x] - ref);
      sm.logit[threadIdx.x] = p;
      l += p;
    }
    __syncthreads();
    acc = make_float4(acc.x * alpha, acc.y * alpha, acc.z * alpha, acc.w * alpha);
    if (key_lane < key_lanes) {
      for (int j0 = key_lane; j0 < cnt; j0 += AS_KEYS * key_lanes) {
        float4 x[AS_KEYS];
        float p[AS_KEYS];
#pragma unroll
        for (int i = 0; i < AS_KEYS; ++i) {
          const int j = j0 + i * key_lanes;
          const T *row = j < cnt ? sm.v_row[j] : nullptr;
          x[i] = row ? as_load4(row + quad * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
          p[i] = row ? sm.logit[j] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < AS_KEYS; ++i)
          acc = make_float4(fmaf(p[i], x[i].x, acc.x), fmaf(p[i], x[i].y, acc.y), fmaf(p[i], x[i].z, acc.z), fmaf(p[i], x[i].w, acc.w));
      }
    }
  }
  sm.sum[threadIdx.x] = acc;
  l = warp_sum(l);
  if (lane == 0) sm.l[warp] = l;
  __syncthreads();
  if ((int)threadIdx.x < quads) {
    float4 o = sm.sum[threadIdx.x];
    for (int i = 1; i < key_lanes; ++i) {
      const float4 x = sm.sum[i * quads + threadIdx.x];
      o = make_float4(o.x + x.x, o.y + x.y, o.z + x.z, o.w + x.w);
    }
    part_o[threadIdx.x * 4] = o.x;  // parts may start anywhere in the scratch
    part_o[threadIdx.x * 4 + 1] = o.y;
    part_o[threadIdx.x * 4 + 2] = o.z;
    part_o[threadIdx.x * 4 + 3] = o.w;
  }
  if (threadIdx.x == 0) {
    part_ml[0] = m;
    part_ml[1] = sm.l[0] + sm.l[1] + sm.l[2] + sm.l[3];
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
  long long want = (4LL * sm_count() + rows_heads - 1) / (rows_heads > 0 ? rows_heads : 1);
  if (want < 1) want = 1;
  if (want > tiles) want = tiles;
  const long long per = (tiles + want - 1) / want;
  return (int)((tiles + per - 1) / per);
}
// The most ranges that any number of pairs up to rows_heads makes of up to n_keys, times the pairs.
inline size_t attn_split_parts(long long rows_heads, int n_keys) {
  const long long tiles = cdiv(n_keys > 0 ? n_keys : 1, AS_TILE), all = rows_heads * tiles, most = rows_heads + 4LL * sm_count() - 1;
  return (size_t)(rows_heads < 1 ? 0 : (all < most ? all : most));
}
// Keys per range when n_keys are cut into `splits` ranges of whole tiles.
inline int attn_split_keys(int n_keys, int splits) {
  return cdiv(cdiv(n_keys > 0 ? n_keys : 1, AS_TILE), splits) * AS_TILE;
}

}  // namespace lazy
