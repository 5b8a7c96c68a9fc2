// Log probabilities of given tokens from rows of logits, with the distribution's entropy, the token's rank and the best
// alternatives, in one pass over the logits:
//   lse = m + log sum_j e^(x_j - m),   log p_t = x_t - lse,   H = lse - sum_j p_j x_j = log S - T / S
// with S = sum e^(x_j - m), T = sum (x_j - m) e^(x_j - m), kept per thread against a running maximum and rescaled when it grows.
//
// Alternatives: the k-th largest of the threads' own maxima over the first loads is a bound that at least k logits reach; what reaches it
// on the way goes to a short list in shared memory, and the list's k best, by (logit, lower id), are found by counting
// at the end, once the bound has been raised to the k-th largest of the threads' maxima over the whole row.  A list that overflows
// (many equal logits) is filled again with the better bound.
#include "attn_common.cuh"
#include "cache_ops.cuh"

namespace lazy {

namespace {

constexpr int LP_THREADS = 256, LP_WARPS = LP_THREADS / 32;
constexpr int LP_LOADS = 4;      // 16-byte loads of a thread in flight
constexpr int LP_LIST = 1024;    // candidates in shared memory
constexpr float LP_LN2 = 0.6931471805599453f;
constexpr float LP_LOWEST = -3.402823466e38f;

typedef unsigned long long u64;

// Order of candidates as one number: larger logit first, then the lower id.
__device__ __forceinline__ u64 lp_key(float x, int id) { return ((u64)co_weight_key(x) << 32) | (uint32_t)~id; }
__device__ __forceinline__ int lp_key_id(u64 key) { return (int)~(uint32_t)key; }
__device__ __forceinline__ float lp_unkey(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? k ^ 0x80000000u : ~k); }

// Running softmax sums of one thread: s = sum 2^d, t = sum d 2^d with d = (x - m) log2(e), either as a pair of partial sums.
struct LpSums {
  float m;
  u64 s, t;
  __device__ __forceinline__ void raise(float to) {
    const float delta = fmaxf((m - to) * CO_LOG2E, -200.f), f = ex2_approx(delta);
    const u64 f2 = f32x2_pack(f, f);
    t = f32x2_mul(f32x2_fma(f32x2_pack(delta, delta), s, t), f2);
    s = f32x2_mul(s, f2);
    m = to;
  }
  // minus_ref: -m, or 0 while m is -infinity.  2^-200 is 0 here: what is impossible adds 0 to both, a NaN makes s NaN
  __device__ __forceinline__ void add(float x0, float x1, float minus_ref) {
    const u64 d = f32x2_mul(f32x2_add(f32x2_pack(x0, x1), f32x2_pack(minus_ref, minus_ref)), f32x2_pack(CO_LOG2E, CO_LOG2E));
    float d0, d1;
    f32x2_unpack(d, d0, d1);
    const u64 e = f32x2_pack(ex2_approx(d0), ex2_approx(d1));
    s = f32x2_add(s, e);
    t = f32x2_fma(e, f32x2_pack(fmaxf(d0, -200.f), fmaxf(d1, -200.f)), t);
  }
  __device__ __forceinline__ float minus_ref() const { return m == -INFINITY ? 0.f : -m; }
};
// The same of several threads together.
struct LpTotal {
  float m, s, t;
  __device__ __forceinline__ void merge(const LpTotal &o) {
    const float mn = fmaxf(m, o.m), r = mn == -INFINITY ? 0.f : mn;
    const float da = fmaxf((m - r) * CO_LOG2E, -200.f), db = fmaxf((o.m - r) * CO_LOG2E, -200.f);
    const float fa = ex2_approx(da), fb = ex2_approx(db);
    t = fmaf(da, s, t) * fa + fmaf(db, o.s, o.t) * fb;
    s = s * fa + o.s * fb;
    m = mn;
  }
};

struct LpShared {
  u64 list[LP_LIST];
  u64 best[LAZY_MAX_TOP];
  uint32_t most[LP_THREADS];  // keys of the threads' maxima
  LpTotal sums[LP_WARPS];
  int higher[LP_WARPS];
  int count;
  uint32_t bound;
  u64 kth;
};

// A number that at least k of the threads' maxima reach, next to the k-th largest of them: its key's upper 16 bits.  By one
// warp; 0 where fewer than k threads have seen anything.
__device__ __forceinline__ uint32_t lp_bound(const uint32_t *most, int k) {
  const int lane = threadIdx.x & 31;
  uint32_t v[LP_WARPS], hi = 0;
#pragma unroll
  for (int i = 0; i < LP_WARPS; ++i) {
    v[i] = most[i * 32 + lane];
    hi = max(hi, v[i]);
  }
  hi = __reduce_max_sync(0xffffffffu, hi);
  uint32_t t = 0;
  for (int b = 31; b >= 16; --b) {
    const uint32_t c = t | (1u << b);
    if (c > hi) continue;  // the whole warp alike
    int n = 0;
#pragma unroll
    for (int i = 0; i < LP_WARPS; ++i) n += v[i] >= c;
    if ((int)__reduce_add_sync(0xffffffffu, n) >= k) t = c;
  }
  return t;
}

template <typename T>
__global__ void __launch_bounds__(LP_THREADS)
token_logprobs_kernel(const LogprobArgs a, DevStatus *status) {
  constexpr int V = Elem<T>::kPerVec;
  __shared__ LpShared sh;
  const int r = blockIdx.x, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, k = a.n_top;
  const T *x = (const T *)a.logits + (size_t)r * a.ld;
  int token = a.tokens ? a.tokens[r] : -1;
  if (token >= a.vocab) {
    if (tid == 0) dev_fail(status, LAZY_E_BADARG, W_LOGPROBS, r, token);
    token = -1;
  }
  const float given = token >= 0 ? Elem<T>::to_f(x[token]) : NAN;
  const float above = given == INFINITY ? NAN : nextafterf(given, INFINITY);  // the least number that is larger
  // ids [0, head) and [vocab - tail, vocab) one by one, the others in 16-byte pieces
  const int mis = (int)(((uintptr_t)x & 15) / sizeof(T)), head = min(mis ? V - mis : 0, a.vocab);
  const int pieces = (a.vocab - head) / V, tail = a.vocab - head - pieces * V;
  const uint4 *body = reinterpret_cast<const uint4 *>(x + head);
  const int token_piece = token < head ? -1 : (token - head) / V;
  LpSums sums = {-INFINITY, 0ull, 0ull};
  int higher = 0;
  float top = -INFINITY;  // this thread's largest
  auto push = [&](float v, int id, u64 bound) {
    const u64 key = lp_key(v, id);
    if (key < bound || id >= a.vocab) return;
    const int i = atomicAdd(&sh.count, 1);
    if (i < LP_LIST) sh.list[i] = key;
  };
  const int edge = tid < head ? tid : (tid < head + tail ? a.vocab - tail + (tid - head) : -1);
  const float edge_x = edge >= 0 ? Elem<T>::to_f(x[edge]) : -INFINITY;
  // visits the pieces in rounds of LP_LOADS loads that lie far apart, so that the first round samples the whole row
  const int rounds = (pieces + LP_THREADS * LP_LOADS - 1) / (LP_THREADS * LP_LOADS);
  const uint32_t none = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;  // -infinity
  auto load = [&](int i, uint4 *raw) {
#pragma unroll
    for (int u = 0; u < LP_LOADS; ++u) {
      const int p = (u * rounds + i) * LP_THREADS + tid;
      raw[u] = p < pieces ? __ldcs(body + p) : make_uint4(none, none, none, none);
    }
  };
  float thr = INFINITY;
  u64 bound = ~0ull;
  if (tid == 0) sh.count = 0;
  if (edge >= 0) {
    top = fmaxf(top, edge_x);
    if (edge_x > -INFINITY) sums.raise(edge_x);
    sums.add(edge_x, -INFINITY, sums.minus_ref());
    if (token >= 0) higher += edge_x > given || (edge_x == given && edge < token);
  }
  for (int i = 0; i < rounds; ++i) {
    uint4 raw[LP_LOADS];
    load(i, raw);
    float f[LP_LOADS][V], big = -INFINITY;
#pragma unroll
    for (int u = 0; u < LP_LOADS; ++u) {
      Vec16<T> z;
      z.raw = raw[u];
      z.unpack(f[u]);
#pragma unroll
      for (int j = 0; j < V; j += 2) big = fmax3(big, f[u][j], f[u][j + 1]);
    }
    if (big > sums.m) sums.raise(big);
    top = fmaxf(top, big);
    if (i == 0 && k > 0) {  // the whole CTA alike
      sh.most[tid] = co_weight_key(top);
      __syncthreads();
      if (warp == 0) {
        const uint32_t b = lp_bound(sh.most, k);
        if (lane == 0) sh.bound = b;
      }
      __syncthreads();
      bound = sh.bound > 0x007fffffu ? (u64)sh.bound << 32 : 0ull;  // above -infinity
      thr = bound ? lp_unkey(sh.bound) : LP_LOWEST;
      if (edge >= 0 && edge_x >= thr) push(edge_x, edge, bound);
    }
    const float minus_ref = sums.minus_ref();
#pragma unroll
    for (int u = 0; u < LP_LOADS; ++u)
#pragma unroll
      for (int j = 0; j < V; j += 2) sums.add(f[u][j], f[u][j + 1], minus_ref);
    if (big >= given) {
#pragma unroll
      for (int u = 0; u < LP_LOADS; ++u) {
        const int p = (u * rounds + i) * LP_THREADS + tid;
        if (p == token_piece && p < pieces) {
#pragma unroll
          for (int j = 0; j < V; ++j) higher += f[u][j] > given || (f[u][j] == given && head + p * V + j < token);
        } else {
          const float bar = p < token_piece ? given : above;
#pragma unroll
          for (int j = 0; j < V; ++j) higher += p < pieces && f[u][j] >= bar;
        }
      }
    }
    if (big >= thr) {
#pragma unroll
      for (int u = 0; u < LP_LOADS; ++u) {
        const int p = (u * rounds + i) * LP_THREADS + tid;
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (f[u][j] >= thr && p < pieces) push(f[u][j], head + p * V + j, bound);
      }
    }
  }
  // ---- the row's sums
  LpTotal total;
  {
    float s0, s1, t0, t1;
    f32x2_unpack(sums.s, s0, s1);
    f32x2_unpack(sums.t, t0, t1);
    total = {sums.m, s0 + s1, t0 + t1};
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    LpTotal other;
    other.m = __shfl_xor_sync(0xffffffffu, total.m, o);
    other.s = __shfl_xor_sync(0xffffffffu, total.s, o);
    other.t = __shfl_xor_sync(0xffffffffu, total.t, o);
    total.merge(other);
  }
  higher = __reduce_add_sync(0xffffffffu, higher);
  if (lane == 0) {
    sh.sums[warp] = total;
    sh.higher[warp] = higher;
  }
  if (k > 0) sh.most[tid] = co_weight_key(top);
  __syncthreads();
  total = sh.sums[0];
  higher = sh.higher[0];
#pragma unroll
  for (int w = 1; w < LP_WARPS; ++w) {
    total.merge(sh.sums[w]);
    higher += sh.higher[w];
  }
  const float log2_s = log2f(total.s), log_s = LP_LN2 * log2_s;
  if (tid == 0) {
    if (a.logprob) a.logprob[r] = token >= 0 ? (given - total.m) - log_s : 0.f;
    if (a.entropy) a.entropy[r] = LP_LN2 * (log2_s - total.t / total.s);
    if (a.rank) a.rank[r] = token >= 0 && given == given ? higher : -1;
  }
  if (k == 0) return;
  // ---- the list's best
  if (warp == 0) {
    const uint32_t b = lp_bound(sh.most, k);
    if (lane == 0) sh.bound = b;
  }
  __syncthreads();
  int n = sh.count;
  u64 low = sh.bound > 0x007fffffu ? (u64)sh.bound << 32 : 0ull;  // at least k reach it, or it is 0
  bool by_count = false;
  while (n < k || n > LP_LIST) {
    if (n < k) low = 0ull;
    else if (by_count || low == 0ull) {  // the bound is no better than before: the k-th of those in the list
      for (int i = tid; i < LP_LIST; i += LP_THREADS) {
        const u64 mine = sh.list[i];
        int at = 0;
        for (int j = 0; j < LP_LIST; ++j) at += sh.list[j] > mine;
        if (at == k - 1) sh.kth = mine;
      }
      __syncthreads();
      low = sh.kth;
    }
    by_count = true;
    __syncthreads();
    if (tid == 0) sh.count = 0;
    __syncthreads();
    if (edge >= 0) push(edge_x, edge, low);
    for (int p = tid; p < pieces; p += LP_THREADS) {
      Vec16<T> z;
      float f[V];
      z.raw = body[p];
      z.unpack(f);
#pragma unroll
      for (int j = 0; j < V; ++j) push(f[j], head + p * V + j, low);
    }
    __syncthreads();
    n = sh.count;
  }
  for (int i = tid; i < n; i += LP_THREADS) {
    const u64 mine = sh.list[i];
    if (mine < low) continue;
    int at = 0;
    for (int j = 0; j < n; ++j) at += sh.list[j] > mine;
    if (at < k) {
      const int id = lp_key_id(mine);
      a.top_id[(size_t)r * k + at] = id;
      a.top_logprob[(size_t)r * k + at] = (Elem<T>::to_f(x[id]) - total.m) - log_s;
    }
  }
}

}  // namespace

int launch_token_logprobs(cudaStream_t st, int dtype, const LogprobArgs &a, DevStatus *status) {
  if (a.n_rows == 0) return LAZY_OK;
  return co_launch(dtype == LAZY_F32 ? token_logprobs_kernel<float> : token_logprobs_kernel<bf16>, dim3((unsigned)a.n_rows),
                   dim3(LP_THREADS), 0, st, 1, false, a, status);
}

}  // namespace lazy
