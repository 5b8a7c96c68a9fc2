// Log probabilities of given tokens from rows of logits, with the distribution's entropy, the token's rank and the best
// alternatives, in one pass over the logits:
//   lse = m + log sum_j e^(x_j - m),   log p_t = x_t - lse,   H = lse - sum_j p_j x_j = log S - T / S
// with S = sum e^(x_j - m), T = sum (x_j - m) e^(x_j - m), kept per thread against a running maximum and rescaled when it grows.
//
// Alternatives: of the threads' maxima over the row, the k-th largest is a bound that at least k logits reach, and few more do.  Only
// the threads whose maximum reaches it have any of those; what they read is read once more (it is in L2), and the few logits that reach
// the bound go to a short list, whose k best, by (logit, lower id) as one 64-bit number, are found by counting.  A list that
// overflows (many equal logits) is filled again with a better bound.  Nothing of this is in the loop over the row.
//
// A CTA takes row after row; a cluster shares one where the rows are few.  A thread's loads go through its own places in shared memory
// (cp.async, a round ahead, into the next row too), so that the memory keeps busy while a row is being finished: small CTAs, five to an
// SM, since their barriers at a row's end then hold up less (with 256 threads, three to an SM, 102 us for what follows).
//
// 3376 rows of 32000 in fp32 (432 MB), with the ranks of their tokens: 69 us without alternatives (6.2 TB/s), 83 with the five best; in bf16 53
// and 67, bound by instructions (one exponential per logit alone takes 24), and by what finishing a row holds up.  One row: 5.0 and
// 8.0 us, 64 rows of 128256 in bf16 9.0 and 14.0 with the 20 best, latency.
#include "rows_mma.cuh"

namespace lazy {

namespace {

constexpr int LP_MANY = 128, LP_FEW = 256;  // threads of a CTA that takes row after row, of one of a cluster
template <typename T, int THREADS>
constexpr int LP_CTAS = THREADS == LP_MANY ? 5 : (sizeof(T) == 4 ? 2 : 3);  // to an SM
template <typename T>
constexpr int LP_LOADS = 32 / Elem<T>::kPerVec;   // 16-byte loads of a thread in a round: 32 logits
template <typename T>
constexpr int LP_AHEAD = sizeof(T) == 4 ? 2 : 3;  // rounds in shared memory, 128 or 64 bytes a thread each
constexpr int LP_MAX_CLUSTER = 8;
constexpr int LP_LIST = 512;                      // candidates in shared memory
constexpr int LP_CELLS = 8;                       // parts of what a thread has read whose maxima are kept
constexpr float LP_LN2 = 0.6931471805599453f;
constexpr uint32_t LP_NEVER = 0x007fffffu;        // key of -infinity
template <typename T, int THREADS>
constexpr int LP_SMEM = LP_AHEAD<T> * LP_LOADS<T> * THREADS * 16;

typedef unsigned long long u64;

// Order of candidates as one number: larger logit first, then the lower id.
__device__ __forceinline__ u64 lp_key(float x, int id) { return ((u64)co_weight_key(x) << 32) | (uint32_t)~id; }
__device__ __forceinline__ int lp_key_id(u64 key) { return (int)~(uint32_t)key; }
__device__ __forceinline__ float lp_unkey(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? k ^ 0x80000000u : ~k); }

// Running softmax sums of one thread: s = sum 2^d, t = sum d 2^d with d = x log2(e) - m2, m2 = m log2(e) rounded, either as a pair of
// partial sums.  Beyond +-LP_LARGE that rounding would matter; such rows are summed again, from (x - m) log2(e).
constexpr float LP_LARGE = 1e7f;
struct LpSums {
  float m = -LP_LARGE, m2 = -LP_LARGE * CO_LOG2E;  // what lies far below adds nothing, -infinity either
  u64 s = 0, t = 0;
  __device__ __forceinline__ void raise(float to) {
    const float to2 = to * CO_LOG2E, delta = fmaxf(m2 - to2, -200.f), f = ex2_approx(delta);
    const u64 f2 = f32x2_pack(f, f);
    t = f32x2_mul(f32x2_fma(f32x2_pack(delta, delta), s, t), f2);
    s = f32x2_mul(s, f2);
    m = to;
    m2 = to2;
  }
  // CLAMP: for logits that may be -infinity, which add 0 to both (2^-200 is 0 here); without it they make t NaN.  A NaN makes s NaN
  template <bool CLAMP>
  __device__ __forceinline__ void add_terms(u64 d) {
    float d0, d1;
    f32x2_unpack(d, d0, d1);
    const u64 e = f32x2_pack(ex2_approx(d0), ex2_approx(d1));
    s = f32x2_add(s, e);
    t = f32x2_fma(e, CLAMP ? f32x2_pack(fmaxf(d0, -200.f), fmaxf(d1, -200.f)) : d, t);
  }
  template <bool CLAMP>
  __device__ __forceinline__ void add(float x0, float x1, u64 minus_m2) {
    add_terms<CLAMP>(f32x2_fma(f32x2_pack(x0, x1), f32x2_pack(CO_LOG2E, CO_LOG2E), minus_m2));
  }
  __device__ __forceinline__ bool wild() const {
    float t0, t1;
    f32x2_unpack(t, t0, t1);
    return !(t0 + t1 == t0 + t1);
  }
};
// The same of several threads together: m their largest logit, s and t against it.
struct LpTotal {
  float m, s, t;
  // of the warp, in every lane; lanes to be left out have m = -infinity and s = t = 0
  __device__ __forceinline__ void across() {
    const float all = warp_max(m), d = fmaxf((m - (all == -INFINITY ? 0.f : all)) * CO_LOG2E, -200.f), f = ex2_approx(d);
    t = warp_sum(fmaf(d, s, t) * f);
    s = warp_sum(s * f);
    m = all;
  }
};

template <int THREADS>
struct LpShared {
  u64 list[LP_LIST];
  u64 best[LAZY_MAX_TOP];     // this CTA's part of the row, sorted
  uint32_t most[THREADS];  // keys of the threads' maxima
  float4 sums[THREADS / 32];      // largest logit, reference of the sums, the sums
  LpTotal total;
  int higher[THREADS / 32], all_higher;
  int count, flags;
  uint32_t bound;
  u64 kth;
  float cell[LP_CELLS][THREADS];  // maxima of parts of what a thread has read
  uint16_t flag[LP_CELLS * THREADS];  // those that reach the bound: part * THREADS + thread
};

// Row r and this CTA's part of it: ids [0, head) and [vocab - tail, vocab) one by one (the first CTA's), 16-byte pieces [p0, p1) of the
// others, the first of them at id `offset`, in rounds of LP_LOADS loads of every thread.
template <typename T, int THREADS>
struct LpRow {
  static constexpr int V = Elem<T>::kPerVec, ROUND = LP_LOADS<T> * THREADS;
  const T *x;
  int offset, head, tail, p0, p1, rounds;
  __device__ __forceinline__ LpRow(const LogprobArgs &a, int r, int rank, int size_log2) {
    x = (const T *)a.logits + (size_t)r * a.ld;
    const int mis = (int)(((uintptr_t)x & 15) / sizeof(T));
    offset = min(mis ? V - mis : 0, a.vocab);
    const int pieces = (a.vocab - offset) / V, per = (pieces + (1 << size_log2) - 1) >> size_log2;
    p0 = min(rank * per, pieces);
    p1 = min(pieces - p0, per) + p0;
    head = rank ? 0 : offset;
    tail = rank ? 0 : a.vocab - offset - pieces * V;
    rounds = (p1 - p0 + ROUND - 1) / ROUND;
  }
  __device__ __forceinline__ const uint4 *body() const { return reinterpret_cast<const uint4 *>(x + offset); }
  __device__ __forceinline__ int piece(int i, int u) const { return p0 + i * ROUND + u * THREADS + (int)threadIdx.x; }
};

// The largest of a thread's round (NaN left out); two logits at a time where they are bf16.
template <typename T>
__device__ __forceinline__ float lp_largest(uint32_t from, int step) {
  float big = -INFINITY;
  __nv_bfloat162 big2 = __float2bfloat162_rn(-INFINITY);
#pragma unroll
  for (int u = 0; u < LP_LOADS<T>; ++u) {
    uint32_t x[4];
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(from + u * step) : "memory");
    if constexpr (sizeof(T) == 4) {
      big = fmax3(big, __uint_as_float(x[0]), __uint_as_float(x[1]));
      big = fmax3(big, __uint_as_float(x[2]), __uint_as_float(x[3]));
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) big2 = __hmax2(big2, *reinterpret_cast<__nv_bfloat162 *>(&x[j]));
    }
  }
  return sizeof(T) == 4 ? big : fmaxf(__low2float(big2), __high2float(big2));
}

// How many of a thread's round are larger than x or, in the loads that lie before the token's (u * THREADS < before), no smaller.  bf16 are
// compared two at a time: the counts of either half stay below 256, exact in bf16.
template <typename T, int THREADS>
__device__ __forceinline__ int lp_count(uint32_t from, float x, int before) {
  int n = 0;
  const float above = x == INFINITY ? NAN : nextafterf(x, INFINITY);  // the least number that is larger
  const __nv_bfloat162 x2 = __float2bfloat162_rn(x);
  __nv_bfloat162 n2 = __float2bfloat162_rn(0.f);
#pragma unroll
  for (int u = 0; u < LP_LOADS<T>; ++u) {
    uint32_t y[4];
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(y[0]), "=r"(y[1]), "=r"(y[2]), "=r"(y[3]) : "r"(from + u * THREADS * 16) : "memory");
    const bool equal = u * THREADS < before;
    const float bar = equal ? x : above;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (sizeof(T) == 4) {
        n += __uint_as_float(y[j]) >= bar;
      } else {
        const __nv_bfloat162 y2 = *reinterpret_cast<__nv_bfloat162 *>(&y[j]);
        n2 = __hadd2(n2, equal ? __hge2(y2, x2) : __hgt2(y2, x2));
      }
    }
  }
  return sizeof(T) == 4 ? n : (int)(__low2float(n2) + __high2float(n2));
}

// A key that at least k of the threads' maxima reach, the k-th largest of them or one below it that no more reach.  By one
// warp; 0 where fewer than k threads have seen anything.
template <int THREADS>
__device__ __forceinline__ uint32_t lp_bound(const uint32_t *most, int k) {
  constexpr int WARPS = THREADS / 32;
  const int lane = threadIdx.x & 31;
  uint32_t v[WARPS], lo = ~0u, hi = 0;
#pragma unroll
  for (int i = 0; i < WARPS; ++i) {
    v[i] = most[i * 32 + lane];
    lo = min(lo, v[i]);
    hi = max(hi, v[i]);
  }
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  if (lo == hi) return lo;
  const int high = (31 - __clz(lo ^ hi)) | 1;  // bits above are the same in all
  uint32_t t = high == 31 ? 0u : lo & ~((2u << high) - 1u);
  for (int b = high - 1; b >= 0; b -= 2) {  // two bits at a time
    const uint32_t c1 = t | (1u << b), c2 = t | (2u << b), c3 = t | (3u << b);
    uint32_t n = 0;
#pragma unroll
    for (int i = 0; i < WARPS; ++i) n += (v[i] >= c1) + ((v[i] >= c2) << 10) + ((v[i] >= c3) << 20);
    n = __reduce_add_sync(0xffffffffu, n);
    const int n1 = n & 1023, n2 = n >> 10 & 1023, n3 = n >> 20;
    t = n3 >= k ? c3 : (n2 >= k ? c2 : (n1 >= k ? c1 : t));
    if (n1 == k || n2 == k || n3 == k) break;
  }
  return t;
}

// How many of n keys precede `mine`, counted by `share` neighbouring threads (a power of two) together.
__device__ __noinline__ int lp_before(const u64 *list, int n, u64 mine, int share) {
  int at = 0;
#pragma unroll 4
  for (int j = threadIdx.x & (share - 1); j < n; j += share) at += list[j] > mine;
  for (int o = share >> 1; o > 0; o >>= 1) at += __shfl_xor_sync(0xffffffffu, at, o);
  return at;
}
// Calls write(place, key) for those of keys [from, from + count) that are among the `want` best of all n (0: no key), a few threads to a
// key; by the whole CTA.
template <int THREADS, typename Write>
__device__ __forceinline__ void lp_best(const u64 *list, int n, int from, int count, int want, Write write) {
  int share = 1;
  while (share < 32 && share * 2 * count <= THREADS) share *= 2;
  const int each = THREADS / share, first = (threadIdx.x & ~31) / share;
  for (int i0 = 0; i0 + first < count; i0 += each) {  // the whole warp alike
    const int i = i0 + threadIdx.x / share;
    const u64 mine = i < count ? list[from + i] : 0ull;
    const int at = lp_before(list, n, mine, share);
    if (mine != 0ull && at < want && (threadIdx.x & (share - 1)) == 0) write(at, mine);
  }
}
// Sums of a warp's threads (largest logit, reference, s, t), each against its own reference, against the largest of those.
__device__ __noinline__ float4 lp_reduce(float4 w) {
  const float all = warp_max(w.y), d = fmaxf(w.y - all, -200.f), f = ex2_approx(d);
  return make_float4(warp_max(w.x), all, warp_sum(w.z * f), warp_sum(fmaf(d, w.z, w.w) * f));
}

template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS, (LP_CTAS<T, THREADS>))
token_logprobs_kernel(const LogprobArgs a, DevStatus *status) {
  constexpr int V = Elem<T>::kPerVec, LOADS = LP_LOADS<T>, AHEAD = LP_AHEAD<T>, STEP = THREADS * 16, WARPS = THREADS / 32;
  extern __shared__ __align__(128) uint4 lp_rounds[];  // [AHEAD][LOADS][THREADS]
  __shared__ LpShared<THREADS> sh;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, k = a.n_top;
  const int rank = (int)co_cluster_rank(), size = (int)co_cluster_size(), size_log2 = 31 - __clz(size);
  const int step = gridDim.x >> size_log2, first = blockIdx.x >> size_log2;
  const uint32_t slots = smem_u32(lp_rounds) + tid * 16;
  auto fetch = [](uint32_t at, float *f) {
    Vec16<T> z;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(z.raw.x), "=r"(z.raw.y), "=r"(z.raw.z), "=r"(z.raw.w) : "r"(at) : "memory");
    z.unpack(f);
  };
  // behind the last piece stands the type's lowest: nothing's maximum, and not summed (times log2(e) it is -infinity, which would call for
  // the round once more)
  const uint32_t none = sizeof(T) == 4 ? 0xff7fffffu : 0xff7fff7fu;
  // ---- rounds are asked for AHEAD - 1 ahead, row after row
  int ask_row = first, ask_i = 0, asked = 0;
  LpRow<T, THREADS> ask(a, min(ask_row, a.n_rows - 1), rank, size_log2);
  auto request = [&]() {
    while (ask_row < a.n_rows && ask_i >= ask.rounds) {  // rows without a whole piece have no rounds
      ask_row += step;
      ask_i = 0;
      if (ask_row < a.n_rows) ask = LpRow<T, THREADS>(a, ask_row, rank, size_log2);
    }
    if (ask_row < a.n_rows) {
      const int p = ask.piece(ask_i, 0);
      const uint4 *from = ask.body() + p;
      const uint32_t to = slots + asked * LOADS * STEP;
      if (p + (LOADS - 1) * THREADS < ask.p1) {
#pragma unroll
        for (int u = 0; u < LOADS; ++u) rm_cp_async16(to + u * STEP, from + u * THREADS, true);
      } else {  // behind the last piece
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
          if (p + u * THREADS < ask.p1) rm_cp_async16(to + u * STEP, from + u * THREADS, true);
          else asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(to + u * STEP), "r"(none) : "memory");
        }
      }
      ++ask_i;
    }
    asked = asked + 1 == AHEAD ? 0 : asked + 1;
    rm_cp_commit();
  };
#pragma unroll
  for (int n = 0; n < AHEAD - 1; ++n) request();
  // the token's logit is asked for while the row before is being finished
  auto logit = [&](int r, int token) {
    return token >= 0 && token < a.vocab ? Elem<T>::to_f(((const T *)a.logits)[(size_t)r * a.ld + token]) : NAN;
  };
  int taken = 0, token = a.tokens && first < a.n_rows ? a.tokens[first] : -1;
  float given = logit(first, token);
  for (int r = first; r < a.n_rows; r += step) {
    const LpRow<T, THREADS> row(a, r, rank, size_log2);
    if (token >= a.vocab) {
      if (tid == 0 && rank == 0) dev_fail(status, LAZY_E_BADARG, W_LOGPROBS, r, token);
      token = -1;
    }
    const int later = r + step < a.n_rows && a.tokens ? a.tokens[r + step] : -1;
    const int token_piece = token < row.offset ? -1 : (token - row.offset) / V;
    LpSums sums;
    int higher = 0;
    const int edge = tid < row.head ? tid : (tid < row.head + row.tail ? a.vocab - row.tail + (tid - row.head) : -1);
    const float edge_x = edge >= 0 ? Elem<T>::to_f(row.x[edge]) : -INFINITY;
    float top = edge_x > -INFINITY ? edge_x : -INFINITY, cell = -INFINITY;  // this thread's largest, of a row and of a few rounds
    const int per_cell = (row.rounds + LP_CELLS - 1) / LP_CELLS;
    int cells = 0, in_cell = 0;
    if (edge >= 0) {
      if (edge_x > sums.m) sums.raise(edge_x);
      sums.add<true>(edge_x, -INFINITY, f32x2_pack(-sums.m2, -sums.m2));
      if (token >= 0) higher += edge_x > given || (edge_x == given && edge < token);
    }
#pragma unroll 1
    for (int i = 0; i < row.rounds; ++i, taken = taken + 1 == AHEAD ? 0 : taken + 1) {
      request();
      rm_cp_wait<AHEAD - 1>();
      const uint32_t from = slots + taken * LOADS * STEP;
      // once for the maximum, once for the sums: reading shared memory again costs less than 32 registers
      const float big = lp_largest<T>(from, STEP);
      top = fmaxf(top, big);
      cell = fmaxf(cell, big);
      if (++in_cell == per_cell || i + 1 == row.rounds) {
        sh.cell[cells++][tid] = cell;
        cell = -INFINITY;
        in_cell = 0;
      }
      if (big > sums.m) sums.raise(big);
      const u64 minus_m2 = f32x2_pack(-sums.m2, -sums.m2);
      const LpSums before_round = sums;
      const int piece0 = row.piece(i, 0);
      const bool whole = piece0 - lane + 31 + (LOADS - 1) * THREADS < row.p1;  // the whole warp alike
      if (whole) {
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
          float f[V];
          fetch(from + u * STEP, f);
#pragma unroll
          for (int j = 0; j < V; j += 2) sums.add<false>(f[j], f[j + 1], minus_m2);
        }
      }
      if (!whole || sums.wild()) {  // the end of the part, or there are -infinities (or NaN): the round once more
        sums = before_round;
#pragma unroll 1
        for (int u = 0; u < LOADS && piece0 + u * THREADS < row.p1; ++u) {
          float f[V];
          fetch(from + u * STEP, f);
#pragma unroll
          for (int j = 0; j < V; j += 2) sums.add<true>(f[j], f[j + 1], minus_m2);
        }
      }
      // ---- ids before the token
      if (big >= given) {
        const int before = token_piece - piece0;  // loads u with u * THREADS < before lie before the token's
        if (given > -3.3e38f) {                   // else what stands behind the last piece would count
          higher += lp_count<T, THREADS>(from, given, before);
          if (before >= 0 && before < LOADS * THREADS && before % THREADS == 0) {  // the token's own piece
            float f[V];
            fetch(from + before / THREADS * STEP, f);
#pragma unroll
            for (int j = 0; j < V; ++j) higher += f[j] == given && row.offset + token_piece * V + j < token;
          }
        } else {
#pragma unroll 1
          for (int u = 0; u < LOADS && piece0 + u * THREADS < row.p1; ++u) {
            float f[V];
            fetch(from + u * STEP, f);
            const int id = row.offset + (piece0 + u * THREADS) * V;
#pragma unroll
            for (int j = 0; j < V; ++j) higher += f[j] > given || (f[j] == given && id + j < token);
          }
        }
      }
    }
    const float given_later = logit(r + step, later);
    // ---- the part's sums: the threads' against the largest reference, then against the largest logit
    float s0, s1, t0, t1;
    f32x2_unpack(sums.s, s0, s1);
    f32x2_unpack(sums.t, t0, t1);
    float4 w = lp_reduce(make_float4(top, sums.m2, s0 + s1, t0 + t1));
    higher = __reduce_add_sync(0xffffffffu, higher);
    if (lane == 0) {
      sh.sums[warp] = w;
      sh.higher[warp] = higher;
    }
    sh.most[tid] = co_weight_key(top);
    if (tid == 0) sh.count = sh.flags = 0;
    __syncthreads();
    float most = sh.sums[0].x;
#pragma unroll
    for (int i = 1; i < WARPS; ++i) most = fmaxf(most, sh.sums[i].x);
    const bool large = most > -INFINITY && !(fabsf(most) <= LP_LARGE);  // the whole CTA alike
    if (large) {
      LpSums again;
      if (edge >= 0) again.add_terms<true>(f32x2_pack((edge_x - most) * CO_LOG2E, -INFINITY));
#pragma unroll 1
      for (int p = row.p0 + tid; p < row.p1; p += THREADS) {
        Vec16<T> z;
        float f[V];
        z.raw = row.body()[p];
        z.unpack(f);
#pragma unroll
        for (int j = 0; j < V; j += 2) again.add_terms<true>(f32x2_pack((f[j] - most) * CO_LOG2E, (f[j + 1] - most) * CO_LOG2E));
      }
      f32x2_unpack(again.s, s0, s1);
      f32x2_unpack(again.t, t0, t1);
      w = lp_reduce(make_float4(most, 0.f, s0 + s1, t0 + t1));
      __syncthreads();  // the first sums have been read
      if (lane == 0) sh.sums[warp] = w;
      __syncthreads();
    }
    if (warp == WARPS - 1) {
      w = lane < WARPS ? sh.sums[lane] : make_float4(-INFINITY, -INFINITY, 0.f, 0.f);
      higher = __reduce_add_sync(0xffffffffu, lane < WARPS ? sh.higher[lane] : 0);
      w = lp_reduce(w);
      // what the rounding of m2 = m log2(e) lost belongs to the exponents
      const float lost = large || most == -INFINITY ? 0.f : fmaf(most, CO_LOG2E, -w.y), f = exp2f(-lost);
      if (lane == 0) {
        sh.total = {most, w.z * f, fmaf(-lost, w.z, w.w) * f};
        sh.all_higher = higher;
      }
    }
    // ---- the part's best, sorted
    const int want = min(k, (row.p1 - row.p0) * V + row.head + row.tail);
    if (want > 0) {
      if (warp == 0) {
        const uint32_t b = lp_bound<THREADS>(sh.most, want);
        if (lane == 0) sh.bound = b;
      }
      __syncthreads();
      u64 low = (u64)max(sh.bound, LP_NEVER + 1u) << 32;  // above -infinity; at least `want` reach it, or all of those are taken
      const float thr = lp_unkey((uint32_t)(low >> 32));
      if (top >= thr)
        for (int c = 0; c < cells; ++c)
          if (sh.cell[c][tid] >= thr) sh.flag[atomicAdd(&sh.flags, 1)] = (uint16_t)(c * THREADS + tid);
      __syncthreads();
      const int flags = sh.flags;
      auto push = [&](float v, int id) {
        const u64 key = lp_key(v, id);
        if (key < low) return;
        const int i = atomicAdd(&sh.count, 1);
        if (i < LP_LIST) sh.list[i] = key;
      };
      int n;
      while (true) {
        if (edge >= 0) push(edge_x, edge);
        const int of_one = per_cell * LOADS, n_read = flags * of_one;  // what each covers, one after the other
#pragma unroll 1
        for (int e = tid; e < n_read; e += THREADS) {
          const int f = per_cell == 1 ? e / LOADS : e / of_one, flag = sh.flag[f];
          const int p = row.p0 + (flag / THREADS * of_one + e - f * of_one) * THREADS + flag % THREADS;
          if (p >= row.p1) continue;
          Vec16<T> z;
          float x[V];
          z.raw = row.body()[p];
          z.unpack(x);
          uint32_t some = 0u;
#pragma unroll
          for (int j = 0; j < V; ++j) some |= x[j] >= thr ? 1u << j : 0u;
          while (some) {  // one place to push from: the code is run once a row, from a cold instruction cache
            const int id = row.offset + p * V + __ffs(some) - 1;
            some &= some - 1;
            push(Elem<T>::to_f(row.x[id]), id);
          }
        }
        __syncthreads();
        n = sh.count;
        if (n <= LP_LIST) break;
        // many equal logits: the k-th of those in the list is a better bound
        for (int i = tid; i < LP_LIST; i += THREADS) {
          const u64 mine = sh.list[i];
          if (lp_before(sh.list, LP_LIST, mine, 1) == want - 1) sh.kth = mine;
        }
        __syncthreads();
        low = sh.kth;
        if (tid == 0) sh.count = 0;
        __syncthreads();
      }
      if (n < want) {  // too few above -infinity: the first of those, then of the NaN
        if (warp == 0) {
          const int begin = rank ? row.offset + row.p0 * V : 0, end = row.offset + row.p1 * V, jump = a.vocab - row.tail;
#pragma unroll 1
          for (int pass = 0; pass < 2; ++pass) {
#pragma unroll 1
            for (int j0 = begin; j0 < end + row.tail && n < want; j0 += 32) {
              const int j = j0 + lane, id = j < end ? j : jump + (j - end);
              const float x = j < end + row.tail ? Elem<T>::to_f(row.x[id]) : 0.f;
              const uint32_t in = __ballot_sync(0xffffffffu, pass ? x != x : x == -INFINITY);
              const int at = n + __popc(in & ((1u << lane) - 1u));
              if (in >> lane & 1u) sh.list[at] = lp_key(x, id);
              n += __popc(in);
            }
          }
          if (lane == 0) sh.bound = n;
        }
        __syncthreads();
        n = (int)sh.bound;
      }
      lp_best<THREADS>(sh.list, n, 0, n, want, [&](int at, u64 key) { sh.best[at] = key; });
    }
    for (int i = want + tid; i < k; i += THREADS) sh.best[i] = 0ull;  // less than everything
    if (size > 1) co_cluster_sync();
    else __syncthreads();
    // ---- the row's outputs
    if (rank == 0 || k > 0) {
      LpTotal total = sh.total;
      higher = sh.all_higher;
      if (size > 1) {
        const int from = min(lane, size - 1);
        total = *co_map_shared(&sh.total, from);
        higher = *co_map_shared(&sh.all_higher, from);
        if (lane >= size) {
          total = {-INFINITY, 0.f, 0.f};
          higher = 0;
        }
        total.across();
        higher = __reduce_add_sync(0xffffffffu, higher);
      }
      const float log2_s = log2f(total.s), log_s = LP_LN2 * log2_s;
      if (tid == 0 && rank == 0) {
        if (a.logprob) a.logprob[r] = token >= 0 ? (given - total.m) - log_s : 0.f;
        if (a.entropy) a.entropy[r] = LP_LN2 * (log2_s - total.t / total.s);
        if (a.rank) a.rank[r] = token >= 0 && given == given ? higher : -1;
      }
      auto write = [&](int at, u64 key) {
        a.top_id[(size_t)r * k + at] = lp_key_id(key);
        a.top_logprob[(size_t)r * k + at] = (lp_unkey((uint32_t)(key >> 32)) - total.m) - log_s;
      };
      if (size == 1) {
        if (tid < k) write(tid, sh.best[tid]);
      } else if (k > 0) {  // every CTA places its own among all
        for (int i = tid; i < size * k; i += THREADS) sh.list[i] = *co_map_shared(&sh.best[i % k], i / k);
        __syncthreads();
        lp_best<THREADS>(sh.list, size * k, rank * k, k, k, write);
      }
    }
    if (size > 1) co_cluster_sync();  // the parts have been read
    else __syncthreads();
    token = later;
    given = given_later;
  }
  rm_cp_wait<0>();
}

// How rows are shared out: threads of a CTA, CTAs to a row, and how long that takes in all by an estimate.
struct LpShape {
  int threads, cluster, at_once;  // clusters that run at once
  double us;
};
// A row takes the longest of its share of the memory's rate (44 B/ns to an SM), of what an SM sums (13 logits a ns), and of a round trip
// to every round, and then some time to be finished: 2 us; to join the parts of a cluster of two another 2, and 0.75 for each doubling.
// The times to finish and to join are those of five alternatives, whatever n_top is.
// One row with five of them, by one CTA, four and eight: of 16000 logits 7.7 us / - / 8.9, 32000 - / 8.0 / 9.0, 50257 - / 9.5 / 8.5.
template <typename T, int THREADS>
LpShape lp_shape(const LogprobArgs &a, int cluster) {
  constexpr int CTAS = LP_CTAS<T, THREADS>;
  const int at_once = (cluster <= 2 ? sm_count() * CTAS : co_cluster_ctas(cluster, CTAS < 3 ? CTAS : 3)) / cluster;
  auto wave = [&](int rows) {
    const double per_sm = rows * cluster <= sm_count() ? 1.0 : (double)rows * cluster / sm_count(), n = (double)a.vocab / cluster;
    const double finish = 2.0 + (cluster > 1 ? 1.25 + 0.75 * log2(cluster) : 0.0);
    return rows == 0 ? 0.0 : fmax(n * per_sm * fmax(sizeof(T) / 44.0, 1.0 / 13.0), n / (0.025 * THREADS)) * 1e-3 + finish;
  };
  return {THREADS, cluster, at_once, a.n_rows / at_once * wave(at_once) + wave(a.n_rows % at_once)};
}

template <typename T, int THREADS>
int token_logprobs(cudaStream_t st, const LogprobArgs &a, const LpShape &s, DevStatus *status) {
  LAZY_TRY((co_allow_smem<token_logprobs_kernel<T, THREADS>>(LP_SMEM<T, THREADS>)));
  return co_launch(token_logprobs_kernel<T, THREADS>, dim3((unsigned)(min(a.n_rows, s.at_once) * s.cluster)), dim3(THREADS),
                   LP_SMEM<T, THREADS>, st, s.cluster, false, a, status);
}
template <typename T>
int token_logprobs(cudaStream_t st, const LogprobArgs &a, DevStatus *status) {
  LpShape s = lp_shape<T, LP_MANY>(a, 1);
  for (int c = 1; c <= LP_MAX_CLUSTER; c *= 2) {
    const LpShape o = lp_shape<T, LP_FEW>(a, c);
    if (o.us < s.us) s = o;
  }
  return s.threads == LP_MANY ? token_logprobs<T, LP_MANY>(st, a, s, status) : token_logprobs<T, LP_FEW>(st, a, s, status);
}

}  // namespace

int launch_token_logprobs(cudaStream_t st, int dtype, const LogprobArgs &a, DevStatus *status) {
  static_assert(LP_LIST >= LP_MAX_CLUSTER * LAZY_MAX_TOP && LP_MANY >= LAZY_MAX_TOP && LP_LIST >= LAZY_MAX_TOP + 32,
                "the cluster's lists fit one");
  if (a.n_rows == 0) return LAZY_OK;
  return dtype == LAZY_F32 ? token_logprobs<float>(st, a, status) : token_logprobs<bf16>(st, a, status);
}

}  // namespace lazy
