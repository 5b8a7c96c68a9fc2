// Verification of drafted tokens.  Draft t (token x_t, drawn from q_t) is accepted iff u_t q_t(x_t) < p_t(x_t) and
// every draft before it was; behind the accepted ones comes one token from the distribution that makes the
// whole sequence a sample of the target: max(p - q, 0) (normalised) after a rejection, p behind the last draft.  It is
// taken by inversion: the first id whose running sum exceeds u times the total.
//
// What has to be read is one row of p (and one of q after a rejection) per sequence, wherever the scan ends; the
// other rows are touched at the drafted ids only.  A cluster of CTAs shares the row: each sums its contiguous
// part, the totals meet in distributed shared memory, and the one warp whose part holds the crossing reads its
// few hundred values again (from L2).  Sums run in 64 bits, differences included: with 32 the running sum's rounding would
// move the crossing to a neighbouring id about once in a few hundred draws at a vocabulary of 32000.  One request, 32000
// ids: 6.4 us, the latency of three rounds of loads and two scans; 128 requests of up to 7 drafts: 12.6 us (31 MB).
#include "attn_common.cuh"
#include "cache_ops.cuh"

namespace lazy {

namespace {

constexpr int VF_THREADS = 512, VF_WARPS = VF_THREADS / 32, VF_MAX_CLUSTER = 8;

__device__ __forceinline__ double warp_sum_f64(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// A probability as the caller has it: negative ones and NaN count as 0 (a negative one of the draft model's would give its id
// a weight that the target does not).
__device__ __forceinline__ float vf_prob(float x) { return fmaxf(x, 0.f); }
// The same in 64 bits, an infinite one as the largest number.
__device__ __forceinline__ double vf_prob_f64(float x) { return (double)fminf(vf_prob(x), 3.402823466e38f); }

// Weights max(p - q, 0) of two ids after a rejection, as the sum of the result and `rest`, what the subtraction in 32 bits
// rounded off (exact, as the larger of p and q is subtracted from).  Infinities make one of them infinite or NaN.
__device__ __forceinline__ unsigned long long vf_less_x2(float p0, float p1, float q0, float q1, unsigned long long &rest) {
  const unsigned long long minus = f32x2_pack(-1.f, -1.f);
  q0 = vf_prob(q0);
  q1 = vf_prob(q1);
  const unsigned long long q = f32x2_pack(q0, q1), most = f32x2_pack(fmaxf(p0, q0), fmaxf(p1, q1)), w = f32x2_fma(q, minus, most);
  rest = f32x2_fma(q, minus, f32x2_fma(w, minus, most));
  return w;
}

// The weights of one row.  VEC: rows and vocabulary are multiples of four ids and 16-byte aligned.
template <bool VEC>
struct VfRow {
  const float *p, *q;  // q NULL: nothing is taken off
  int zeroed;          // id without weight, or -1 (always, where q is there)
  bool wild;           // there are infinities among the weights
  __device__ __forceinline__ double at(int j) const {
    return j == zeroed ? 0.0 : fmax(vf_prob_f64(p[j]) - (q ? vf_prob_f64(q[j]) : 0.0), 0.0);
  }
  // Sum over ids first, first + stride, ... < end (four consecutive ones each with VEC).  What 32 bits lose of the
  // differences is added up as well (2^-44 of the sum is left): without it a crossing would move to a neighbouring id now
  // and then.  Subtracting in 64 bits throughout, with another conversion per id, takes 128 requests 12.5 us with their rows
  // in L2, 10.3 so.
  __device__ __forceinline__ double sum(int first, int end, int stride) const {
    if (wild) {
      double total = 0.0;
      for (int j0 = first; j0 < end; j0 += stride)
        for (int j = j0; j < j0 + (VEC ? 4 : 1); ++j) total += at(j);
      return total;
    }
    return q ? sum_of<true>(first, end, stride) : sum_of<false>(first, end, stride);
  }
  template <bool Q>
  __device__ __forceinline__ double sum_of(int first, int end, int stride) const {
    constexpr int UNROLL = 8, W = VEC ? 4 : 2;  // loads of a row in flight; of two ids the second is not there without VEC
    double total = 0.0;
    for (int j0 = first; j0 < end; j0 += UNROLL * stride) {
      float x[UNROLL][W], y[UNROLL][W];
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        const int j = j0 + u * stride;
        if (VEC) {
          float4 z = make_float4(0.f, 0.f, 0.f, 0.f);
          *reinterpret_cast<float4 *>(x[u]) = j < end ? *reinterpret_cast<const float4 *>(p + j) : z;
          if (Q) *reinterpret_cast<float4 *>(y[u]) = j < end ? *reinterpret_cast<const float4 *>(q + j) : z;
        } else {
          x[u][0] = j < end ? p[j] : 0.f;
          if (Q) y[u][0] = j < end ? q[j] : 0.f;
          x[u][1] = y[u][1] = 0.f;
        }
      }
      unsigned long long rests = 0ull;
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        const int j = j0 + u * stride;
        float w[W];
#pragma unroll
        for (int i = 0; i < W; i += 2) {
          if (Q) {
            unsigned long long rest;
            f32x2_unpack(vf_less_x2(x[u][i], x[u][i + 1], y[u][i], y[u][i + 1], rest), w[i], w[i + 1]);
            rests = f32x2_add(rests, rest);
          } else {
            w[i] = j + i == zeroed ? 0.f : vf_prob(x[u][i]);
            w[i + 1] = j + i + 1 == zeroed ? 0.f : vf_prob(x[u][i + 1]);
          }
        }
        if (VEC) total += ((double)w[0] + (double)w[1]) + ((double)w[2] + (double)w[3]);
        else total += (double)w[0];
      }
      if (Q) {
        float r0, r1;
        f32x2_unpack(rests, r0, r1);
        total += (double)(r0 + r1);
      }
    }
    return total;
  }
};

__device__ __forceinline__ double warp_inclusive_f64(double v) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const double up = __shfl_up_sync(0xffffffffu, v, o);
    if ((int)(threadIdx.x & 31) >= o) v += up;
  }
  return v;
}

// First id of [begin, end) whose running sum, from `run` on, exceeds the bar; if rounding leaves none, the last one with any
// weight (-1: none has).  By a warp: every lane sums a contiguous piece, one scan finds the piece, then its ids 32 at a time.
template <bool VEC>
__device__ __forceinline__ int vf_crossing(const VfRow<VEC> &row, int begin, int end, double run, double bar) {
  const int lane = threadIdx.x & 31;
  const int piece = ((end - begin + 31) / 32 + 3) / 4 * 4;
  const int b = min(begin + lane * piece, end), e = min(b + piece, end);
  const double mine = row.sum(b, e, VEC ? 4 : 1), incl = warp_inclusive_f64(mine);
  const uint32_t over = __ballot_sync(0xffffffffu, mine > 0.0 && run + incl > bar), any = __ballot_sync(0xffffffffu, mine > 0.0);
  if (!any) return -1;
  const int who = over ? __ffs(over) - 1 : 31 - __clz(any);
  run += __shfl_sync(0xffffffffu, incl - mine, who);
  const int b0 = begin + who * piece, e0 = min(b0 + piece, end);
  int last = -1;
  for (int j0 = b0; j0 < e0; j0 += 32) {
    const int j = j0 + lane;
    const double w = j < e0 ? row.at(j) : 0.0;
    const double at = run + warp_inclusive_f64(w);
    const uint32_t hit = __ballot_sync(0xffffffffu, w > 0.0 && at > bar), some = __ballot_sync(0xffffffffu, w > 0.0);
    if (hit) return j0 + __ffs(hit) - 1;
    if (some) last = j0 + 31 - __clz(some);
    run = __shfl_sync(0xffffffffu, at, 31);
  }
  return last;
}

// One cluster per sequence.
template <bool VEC>
__global__ void __launch_bounds__(VF_THREADS)
verify_kernel(const float *__restrict__ p, int ldp, const float *__restrict__ q, int ldq,
              const int32_t *__restrict__ draft, const int32_t *__restrict__ cu, int n_draft, int max_draft, int vocab,
              const float *__restrict__ u_accept, const float *__restrict__ u_sample, int32_t *__restrict__ n_accept,
              int32_t *__restrict__ tokens, DevStatus *status) {
  __shared__ double warp_total[VF_WARPS];
  __shared__ double cta_total;
  __shared__ int s_acc;
  const int rank = (int)co_cluster_rank(), size = (int)co_cluster_size();
  const int s = blockIdx.x / size, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int d0, T;
  if (!co_span(cu, s, n_draft, max_draft, status, W_VERIFY, d0, T)) return;  // the whole cluster alike
  // ---- accepted drafts: every CTA finds the same count
  if (warp == 0) {
    int acc = 0;
    for (int t0 = 0; t0 < T; t0 += 32) {
      const int t = t0 + lane;
      bool ok = false;
      if (t < T) {
        const int x = draft[d0 + t];
        if (x >= 0 && x < vocab) {
          const double px = vf_prob(p[(size_t)(d0 + s + t) * ldp + x]);
          const double qx = q ? (double)vf_prob(q[(size_t)(d0 + t) * ldq + x]) : 1.0;
          ok = (double)u_accept[d0 + t] * qx < px;  // exact: 24 by 24 bits in 53
        } else if (rank == 0) {
          dev_fail(status, LAZY_E_BADARG, W_VERIFY, d0 + t, x);
        }
      }
      const uint32_t good = __ballot_sync(0xffffffffu, ok);
      if (good != 0xffffffffu) {
        acc = t0 + __ffs(~good) - 1;
        break;
      }
      acc = t0 + 32;
    }
    if (lane == 0) s_acc = min(acc, T);
  }
  __syncthreads();
  const int acc = s_acc;
  VfRow<VEC> row = {p + (size_t)(d0 + s + acc) * ldp, acc < T && q ? q + (size_t)(d0 + acc) * ldq : nullptr,
                    acc < T && !q ? draft[d0 + acc] : -1, false};
  // ---- this warp's contiguous part of the row, in multiples of 128 ids
  const int parts = size * VF_WARPS, part = rank * VF_WARPS + warp;
  const int len = ((vocab + parts - 1) / parts + 127) / 128 * 128;
  const int begin = (int)min((long long)part * len, (long long)vocab), end = min(vocab - begin, len) + begin;
  while (true) {
    const double sum = warp_sum_f64(row.sum(begin + lane * (VEC ? 4 : 1), end, VEC ? 128 : 32));
    if (lane == 0) warp_total[warp] = sum;
    __syncthreads();
    const double mine = lane < VF_WARPS ? warp_total[lane] : 0.0;
    if (warp == 0) {
      const double t = warp_sum_f64(mine);
      if (lane == 0) cta_total = t;
    }
    co_cluster_sync();
    double cta[VF_MAX_CLUSTER], total = 0.0;
#pragma unroll
    for (int r = 0; r < VF_MAX_CLUSTER; ++r) {
      cta[r] = r < size ? *co_map_shared(&cta_total, r) : 0.0;
      total += cta[r];
    }
    co_cluster_arrive();  // when all have, every total has been read: a second pass may write again, a CTA may leave
    if (!row.wild && !(total <= 1.7976931348623157e308)) {
      co_cluster_wait();
      row.wild = true;
      continue;
    }
    if (!(total > 0.0) && (row.q || row.zeroed >= 0)) {
      co_cluster_wait();
      row.q = nullptr;  // the draft's distribution covers the target's (equal but for rounding): the target's itself
      row.zeroed = -1;
      continue;
    }
    // ---- the crossing lies in the first CTA, and there in the first warp's part, whose running sum exceeds the
    // bar; where rounding leaves none, in the last with any weight.  All threads decide
    // alike from the same numbers.
    const double bar = (double)u_sample[s] * total;
    int owner_cta = -1, owner = -1;
    double base = 0.0, run0 = 0.0;
    bool crossed = false;
#pragma unroll
    for (int r = 0; r < VF_MAX_CLUSTER; ++r) {
      if (!crossed && cta[r] > 0.0) {
        owner_cta = r;
        base = run0;
        crossed = run0 + cta[r] > bar;
      }
      run0 += cta[r];
    }
    if (owner_cta == rank) {  // lane w: warp w
      const double incl = warp_inclusive_f64(mine);
      const uint32_t over = __ballot_sync(0xffffffffu, mine > 0.0 && base + incl > bar), any = __ballot_sync(0xffffffffu, mine > 0.0);
      owner = over ? __ffs(over) - 1 : 31 - __clz(any);
      base += __shfl_sync(0xffffffffu, incl - mine, owner & 31);
    }
    if (owner == warp) {
      const int token = vf_crossing<VEC>(row, begin, end, base, bar);
      if (lane == 0) tokens[(size_t)s * (max_draft + 1) + acc] = token;
    }
    if (rank == 0) {
      if (threadIdx.x == 0) {
        n_accept[s] = acc;
        if (!(total > 0.0)) {
          tokens[(size_t)s * (max_draft + 1) + acc] = -1;
          dev_fail(status, LAZY_E_BADARG, W_VERIFY, d0 + s + acc, -1);
        }
      }
      for (int t = threadIdx.x; t <= max_draft; t += VF_THREADS)
        if (t != acc) tokens[(size_t)s * (max_draft + 1) + t] = t < acc ? draft[d0 + t] : -1;
    }
    __syncwarp();
    co_cluster_wait();
    return;
  }
}

}  // namespace

int launch_verify(cudaStream_t st, const float *p, int ldp, const float *q, int ldq, const int32_t *draft,
                  const int32_t *cu_draft, int n_seqs, int n_draft, int max_draft, int vocab, const float *u_accept,
                  const float *u_sample, int32_t *n_accept, int32_t *tokens, DevStatus *status) {
  if (n_seqs == 0) return LAZY_OK;
  int cluster = 1;
  while (cluster < VF_MAX_CLUSTER && (long long)n_seqs * cluster < sm_count() && vocab > cluster * VF_WARPS * 128) cluster *= 2;
  const bool vec = vocab % 4 == 0 && !((uintptr_t)p & 15) && ldp % 4 == 0 && (!q || (!((uintptr_t)q & 15) && ldq % 4 == 0));
  return co_launch(vec ? verify_kernel<true> : verify_kernel<false>, dim3((unsigned)n_seqs * cluster), dim3(VF_THREADS), 0, st,
                   cluster, false, p, ldp, q, ldq, draft, cu_draft, n_draft, max_draft, vocab, u_accept, u_sample, n_accept,
                   tokens, status);
}

}  // namespace lazy
