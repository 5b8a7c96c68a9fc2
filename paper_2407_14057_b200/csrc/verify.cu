// Verification of drafted tokens.  Draft t (token x_t, drawn from q_t) is accepted iff u_t q_t(x_t) < p_t(x_t) and
// every draft before it was; behind the accepted ones comes one token from the distribution that makes the
// whole sequence a sample of the target: max(p - q, 0) (normalised) after a rejection, p behind the last draft.  It is
// taken by inversion: the first id whose running sum exceeds u times the total.
//
// What has to be read is one row of p (and one of q after a rejection) per sequence, wherever the scan ends; the
// other rows are touched at the drafted ids only.  A cluster of CTAs shares the row: each sums its contiguous
// part, the totals meet in distributed shared memory, and the one warp whose part holds the crossing reads its
// few hundred values again (from L2).  Sums run in 64 bits: with 32 the running sum's rounding would move the crossing to a
// neighbouring id about once in a few hundred draws at a vocabulary of 32000.
#include "cache_ops.cuh"

namespace lazy {

namespace {

constexpr int VF_THREADS = 512, VF_WARPS = VF_THREADS / 32, VF_MAX_CLUSTER = 8;

__device__ __forceinline__ double warp_sum_f64(double v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Weight of id j: p[j], less q[j] (row_q) or nothing at all for the one rejected id; never negative, NaN counts 0.
__device__ __forceinline__ float vf_weight(float p, float q, int j, int zeroed) {
  return j == zeroed ? 0.f : fmaxf(p - q, 0.f);
}

// Four consecutive weights from id j on (j a multiple of 4); ids past `end` weigh nothing.
__device__ __forceinline__ void vf_load4(const float *row_p, const float *row_q, int j, int end, bool vec, int zeroed,
                                         float *w) {
  if (vec && j + 4 <= end) {
    const float4 a = *reinterpret_cast<const float4 *>(row_p + j);
    float4 b = make_float4(0.f, 0.f, 0.f, 0.f);
    if (row_q) b = *reinterpret_cast<const float4 *>(row_q + j);
    w[0] = vf_weight(a.x, b.x, j, zeroed);
    w[1] = vf_weight(a.y, b.y, j + 1, zeroed);
    w[2] = vf_weight(a.z, b.z, j + 2, zeroed);
    w[3] = vf_weight(a.w, b.w, j + 3, zeroed);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = j + i < end ? vf_weight(row_p[j + i], row_q ? row_q[j + i] : 0.f, j + i, zeroed) : 0.f;
  }
}

// One cluster per sequence.
__global__ void __launch_bounds__(VF_THREADS)
verify_kernel(const float *__restrict__ p, int ldp, const float *__restrict__ q, int ldq,
              const int32_t *__restrict__ draft, const int32_t *__restrict__ cu, int n_draft, int max_draft, int vocab,
              const float *__restrict__ u_accept, const float *__restrict__ u_sample, int32_t *__restrict__ n_accept,
              int32_t *__restrict__ tokens, int vec, DevStatus *status) {
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
          const double px = p[(size_t)(d0 + s + t) * ldp + x];
          const double qx = q ? (double)q[(size_t)(d0 + t) * ldq + x] : 1.0;
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
  const float *row_p = p + (size_t)(d0 + s + acc) * ldp;
  const float *row_q = acc < T && q ? q + (size_t)(d0 + acc) * ldq : nullptr;
  int zeroed = acc < T && !q ? draft[d0 + acc] : -1;
  // ---- this warp's contiguous part of the row, in multiples of 128 ids
  const int parts = size * VF_WARPS, part = rank * VF_WARPS + warp;
  const int len = ((vocab + parts - 1) / parts + 127) / 128 * 128;
  const int begin = (int)min((long long)part * len, (long long)vocab), end = min(vocab - begin, len) + begin;
  for (int pass = 0;; ++pass) {
    double sum = 0.0;
    for (int j0 = begin; j0 < end; j0 += 128) {
      float w[4];
      vf_load4(row_p, row_q, j0 + lane * 4, end, vec != 0, zeroed, w);
      sum += ((double)w[0] + (double)w[1]) + ((double)w[2] + (double)w[3]);
    }
    sum = warp_sum_f64(sum);
    if (lane == 0) warp_total[warp] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
      double t = 0.0;
      for (int w = 0; w < VF_WARPS; ++w) t += warp_total[w];
      cta_total = t;
    }
    co_cluster_sync();
    double cta[VF_MAX_CLUSTER], total = 0.0;
#pragma unroll
    for (int r = 0; r < VF_MAX_CLUSTER; ++r) {
      cta[r] = r < size ? *co_map_shared(&cta_total, r) : 0.0;
      total += cta[r];
    }
    co_cluster_sync();  // every total has been read: a second pass may write again, a CTA may leave
    if (!(total > 0.0) && (row_q || zeroed >= 0) && pass == 0) {
      row_q = nullptr;  // the draft's distribution covers the target's (equal but for rounding): the target's itself
      zeroed = -1;
      continue;
    }
    // ---- the crossing lies in the first CTA, and there in the first warp's part, whose running sum exceeds the
    // bar; where rounding (or an infinite total) leaves none, in the last with any weight.  All threads decide
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
    if (owner_cta == rank) {
      double run = base;
      crossed = false;
      for (int w = 0; w < VF_WARPS && !crossed; ++w) {
        const double t = warp_total[w];
        if (t > 0.0) {
          owner = w;
          base = run;
          crossed = run + t > bar;
        }
        run += t;
      }
    }
    if (owner == warp) {
      double run = base;
      int found = -1, last_pos = -1;
      for (int j0 = begin; j0 < end && found < 0; j0 += 128) {
        const int j = j0 + lane * 4;
        float w[4];
        vf_load4(row_p, row_q, j, end, vec != 0, zeroed, w);
        const double mine = ((double)w[0] + (double)w[1]) + ((double)w[2] + (double)w[3]);
        double incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const double up = __shfl_up_sync(0xffffffffu, incl, o);
          if (lane >= o) incl += up;
        }
        double at = run + (incl - mine);
        int hit = -1;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          at += (double)w[i];
          if (hit < 0 && w[i] > 0.f && at > bar) hit = j + i;
          if (w[i] > 0.f) last_pos = j + i;
        }
        const uint32_t hits = __ballot_sync(0xffffffffu, hit >= 0);
        if (hits) found = __shfl_sync(0xffffffffu, hit, __ffs(hits) - 1);
        run += __shfl_sync(0xffffffffu, incl, 31);
      }
      if (found < 0) {  // the two orders of summation round apart at the part's very end
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) last_pos = max(last_pos, __shfl_xor_sync(0xffffffffu, last_pos, o));
        found = last_pos;
      }
      if (lane == 0) tokens[(size_t)s * (max_draft + 1) + acc] = found;
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
  const int vec = !((uintptr_t)p & 15) && ldp % 4 == 0 && (!q || (!((uintptr_t)q & 15) && ldq % 4 == 0));
  return co_launch(verify_kernel, dim3((unsigned)n_seqs * cluster), dim3(VF_THREADS), 0, st, cluster, false, p, ldp, q,
                   ldq, draft, cu_draft, n_draft, max_draft, vocab, u_accept, u_sample, n_accept, tokens, vec, status);
}

}  // namespace lazy
