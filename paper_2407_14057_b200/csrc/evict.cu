// Eviction from a prompt's cache by accumulated attention weight: of every (sequence, key/value head) the newest
// n_recent rows stay, and of the older ones those with the largest weight, up to the budget; equal weights go
// to the lower row.  Heads choose for themselves, so slot t of two heads may hold different tokens.
//
// One launch, a few CTAs per (sequence, head).  Each of them makes the whole selection for itself (which needs no word
// between them): a radix select over order-preserving keys held in shared memory (of few keys, a comparison of each with all)
// finds the weight at the last kept rank, every warp counts the kept rows of its contiguous part, and after one scan over the warps the rows are listed
// in row order without a barrier per chunk.  A CTA lists and then copies only its share of the slots.  The copy is what
// is bound by memory: kept rows are read and written once.  A prompt of 3376 rows on 32 heads cut to 1024 slots: 15.2 us (34 MB,
// 4.6 us of it the selection, 5.3 the copy); eight prompts of 1 to 16384 rows on 8 heads cut to 2048: 31.5 us (119 MB, 3.8 TB/s).
#include "cache_ops.cuh"

namespace lazy {

namespace {

constexpr int ES_THREADS = 1024, ES_WARPS = ES_THREADS / 32;
constexpr int ES_BINS = 2048;      // 11-bit digits
constexpr int ES_COPIES = 4;       // of the histogram, by lane: weights crowd in a few exponents
constexpr int ES_KEYS = 45056;     // keys held in shared memory (176 KiB); longer sequences are read again per pass
constexpr int ES_PITCH = ES_BINS + 8;  // copies start 8 banks apart
constexpr int ES_HIST = ES_COPIES * ES_PITCH;
constexpr int ES_SMEM = (ES_HIST + ES_KEYS) * 4;
// Keys that are compared one with another instead of by digits: a bin of a 3376-row prompt's weights holds a hundred, and two
// more digits would take 2.1 us where comparing takes 1; comparing 250 takes as long as a digit.
constexpr int ES_FEW = 192;
constexpr int ES_BATCH = 8;        // weights in flight per thread
constexpr int EG_PIECES = 4;       // 16-byte pieces of K and of V in flight per thread
constexpr int ES_MAX_PARTS = 8;    // CTAs per (sequence, head)

// The bin that holds rank `left` (1 = the largest) when counted from the top, by the first ES_SCAN threads (all 1024 would
// take four times as long: the scan is bound by instruction issue).  Writes {bin, rows above it, rows in it} to found.
constexpr int ES_SCAN = 256, ES_PER = ES_BINS / ES_SCAN;
__device__ __forceinline__ void find_bin(const int *hist, int copies, int bins, int left, int *warp_sums, int *found) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int b0 = bins - ES_PER * ((int)threadIdx.x + 1);  // this thread's bins: [b0, b0 + ES_PER)
  int c[ES_PER], sum = 0;
#pragma unroll
  for (int i = 0; i < ES_PER; ++i) c[i] = 0;
  if (b0 >= 0)
    for (int k = 0; k < copies; ++k)
#pragma unroll
      for (int i = 0; i < ES_PER; i += 4) {
        const int4 x = *reinterpret_cast<const int4 *>(&hist[k * ES_PITCH + b0 + i]);
        c[i] += x.x;
        c[i + 1] += x.y;
        c[i + 2] += x.z;
        c[i + 3] += x.w;
      }
#pragma unroll
  for (int i = 0; i < ES_PER; ++i) sum += c[i];
  int incl = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int up = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += up;
  }
  if (lane == 31) warp_sums[warp] = incl;
  asm volatile("bar.sync 1, %0;" ::"n"(ES_SCAN) : "memory");
  int above = __reduce_add_sync(0xffffffffu, lane < warp ? warp_sums[lane] : 0) + incl - sum;
  if (above < left && left <= above + sum) {
#pragma unroll
    for (int i = ES_PER - 1; i >= 0; --i) {
      if (above < left && left <= above + c[i]) {
        found[0] = b0 + i;
        found[1] = above;
        found[2] = c[i];
      }
      above += c[i];
    }
  }
}

// The key at rank `left` of m <= ES_FEW of them (zeros behind them), each compared with all; written to found as find_bin does.
__device__ __forceinline__ void find_key(const uint32_t *few, int m, int left, int *found) {
  if ((int)threadIdx.x >= m) return;
  const uint32_t mine = few[threadIdx.x];
  int above = 0, reach = 0;  // keys above, and above or equal
#pragma unroll 2
  for (int j = 0; j < m; j += 8) {
    const uint4 a = *reinterpret_cast<const uint4 *>(few + j), b = *reinterpret_cast<const uint4 *>(few + j + 4);
    const uint32_t key[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      above += key[i] > mine;
      reach += key[i] >= mine;
    }
  }
  if (mine == 0u) reach = m;  // without the zeros behind
  if (above < left && left <= reach) {  // equal keys write the same
    found[0] = (int)mine;
    found[1] = above;
    found[2] = reach - above;
  }
}

// grid (parts, n_kv_heads, n_seqs).  idx[s, g]: the kept rows by slot; vecs: 16-byte pieces per row.
__global__ void __launch_bounds__(ES_THREADS, 1)
evict_kernel(const uint4 *__restrict__ k, const uint4 *__restrict__ v, long long ld, int vecs,
             const int32_t *__restrict__ pos, const float *__restrict__ mass, int n_total, const int32_t *__restrict__ cu,
             int max_len, int budget, int n_recent, int32_t *__restrict__ idx, uint4 *__restrict__ kc,
             uint4 *__restrict__ vc, float *__restrict__ cmass, int32_t *__restrict__ cpos, int32_t *__restrict__ clen, int cap,
             DevStatus *status) {
  extern __shared__ __align__(16) uint32_t es_smem[];
  int *hist = reinterpret_cast<int *>(es_smem);
  uint32_t *keys = es_smem + ES_HIST;
  __shared__ int warp_sums[2][ES_WARPS];
  __shared__ int found[3];  // by find_bin, find_key
  __shared__ __align__(16) uint32_t few[ES_FEW];
  __shared__ int n_few;
  const int g = blockIdx.y, s = blockIdx.z, Hkv = gridDim.y;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const size_t sg = (size_t)s * Hkv + g;
  int32_t *list = idx + sg * budget;
  int start, n;
  if (!co_span(cu, s, n_total, max_len, status, W_EVICT, start, n)) return;
  const int keep = min(n, budget);
  if (blockIdx.x == 0 && threadIdx.x == 0) clen[sg] = keep;
  const int share = (keep + gridDim.x - 1) / gridDim.x;
  const int first = min((int)blockIdx.x * share, keep), last = min(first + share, keep);  // this CTA's slots
  if (first == last) return;
  const float *m = mass + (size_t)g * n_total + start;
  const int old = n - min(n_recent, keep);  // rows that compete
  const int need = keep - (n - old);        // how many of them stay
  // the newest rows, and all rows where all stay: slot t holds row t + (n - keep)
  for (int t = max(first, need == old ? 0 : need) + threadIdx.x; t < last; t += ES_THREADS) list[t] = start + n - keep + t;
  if (need > 0 && need < old && first < need) {
    const bool held = old <= ES_KEYS;
    if (held)
      for (int i0 = threadIdx.x; i0 < old; i0 += ES_THREADS * ES_BATCH) {
        float w[ES_BATCH];
#pragma unroll
        for (int i = 0; i < ES_BATCH; ++i) w[i] = i0 + i * ES_THREADS < old ? m[i0 + i * ES_THREADS] : 0.f;
#pragma unroll
        for (int i = 0; i < ES_BATCH; ++i)
          if (i0 + i * ES_THREADS < old) keys[i0 + i * ES_THREADS] = co_weight_key(w[i]);
      }
    auto key_of = [&](int i) { return held ? keys[i] : co_weight_key(m[i]); };
    uint32_t prefix = 0u, mask = 0u;
    int left = need;
    if (threadIdx.x < ES_FEW) few[threadIdx.x] = 0u;
    if (old <= ES_FEW) {
      __syncthreads();
      if ((int)threadIdx.x < old) few[threadIdx.x] = keys[threadIdx.x];
      __syncthreads();
      find_key(few, old, left, found);
      __syncthreads();
      prefix = (uint32_t)found[0];
      left -= found[1];
    } else {
      for (int pass = 0; pass < 3; ++pass) {  // digits of 11, 11 and 10 bits from the top
        const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0), bins = pass == 2 ? 1024 : ES_BINS;
        const int copies = pass == 0 ? ES_COPIES : 1;  // later passes count the few rows of one bin
        for (int i = threadIdx.x; i < copies * ES_PITCH; i += ES_THREADS) hist[i] = 0;
        if (threadIdx.x == 0) n_few = 0;
        __syncthreads();
#pragma unroll 4
        for (int i = threadIdx.x; i < old; i += ES_THREADS) {
          const uint32_t key = key_of(i);
          if ((key & mask) == prefix) atomicAdd(&hist[(lane & (copies - 1)) * ES_PITCH + ((key >> shift) & (bins - 1))], 1);
        }
        __syncthreads();
        if (threadIdx.x < ES_SCAN) find_bin(hist, copies, bins, left, warp_sums[0], found);
        __syncthreads();
        left -= found[1];
        prefix |= (uint32_t)found[0] << shift;
        mask |= (uint32_t)(bins - 1) << shift;
        const int m = found[2];
        if (pass < 2 && m <= ES_FEW) {  // in any order: only the key at the rank is looked for
          for (int i = threadIdx.x; i < old; i += ES_THREADS) {
            const uint32_t key = key_of(i);
            if ((key & mask) == prefix) few[atomicAdd(&n_few, 1)] = key;
          }
          __syncthreads();
          find_key(few, m, left, found);
          __syncthreads();
          prefix = (uint32_t)found[0];
          left -= found[1];
          break;
        }
      }
    }
    // ---- keys above `prefix` stay, and of those equal to it the first `left`; warp w walks rows [w part, (w + 1) part).
    // Where all equal ones stay (no tie is cut) "above" takes them in, and one vote per 32 rows is enough.
    const bool cut = found[2] != left;
    const int part = ((old + ES_WARPS - 1) / ES_WARPS + 31) / 32 * 32;
    const int begin = min(warp * part, old), end = min(begin + part, old);
    int n_above = 0, n_equal = 0;
#pragma unroll 4
    for (int i = begin + lane; i < end; i += 32) {
      const uint32_t key = key_of(i);
      n_above += cut ? key > prefix : key >= prefix;
      n_equal += key == prefix;
    }
    n_above = __reduce_add_sync(0xffffffffu, n_above);
    n_equal = cut ? __reduce_add_sync(0xffffffffu, n_equal) : 0;
    __syncthreads();  // warp_sums may still be read from the last pass
    if (lane == 0) {
      warp_sums[0][warp] = n_above;
      warp_sums[1][warp] = n_equal;
    }
    __syncthreads();
    // rows above, and equal ones, before this warp's
    int at = __reduce_add_sync(0xffffffffu, lane < warp ? warp_sums[0][lane] : 0);
    int ties = __reduce_add_sync(0xffffffffu, lane < warp ? warp_sums[1][lane] : 0);
    const uint32_t below = (1u << lane) - 1u;
    if (!cut) {
      if (at < last && at + n_above > first) {
#pragma unroll 4
        for (int i0 = begin; i0 < end; i0 += 32) {
          const int i = i0 + lane;
          const bool stays = i < end && key_of(i) >= prefix;
          const uint32_t all = __ballot_sync(0xffffffffu, stays);
          const int slot = at + __popc(all & below);
          if (stays && slot >= first && slot < last) list[slot] = start + i;
          at += __popc(all);
        }
      }
    } else {
      for (int i0 = begin; i0 < end; i0 += 32) {
        const int i = i0 + lane;
        const uint32_t key = i < end ? key_of(i) : 0u;
        const uint32_t above = __ballot_sync(0xffffffffu, i < end && key > prefix);
        const uint32_t equal = __ballot_sync(0xffffffffu, i < end && key == prefix);
        const int my_ties = ties + __popc(equal & below);
        const int slot = at + __popc(above & below) + min(my_ties, left);
        if (((above >> lane & 1u) || ((equal >> lane & 1u) && my_ties < left)) && slot >= first && slot < last)
          list[slot] = start + i;
        at += __popc(above);
        ties += __popc(equal);
      }
    }
  }
  __syncthreads();  // the share's list is complete
  const int pieces = (last - first) * vecs;
  for (int i0 = threadIdx.x; i0 < pieces; i0 += ES_THREADS * EG_PIECES) {
    uint4 a[EG_PIECES], b[EG_PIECES];
#pragma unroll
    for (int p = 0; p < EG_PIECES; ++p) {
      const int i = min(i0 + p * ES_THREADS, pieces - 1);
      const size_t from = (size_t)list[first + i / vecs] * ld + (size_t)g * vecs + i % vecs;
      a[p] = k[from];
      b[p] = v[from];
    }
#pragma unroll
    for (int p = 0; p < EG_PIECES; ++p) {
      const int i = i0 + p * ES_THREADS;
      if (i < pieces) {
        const size_t to = (((size_t)s * cap + first + i / vecs) * Hkv + g) * vecs + i % vecs;
        kc[to] = a[p];
        vc[to] = b[p];
      }
    }
  }
  for (int slot = first + threadIdx.x; slot < last; slot += ES_THREADS) {
    const int row = list[slot];
    cmass[sg * cap + slot] = mass[(size_t)g * n_total + row];
    cpos[sg * cap + slot] = pos[row];
  }
}

}  // namespace

size_t evict_scratch_ints(int n_seqs, int n_kv_heads, int budget) {
  return (size_t)n_seqs * n_kv_heads * budget;
}

int launch_evict(cudaStream_t st, int dtype, const void *k, const void *v, int ldkv, const int32_t *pos,
                 const float *mass, const int32_t *cu, int n_seqs, int max_len, int n_total, int n_kv_heads,
                 int head_dim, int budget, int n_recent, int32_t *idx, void *kc, void *vc, float *cmass, int32_t *cpos,
                 int32_t *clen, int cap, DevStatus *status) {
  if (n_seqs == 0) return LAZY_OK;
  LAZY_TRY(co_allow_smem<evict_kernel>(ES_SMEM));
  const size_t smem = (size_t)(ES_HIST + (max_len < ES_KEYS ? max_len : ES_KEYS)) * 4;
  // as many CTAs per (sequence, head) as run at once on the machine, one per SM; a part copies 64 slots at least
  const long long heads = (long long)n_seqs * n_kv_heads;
  const int most = budget < max_len ? budget : max_len;
  long long parts = sm_count() / heads;
  if (parts > ES_MAX_PARTS) parts = ES_MAX_PARTS;
  if (parts > cdiv(most, 64)) parts = cdiv(most, 64);
  if (parts < 1) parts = 1;
  return co_launch(evict_kernel, dim3((unsigned)parts, n_kv_heads, n_seqs), dim3(ES_THREADS), smem, st, 1, false,
                   (const uint4 *)k, (const uint4 *)v, (long long)ldkv * elem_bytes(dtype) / 16,
                   head_dim * elem_bytes(dtype) / 16, pos, mass, n_total, cu, max_len, budget, n_recent, idx, (uint4 *)kc,
                   (uint4 *)vc, cmass, cpos, clen, cap, status);
}

}  // namespace lazy
