// Attention of a batch of requests that share one prefix.  Every query row sees the whole prefix and the first part of
// its request's own key list (row i of T rows: keys j <= C - T + i of C), so the prefix part is one product of all
// rows with the prefix's keys: in the tensor-core form it is computed for the batch together and read once for every 256 (row,
// head) pairs of a key/value head (64 rows of a group of four), not once per request.  The general form (fp32, widths above 128,
// groups above 128) reads it for every row and head.
//
// bf16, head width up to 128: three launches; one for a few requests without a prefix, two for more of them or for requests
// without own keys.  (1) The prefix on tcgen05: the
// batch's (row, head) pairs of one key/value head are the lanes of 128-lane tiles, the prefix's keys are cut into ranges, every
// CTA leaves the partial softmax of its lanes over its range.  (2) The requests' own keys on the warp-level path of
// rows_mma.cuh, launched as a dependent that does not wait for (1): a CTA of it fits beside one of (1).  (3) A merge of the
// parts, one warp per (row, head).  64 requests of one row behind 16384 keys, 8 heads of 128 in groups of 4, 1 to 500 own keys
// each: 47.8 us (139 MB; 33 us without own keys, 24 without the prefix); four requests of five rows behind 1000 keys, 32 heads:
// 16.6 us (24 MB).
#include "attn_split.cuh"
#include "rows_mma.cuh"

namespace lazy {

namespace {

__device__ __forceinline__ int px_seq_of_row(const int32_t *cu, int n_seqs, int r) {
  int lo = 0, hi = n_seqs;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cu[mid] <= r) lo = mid;
    else hi = mid;
  }
  return lo;
}

// The same by a warp: 32 entries are looked at in one round.
__device__ __forceinline__ int px_seq_of_row_warp(const int32_t *cu, int n_seqs, int r) {
  const int lane = threadIdx.x & 31;
  int lo = 0, n = n_seqs;  // the sequence is one of [lo, lo + n)
  while (n > 1) {
    const int step = (n + 31) / 32, i = lo + lane * step;
    const uint32_t le = __ballot_sync(0xffffffffu, lane == 0 || (lane * step < n && cu[i] <= r));
    const int k = 31 - __clz(le);
    n = min(step, n - k * step);
    lo += k * step;
  }
  return lo;
}

// Own keys that row r sees, as a range of the key list: [*first, *first + return value).  Tables that do not fit
// their declared sizes are reported and give no keys.
__device__ __forceinline__ int px_own_keys(const PrefixArgs &a, int r, int s, int *first, DevStatus *status) {
  const int q0 = a.cu_q[s], q1 = a.cu_q[s + 1], c0 = a.cu_kv[s], c1 = a.cu_kv[s + 1];
  *first = c0;
  if (q0 < 0 || q1 > a.n_rows || r < q0 || r >= q1 || q1 - q0 > a.max_q || c0 < 0 || c1 < c0 || c1 > a.n_kv || c1 - c0 > a.max_kv) {
    dev_fail(status, LAZY_E_BADARG, W_PREFIX, r, s);
    return 0;
  }
  return max((c1 - c0) - (q1 - q0) + (r - q0) + 1, 0);
}

// ---- general form ---------------------------------------------------------------------------------------------
// grid (splits, n_heads, n_rows)
template <typename T>
__global__ void __launch_bounds__(AS_THREADS)
prefix_partial_kernel(const PrefixArgs a, int per_split, float *__restrict__ part_o, float *__restrict__ part_ml,
                      DevStatus *status) {
  __shared__ AttnSplitSmem<T> sm;
  __shared__ int s_first, s_own;
  const int r = blockIdx.z, h = blockIdx.y, H = gridDim.y, g = h / (H / a.n_kv_heads);
  if (threadIdx.x == 0) s_own = px_own_keys(a, r, px_seq_of_row(a.cu_q, a.n_seqs, r), &s_first, status);
  __syncthreads();
  const int first = s_first, n = a.n_pre + s_own;
  const int k0 = blockIdx.x * per_split;
  const size_t part = ((size_t)r * H + h) * gridDim.x + blockIdx.x;
  const size_t col = (size_t)g * a.head_dim;
  auto row = [&](const void *pre, const void *own, int j) -> const T * {
    if (j < a.n_pre) return (const T *)pre + (size_t)j * a.ld_pre + col;
    const int i = a.kv_idx[first + (j - a.n_pre)];
    if (i < 0 || i >= a.kv_rows) {
      dev_fail(status, LAZY_E_BADARG, W_PREFIX, first + (j - a.n_pre), i);
      return nullptr;
    }
    return (const T *)own + (size_t)i * a.ldkv + col;
  };
  attn_split_partial<T>(sm, (const T *)a.q + (size_t)r * a.ldq + (size_t)h * a.head_dim, a.head_dim, k0,
                        k0 + min(n - k0, per_split), [&](int j) { return row(a.k_pre, a.k, j); },
                        [&](int j) { return row(a.v_pre, a.v, j); }, part_o + part * a.head_dim, part_ml + part * 2,
                        nullptr);
}

// grid (n_heads, n_rows)
template <typename T>
__global__ void __launch_bounds__(AS_THREADS)
prefix_merge_kernel(const float *__restrict__ part_o, const float *__restrict__ part_ml, int n_splits, int head_dim,
                    T *__restrict__ o) {
  const size_t rh = (size_t)blockIdx.y * gridDim.x + blockIdx.x;
  attn_split_merge<T>(part_o + rh * n_splits * head_dim, part_ml + rh * n_splits * 2, n_splits, head_dim,
                      o + rh * head_dim, nullptr);
}

template <typename T>
int prefix_general(cudaStream_t st, const PrefixArgs &a, float *scratch, DevStatus *status) {
  const int keys = a.n_pre + a.max_kv;
  const int splits = attn_split_count((long long)a.n_rows * a.n_heads, keys);
  float *part_ml = scratch + (size_t)a.n_rows * a.n_heads * splits * a.head_dim;
  prefix_partial_kernel<T><<<dim3(splits, a.n_heads, a.n_rows), AS_THREADS, 0, st>>>(
      a, attn_split_keys(keys, splits), scratch, part_ml, status);
  LAZY_COUNT_LAUNCH();
  prefix_merge_kernel<T><<<dim3(a.n_heads, a.n_rows), AS_THREADS, 0, st>>>(scratch, part_ml, splits, a.head_dim, (T *)a.o);
  LAZY_COUNT_LAUNCH();
  return launch_ok();
}


// ---- (1) the prefix on tcgen05 ------------------------------------------------------------------------------------
// One CTA: TILES lane tiles (one or two) of 128 lanes = R rows x group heads of one key/value head, 64 keys at a time.
//   warp 0      TMA: the queries as one 3-d box per tile, then K and V tiles through a ring each (lanes 0 and 1);
//   warp 1      owns TMEM, issues S = Q K^T (M128 N64) of every tile as soon as its logits have been taken to registers;
//   warp 2      issues O += P V (M128 N = head width, P from TMEM);
//   warps 3..   softmax, one thread per lane; running maximum raised only when it grows by more than 2^8.
// TMEM columns of a tile: S (64) | P high (32) | P low (32) | O (head width).  P enters as the sum of two bf16 numbers (see
// WEIGHT_REST), so that the only rounding of an output that counts is its own; without the low part the 64 requests above
// would take 2.7 % less.  Two lane tiles in one CTA share the K and V tiles in shared memory.  64 keys take a CTA 1.17 us
// with two tiles, 0.9 with one: the products alone would take 0.8 and 0.4, the softmax threads' instructions about as much,
// and neither hides all of the other.
constexpr int PT_Q = 128, PT_K = 64;
constexpr float PT_RESCALE = 8.f;
constexpr int PT_REGS = 120;  // of 352 threads, which leaves the registers of a CTA of the own keys (168 x 128)

template <int HD, int TILES>
struct PrefixShape {
  static constexpr int CH = (HD + 63) / 64;  // 64-column chunks of the head, the last one filled up with zeros
  static constexpr int Q_CHUNK = PT_Q * 128, Q_BYTES = CH * Q_CHUNK;
  static constexpr int KV_CHUNK = PT_K * 128, KV_BYTES = CH * KV_CHUNK;
  static constexpr int STAGES = TILES == 1 ? 4 : 3;     // 160 KiB, beside which a CTA of the own keys fits (head width 128)
  static constexpr int THREADS = 96 + TILES * 128;
  static constexpr int TMEM_COLS = 256 * TILES;
  static constexpr int RING = TILES * Q_BYTES;          // offset of the K ring, the V ring behind it
  static constexpr int BARRIERS = RING + 2 * STAGES * KV_BYTES;
};
template <int STAGES, int TILES>
struct __align__(8) PrefixBarriers {
  unsigned long long q_full, k_full[STAGES], k_empty[STAGES], v_full[STAGES], v_empty[STAGES];
  unsigned long long s_full[TILES], s_free[TILES], p_full[TILES], pv_done[TILES], done[2];
  uint32_t tmem_base;
  int abort_flag, last_flag;  // last_flag: of the waits after an abort
};
template <int HD, int TILES>
constexpr int prefix_smem = PrefixShape<HD, TILES>::BARRIERS + 1024 +
                            (int)sizeof(PrefixBarriers<PrefixShape<HD, TILES>::STAGES, TILES>);

// grid (n_kv_heads, lane groups of TILES tiles, splits).  Parts: part_o [split][n_rows * n_heads][HD], part_ml
// [split][n_rows * n_heads] (maximum in log2 units, sum); pair (row, head) at row * n_heads + head.
template <int HD, int TILES>
__global__ void __maxnreg__(PT_REGS)
prefix_tc_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                 const __grid_constant__ CUtensorMap map_v, int n_rows, int group, int rows_per_tile, int n_pre,
                 int tiles_per_split, float *__restrict__ part_o, float2 *__restrict__ part_ml, DevStatus *status) {
  using Shape = PrefixShape<HD, TILES>;
  constexpr int STAGES = Shape::STAGES;
  extern __shared__ uint8_t prefix_smem_raw[];
  const uint32_t raw_addr = smem_u32(prefix_smem_raw);
  uint8_t *smem = prefix_smem_raw + (((raw_addr + 1023u) & ~1023u) - raw_addr);
  const uint32_t sQ = smem_u32(smem), sK = sQ + Shape::RING, sV = sK + STAGES * Shape::KV_BYTES;
  auto *bars = reinterpret_cast<PrefixBarriers<STAGES, TILES> *>(smem + Shape::BARRIERS);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = blockIdx.x, R = rows_per_tile, H = gridDim.x * group;
  const int row0 = blockIdx.y * TILES * R;  // first row of the CTA's first tile
  const int t0 = blockIdx.z * tiles_per_split, nt = min(tiles_per_split, (n_pre + PT_K - 1) / PT_K - t0);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  if (threadIdx.x == 0) {
    mbar_init(smem_u32(&bars->q_full), 1);
    for (int i = 0; i < STAGES; ++i) {
      mbar_init(smem_u32(&bars->k_full[i]), 1);
      mbar_init(smem_u32(&bars->k_empty[i]), 1);
      mbar_init(smem_u32(&bars->v_full[i]), 1);
      mbar_init(smem_u32(&bars->v_empty[i]), 1);
    }
    for (int t = 0; t < TILES; ++t) {
      mbar_init(smem_u32(&bars->s_full[t]), 1);
      mbar_init(smem_u32(&bars->s_free[t]), 4);
      mbar_init(smem_u32(&bars->p_full[t]), 4);
      mbar_init(smem_u32(&bars->pv_done[t]), 1);
    }
    for (int i = 0; i < 2; ++i) mbar_init(smem_u32(&bars->done[i]), 1);
    bars->abort_flag = bars->last_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    tma_prefetch_desc(&map_q);
    tma_prefetch_desc(&map_k);
    tma_prefetch_desc(&map_v);
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars->tmem_base)),
                 "r"((uint32_t)Shape::TMEM_COLS)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *reinterpret_cast<volatile uint32_t *>(&bars->tmem_base);
  volatile int *abort_flag = &bars->abort_flag;
  int loads = 0;  // by a loading thread

  if (warp == 0) {
    if (lane < 2) {
      const CUtensorMap *map = lane == 0 ? &map_k : &map_v;
      const uint32_t ring = lane == 0 ? sK : sV;
      unsigned long long *fulls = lane == 0 ? bars->k_full : bars->v_full, *empties = lane == 0 ? bars->k_empty : bars->v_empty;
      if (lane == 0) {
        const uint32_t qf = smem_u32(&bars->q_full);
        mbar_expect_tx(qf, (uint32_t)(TILES * Shape::CH * R * group * 128));
        for (int t = 0; t < TILES; ++t)
#pragma unroll
          for (int c = 0; c < Shape::CH; ++c)
            tma_load_3d(sQ + t * Shape::Q_BYTES + c * Shape::Q_CHUNK, &map_q, qf, c * 64, g * group, row0 + t * R);
      }
      for (int j = 0; j < nt; ++j) {
        const int st = j % STAGES;
        if (!mbar_wait(smem_u32(&empties[st]), (uint32_t)((j / STAGES) & 1) ^ 1u, abort_flag, status, W_PREFIX)) break;
        const uint32_t full = smem_u32(&fulls[st]);
        mbar_expect_tx(full, Shape::KV_BYTES);
#pragma unroll
        for (int c = 0; c < Shape::CH; ++c)
          tma_load_3d(ring + st * Shape::KV_BYTES + c * Shape::KV_CHUNK, map, full, c * 64, g, (t0 + j) * PT_K);
        ++loads;
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = idesc_bf16(PT_Q, PT_K, 0, 0);
      bool ok = mbar_wait(smem_u32(&bars->q_full), 0, abort_flag, status, W_PREFIX);
      for (int j = 0; j < nt && ok; ++j) {
        const int st = j % STAGES;
        ok = mbar_wait(smem_u32(&bars->k_full[st]), (uint32_t)((j / STAGES) & 1), abort_flag, status, W_PREFIX);
        for (int t = 0; t < TILES && ok; ++t) {
          ok = mbar_wait(smem_u32(&bars->s_free[t]), (uint32_t)(j & 1) ^ 1u, abort_flag, status, W_PREFIX);
          if (!ok) break;
          tc_fence_after();
#pragma unroll
          for (int k = 0; k < HD / 16; ++k) {
            const uint64_t ad = umma_smem_desc(sQ + t * Shape::Q_BYTES + (k >> 2) * Shape::Q_CHUNK + (k & 3) * 32);
            const uint64_t bd = umma_smem_desc(sK + st * Shape::KV_BYTES + (k >> 2) * Shape::KV_CHUNK + (k & 3) * 32);
            umma_bf16(tmem_base + (uint32_t)(t * 256), ad, bd, idesc, k != 0 ? 1u : 0u);
          }
          umma_commit(smem_u32(&bars->s_full[t]));
        }
        if (ok) umma_commit(smem_u32(&bars->k_empty[st]));
      }
    }
  } else if (warp == 2) {
    if (lane == 0) {
      const uint32_t idesc = idesc_bf16(PT_Q, HD, 0, 1);
      bool ok = true;
      for (int j = 0; j < nt && ok; ++j) {
        const int st = j % STAGES;
        ok = mbar_wait(smem_u32(&bars->v_full[st]), (uint32_t)((j / STAGES) & 1), abort_flag, status, W_PREFIX);
        for (int t = 0; t < TILES && ok; ++t) {
          ok = mbar_wait(smem_u32(&bars->p_full[t]), (uint32_t)(j & 1), abort_flag, status, W_PREFIX);
          if (!ok) break;
          tc_fence_after();
          const uint32_t tile = tmem_base + (uint32_t)(t * 256);
#pragma unroll
          for (int part = 0; part < 2; ++part)
#pragma unroll
            for (int k = 0; k < PT_K / 16; ++k) {
              const uint64_t vd = umma_smem_desc_mn(sV + st * Shape::KV_BYTES + k * 2048, Shape::KV_CHUNK, 1024);
              umma_bf16_a_tmem(tile + 128u, tile + 64u + (uint32_t)(part * 32 + k * 8), vd, idesc, (j | part | k) != 0 ? 1u : 0u);
            }
          umma_commit(smem_u32(&bars->pv_done[t]));
        }
        if (ok) umma_commit(smem_u32(&bars->v_empty[st]));
      }
    }
  } else {
    const int t = (warp - 3) >> 2, quarter = warp & 3;
    const uint32_t tile = tmem_base + (uint32_t)(t * 256) + ((uint32_t)(quarter * 32) << 16);
    const int f = quarter * 32 + lane;  // lane of the tile
    const int row = row0 + t * R + f / group;
    const bool used = f < R * group && row < n_rows;
    const bool warp_used = __any_sync(0xffffffffu, used);  // a warp without lanes only keeps the hand-over going
    const float sl2 = rsqrtf((float)HD) * CO_LOG2E;
    const unsigned long long sl2x2 = f32x2_pack(sl2, sl2);
    float m = -INFINITY, l = 0.f;
    bool ok = true;
    for (int j = 0; j < nt && ok; ++j) {
      ok = mbar_wait(smem_u32(&bars->s_full[t]), (uint32_t)(j & 1), abort_flag, status, W_PREFIX);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      tc_fence_after();
      if (!warp_used) {
        // not before the phase of P_{j-1} is over: the arrival would count for that one
        if (j > 0) {
          ok = mbar_wait(smem_u32(&bars->pv_done[t]), (uint32_t)((j - 1) & 1), abort_flag, status, W_PREFIX);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(smem_u32(&bars->s_free[t]));
          mbar_arrive(smem_u32(&bars->p_full[t]));
        }
        continue;
      }
      uint32_t raw[64];
      tmem_ld_32x32_raw(tile, raw);
      tmem_ld_32x32_raw(tile + 32u, raw + 32);
      tmem_ld_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bars->s_free[t]));
      const int there = n_pre - (t0 + j) * PT_K;  // keys of this tile
      if (there < PT_K) {
#pragma unroll
        for (int c = 0; c < 64; ++c)
          if (c >= there) raw[c] = 0xff800000u;  // -inf
      }
      float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int c = 0; c < 64; c += 8) {
        mx[0] = fmax3(mx[0], __uint_as_float(raw[c]), __uint_as_float(raw[c + 1]));
        mx[1] = fmax3(mx[1], __uint_as_float(raw[c + 2]), __uint_as_float(raw[c + 3]));
        mx[2] = fmax3(mx[2], __uint_as_float(raw[c + 4]), __uint_as_float(raw[c + 5]));
        mx[3] = fmax3(mx[3], __uint_as_float(raw[c + 6]), __uint_as_float(raw[c + 7]));
      }
      const float mj = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * sl2;
      // The reference exponent is settled before the exponentials; P_{j-1} V_{j-1} has to be done only where O is rescaled
      // and, below, where P_j takes the place of P_{j-1}: the exponentials run while it does.
      float alpha = 1.f;
      bool waited = j == 0;
      if (j == 0) m = mj;
      else {
        const bool need = mj - m > PT_RESCALE;
        if (need) {
          alpha = ex2_approx(m - mj);
          m = mj;
        }
        if (__any_sync(0xffffffffu, need)) {
          ok = mbar_wait(smem_u32(&bars->pv_done[t]), (uint32_t)((j - 1) & 1), abort_flag, status, W_PREFIX);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          tc_fence_after();
          waited = true;
#pragma unroll 1
          for (int c = 0; c < HD; c += 32) {
            uint32_t ov[32];
            tmem_ld_32x32_raw(tile + 128u + (uint32_t)c, ov);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; ++i) ov[i] = __float_as_uint(__uint_as_float(ov[i]) * alpha);
            tmem_st_32x32(tile + 128u + (uint32_t)c, ov);
          }
          tmem_st_wait();
        }
      }
      const float ref = m == -INFINITY ? 0.f : m;
      const unsigned long long neg = f32x2_pack(-ref, -ref);
      unsigned long long sum = 0ull;
      const unsigned long long rest = f32x2_pack(-WEIGHT_REST, -WEIGHT_REST);
      uint32_t hi[32];
#pragma unroll
      for (int c = 0; c < 64; c += 2) {
        const unsigned long long x = f32x2_fma(f32x2_pack(__uint_as_float(raw[c]), __uint_as_float(raw[c + 1])), sl2x2, neg);
        const unsigned long long p = ex2_approx_x2(x);
        float p0, p1, h0, h1;
        sum = f32x2_add(sum, p);
        f32x2_unpack(p, p0, p1);
        hi[c >> 1] = bf16x2_pack_rz(p0, p1);
        bf16x2_unpack(hi[c >> 1], h0, h1);
        f32x2_unpack(f32x2_fma(f32x2_pack(h0, h1), rest, p), p0, p1);
        raw[c >> 1] = bf16x2_pack(p0, p1);  // entry c / 2 has been used by now
      }
      float sm0, sm1;
      f32x2_unpack(sum, sm0, sm1);
      l = l * alpha + (sm0 + sm1);
      if (!waited) {
        ok = mbar_wait(smem_u32(&bars->pv_done[t]), (uint32_t)((j - 1) & 1), abort_flag, status, W_PREFIX);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc_fence_after();
      }
      tmem_st_32x32(tile + 64u, hi);
      tmem_st_32x32(tile + 96u, raw);
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bars->p_full[t]));
    }
    if (ok && nt > 0) {
      ok = mbar_wait(smem_u32(&bars->pv_done[t]), (uint32_t)((nt - 1) & 1), abort_flag, status, W_PREFIX);
      ok = __all_sync(0xffffffffu, ok);
    }
    if (warp_used) {
      tc_fence_after();
      const size_t part0 = (size_t)blockIdx.z * n_rows * H;
      const int pair = used ? row * H + g * group + f % group : -1;
      if (used) part_ml[part0 + pair] = make_float2(m, ok ? l : NAN);  // a wait ran out: nothing like a result
      // O leaves in whole 128-byte lines: 32 lanes x 32 columns at a time are turned around in the tile's query rows, which
      // no product reads any more (16-byte pieces swizzled: no conflicts either way)
      const uint32_t turn = sQ + t * Shape::Q_BYTES + quarter * 4096;
      if (ok) {
#pragma unroll 1
        for (int c = 0; c < HD; c += 32) {
          float v[32];
          tmem_ld_32x32(tile + 128u + (uint32_t)c, v);
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] *= WEIGHT_UNLIFT;
          __syncwarp();
#pragma unroll
          for (int i = 0; i < 8; ++i)
            asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(turn + lane * 128 + ((i ^ (lane & 7)) << 4)),
                         "f"(v[4 * i]), "f"(v[4 * i + 1]), "f"(v[4 * i + 2]), "f"(v[4 * i + 3])
                         : "memory");
          __syncwarp();
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int fl = i * 4 + (lane >> 3);  // the lane whose line this is
            const int to = __shfl_sync(0xffffffffu, pair, fl);
            float4 x;
            asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                         : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w)
                         : "r"(turn + fl * 128 + (((lane & 7) ^ (fl & 7)) << 4))
                         : "memory");
            if (to >= 0) *reinterpret_cast<float4 *>(part_o + (part0 + to) * HD + c + (lane & 7) * 4) = x;
          }
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {  // a wait ran out: what this CTA has in flight ends before it leaves
    if (threadIdx.x == 0) {
      ring_landed(&bars->q_full, 1, 1, &bars->last_flag, status, W_PREFIX);
      ring_landed(bars->k_full, STAGES, loads, &bars->last_flag, status, W_PREFIX);
    } else if (threadIdx.x == 1) {
      ring_landed(bars->v_full, STAGES, loads, &bars->last_flag, status, W_PREFIX);
    } else if (lane == 0 && (warp == 1 || warp == 2)) {
      umma_commit(smem_u32(&bars->done[warp - 1]));
      mbar_wait(smem_u32(&bars->done[warp - 1]), 0, &bars->last_flag, status, W_PREFIX);
    }
    __syncthreads();
  }
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)Shape::TMEM_COLS)
                 : "memory");
  }
}

// ---- (2) the requests' own keys -----------------------------------------------------------------------------------
// One CTA: 8 NT columns (row, head) of one (request, key/value head) over one range of its list; warps take every fourth group of
// 16 keys, and their parts are added in shared memory.
constexpr int PO_WARPS = 4, PO_THREADS = PO_WARPS * 32, PO_STAGES = 2, PO_CLUSTER = 8;
// Keys of a part; 64 requests with 1 to 500 keys of their own: 69 us with 64, 55 with 128, 50 with 256, 51 with 512
constexpr int PO_KEYS = 256;

template <int HD, int NT>
struct PrefixOwnShared {
  float wm[PO_WARPS][NT * 8], wl[PO_WARPS][NT * 8];
  float m[NT * 8], l[NT * 8];  // of the CTA, read by the cluster
  size_t pair[NT * 8];         // where a column's part goes
};

// grid (n_kv_heads * column blocks, splits, n_seqs).  DIRECT, without a prefix and with lists of few parts: the parts are the
// CTAs of a cluster, grid (n_kv_heads * column blocks * parts, 1, n_seqs), which leave the outputs themselves and no merge is
// needed: one row with 20 keys, 8 heads of 64, 3.7 us, 4.4 with a merge (among calls from Python 4.7 and 6.7); with 300 keys, 8
// heads of 128, 4.9 and 5.7.  More CTAs than run at once lose by it: 32 requests of five rows, 200 keys 34.4 us, with a merge 27.8.
template <int HD, int NT, bool DIRECT>
__global__ void __launch_bounds__(PO_THREADS, NT == 1 ? 4 : 2)
prefix_own_kernel(const PrefixArgs a, int group, int col_blocks, int per_split, float *__restrict__ part_o,
                  float2 *__restrict__ part_ml, DevStatus *status) {
  using Rows = RowsMma<HD, NT>;
  extern __shared__ __align__(128) uint8_t own_smem[];
  __shared__ PrefixOwnShared<HD, NT> sh;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int csize = DIRECT ? (int)co_cluster_size() : 1, split = DIRECT ? (int)co_cluster_rank() : (int)blockIdx.y;
  const int unit = blockIdx.x / csize, g = unit / col_blocks, cb = unit - g * col_blocks, s = blockIdx.z;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int q0 = a.cu_q[s], T = a.cu_q[s + 1] - q0, c0 = a.cu_kv[s], C = a.cu_kv[s + 1] - c0;
  const bool fits = q0 >= 0 && T >= 0 && q0 + T <= a.n_rows && T <= a.max_q && c0 >= 0 && C >= 0 && c0 + C <= a.n_kv &&
                    C <= a.max_kv;
  if (!fits && threadIdx.x == 0) dev_fail(status, LAZY_E_BADARG, W_PREFIX, s, -1);
  const int n_cols = T * group, col0 = cb * NT * 8;
  const int lo = split * per_split, hi = min(lo + per_split, C);
  bf16 *o = (bf16 *)a.o;
  if (DIRECT && blockIdx.x == 0) {  // rows that belong to nobody, or to a list that does not fit, are zero
    const int before = s == 0 ? min(max(q0, 0), a.n_rows) : 0, behind = s == a.n_seqs - 1 ? max(q0 + T, 0) : a.n_rows;
    const int bad0 = fits ? 0 : max(q0, 0), bad1 = fits ? 0 : min(q0 + T, a.n_rows);
    if ((before > 0 || behind < a.n_rows) && threadIdx.x == 0) dev_fail(status, LAZY_E_BADARG, W_PREFIX, s, behind);
    const size_t width = (size_t)a.n_heads * HD;
    for (size_t i = threadIdx.x; i < before * width; i += PO_THREADS) o[i] = __float2bfloat16_rn(0.f);
    for (size_t i = behind * width + threadIdx.x; i < a.n_rows * width; i += PO_THREADS) o[i] = __float2bfloat16_rn(0.f);
    for (size_t i = bad0 * width + threadIdx.x; bad1 > bad0 && i < bad1 * width; i += PO_THREADS) o[i] = __float2bfloat16_rn(0.f);
  }
  if (fits && col0 < n_cols) {
    const uint32_t stages = smem_u32(own_smem) + warp * PO_STAGES * Rows::STAGE;
    Rows rows;
    rows.init([&](int c) -> const bf16 * {
      const int f = col0 + c;
      return f < n_cols ? (const bf16 *)a.q + (size_t)(q0 + f / group) * a.ldq + (size_t)(g * group + f % group) * HD : nullptr;
    });
    int vis[NT][2];  // keys of the list that this lane's columns see
    int least = C, most = 0;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int f = col0 + t * 8 + (lane & 3) * 2 + i;
        vis[t][i] = f < n_cols ? max(C - T + f / group + 1, 0) : 0;
      }
    {  // the block's first and last column bound all of them
      const int last = min(col0 + NT * 8, n_cols) - 1;
      least = max(C - T + col0 / group + 1, 0);
      most = max(C - T + last / group + 1, 0);
    }
    const int end = min(hi, most);
    const bf16 *kb = (const bf16 *)a.k + (size_t)g * HD, *vb = (const bf16 *)a.v + (size_t)g * HD;
    // list entry of key lane % 16 of group warp + 4 i (-1: not there or out of range), fetched one group ahead
    auto entry = [&](int i) {
      const int j = lo + (warp + i * PO_WARPS) * RM_KEYS + (lane & 15);
      int e = -1;
      if (j < end) {
        e = a.kv_idx[c0 + j];
        if (e < 0 || e >= a.kv_rows) {
          dev_fail(status, LAZY_E_BADARG, W_PREFIX, c0 + j, e);
          e = -1;
        }
      }
      return e;
    };
    auto request = [&](int i, int e, uint32_t &mask) {
      const int j0 = lo + (warp + i * PO_WARPS) * RM_KEYS;
      mask = __ballot_sync(0xffffffffu, e >= 0) & 0xffffu;
      if (j0 < end)
        rows_load<HD>(stages + (i & 1) * Rows::STAGE, [&](int r, const bf16 *&kr, const bf16 *&vr) {
          const int row = __shfl_sync(0xffffffffu, e, r);
          const size_t at = (size_t)max(row, 0) * a.ldkv;
          kr = kb + at;
          vr = vb + at;
          return row >= 0;
        });
      rm_cp_commit();
    };
    static_assert(PO_STAGES == 2, "one group is requested while another is used");
    uint32_t there, there_next;
    request(0, entry(0), there);
    int e_next = entry(1);
    for (int i = 0; lo + (warp + i * PO_WARPS) * RM_KEYS < end; ++i) {
      request(i + 1, e_next, there_next);
      e_next = entry(i + 2);
      rm_cp_wait<1>();
      __syncwarp();
      const int j0 = lo + (warp + i * PO_WARPS) * RM_KEYS;
      int seen[NT][2];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int k = 0; k < 2; ++k) seen[t][k] = min(vis[t][k], hi) - j0;
      const uint32_t stage = stages + (i & 1) * Rows::STAGE;
      auto none = [](int, int, float, float) {};
      if (least >= min(j0 + RM_KEYS, end)) rows.template process<false>(stage, seen, there, none);
      else rows.template process<true>(stage, seen, there, none);
      there = there_next;
      __syncwarp();
    }
    rm_cp_wait<0>();
    rows.finish();
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
    float *wo = reinterpret_cast<float *>(own_smem);  // [warp][column][HD]
    const size_t base = DIRECT ? 0 : (size_t)split * a.n_rows * a.n_heads;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int c = t * 8 + (lane & 3) * 2 + i;
        float mx = sh.wm[0][c];
#pragma unroll
        for (int w = 1; w < PO_WARPS; ++w) mx = fmaxf(mx, sh.wm[w][c]);
        const float ref = mx == -INFINITY ? 0.f : mx;
        const float scale = ex2_approx(rows.m[t][i] - ref) * WEIGHT_UNLIFT;
#pragma unroll
        for (int k = 0; k < HD / 16; ++k) {
          wo[((size_t)warp * NT * 8 + c) * HD + k * 16 + (lane >> 2)] = rows.o[t][k][i] * scale;
          wo[((size_t)warp * NT * 8 + c) * HD + k * 16 + 8 + (lane >> 2)] = rows.o[t][k][2 + i] * scale;
        }
        const int f = col0 + c;
        if (warp == 0 && lane < 4 && f < n_cols) {
          float sum = 0.f;
#pragma unroll
          for (int w = 0; w < PO_WARPS; ++w) sum += sh.wl[w][c] * ex2_approx(sh.wm[w][c] - ref);
          const size_t pair = base + (size_t)(q0 + f / group) * a.n_heads + g * group + f % group;
          if (!DIRECT) part_ml[pair] = make_float2(mx, sum);
          sh.pair[c] = pair;
          sh.m[c] = mx;
          sh.l[c] = sum;
        }
      }
    __syncthreads();
    const int outputs = min(NT * 8, n_cols - col0) * HD;
    float *co = wo + PO_WARPS * NT * 8 * HD;  // [column][HD]: the CTA's part, read by the cluster
    static_assert((PO_WARPS + 1) * NT * 8 * HD * 4 <= PO_WARPS * PO_STAGES * Rows::STAGE, "the stages hold the outputs in the end");
    for (int i = threadIdx.x; i < outputs; i += PO_THREADS) {
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < PO_WARPS; ++w) sum += wo[(size_t)w * NT * 8 * HD + i];
      if (DIRECT) co[i] = sum;
      else part_o[sh.pair[i / HD] * HD + i % HD] = sum;
    }
    if (DIRECT) {
      co_cluster_sync();
      for (int i = split * PO_THREADS + threadIdx.x; i < outputs; i += csize * PO_THREADS) {
        float part[PO_CLUSTER], m[PO_CLUSTER], l[PO_CLUSTER], mx = -INFINITY, sum = 0.f, total = 0.f;
#pragma unroll
        for (int r = 0; r < PO_CLUSTER; ++r) {
          part[r] = r < csize ? *co_map_shared(co + i, r) : 0.f;
          m[r] = r < csize ? *co_map_shared(&sh.m[i / HD], r) : -INFINITY;
          l[r] = r < csize ? *co_map_shared(&sh.l[i / HD], r) : 0.f;
        }
#pragma unroll
        for (int r = 0; r < PO_CLUSTER; ++r) mx = fmaxf(mx, m[r]);
        const float ref = mx == -INFINITY ? 0.f : mx;
#pragma unroll
        for (int r = 0; r < PO_CLUSTER; ++r) {
          const float scale = ex2_approx(m[r] - ref);
          sum += part[r] * scale;
          total += l[r] * scale;
        }
        const float inv = total > 0.f ? 1.f / total : (total != total ? NAN : 0.f);
        o[sh.pair[i / HD] * HD + i % HD] = __float2bfloat16_rn(sum * inv);
      }
      co_cluster_sync();  // nobody leaves while its part is being read
    }
  }
  // the merge waits for this kernel alone: its end has to mean the end of the one before it.  One CTA sees to that; the
  // others leave their SMs to the next ones.
  if (!DIRECT && blockIdx.x + blockIdx.y + blockIdx.z == 0) asm volatile("griddepcontrol.wait;" ::: "memory");
}

// ---- (3) the merge: one warp per (row, head) ------------------------------------------------------------------------
// The parts are still being written when it starts: they must not be __restrict__, which with const says that nobody
// writes them while it runs and lets their loads go ahead of the wait.
template <int HD>
__global__ void __launch_bounds__(128)
prefix_tc_merge_kernel(const PrefixArgs a, const float *part_o, const float2 *part_ml, int n_pre_parts, int n_parts,
                       int own_split, DevStatus *status) {
  constexpr int V = HD / 32;
  constexpr bool WIDE = V % 2 == 0;  // a lane's columns: V in a row, or every 32nd where V is odd
  const int lane = threadIdx.x & 31;
  const long long pairs = (long long)a.n_rows * a.n_heads, pair = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (pair >= pairs) return;
  int first;
  const int row = (int)(pair / a.n_heads);  // the tables are inputs: they are read before the parts are there
  const int own = px_own_keys(a, row, px_seq_of_row_warp(a.cu_q, a.n_seqs, row), &first, status);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  // parts of own keys that hold any for this row (the others may not have been written)
  const int n = n_pre_parts + (own > 0 ? min((own + own_split - 1) / own_split, n_parts - n_pre_parts) : 0);
  // The outputs' loads do not wait for the weights: a batch is in flight while the (maximum, sum) pairs arrive, and the next
  // one while a batch is added up.
  constexpr int BATCH = 8;
  const float *first_o = part_o + pair * HD + (WIDE ? lane * V : lane);
  auto fetch = [&](int i0, float (&x)[BATCH][V]) {
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const float *p = first_o + (size_t)min(i0 + i, n - 1) * pairs * HD;
      if (V == 4) *reinterpret_cast<float4 *>(x[i]) = *reinterpret_cast<const float4 *>(p);
      else if (V == 2) *reinterpret_cast<float2 *>(x[i]) = *reinterpret_cast<const float2 *>(p);
      else {
#pragma unroll
        for (int c = 0; c < V; ++c) x[i][c] = p[c * 32];
      }
    }
  };
  float x[BATCH][V], next[BATCH][V];
  float m = -INFINITY, l = 0.f;
  bool bad = false;
  float2 ml = make_float2(-INFINITY, 0.f);
  if (lane < n) ml = part_ml[lane * pairs + pair];
  if (n > 0) fetch(0, x);
  for (int i = lane; i < n; i += 32) {
    const float2 y = i == lane ? ml : part_ml[i * pairs + pair];
    bad |= y.y != y.y;
    if (y.y > 0.f) m = fmaxf(m, y.x);
  }
  m = warp_max(m);
  bad = __any_sync(0xffffffffu, bad);
  float acc[V];
#pragma unroll
  for (int i = 0; i < V; ++i) acc[i] = 0.f;
  for (int i0 = 0; i0 < n; i0 += 32) {
    if (i0 > 0) ml = i0 + lane < n ? part_ml[(i0 + lane) * pairs + pair] : make_float2(-INFINITY, 0.f);
    float w = 0.f;
    if (ml.y > 0.f) {
      w = ex2_approx(ml.x - m);
      l = fmaf(ml.y, w, l);
    }
    for (int k = 0; k < min(32, n - i0); k += BATCH) {
      fetch(i0 + k + BATCH, next);  // past the end: the last part again, not used
#pragma unroll
      for (int i = 0; i < BATCH; ++i) {
        const float wi = __shfl_sync(0xffffffffu, w, k + i);  // 0 past the end
        if (i0 + k + i < n) {
#pragma unroll
          for (int c = 0; c < V; ++c) acc[c] = fmaf(x[i][c], wi, acc[c]);
        }
#pragma unroll
        for (int c = 0; c < V; ++c) x[i][c] = next[i][c];
      }
    }
  }
  l = warp_sum(l);
  const float inv = bad ? NAN : (l > 0.f ? 1.f / l : 0.f);
  bf16 *o = (bf16 *)a.o + pair * HD + (WIDE ? lane * V : lane);
  if (V == 4)
    *reinterpret_cast<uint2 *>(o) = make_uint2(bf16x2_pack(acc[0] * inv, acc[1] * inv), bf16x2_pack(acc[2] * inv, acc[3] * inv));
  else if (V == 2) *reinterpret_cast<uint32_t *>(o) = bf16x2_pack(acc[0] * inv, acc[1] * inv);
  else {
#pragma unroll
    for (int c = 0; c < V; ++c) o[c * 32] = __float2bfloat16_rn(acc[c] * inv);
  }
}

bool prefix_tc_eligible(int dtype, int head_dim, int group) {
  return dtype == LAZY_BF16 && head_dim <= 128 && group <= PT_Q;
}

// How the work is cut: key ranges of the prefix and of the own lists, so that every launch fills the machine once.
struct PrefixPlan {
  int tiles, lane_groups, pre_parts, tiles_per_split, nt, col_blocks, own_parts, own_split;
  bool direct;  // no prefix, and clusters of the own keys' parts all run at once: one launch
  size_t pairs, parts;
};
PrefixPlan prefix_plan(int n_rows, int n_seqs, int max_q, int n_pre, int max_kv, int n_heads, int n_kv_heads) {
  PrefixPlan p;
  const int group = n_heads / n_kv_heads, R = PT_Q / group;
  const int lane_tiles = cdiv(n_rows, R), key_tiles = cdiv(n_pre, PT_K);
  if (max_q > n_rows) max_q = n_rows;  // a bound may be any number
  p.tiles = lane_tiles > 1 ? 2 : 1;
  p.lane_groups = cdiv(lane_tiles, p.tiles);
  p.pre_parts = p.tiles_per_split = 0;
  if (key_tiles > 0) {
    const long long ctas = (long long)n_kv_heads * p.lane_groups, slots = sm_count();
    long long want = slots / ctas;
    if (want < 1) want = 1;
    if (want > key_tiles) want = key_tiles;
    p.tiles_per_split = cdiv(key_tiles, (int)want);
    p.pre_parts = cdiv(key_tiles, p.tiles_per_split);
  }
  p.nt = max_q * group <= 8 ? 1 : 2;
  p.col_blocks = cdiv(max_q * group, p.nt * 8);
  p.own_parts = p.own_split = 0;
  p.direct = false;
  if (max_kv > 0) {
    const long long ctas = (long long)n_kv_heads * p.col_blocks * n_seqs;
    long long want = (2LL * sm_count() + ctas - 1) / ctas;
    if (want < cdiv(max_kv, PO_KEYS)) want = cdiv(max_kv, PO_KEYS);
    if (want > 64) want = 64;
    const int most = cdiv(max_kv, PO_WARPS * RM_KEYS);  // a group of keys per warp at least
    if (want > most) want = most;
    if (key_tiles == 0) {
      const int per_sm = p.nt == 1 ? 3 : 2;
      long long c = 1;
      while (c < PO_CLUSTER && c < want && ctas * c * 2 <= co_cluster_ctas((int)c * 2, per_sm)) c *= 2;
      p.direct = c * PO_KEYS * 2 >= max_kv && ctas * c <= co_cluster_ctas((int)c, per_sm);
      if (p.direct) want = c;
    }
    p.own_split = cdiv(cdiv(max_kv, (int)want), RM_KEYS) * RM_KEYS;
    p.own_parts = p.direct ? (int)want : cdiv(max_kv, p.own_split);
  }
  p.pairs = (size_t)n_rows * n_heads;
  p.parts = (size_t)p.pre_parts + p.own_parts;
  return p;
}

template <int HD, int TILES>
int prefix_tc_launch(cudaStream_t st, const PrefixArgs &a, const PrefixPlan &p, int group, float *part_o, float2 *part_ml,
                     DevStatus *status) {
  const int R = PT_Q / group;
  CUtensorMap mq, mk, mv;
  LAZY_TRY(tma_map_heads_bf16(&mq, a.q, a.n_rows, a.n_heads, HD, a.ldq, group, R));
  LAZY_TRY(tma_map_heads_bf16(&mk, a.k_pre, a.n_pre, a.n_kv_heads, HD, a.ld_pre, 1, PT_K));
  LAZY_TRY(tma_map_heads_bf16(&mv, a.v_pre, a.n_pre, a.n_kv_heads, HD, a.ld_pre, 1, PT_K));
  LAZY_TRY((co_allow_smem<prefix_tc_kernel<HD, TILES>>(prefix_smem<HD, TILES>, true)));
  return co_launch(prefix_tc_kernel<HD, TILES>, dim3(a.n_kv_heads, p.lane_groups, p.pre_parts),
                   dim3(PrefixShape<HD, TILES>::THREADS), prefix_smem<HD, TILES>, st, 1, false, mq, mk, mv, a.n_rows, group, R,
                   a.n_pre, p.tiles_per_split, part_o, part_ml, status);
}
template <int HD, int NT, bool DIRECT>
int prefix_own_launch(cudaStream_t st, const PrefixArgs &a, const PrefixPlan &p, int group, float *part_o, float2 *part_ml,
                      DevStatus *status) {
  constexpr int SMEM = PO_WARPS * PO_STAGES * RowsMma<HD, NT>::STAGE;
  const int units = a.n_kv_heads * p.col_blocks;
  LAZY_TRY((co_allow_smem<prefix_own_kernel<HD, NT, DIRECT>>(SMEM, true)));
  const dim3 grid = DIRECT ? dim3(units * p.own_parts, 1, a.n_seqs) : dim3(units, p.own_parts, a.n_seqs);
  return co_launch(prefix_own_kernel<HD, NT, DIRECT>, grid, dim3(PO_THREADS), SMEM, st, DIRECT ? p.own_parts : 1, p.pre_parts > 0,
                   a, group, p.col_blocks, p.own_split, part_o, part_ml, status);
}

template <int HD>
int prefix_tc(cudaStream_t st, const PrefixArgs &a, float *scratch, DevStatus *status) {
  const int group = a.n_heads / a.n_kv_heads;
  const PrefixPlan p = prefix_plan(a.n_rows, a.n_seqs, a.max_q, a.n_pre, a.max_kv, a.n_heads, a.n_kv_heads);
  float *part_o = reinterpret_cast<float *>(align_up((uintptr_t)scratch, 16));
  float2 *part_ml = reinterpret_cast<float2 *>(part_o + p.parts * p.pairs * HD);
  if (p.pre_parts > 0)
    LAZY_TRY((p.tiles == 1 ? prefix_tc_launch<HD, 1>(st, a, p, group, part_o, part_ml, status)
                           : prefix_tc_launch<HD, 2>(st, a, p, group, part_o, part_ml, status)));
  if (p.direct)
    return p.nt == 1 ? prefix_own_launch<HD, 1, true>(st, a, p, group, nullptr, nullptr, status)
                     : prefix_own_launch<HD, 2, true>(st, a, p, group, nullptr, nullptr, status);
  if (p.own_parts > 0) {
    float *own_o = part_o + (size_t)p.pre_parts * p.pairs * HD;
    float2 *own_ml = part_ml + (size_t)p.pre_parts * p.pairs;
    LAZY_TRY((p.nt == 1 ? prefix_own_launch<HD, 1, false>(st, a, p, group, own_o, own_ml, status)
                        : prefix_own_launch<HD, 2, false>(st, a, p, group, own_o, own_ml, status)));
  }
  const long long warps = (long long)p.pairs;
  return co_launch(prefix_tc_merge_kernel<HD>, dim3((unsigned)((warps + 3) / 4)), dim3(128), 0, st, 1, p.parts > 0, a,
                   (const float *)part_o, (const float2 *)part_ml, p.pre_parts, (int)p.parts, p.own_split > 0 ? p.own_split : 1,
                   status);
}

}  // namespace

size_t attention_prefix_scratch_need(int n_rows, int n_seqs, int max_q, int n_pre, int max_kv, int n_heads,
                                     int n_kv_heads, int head_dim) {
  const size_t general =
      (size_t)n_rows * n_heads * attn_split_count((long long)n_rows * n_heads, n_pre + max_kv) * (head_dim + 2);
  if (n_heads / n_kv_heads > PT_Q || max_q < 1 || n_seqs < 1 || n_rows < 1) return general;
  const PrefixPlan p = prefix_plan(n_rows, n_seqs, max_q, n_pre, max_kv, n_heads, n_kv_heads);
  const size_t tiled = p.parts * p.pairs * (head_dim + 2) + 4;  // + 4: parts start on a 16-byte boundary
  return general > tiled ? general : tiled;
}

// As much as any batch no larger needs (of n_rows <= n_seqs * max_q rows), although fewer rows are cut into more parts: parts
// times (row, head) pairs of the prefix at the row counts that a number of lane groups ends with, and of the own keys, whose
// parts fill the machine twice or hold PO_KEYS keys (prefix_plan; 16 or fewer pairs make a column block).
size_t attention_prefix_scratch_floats(int n_rows, int n_seqs, int max_q, int n_pre, int max_kv, int n_heads,
                                       int n_kv_heads, int head_dim) {
  const size_t need = attention_prefix_scratch_need(n_rows, n_seqs, max_q, n_pre, max_kv, n_heads, n_kv_heads, head_dim);
  const size_t general = attn_split_parts((long long)n_rows * n_heads, n_pre + max_kv) * (head_dim + 2);
  size_t tiled = 0;
  if (n_heads / n_kv_heads <= PT_Q) {
    const long long R = PT_Q / (n_heads / n_kv_heads), sms = sm_count(), key_tiles = cdiv(n_pre, PT_K), rows = n_rows;
    auto least = [](long long a, long long b) { return a < b ? a : b; };
    auto most = [](long long a, long long b) { return a > b ? a : b; };
    long long pre = 0;
    for (long long g = 1; g == 1 || ((g - 1) * 2 * R < rows && g <= sms / n_kv_heads); ++g)
      pre = most(pre, least(rows, 2 * R * g) * least(key_tiles, most(sms / (n_kv_heads * g), 1)));
    if (key_tiles > 0) pre = most(pre, rows);
    const long long pairs = rows * n_heads, by_warps = least(64, cdiv(max_kv, PO_WARPS * RM_KEYS)),
                    by_keys = least(64, cdiv(max_kv, PO_KEYS));
    const long long own = least(pairs * by_warps, most(pairs + 2 * 16 * sms, pairs * by_keys));
    tiled = (size_t)(pre * n_heads + own) * (head_dim + 2) + 4;
  }
  const size_t any = general > tiled ? general : tiled;
  return any > need ? any : need;
}

int launch_attention_prefix(cudaStream_t st, int dtype, const PrefixArgs &a, float *scratch, DevStatus *status) {
  if (a.n_rows == 0) return LAZY_OK;
  if (prefix_tc_eligible(dtype, a.head_dim, a.n_heads / a.n_kv_heads))
    return co_head_dim(a.head_dim, [&](auto hd) { return prefix_tc<hd.value>(st, a, scratch, status); });
  return dtype == LAZY_F32 ? prefix_general<float>(st, a, scratch, status) : prefix_general<bf16>(st, a, scratch, status);
}

}  // namespace lazy
