// Accumulated attention weight of prompts: mass[g, j] = sum over the last `window` rows i >= j of a sequence (0 = all rows)
// and over the query heads h of key/value head g of softmax_j(q_i,h . k_j,g / sqrt(dh)).  window = 1 with a
// division by the heads is the Eq. 1 score.  No probability matrix is written: pass 1 leaves each (row, head)'s
// log-sum-exp, pass 2 forms the logits again, key-major, so that a thread owns a key and sums over the rows in registers.
// Each key's sum is taken by one thread group in a fixed order: no atomics, the same bits every time.
//
// A "lane" is one (row, head of the group) pair; lanes of a key/value head are numbered row-major, f = row * group +
// head.  lse[g][f] (log2 units) of all rows of the batch is the scratch between the passes.
#include "attn_common.cuh"
#include "cache_ops.cuh"

namespace lazy {

namespace {

// ---- general form: CUDA cores, any storage type and head width -------------------------------------------------
// 32 rows of one side stay in shared memory, 64-row tiles of the other stream past them through two buffers; 256
// threads hold 2 x 4 logits each and read both sides 16 bytes at a time (rows are padded by 16 bytes: no conflicts).
// Small tiles and a cluster that shares the streamed tiles keep a short prompt from running on a few SMs: three prompts of
// 278 rows in all, 4 heads of 64 in fp32, took 48.7 us with 64 x 64 tiles and one CTA per tile.
constexpr int MG_A = 32, MG_B = 64, MG_THREADS = 256;
// See mass_cluster.  Four prompts of 400 to 700 rows, 4 on 2 heads of 128: 103 us, 149 with a start of 5; one prompt of 700, 8 on
// 2 heads of 64: 60 and 55.
constexpr double MG_START = 0.5, MG_JOIN = 0.25;
constexpr int MT_MAX_CLUSTER = 8;

// Tile blockIdx.y of sequence blockIdx.z, or the other way round (by_tile): tiles then start in the order of their work over all
// sequences, so that none of the longest starts late because of the sequence it belongs to (3309, 1968, 4079 and 2232 rows:
// 415 us one sequence after the other, 391 so).  CTAs without a tile then lie between the others, though, which
// costs more than it gives where the lengths differ much (3402 and 85 rows: 131 us and 143).  The two batches fill 0.71 and
// 0.51 of n_seqs * max_len rows; the rule divides at 2/3, between them nothing was measured.
struct MassGrid {
  bool by_tile;
  MassGrid(int n_seqs, int max_len, long long n_total) : by_tile(3 * n_total >= 2LL * n_seqs * max_len) {}
  dim3 grid(int x, int n_seqs, long long tiles) const {
    return by_tile ? dim3((unsigned)x, n_seqs, (unsigned)tiles) : dim3((unsigned)x, (unsigned)tiles, n_seqs);
  }
};
// Tiles of `rows` that a batch can hold at most: `longest` per sequence, but no more than all rows make up.
long long mass_tiles(long long longest, int rows, int n_seqs, long long all_rows) {
  const long long a = longest * n_seqs, b = all_rows / rows + n_seqs;
  return a < b ? a : b;
}
struct MassGeneralShared {
  float m[MG_A], l[MG_A];  // this CTA's part, read by the cluster
};

// Rows [r0, r0 + ROWS) of one side into shared memory; row_of(r) gives a row or NULL (reads as zeros).
template <typename T, int ROWS, typename RowOf>
__device__ __forceinline__ void mg_load(T *dst, int head_dim, RowOf row_of) {
  constexpr int V = Elem<T>::kPerVec;
  const int pieces = head_dim / V, pitch = head_dim + V;
  for (int i = threadIdx.x; i < ROWS * pieces; i += MG_THREADS) {
    const int r = i / pieces, c = i - r * pieces;
    const T *row = row_of(r);
    const uint32_t to = smem_u32(dst + r * pitch + c * V);
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(row ? row + c * V : dst), "r"(row ? 16 : 0)
                 : "memory");
  }
}

// grid (n_kv_heads * cluster, tiles of the stationary side and sequences).  PASS 1: stationary lanes, streamed keys.  PASS 2:
// stationary keys, streamed lanes.
template <typename T, int PASS>
__global__ void __launch_bounds__(MG_THREADS)
mass_general_kernel(const T *__restrict__ q, int ldq, const T *__restrict__ k, int ldkv,
                    const int32_t *__restrict__ cu, int max_len, int n_total, int group, int head_dim, int window,
                    bool by_tile, float *lse, float *__restrict__ mass, DevStatus *status) {
  constexpr int V = Elem<T>::kPerVec;
  extern __shared__ __align__(128) uint8_t mg_smem[];
  __shared__ MassGeneralShared sh;
  const int rank = (int)co_cluster_rank(), csize = (int)co_cluster_size();
  const int g = blockIdx.x / csize, pitch = head_dim + V;
  const int s = by_tile ? blockIdx.y : blockIdx.z, z = by_tile ? blockIdx.z : blockIdx.y;
  if (PASS == 1) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  auto rows_of = [&](int n) { return window > 0 ? min(n, window) : n; };  // the last ones accumulate
  auto tiles_of = [&](int n) { return ((PASS == 1 ? rows_of(n) * group : n) + MG_A - 1) / MG_A; };
  int start, n;
  if (!co_span(cu, s, n_total, max_len, status, W_MASS, start, n) ) return;  // the whole cluster alike
  const int at = PASS == 1 ? (by_tile ? (int)gridDim.z : tiles_of(n)) - 1 - z : z;  // most work first
  if (at < 0 || at >= tiles_of(n)) return;
  const int first = n - rows_of(n), n_lanes = rows_of(n) * group;
  const int n_a = PASS == 1 ? n_lanes : n, a0 = at * MG_A;
  const float *lse_g = lse + ((size_t)g * n_total + start + first) * group;  // lane f of this sequence at lse_g[f]
  const float scale = rsqrtf((float)head_dim) * CO_LOG2E;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  // streamed rows [all0, all1) that matter to this tile, and this CTA's share of them in whole tiles
  int all0 = 0, all1;
  if (PASS == 1) all1 = min(n, first + (min(a0 + MG_A, n_a) - 1) / group + 1);
  else {
    all0 = max(a0 - first, 0) * group;  // the first lane whose row sees key a0
    all1 = n_lanes;
  }
  const int tiles = (all1 - all0 + MG_B - 1) / MG_B, per = (tiles + csize - 1) / csize;
  const int b_begin = min(all0 + rank * per * MG_B, all1), b_end = min(b_begin + per * MG_B, all1);
  auto lane_row = [&](int f) -> const T * {
    return f < n_lanes ? q + (size_t)(start + first + f / group) * ldq + (size_t)(g * group + f % group) * head_dim : nullptr;
  };
  auto key_row = [&](int j) -> const T * { return j < n ? k + (size_t)(start + j) * ldkv + (size_t)g * head_dim : nullptr; };
  T *sa = reinterpret_cast<T *>(mg_smem), *sb = sa + MG_A * pitch;
  auto load_b = [&](int b0, int buf) {
    if (b0 < b_end)
      mg_load<T, MG_B>(sb + buf * MG_B * pitch, head_dim, [&](int r) { return PASS == 1 ? key_row(b0 + r) : lane_row(b0 + r); });
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  mg_load<T, MG_A>(sa, head_dim, [&](int r) { return PASS == 1 ? lane_row(a0 + r) : key_row(a0 + r); });
  load_b(b_begin, 0);
  if (PASS == 2) asm volatile("griddepcontrol.wait;" ::: "memory");  // the log-sum-exps of pass 1
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
  int buf = 0;
  for (int b0 = b_begin; b0 < b_end; b0 += MG_B, buf ^= 1) {
    load_b(b0 + MG_B, buf ^ 1);
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    __syncthreads();
    const T *pa = sa + ty * 2 * pitch, *pb = sb + (buf * MG_B + tx) * pitch;
    float x[2][4] = {};
#pragma unroll 4
    for (int c = 0; c < head_dim; c += V) {
      float av[2][V], bv[4][V];
      Vec16<T> t;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        t.load(pa + i * pitch + c);
        t.unpack(av[i]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        t.load(pb + j * 16 * pitch + c);
        t.unpack(bv[j]);
      }
#pragma unroll
      for (int e = 0; e < V; ++e)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) x[i][j] = fmaf(av[i][e], bv[j][e], x[i][j]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int a = a0 + ty * 2 + i;
      if (PASS == 1) {
        const int row = first + a / group;
        float mt = m[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int key = b0 + tx + j * 16;
          x[i][j] = key <= row && key < n && a < n_a ? x[i][j] * scale : -INFINITY;
          mt = fmaxf(mt, x[i][j]);
        }
        const float ref = mt == -INFINITY ? 0.f : mt;
        float sum = l[i] * exp2f(m[i] - ref);
#pragma unroll
        for (int j = 0; j < 4; ++j) sum += exp2f(x[i][j] - ref);
        m[i] = mt;
        l[i] = sum;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int f = b0 + tx + j * 16;
          if (f < n_lanes && first + f / group >= a) l[i] += exp2f(x[i][j] * scale - lse_g[f]);
        }
      }
    }
    __syncthreads();  // the buffer may be filled again
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
#pragma unroll
  for (int i = 0; i < 2; ++i) {
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) {
      const float lo = __shfl_xor_sync(0xffffffffu, l[i], o);
      if (PASS == 1) {
        const float mo = __shfl_xor_sync(0xffffffffu, m[i], o);
        const float mt = fmaxf(m[i], mo), ref = mt == -INFINITY ? 0.f : mt;
        l[i] = l[i] * exp2f(m[i] - ref) + lo * exp2f(mo - ref);
        m[i] = mt;
      } else {
        l[i] += lo;
      }
    }
    if (tx == 0) {
      sh.m[ty * 2 + i] = m[i];
      sh.l[ty * 2 + i] = l[i];
    }
  }
  if (csize > 1) co_cluster_sync();
  else __syncthreads();
  if (rank == 0 && threadIdx.x < MG_A && a0 + (int)threadIdx.x < n_a) {
    float mm = -INFINITY, ll = 0.f;
    for (int r = 0; r < csize; ++r) {
      const float lr = *co_map_shared(&sh.l[threadIdx.x], r);
      if (PASS == 1) {
        const float mr = *co_map_shared(&sh.m[threadIdx.x], r);
        const float mt = fmaxf(mm, mr), ref = mt == -INFINITY ? 0.f : mt;
        ll = ll * exp2f(mm - ref) + lr * exp2f(mr - ref);
        mm = mt;
      } else {
        ll += lr;
      }
    }
    const size_t a = a0 + threadIdx.x;
    if (PASS == 1) lse[((size_t)g * n_total + start + first) * group + a] = mm + log2f(ll);
    else mass[(size_t)g * n_total + start + a] = ll;
  }
  if (csize > 1) co_cluster_sync();  // nobody leaves while its part is being read
}

// CTAs per stationary tile, for `tiles` of them that stream up to `streamed` tiles each and `seen` of that on average, the
// longest first: the number whose estimated time is the least.  The unit is a streamed tile; `start` is what starting and leaving a
// CTA costs, `join` what every doubling of the cluster adds.  A launch takes its longest CTA, or the CTAs' time shared out,
// or, when a part of the CTAs starts after the others, the shortest of the first with the longest of the second.  Longest CTAs that
// all run at once are not the best choice for triangles (us, clusters filling the machine once | by this rule): 3402 + 85 rows of
// 32 heads in groups of 4 171 | 131, 4100 rows of 12 in groups of 3 109 | 87, 2328 rows of 8 in groups of 4 50 | 32.
int mass_cluster(long long tiles, int streamed, double seen, int per_sm, double start, double join) {
  int best = 1;
  double least = 0.;
  for (int c = 1, log2c = 0; c <= MT_MAX_CLUSTER; c *= 2, ++log2c) {
    const double over = start + join * log2c, longest = (streamed + c - 1) / c;
    const double waves = (double)tiles * c / co_cluster_ctas(c, per_sm);
    double t = longest + over;
    if (waves > 1.) {
      t = fmax(t, waves * (streamed * seen / c + over));
      t = fmax(t, 2. * (over + longest * (1. - 2. * (1. - seen) / waves)));
    }
    if (c == 1 || t < least) {
      best = c;
      least = t;
    }
  }
  return best;
}
// The part of a rectangle of `rows` last rows and n keys that is seen.
double mass_seen(int rows, int n) { return 1. - rows / (2. * n); }

template <typename T>
int mass_general(cudaStream_t st, const T *q, int ldq, const T *k, int ldkv, const int32_t *cu, int n_seqs, int max_len,
                 int n_total, int n_heads, int n_kv_heads, int head_dim, int window, float *lse, float *mass,
                 DevStatus *status) {
  const int group = n_heads / n_kv_heads;
  const int rows = window > 0 && window < max_len ? window : max_len;
  const long long lanes = (long long)rows * group;
  const int smem = (MG_A + 2 * MG_B) * (head_dim + Elem<T>::kPerVec) * (int)sizeof(T);
  constexpr int MOST = (MG_A + 2 * MG_B) * (256 + Elem<T>::kPerVec) * (int)sizeof(T);
  LAZY_TRY((co_allow_smem<mass_general_kernel<T, 1>>(MOST)));
  LAZY_TRY((co_allow_smem<mass_general_kernel<T, 2>>(MOST)));
  const long long lane_tiles = (lanes + MG_A - 1) / MG_A, key_tiles = cdiv(max_len, MG_A);
  if (lane_tiles > 65535 || key_tiles > 65535) return LAZY_E_CAPACITY;
  const int per_sm = smem <= 100 * 1024 ? 2 : 1;
  const double seen = mass_seen(rows, max_len);
  const long long all_lane = mass_tiles(lane_tiles, MG_A, n_seqs, n_total * (long long)group);
  const long long all_key = mass_tiles(key_tiles, MG_A, n_seqs, n_total);
  const int c1 = mass_cluster(all_lane * n_kv_heads, cdiv(max_len, MG_B), seen, per_sm, MG_START, MG_JOIN);
  const int c2 = mass_cluster(all_key * n_kv_heads, (int)((lanes + MG_B - 1) / MG_B), seen, per_sm, MG_START, MG_JOIN);
  const MassGrid grid(n_seqs, max_len, n_total);
  LAZY_TRY(co_launch(mass_general_kernel<T, 1>, grid.grid(n_kv_heads * c1, n_seqs, lane_tiles), dim3(MG_THREADS), smem, st, c1,
                     false, q, ldq, k, ldkv, cu, max_len, n_total, group, head_dim, window, grid.by_tile, lse, mass, status));
  return co_launch(mass_general_kernel<T, 2>, grid.grid(n_kv_heads * c2, n_seqs, key_tiles), dim3(MG_THREADS), smem, st, c2,
                   true, q, ldq, k, ldkv, cu, max_len, n_total, group, head_dim, window, grid.by_tile, lse, mass, status);
}

// ---- tensor-core form: bf16, head width up to 128 ----------------------------------------------------------------
// One CTA holds 128 rows of one side (pass 1: lanes, pass 2: keys) in shared memory as the M side of the product and
// streams 128-row tiles of the other side past them; a logit tile S (128 x 128, fp32) lands in TMEM and is consumed from
// there, so every row's reduction stays inside one thread: pass 1 keeps a lane's running maximum and sum, pass 2 a
// key's running sum.  Warp roles:
//   warp 0     TMA: the stationary tile once, the streamed tiles through a two-stage ring (and, in pass 2, their
//              lanes' log-sum-exps through a four-stage ring);
//   warp 1     owns TMEM and issues S_j = A B_j^T (M128 N128 K16) from one lane into two buffers of 128 columns;
//   warps 2-9  two threads per TMEM lane, 64 columns each: tcgen05.ld, then one exponential per logit.
// Two CTAs share an SM.  The bound is what the softmax threads issue: one exponential per (row, key, head) and pass is 1024
// clocks of the special-function unit per tile against 514 of the tensor cores (head width 128), so a quarter of them is
// taken on the FMA pipe (a 3376-row prompt of 32 heads: 131 us with none, 122 with a quarter, 142 with half), which
// leaves 768 clocks of that unit and about as many of instruction issue; a tile takes some 1350.  What does not change that:
// persistent CTAs (128 us), 256 stationary rows with one streamed tile for both and rings for both sides (128 to 135 us, the
// stationary side in shared or tensor memory, one or two issuing warps), 32 or 128 columns to a thread (130 and 137), half
// of a thread's columns loaded while the other half is used (141).
// Lane tiles hold R = 128 / group rows x group heads, loaded as one 3-d box; with a group that does not divide 128
// the last lanes of a tile are unused.  A short grid is filled up by clusters: the CTAs of a cluster share a
// stationary tile, split the streamed tiles and add their parts in rank order through distributed shared memory.
//
// DEEP is the form for few lanes over many keys (a window of a long prompt), where a CTA would spend its time on starting up:
// one CTA per SM with four stages; pass 1 cuts the keys into ranges (no clusters: eight to a cluster only 120 of the 148 SMs
// can be used) and leaves each range's (maximum, sum), pass 2 merges them and takes a range of key tiles, the next one
// loaded while the last is used.  Ranges are of one length for all sequences, so that long and short ones share the SMs (a one-row
// window of five sequences of 16169 to 9 rows: 46 us with as many ranges to each, 28 so).  A 64-row window over 16384 keys of 8
// heads, group 4: 35 us, 49 without this form.
constexpr int MT = 128;                       // tile rows of either side, columns of S
constexpr int MT_LSE_STAGES = 4, MT_DEEP_TILES = 4, MT_DEEP_SPLITS = 32;  // lane tiles that DEEP pass 2 takes at most
static_assert(MT_DEEP_TILES <= MT_LSE_STAGES, "DEEP pass 2 keeps all lanes' log-sum-exps where the ring would be");
constexpr int MT_POLY = 8;  // of as many columns, two exponentials are taken on the FMA pipe (a quarter): see ex2_poly_x2
constexpr double MT_START = 7., MT_JOIN = 1.;  // see mass_cluster
constexpr int MT_THREADS = 320;
constexpr int MT_TMEM_COLS = 256;

struct MassDeep {
  int splits, split_tiles;   // pass 1: key ranges per lane tile, key tiles in each
  int ranges, range_tiles;   // pass 2: ranges of key tiles per head
};
template <bool DEEP>
struct MassShape {
  static constexpr int A_BUFS = DEEP ? 2 : 1, STAGES = DEEP ? 4 : 2, CTAS = DEEP ? 1 : 2;
};
template <bool DEEP>
struct __align__(16) MassShared {
  using Shape = MassShape<DEEP>;
  float lse[MT_LSE_STAGES][MT];
  float part_m[2][MT], part_l[2][2][MT];  // per column half: a lane's (maximum, sum), a key's sum (two tiles' in turn)
  unsigned long long a_full[Shape::A_BUFS], a_empty[Shape::A_BUFS], b_full[Shape::STAGES], b_empty[Shape::STAGES], s_full[2],
      s_free[2], l_full[MT_LSE_STAGES], l_free[MT_LSE_STAGES], done;
  uint32_t tmem_base;
  int abort_flag, last_flag;  // last_flag: of the waits after an abort
};
template <int HD, bool DEEP>
constexpr int mass_smem =
    (MassShape<DEEP>::A_BUFS + MassShape<DEEP>::STAGES) * MT * ((HD + 63) / 64) * 128 + 1024 + (int)sizeof(MassShared<DEEP>);

// grid (n_kv_heads * cluster, tiles and sequences); DEEP, no clusters: pass 1 (n_kv_heads * splits, the same), pass 2 (n_kv_heads,
// ranges of key tiles and sequences).  parts: (maximum, sum) of tile t's lanes over key range i at (((s * n_kv_heads + g) *
// deep_tiles + t) * splits + i) * 128; a range that holds none of a sequence's tiles is not written.
// lse: tiles of 128 floats (minus the log-sum-exps, log2 units), tile t of sequence s of key/value head g at ((g * seq_tiles)
// + start_s / R + s + t) * 128: sequences' tiles cannot overlap and every tile is 512-byte aligned.
template <int PASS, int HD, bool DEEP>
__global__ void __launch_bounds__(MT_THREADS, MassShape<DEEP>::CTAS)
mass_tc_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
               const int32_t *__restrict__ cu, int max_len, int n_total, int group, int rows_per_tile, int window,
               bool by_tile, float *lse, int seq_tiles, const MassDeep deep, float2 *parts, int deep_tiles,
               float *__restrict__ mass, DevStatus *status) {
  extern __shared__ uint8_t mass_smem_raw[];
  constexpr int A_BUFS = MassShape<DEEP>::A_BUFS, STAGES = MassShape<DEEP>::STAGES;
  constexpr int CH = (HD + 63) / 64;         // 64-column chunks of the head, the last one filled up with zeros
  constexpr int CHUNK = MT * 128;            // bytes of one chunk of a tile
  const uint32_t raw_addr = smem_u32(mass_smem_raw);
  uint8_t *smem = mass_smem_raw + (((raw_addr + 1023u) & ~1023u) - raw_addr);
  const uint32_t sA = smem_u32(smem), sB = sA + A_BUFS * CH * CHUNK;
  auto *sh = reinterpret_cast<MassShared<DEEP> *>(smem + (A_BUFS + STAGES) * CH * CHUNK);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr bool SPLIT = DEEP && PASS == 1;
  const int csize = SPLIT ? deep.splits : (int)co_cluster_size();  // CTAs that share a stationary tile
  const int g = blockIdx.x / csize, rank = blockIdx.x - g * csize, R = rows_per_tile, Hkv = gridDim.x / csize;
  const int s = by_tile ? blockIdx.y : blockIdx.z, z = by_tile ? blockIdx.z : blockIdx.y;
  if (PASS == 1) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  auto rows_of = [&](int n) { return window > 0 ? min(n, window) : n; };  // the last ones accumulate
  auto tiles_of = [&](int n) { return PASS == 1 ? (rows_of(n) + R - 1) / R : (n + MT - 1) / MT; };
  const int range = DEEP && PASS == 2 ? deep.range_tiles : 1;  // stationary tiles of a CTA
  int start, n;
  if (!co_span(cu, s, n_total, max_len, status, W_MASS, start, n) ) return;  // the whole cluster alike
  const int first = n - rows_of(n), a_tiles = tiles_of(n);
  const int lane_tiles = (n - first + R - 1) / R, key_tiles = (n + MT - 1) / MT;
  // stationary tiles [at0, at1): one, most work first, or in DEEP pass 2 a range of them
  const int at0 = PASS == 1 ? (by_tile ? (int)gridDim.z : a_tiles) - 1 - z : z * range;
  const int at1 = DEEP && PASS == 2 ? min(at0 + range, a_tiles) : at0 + 1;
  if (at0 < 0 || at0 >= a_tiles) return;
  // key tiles that some lane of a lane tile sees; streamed tiles [b0, b1) of this CTA for a stationary one
  auto keys_of = [&](int lane_tile) { return min(key_tiles, (min(first + (lane_tile + 1) * R, n) + MT - 1) / MT); };
  auto streamed = [&](int at, int &b0, int &b1) {
    const int all0 = PASS == 1 ? 0 : max(at * MT - first, 0) / R;
    const int all1 = PASS == 1 ? keys_of(at) : lane_tiles;
    const int per = SPLIT ? deep.split_tiles : (all1 - all0 + csize - 1) / csize;
    b0 = min(all0 + rank * per, all1);
    b1 = min(b0 + per, all1);
  };
  if (SPLIT) {
    int b0, b1;
    streamed(at0, b0, b1);
    if (b0 == b1) return;
  }
  const size_t lse_base = ((size_t)g * seq_tiles + start / R + s) * MT;

  if (threadIdx.x == 0) {
    for (int i = 0; i < A_BUFS; ++i) {
      mbar_init(smem_u32(&sh->a_full[i]), 1);
      mbar_init(smem_u32(&sh->a_empty[i]), 1);
    }
    for (int i = 0; i < STAGES; ++i) {
      mbar_init(smem_u32(&sh->b_full[i]), 1);
      mbar_init(smem_u32(&sh->b_empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&sh->s_full[i]), 1);
      mbar_init(smem_u32(&sh->s_free[i]), 8);
    }
    for (int i = 0; i < MT_LSE_STAGES; ++i) {
      mbar_init(smem_u32(&sh->l_full[i]), 1);
      mbar_init(smem_u32(&sh->l_free[i]), 8);
    }
    mbar_init(smem_u32(&sh->done), 1);
    sh->abort_flag = sh->last_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    tma_prefetch_desc(&map_q);
    tma_prefetch_desc(&map_k);
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh->tmem_base)),
                 "r"((uint32_t)MT_TMEM_COLS)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *reinterpret_cast<volatile uint32_t *>(&sh->tmem_base);
  volatile int *abort_flag = &sh->abort_flag;

  // Every role walks the same (stationary, streamed) pairs: `t` counts pairs, `ai` stationary tiles.
  int a_loads = 0, b_loads = 0, l_loads = 0;  // by the loading thread
  if (warp == 0) {
    if (lane == 0) {
      const uint32_t lane_bytes = (uint32_t)(R * group * 128 * CH), key_bytes = (uint32_t)(CH * CHUNK);
      auto load = [&](bool lanes, int tile, uint32_t dst, uint32_t bar) {
        mbar_expect_tx(bar, lanes ? lane_bytes : key_bytes);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          if (lanes) tma_load_3d(dst + c * CHUNK, &map_q, bar, c * 64, g * group, start + first + tile * R);
          else tma_load_3d(dst + c * CHUNK, &map_k, bar, c * 64, g, start + tile * MT);
        }
      };
      bool ok = true, waited = PASS == 1 || DEEP;
      int t = 0, ai = 0;
      for (int at = at0; at < at1 && ok; ++at) {
        int b0, b1;
        streamed(at, b0, b1);
        if (b0 == b1) continue;
        ok = mbar_wait(smem_u32(&sh->a_empty[ai % A_BUFS]), (uint32_t)((ai / A_BUFS) & 1) ^ 1u, abort_flag, status, W_MASS);
        if (!ok) break;
        load(PASS == 1, at, sA + (ai % A_BUFS) * CH * CHUNK, smem_u32(&sh->a_full[ai % A_BUFS]));
        a_loads = ++ai;
        if (!waited) {
          asm volatile("griddepcontrol.wait;" ::: "memory");  // the log-sum-exps of pass 1
          waited = true;
        }
        for (int b = b0; b < b1; ++b, ++t) {
          const int st = t % STAGES;
          ok = mbar_wait(smem_u32(&sh->b_empty[st]), (uint32_t)((t / STAGES) & 1) ^ 1u, abort_flag, status, W_MASS);
          if (!ok) break;
          load(PASS == 2, b, sB + st * CH * CHUNK, smem_u32(&sh->b_full[st]));
          ++b_loads;
          if (PASS == 2 && !DEEP) {
            const int ls = t % MT_LSE_STAGES;
            ok = mbar_wait(smem_u32(&sh->l_free[ls]), (uint32_t)((t / MT_LSE_STAGES) & 1) ^ 1u, abort_flag, status, W_MASS);
            if (!ok) break;
            mbar_expect_tx(smem_u32(&sh->l_full[ls]), MT * 4);
            bulk_load(smem_u32(sh->lse[ls]), lse + lse_base + (size_t)b * MT, MT * 4, smem_u32(&sh->l_full[ls]));
            ++l_loads;
          }
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = idesc_bf16(MT, MT, 0, 0);
      bool ok = true;
      int t = 0, ai = 0;
      for (int at = at0; at < at1 && ok; ++at) {
        int b0, b1;
        streamed(at, b0, b1);
        if (b0 == b1) continue;
        const uint32_t a_tile = sA + (ai % A_BUFS) * CH * CHUNK;
        ok = mbar_wait(smem_u32(&sh->a_full[ai % A_BUFS]), (uint32_t)((ai / A_BUFS) & 1), abort_flag, status, W_MASS);
        for (int b = b0; b < b1 && ok; ++b, ++t) {
          const int st = t % STAGES, sb = t & 1;
          ok = mbar_wait(smem_u32(&sh->b_full[st]), (uint32_t)((t / STAGES) & 1), abort_flag, status, W_MASS);
          if (!ok) break;
          ok = mbar_wait(smem_u32(&sh->s_free[sb]), (uint32_t)((t >> 1) & 1) ^ 1u, abort_flag, status, W_MASS);
          if (!ok) break;
          tc_fence_after();
#pragma unroll
          for (int k = 0; k < HD / 16; ++k) {
            const uint64_t ad = umma_smem_desc(a_tile + (k >> 2) * CHUNK + (k & 3) * 32);
            const uint64_t bd = umma_smem_desc(sB + st * CH * CHUNK + (k >> 2) * CHUNK + (k & 3) * 32);
            umma_bf16(tmem_base + (uint32_t)(sb * MT), ad, bd, idesc, k != 0 ? 1u : 0u);
          }
          umma_commit(smem_u32(&sh->b_empty[st]));
          if (b + 1 == b1) umma_commit(smem_u32(&sh->a_empty[ai % A_BUFS]));
          umma_commit(smem_u32(&sh->s_full[sb]));
        }
        ++ai;
      }
    }
  } else {
    const int quarter = warp & 3, half = (warp - 2) >> 2;
    const uint32_t t_s = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(half * 64);
    const int row = quarter * 32 + lane;  // row of the stationary tile
    const float sl2 = rsqrtf((float)HD) * CO_LOG2E;
    const unsigned long long sl2x2 = f32x2_pack(sl2, sl2);
    float m = -INFINITY, l = 0.f;
    bool ok = true;
    int t = 0;
    if (PASS == 2 && DEEP) {  // minus the lanes' log-sum-exps, from the key ranges of pass 1
      asm volatile("griddepcontrol.wait;" ::: "memory");
      const float2 *p = parts + ((size_t)s * Hkv + g) * deep_tiles * deep.splits * MT;
      for (int i = threadIdx.x - 64; i < lane_tiles * MT; i += 256) {
        const float2 *pi = p + (size_t)(i / MT) * deep.splits * MT + i % MT;
        const int written = (keys_of(i / MT) + deep.split_tiles - 1) / deep.split_tiles;
        float mm = -INFINITY, ll = 0.f;
#pragma unroll 8
        for (int r = 0; r < written; ++r) {
          const float2 x = pi[(size_t)r * MT];
          const float mt = fmaxf(mm, x.x), ref = mt == -INFINITY ? 0.f : mt;
          ll = ll * ex2_approx(mm - ref) + x.y * ex2_approx(x.x - ref);
          mm = mt;
        }
        sh->lse[i / MT][i % MT] = -(mm + log2f(ll));
      }
      asm volatile("bar.sync 1, 256;" ::: "memory");
    }
    for (int at = at0; at < at1; ++at) {
      int b0, b1;
      streamed(at, b0, b1);
      // pass 1: this lane's row inside the sequence, -1 for a lane that does not exist (it sees no key); pass 2: the key
      int own = PASS == 1 ? first + at * R + row / group : at * MT + row;
      if (PASS == 1 && (row >= R * group || own >= n)) own = -1;
      l = 0.f;
      for (int b = b0; b < b1 && ok; ++b, ++t) {
        const int sb = t & 1;
        ok = mbar_wait(smem_u32(&sh->s_full[sb]), (uint32_t)((t >> 1) & 1), abort_flag, status, W_MASS);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        tc_fence_after();
        // columns [lo, hi) of this thread's 64 are seen
        int lo = 0, hi = 64;
        if (PASS == 1) hi = own + 1 - (b * MT + half * 64);
        else {
          const int row0 = first + b * R;  // first row of the streamed tile
          lo = (own - row0) * group - half * 64;
          hi = min(R, n - row0) * group - half * 64;
        }
        // a warp that sees nothing has nothing to do: in DEEP, whose lanes can be few (elsewhere the test costs more than it saves)
        const bool any = !DEEP || __any_sync(0xffffffffu, hi > max(lo, 0) && lo < 64);
        uint32_t raw[64];
        if (any) {
          tmem_ld_32x32_raw(t_s + (uint32_t)(sb * MT), raw);
          tmem_ld_32x32_raw(t_s + (uint32_t)(sb * MT) + 32u, raw + 32);
          tmem_ld_wait();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sh->s_free[sb]));
        if (PASS == 1) {
          if (!any) continue;
          if (hi < 64) {
#pragma unroll
            for (int c = 0; c < 64; ++c)
              if (c >= hi) raw[c] = 0xff800000u;  // -inf
          }
          float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int c = 0; c < 64; c += 8) {
            mx[0] = fmax3(mx[0], __uint_as_float(raw[c]), __uint_as_float(raw[c + 1]));
            mx[1] = fmax3(mx[1], __uint_as_float(raw[c + 2]), __uint_as_float(raw[c + 3]));
            mx[2] = fmax3(mx[2], __uint_as_float(raw[c + 4]), __uint_as_float(raw[c + 5]));
            mx[3] = fmax3(mx[3], __uint_as_float(raw[c + 6]), __uint_as_float(raw[c + 7]));
          }
          const float mt = fmaxf(m, fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * sl2);
          const float ref = mt == -INFINITY ? 0.f : mt;
          const unsigned long long neg = f32x2_pack(-ref, -ref);
          unsigned long long sum0 = 0ull, sum1 = 0ull;
#pragma unroll
          for (int c = 0; c < 64; c += 4) {
            const unsigned long long x0 = f32x2_fma(f32x2_pack(__uint_as_float(raw[c]), __uint_as_float(raw[c + 1])), sl2x2, neg);
            const unsigned long long x1 = f32x2_fma(f32x2_pack(__uint_as_float(raw[c + 2]), __uint_as_float(raw[c + 3])), sl2x2, neg);
            sum0 = f32x2_add(sum0, ex2_approx_x2(x0));
            sum1 = f32x2_add(sum1, c % MT_POLY == MT_POLY - 4 ? ex2_poly_x2(x1) : ex2_approx_x2(x1));
          }
          float u0, u1;
          f32x2_unpack(f32x2_add(sum0, sum1), u0, u1);
          l = l * ex2_approx(m - ref) + (u0 + u1);
          m = mt;
        } else {
          const int ls = DEEP ? b : t % MT_LSE_STAGES;
          if (!DEEP) {
            ok = mbar_wait(smem_u32(&sh->l_full[ls]), (uint32_t)((t / MT_LSE_STAGES) & 1), abort_flag, status, W_MASS);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
          }
          const float4 *le = reinterpret_cast<const float4 *>(sh->lse[ls] + half * 64);
          if (!any) {
          } else if (lo <= 0 && hi >= 64) {
            unsigned long long sum0 = 0ull, sum1 = 0ull;
#pragma unroll
            for (int c = 0; c < 64; c += 4) {
              const float4 e = le[c >> 2];
              const unsigned long long x0 = f32x2_fma(f32x2_pack(__uint_as_float(raw[c]), __uint_as_float(raw[c + 1])), sl2x2,
                                                      f32x2_pack(e.x, e.y));
              const unsigned long long x1 = f32x2_fma(f32x2_pack(__uint_as_float(raw[c + 2]), __uint_as_float(raw[c + 3])), sl2x2,
                                                      f32x2_pack(e.z, e.w));
              sum0 = f32x2_add(sum0, ex2_approx_x2(x0));
              sum1 = f32x2_add(sum1, c % MT_POLY == MT_POLY - 4 ? ex2_poly_x2(x1) : ex2_approx_x2(x1));
            }
            float u0, u1;
            f32x2_unpack(f32x2_add(sum0, sum1), u0, u1);
            l += u0 + u1;
          } else {  // a tile on the diagonal or at the end: unseen columns are left out, whatever they hold
            float sum = 0.f;
#pragma unroll
            for (int c0 = 0; c0 < 64; c0 += 16) {
              if (c0 >= hi || c0 + 16 <= lo) continue;
#pragma unroll
              for (int c = c0; c < c0 + 16; ++c) {
                const float x = fmaf(__uint_as_float(raw[c]), sl2, sh->lse[ls][half * 64 + c]);
                sum += c >= lo && c < hi ? ex2_approx(x) : 0.f;
              }
            }
            l += sum;
          }
          if (!DEEP) {
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh->l_free[ls]));
          }
        }
      }
      if (!ok) l = NAN;  // a wait ran out (reported): nothing that looks like a result
      const int buf = (at - at0) & 1;
      sh->part_l[buf][half][row] = l;
      if (DEEP && PASS == 2) {
        // the two halves of the columns meet; two buffers, so that nobody overwrites what is still being read
        asm volatile("bar.sync 1, 256;" ::: "memory");
        if (half == 0 && own < n) mass[(size_t)g * n_total + start + own] = l + sh->part_l[buf][1][row];
      }
    }
    sh->part_m[half][row] = m;
  }
  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {  // a wait ran out: what this CTA has in flight ends before it leaves
    if (threadIdx.x == 0) {
      ring_landed(sh->a_full, A_BUFS, a_loads, &sh->last_flag, status, W_MASS);
      ring_landed(sh->b_full, STAGES, b_loads, &sh->last_flag, status, W_MASS);
      ring_landed(sh->l_full, MT_LSE_STAGES, l_loads, &sh->last_flag, status, W_MASS);
    } else if (threadIdx.x == 32) {
      umma_commit(smem_u32(&sh->done));
      mbar_wait(smem_u32(&sh->done), 0, &sh->last_flag, status, W_MASS);
    }
    __syncthreads();
  }
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)MT_TMEM_COLS)
                 : "memory");
  }
  if (DEEP && PASS == 2) return;
  if (csize > 1 && !SPLIT) co_cluster_sync();
  if ((rank == 0 || SPLIT) && threadIdx.x < MT) {
    const int row = threadIdx.x;
    float m = -INFINITY, l = 0.f;
    for (int r = 0; r < (SPLIT ? 1 : csize); ++r)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float lr = SPLIT ? sh->part_l[0][h][row] : *co_map_shared(&sh->part_l[0][h][row], r);
        if (PASS == 1) {
          const float mr = SPLIT ? sh->part_m[h][row] : *co_map_shared(&sh->part_m[h][row], r);
          const float mt = fmaxf(m, mr), ref = mt == -INFINITY ? 0.f : mt;
          l = l * ex2_approx(m - ref) + lr * ex2_approx(mr - ref);
          m = mt;
        } else {
          l += lr;
        }
      }
    if (SPLIT) parts[((((size_t)s * Hkv + g) * deep_tiles + at0) * deep.splits + rank) * MT + row] = make_float2(m, l);
    else if (PASS == 1) lse[lse_base + (size_t)at0 * MT + row] = -(m + log2f(l));  // lanes that do not exist: never looked at
    else if (at0 * MT + row < n) mass[(size_t)g * n_total + start + at0 * MT + row] = l;
  }
  if (csize > 1 && !SPLIT) co_cluster_sync();  // nobody leaves while its parts are being read
}

bool mass_tc_eligible(int dtype, int head_dim, int group) {
  return dtype == LAZY_BF16 && head_dim <= 128 && group <= MT;
}
int mass_seq_tiles(int n_seqs, int n_total, int group) { return n_total / (MT / group) + n_seqs + 1; }

// Key tiles per CTA so that all of them run at once: `most` to a sequence and `all` in all, `ctas` CTAs if none is cut.
int mass_range(int most, long long all, long long ctas) {
  const long long sms = sm_count();
  long long per = ctas < sms ? cdiv(most, (int)(sms / ctas)) : most;  // every sequence with as many ranges as the longest
  if (ctas < sms) {  // or as many as its length fills, one more for what is left over
    const long long b = (all + (sms - ctas) - 1) / (sms - ctas);
    if (b < per) per = b;
  }
  return (int)(per < 1 ? 1 : per);
}
// Whether both passes take the DEEP form (splits > 0): few lane tiles, many key tiles, a CTA for every (sequence, head).
MassDeep mass_deep(int n_seqs, int n_total, int max_len, int n_heads, int n_kv_heads, int window) {
  const int R = MT / (n_heads / n_kv_heads), rows = window > 0 && window < max_len ? window : max_len;
  const int lane_tiles = cdiv(rows, R), key_tiles = cdiv(max_len, MT);
  const long long heads = (long long)n_kv_heads * n_seqs, sms = sm_count();
  const long long all_lane = mass_tiles(lane_tiles, R, n_seqs, n_total) * n_kv_heads;
  const long long all_key = mass_tiles(key_tiles, MT, n_seqs, n_total) * n_kv_heads;
  if (lane_tiles > MT_DEEP_TILES || all_key <= 2 * sms || heads > sms) return {0, 0, 0, 0};
  MassDeep d;
  d.split_tiles = mass_range(key_tiles, all_key * lane_tiles, all_lane);
  if (d.split_tiles < cdiv(key_tiles, MT_DEEP_SPLITS)) d.split_tiles = cdiv(key_tiles, MT_DEEP_SPLITS);
  d.splits = cdiv(key_tiles, d.split_tiles);
  d.range_tiles = mass_range(key_tiles, all_key, heads);
  d.ranges = cdiv(key_tiles, d.range_tiles);
  return d;
}

template <int HD>
int mass_tc(cudaStream_t st, const void *q, int ldq, const void *k, int ldkv, const int32_t *cu, int n_seqs, int max_len,
            int n_total, int n_heads, int n_kv_heads, int window, float *lse, float *mass, DevStatus *status) {
  const int group = n_heads / n_kv_heads, R = MT / group;
  CUtensorMap mq, mk;
  LAZY_TRY(tma_map_heads_bf16(&mq, q, n_total, n_heads, HD, ldq, group, R));
  LAZY_TRY(tma_map_heads_bf16(&mk, k, n_total, n_kv_heads, HD, ldkv, 1, MT));
  const int rows = window > 0 && window < max_len ? window : max_len;
  const int lane_tiles = cdiv(rows, R), key_tiles = cdiv(max_len, MT), seq_tiles = mass_seq_tiles(n_seqs, n_total, group);
  const long long all_lane = mass_tiles(lane_tiles, R, n_seqs, n_total), all_key = mass_tiles(key_tiles, MT, n_seqs, n_total);
  if (lane_tiles > 65535 || key_tiles > 65535) return LAZY_E_CAPACITY;
  const MassDeep deep = mass_deep(n_seqs, n_total, max_len, n_heads, n_kv_heads, window);
  float2 *parts = reinterpret_cast<float2 *>(lse + (size_t)n_kv_heads * seq_tiles * MT);
  const MassGrid grid(n_seqs, max_len, n_total);
  auto launch = [&](auto kernel, int x, int tiles, int smem, int cluster, bool dependent) {
    return co_launch(kernel, grid.grid(x, n_seqs, tiles), dim3(MT_THREADS), smem, st, cluster, dependent, mq, mk, cu, max_len,
                     n_total, group, R, window, grid.by_tile, lse, seq_tiles, deep, parts, lane_tiles, mass, status);
  };
  if (deep.splits) {
    LAZY_TRY((co_allow_smem<mass_tc_kernel<1, HD, true>>(mass_smem<HD, true>)));
    LAZY_TRY((co_allow_smem<mass_tc_kernel<2, HD, true>>(mass_smem<HD, true>)));
    LAZY_TRY(launch(mass_tc_kernel<1, HD, true>, n_kv_heads * deep.splits, lane_tiles, mass_smem<HD, true>, 1, false));
    return launch(mass_tc_kernel<2, HD, true>, n_kv_heads, deep.ranges, mass_smem<HD, true>, 1, true);
  }
  const double seen = mass_seen(rows, max_len);
  const int c1 = mass_cluster(all_lane * n_kv_heads, key_tiles, seen, 2, MT_START, MT_JOIN);
  const int c2 = mass_cluster(all_key * n_kv_heads, lane_tiles, seen, 2, MT_START, MT_JOIN);
  LAZY_TRY((co_allow_smem<mass_tc_kernel<1, HD, false>>(mass_smem<HD, false>)));
  LAZY_TRY((co_allow_smem<mass_tc_kernel<2, HD, false>>(mass_smem<HD, false>)));
  LAZY_TRY(launch(mass_tc_kernel<1, HD, false>, n_kv_heads * c1, lane_tiles, mass_smem<HD, false>, c1, false));
  return launch(mass_tc_kernel<2, HD, false>, n_kv_heads * c2, key_tiles, mass_smem<HD, false>, c2, true);
}

}  // namespace

size_t attention_mass_scratch_need(int n_seqs, int n_total, int max_len, int n_heads, int n_kv_heads, int window) {
  const int group = n_heads / n_kv_heads;
  if (max_len > n_total) max_len = n_total;  // a bound may be any number
  const size_t general = (size_t)n_total * n_heads;
  if (group > MT) return general;
  const MassDeep deep = mass_deep(n_seqs, n_total, max_len, n_heads, n_kv_heads, window);
  const int lane_tiles = cdiv(window > 0 && window < max_len ? window : max_len, MT / group);
  const size_t tiled = (size_t)n_kv_heads * mass_seq_tiles(n_seqs, n_total, group) * MT +
                       (size_t)n_seqs * n_kv_heads * lane_tiles * deep.splits * MT * 2;
  return (general > tiled ? general : tiled) + 4;  // + 4: tiles start on a 16-byte boundary
}

// As much as any batch no larger needs: of the DEEP form's parts, which a larger batch may do without, the most there can be.
size_t attention_mass_scratch_floats(int n_seqs, int n_total, int max_len, int n_heads, int n_kv_heads, int window) {
  const int group = n_heads / n_kv_heads;
  if (max_len > n_total) max_len = n_total;
  const size_t general = (size_t)n_total * n_heads;
  if (group > MT) return general;
  size_t tiled = (size_t)n_kv_heads * mass_seq_tiles(n_seqs, n_total, group) * MT;
  const int key_tiles = cdiv(max_len, MT), sms = sm_count();
  if (mass_tiles(key_tiles, MT, n_seqs, n_total) * n_kv_heads > 2 * sms) {
    const int lane_tiles = cdiv(window > 0 && window < max_len ? window : max_len, MT / group);
    const size_t heads = (size_t)(n_seqs < sms / n_kv_heads ? n_seqs : sms / n_kv_heads) * n_kv_heads;
    tiled += heads * (lane_tiles < MT_DEEP_TILES ? lane_tiles : MT_DEEP_TILES) *
             (key_tiles < MT_DEEP_SPLITS ? key_tiles : MT_DEEP_SPLITS) * MT * 2;
  }
  return (general > tiled ? general : tiled) + 4;
}

int launch_attention_mass(cudaStream_t st, int dtype, const void *q, int ldq, const void *k, int ldkv,
                          const int32_t *cu, int n_seqs, int max_len, int n_total, int n_heads, int n_kv_heads,
                          int head_dim, int window, float *scratch, float *mass, DevStatus *status) {
  if (max_len > n_total) max_len = n_total;  // a bound may be any number
  if (n_seqs == 0 || max_len == 0) return LAZY_OK;
  if (mass_tc_eligible(dtype, head_dim, n_heads / n_kv_heads)) {
    float *lse = reinterpret_cast<float *>(align_up((uintptr_t)scratch, 16));
    return co_head_dim(head_dim, [&](auto hd) {
      return mass_tc<hd.value>(st, q, ldq, k, ldkv, cu, n_seqs, max_len, n_total, n_heads, n_kv_heads, window, lse, mass, status);
    });
  }
  if (dtype == LAZY_F32)
    return mass_general<float>(st, (const float *)q, ldq, (const float *)k, ldkv, cu, n_seqs, max_len, n_total, n_heads,
                               n_kv_heads, head_dim, window, scratch, mass, status);
  return mass_general<bf16>(st, (const bf16 *)q, ldq, (const bf16 *)k, ldkv, cu, n_seqs, max_len, n_total, n_heads,
                            n_kv_heads, head_dim, window, scratch, mass, status);
}

}  // namespace lazy
