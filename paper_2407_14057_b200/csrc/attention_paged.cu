// Attention of one or several new rows per sequence over a paged cache, softmax(q k / sqrt(dh)) v: row i of a sequence's T
// sees the first len - T + i + 1 of its tokens.
#include "attn_split.cuh"
#include "paged.cuh"
#include "rows_mma.cuh"

namespace lazy {

namespace {

typedef unsigned long long u64;

// ---- general form: fp32 and wide heads, on CUDA cores; partial softmaxes of split key ranges, then their merge ----------------------
// A CTA takes a range of keys for four columns (a column being one (row, query head)) of a key/value head, a warp eight keys at a time
// with its lanes along the head: 32 dot products, whose sums over the lanes are scattered to one a lane in 31 exchanges (each on its own
// takes five); the weights go back by 32 broadcasts.  16 sequences of 3000 tokens, 8 on 2 heads of 64, fp32 (49 MB): 25 us, with a row and
// head to a CTA 63.
constexpr int PW_COLS = 4, PW_KEYS = 8, PW_WARPS = 4, PW_THREADS = PW_WARPS * 32;

// Key ranges: enough CTAs for four on every SM, in whole tiles of keys.
inline int paged_wide_splits(long long pairs, int max_kv) { return attn_split_count(pairs, max_kv); }
inline long long paged_wide_tiles(int max_q, int n_heads, int n_kv_heads) {
  return ((long long)max_q * (n_heads / n_kv_heads) + PW_COLS - 1) / PW_COLS;
}

// grid (n_kv_heads * column tiles * splits, n_seqs); head width 32 E
template <typename T, int E>
__global__ void __launch_bounds__(PW_THREADS)
paged_wide_kernel(const PagedArgs a, int group, int tiles, int splits, int per_split, float *__restrict__ part_o,
                  float *__restrict__ part_ml, DevStatus *status) {
  constexpr int HD = 32 * E;
  __shared__ float so[PW_WARPS][PW_COLS][HD];
  __shared__ float2 sml[PW_WARPS][PW_COLS];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, s = blockIdx.y;
  int x = blockIdx.x;
  const int split = x % splits;
  x /= splits;
  const int g = x / tiles, c0 = (x - g * tiles) * PW_COLS;
  int start, rows, len;
  if (!paged_seq(a.kv, a.cu_q, s, a.n_rows, a.max_q, a.max_kv, blockIdx.x == 0 && threadIdx.x == 0, status, start, rows, len)) return;
  const int cols = min(PW_COLS, (int)min((long long)rows * group - c0, (long long)PW_COLS));
  if (cols <= 0) return;
  const int k0 = split * per_split, k1 = k0 + min(len - k0, per_split);  // k0 + per_split may pass 2^31
  const int32_t *table = a.kv.table + (size_t)s * a.kv.ld_table;
  const T *kp = (const T *)a.kv.k + (long long)g * a.kv.head_stride + lane, *vp = (const T *)a.kv.v + (long long)g * a.kv.head_stride + lane;
  auto row_of = [&](int c) { return (c0 + c) / group; };
  auto head_of = [&](int c) { return g * group + (c0 + c) % group; };
  float q[PW_COLS][E], o[PW_COLS][E], m = -INFINITY, l = 0.f;  // m and l of column lane % 4, l of this lane's keys
  const float scale = rsqrtf((float)HD) * CO_LOG2E;
#pragma unroll
  for (int c = 0; c < PW_COLS; ++c)
#pragma unroll
    for (int e = 0; e < E; ++e) {
      q[c][e] = c < cols ? Elem<T>::to_f(((const T *)a.q)[(size_t)(start + row_of(c)) * a.ldq + (size_t)head_of(c) * HD + e * 32 + lane]) * scale : 0.f;
      o[c][e] = 0.f;
    }
  const int my_c = lane & 3, my_key = lane >> 2;
  const int vis = my_c < cols ? min(len - rows + row_of(my_c) + 1, k1) : 0;  // keys below it are seen by this lane's column
  for (int j0 = k0 + warp * PW_KEYS; j0 < k1; j0 += PW_WARPS * PW_KEYS) {
    const int j = min(j0 + (lane & 7), k1 - 1), nth = j / a.kv.page_size, page = table[nth];
    const bool in = page >= 0 && page < a.kv.n_pages;
    if (!in && lane < PW_KEYS) dev_fail(status, LAZY_E_BADARG, W_PAGED, s, page);
    const long long off = (long long)page * a.kv.page_stride + (long long)(j - nth * a.kv.page_size) * a.kv.slot_stride;
    const uint32_t there = __ballot_sync(0xffffffffu, in && j0 + (lane & 7) < k1) & 0xffu;
    float v[PW_KEYS][E], d[PW_KEYS * PW_COLS];
    {
      float k[PW_KEYS][E];
#pragma unroll
      for (int i = 0; i < PW_KEYS; ++i) {
        const long long at = __shfl_sync(0xffffffffu, off, i);
#pragma unroll
        for (int e = 0; e < E; ++e) k[i][e] = there >> i & 1u ? Elem<T>::to_f(kp[at + e * 32]) : 0.f;
        if (E <= 4) {
#pragma unroll
          for (int e = 0; e < E; ++e) v[i][e] = there >> i & 1u ? Elem<T>::to_f(vp[at + e * 32]) : 0.f;
        }
      }
#pragma unroll
      for (int i = 0; i < PW_KEYS; ++i)
#pragma unroll
        for (int c = 0; c < PW_COLS; ++c) {
          float sum = q[c][0] * k[i][0];
#pragma unroll
          for (int e = 1; e < E; ++e) sum = fmaf(q[c][e], k[i][e], sum);
          d[i * PW_COLS + c] = sum;
        }
    }
    if (E > 4) {
#pragma unroll
      for (int i = 0; i < PW_KEYS; ++i) {
        const long long at = __shfl_sync(0xffffffffu, off, i);
#pragma unroll
        for (int e = 0; e < E; ++e) v[i][e] = there >> i & 1u ? Elem<T>::to_f(vp[at + e * 32]) : 0.f;
      }
    }
    // sums over the lanes, that of key i and column c to lane 4 i + c
#pragma unroll
    for (int n = 16; n > 0; n >>= 1)
#pragma unroll
      for (int i = 0; i < n; ++i) {
        const float keep = lane & n ? d[i + n] : d[i], give = lane & n ? d[i] : d[i + n];
        d[i] = keep + __shfl_xor_sync(0xffffffffu, give, n);
      }
    const float logit = (there >> my_key & 1u) && j0 + my_key < vis ? d[0] : -INFINITY;
    float most = fmaxf(logit, __shfl_xor_sync(0xffffffffu, logit, 4));
    most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 8));
    most = fmaxf(m, fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 16)));
    const float ref = most == -INFINITY ? 0.f : most;  // nothing seen so far: every weight is 2^-inf = 0
    const float alpha = exp2f(m - ref), p = exp2f(logit - ref);
    m = most;
    l = fmaf(l, alpha, p);
    if (__any_sync(0xffffffffu, alpha != 1.f)) {
#pragma unroll
      for (int c = 0; c < PW_COLS; ++c) {
        const float f = __shfl_sync(0xffffffffu, alpha, c);
#pragma unroll
        for (int e = 0; e < E; ++e) o[c][e] *= f;
      }
    }
#pragma unroll
    for (int i = 0; i < PW_KEYS; ++i)
#pragma unroll
      for (int c = 0; c < PW_COLS; ++c) {
        const float w = __shfl_sync(0xffffffffu, p, i * PW_COLS + c);
        if (w != 0.f) {  // the whole warp alike; a value that a column does not see must not reach it as 0 x inf
#pragma unroll
          for (int e = 0; e < E; ++e) o[c][e] = fmaf(w, v[i][e], o[c][e]);
        }
      }
  }
  l += __shfl_xor_sync(0xffffffffu, l, 4);
  l += __shfl_xor_sync(0xffffffffu, l, 8);
  l += __shfl_xor_sync(0xffffffffu, l, 16);
  if (lane < PW_COLS) sml[warp][lane] = make_float2(m, l);
#pragma unroll
  for (int c = 0; c < PW_COLS; ++c)
#pragma unroll
    for (int e = 0; e < E; ++e) so[warp][c][e * 32 + lane] = o[c][e];
  __syncthreads();
  for (int i = threadIdx.x; i < cols * HD; i += PW_THREADS) {
    const int c = i / HD, at = i - c * HD;
    float top = -INFINITY, sum = 0.f, out = 0.f;
#pragma unroll
    for (int w = 0; w < PW_WARPS; ++w) top = fmaxf(top, sml[w][c].x);
#pragma unroll
    for (int w = 0; w < PW_WARPS; ++w) {
      const float f = exp2f(sml[w][c].x - (top == -INFINITY ? 0.f : top));
      sum = fmaf(sml[w][c].y, f, sum);
      if (f != 0.f) out = fmaf(so[w][c][at], f, out);
    }
    if (splits == 1) {
      ((T *)a.o)[((size_t)(start + row_of(c)) * a.n_heads + head_of(c)) * HD + at] = Elem<T>::from_f(sum == 0.f ? 0.f : out / sum);
    } else {
      const size_t part = (((size_t)s * (gridDim.x / splits) + x) * PW_COLS + c) * splits + split;
      part_o[part * HD + at] = out;
      if (at == 0) {
        part_ml[part * 2] = top;
        part_ml[part * 2 + 1] = sum;
      }
    }
  }
}

// grid (n_heads, n_rows)
template <typename T>
__global__ void __launch_bounds__(AS_THREADS)
paged_merge_kernel(const PagedArgs a, const float *__restrict__ part_o, const float *__restrict__ part_ml, int tiles, int splits) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int h = blockIdx.x, r = blockIdx.y;
  const int s = a.cu_q ? paged_find_seq(a.cu_q, a.n_seqs, r) : r;
  int start, rows, len;
  if (s < 0 || !paged_seq(a.kv, a.cu_q, s, a.n_rows, a.max_q, a.max_kv, false, nullptr, start, rows, len) || r < start || r >= start + rows)
    return;  // the row is left as it was
  const int group = a.n_heads / a.n_kv_heads, g = h / group, c = (r - start) * group + h - g * group;
  const size_t part = ((((size_t)s * a.n_kv_heads + g) * tiles + c / PW_COLS) * PW_COLS + c % PW_COLS) * splits;
  attn_split_merge<T>(part_o + part * a.head_dim, part_ml + part * 2, splits, a.head_dim, (T *)a.o + ((size_t)r * gridDim.x + h) * a.head_dim,
                      nullptr);
}

template <typename T, int E>
int paged_wide(cudaStream_t st, const PagedArgs &a, float *scratch, DevStatus *status) {
  const long long tiles = paged_wide_tiles(a.max_q, a.n_heads, a.n_kv_heads), pairs = tiles * a.n_kv_heads;  // of a sequence
  const int splits = paged_wide_splits(pairs * a.n_seqs, a.max_kv);
  if (pairs * splits > 0x7fffffffLL) return LAZY_E_CAPACITY;
  float *part_o = scratch, *part_ml = scratch + (size_t)pairs * a.n_seqs * PW_COLS * splits * a.head_dim;
  LAZY_TRY(co_launch(paged_wide_kernel<T, E>, dim3((unsigned)(pairs * splits), a.n_seqs), dim3(PW_THREADS), 0, st, 1, false, a,
                     a.n_heads / a.n_kv_heads, (int)tiles, splits, attn_split_keys(a.max_kv, splits), part_o, part_ml, status));
  if (splits == 1) return LAZY_OK;
  return co_launch(paged_merge_kernel<T>, dim3(a.n_heads, a.n_rows), dim3(AS_THREADS), 0, st, 1, true, a, part_o, part_ml, (int)tiles, splits);
}
int paged_f32(cudaStream_t st, const PagedArgs &a, float *scratch, DevStatus *status) {
  switch (a.head_dim) {
    case 32: return paged_wide<float, 1>(st, a, scratch, status);
    case 64: return paged_wide<float, 2>(st, a, scratch, status);
    case 96: return paged_wide<float, 3>(st, a, scratch, status);
    case 128: return paged_wide<float, 4>(st, a, scratch, status);
    case 160: return paged_wide<float, 5>(st, a, scratch, status);
    case 192: return paged_wide<float, 6>(st, a, scratch, status);
    case 224: return paged_wide<float, 7>(st, a, scratch, status);
    case 256: return paged_wide<float, 8>(st, a, scratch, status);
  }
  return LAZY_E_BADARG;
}

// ---- bf16, head width up to 128: warp-level MMA over equal shares of the batch's keys -------------------------------------------
// The work is cut into units of 64 keys of one (sequence, key/value head, tile of columns), a column being one (row, query head); units
// lie in the order of sequences, heads, column tiles and keys, and every CTA takes an equal range of them, whatever the
// lengths: it runs through the end of one pair, whole pairs, and the start of another.  A warp takes every fourth 16 keys.  What a CTA
// has of a whole pair it writes to o; of a part, the maximum, sum and unnormalised output go to the scratch, a
// pair's first to place 1, a later one to place 0.  A second launch has a CTA per place 1 and adds the parts up in order.
// Bound by reading the keys and values: 16 sequences of up to 16384 tokens, 32 on 8 heads (981 MB) 155 us, 6.3 TB/s, 96 % of the copy rate; 32
// sequences of 1 to 4094 (238 MB) 46 us, of which the first loads wait 4 and the second launch takes 4.
constexpr int PG_UNIT = 64;
constexpr int PG_LEAST = 4;  // units that a CTA is worth starting for (2 to 16: the same but for calls of a few microseconds)
// Units that go by while a CTA turns to another pair: they count at the pair's start, so that a CTA with many short sequences has fewer keys
// (the 32 sequences above: 54 us with none, 48 with one or three, 47 with two).
constexpr int PG_SWITCH = 2;
constexpr int PG_MERGE_THREADS = 512;
// Where all pairs run at once in clusters of up to 16 CTAs, and a CTA has few units of its pair, a cluster holds a pair, its CTAs
// taking turns at the units, and the parts meet in distributed shared memory: one launch, and the first pages are asked for with the
// length.  One sequence of 1024 tokens, 32 heads: 6.4 us, 10.4 in two launches; 16 of 2000 on 8 heads: 25 and 31; with more than 16 units
// to a CTA the two launches are as fast (one sequence of 16000: 21 either way), and know the lengths.
constexpr int PG_MAX_CLUSTER = 16;
constexpr int PG_JOIN_UNITS = 16;
// Warps of a CTA, groups of 16 keys that a warp has asked for or at hand, CTAs to an SM.  12 warps keep the memory busy; a warp by itself
// takes a microsecond for 16 keys, whatever is at hand, so that a few large CTAs finish sooner than as many small ones.
struct PgDepth {
  int warps, stages, ctas;
};
constexpr PgDepth PG_WIDE = {4, 2, 3};
constexpr PgDepth PG_DEEP = {8, 2, 1};

// A part that other CTAs continue, as many of them as `more`, and where the pair's outputs are: columns [c0, c0 + cols) of key/value
// head g for the rows from `start` on.
struct __align__(16) PgSplit {
  int more, start, g, c0, cols, unused[3];
};
struct PgScratch {
  PgSplit *split;    // [CTAs]
  float *ml, *o;     // [CTAs][2][columns][2], [CTAs][2][columns][HD]
};
// Blocks of eight columns that a CTA takes, by the columns that a key/value head may have.  Four at a time read the keys of 32 columns
// once instead of twice, but take the registers of a third CTA and spill: when tried, 16 sequences of 3000 tokens, 8 rows of 4 heads, took 66 us
// with four blocks and 69 with two, four sequences with drafts 25 and 20.  With two, later steps have brought them to 65 and 18.6.
inline int pg_blocks(long long columns) { return columns <= 8 ? 1 : 2; }
inline int pg_grid() { return sm_count() * PG_WIDE.ctas; }
// floats; the parts' order in memory is splits, maxima and sums, outputs (+ 4: they start on a 16-byte boundary)
inline size_t pg_scratch_floats(int blocks, int head_dim) { return (size_t)pg_grid() * (8 + 16 * blocks * (2 + head_dim)) + 4; }
inline PgScratch pg_scratch(float *scratch, int blocks) {
  PgScratch c;
  c.split = reinterpret_cast<PgSplit *>(align_up((uintptr_t)scratch, 16));
  c.ml = reinterpret_cast<float *>(c.split + pg_grid());
  c.o = c.ml + (size_t)pg_grid() * 16 * blocks * 2;
  return c;
}

struct PgSeq {
  int start, rows, len, tiles, cts;  // cts: column tiles
  // what a pair counts for in the CTAs' shares, and the sequence
  __device__ __forceinline__ int share() const { return tiles + PG_SWITCH; }
  __device__ __forceinline__ long long units(int n_kv_heads) const { return rows ? (long long)share() * cts * n_kv_heads : 0; }
};
template <int COLS>
__device__ __forceinline__ PgSeq pg_seq(const PagedArgs &a, int s, int group, bool report, DevStatus *status) {
  PgSeq q;
  if (!paged_seq(a.kv, a.cu_q, s, a.n_rows, a.max_q, a.max_kv, report, status, q.start, q.rows, q.len)) q.rows = 0;
  q.tiles = q.rows ? (q.len + PG_UNIT - 1) / PG_UNIT : 0;
  q.cts = (int)(((long long)q.rows * group + COLS - 1) / COLS);
  return q;
}

template <int HD, int NT, int WARPS>
struct PgShared {
  float m[NT * 8], l[NT * 8];  // the CTA's part, read by the cluster
  float wm[WARPS][NT * 8], wl[WARPS][NT * 8];
  long long scan[WARPS];
  long long base;  // units of the sequences before `s`
  int s;
};

// JOIN: a cluster per pair, see above.  WHOLE: 16 keys from a multiple of 16 on lie in one page.
template <int HD, int NT, bool WHOLE, bool JOIN, int WARPS, int STAGES, int CTAS>
__global__ void __launch_bounds__(WARPS * 32, CTAS)
paged_mma_kernel(const PagedArgs a, int group, int max_cts, PgScratch scratch, DevStatus *status) {
  using Rows = RowsMma<HD, NT>;
  constexpr int COLS = NT * 8, THREADS = WARPS * 32, PER_UNIT = PG_UNIT / RM_KEYS;  // a unit is four groups of 16 keys
  extern __shared__ __align__(128) uint8_t paged_smem[];
  __shared__ PgShared<HD, NT, WARPS> sh;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, Hkv = a.n_kv_heads;
  const int csize = JOIN ? (int)co_cluster_size() : 1, rank = JOIN ? (int)co_cluster_rank() : 0, cta = blockIdx.x;
  int s, g, ct, first, jump, early = 0;  // the pair, and this CTA's units of it: first, first + jump, ...
  long long base = 0, total = 0, u0 = 0, u1 = 1;
  int ctas = 1;
  PgSeq seq;
  const int shift = (a.kv.page_size & (a.kv.page_size - 1)) == 0 ? __ffs(a.kv.page_size) - 1 : -1;  // of a power of two: no divisions
  auto nth_page = [&](int j) { return shift >= 0 ? j >> shift : j / a.kv.page_size; };
  auto page_of = [&](int s, int j) { return a.kv.table[(size_t)s * a.kv.ld_table + nth_page(j)]; };
  const long long slot_stride = a.kv.slot_stride, mine_in_run = rows_mine<HD>(slot_stride);
  auto first_of = [&](int c) { return total * c / ctas; };
  if (JOIN) {
    int pair = blockIdx.x / csize;
    ct = pair % max_cts;
    pair /= max_cts;
    s = pair / Hkv;
    g = pair - s * Hkv;
    first = rank;
    jump = csize;
    // asked for before the length is known: it may name a page that the sequence has not
    first += warp / PER_UNIT * jump;  // four warps to a unit
    jump *= WARPS / PER_UNIT;
    early = page_of(s, min((first * PER_UNIT + warp % PER_UNIT) * RM_KEYS + (WHOLE ? 0 : lane & 15), a.max_kv - 1));
    seq = pg_seq<COLS>(a, s, group, g == 0 && ct == 0 && rank == 0 && threadIdx.x == 0, status);
    if (ct >= seq.cts) return;  // the whole cluster alike
  } else {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    // ---- this CTA's range of units
    const int per = (a.n_seqs + THREADS - 1) / THREADS, s0 = threadIdx.x * per, s1 = min(s0 + per, a.n_seqs);
    long long mine = 0;
    for (int i = s0; i < s1; ++i) mine += pg_seq<COLS>(a, i, group, cta == 0, status).units(Hkv);
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long up = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += up;
    }
    if (lane == 31) sh.scan[warp] = incl;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
      if (w < warp) incl += sh.scan[w];
      total += sh.scan[w];
    }
    ctas = (int)min((long long)gridDim.x, (total + PG_LEAST - 1) / PG_LEAST);
    if (cta >= ctas) {
      if (threadIdx.x == 0) scratch.split[cta].more = 0;
      return;
    }
    u0 = first_of(cta);
    u1 = first_of(cta + 1);
    if (incl - mine <= u0 && u0 < incl) {
      long long at = incl - mine;
      int i = s0;
      while (i + 1 < s1) {
        const long long n = pg_seq<COLS>(a, i, group, false, status).units(Hkv);
        if (u0 < at + n) break;
        at += n;
        ++i;
      }
      sh.s = i;
      sh.base = at;
    }
    __syncthreads();
    s = sh.s;
    base = sh.base;
    seq = pg_seq<COLS>(a, s, group, false, status);
    jump = 1;
  }
  const uint32_t stages = smem_u32(paged_smem) + warp * STAGES * Rows::STAGE;
  PgSplit split = {};
  for (long long u = u0; u < u1; u = JOIN ? u1 : u) {
    int count;           // units of this CTA
    long long pair0 = 0;  // the pair's first unit
    if (JOIN) {
      count = first < seq.tiles ? (seq.tiles - first + jump - 1) / jump : 0;
    } else {
      while (u >= base + seq.units(Hkv)) {
        if (s + 1 >= a.n_seqs) {  // the tables changed meanwhile
          if (threadIdx.x == 0) scratch.split[cta].more = 0;
          return;
        }
        base += seq.units(Hkv);
        seq = pg_seq<COLS>(a, ++s, group, false, status);
      }
      const int pair = (int)((u - base) / seq.share());
      g = pair / seq.cts;
      ct = pair - g * seq.cts;
      pair0 = base + (long long)pair * seq.share();
      first = max((int)(u - pair0) - PG_SWITCH, 0);
      const int share_end = (int)min((long long)seq.share(), u1 - pair0);
      u = pair0 + share_end;
      count = share_end - PG_SWITCH - first;
      if (count <= 0) continue;  // the range ends before the pair's keys
    }
    const int c0 = ct * COLS, cols = min(COLS, seq.rows * group - c0);
    const bf16 *kp = (const bf16 *)a.kv.k + (long long)g * a.kv.head_stride, *vp = (const bf16 *)a.kv.v + (long long)g * a.kv.head_stride;
    // group i of this warp: keys [j0, j0 + 16); the page of its keys (WHOLE: one for all of them) is asked for a group ahead
    auto first_key = [&](int i) { return ((first + i * jump) * PER_UNIT + warp % PER_UNIT) * RM_KEYS; };
    auto ask = [&](int i) { return i < count ? page_of(s, min(first_key(i) + (WHOLE ? 0 : lane & 15), seq.len - 1)) : 0; };
    int next = JOIN && WHOLE ? early : ask(0);  // an early page beyond the length is not looked at
    u64 there = 0;  // of the stages in flight, 16 bits each: keys whose pages are in the pool
    int put = 0, take = 0;
    auto request = [&](int i) {
      const int j0 = first_key(i), page = next;
      next = ask(i + 1);
      if (i < count && j0 < seq.len) {
        const bool in = (uint32_t)page < (uint32_t)a.kv.n_pages;
        const int j = WHOLE ? j0 : min(j0 + (lane & 15), seq.len - 1), left = seq.len - j0;
        const int at = shift >= 0 ? j & (a.kv.page_size - 1) : j - nth_page(j) * a.kv.page_size;
        const long long off = page * a.kv.page_stride + at * slot_stride;
        const uint32_t to = stages + put * Rows::STAGE;
        uint32_t ok = 0xffffu;
        if (WHOLE && in && left >= RM_KEYS) {
          rows_load_run<HD>(to, kp + off, vp + off, slot_stride, mine_in_run);
        } else {
          if (!in && (WHOLE ? lane == 0 : j0 + (lane & 15) < seq.len)) dev_fail(status, LAZY_E_BADARG, W_PAGED, s, page);
          ok &= __ballot_sync(0xffffffffu, in);  // WHOLE: all lanes alike
          rows_load<HD>(to, [&](int r, const bf16 *&kr, const bf16 *&vr) {
            const long long o = WHOLE ? off + r * slot_stride : __shfl_sync(0xffffffffu, off, r);
            const bool there = (ok >> r & 1u) && r < left;
            kr = kp + (there ? o : 0);
            vr = vp + (there ? o : 0);
            return there;
          });
        }
        there = (there & ~(0xffffull << (16 * put))) | (u64)ok << (16 * put);
      }
      put = put + 1 == STAGES ? 0 : put + 1;
      rm_cp_commit();
    };
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) request(i);
    Rows rows;
    int t_vis[NT][2];  // tokens that this lane's columns see
    rows.init([&](int c) -> const bf16 * {
      if (c >= cols) return nullptr;
      const int t = (c0 + c) / group, h = c0 + c - t * group;
      return (const bf16 *)a.q + (size_t)(seq.start + t) * a.ldq + (size_t)(g * group + h) * HD;
    });
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        t_vis[t][i] = seq.len - seq.rows + min((c0 + t * 8 + (lane & 3) * 2 + i) / group, seq.rows - 1) + 1;
    const int least = seq.len - seq.rows + 1;  // what every row sees
#pragma unroll 1
    for (int i = 0; i < count; ++i) {
      request(i + STAGES - 1);
      rm_cp_wait<STAGES - 1>();
      __syncwarp();
      const int j0 = first_key(i);
      if (j0 < seq.len) {
        int vis[NT][2];
        const uint32_t stage = stages + take * Rows::STAGE, ok = (uint32_t)(there >> (16 * take)) & 0xffffu;
        if (j0 + RM_KEYS <= least && ok == 0xffffu) {
          rows.template step<false, true>(stage, vis, ok);
        } else {
#pragma unroll
          for (int t = 0; t < NT; ++t) vis[t][0] = t_vis[t][0] - j0, vis[t][1] = t_vis[t][1] - j0;
          if (j0 + RM_KEYS > least && seq.rows > 1) rows.template step<true, false>(stage, vis, ok);
          else rows.template step<false, false>(stage, vis, ok);
        }
      }
      take = take + 1 == STAGES ? 0 : take + 1;
      __syncwarp();  // the stage may be requested again
    }
    rm_cp_wait<0>();
    rows.finish();
    // ---- the CTA's part: the warps' outputs against the common maximum, added in warp order
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
    float *wo = reinterpret_cast<float *>(paged_smem);  // [warp][column][HD]
    float *co = wo;                                     // [column][HD]: the part, read by the cluster; written where warp 0's was
    static_assert(WARPS * COLS * HD * 4 <= WARPS * STAGES * Rows::STAGE, "the stages hold the outputs in the end");
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int c = t * 8 + (lane & 3) * 2 + i;
        if (c >= cols) continue;
        float mx = sh.wm[0][c];
#pragma unroll
        for (int w = 1; w < WARPS; ++w) mx = fmaxf(mx, sh.wm[w][c]);
        const float f = ex2_approx(rows.m[t][i] - (mx == -INFINITY ? 0.f : mx)) * WEIGHT_UNLIFT;
#pragma unroll
        for (int k = 0; k < HD / 16; ++k) {
          wo[(warp * COLS + c) * HD + k * 16 + (lane >> 2)] = rows.o[t][k][i] * f;
          wo[(warp * COLS + c) * HD + k * 16 + 8 + (lane >> 2)] = rows.o[t][k][2 + i] * f;
        }
      }
    __syncthreads();
    const bool all = !JOIN && first == 0 && count == seq.tiles;
    const size_t place = JOIN ? 0 : ((size_t)cta * 2 + (first == 0)) * COLS;
    auto output = [&](int c, int d) {
      const int t = (c0 + c) / group, h = c0 + c - t * group;
      return (bf16 *)a.o + ((size_t)(seq.start + t) * a.n_heads + g * group + h) * HD + d;
    };
    for (int e = threadIdx.x; e < cols * (HD / 8); e += THREADS) {
      const int c = e / (HD / 8), d = e % (HD / 8) * 8;
      float m = -INFINITY, l = 0.f, x[8];
#pragma unroll
      for (int w = 0; w < WARPS; ++w) m = fmaxf(m, sh.wm[w][c]);
#pragma unroll
      for (int w = 0; w < WARPS; ++w) l += sh.wl[w][c] * ex2_approx(sh.wm[w][c] - (m == -INFINITY ? 0.f : m));
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = 0.f;
#pragma unroll
      for (int w = 0; w < WARPS; ++w)
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] += wo[(w * COLS + c) * HD + d + i];
      if (all || (JOIN && csize == 1)) {
        const float inv = l == 0.f ? 0.f : 1.f / l;
        Vec16<bf16> y;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= inv;
        y.pack(x);
        y.store(output(c, d));
      } else {
        if (d == 0) {
          if (JOIN) sh.m[c] = m, sh.l[c] = l;
          else *reinterpret_cast<float2 *>(scratch.ml + (place + c) * 2) = make_float2(m, l);
        }
        float4 *o = reinterpret_cast<float4 *>(JOIN ? co + c * HD + d : scratch.o + (place + c) * HD + d);
        o[0] = make_float4(x[0], x[1], x[2], x[3]);
        o[1] = make_float4(x[4], x[5], x[6], x[7]);
      }
    }
    if (JOIN) {
      if (csize == 1) return;
      co_cluster_sync();
      // every CTA a share of the outputs, four elements to a thread; all reads of the others' memory are in flight together
      for (int e = rank * THREADS + threadIdx.x; e < cols * (HD / 4); e += csize * THREADS) {
        const int c = e / (HD / 4), d = e % (HD / 4) * 4;
        float m[PG_MAX_CLUSTER], l[PG_MAX_CLUSTER];
#pragma unroll
        for (int r = 0; r < PG_MAX_CLUSTER; ++r) {
          m[r] = r < csize ? *co_map_shared(&sh.m[c], r) : -INFINITY;
          l[r] = r < csize ? *co_map_shared(&sh.l[c], r) : 0.f;
        }
        float most = -INFINITY, sum = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int r0 = 0; r0 < PG_MAX_CLUSTER; r0 += 8) {
          if (r0 >= csize) break;
          float4 x[8];
#pragma unroll
          for (int r = 0; r < 8; ++r)
            x[r] = r0 + r < csize ? *co_map_shared(reinterpret_cast<float4 *>(co + c * HD + d), r0 + r) : make_float4(0.f, 0.f, 0.f, 0.f);
          if (r0 == 0) {
#pragma unroll
            for (int r = 0; r < PG_MAX_CLUSTER; ++r) most = fmaxf(most, m[r]);
          }
#pragma unroll
          for (int r = 0; r < 8; ++r) {
            const float f = ex2_approx(m[r0 + r] - (most == -INFINITY ? 0.f : most));
            sum = fmaf(l[r0 + r], f, sum);
            o = make_float4(fmaf(x[r].x, f, o.x), fmaf(x[r].y, f, o.y), fmaf(x[r].z, f, o.z), fmaf(x[r].w, f, o.w));
          }
        }
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        *reinterpret_cast<uint2 *>(output(c, d)) = make_uint2(bf16x2_pack(o.x * inv, o.y * inv), bf16x2_pack(o.z * inv, o.w * inv));
      }
      co_cluster_sync();  // nobody leaves while its part is being read
      return;
    }
    if (first == 0 && !all) {  // the range ends here; the pair's last unit is that of the last CTA that begins before it
      const long long last = pair0 + seq.share() - 1;
      split = {(int)(((last + 1) * ctas + total - 1) / total) - 1 - cta, seq.start, g, c0, cols, {}};
    }
    if (u < u1) __syncthreads();  // the stages and the maxima have been read
  }
  if (threadIdx.x == 0) scratch.split[cta] = split;
}

// Adds up the parts of the pair that CTA blockIdx.x began and did not finish.  A warp per column, several to one where there are few.
template <int HD, int COLS>
__global__ void __launch_bounds__(PG_MERGE_THREADS)
paged_mma_merge_kernel(const PagedArgs a, int group, PgScratch scratch) {
  constexpr int WARPS = PG_MERGE_THREADS / 32, WIDE = HD / 4, BATCH = 8;  // lanes 0..WIDE-1 hold four of a column's elements each
  static_assert(COLS <= WARPS, "a warp per column");
  __shared__ float4 part[WARPS][32];
  __shared__ float2 part_ml[WARPS];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int cta = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const PgSplit p = scratch.split[cta];
  if (p.more == 0) return;
  const int n = p.more + 1;
  int share = 1;  // warps to a column
  while (share * 2 * p.cols <= WARPS) share *= 2;
  const int c = warp / share, first = warp % share;
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  auto place = [&](int i) { return ((size_t)(cta + i) * 2 + (i == 0)) * COLS + c; };
  if (c < p.cols) {
    for (int i0 = first; i0 < n; i0 += share * BATCH) {
      float2 ml[BATCH];
      float4 x[BATCH];
#pragma unroll
      for (int b = 0; b < BATCH; ++b) {
        const int i = i0 + b * share;
        ml[b] = i < n ? *reinterpret_cast<const float2 *>(scratch.ml + place(i) * 2) : make_float2(-INFINITY, 0.f);
        x[b] = i < n && lane < WIDE ? *reinterpret_cast<const float4 *>(scratch.o + place(i) * HD + lane * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
      float mx = m;
#pragma unroll
      for (int b = 0; b < BATCH; ++b) mx = fmaxf(mx, ml[b].x);
      const float ref = mx == -INFINITY ? 0.f : mx, f = ex2_approx(m - ref);
      l *= f;
      o = make_float4(o.x * f, o.y * f, o.z * f, o.w * f);
      m = mx;
#pragma unroll
      for (int b = 0; b < BATCH; ++b) {
        const float w = ex2_approx(ml[b].x - ref);
        l = fmaf(ml[b].y, w, l);
        o = make_float4(fmaf(x[b].x, w, o.x), fmaf(x[b].y, w, o.y), fmaf(x[b].z, w, o.z), fmaf(x[b].w, w, o.w));
      }
    }
  }
  part[warp][lane] = o;
  if (lane == 0) part_ml[warp] = make_float2(m, l);
  __syncthreads();
  if (c >= p.cols || first != 0 || lane >= WIDE) return;
  for (int w = 0; w < share; ++w) m = fmaxf(m, part_ml[warp + w].x);
  const float ref = m == -INFINITY ? 0.f : m;
  l = 0.f;
  o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int w = 0; w < share; ++w) {
    const float2 ml = part_ml[warp + w];
    const float f = ex2_approx(ml.x - ref);
    const float4 x = part[warp + w][lane];
    l = fmaf(ml.y, f, l);
    o = make_float4(fmaf(x.x, f, o.x), fmaf(x.y, f, o.y), fmaf(x.z, f, o.z), fmaf(x.w, f, o.w));
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const int t = (p.c0 + c) / group, h = p.c0 + c - t * group;
  *reinterpret_cast<uint2 *>((bf16 *)a.o + ((size_t)(p.start + t) * a.n_heads + p.g * group + h) * HD + lane * 4) =
      make_uint2(bf16x2_pack(o.x * inv, o.y * inv), bf16x2_pack(o.z * inv, o.w * inv));
}

// How a launch is shaped: CTAs of a cluster per pair (0: equal shares of all keys), and whether they are the large ones.
struct PgShape {
  int cluster;
  bool deep;
};
PgShape paged_shape(const PagedArgs &a, int max_cts) {
  const long long pairs = (long long)a.n_seqs * a.n_kv_heads * max_cts;
  if (a.max_kv < 1) return {0, false};
  auto largest = [&](PgDepth d) {  // of which all run at once, and every warp has something to do
    int c = 1;
    while (c < PG_MAX_CLUSTER && pairs * c * 2 <= co_cluster_ctas(c * 2, d.ctas) && a.max_kv > c * d.warps * RM_KEYS) c *= 2;
    return pairs * c <= co_cluster_ctas(c, d.ctas) ? c : 0;
  };
  const PgDepth d = PG_WIDE;
  const int wide = largest(d), deep = largest(PG_DEEP);
  // as many SMs as possible, then as many warps
  const long long sms = sm_count(), wide_sms = min(pairs * wide, sms), deep_sms = min(pairs * deep, sms);
  const bool large = deep_sms > wide_sms || (deep_sms == wide_sms && deep * PG_DEEP.warps >= wide * d.warps);
  const int c = large ? deep : wide, warps = c * (large ? PG_DEEP : d).warps;
  if (c == 0 || a.max_kv > warps * RM_KEYS * PG_JOIN_UNITS) return {0, false};
  return {c, large};
}

template <int HD, int NT, bool WHOLE>
int paged_mma_launch(cudaStream_t st, const PagedArgs &a, float *scratch, DevStatus *status) {
  constexpr PgDepth D = PG_WIDE, E = PG_DEEP;
  constexpr int GROUP = RowsMma<HD, NT>::STAGE, SMEM = GROUP * D.warps * D.stages, DEEP = GROUP * E.warps * E.stages;
  const int group = a.n_heads / a.n_kv_heads, max_cts = (int)(((long long)a.max_q * group + NT * 8 - 1) / (NT * 8));
  const PgScratch c = pg_scratch(scratch, NT);
  const PgShape shape = paged_shape(a, max_cts);
  if (shape.cluster) {
    const dim3 grid((unsigned)(a.n_seqs * a.n_kv_heads * max_cts * shape.cluster));
    if (shape.deep) {
      constexpr auto kernel = paged_mma_kernel<HD, NT, WHOLE, true, E.warps, E.stages, E.ctas>;
      LAZY_TRY((co_allow_smem<kernel>(DEEP, false, true)));
      return co_launch(kernel, grid, dim3(E.warps * 32), DEEP, st, shape.cluster, false, a, group, max_cts, c, status);
    }
    constexpr auto kernel = paged_mma_kernel<HD, NT, WHOLE, true, D.warps, D.stages, D.ctas>;
    LAZY_TRY((co_allow_smem<kernel>(SMEM, false, true)));
    return co_launch(kernel, grid, dim3(D.warps * 32), SMEM, st, shape.cluster, false, a, group, max_cts, c, status);
  }
  constexpr auto kernel = paged_mma_kernel<HD, NT, WHOLE, false, D.warps, D.stages, D.ctas>;
  LAZY_TRY((co_allow_smem<kernel>(SMEM)));
  LAZY_TRY(co_launch(kernel, dim3(pg_grid()), dim3(D.warps * 32), SMEM, st, 1, false, a, group, 0, c, status));
  return co_launch(paged_mma_merge_kernel<HD, NT * 8>, dim3(pg_grid()), dim3(PG_MERGE_THREADS), 0, st, 1, true, a, group, c);
}

bool paged_mma_eligible(int dtype, int head_dim) { return dtype == LAZY_BF16 && head_dim <= 128; }

}  // namespace

// What the call needs: parts of keys that are not split go straight to the outputs.
size_t attention_paged_scratch_need(int dtype, int n_rows, int n_seqs, int max_q, int max_kv, int n_heads, int n_kv_heads, int head_dim) {
  max_q = min(max_q, n_rows);
  if (paged_mma_eligible(dtype, head_dim)) return pg_scratch_floats(pg_blocks((long long)max_q * (n_heads / n_kv_heads)), head_dim);
  const long long pairs = paged_wide_tiles(max_q, n_heads, n_kv_heads) * n_kv_heads * n_seqs;
  const int splits = paged_wide_splits(pairs, max_kv);
  return splits == 1 ? 0 : (size_t)pairs * splits * PW_COLS * (head_dim + 2);
}
// As much as that call or any smaller one needs, of either type.
size_t attention_paged_scratch_floats(int n_rows, int n_seqs, int max_q, int max_kv, int n_heads, int n_kv_heads, int head_dim) {
  max_q = min(max_q, n_rows);
  const long long pairs = paged_wide_tiles(max_q, n_heads, n_kv_heads) * n_kv_heads * n_seqs;
  const size_t wide = attn_split_parts(min(pairs, attn_split_most()), max_kv) * PW_COLS * (head_dim + 2);
  const size_t mma = head_dim <= 128 ? pg_scratch_floats(pg_blocks((long long)max_q * (n_heads / n_kv_heads)), head_dim) : 0;
  return wide > mma ? wide : mma;
}

template <int HD, bool WHOLE>
static int paged_mma(cudaStream_t st, const PagedArgs &a, float *scratch, DevStatus *status) {
  return pg_blocks((long long)a.max_q * (a.n_heads / a.n_kv_heads)) == 1 ? paged_mma_launch<HD, 1, WHOLE>(st, a, scratch, status)
                                                                        : paged_mma_launch<HD, 2, WHOLE>(st, a, scratch, status);
}

int launch_attention_paged(cudaStream_t st, int dtype, const PagedArgs &a, float *scratch, DevStatus *status) {
  if (a.n_rows == 0) return LAZY_OK;
  if (paged_mma_eligible(dtype, a.head_dim)) {
    const bool whole = a.kv.page_size % RM_KEYS == 0;
    return co_head_dim(a.head_dim, [&](auto hd) {
      return whole ? paged_mma<hd.value, true>(st, a, scratch, status) : paged_mma<hd.value, false>(st, a, scratch, status);
    });
  }
  if (dtype == LAZY_F32) return paged_f32(st, a, scratch, status);
  switch (a.head_dim) {
    case 160: return paged_wide<bf16, 5>(st, a, scratch, status);
    case 192: return paged_wide<bf16, 6>(st, a, scratch, status);
    case 224: return paged_wide<bf16, 7>(st, a, scratch, status);
    case 256: return paged_wide<bf16, 8>(st, a, scratch, status);
  }
  return LAZY_E_BADARG;
}

}  // namespace lazy
