// Attention of a few query rows over keys that lie anywhere in memory, one warp at a time: the inner loop shared by
// the step on bounded caches, the requests' own keys behind a shared prefix, and new rows over paged caches.
//
// A warp takes 16 keys at a time and up to 8 NT columns, a column being one (query row, head) that reads the same
// key/value head.  Keys are the M side of both products, so few columns waste nothing of the instruction:
//   S^T [16 keys x 8] = K [16 x HD] Q^T,   O^T [HD x 8] += V^T [HD x 16] P^T       (m16n8k16, bf16, fp32 accumulators)
// The accumulator of S^T holds P with keys along the rows; one 8 x 8 transpose per half turns it into the second
// product's operand without shared memory.  P enters as the sum of two bf16 numbers (see WEIGHT_REST), so that the only
// rounding of an output that counts is its own: the step is bound by reading K and V, and the second product's extra
// instructions (24 instead of 16 per 16 keys of a head width of 128, about 3 clocks per key of an SM against 22 that
// the key's 512 bytes take) cost no time.  This is the warp-level tensor path, not tcgen05: with at most 16 columns the step is bound by
// reading the keys, which a warp alone does without a wait for others, whereas a 128-row instruction wants 128 keys brought
// together by a CTA, a tile's P back through shared or tensor memory, and barriers between.  Keys named by lists cannot come through
// tensor maps either way.  With many columns (drafts, chunks of a prompt) the products bound the step, and that reason ends.
//
// Every warp owns its shared memory stages (cp.async, 16 bytes a lane, rows that do not exist read as zeros), so the
// loop has no barrier wider than the warp.
#pragma once
#include "attn_common.cuh"
#include "cache_ops.cuh"

namespace lazy {

constexpr int RM_KEYS = 16;  // keys per stage

__device__ __forceinline__ void rm_cp_async16(uint32_t dst, const void *src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void rm_cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void rm_cp_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void rm_ldmatrix(uint32_t addr, uint32_t *r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void rm_ldmatrix_trans(uint32_t addr, uint32_t *r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ uint32_t rm_transpose(uint32_t a) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
__device__ __forceinline__ void rm_mma(float *c, const uint32_t *a, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// 16-byte piece c of row r of a stage's half (K, then V).  Rows lie 128 or 256 bytes apart: the swizzle moves a piece by up
// to eight places, which a head width of 32 or 96 has no room for by itself.
template <int HD>
constexpr int rows_pitch = HD <= 64 ? 128 : 256;
template <int HD>
__device__ __forceinline__ uint32_t rows_at(int r, int c) {
  return (uint32_t)(r * rows_pitch<HD> + ((c ^ (r & 7)) << 4));
}
// Requests one stage: rows(r) gives (K row, V row, exists) of key r; call with the whole warp, then rm_cp_commit().
template <int HD, typename Rows>
__device__ __forceinline__ void rows_load(uint32_t stage, Rows rows) {
  const int lane = threadIdx.x & 31;
  constexpr int CHUNKS = HD / 8;
#pragma unroll
  for (int i = 0; i < RM_KEYS * CHUNKS / 32; ++i) {
    const int r = (i * 32 + lane) / CHUNKS, c = (i * 32 + lane) % CHUNKS;
    const bf16 *kr, *vr;
    const bool there = rows(r, kr, vr);
    rm_cp_async16(stage + rows_at<HD>(r, c), kr + c * 8, there);
    rm_cp_async16(stage + RM_KEYS * rows_pitch<HD> + rows_at<HD>(r, c), vr + c * 8, there);
  }
}

// The same for 16 rows that lie `stride` elements apart from kr / vr on, all of them there: fewer instructions to an address.  `mine` is
// rows_mine(stride), this lane's place in the first of them.
template <int HD>
__device__ __forceinline__ long long rows_mine(long long stride) {
  const int lane = threadIdx.x & 31;
  constexpr int CHUNKS = HD / 8;
  return 32 % CHUNKS == 0 ? (lane / CHUNKS) * stride + lane % CHUNKS * 8 : 0;
}
template <int HD>
__device__ __forceinline__ void rows_load_run(uint32_t stage, const bf16 *kr, const bf16 *vr, long long stride, long long mine) {
  constexpr int CHUNKS = HD / 8;
  if constexpr (32 % CHUNKS == 0) {  // a lane stays in its column, rows advance by 32 / CHUNKS
    constexpr int STEP = 32 / CHUNKS;
    const int lane = threadIdx.x & 31, r0 = lane / CHUNKS, c = lane % CHUNKS;
    kr += mine;
    vr += mine;
#pragma unroll
    for (int i = 0; i < RM_KEYS / STEP; ++i) {
      const uint32_t to = stage + rows_at<HD>(r0 + i * STEP, c);
      rm_cp_async16(to, kr, true);
      rm_cp_async16(to + RM_KEYS * rows_pitch<HD>, vr, true);
      kr += STEP * stride;
      vr += STEP * stride;
    }
  } else {
    rows_load<HD>(stage, [&](int r, const bf16 *&k, const bf16 *&v) {
      k = kr + r * stride;
      v = vr + r * stride;
      return true;
    });
  }
}

constexpr float RM_SLACK = 8.f;

template <int HD, int NT>
struct RowsMma {
  static constexpr int CHUNKS = HD / 8;              // 16-byte pieces per row
  static constexpr int HALF = RM_KEYS * rows_pitch<HD>;  // bytes of a stage's K (or V)
  static constexpr int STAGE = 2 * HALF;
  uint32_t qf[NT][HD / 16][2];
  float m[NT][2], l[NT][2];   // of columns (lane % 4) * 2 + {0, 1} of each block of 8; l is this lane's keys' only
  float o[NT][HD / 16][4];    // times WEIGHT_LIFT

  __device__ static __forceinline__ uint32_t at(int r, int c) { return rows_at<HD>(r, c); }

  // q_of(column): the column's query, or NULL for a column that is not used (reads as zeros)
  template <typename QOf>
  __device__ __forceinline__ void init(QOf q_of) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const bf16 *q = q_of(t * 8 + (lane >> 2));
#pragma unroll
      for (int k = 0; k < HD / 16; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          qf[t][k][h] = q ? *reinterpret_cast<const uint32_t *>(q + k * 16 + h * 8 + (lane & 3) * 2) : 0u;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        m[t][i] = -INFINITY;
        l[t][i] = 0.f;
      }
#pragma unroll
      for (int k = 0; k < HD / 16; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[t][k][i] = 0.f;
    }
  }

  // One stage of keys.  Key r of the stage is seen by this lane's column i of block t iff r < vis[t][i] and bit r of
  // `there` is set.  logits(t, r, x0, x1): the two columns' logits (log2 units) of key r, as they are before the mask.
  // CUT: columns may differ in what they see.  A value row that some column does not see must then not reach it even as
  // 0 x inf or 0 x NaN, so rows with such values (bits of `wild`) are taken out of the product and added one by one
  // to the columns that see them.
  template <bool CUT, typename Logits>
  __device__ __forceinline__ void process(uint32_t stage, const int (&vis)[NT][2], uint32_t there, Logits logits) {
    const int lane = threadIdx.x & 31, kr = lane >> 2;
    const float sl2 = rsqrtf((float)HD) * CO_LOG2E;
    float s[NT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[t][i] = 0.f;
#pragma unroll
    for (int k = 0; k < HD / 16; ++k) {
      uint32_t a[4];  // keys 0-7 | 8-15 of columns k * 16 .. + 7, then of the next eight
      rm_ldmatrix(stage + at(lane & 15, k * 2 + (lane >> 4)), a);
#pragma unroll
      for (int t = 0; t < NT; ++t) rm_mma(s[t], a, qf[t][k][0], qf[t][k][1]);
    }
    const uint32_t wild = CUT ? take_out_wild(stage) : 0u;
    uint32_t hi[NT][2], lo[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[t][i] *= sl2;
      logits(t, kr, s[t][0], s[t][1]);
      logits(t, kr + 8, s[t][2], s[t][3]);
      float alpha[2], p[4];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (kr >= vis[t][i] || !(there >> kr & 1u)) s[t][i] = -INFINITY;
        if (kr + 8 >= vis[t][i] || !(there >> (kr + 8) & 1u)) s[t][2 + i] = -INFINITY;
        float mx = fmaxf(s[t][i], s[t][2 + i]);
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
        mx = fmaxf(mx, m[t][i]);
        const float ref = mx == -INFINITY ? 0.f : mx;  // nothing seen so far: every weight is 2^-inf = 0
        alpha[i] = ex2_approx(m[t][i] - ref);
        m[t][i] = mx;
        p[i] = ex2_approx(s[t][i] - ref);
        p[2 + i] = ex2_approx(s[t][2 + i] - ref);
        l[t][i] = l[t][i] * alpha[i] + (p[i] + p[2 + i]);
      }
      if (__any_sync(0xffffffffu, alpha[0] != 1.f || alpha[1] != 1.f)) {
#pragma unroll
        for (int k = 0; k < HD / 16; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[t][k][i] *= alpha[i & 1];
      }
      if (CUT && wild) add_wild(stage, wild, t, vis[t], there, p);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t h = bf16x2_pack_rz(p[2 * i], p[2 * i + 1]);
        float h0, h1;
        bf16x2_unpack(h, h0, h1);
        hi[t][i] = rm_transpose(h);
        lo[t][i] = rm_transpose(bf16x2_pack(fmaf(h0, -WEIGHT_REST, p[2 * i]), fmaf(h1, -WEIGHT_REST, p[2 * i + 1])));
      }
    }
#pragma unroll
    for (int k = 0; k < HD / 16; ++k) {
      uint32_t a[4];  // head columns 0-7 | 8-15 of keys 0-7, then of keys 8-15
      rm_ldmatrix_trans(stage + HALF + at((lane & 7) + ((lane >> 4) << 3), k * 2 + ((lane >> 3) & 1)), a);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        rm_mma(o[t][k], a, hi[t][0], hi[t][1]);
        rm_mma(o[t][k], a, lo[t][0], lo[t][1]);
      }
    }
  }

  // The same without logits for the caller, with less between its products: a column's reference m is raised only when a logit exceeds it
  // by more than RM_SLACK (weights are then up to 2^RM_SLACK), so that most groups need neither their maximum nor a pass over the
  // outputs, and products that depend on one another have others between them.  ALL: every column sees all 16 keys.
  template <bool CUT, bool ALL>
  __device__ __forceinline__ void step(uint32_t stage, const int (&vis)[NT][2], uint32_t there) {
    const int lane = threadIdx.x & 31, kr = lane >> 2;
    const float sl2 = rsqrtf((float)HD) * CO_LOG2E;
    constexpr int CHAINS = NT == 1 ? 2 : 1;  // sums over the head that run side by side
    float s[NT][4], x[CHAINS][NT][4];
#pragma unroll
    for (int c = 0; c < CHAINS; ++c)
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[c][t][i] = 0.f;
#pragma unroll
    for (int k = 0; k < HD / 16; ++k) {
      uint32_t a[4];  // keys 0-7 | 8-15 of columns k * 16 .. + 7, then of the next eight
      rm_ldmatrix(stage + at(lane & 15, k * 2 + (lane >> 4)), a);
#pragma unroll
      for (int t = 0; t < NT; ++t) rm_mma(x[k % CHAINS][t], a, qf[t][k][0], qf[t][k][1]);
    }
    const uint32_t wild = CUT ? take_out_wild(stage) : 0u;
    bool grown = false;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[t][i] = (CHAINS == 2 ? x[0][t][i] + x[CHAINS - 1][t][i] : x[0][t][i]) * sl2;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (!ALL) {
          if (kr >= vis[t][i] || !(there >> kr & 1u)) s[t][i] = -INFINITY;
          if (kr + 8 >= vis[t][i] || !(there >> (kr + 8) & 1u)) s[t][2 + i] = -INFINITY;
        }
        grown |= fmaxf(s[t][i], s[t][2 + i]) > m[t][i] + RM_SLACK;
      }
    }
    if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          float mx = fmaxf(s[t][i], s[t][2 + i]);
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
          mx = fmaxf(mx, m[t][i]);
          const float alpha = ex2_approx(m[t][i] - (mx == -INFINITY ? 0.f : mx));
          m[t][i] = mx;
          l[t][i] *= alpha;
#pragma unroll
          for (int k = 0; k < HD / 16; ++k) {
            o[t][k][i] *= alpha;
            o[t][k][2 + i] *= alpha;
          }
        }
    }
    uint32_t hi[NT][2], lo[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float p[4];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float ref = m[t][i] == -INFINITY ? 0.f : m[t][i];  // nothing seen so far: every weight is 2^-inf = 0
        p[i] = ex2_approx(s[t][i] - ref);
        p[2 + i] = ex2_approx(s[t][2 + i] - ref);
        l[t][i] += p[i] + p[2 + i];
      }
      if (CUT && wild) add_wild(stage, wild, t, vis[t], there, p);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t h = bf16x2_pack_rz(p[2 * i], p[2 * i + 1]);
        float h0, h1;
        bf16x2_unpack(h, h0, h1);
        hi[t][i] = rm_transpose(h);
        lo[t][i] = rm_transpose(bf16x2_pack(fmaf(h0, -WEIGHT_REST, p[2 * i]), fmaf(h1, -WEIGHT_REST, p[2 * i + 1])));
      }
    }
    constexpr int BATCH = HD % 64 == 0 ? 4 : 2;  // pieces of the head at a time
#pragma unroll
    for (int k0 = 0; k0 < HD / 16; k0 += BATCH) {
      uint32_t a[BATCH][4];  // head columns 0-7 | 8-15 of keys 0-7, then of keys 8-15
#pragma unroll
      for (int b = 0; b < BATCH; ++b)
        rm_ldmatrix_trans(stage + HALF + at((lane & 7) + ((lane >> 4) << 3), (k0 + b) * 2 + ((lane >> 3) & 1)), a[b]);
#pragma unroll
      for (int b = 0; b < BATCH; ++b)
#pragma unroll
        for (int t = 0; t < NT; ++t) rm_mma(o[t][k0 + b], a[b], hi[t][0], hi[t][1]);
#pragma unroll
      for (int b = 0; b < BATCH; ++b)
#pragma unroll
        for (int t = 0; t < NT; ++t) rm_mma(o[t][k0 + b], a[b], lo[t][0], lo[t][1]);
    }
  }

  // Value rows of the stage that hold an infinity or a NaN, as a bit per key; they are copied over the stage's K rows
  // (which have been used) and replaced by zeros.
  __device__ __forceinline__ uint32_t take_out_wild(uint32_t stage) const {
    const int lane = threadIdx.x & 31;
    constexpr int PER = 32 / CHUNKS;
    uint32_t wild = 0u;
#pragma unroll
    for (int i = 0; i < RM_KEYS / PER; ++i) {
      const int k0 = lane / CHUNKS, r = i * PER + min(k0, PER - 1), c = lane % CHUNKS;  // head width 96: eight lanes are left over
      const uint32_t addr = stage + HALF + at(r, c);
      uint32_t x[4];
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(addr) : "memory");
      bool bad = false;
#pragma unroll
      for (int k = 0; k < 4; ++k) bad |= (x[k] & 0x7f80u) == 0x7f80u || (x[k] & 0x7f800000u) == 0x7f800000u;
      const uint32_t lanes = __ballot_sync(0xffffffffu, bad);
#pragma unroll
      for (int k = 0; k < PER; ++k)
        if (lanes >> (k * CHUNKS) & ((1u << CHUNKS) - 1u)) {
          wild |= 1u << (i * PER + k);
          if (k0 == k) {
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(stage + at(r, c)), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]) : "memory");
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(addr), "r"(0u) : "memory");
          }
        }
    }
    __syncwarp();
    return wild;
  }
  // o += p v for the value rows that were taken out, in the columns that see them.
  __device__ __forceinline__ void add_wild(uint32_t stage, uint32_t wild, int t, const int (&vis)[2], uint32_t there,
                                           const float (&p)[4]) {
    const int lane = threadIdx.x & 31;
    for (int r = 0; r < RM_KEYS; ++r) {
      if (!(wild >> r & 1u)) continue;
      const int from = (r & 7) * 4 + (lane & 3);
      const float p0 = __shfl_sync(0xffffffffu, r < 8 ? p[0] : p[2], from) * WEIGHT_LIFT;
      const float p1 = __shfl_sync(0xffffffffu, r < 8 ? p[1] : p[3], from) * WEIGHT_LIFT;
#pragma unroll
      for (int k = 0; k < HD / 16; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int d = k * 16 + h * 8 + (lane >> 2);
          uint16_t u;
          asm volatile("ld.shared.u16 %0, [%1];" : "=h"(u) : "r"(stage + at(r, d >> 3) + (d & 7) * 2) : "memory");
          const float v = __uint_as_float((uint32_t)u << 16);
          if ((there >> r & 1u) && r < vis[0]) o[t][k][2 * h] += p0 * v;
          if ((there >> r & 1u) && r < vis[1]) o[t][k][2 * h + 1] += p1 * v;
        }
    }
  }

  // Sums l over the warp's keys; afterwards every lane of a column pair holds it.
  __device__ __forceinline__ void finish() {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        l[t][i] += __shfl_xor_sync(0xffffffffu, l[t][i], 4);
        l[t][i] += __shfl_xor_sync(0xffffffffu, l[t][i], 8);
        l[t][i] += __shfl_xor_sync(0xffffffffu, l[t][i], 16);
      }
  }
};

}  // namespace lazy
