// New rows of a fused projection on their way into a paged cache: every head of q and k is normalised (where there are gains),
// rotated by the row's original position, and q goes to its own rows, k and v to the slot that the row takes in its
// sequence's pages.
//   y = x rsqrt(mean(x^2) + eps) g,   (y_i, y_{i + dh/2}) -> (y_i c_i - y_{i + dh/2} s_i, y_{i + dh/2} c_i + y_i s_i)
// Everything in fp32, rounded once when it is stored.
//
// A few lanes hold a head: lane i the 16-byte pieces i and i + half, so that a pair never leaves its lane, the mean is a
// reduction over those lanes, and a row's cosines and sines are loaded once for all its heads.  A warp takes a row, or a part of one
// where the rows are few.  Bound by memory, every element read and written once: 3376 rows of 32 heads (166 MB) 31 us, 5.4 TB/s, 9000 rows
// 79 (5.6).  Normalised heads: 9427 rows of 32 on 8 heads (232 MB) 52 us, without 43.  That is latency: 235 instructions to four heads of a
// warp, which 20 warps to an SM issue in 55 % of its cycles, with the memory at 45 % of its peak.  Of 9.4 cycles that a warp takes for
// one, 2.8 wait for loads, 2.3 for an arithmetic result, 1.3 for shuffles of the mean, 1.1 for their turn.
#include "paged.cuh"

namespace lazy {

namespace {

constexpr int PA_THREADS = 256, PA_WARPS = PA_THREADS / 32;
constexpr int PA_BATCH = 2;  // heads of a lane in flight; four at two CTAs to an SM: 32 and 54 us for the two above
constexpr int PA_CTAS = 3;   // to an SM

template <typename T>
__global__ void __launch_bounds__(PA_THREADS, PA_CTAS)
paged_append_kernel(const AppendArgs a, int lanes_log2, int parts, int steps, DevStatus *status) {
  constexpr int V = Elem<T>::kPerVec;
  const int lane = threadIdx.x & 31;
  const long long w = (long long)blockIdx.x * PA_WARPS + (threadIdx.x >> 5);
  const int r = (int)(w / parts), part = (int)(w - (long long)r * parts);
  if (r >= a.n_rows) return;
  const int half = a.head_dim >> 1, i0 = (lane & ((1 << lanes_log2) - 1)) * V;  // this lane's place in a head
  const bool on = i0 < half;
  const int per_step = 32 >> lanes_log2, sub = lane >> lanes_log2;
  const int heads = a.n_heads + 2 * a.n_kv_heads;
  const int h_end = min(heads, (part + 1) * steps * per_step);
  auto source = [&](int h) -> const T * {
    if (h < a.n_heads) return (const T *)a.q + (size_t)r * a.ldq + (size_t)h * a.head_dim;
    h -= a.n_heads;
    if (h < a.n_kv_heads) return (const T *)a.k + (size_t)r * a.ldkv + (size_t)h * a.head_dim;
    return (const T *)a.v + (size_t)r * a.ldkv + (size_t)(h - a.n_kv_heads) * a.head_dim;
  };
  Vec16<T> x[PA_BATCH], y[PA_BATCH];
  auto fetch = [&](int h0) {
#pragma unroll
    for (int u = 0; u < PA_BATCH; ++u) {
      const int h = h0 + u * per_step;
      if (h < h_end && on) {
        const T *p = source(h) + i0;
        x[u].load(p);
        y[u].load(p + half);
      }
    }
  };
  int h0 = part * steps * per_step + sub;
  fetch(h0);  // needs no table
  // ---- the row's place
  const int s = a.cu_q ? paged_find_seq(a.cu_q, a.n_seqs, r) : r;
  if (a.cu_q) paged_check_bounds(a.cu_q, a.n_seqs, a.n_rows, w * 32 + lane, (long long)a.n_rows * parts * 32, status);
  if (s < 0) return;
  const int p = a.pos[r];
  int start, rows, len;
  if (!paged_seq(a.kv, a.cu_q, s, a.n_rows, a.n_rows, a.max_len, lane == 0, status, start, rows, len) || rows == 0) return;
  if (r < start || r >= start + rows) {  // boundaries that do not ascend
    if (lane == 0) dev_fail(status, LAZY_E_BADARG, W_PAGED, s, r);
    return;
  }
  if (p < 0 || p >= a.max_pos) {
    if (lane == 0) dev_fail(status, LAZY_E_CAPACITY, W_ROPE_POS, r, p);
    return;
  }
  const int slot = len - rows + (r - start), nth = slot / a.kv.page_size, in_page = slot - nth * a.kv.page_size;
  const int page = a.kv.table[(size_t)s * a.kv.ld_table + nth];
  float2 cs[V];
  if (on) {
    const float4 *t = reinterpret_cast<const float4 *>(a.rope_table + (size_t)p * a.head_dim + 2 * i0);
#pragma unroll
    for (int j = 0; j < V / 2; ++j) {
      const float4 c = t[j];
      cs[2 * j] = make_float2(c.x, c.y);
      cs[2 * j + 1] = make_float2(c.z, c.w);
    }
  }
  const bool there = page >= 0 && page < a.kv.n_pages;
  if (!there && lane == 0) dev_fail(status, LAZY_E_BADARG, W_PAGED, s, page);
  const long long at = (long long)page * a.kv.page_stride + (long long)in_page * a.kv.slot_stride;
  const float inv_dh = 1.f / (float)a.head_dim;
  for (; h0 - sub < h_end; h0 += PA_BATCH * per_step) {
    if (h0 != part * steps * per_step + sub) fetch(h0);
#pragma unroll
    for (int u = 0; u < PA_BATCH; ++u) {
      const int h = h0 + u * per_step;
      if (h - sub >= h_end) break;  // the whole warp alike
      const bool is_q = h < a.n_heads, is_v = h >= a.n_heads + a.n_kv_heads, mine = on && h < h_end;
      float fx[V], fy[V];
      if (mine && !is_v) {
        x[u].unpack(fx);
        y[u].unpack(fy);
      }
      const T *gain = (const T *)(is_q ? a.g_q : a.g_k);
      if (a.g_q || a.g_k) {  // the whole warp alike: lanes of other heads take part in the shuffles
        float sum = 0.f;
        if (mine && !is_v) {
#pragma unroll
          for (int j = 0; j < V; ++j) sum = fmaf(fx[j], fx[j], fmaf(fy[j], fy[j], sum));
        }
        for (int o = 1 << lanes_log2 >> 1; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (mine && !is_v && gain) {
          const float f = rsqrtf(fmaf(sum, inv_dh, a.eps));
          Vec16<T> gx, gy;
          gx.load(gain + i0);
          gy.load(gain + half + i0);
          float ga[V], gb[V];
          gx.unpack(ga);
          gy.unpack(gb);
#pragma unroll
          for (int j = 0; j < V; ++j) {
            fx[j] *= f * ga[j];
            fy[j] *= f * gb[j];
          }
        }
      }
      if (!mine) continue;
      if (!is_v) {
        float ox[V], oy[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
          ox[j] = fx[j] * cs[j].x - fy[j] * cs[j].y;
          oy[j] = fy[j] * cs[j].x + fx[j] * cs[j].y;
        }
        x[u].pack(ox);
        y[u].pack(oy);
      }
      if (is_q) {
        T *o = (T *)a.q_out + (size_t)r * a.ldq_out + (size_t)h * a.head_dim + i0;
        x[u].store(o);
        y[u].store(o + half);
        continue;
      }
      const int g = h - a.n_heads - (is_v ? a.n_kv_heads : 0);
      if (!is_v && a.k_out) {
        T *o = (T *)a.k_out + (size_t)r * a.ldk_out + (size_t)g * a.head_dim + i0;
        x[u].store(o);
        y[u].store(o + half);
      }
      if (there) {
        T *o = (T *)(is_v ? a.kv.v : a.kv.k) + at + (long long)g * a.kv.head_stride + i0;
        x[u].store(o);
        y[u].store(o + half);
      }
    }
  }
}

}  // namespace

int launch_paged_append(cudaStream_t st, int dtype, const AppendArgs &a, DevStatus *status) {
  if (a.n_rows == 0) return LAZY_OK;
  const int pieces = a.head_dim / 2 / (dtype == LAZY_F32 ? 4 : 8);
  int lanes_log2 = 0;
  while ((1 << lanes_log2) < pieces) ++lanes_log2;
  const int all = cdiv(a.n_heads + 2 * a.n_kv_heads, 32 >> lanes_log2);  // steps of a row
  // a warp per row, several where the rows leave SMs without a warp's worth of loads
  int parts = cdiv(32 * sm_count(), a.n_rows);
  if (parts > all) parts = all;
  const int steps = cdiv(all, parts);
  parts = cdiv(all, steps);
  const long long warps = (long long)a.n_rows * parts, blocks = (warps + PA_WARPS - 1) / PA_WARPS;
  if (blocks > 0x7fffffffLL) return LAZY_E_CAPACITY;
  return co_launch(dtype == LAZY_F32 ? paged_append_kernel<float> : paged_append_kernel<bf16>, dim3((unsigned)blocks),
                   dim3(PA_THREADS), 0, st, 1, false, a, lanes_log2, parts, steps, status);
}

}  // namespace lazy
