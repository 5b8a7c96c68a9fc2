// Caches in pages, shared by the operators that write and read them: where a sequence's rows, slots and pages are, and the
// checks of the device-side tables that say so.
#pragma once
#include "cache_ops.cuh"

namespace lazy {

// Sequence that row r belongs to: the last s with cu[s] <= r, found by the whole warp 32 boundaries at a time (two rounds of
// loads up to 1024 sequences).  -1: before the first sequence or behind the last, a row that belongs to none.
__device__ __forceinline__ int paged_find_seq(const int32_t *cu, int n_seqs, int r) {
  const int lane = threadIdx.x & 31;
  int lo = 0, n = n_seqs + 1;  // boundaries [lo, lo + n)
  while (true) {
    const int step = (n + 31) / 32, at = lane * step;
    const uint32_t under = __ballot_sync(0xffffffffu, at < n && cu[lo + min(at, n - 1)] <= r);
    if (!under) return -1;
    const int last = 31 - __clz(under);
    lo += last * step;
    n = min(step, n - last * step);
    if (step == 1) return lo < n_seqs ? lo : -1;
  }
}

// The rows and cached tokens of sequence s: rows [start, start + rows) of the batch (without cu: row s, none where len is 0), the
// last of its `len` tokens.  False, and reported, where the tables do not fit; true with rows = 0 where there is nothing to do.
__device__ __forceinline__ bool paged_seq(const PagedKV &kv, const int32_t *cu, int s, int n_rows, int max_rows, int max_len,
                                          bool report, DevStatus *status, int &start, int &rows, int &len) {
  bool ok = true;
  len = kv.len[s];
  start = s;
  rows = len != 0;
  if (cu) {
    start = cu[s];
    const int end = cu[s + 1];
    ok = start >= 0 && end >= start && end <= n_rows;
    rows = end - start;
    ok = ok && rows <= max_rows;
  }
  if (ok && rows > 0) ok = len >= rows && len <= max_len;
  if (!ok && report) dev_fail(status, LAZY_E_BADARG, W_PAGED, s, len);
  return ok;
}

// Reports boundaries that do not ascend or leave the rows, those that no row leads to among them: thread `id` of `n` takes every n-th.
__device__ __forceinline__ void paged_check_bounds(const int32_t *cu, int n_seqs, int n_rows, long long id, long long n, DevStatus *status) {
  for (long long s = id; s < n_seqs; s += n) {
    const int start = cu[s], end = cu[s + 1];
    if (start < 0 || end < start || end > n_rows) dev_fail(status, LAZY_E_BADARG, W_PAGED, (int)s, end);
  }
}

// Most tokens that a sequence's row of the table names.
inline int paged_capacity(const PagedKV &kv) {
  const long long n = (long long)kv.table_pages * kv.page_size;
  return n > 0x7fffff00LL ? 0x7fffff00 : (int)n;
}

}  // namespace lazy
