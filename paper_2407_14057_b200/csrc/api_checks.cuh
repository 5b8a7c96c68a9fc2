// Argument checks shared by the entry points of the operators on bounded, shared and paged caches.
#pragma once
#include "cache_ops.cuh"

namespace lazy {

constexpr int MAX_GRID_YZ = 65535;

inline bool bad_dtype(int dtype) { return dtype != LAZY_BF16 && dtype != LAZY_F32; }

// Head layout shared by the calls; n_kv_heads = 0 stands for n_heads.
inline int check_heads(int n_heads, int &n_kv_heads, int head_dim) {
  if (n_kv_heads == 0) n_kv_heads = n_heads;
  if (n_heads < 1 || n_kv_heads < 1 || n_heads % n_kv_heads) return LAZY_E_BADARG;
  if (head_dim < 32 || head_dim > 256 || head_dim % 32) return LAZY_E_BADARG;
  if (n_heads > MAX_GRID_YZ) return LAZY_E_CAPACITY;
  return LAZY_OK;
}

inline bool bad_rows(const void *p, long long ld, long long width, int dtype) {
  return !p || ld < width || !co_rows_ok(p, ld, dtype);
}

}  // namespace lazy
