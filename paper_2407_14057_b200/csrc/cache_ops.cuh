// Pieces shared by the operators on bounded and shared caches: checks of device-side length tables, the
// order of accumulated weights, per-device kernel attributes, launch shapes with clusters.
#pragma once
#include <atomic>
#include <type_traits>

#include "common.cuh"

namespace lazy {

constexpr float CO_LOG2E = 1.4426950408889634f;

// Rows [start, start + n) of sequence s in a table of cumulative lengths.  A table that is not ascending, leaves
// [0, n_total] or holds a sequence longer than max_len is reported; the caller then skips the sequence.
__device__ __forceinline__ bool co_span(const int32_t *cu, int s, int n_total, int max_len, DevStatus *status,
                                        int where, int &start, int &n) {
  const int a = cu[s], b = cu[s + 1];
  start = a;
  n = b - a;
  const bool ok = a >= 0 && b >= a && b <= n_total && b - a <= max_len;
  if (!ok && threadIdx.x == 0) dev_fail(status, LAZY_E_BADARG, where, s, b);
  return ok;
}

// Unsigned key whose order is that of the weights: -0 counts as 0, NaN as less than everything.
__device__ __forceinline__ uint32_t co_weight_key(float w) {
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.f);  // -0 + 0 = +0
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// Opts a kernel in to `bytes` of dynamic shared memory, once per device (the attribute belongs to the device's
// context).  More than 64 devices simply set it again each time.
// `beside`: asks for the largest split of the SM's memory in favour of shared memory, so that a CTA of another kernel finds
// room beside this one's (both have to ask; it takes L1 from kernels that want it).  `large_clusters`: lets it run in clusters of
// more than eight.
template <auto Kernel>
inline int co_allow_smem(int bytes, bool beside = false, bool large_clusters = false) {
  static std::atomic<unsigned long long> done{0};
  int dev = 0;
  LAZY_CUDA_OK(cudaGetDevice(&dev));
  const unsigned long long bit = dev < 64 ? 1ull << dev : 0ull;
  if (done.load(std::memory_order_acquire) & bit) return LAZY_OK;
  LAZY_CUDA_OK(cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
  if (beside)
    LAZY_CUDA_OK(cudaFuncSetAttribute(Kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared));
  if (large_clusters) LAZY_CUDA_OK(cudaFuncSetAttribute(Kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1));
  done.fetch_or(bit, std::memory_order_release);
  return LAZY_OK;
}

// Calls f(std::integral_constant<int, HD>) for a head width of 32, 64, 96 or 128.
template <typename F>
inline int co_head_dim(int head_dim, F f) {
  switch (head_dim) {
    case 32: return f(std::integral_constant<int, 32>{});
    case 64: return f(std::integral_constant<int, 64>{});
    case 96: return f(std::integral_constant<int, 96>{});
    case 128: return f(std::integral_constant<int, 128>{});
  }
  return LAZY_E_BADARG;
}

// Launch with a cluster of `cluster` CTAs along x and, on request, as a programmatic dependent.
template <typename... KArgs, typename... Args>
inline int co_launch(void (*kfn)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, int cluster, bool pdl,
                     Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  int n = 0;
  if (cluster > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = cluster;
    attr[n].val.clusterDim.y = 1;
    attr[n].val.clusterDim.z = 1;
    ++n;
  }
  if (pdl) {
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n].val.programmaticStreamSerializationAllowed = 1;
    ++n;
  }
  cfg.attrs = attr;
  cfg.numAttrs = n;
  if (cudaLaunchKernelEx(&cfg, kfn, static_cast<KArgs>(args)...) != cudaSuccess) {
    cudaGetLastError();  // reported here and now: a later call must not find it
    return LAZY_E_CUDA;
  }
  LAZY_COUNT_LAUNCH();
  return LAZY_OK;
}

// CTAs that run at once in clusters of `size` (1, 2, 4, 8 or 16), up to three to an SM: a cluster stays within a group of SMs, and
// the groups are not multiples of it (as the occupancy calculator has it for 148 SMs and a kernel that fits one, two or
// three times on an SM).  An estimate for choosing a launch's shape: a launch of more runs its last clusters after the others.
inline int co_cluster_ctas(int size, int per_sm) {
  constexpr int TABLE[3][3] = {{132, 284, 416}, {120, 264, 384}, {112, 224, 336}};
  if (size <= 2) return sm_count() * per_sm;
  return sm_count() * TABLE[size == 4 ? 0 : (size == 8 ? 1 : 2)][per_sm - 1] / 148;
}

__device__ __forceinline__ uint32_t co_cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t co_cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
// All threads of all CTAs of the cluster; shared-memory writes before it are visible cluster-wide after it.
__device__ __forceinline__ void co_cluster_sync() {
  asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}
// The same in two steps, with work between them that needs no word from the others.
__device__ __forceinline__ void co_cluster_arrive() { asm volatile("barrier.cluster.arrive.aligned;" ::: "memory"); }
__device__ __forceinline__ void co_cluster_wait() { asm volatile("barrier.cluster.wait.aligned;" ::: "memory"); }
// Address of `p` (this CTA's shared memory) in CTA `rank` of the cluster.
template <typename T>
__device__ __forceinline__ T *co_map_shared(T *p, uint32_t rank) {
  uint64_t out;
  asm volatile("mapa.u64 %0, %1, %2;" : "=l"(out) : "l"((uint64_t)p), "r"(rank));
  return reinterpret_cast<T *>(out);
}

// Pitch and base of rows that are read in 16-byte pieces.
inline bool co_rows_ok(const void *p, long long ld, int dtype) {
  return !((uintptr_t)p & 15) && ld % (dtype == LAZY_F32 ? 4 : 8) == 0;
}

}  // namespace lazy
