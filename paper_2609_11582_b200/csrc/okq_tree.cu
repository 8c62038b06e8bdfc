// What the nodes of a drafted tree see (okq_tree_ancestors): from each node's parent the bits of its ancestors, and its depth.
//
// A block per sequence, its parents in shared memory; a thread per node walks to the root.  Parents come before their nodes, so the walk meets
// descending numbers and fills a row's words from the last to the first.  Bound by latency: a launch, one load, and a walk as long as the
// tree is deep.
#include "okq_paged.cuh"

namespace okq {

namespace {

constexpr int NT = 128, MOST = 4096;

__global__ void __launch_bounds__(NT) k_tree_ancestors(const PagedView c, const int32_t* parents, int n, const int32_t* q_len, unsigned long long* seen,
                                                        int32_t* depth) {
  __shared__ int parent[MOST];
  depend_wait();
  const int b = blockIdx.x, m = count_of(q_len, b, n), words = (n + 63) / 64;
  int bad = 0;
  for (int i = threadIdx.x; i < m; i += NT) {
    const int p = __ldcg(&parents[(size_t)b * n + i]);
    bad |= p < -1 || p >= i;
    parent[i] = p < i ? p : -1;
  }
  if (bad) set_status(c.status, OKQ_ERR_INVALID_ARG);
  __syncthreads();
  for (int i = threadIdx.x; i < m; i += NT) {
    unsigned long long* row = seen + ((size_t)b * n + i) * words;
    int at = i, steps = -1;
    for (int w = words - 1; w >= 0; w--) {
      unsigned long long bits = 0;
      for (; at >= 64 * w; at = parent[at]) {
        bits |= 1ull << (at & 63);
        steps++;
      }
      row[w] = bits;
    }
    if (depth) depth[(size_t)b * n + i] = steps;
  }
}

}  // namespace

}  // namespace okq

extern "C" okq_status okq_tree_ancestors(const okq_paged* cache, const int32_t* parents, int32_t n_new, const int32_t* q_len, uint64_t* seen,
                                         int32_t* depth, void* stream) {
  using namespace okq;
  const okq_status st = check_paged(cache, true);
  if (st != OKQ_OK) return st;
  if (n_new < 0 || (n_new > 0 && (!parents || !seen))) return OKQ_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(parents) & 3) || (reinterpret_cast<uintptr_t>(q_len) & 3) || (reinterpret_cast<uintptr_t>(depth) & 3) ||
      (reinterpret_cast<uintptr_t>(seen) & 7))
    return OKQ_ERR_ALIGNMENT;
  if (n_new > MOST) return OKQ_ERR_UNSUPPORTED;
  if (n_new == 0) return OKQ_OK;
  const cudaError_t e = launch_dependent(k_tree_ancestors, dim3(cache->batch), NT, 0, static_cast<cudaStream_t>(stream), 1, paged_view(cache), parents, n_new,
                                         q_len, reinterpret_cast<unsigned long long*>(seen), depth);
  if (e != cudaSuccess) {
    set_last_cuda_error((int)e);
    (void)cudaGetLastError();
    return OKQ_ERR_CUDA;
  }
  return launch_status();
}
