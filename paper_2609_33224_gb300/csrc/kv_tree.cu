// Masks and positions of trees of drafted tokens, from their parents.
#include "kv_internal.cuh"

namespace pskv {
namespace {

// A CTA takes a tree, its parents in shared memory; a thread takes a node and walks up to the root.  Ancestors come in
// falling order, so that each word of the node's row is complete, and written, before the next one.  The walk ends, as
// every step goes to a smaller number.  Bound by latency: the load of the parents, a shared-memory load per step.  A tree
// of 24 nodes 2.0 us, 256 of 200 nodes 4.3.  The steps of a node are its depth: a chain of 64 nodes takes 7.6 us, 256 chains
// of 200 26, one of 300 39, of 1000 318, and of 8192, the longest there may be, 18 ms.
__global__ void __launch_bounds__(256) tree_kernel(const TreeArgs a) {
  extern __shared__ int32_t parent[];
  const uint32_t b = blockIdx.x;
  int64_t first = (int64_t)a.each * b, last = first + a.each;
  if (a.offsets) {
    first = a.offsets[b];
    last = a.offsets[b + 1];
  }
  if (first < 0 || last < first || last > (int64_t)a.nodes || last - first > (int64_t)a.words * 32) {
    if (threadIdx.x == 0) atomicOr_system(a.err, kErrTree);
    return;
  }
  const int32_t n = (int32_t)(last - first);
  for (int32_t i = threadIdx.x; i < n; i += blockDim.x) {
    int32_t p = a.parents[first + i];
    if (p >= i) {
      atomicOr_system(a.err, kErrTree);
      p = -1;
    }
    parent[i] = p;
  }
  __syncthreads();
  const int64_t start = a.start ? a.start[b] : 0;
  for (int32_t i = threadIdx.x; i < n; i += blockDim.x) {
    uint32_t* row = a.mask + (first + i) * a.stride;
    uint32_t word = a.words - 1, bits = 0;
    int64_t depth = -1;
    int32_t j = parent[i] < -1 ? -1 : i;
    for (; j >= 0; j = parent[j]) {
      const uint32_t w = (uint32_t)j / 32;
      while (word != w) {
        row[word--] = bits;
        bits = 0;
      }
      bits |= 1u << (j % 32);
      ++depth;
    }
    if (j < -1) atomicOr_system(a.err, kErrTree);  // an ancestor is no node
    for (;; bits = 0) {
      row[word] = bits;
      if (word-- == 0) break;
    }
    if (a.positions) a.positions[first + i] = start + (depth < 0 ? 0 : depth);
  }
}

}  // namespace

cudaError_t launch_tree(const TreeArgs& a, uint32_t trees, cudaStream_t s) {
  tree_kernel<<<trees, a.words * 32 < 256 ? a.words * 32 : 256, a.words * 32 * sizeof(int32_t), s>>>(a);
  return cudaGetLastError();
}

}  // namespace pskv
