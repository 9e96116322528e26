// Where a kept node's row comes from and goes to: plain arithmetic, so that a host compiler takes it too.
#pragma once

#ifdef __CUDACC__
#define JD_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define JD_HOST_DEVICE inline
#endif

namespace jd {

// Node number i of a path (`before`: the node in front of it, 0 for the first) of a sequence of `len` tokens that holds rows for `limit`:
// entries of its page table that its row is moved from and to. False where the path is cut. Every thread judges its own node,
// those behind a cut among them: its own number bounds the target's row by the source's, which `before` alone does only while all in
// front of it rise from 1.
JD_HOST_DEVICE bool path_entries(int len, int limit, int i, int node, int before, int max_nodes, int page_shift, int* from, int* to) {
  if (node <= before || node <= i || node >= max_nodes || len + node >= limit) return false;
  *from = (len + node) >> page_shift;
  *to = (len + 1 + i) >> page_shift;
  return true;
}

}  // namespace jd
