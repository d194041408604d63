// The end of a step with drafted tokens: which of them the model agrees with, and their rows of the response caches moved to
// where the next step expects them.
//
// From node 0, the last token that is certain, the walk goes to the child (the first, if several) that drafted what was sampled
// at the node, as long as there is one: a lane per node, one comparison and a ballot a step.  Node path[j] becomes row
// len + j of the cache.  path ascends and path[j] >= j, so whoever owns a column of the rows may move them one after the
// other (in batches, each read before it is written) and never overwrites a row that is still to be read.
// Bound by latency: a tree's three tables, the walk, the rows.  Every workgroup walks by itself: a second launch would cost more.
// Measured, us of the kernel: one prompt over 32 layers 3.3; 64 prompts of 8 KV heads over 32 layers 8.8 (30 MB to move: 5.8 at a copy's
// rate); 16 fp32 prompts over 8 layers 6.4.  The call takes 7.4 through the binding, so one prompt is bound by the host.
// Lengths in place: 2.0 / 2.9 / 2.6 more, the second launch.
#include <algorithm>

#include "sp_device.h"
#include "sp_internal.h"

namespace sp {

namespace {

constexpr int kAcceptThreads = 256;
constexpr int kMoveBatch = 8;          // rows in flight

struct Walk {
  int32_t path[kMaxNodes];
  int32_t n, next, len;
};

// by the first wave; kMaxNodes is its width
__device__ __forceinline__ void walk_tree(const AcceptArgs &a, int b, Walk &w) {
  static_assert(kMaxNodes == 64, "a lane per node");
  const int i = threadIdx.x, N = a.max_nodes;
  const int n = a.n_nodes ? min(max(a.n_nodes[b], 0), N) : N;
  const int len = (a.resp_len ? a.resp_len[b] : 0) + a.resp_len_add;
  // a node whose K and V found no place in the cache cannot be taken
  const bool there = i < n && len >= 0 && len + i < a.resp_capacity;
  const int64_t at = int64_t(b) * N + i;
  const int draft = there ? a.draft[at] : -1, sampled = there ? a.sampled[at] : -1;
  const int parent = there ? (a.parent ? a.parent[at] : i - 1) : -1;
  int cur = 0, count = 0, next = -1;
  uint64_t left = __ballot(there);
  if (left & 1) {
    while (true) {
      if (i == 0) w.path[count] = cur;
      ++count;
      next = __shfl(sampled, cur);
      const uint64_t child = __ballot(there && i > cur && parent == cur && draft == next && next >= 0);
      if (!child) break;
      cur = __builtin_ctzll(child);
    }
  }
  if (i == 0) { w.n = count; w.next = next; w.len = len; }
}

}  // namespace

// MOVE: blockIdx.x = prompt, y = part of its columns (16 bytes of a row of a layer's K or V).  Without it a workgroup per prompt writes
// the results alone: where resp_len_out is resp_len itself they come behind the moves of all workgroups, which read resp_len.
template <bool MOVE, bool RESULTS>
__global__ __launch_bounds__(kAcceptThreads) void accept_kernel(AcceptArgs a) {
  __shared__ Walk w;
  const int b = blockIdx.x;
  if (threadIdx.x < 64) walk_tree(a, b, w);
  __syncthreads();
  if (RESULTS && blockIdx.y == 0) {
    if (int(threadIdx.x) < a.max_nodes)
      a.path[int64_t(b) * a.max_nodes + threadIdx.x] = int(threadIdx.x) < w.n ? w.path[threadIdx.x] : -1;
    if (threadIdx.x == 0) {
      a.n_accepted[b] = w.n;
      a.next_token[b] = w.next;
      a.resp_len_out[b] = w.len + w.n;
    }
  }
  if (!MOVE) return;
  if (a.pos_resp && blockIdx.y == 0 && threadIdx.x < 64) {    // all positions are read before the first is written
    float *pos = a.pos_resp + int64_t(b) * a.resp_capacity + w.len;
    const bool mine = int(threadIdx.x) < w.n;
    const float x = mine ? pos[w.path[threadIdx.x]] : 0.f;
    if (mine) pos[threadIdx.x] = x;
  }
  int first = 0;                                              // rows that stay where they are
  while (first < w.n && w.path[first] == first) ++first;
  if (first == w.n) return;
  const int per_layer = a.row_bytes / 16;
  const int64_t columns = int64_t(2) * a.n_layers * per_layer, at = (int64_t(b) * a.resp_capacity + w.len) * a.row_bytes;
  for (int64_t c = int64_t(blockIdx.y) * kAcceptThreads + threadIdx.x; c < columns; c += int64_t(gridDim.y) * kAcceptThreads) {
    const int64_t block = c / per_layer;
    char *base = static_cast<char *>(block & 1 ? a.Vr : a.Kr) + (block >> 1) * a.layer_bytes + at + (c - block * per_layer) * 16;
    for (int j0 = first; j0 < w.n; j0 += kMoveBatch) {
      u32x4 v[kMoveBatch];
#pragma unroll
      for (int j = 0; j < kMoveBatch; ++j)
        if (j0 + j < w.n) v[j] = ld16(base + int64_t(w.path[j0 + j]) * a.row_bytes);
#pragma unroll
      for (int j = 0; j < kMoveBatch; ++j)
        if (j0 + j < w.n) st16(base + int64_t(j0 + j) * a.row_bytes, v[j]);
    }
  }
}

hipError_t launch_accept(const AcceptArgs &a, int32_t n_prompts, int n_cu, hipStream_t s) {
  // as many workgroups as are resident together (eight to a compute unit): each walks the tree for itself
  const int64_t columns = int64_t(2) * a.n_layers * (a.row_bytes / 16), most = (columns + kAcceptThreads - 1) / kAcceptThreads;
  const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(most, int64_t(8) * n_cu / n_prompts));
  const dim3 grid(unsigned(n_prompts), unsigned(std::min<int64_t>(parts, 65535))), block(kAcceptThreads);
  if (a.resp_len_out != a.resp_len) {
    hipLaunchKernelGGL((accept_kernel<true, true>), grid, block, 0, s, a);
  } else {
    hipLaunchKernelGGL((accept_kernel<true, false>), grid, block, 0, s, a);
    hipLaunchKernelGGL((accept_kernel<false, true>), dim3(unsigned(n_prompts)), block, 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace sp
