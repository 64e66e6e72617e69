// Masks and positions of drafted trees, and the path of a tree that the model's
// choices confirm: a workgroup to a request.
//
// The ancestors of a node are found in two steps. Within a block of 64 nodes, a lane
// each, by doubling: after r rounds a lane has the bits of its 2^r nearest ancestors of
// the block and the one above them. The block's highest ancestor hangs from a node of an
// earlier block, whose own bits of that block are complete: at most one step a block.
//
// Both are chains of loads: 2.2 us for one request, 3.6 for 200 trees of 65-250 nodes (1.3 MB); the
// rest of a call (7.7 us) is its launch and the binding.
#include "tree_kernels.h"

#include <algorithm>
#include <climits>

namespace ema {
namespace {

constexpr int kThreads = 256;
constexpr int kNodes = EMA_TREE_NODES;

// Rows of request b, clamped to what is there; 1 if the starts are out of range.
__device__ __forceinline__ int rows_of(const int32_t* starts, int tokens, int b, int& s, int& n) {
  const int from = starts[b], to = starts[b + 1];
  s = min(max(from, 0), tokens);
  n = max(0, min(max(to, 0), tokens) - s);
  return from < 0 || to < from || to > tokens || (b == 0 && from != 0);
}

__device__ __forceinline__ uint64_t shuffle64(uint64_t x, int lane) {
  return uint64_t(uint32_t(__shfl(int(uint32_t(x)), lane))) |
         uint64_t(uint32_t(__shfl(int(uint32_t(x >> 32)), lane))) << 32;
}

__global__ __launch_bounds__(kThreads) void tree_tables_kernel(TreeTablesArgs a) {
  __shared__ uint64_t s_own[kNodes];       // the node's ancestors (and itself) in its block
  __shared__ int s_above[kNodes];          // the parent of the first of them, -1: a root
  const int tid = threadIdx.x, lane = tid & 63, b = blockIdx.x;
  int s, n;
  const int wrong = rows_of(a.starts, a.tokens, b, s, n);
  const int given = a.seq_lens[b], base = max(given, INT_MIN + n) - n;
  const int known = min(n, 64 * a.words);
  if (tid == 0) {
    if (a.base) a.base[b] = base;
    const int bad = wrong + (given < n) + (known < n);
    if (bad > 0) atomicAdd(a.err_count, bad);
  }
  for (int i0 = 0; i0 < known; i0 += kThreads) {
    const int i = i0 + tid, first = i - lane;
    if (first >= known) continue;          // a whole wave
    int p = -1;
    bool bad = false;
    if (i < known) {
      p = a.parents[s + i];
      bad = p < -1 || p >= i;
      if (bad) p = -1;
    }
    const unsigned long long m = __ballot(bad);
    if (m != 0 && lane == 0) atomicAdd(a.err_count, __popcll(m));
    uint64_t own = 1ull << lane;
    int up = p >= first ? p - first : -1;  // its lane
    while (__ballot(up >= 0) != 0) {
      const int from = max(up, 0);
      const uint64_t more = shuffle64(own, from);
      const int next = __shfl(up, from);
      if (up >= 0) {
        own |= more;
        up = next;
      }
    }
    const int above = __shfl(p, int(__builtin_ctzll(own)));
    if (i < known) {
      s_own[i] = own;
      s_above[i] = above;
    }
  }
  __syncthreads();
  for (int i = tid; i < n; i += kThreads) {
    uint64_t* const out = a.mask + int64_t(s + i) * a.words;
    int depth = 1, at = i < known ? i : -1;
    for (int w = a.words - 1; w >= 0; --w) {
      uint64_t x = 0;
      if (at >= 0 && at >> 6 == w) {
        x = s_own[at];
        at = s_above[at];
        depth += __popcll(x);
      }
      out[w] = x;
    }
    if (a.positions) a.positions[s + i] = base + (i < known ? depth - 2 : 0);
  }
}

__global__ __launch_bounds__(kThreads) void tree_accept_kernel(TreeAcceptArgs a) {
  __shared__ int s_next[kNodes + 1];       // after node i - 1: its lowest child that is confirmed
  __shared__ int s_n;
  const int tid = threadIdx.x, b = blockIdx.x;
  int s, n;
  const int wrong = rows_of(a.starts, a.tokens, b, s, n);
  const int known = min(n, kNodes);
  if (tid == 0) {
    const int bad = wrong + (known < n);
    if (bad > 0) atomicAdd(a.err_count, bad);
  }
  for (int i = tid; i <= known; i += kThreads) s_next[i] = INT_MAX;
  __syncthreads();
  const bool rooted = a.root_choice == nullptr;
  const int root = rooted ? -1 : a.root_choice[b];
  for (int i = tid; i < known; i += kThreads) {
    const int p = a.parents[s + i], token = a.drafted[s + i];
    const bool bad = p < -1 || p >= i;
    if (bad) atomicAdd(a.err_count, 1);
    if (rooted && i == 0) s_next[0] = 0;
    else if (!bad && !(rooted && p < 0) && token == (p < 0 ? root : a.choice[s + p]))
      atomicMin(&s_next[p + 1], i);
  }
  __syncthreads();
  if (tid == 0) {
    int k = 0, last = -1;
    for (int at = s_next[0]; at != INT_MAX && k < a.cap; at = s_next[at + 1]) {
      a.path[int64_t(b) * a.cap + k++] = at;
      last = at;
    }
    a.n_path[b] = k;
    a.next[b] = last >= 0 ? a.choice[s + last] : root;
    s_n = k;
  }
  __syncthreads();
  for (int k = s_n + tid; k < a.cap; k += kThreads) a.path[int64_t(b) * a.cap + k] = -1;
}

}  // namespace

hipError_t launch_tree_tables(const TreeTablesArgs& a, hipStream_t stream) {
  if (a.batch <= 0) return hipSuccess;
  hipLaunchKernelGGL(tree_tables_kernel, dim3(a.batch), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_tree_accept(const TreeAcceptArgs& a, hipStream_t stream) {
  if (a.batch <= 0) return hipSuccess;
  hipLaunchKernelGGL(tree_accept_kernel, dim3(a.batch), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace ema
