// Kept tokens moved together in the cache, in place: token base + k becomes what token
// base + keep[k] was. keep[k] >= k, and both ascend, so no place that a token is
// written to is read by a later one: a (layer, request, head) goes through its list
// in order, a chunk of it read before any of it is written.
//
// K is a row of 256 bytes per token and head in either layout, V such a row in the
// token-major one and a column of 128 elements, a row apart each, in the other.
#include "tree_kernels.h"

namespace ema {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kChunk = 16;               // list entries

// Elements of a token's K and V of one head, from the block's first on.
struct Place {
  uint16_t* block;                       // nullptr: nothing to move
  int tok;
  int nhd;
};

__global__ __launch_bounds__(kThreads) void compact_kernel(CompactArgs a) {
  __shared__ Place s_src[kChunk], s_dst[kChunk];
  const int tid = threadIdx.x, b = blockIdx.x, l = blockIdx.y, h = blockIdx.z;
  const PoolView& pv = a.pools;
  const int BS = pv.block_size, H = pv.kv_heads;
  const int base = a.base[b], given = a.n_keep[b], n = max(0, min(given, a.cap));
  const bool counts = h == 0, first = counts && l == 0;
  if (first && tid == 0) {
    if (a.new_lens) a.new_lens[b] = base + n;
    const int bad = (base < 0) + (n != given);
    if (bad > 0) atomicAdd(a.err_count, bad);
  }
  if (base < 0) return;
  const int32_t* table = a.table + (int64_t(l) * a.batch + b) * a.max_blocks;
  const int64_t room = int64_t(a.max_blocks) << a.block_shift;
  const int n_total = pv.n_local + pv.n_slice;
  auto place = [&](int64_t t, Place& p) {
    const int id = table[t >> a.block_shift];
    p.tok = int(t) & (BS - 1);
    p.nhd = id >= pv.n_local ? pv.slice_layout : 0;
    if (id < 0 || id >= n_total) return false;
    p.block = reinterpret_cast<uint16_t*>(
        id < pv.n_local ? pv.local + int64_t(id) * pv.block_bytes
                        : pv.slice + int64_t(id - pv.n_local) * pv.block_bytes);
    return true;
  };
  const int64_t half = int64_t(BS) * H * 128;
  auto k_at = [&](const Place& p) { return p.block + (p.nhd ? int64_t(p.tok) * H + h : int64_t(h) * BS + p.tok) * 128; };
  auto v_at = [&](const Place& p, int ch) {
    return p.block + half + (p.nhd ? (int64_t(p.tok) * H + h) * 128 + ch
                                   : (int64_t(h) * 128 + ch) * BS + p.tok);
  };
  for (int k0 = 0; k0 < n; k0 += kChunk) {
    if (tid < kChunk) {
      const int k = k0 + tid;
      Place src{}, dst{};
      if (k < n) {
        const int32_t* list = a.keep + int64_t(b) * a.cap;
        const int from = list[k], before = k > 0 ? list[k - 1] : -1;
        const bool good = from >= k && from > before && int64_t(base) + from < room;
        if (!good && first) atomicAdd(a.err_count, 1);
        if (good && from != k && (!place(int64_t(base) + from, src) || !place(int64_t(base) + k, dst))) {
          src.block = nullptr;
          if (counts) atomicAdd(a.err_count, 1);
        }
      }
      s_src[tid] = src;
      s_dst[tid] = dst;
    }
    __syncthreads();
    u32x4 kx;
    uint16_t vx[kChunk / 2];
    const int e = tid >> 4, piece = tid & 15, ch = tid & 127, e0 = tid >> 7;
    if (s_src[e].block) kx = *reinterpret_cast<const u32x4*>(k_at(s_src[e]) + piece * 8);
#pragma unroll
    for (int i = 0; i < kChunk / 2; ++i)
      if (s_src[e0 + 2 * i].block) vx[i] = *v_at(s_src[e0 + 2 * i], ch);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // read before any wave writes
    __syncthreads();
    if (s_src[e].block) *reinterpret_cast<u32x4*>(k_at(s_dst[e]) + piece * 8) = kx;
#pragma unroll
    for (int i = 0; i < kChunk / 2; ++i)
      if (s_src[e0 + 2 * i].block) *v_at(s_dst[e0 + 2 * i], ch) = vx[i];
    __syncthreads();
  }
}

}  // namespace

hipError_t launch_kv_compact(const CompactArgs& a, hipStream_t stream) {
  if (a.batch <= 0) return hipSuccess;
  hipLaunchKernelGGL(compact_kernel, dim3(a.batch, a.layers, a.pools.kv_heads), dim3(kThreads), 0,
                     stream, a);
  return hipGetLastError();
}

}  // namespace ema
