// The K and V of a chunk's tokens into their blocks.
//
// K rows are copied as they are, 16 bytes a lane. V rows become columns of the
// transposed V block: a workgroup takes a tile of tokens of one head, in LDS,
// and wherever eight consecutive tokens of the list fill eight consecutive,
// aligned rows of a block (all of a prompt but its ragged ends) writes them as one
// 16-byte piece per channel; other tokens are written element by element. A
// group of eight may straddle two tiles: the one it begins in reads on
// past its end for it, and the other leaves those tokens out, both by the same
// test of the slots alone.
//
// Bound by HBM: 8195 tokens of 8 heads, 67 MB, 13.6 us = 4.9 TB/s, what a plain copy of
// that size in one piece takes. Tiles of 64 tokens (K and V rows of a head, 36 KB in flight
// a workgroup): all loads of a tile are issued before the first store (a load and its store at a time: 15.8).
#include "op_kernels.h"

namespace ema {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;

template <int TILE>
__global__ __launch_bounds__(kThreads, 4) void kv_store_kernel(StoreArgs a) {
  constexpr int kRows = TILE + 7;                    // and what a group reads past the tile
  __shared__ int s_slot[7 + kRows];                  // tokens t0 - 7 .. t0 + TILE + 6
  __shared__ __attribute__((aligned(16))) uint16_t s_v[kRows][128];
  __shared__ int s_lead[TILE / 8 + 1], s_one[TILE], s_n[2];
  const int tid = threadIdx.x;
  const int t0 = blockIdx.x * TILE, h = blockIdx.y;
  const int BS = a.block_size, H = a.kv_heads;
  const int n = min(TILE, a.tokens - t0);
  for (int i = tid; i < 7 + kRows; i += kThreads) {
    const int t = t0 + i - 7;
    int s = t >= 0 && t < a.tokens ? a.slots[t] : -1;
    if (s < -1 || s >= a.n_slots) {
      if (h == 0 && t >= t0 && t < t0 + n) atomicAdd(a.err_count, 1);
      s = -1;
    }
    s_slot[i] = s;
  }
  if (tid < 2) s_n[tid] = 0;
  __syncthreads();
  if (tid < 64) {
    // group: tokens i .. i + 7 (from -7 on) hold rows 8r .. 8r + 7 of a block
    auto whole = [&](int i) {
      const int s = s_slot[i + 7];
      bool ok = s >= 0 && (s & 7) == 0;
#pragma unroll
      for (int k = 1; k < 8; ++k) ok = ok && s_slot[i + 7 + k] == s + k;
      return ok;
    };
    bool lead = false, one = false;
    if (tid < n) {
      const int s = s_slot[tid + 7];
      lead = s >= 0 && (s & 7) == 0 && whole(tid);
      one = s >= 0 && !whole(tid - (s & 7));
    }
    const unsigned long long ml = __ballot(lead), mo = __ballot(one);
    const unsigned long long below = (1ull << tid) - 1ull;
    if (lead) s_lead[__popcll(ml & below)] = tid;
    if (one) s_one[__popcll(mo & below)] = tid;
    if (tid == 0) {
      s_n[0] = __popcll(ml);
      s_n[1] = __popcll(mo);
    }
  }
  // K rows straight on, V rows into LDS: 16 threads to a row, all their loads at once
  const int piece = tid & 15;
  constexpr int kRounds = (kRows + kThreads / 16 - 1) / (kThreads / 16);
  u32x4 kx[kRounds], vx[kRounds];
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int i = (tid >> 4) + r * (kThreads / 16);
    if (i >= kRows || s_slot[min(i, kRows - 1) + 7] < 0) continue;
    const int64_t t = t0 + i;
    vx[r] = __builtin_nontemporal_load(
        reinterpret_cast<const u32x4*>(a.v + t * a.v_stride + h * 128 + piece * 8));
    if (i < n)
      kx[r] = __builtin_nontemporal_load(
          reinterpret_cast<const u32x4*>(a.k + t * a.k_stride + h * 128 + piece * 8));
  }
#pragma unroll
  for (int r = 0; r < kRounds; ++r) {
    const int i = (tid >> 4) + r * (kThreads / 16);
    if (i >= kRows) continue;
    const int s = s_slot[i + 7];
    if (s < 0) continue;
    *reinterpret_cast<u32x4*>(&s_v[i][piece * 8]) = vx[r];
    if (i >= n) continue;
    uint16_t* blk = reinterpret_cast<uint16_t*>(a.local + int64_t(s >> a.block_shift) * a.block_bytes);
    *reinterpret_cast<u32x4*>(blk + (int64_t(h) * BS + (s & (BS - 1))) * 128 + piece * 8) = kx[r];
  }
  __syncthreads();
  const int64_t v_half = int64_t(BS) * H * 128;
  // two groups side by side, whose pieces are often neighbours in a V row
  const int n_lead = s_n[0];
  for (int e = tid; e < (n_lead + 1) / 2 * 256; e += kThreads) {
    const int g = e / 256 * 2 + (e & 1), d = (e >> 1) & 127;
    if (g >= n_lead) continue;
    const int i = s_lead[g], s = s_slot[i + 7];
    uint16_t x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = s_v[i + k][d];
    uint16_t* blk = reinterpret_cast<uint16_t*>(a.local + int64_t(s >> a.block_shift) * a.block_bytes);
    *reinterpret_cast<u32x4*>(blk + v_half + (int64_t(h) * 128 + d) * BS + (s & (BS - 1))) =
        u32x4{x[0] | (uint32_t(x[1]) << 16), x[2] | (uint32_t(x[3]) << 16),
              x[4] | (uint32_t(x[5]) << 16), x[6] | (uint32_t(x[7]) << 16)};
  }
  for (int e = tid; e < s_n[1] * 128; e += kThreads) {
    const int i = s_one[e >> 7], d = e & 127, s = s_slot[i + 7];
    uint16_t* blk = reinterpret_cast<uint16_t*>(a.local + int64_t(s >> a.block_shift) * a.block_bytes);
    blk[v_half + (int64_t(h) * 128 + d) * BS + (s & (BS - 1))] = s_v[i][d];
  }
}

}  // namespace

hipError_t launch_kv_store(const StoreArgs& a, hipStream_t stream) {
  if (a.tokens <= 0) return hipSuccess;
  hipLaunchKernelGGL(kv_store_kernel<64>, dim3((a.tokens + 63) / 64, a.kv_heads), dim3(kThreads), 0,
                     stream, a);
  return hipGetLastError();
}

}  // namespace ema
