// Attention of prompt chunks and differential attention over the paged cache:
// one wavefront per query row and output head, tokens over the lanes for the
// scores, channels over the lanes for the output, in 32 bits throughout.
#include "op_kernels.h"
#include "attn_store.h"

namespace ema {
namespace {

__device__ __forceinline__ float to_f32(uint16_t x, int bf16) {
  return bf16 ? __builtin_bit_cast(float, uint32_t(x) << 16)
              : float(__builtin_bit_cast(_Float16, x));
}

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
  return x;
}
__device__ __forceinline__ float wave_add(float x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
  return x;
}

// MAPS 1: plain attention of 128 channels; 2: differential attention of 256.
template <int MAPS>
__global__ __launch_bounds__(64) void attend_rows(PromptArgs a) {
  constexpr int D = 128, kCh = 2 * MAPS;               // channels of a lane
  __shared__ float s_q[MAPS][D], s_p[MAPS][64];
  const int lane = threadIdx.x, row = blockIdx.x, head = blockIdx.y;
  int b = row, i = 0, n = 1;
  if (a.starts) {
    if (row < a.starts[0] || row >= a.starts[a.batch]) return;
    int lo = 0, hi = a.batch;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (a.starts[mid] <= row) lo = mid; else hi = mid;
    }
    b = lo;
    i = row - a.starts[b];
    n = a.starts[b + 1] - a.starts[b];
  }
  const int BS = a.block_size, H = a.kv_heads, G = a.q_heads / H;
  const int raw = a.seq_lens[b];
  const int len = max(0, min(raw, a.max_blocks * BS));
  if (lane == 0 && head == 0 && ((len != raw && i == 0) || (a.starts && len - n + i < 0)))
    atomicAdd(a.err_count, 1);
  const int seen = a.starts ? len - n + i + 1 : len;   // tokens the row attends
  const int kvh = head / G * MAPS;                     // the (first) KV head
  for (int e = lane; e < MAPS * D; e += 64) {
    const uint16_t* q = reinterpret_cast<const uint16_t*>(a.q) + int64_t(row) * a.q_stride;
    s_q[e / D][e % D] = to_f32(q[head * MAPS * D + e], a.dtype);
  }
  __syncthreads();
  float m[MAPS], l[MAPS], o[MAPS][kCh];
#pragma unroll
  for (int x = 0; x < MAPS; ++x) {
    m[x] = -INFINITY;
    l[x] = 0.0f;
#pragma unroll
    for (int c = 0; c < kCh; ++c) o[x][c] = 0.0f;
  }
  const int64_t half = int64_t(BS) * H * D;
  for (int t0 = 0; t0 < seen; t0 += 64) {
    const int t = t0 + lane;
    int id = -1;
    if (t < seen) {
      id = a.table[int64_t(b) * a.max_blocks + t / BS];
      if (id < 0 || id >= a.n_local) {
        if (t % BS == 0 && head == 0) atomicAdd(a.err_count, 1);
        id = -1;
      }
    }
    const uint16_t* blk = reinterpret_cast<const uint16_t*>(a.local + int64_t(max(id, 0)) * a.block_bytes);
#pragma unroll
    for (int x = 0; x < MAPS; ++x) {
      float s = -INFINITY;
      if (id >= 0) {
        s = 0.0f;
        const uint16_t* k = blk + (int64_t(kvh + x) * BS + t % BS) * D;
        for (int d = 0; d < D; ++d) s = fmaf(to_f32(k[d], a.dtype), s_q[x][d], s);
        s *= a.scale_log2;
      }
      const float mx = fmaxf(m[x], wave_max(s));
      const float at = mx == -INFINITY ? 0.0f : mx;      // NaN scores stay NaN
      const float f = exp2f(m[x] - at);
      const float p = exp2f(s - at);
      m[x] = mx;
      l[x] = l[x] * f + wave_add(p);
#pragma unroll
      for (int c = 0; c < kCh; ++c) o[x][c] *= f;
      s_p[x][lane] = p;
    }
    __syncthreads();
    for (int k = 0; k < 64; ++k) {
      const int kid = __shfl(id, k);
      if (kid < 0) continue;
      const uint16_t* kb = reinterpret_cast<const uint16_t*>(a.local + int64_t(kid) * a.block_bytes) + half;
#pragma unroll
      for (int c = 0; c < kCh; ++c) {
        const float v = to_f32(kb[(int64_t(kvh) * D + c * 64 + lane) * BS + (t0 + k) % BS], a.dtype);
#pragma unroll
        for (int x = 0; x < MAPS; ++x) o[x][c] = fmaf(s_p[x][k], v, o[x][c]);
      }
    }
    __syncthreads();
  }
  AttnArgs st;
  st.out = a.out;
  st.out_dtype = a.out_dtype;
  float r[kCh], sq = 0.0f;
#pragma unroll
  for (int c = 0; c < kCh; ++c) {
    r[c] = l[0] == 0.0f ? 0.0f : o[0][c] / l[0];
    if constexpr (MAPS == 2) r[c] -= l[1] == 0.0f ? 0.0f : a.lam[head] * (o[1][c] / l[1]);
    sq = fmaf(r[c], r[c], sq);
  }
  if (MAPS == 2 && a.norm_weight) {
    const float inv = 1.0f / sqrtf(wave_add(sq) / float(MAPS * D) + a.norm_eps);
#pragma unroll
    for (int c = 0; c < kCh; ++c) r[c] *= inv * a.norm_weight[c * 64 + lane];
  }
#pragma unroll
  for (int c = 0; c < kCh; ++c)
    store_out(st, (int64_t(row) * (a.q_heads / MAPS) + head) * MAPS * D + c * 64 + lane, r[c]);
}

template <int MAPS>
hipError_t launch(const PromptArgs& a, hipStream_t stream) {
  if (a.tokens <= 0 || a.batch <= 0) return hipSuccess;
  hipLaunchKernelGGL(attend_rows<MAPS>, dim3(a.tokens, a.q_heads / MAPS), dim3(64), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

size_t diff_prompt_workspace(const PromptArgs&) { return 0; }
hipError_t launch_diff_prompt_attention(const PromptArgs& a, hipStream_t s) { return launch<2>(a, s); }

}  // namespace ema
