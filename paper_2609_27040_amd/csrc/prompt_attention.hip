// Causal attention of prompt chunks over the paged cache, on the matrix cores.
//
// The G query heads that share a KV head are rows beside each other: row r of a
// sequence's n tokens is (token r / G, head r % G), and a workgroup of eight waves
// takes 256 rows, 32 to a wave, past K and V tiles of 64 tokens staged in LDS:
//   scores   S^T[token][row] = K . Q^T     v_mfma_f32_32x32x16, A = 32 K rows, B = Q^T
//            in registers; the rows of A are taken in an order that leaves every
//            lane with 8 consecutive tokens of one row twice over
//   softmax  online, in the log2 domain: every lane has 32 of its row's 64 scores
//            and the lane 32 away the others
//   output   O^T[channel][row] += V^T . P^T   A = 32 channels of the transposed V
//            block, B = P as the scores left it: nothing moves between lanes
// The output is rescaled only where a row's maximum has grown by more than 2^8 since
// the last time: weights are then at most 256 instead of 1, which costs a
// floating type nothing.
#include "prompt_common.h"

#include <algorithm>
#include <climits>

namespace ema {
namespace {

constexpr int kWaves = 8;
constexpr int kThreads = kWaves * 64;
constexpr int kRows = kWaves * 32;
constexpr float kSlack = 8.0f;

// P of a tile in NP 16-bit parts whose sum keeps 8 (bf16) or 11 (f16) bits each.
template <int NP>
struct Weights {
  u32x4 p[NP][4];        // [part][16 tokens]
};

template <bool BF16, int NP>
__device__ __forceinline__ void put_weights(Weights<NP>& w, int ks, const float (&p)[8]) {
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    float x = p[2 * q], y = p[2 * q + 1];
#pragma unroll
    for (int n = 0; n < NP; ++n) {
      const uint32_t u = pack16<BF16>(x, y);
      w.p[n][ks][q] = u;
      if (n + 1 < NP) {
        x -= low16<BF16>(u);
        y -= high16<BF16>(u);
      }
    }
  }
}

template <bool BF16, int BSC, int NP>
__global__ __launch_bounds__(kThreads, 2) void prompt_kernel(PromptArgs a, int tiles, int splits) {
  __shared__ __attribute__((aligned(16))) u32x4 s_k[2][kTilePieces];
  __shared__ __attribute__((aligned(16))) u32x4 s_v[2][kTilePieces];
  __shared__ int s_find[kFindScratch];
  __shared__ int s_bad[128];             // per channel: the first token not finite there
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int G = a.q_heads / a.kv_heads;
  const int kvh = int(blockIdx.x) % a.kv_heads;
  const int rest = int(blockIdx.x) / a.kv_heads;
  const int split = rest % splits;
  if (tid < 128) s_bad[tid] = INT_MAX;
  // the last tiles of a sequence see the most tokens: they go first
  const RowTile R = find_tile<kThreads>(a, G, kRows, tiles - 1 - rest / splits, s_find);
  if (R.b < 0) return;
  const int past = R.len - R.n;          // tokens before the chunk
  if (R.first == 0 && split == 0 && kvh == 0 && tid == 0 &&
      (past < 0 || R.len != a.seq_lens[R.b]))
    atomicAdd(a.err_count, 1);

  const int r = R.first + wave * 32 + col;
  const bool live = r < R.n * G;
  const int tok = live ? r / G : 0, g = live ? r - tok * G : 0;
  const int pos = live ? past + tok : -1;              // the row attends tokens 0 .. pos
  const int last_row = min(R.n * G, R.first + kRows) - 1;
  const int end = max(0, past + last_row / G + 1);     // tokens the workgroup looks at
  const int from = past + R.first / G;                 // position of its first row
  const int wave_first = R.first + wave * 32;
  const int wave_end = wave_first >= R.n * G
                           ? 0 : max(0, past + min(R.n * G - 1, wave_first + 31) / G + 1);
  const int wave_from = past + wave_first / G;
  const int n_tiles = (end + kKT - 1) / kKT;
  const int j0 = int(int64_t(n_tiles) * split / splits);
  const int j1 = int(int64_t(n_tiles) * (split + 1) / splits);

  u32x4 q[8];
  {
    const char* p = a.q + (int64_t(R.row0 + tok) * a.q_stride + (kvh * G + g) * 128 + half * 8) * 2;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) q[ks] = *reinterpret_cast<const u32x4*>(p + ks * 32);
  }
  f32x16 o[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) o[c] = f32x16{};
  float m = -INFINITY, l = 0.0f;         // l: this lane's half of the tokens

  const int32_t* trow = a.table + int64_t(R.b) * a.max_blocks;
  const int64_t v_half = a.block_bytes / 2;
  u32x4 kr[2], vr[2];
  TileIds<BSC> ids = load_ids<BSC>(a, trow, j0 * kKT, end), next_ids;
  // Issues the loads of tile j into the registers. Wave w's pieces 64w .. 64w + 63 of
  // each half tile lie in one block.
  auto load = [&](int j, TileIds<BSC>& t) {
    check_ids<BSC>(a, t);
    const int tb = BSC == 64 ? (j * kKT) % a.block_size : 0;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int kt = wave * 4 + x * 32 + (lane >> 4);          // K token of the tile
      const int kid = t.id[(wave * 4 + x * 32) / BSC];
      kr[x] = *reinterpret_cast<const u32x4*>(
          a.local + int64_t(max(kid, 0)) * a.block_bytes +
          ((kvh * a.block_size + tb + kt % BSC) * 128 + (lane & 15) * 8) * 2);
      constexpr int per = 16 * BSC;                              // V pieces of a block
      const int p = x * 512 + tid, vb = uniform(p / per);
      const int ch = p % per / (BSC / 8), gi = p % (BSC / 8);
      const int vid = t.id[vb];
      vr[x] = *reinterpret_cast<const u32x4*>(
          a.local + int64_t(max(vid, 0)) * a.block_bytes + v_half +
          (int64_t(kvh * 128 + ch) * a.block_size + tb + gi * 8) * 2);
    }
  };
  // Puts the loaded tile j into buffer x; V of tokens that are not there becomes 0.
  auto stage = [&](int j, const TileIds<BSC>& t, int x) {
    const bool edge = (j + 1) * kKT > from + 1;                  // some row masks some token
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const int kt = wave * 4 + y * 32 + (lane >> 4);
      s_k[x][k_place(kt, lane & 15)] = kr[y];
      constexpr int per = 16 * BSC;
      const int p = y * 512 + tid, vb = uniform(p / per);
      const int ch = p % per / (BSC / 8), gi = p % (BSC / 8);
      u32x4 v = vr[y];
      const int left = end - j * kKT - (vb * BSC + gi * 8);
      if (t.id[vb] < 0) v = u32x4{0, 0, 0, 0};
      if (edge) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          v[i] &= (2 * i < left ? 0xffffu : 0u) | (2 * i + 1 < left ? 0xffff0000u : 0u);
        if (not_finite<BF16>(v)) drop_not_finite<BF16>(v, j * kKT + vb * BSC + gi * 8, &s_bad[ch]);
      }
      s_v[x][v_place<BSC>(ch, vb * (BSC / 8) + gi)] = v;
    }
  };

  if (j0 < j1) {
    load(j0, ids);
    next_ids = load_ids<BSC>(a, trow, (j0 + 1) * kKT, end);
    __syncthreads();                     // s_bad is clear
    stage(j0, ids, 0);
  }
  __syncthreads();
  // A rows of the scores: MFMA row i of a 32-token tile is this token
  const int arow = (col >> 4) * 16 + ((col >> 2) & 1) * 8 + ((col >> 3) & 1) * 4 + (col & 3);
  for (int j = j0; j < j1; ++j) {
    const int buf = (j - j0) & 1;
    const TileIds<BSC> cur = ids;
    if (j + 1 < j1) {
      ids = next_ids;
      load(j + 1, ids);
      if (j + 2 < j1) next_ids = load_ids<BSC>(a, trow, (j + 2) * kKT, end);
    }
    const int t0 = j * kKT;
    bool all_ids = true;
#pragma unroll
    for (int i = 0; i < TileIds<BSC>::N; ++i) all_ids &= cur.id[i] >= 0;
    if (!all_ids && kvh == 0 && R.first == 0 && tid == 0) {
#pragma unroll
      for (int i = 0; i < TileIds<BSC>::N; ++i)
        if (cur.id[i] < 0 && t0 + i * BSC < end) atomicAdd(a.err_count, 1);
    }
    if (t0 < wave_end) {
      f32x16 s[2];
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        s[tt] = f32x16{};
#pragma unroll
        for (int ks = 0; ks < 8; ++ks)
          s[tt] = mfma32<BF16>(s_k[buf][k_place(tt * 32 + arow, ks * 2 + half)], q[ks], s[tt]);
      }
      const bool masked = t0 + kKT > wave_from + 1;
      if (masked || !all_ids) {
        const int rel = pos - t0 - half * 8;           // token 16k + e of this lane: 16k + e <= rel
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int t = tt * 32 + (i >> 3) * 16;     // of 16 tokens, in one block
            const bool ok = t + (i & 7) <= rel && cur.id[t / BSC] >= 0;
            s[tt][i] = ok ? s[tt][i] : -INFINITY;
          }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[tt][i]);
      mx = fmaxf(mx, other_half(mx)) * a.scale_log2;
      if (__ballot(mx > m + kSlack)) {
        const float m_new = fmaxf(m, mx);
        const float alpha = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - m_new);
        m = m_new;
        l *= alpha;
#pragma unroll
        for (int c = 0; c < 4; ++c) o[c] *= alpha;
      }
      const float ref = m == -INFINITY ? 0.0f : m;
      Weights<NP> w;
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = __builtin_amdgcn_exp2f(fmaf(s[ks >> 1][(ks & 1) * 8 + e], a.scale_log2, -ref));
          l += p[e];
        }
        put_weights<BF16, NP>(w, ks, p);
      }
#pragma unroll
      for (int ks = 0; ks < 4; ++ks)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const u32x4 v = s_v[buf][v_place<BSC>(c * 32 + col, ks * 2 + half)];
#pragma unroll
          for (int n = 0; n < NP; ++n) o[c] = mfma32<BF16>(v, w.p[n][ks], o[c]);
        }
    }
    if (j + 1 < j1) stage(j + 1, ids, buf ^ 1);
    __syncthreads();
  }

  l += other_half(l);
  if (!live) return;
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (pos >= s_bad[c * 32 + (i >> 2) * 8 + half * 4 + (i & 3)]) o[c][i] = NAN;
  const int64_t orow = int64_t(R.row0 + tok) * a.q_heads + kvh * G + g;
  if (splits > 1) {
    const int64_t part = int64_t(split) * a.tokens * a.q_heads + orow;
    float* po = a.ws + part * 128;
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4*>(po + c * 32 + i * 8 + half * 4) =
            f32x4{o[c][4 * i], o[c][4 * i + 1], o[c][4 * i + 2], o[c][4 * i + 3]};
    if (half == 0) {
      float* ml = a.ws + int64_t(splits) * a.tokens * a.q_heads * 128 + part * 2;
      ml[0] = m;
      ml[1] = l;
    }
    return;
  }
  AttnArgs st;
  st.out = a.out;
  st.out_dtype = a.out_dtype;
  st.out_vec = 1;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      store_out4(st, orow * 128 + c * 32 + i * 8 + half * 4,
                 out_f32x4{o[c][4 * i] * inv, o[c][4 * i + 1] * inv, o[c][4 * i + 2] * inv,
                           o[c][4 * i + 3] * inv});
}

// Joins the parts of a row: 32 lanes to a row, four channels a lane.
__global__ __launch_bounds__(256) void prompt_join(PromptArgs a, int splits) {
  const int64_t rows = int64_t(a.tokens) * a.q_heads;
  const int64_t row = int64_t(blockIdx.x) * 8 + (threadIdx.x >> 5);
  if (row >= rows) return;
  const int tok = int(row / a.q_heads);
  if (tok < a.starts[0] || tok >= a.starts[a.batch]) return;
  const int d = (threadIdx.x & 31) * 4;
  const float* ml = a.ws + splits * rows * 128;
  float M = -INFINITY;
  for (int s = 0; s < splits; ++s) M = fmaxf(M, ml[(s * rows + row) * 2]);
  const float ref = M == -INFINITY ? 0.0f : M;
  float L = 0.0f;
  f32x4 O = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s = 0; s < splits; ++s) {
    const float f = __builtin_amdgcn_exp2f(ml[(s * rows + row) * 2] - ref);
    L = fmaf(f, ml[(s * rows + row) * 2 + 1], L);
    const f32x4 x = *reinterpret_cast<const f32x4*>(a.ws + (s * rows + row) * 128 + d);
#pragma unroll
    for (int k = 0; k < 4; ++k) O[k] = fmaf(f, x[k], O[k]);
  }
  AttnArgs st;
  st.out = a.out;
  st.out_dtype = a.out_dtype;
  st.out_vec = 1;
  const float inv = L == 0.0f ? 0.0f : 1.0f / L;
  store_out4(st, row * 128 + d, out_f32x4{O[0] * inv, O[1] * inv, O[2] * inv, O[3] * inv});
}

// Tiles of all sequences at most, whatever their lengths.
int64_t tile_bound(const PromptArgs& a) {
  const int64_t rows = int64_t(a.tokens) * (a.q_heads / a.kv_heads);
  return std::min<int64_t>(a.tokens, (rows + kRows - 1) / kRows + a.batch - 1);
}

// Parts that a tile's tokens are cut into: as many as fill the chip's 256 compute
// units, of 256 tokens at least where the table is full.
int split_count(const PromptArgs& a) {
  const int64_t groups = tile_bound(a) * a.kv_heads;
  const int64_t most = int64_t(a.max_blocks) * a.block_size / 256;
  return int(std::max<int64_t>(1, std::min<int64_t>({256 / groups, most, 64})));
}

template <bool BF16, int NP>
hipError_t launch(const PromptArgs& a, hipStream_t stream) {
  const int64_t tiles = tile_bound(a);
  const int splits = split_count(a);
  const dim3 grid(unsigned(tiles * a.kv_heads * splits));
  switch (a.block_size) {
    case 16:
      hipLaunchKernelGGL((prompt_kernel<BF16, 16, NP>), grid, dim3(kThreads), 0, stream, a,
                         int(tiles), splits);
      break;
    case 32:
      hipLaunchKernelGGL((prompt_kernel<BF16, 32, NP>), grid, dim3(kThreads), 0, stream, a,
                         int(tiles), splits);
      break;
    default:
      hipLaunchKernelGGL((prompt_kernel<BF16, 64, NP>), grid, dim3(kThreads), 0, stream, a,
                         int(tiles), splits);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || splits == 1) return e;
  const int64_t rows = int64_t(a.tokens) * a.q_heads;
  hipLaunchKernelGGL(prompt_join, dim3(unsigned((rows + 7) / 8)), dim3(256), 0, stream, a, splits);
  return hipGetLastError();
}

}  // namespace

size_t prompt_workspace(const PromptArgs& a) {
  const int splits = split_count(a);
  return splits == 1 ? 0 : size_t(splits) * a.tokens * a.q_heads * 130 * 4;
}

hipError_t launch_prompt_attention(const PromptArgs& a, hipStream_t stream) {
  if (a.out_dtype != kOutF32)
    return a.dtype == 1 ? launch<true, 1>(a, stream) : launch<false, 1>(a, stream);
  return a.dtype == 1 ? launch<true, 3>(a, stream) : launch<false, 2>(a, stream);
}

}  // namespace ema
