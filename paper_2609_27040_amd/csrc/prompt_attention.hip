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
// floating type nothing. In f16 weights and their sum are 2^7 times as large, so that the
// largest stay below 2^15 and the smallest step, 2^-24, is 2^-31 of the row's largest weight;
// with two parts 2^11 times, from a growth of 2^4 on (2 % slower), for 2^-35. (Without: a row
// whose first token has all the weight and no value, 12 above the other scores, was off by 9e-4
// in 32 bits, now 2e-6.)
//
// 4 * 128 operations per (row, token it attends): bound by the matrix cores, fed from LDS. The
// 32 products of a wave's tile take 1024 cycles at least, its softmax some 1150, so the waves
// take turns in two groups (below), and a tile of 64 tokens and 256 rows takes 1.7 us = 3400
// cycles for 2048 of products. One prompt of 8191 tokens (32 query, 8 KV heads, bf16): 498 us,
// 1100 TFLOP/s; four of 257-3841 tokens 207 us, 947; 512 tokens behind 32001 (8 and 1 heads),
// 16 parts and their join, 81 us, 837. (A large matrix product of the vendor's library:
// 1130-1370.) With 64 rows to a wave the operands would be read half as often, but they spill.
#include "prompt_common.h"

#include <algorithm>
#include <climits>

namespace ema {
namespace {

constexpr int kWaves = 8;
constexpr int kThreads = kWaves * 64;
constexpr int kRows = kWaves * 32;
constexpr int kRing = 3;                 // staged tiles

// P of a tile in NP 16-bit parts whose sum keeps 8 (bf16) or 11 (f16) bits each.
template <int NP>
struct Weights {
  u32x4 p[NP][4];        // [part][16 tokens]
};

template <bool BF16, int NP>
__device__ __forceinline__ void put_weights(Weights<NP>& w, int ks, int q, float x, float y) {
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

// The eight waves are two groups, one of each to a SIMD, that take turns: while one
// has the matrix cores (the last tile's weights times V, then the next scores), the
// other works its scores into weights, puts its share of a later tile into LDS and
// issues the loads of the one after. Phase p: the first group has the products of tile
// p / 2 when p is even and its softmax when p is odd, the second group one phase
// later; a barrier ends each. K of tile j and V of tile j - 1 are read in phases 2j
// and 2j + 1; in those two phases K of j + 2 and V of j + 1 are sent for, straight into
// LDS, to the places of K of j - 1 and V of j - 2, which the phases before were the last
// to read, and in the next two each wave waits for its own before it goes on.
template <bool BF16, int BSC, int NP>
__global__ __launch_bounds__(kThreads, 2) void prompt_kernel(PromptArgs a, int splits) {
  __shared__ __attribute__((aligned(16))) u32x4 s_kv[2][kRing][kTilePieces];
  auto& s_k = s_kv[0];
  auto& s_v = s_kv[1];
  __shared__ int s_find[kFindScratch];
  __shared__ int s_bad[129];             // the first token not finite, per channel and of all
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int G = a.q_heads / a.kv_heads;
  const int kvh = int(blockIdx.x) % a.kv_heads;
  const int rest = int(blockIdx.x) / a.kv_heads;
  const int split = rest % splits;
  if (tid < 129) s_bad[tid] = INT_MAX;
  const RowTile R = find_tile<kThreads, kRows>(a, G, rest / splits, s_find);
  if (blockIdx.x == 0 && R.wrong > 0) atomicAdd(a.err_count, R.wrong);
  if (R.b < 0) return;
  if (R.first == 0 && split == 0 && kvh == 0 && tid == 0 && (R.len < R.n || R.len != R.given))
    atomicAdd(a.err_count, 1);
  const Reach at = reach_of<kRows>(R, G, R.first + wave * 32, split, splits);
  const int j0 = at.j0, j1 = at.j1;
  // the sequence's last rows see all of its tokens
  const bool counts = kvh == 0 && wave == 0 && R.first + kRows >= R.n * G;

  u32x4 q[8];
  {
    const char* p = a.q + (int64_t(R.row0 + at.tok) * a.q_stride + (kvh * G + at.g) * 128 + half * 8) * 2;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) q[ks] = *reinterpret_cast<const u32x4*>(p + ks * 32);
  }

  // ---- staging -------------------------------------------------------------------
  const uint32_t lds_k = lds_address(&s_k[0][0]), lds_v = lds_address(&s_v[0][0]);
  constexpr int kTileBytes = kTilePieces * 16;
  Staging<BSC, kThreads> st;
  typename Staging<BSC, kThreads>::Blocks next_v;   // of the K tile on its way, whose V is next
  // Step j: V of tile j and K of tile j + 1 have arrived; V of j + 1 and K of j + 2 are
  // sent for. s0, s1, s2: places of tiles j, j + 1 and j + 2.
  auto stage = [&](int j, int s0, int s1, int s2) {
    if (j >= j1) return;
    loads_arrived();
    if ((j + 1) * kKT > at.from + 1 || st.window.bad != 0)      // some row masks some token
      st.template clean_v<BF16>(s_v[s0], j, at.end, s_bad, &s_bad[128]);
    if (st.window.bad != 0 && counts) st.count_bad(a, j, at.end);
    if (j + 1 < j1) st.load_v(lds_v + s1 * kTileBytes, j + 1, next_v, 0);
    if (j + 2 < j1) {
      next_v = st.blocks(j + 2);
      st.load_k(lds_k + s2 * kTileBytes, j + 2, next_v, 0);
    }
  };

  // ---- products ------------------------------------------------------------------
  f32x16 o[4], s[2];
#pragma unroll
  for (int c = 0; c < 4; ++c) o[c] = f32x16{};
  s[0] = s[1] = f32x16{};
  Weights<NP> w;
  const int arow = score_row(col);
  // operands this many products ahead of their use (fewer where registers are short)
  constexpr int kAhead = NP == 3 ? 4 : 6;
  auto read_k = [&](int slot, int i) {
    return s_k[slot][k_place((i & 1) * 32 + arow, (i >> 1) * 2 + half)];
  };
  auto read_v = [&](int slot, int i) {
    return s_v[slot][v_place<BSC>((i & 3) * 32 + col, (i >> 2) * 2 + half)];
  };
  auto score = [&](int i, u32x4 f) {
    s[i & 1] = mfma32<BF16>(f, q[i >> 1], i < 2 ? f32x16{} : s[i & 1]);
  };
  auto weigh_v = [&](int i, u32x4 f) {
#pragma unroll
    for (int n = 0; n < NP; ++n) o[i & 3] = mfma32<BF16>(f, w.p[n][i >> 2], o[i & 3]);
  };
  // The products of tile j: V of the tile before, K of this one, from their places.
  auto products = [&](int j, int before, int slot) {
    const bool pv = j > j0 && (j - 1) * kKT < at.wave_end, qk = j < j1 && j * kKT < at.wave_end;
    __builtin_amdgcn_s_setprio(1);
    u32x4 f[16], g[kAhead];
    if (pv) {
#pragma unroll
      for (int i = 0; i < 16; ++i) f[i] = read_v(before, i);
#pragma unroll
      for (int i = 0; i < kAhead; ++i) g[i] = read_k(slot, i);   // not used where !qk
#pragma unroll
      for (int i = 0; i < 16; ++i) weigh_v(i, f[i]);
      EMA_SCHED_LDS_READ(kAhead);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        EMA_SCHED_MFMA(NP);
        EMA_SCHED_LDS_READ(1);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) g[i] = read_k(slot, i);
    }
    if (qk) {
#pragma unroll
      for (int i = 0; i < 16; ++i) f[i] = i < kAhead ? g[i] : read_k(slot, i);
#pragma unroll
      for (int i = 0; i < 16; ++i) score(i, f[i]);
#pragma unroll
      for (int i = 0; i < 16 - kAhead; ++i) {
        EMA_SCHED_MFMA(1);
        EMA_SCHED_LDS_READ(1);
      }
      EMA_SCHED_MFMA(kAhead);
    }
    __builtin_amdgcn_s_setprio(0);
  };

  // ---- softmax -------------------------------------------------------------------
  constexpr float kSlack = BF16 || NP == 1 ? 8.0f : 4.0f, kUp = BF16 ? 0.0f : 15.0f - kSlack;
  float m = -INFINITY, l = 0.0f;         // l: this lane's half of the tokens
  auto softmax = [&](int j) {
    const int t0 = j * kKT;
    if (j >= j1 || t0 >= at.wave_end) return;
    if (t0 + kKT > at.wave_from + 1) {
      const int rel = at.pos - t0 - half * 8;             // token 16k + e of this lane: 16k + e <= rel
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          s[tt][i] = tt * 32 + (i >> 3) * 16 + (i & 7) <= rel ? s[tt][i] : -INFINITY;
    }
    if (st.window.bad != 0) {
#pragma unroll
      for (int x = 0; x < 4; ++x) {                    // 16 tokens, in one block
        if (st.window.good((t0 + x * 16) >> a.block_shift)) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) s[x >> 1][(x & 1) * 8 + i] = -INFINITY;
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
    const float ref = m == -INFINITY ? 0.0f : m - kUp;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        float p[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          p[e] = __builtin_amdgcn_exp2f(
              fmaf(s[ks >> 1][(ks & 1) * 8 + 2 * x + e], a.scale_log2, -ref));
          l += p[e];
        }
        put_weights<BF16, NP>(w, ks, x, p[0], p[1]);
      }
  };

  // ---- the phases ----------------------------------------------------------------
  if (j0 < j1) {
    st.open(a, R.b, kvh, j0, at.end);
    next_v = st.blocks(j0);
    st.load_k(lds_k, j0, next_v, 0);
    st.load_v(lds_v, j0, next_v, 0);
    if (j0 + 1 < j1) {
      next_v = st.blocks(j0 + 1);
      st.load_k(lds_k + kTileBytes, j0 + 1, next_v, 0);
    }
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) arrived(q[ks]);
    loads_arrived();
    __syncthreads();
    // One loop for both groups; the second stages first and starts a phase later.
    const int late = wave >= kWaves / 2 ? 1 : 0;
    if (late) {
      stage(j0, 0, 1, 2);
      __syncthreads();
    }
    int s0 = 0, s1 = 1, s2 = 2;          // places of tiles j, j + 1 and j + 2 (and j - 1)
    for (int j = j0; j < j1; ++j) {
      products(j, s2, s0);
      __syncthreads();
      stage(j + late, late ? s1 : s0, late ? s2 : s1, late ? s0 : s2);
      softmax(j);
      const int t = s0;
      s0 = s1;
      s1 = s2;
      s2 = t;
      __syncthreads();
    }
    products(j1, s2, s0);
    if (!late) __syncthreads();
  }
  __syncthreads();

  l += other_half(l);
  if (s_bad[128] != INT_MAX)
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (at.pos >= s_bad[c * 32 + (i >> 2) * 8 + half * 4 + (i & 3)]) o[c][i] = NAN;
  const int row = at.live ? (R.row0 + at.tok) * a.q_heads + kvh * G + at.g : -1;
  u32x4* const scratch = &s_kv[0][0][0] + wave * 512;
  if (splits == 1) {
    write_rows(scratch, o, l == 0.0f ? 0.0f : 1.0f / l, row, 128, 0, a.out, a.out_dtype);
    return;
  }
  const int64_t rows = int64_t(a.tokens) * a.q_heads;
  write_rows(scratch, o, 1.0f, row, 128, 0, a.ws + split * rows * 128, kOutF32);
  if (at.live && half == 0) {
    float* ml = a.ws + splits * rows * 128 + (split * rows + row) * 2;
    ml[0] = m;
    ml[1] = l;
  }
}

// Joins the parts of a row: 32 lanes to a row, four channels a lane. Bound by reading the
// parts: 4096 rows in 16 parts, 34 MB, 13 us.
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

int split_count(const PromptArgs& a) { return split_parts(a, tile_bound(a, kRows) * a.kv_heads); }

template <bool BF16, int NP>
hipError_t launch(const PromptArgs& a, hipStream_t stream) {
  const int64_t tiles = tile_bound(a, kRows);
  const int splits = split_count(a);
  const dim3 grid(unsigned(tiles * a.kv_heads * splits));
  switch (a.block_size) {
    case 16:
      hipLaunchKernelGGL((prompt_kernel<BF16, 16, NP>), grid, dim3(kThreads), 0, stream, a,
                         splits);
      break;
    case 32:
      hipLaunchKernelGGL((prompt_kernel<BF16, 32, NP>), grid, dim3(kThreads), 0, stream, a,
                         splits);
      break;
    default:
      hipLaunchKernelGGL((prompt_kernel<BF16, 64, NP>), grid, dim3(kThreads), 0, stream, a,
                         splits);
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
  if (!a.full)
    return a.dtype == 1 ? launch<true, 1>(a, stream) : launch<false, 1>(a, stream);
  return a.dtype == 1 ? launch<true, 3>(a, stream) : launch<false, 2>(a, stream);
}

}  // namespace ema
