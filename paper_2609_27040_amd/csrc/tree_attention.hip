// Attention of drafted trees over the paged cache, on the matrix cores.
//
// The G query heads that share a KV head are rows beside each other: row r of a
// request's n nodes is (node r / G, head r % G), and a workgroup takes 32 RT rows
// past the request's tokens in tiles of 64, its four waves in turn:
//   scores   S^T[token][row] = K . Q^T     v_mfma_f32_32x32x16, A = 32 K rows, B = Q^T
//            in registers; the rows of A are taken in an order that leaves every
//            lane with 8 consecutive tokens of one row twice over
//   softmax  online, in the log2 domain: every lane has 32 of its row's 64 scores
//            and the lane 32 away the others
//   output   O^T[channel][row] += V^T . P^T   A = 32 channels of the transposed V
//            block, B = P as the scores left it: nothing moves between lanes
// Each wave loads its own tiles, straight into its own 32 KiB of LDS, and keeps its own
// maximum, sum and output; they are merged in the place of the tiles at the end.
//
// Only tiles that reach past the older tokens look at the mask: 64 bits of it, those of
// the tile's tokens, are shifted into place from two words of the row's. There V is
// cleaned of what is not finite, since 0 times it would be NaN for rows that do not attend
// it; where a tile has such values, a second product, of ones in their places and ones
// for the attended tokens, tells which rows' channels become NaN.
//
// The output is rescaled only where a row's maximum has grown by more than 2^8; in f16
// weights and their sum are kept in a power-of-two scale in which the largest stand just
// below 2^15, as in the prompt kernels.
#include "prompt_common.h"
#include "tree_kernels.h"

#include <algorithm>

namespace ema {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * 64;

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

// A piece's values that are not finite: zeroed in the piece; ones in their places.
template <bool BF16>
__device__ __forceinline__ u32x4 take_not_finite(u32x4& v) {
  constexpr uint32_t kExp = BF16 ? 0x7f80u : 0x7c00u, kOne = BF16 ? 0x3f80u : 0x3c00u;
  u32x4 ones;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool lo = (v[i] & kExp) == kExp, hi = ((v[i] >> 16) & kExp) == kExp;
    ones[i] = (lo ? kOne : 0u) | (hi ? kOne << 16 : 0u);
    v[i] &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
  }
  return ones;
}

template <bool BF16, int BSC, int NP, int RT>
__global__ __launch_bounds__(kThreads, 1) void tree_kernel(TreeAttnArgs a) {
  constexpr int kRows = 32 * RT;
  constexpr uint32_t kOne = BF16 ? 0x3f80u : 0x3c00u;
  // K and V of a tile per wave; at the end each wave's outputs
  __shared__ __attribute__((aligned(16))) u32x4 s_kv[kWaves][2][kTilePieces];
  __shared__ float s_m[kWaves][kRows], s_l[kWaves][kRows];
  __shared__ int s_find[kFindScratch];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int G = a.q_heads / a.kv_heads;
  const int kvh = int(blockIdx.x) % a.kv_heads;
  const RowTile R = find_in_order<kThreads, kRows>(a, G, int(blockIdx.x) / a.kv_heads, s_find);
  if (blockIdx.x == 0 && R.wrong > 0) atomicAdd(a.err_count, R.wrong);
  if (R.b < 0) return;
  if (R.first == 0 && kvh == 0 && tid == 0 && (R.len < R.n || R.len != R.given))
    atomicAdd(a.err_count, 1);
  const int base = R.len - R.n;            // tokens before the tree; negative: nodes without a place
  const int tiles = (R.len + kKT - 1) / kKT;
  const bool counts = kvh == 0 && R.first == 0;

  // this lane's rows
  int tok[RT], head[RT];
  bool live[RT];
  u32x4 q[RT][8];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = R.first + rt * 32 + col;
    live[rt] = r < R.n * G;
    tok[rt] = live[rt] ? r / G : 0;
    head[rt] = kvh * G + (live[rt] ? r - tok[rt] * G : 0);
    const char* p = a.q + (int64_t(R.row0 + tok[rt]) * a.q_stride + head[rt] * 128 + half * 8) * 2;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) q[rt][ks] = *reinterpret_cast<const u32x4*>(p + ks * 32);
  }

  auto& s_k = s_kv[wave][0];
  auto& s_v = s_kv[wave][1];
  const uint32_t lds_k = lds_address(&s_k[0]), lds_v = lds_address(&s_v[0]);
  Staging<BSC, 64> st;
  typename Staging<BSC, 64>::Blocks at;

  f32x16 o[RT][4], s[RT][2];
  float m[RT], l[RT];                      // l: this lane's half of the tokens
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    m[rt] = -INFINITY;
    l[rt] = 0.0f;
#pragma unroll
    for (int c = 0; c < 4; ++c) o[rt][c] = f32x16{};
  }
  const int arow = score_row(col);
  constexpr float kSlack = BF16 || NP == 1 ? 8.0f : 4.0f, kUp = BF16 ? 0.0f : 15.0f - kSlack;

  // Which tokens of the tile from t0 on row rt attends, a bit each.
  auto attended = [&](int rt, int t0) -> uint64_t {
    if (!live[rt] || base + tok[rt] < 0) return 0;
    const uint64_t* words = a.mask + int64_t(R.row0 + tok[rt]) * a.words;
    const int j = t0 - base;               // the node at the tile's first token
    uint64_t x;
    if (j <= -64) {
      x = ~0ull;
    } else if (j < 0) {
      x = (words[0] << -j) | ((1ull << -j) - 1ull);
    } else {
      const int w = j >> 6, by = j & 63;
      x = w < a.words ? words[w] >> by : 0;
      if (by > 0 && w + 1 < a.words) x |= words[w + 1] << (64 - by);
    }
    const int left = R.len - t0;
    if (left < 64) x &= (1ull << left) - 1ull;
    if (st.window.bad != 0)
#pragma unroll
      for (int i = 0; i < 4; ++i)          // 16 tokens, in one block
        if (!st.window.good((t0 + 16 * i) >> a.block_shift)) x &= ~(0xffffull << (16 * i));
    return x;
  };

  if (wave < tiles) {
    st.open(a, R.b, kvh, wave, R.len);
    at = st.blocks(wave);
    st.load_k(lds_k, wave, at, 0);
    st.load_v(lds_v, wave, at, 0);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int ks = 0; ks < 8; ++ks) arrived(q[rt][ks]);
  }
  for (int j = wave; j < tiles; j += kWaves) {
    const int t0 = j * kKT;
    const bool more = j + kWaves < tiles;
    const bool partly = t0 + kKT > base || st.window.bad != 0;
    uint64_t sees[RT];
    loads_arrived();
    if (counts && st.window.bad != 0) st.count_bad(a, j, R.len);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) sees[rt] = partly ? attended(rt, t0) : ~0ull;
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int ks = 0; ks < 8; ++ks) {
        const u32x4 k = s_k[k_place(tt * 32 + arow, ks * 2 + half)];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
          s[rt][tt] = mfma32<BF16>(k, q[rt][ks], ks == 0 ? f32x16{} : s[rt][tt]);
      }
    Weights<NP> w[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      if (partly) {
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
          const uint32_t bits = uint32_t(sees[rt] >> (tt * 32 + half * 8));
#pragma unroll
          for (int i = 0; i < 16; ++i)
            s[rt][tt][i] = (bits >> ((i >> 3) * 16 + (i & 7))) & 1 ? s[rt][tt][i] : -INFINITY;
        }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[rt][tt][i]);
      mx = fmaxf(mx, other_half(mx)) * a.scale_log2;
      if (__ballot(mx > m[rt] + kSlack)) {
        const float m_new = fmaxf(m[rt], mx);
        const float alpha = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[rt] - m_new);
        m[rt] = m_new;
        l[rt] *= alpha;
#pragma unroll
        for (int c = 0; c < 4; ++c) o[rt][c] *= alpha;
      }
      const float ref = m[rt] == -INFINITY ? 0.0f : m[rt] - kUp;
#pragma unroll
      for (int ks = 0; ks < 4; ++ks)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          float p[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            p[e] = __builtin_amdgcn_exp2f(
                fmaf(s[rt][ks >> 1][(ks & 1) * 8 + 2 * x + e], a.scale_log2, -ref));
            l[rt] += p[e];
          }
          put_weights<BF16, NP>(w[rt], ks, x, p[0], p[1]);
        }
    }
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        u32x4 v = s_v[v_place<BSC>(c * 32 + col, ks * 2 + half)];
        if (partly && __ballot(not_finite<BF16>(v))) {
          const u32x4 bad = take_not_finite<BF16>(v);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            const uint32_t bits = uint32_t(sees[rt] >> (ks * 16 + half * 8));
            u32x4 ones;
#pragma unroll
            for (int i = 0; i < 4; ++i)
              ones[i] = (bits >> (2 * i) & 1 ? kOne : 0u) | (bits >> (2 * i + 1) & 1 ? kOne << 16 : 0u);
            const f32x16 hit = mfma32<BF16>(bad, ones, f32x16{});
#pragma unroll
            for (int i = 0; i < 16; ++i) o[rt][c][i] = hit[i] > 0.0f ? NAN : o[rt][c][i];
          }
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int n = 0; n < NP; ++n) o[rt][c] = mfma32<BF16>(v, w[rt].p[n][ks], o[rt][c]);
      }
    reads_done();
    if (more) {
      at = st.blocks(j + kWaves);
      st.load_k(lds_k, j + kWaves, at, 0);
      st.load_v(lds_v, j + kWaves, at, 0);
    }
  }

  // ---- the waves' parts of a row -------------------------------------------------------
  __syncthreads();
  f32x4* const part = reinterpret_cast<f32x4*>(&s_kv[0][0][0]);
  // Four channels 4f .. 4f + 3 of a wave's row, rows off each other's banks.
  auto part_at = [&](int w, int r, int f) -> f32x4& {
    return part[w * (2 * kTilePieces) + r * 32 + (f ^ (r & 31))];
  };
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const float sum = l[rt] + other_half(l[rt]);
    if (half == 0) {
      s_m[wave][rt * 32 + col] = m[rt];
      s_l[wave][rt * 32 + col] = sum;
    }
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        part_at(wave, rt * 32 + col, c * 8 + i * 2 + half) =
            f32x4{o[rt][c][4 * i], o[rt][c][4 * i + 1], o[rt][c][4 * i + 2], o[rt][c][4 * i + 3]};
  }
  __syncthreads();
  AttnArgs out;
  out.out = a.out;
  out.out_dtype = a.out_dtype;
  out.out_vec = 1;
  for (int x = tid; x < kRows * 32; x += kThreads) {
    const int r = x >> 5, f = x & 31;
    if (R.first + r >= R.n * G) break;
    float M = -INFINITY, L = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) M = fmaxf(M, s_m[w][r]);
    const float ref = M == -INFINITY ? 0.0f : M;
    f32x4 O = f32x4{};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float by = __builtin_amdgcn_exp2f(s_m[w][r] - ref);
      L = fmaf(by, s_l[w][r], L);
      O += part_at(w, r, f) * by;
    }
    const float inv = L == 0.0f ? 0.0f : 1.0f / L;
    const int node = (R.first + r) / G, g = R.first + r - node * G;
    store_out4(out, (int64_t(R.row0 + node) * a.q_heads + kvh * G + g) * 128 + 4 * f,
               out_f32x4{O[0] * inv, O[1] * inv, O[2] * inv, O[3] * inv});
  }
}

int row_tiles(const PromptArgs& a) {
  const int64_t rows = (int64_t(a.tokens) + a.batch - 1) / a.batch * (a.q_heads / a.kv_heads);
  return rows <= 32 ? 1 : 2;
}

template <bool BF16, int NP, int RT>
void launch_sizes(const TreeAttnArgs& a, hipStream_t stream) {
  const dim3 grid(unsigned(tile_bound(a, 32 * RT) * a.kv_heads));
  if (a.block_size == 16)
    hipLaunchKernelGGL((tree_kernel<BF16, 16, NP, RT>), grid, dim3(kThreads), 0, stream, a);
  else if (a.block_size == 32)
    hipLaunchKernelGGL((tree_kernel<BF16, 32, NP, RT>), grid, dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((tree_kernel<BF16, 64, NP, RT>), grid, dim3(kThreads), 0, stream, a);
}

template <bool BF16, int NP>
void launch_rows(const TreeAttnArgs& a, hipStream_t stream) {
  if (row_tiles(a) == 1) launch_sizes<BF16, NP, 1>(a, stream);
  else launch_sizes<BF16, NP, 2>(a, stream);
}

}  // namespace

size_t tree_workspace(const PromptArgs&) { return 0; }

hipError_t launch_tree_attention(const TreeAttnArgs& a, hipStream_t stream) {
  if (a.dtype == 1) {
    if (a.full) launch_rows<true, 3>(a, stream);
    else launch_rows<true, 1>(a, stream);
  } else {
    if (a.full) launch_rows<false, 2>(a, stream);
    else launch_rows<false, 1>(a, stream);
  }
  return hipGetLastError();
}

}  // namespace ema
