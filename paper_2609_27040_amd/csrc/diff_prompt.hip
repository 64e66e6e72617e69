// Differential attention of prompt chunks over the paged cache, on the matrix cores, in
// two launches.
//
// The maps' difference is smaller than the maps, so it is formed in 32 bits before anything
// is rounded: the first launch finds each row's maximum m and sum l for each map (scores
// only), the second computes the scores again and multiplies
//   P = 2^(s1 - m1) / l1 - lambda 2^(s2 - m2) / l2,   rounded once,
// with V, once for both maps. In f16 a row's P is multiplied by a power of two before it is
// rounded, which the outputs are divided by: P is about 1 / length, where f16's steps of 2^-24
// show (32-bit outputs, 8191 tokens of scores of deviation 1/4: off by 2e-4 without). The
// maxima are a row's own there, not the last that its sum was scaled by, so the larger map's
// largest weight stands at 2^13 at least, and the step is 2^-37 of it. Against running both
// softmaxes beside each other with an output for each, that is the same number of products
// (scores of 2 x 128 twice, V of 256 once, instead of scores once and V twice), half the
// registers for outputs, no rescaling, and an error of the weights that is relative to the
// difference.
//
// First launch: as prompt attention without its V half; 256 rows of one KV head to a
// workgroup. Second: rows are (token, head of the group) of a pair of KV heads, 32 of them
// to two waves; either wave weighs 32 of a tile's 64 tokens for both maps and leaves its
// weights in LDS, and multiplies all 64 with one of the two V heads: as many products of
// scores as of V, none done twice. Waves take turns in two groups as in prompt
// attention, but with two places for tiles: a tile's K, and V of the one before, are sent for
// at the start of the two phases before those that read it and have arrived at their end. The
// group that has its softmax then sends for all of it, so that nothing stands before the
// other's products (each sending for half: three 8B prompts 141 us a call, so: 130).
// Outputs of 32 bits keep the weights in 2 (f16) or 3 (bf16) 16-bit parts, whose place in LDS
// leaves room for four waves only.
//
// Bound by the matrix cores and the exponentials in turns. Three prompts of 301-2047 tokens (32
// query, 8 KV heads, bf16) 120 us, 440 TFLOP/s of the 1024 operations per (head, token) that
// one pass with the sums known would take, 660 of those done; one of 4096 tokens 238 us, 580 and
// 870. The first launch takes 35 % of it. A first launch without turns, one barrier a tile: 243.
#include "prompt_common.h"

#include <algorithm>
#include <climits>

namespace ema {
namespace {

constexpr int kRing = 3;                 // K tiles of the first launch
constexpr int kStatWaves = 8;
constexpr int kStatThreads = kStatWaves * 64;
constexpr int kStatRows = kStatWaves * 32;
constexpr float kSlack = 8.0f;

// The query head that is head g of KV head kvh's group: heads 2i and 2i + 1 are a pair.
__device__ __forceinline__ int query_head(int kvh, int group, int g) {
  return 2 * ((kvh >> 1) * group + g) + (kvh & 1);
}

// Scores of the lane's row that it does not attend become -inf: token 8 * half + t0 + i.
template <int N>
__device__ __forceinline__ void mask_scores(f32x16 (&s)[N], int pos, int t0, int half) {
  const int rel = pos - t0 - half * 8;
#pragma unroll
  for (int x = 0; x < N; ++x)
#pragma unroll
    for (int i = 0; i < 16; ++i)
      s[x][i] = x * 32 + (i >> 3) * 16 + (i & 7) <= rel ? s[x][i] : -INFINITY;
}

// The first launch leaves (m, l) of every part of a row's tokens side by side, in an even
// number of places: a row's are then read 16 bytes at a time. (Parts apart, and each lane both
// maps: 10-14 us of a call of 62 with 21 parts.)
__host__ __device__ constexpr int stat_room(int splits) { return (splits + 1) & ~1; }

template <bool BF16, int BSC>
__global__ __launch_bounds__(kStatThreads, 2) void diff_stats(PromptArgs a, int splits) {
  __shared__ __attribute__((aligned(16))) u32x4 s_k[kRing][kTilePieces];
  __shared__ int s_find[kFindScratch];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int G = a.q_heads / a.kv_heads;
  const int kvh = int(blockIdx.x) % a.kv_heads, rest = int(blockIdx.x) / a.kv_heads;
  const int split = rest % splits;
  const RowTile R = find_tile<kStatThreads, kStatRows>(a, G, rest / splits, s_find);
  if (blockIdx.x == 0 && R.wrong > 0) atomicAdd(a.err_count, R.wrong);
  if (R.b < 0) return;
  if (R.first == 0 && split == 0 && kvh == 0 && tid == 0 && (R.len < R.n || R.len != R.given))
    atomicAdd(a.err_count, 1);
  const Reach at = reach_of<kStatRows>(R, G, R.first + wave * 32, split, splits);
  const int j0 = at.j0, j1 = at.j1, head = query_head(kvh, G, at.g);
  // the sequence's last rows see all of its tokens
  const bool counts = kvh == 0 && wave == 0 && R.first + kStatRows >= R.n * G;

  u32x4 q[8];
  {
    const char* p = a.q + (int64_t(R.row0 + at.tok) * a.q_stride + head * 128 + half * 8) * 2;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) q[ks] = *reinterpret_cast<const u32x4*>(p + ks * 32);
  }
  const uint32_t lds_k = lds_address(&s_k[0][0]);
  constexpr int kTileBytes = kTilePieces * 16;
  Staging<BSC, kStatThreads> st;
  // K of tile j + 1 has arrived, K of j + 2 is sent for.
  auto stage = [&](int j, int s2) {
    if (j >= j1) return;
    loads_arrived();
    if (st.window.bad != 0 && counts) st.count_bad(a, j, at.end);
    if (j + 2 < j1) st.load_k(lds_k + s2 * kTileBytes, j + 2, st.blocks(j + 2), 0);
  };
  f32x16 s[2] = {f32x16{}, f32x16{}};
  const int arow = score_row(col);
  constexpr int kAhead = 6;
  auto products = [&](int j, int slot) {
    if (j >= j1 || j * kKT >= at.wave_end) return;
    __builtin_amdgcn_s_setprio(1);
    u32x4 f[16];
#pragma unroll
    for (int i = 0; i < 16; ++i)
      f[i] = s_k[slot][k_place((i & 1) * 32 + arow, (i >> 1) * 2 + half)];
#pragma unroll
    for (int i = 0; i < 16; ++i)
      s[i & 1] = mfma32<BF16>(f[i], q[i >> 1], i < 2 ? f32x16{} : s[i & 1]);
    EMA_SCHED_LDS_READ(kAhead);
#pragma unroll
    for (int i = 0; i < 16 - kAhead; ++i) {
      EMA_SCHED_MFMA(1);
      EMA_SCHED_LDS_READ(1);
    }
    EMA_SCHED_MFMA(kAhead);
    __builtin_amdgcn_s_setprio(0);
  };
  float m = -INFINITY, l = 0.0f, top = -INFINITY;      // top: the largest score so far
  auto softmax = [&](int j) {
    const int t0 = j * kKT;
    if (t0 >= at.wave_end) return;
    if (t0 + kKT > at.wave_from + 1) mask_scores(s, at.pos, t0, half);
    if (st.window.bad != 0) {
#pragma unroll
      for (int x = 0; x < 4; ++x) {
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
    top = fmaxf(top, mx);
    if (__ballot(mx > m + kSlack)) {
      const float m_new = fmaxf(m, mx);
      l *= m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - m_new);
      m = m_new;
    }
    const float ref = m == -INFINITY ? 0.0f : m;
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        sum[i & 3] += __builtin_amdgcn_exp2f(fmaf(s[tt][i], a.scale_log2, -ref));
    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
  };
  if (j0 < j1) {
    st.open(a, R.b, kvh, j0, at.end);
    st.load_k(lds_k, j0, st.blocks(j0), 0);
    if (j0 + 1 < j1) st.load_k(lds_k + kTileBytes, j0 + 1, st.blocks(j0 + 1), 0);
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) arrived(q[ks]);
    loads_arrived();
    __syncthreads();
    const int late = wave >= kStatWaves / 2 ? 1 : 0;
    if (late) {
      stage(j0, 2);
      __syncthreads();
    }
    int s0 = 0, s1 = 1, s2 = 2;          // places of tiles j, j + 1 and j + 2
    for (int j = j0; j < j1; ++j) {
      products(j, s0);
      __syncthreads();
      stage(j + late, late ? s0 : s2);
      softmax(j);
      const int t = s0;
      s0 = s1;
      s1 = s2;
      s2 = t;
      __syncthreads();
    }
    if (!late) __syncthreads();
  }
  l += other_half(l);
  if constexpr (!BF16) {
    if (top > m) {
      l *= __builtin_amdgcn_exp2f(m - top);
      m = top;
    }
  }
  if (!at.live || half != 0) return;
  const int64_t row = int64_t(R.row0 + at.tok) * a.q_heads + head;
  reinterpret_cast<float2*>(a.ws)[row * stat_room(splits) + split] = float2{m, l};
}

template <int NP>
constexpr int kMulWaves = NP == 1 ? 8 : 4;
template <int NP>
constexpr int kMulRows = kMulWaves<NP> / 2 * 32;

template <bool BF16, int BSC, int NP>
__global__ __launch_bounds__(kMulWaves<NP> * 64, NP == 1 ? 2 : 1)
void diff_multiply(PromptArgs a, int stat_splits, int splits) {
  constexpr int kWaves = kMulWaves<NP>, kThreads = kWaves * 64, kRows = kMulRows<NP>;
  constexpr int kTileBytes = kTilePieces * 16;
  __shared__ __attribute__((aligned(16))) u32x4 s_k[2][2][kTilePieces];    // [place][KV head]
  __shared__ __attribute__((aligned(16))) u32x4 s_v[2][2][kTilePieces];
  __shared__ __attribute__((aligned(16))) u32x4 s_p[kWaves][2][NP][64];    // a wave's weights
  __shared__ int s_find[kFindScratch];
  // f16: what a lane's outputs are multiplied by at the end (registers are short)
  __shared__ float s_back[BF16 ? 1 : kThreads];
  __shared__ int s_bad[2 * 128 + 1];     // the first token not finite, per channel and of all
  float* const s_sq = reinterpret_cast<float*>(&s_p[0][0][0][0]);          // at the end
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int col = lane & 31, half = lane >> 5;
  const int G = a.q_heads / a.kv_heads, P = a.kv_heads / 2;
  const int pair = int(blockIdx.x) % P, rest = int(blockIdx.x) / P;
  const int split = rest % splits;
  for (int i = tid; i < 2 * 128 + 1; i += kThreads) s_bad[i] = INT_MAX;
  const RowTile R = find_tile<kThreads, kRows>(a, G, rest / splits, s_find);
  if (R.b < 0) return;
  const int mine = wave & 1;             // the half of a tile's tokens, and the V head
  const Reach at = reach_of<kRows>(R, G, R.first + (wave >> 1) * 32, split, splits);
  const int j0 = at.j0, j1 = at.j1;
  const int64_t row = int64_t(R.row0 + at.tok);
  const int head = pair * G + at.g;      // of the output; its maps are query heads 2h, 2h + 1

  u32x4 q[2][8];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const char* p = a.q + (row * a.q_stride + (2 * head + x) * 128 + half * 8) * 2;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) q[x][ks] = *reinterpret_cast<const u32x4*>(p + ks * 32);
  }
  // m, and 1 / l (the second map's times lambda): each half of the wave joins one map's parts,
  // the first of which are on their way while the first tile is sent for
  const f32x4* const ml = reinterpret_cast<const f32x4*>(
      a.ws + (row * a.q_heads + 2 * head + half) * stat_room(stat_splits) * 2);
  const int n_ml = stat_room(stat_splits) / 2;
  f32x4 part[4];
#pragma unroll
  for (int y = 0; y < 4; ++y) part[y] = ml[min(y, n_ml - 1)];
  const float factor = half == 0 ? 1.0f : a.lam[head];
  float ref[2], by[2];

  const uint32_t lds_k = lds_address(&s_k[0][0][0]), lds_v = lds_address(&s_v[0][0][0]);
  constexpr int kSenders = 256;          // threads: the second group, or all
  const int late = NP == 1 && wave >= kWaves / 2 ? 1 : 0;
  const bool sends = NP > 1 || late != 0;
  Staging<BSC, kSenders> st;
  typename Staging<BSC, kSenders>::Blocks next_v;
  auto place = [&](int j) { return (j - j0) & 1; };
  // K of tile j + 1 and V of tile j are sent for. The others follow in the table, to know of
  // entries that are no block.
  auto send = [&](int j) {
    if (j >= j1) return;
    if (!sends) {
      st.pass(j);
      return;
    }
#pragma unroll
    for (int x = 0; x < 2; ++x)
      st.load_v(lds_v + (place(j) * 2 + x) * kTileBytes, j, next_v, x);
    if (j + 1 < j1) {
      next_v = st.blocks(j + 1);
#pragma unroll
      for (int x = 0; x < 2; ++x)
        st.load_k(lds_k + (place(j + 1) * 2 + x) * kTileBytes, j + 1, next_v, x);
    }
  };
  // They are there.
  auto receive = [&](int j) {
    if (j >= j1 || !sends) return;
    loads_arrived();
    if ((j + 1) * kKT > at.from + 1 || st.window.bad != 0)
#pragma unroll 1
      for (int x = 0; x < 2; ++x)
        st.template clean_v<BF16>(s_v[place(j)][x], j, at.end, s_bad + x * 128, &s_bad[256]);
  };

  f32x16 o[4], s[2];
#pragma unroll
  for (int c = 0; c < 4; ++c) o[c] = f32x16{};
  s[0] = s[1] = f32x16{};
  const int arow = mine * 32 + score_row(col);
  constexpr int kAhead = NP == 1 ? 6 : 4;
  auto read_k = [&](int j, int i) {
    return s_k[place(j)][i & 1][k_place(arow, (i >> 1) * 2 + half)];
  };
  auto read_v = [&](int j, int i) {
    return s_v[place(j)][mine][v_place<BSC>((i & 3) * 32 + col, (i >> 2) * 2 + half)];
  };
  // The products of tile j: V of the tile before, K of this one.
  auto products = [&](int j) {
    const bool pv = j > j0 && (j - 1) * kKT < at.wave_end, qk = j < j1 && j * kKT < at.wave_end;
    __builtin_amdgcn_s_setprio(1);
    u32x4 f[16], g[kAhead];
    if (pv) {
      u32x4 w[4][NP];
#pragma unroll
      for (int ks = 0; ks < 4; ++ks)
#pragma unroll
        for (int n = 0; n < NP; ++n) w[ks][n] = s_p[(wave & ~1) + (ks >> 1)][ks & 1][n][lane];
#pragma unroll
      for (int i = 0; i < 16; ++i) f[i] = read_v(j - 1, i);
#pragma unroll
      for (int i = 0; i < kAhead; ++i) g[i] = read_k(j, i);    // not used where !qk
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int n = 0; n < NP; ++n) o[i & 3] = mfma32<BF16>(f[i], w[i >> 2][n], o[i & 3]);
      EMA_SCHED_LDS_READ(4 * NP + kAhead);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        EMA_SCHED_MFMA(NP);
        EMA_SCHED_LDS_READ(1);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) g[i] = read_k(j, i);
    }
    if (qk) {
#pragma unroll
      for (int i = 0; i < 16; ++i) f[i] = i < kAhead ? g[i] : read_k(j, i);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        s[i & 1] = mfma32<BF16>(f[i], q[i & 1][i >> 1], i < 2 ? f32x16{} : s[i & 1]);
#pragma unroll
      for (int i = 0; i < 16 - kAhead; ++i) {
        EMA_SCHED_MFMA(1);
        EMA_SCHED_LDS_READ(1);
      }
      EMA_SCHED_MFMA(kAhead);
    }
    __builtin_amdgcn_s_setprio(0);
  };
  // The weights of this wave's 32 tokens of tile j.
  auto weigh = [&](int j) {
    const int t0 = j * kKT + mine * 32;
    if (j * kKT >= at.wave_end) return;
    if (t0 + 32 > at.wave_from + 1) {
      const int rel = at.pos - t0 - half * 8;
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          s[x][i] = (i >> 3) * 16 + (i & 7) <= rel ? s[x][i] : -INFINITY;
    }
    if (st.window.bad != 0) {
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        if (st.window.good((t0 + y * 16) >> a.block_shift)) continue;
#pragma unroll
        for (int i = 0; i < 8; ++i) s[0][y * 8 + i] = s[1][y * 8 + i] = -INFINITY;
      }
    }
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      u32x4 w[NP];
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        float p[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int i = ks * 8 + 2 * y + e;
          const float p1 = __builtin_amdgcn_exp2f(fmaf(s[0][i], a.scale_log2, -ref[0]));
          const float p2 = __builtin_amdgcn_exp2f(fmaf(s[1][i], a.scale_log2, -ref[1]));
          p[e] = fmaf(p1, by[0], -(p2 * by[1]));
        }
#pragma unroll
        for (int n = 0; n < NP; ++n) {
          const uint32_t u = pack16<BF16>(p[0], p[1]);
          w[n][y] = u;
          p[0] -= low16<BF16>(u);
          p[1] -= high16<BF16>(u);
        }
      }
#pragma unroll
      for (int n = 0; n < NP; ++n) s_p[wave][ks][n][lane] = w[n];
    }
  };

  if (j0 < j1) {
    st.open(a, R.b, 2 * pair, j0, at.end);
    next_v = st.blocks(j0);
    if (sends)
#pragma unroll
      for (int x = 0; x < 2; ++x) st.load_k(lds_k + x * kTileBytes, j0, next_v, x);
  }
  {
    float m = -INFINITY, l = 0.0f;
    for (int y0 = 0; y0 < n_ml; y0 += 4) {
      if (y0 > 0)
#pragma unroll
        for (int y = 0; y < 4; ++y) part[y] = ml[min(y0 + y, n_ml - 1)];
#pragma unroll
      for (int y = 0; y < 4; ++y)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          if (2 * (y0 + y) + e >= stat_splits) continue;
          const float pm = part[y][2 * e], pl = part[y][2 * e + 1];
          const float m_new = fmaxf(m, pm), r = m_new == -INFINITY ? 0.0f : m_new;
          l = l * __builtin_amdgcn_exp2f(m - r) + pl * __builtin_amdgcn_exp2f(pm - r);
          m = m_new;
        }
    }
    const float mine_ref = m == -INFINITY ? 0.0f : m;
    const float mine_by = l == 0.0f ? 0.0f : factor / l;
    const float other_ref = other_half(mine_ref), other_by = other_half(mine_by);
    ref[0] = half == 0 ? mine_ref : other_ref;
    ref[1] = half == 0 ? other_ref : mine_ref;
    by[0] = half == 0 ? mine_by : other_by;
    by[1] = half == 0 ? other_by : mine_by;
    if constexpr (!BF16) {
      // 2^(s - m) is at most 1, so with the larger factor in [2^13, 2^14) P stays below 2^15
      const int up = 14 - __builtin_amdgcn_frexp_expf(fmaxf(by[0], fabsf(by[1])));
      by[0] = __builtin_amdgcn_ldexpf(by[0], up);
      by[1] = __builtin_amdgcn_ldexpf(by[1], up);
      s_back[tid] = __builtin_amdgcn_ldexpf(1.0f, -up);
    }
  }
  if (j0 < j1) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
#pragma unroll
      for (int ks = 0; ks < 8; ++ks) arrived(q[x][ks]);
      arrived(ref[x]);
      arrived(by[x]);
    }
    loads_arrived();
    __syncthreads();
    // Phase 2j: the first group has the products of tile j, the second weighs tile j - 1;
    // 2j + 1: the other way round. Tiles are sent for at the start of 2j and received at the
    // end of 2j + 1.
    if (late) {
      send(j0);
      __syncthreads();
    }
    for (int j = j0; j < j1; ++j) {
      if (!late) send(j);
      products(j);
      if (late) receive(j);
      __syncthreads();
      if (late) send(j + 1);
      weigh(j);
      if (!late) receive(j);
      __syncthreads();
    }
    products(j1);
    if (!late) __syncthreads();
  }
  __syncthreads();

  if constexpr (!BF16) {
    const float back = s_back[tid];
#pragma unroll
    for (int c = 0; c < 4; ++c) o[c] *= back;
  }
  if (s_bad[256] != INT_MAX)
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (at.pos >= s_bad[mine * 128 + c * 32 + (i >> 2) * 8 + half * 4 + (i & 3)]) o[c][i] = NAN;
  u32x4* const scratch = &s_k[0][0][0] + wave * 512;
  const int out_row = at.live ? int(row) * (a.q_heads / 2) + head : -1;
  if (splits > 1) {
    const int64_t rows = int64_t(a.tokens) * (a.q_heads / 2);
    write_rows(scratch, o, 1.0f, out_row, 256, mine * 128,
               a.ws + int64_t(stat_room(stat_splits)) * a.tokens * a.q_heads * 2 + split * rows * 256,
               kOutF32);
    return;
  }
  float inv = 1.0f;
  if (a.norm_weight) {
    float sq = 0.0f;
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) sq = fmaf(o[c][i], o[c][i], sq);
    sq += other_half(sq);
    s_sq[wave * 64 + lane] = sq;
    __syncthreads();
    sq += s_sq[(wave ^ 1) * 64 + lane];
    inv = sq == 0.0f ? 0.0f : 1.0f / sqrtf(sq / 256.0f + a.norm_eps);
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(a.norm_weight + mine * 128 + c * 32 + i * 8 +
                                                        half * 4);
#pragma unroll
        for (int k = 0; k < 4; ++k) o[c][4 * i + k] *= x[k];
      }
  }
  write_rows(scratch, o, inv, out_row, 256, mine * 128, a.out, a.out_dtype);
}

// Adds up the parts of a row: a wave to a row, four channels a lane (98 tokens, 8 heads, 25
// parts: 6 us).
__global__ __launch_bounds__(256) void diff_add(PromptArgs a, int stat_splits, int splits) {
  const int64_t rows = int64_t(a.tokens) * (a.q_heads / 2);
  const int64_t row = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (row >= rows) return;
  const int tok = int(row / (a.q_heads / 2));
  if (tok < a.starts[0] || tok >= a.starts[a.batch]) return;
  const int lane = threadIdx.x & 63;
  const float* parts = a.ws + int64_t(stat_room(stat_splits)) * a.tokens * a.q_heads * 2;
  f32x4 r = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int s = 0; s < splits; ++s)
    r += *reinterpret_cast<const f32x4*>(parts + (s * rows + row) * 256 + 4 * lane);
  if (a.norm_weight) {
    float sq = r[0] * r[0] + r[1] * r[1] + r[2] * r[2] + r[3] * r[3];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sq += __shfl_xor(sq, o);
    const float inv = sq == 0.0f ? 0.0f : 1.0f / sqrtf(sq / 256.0f + a.norm_eps);
    r *= *reinterpret_cast<const f32x4*>(a.norm_weight + 4 * lane) * inv;
  }
  AttnArgs to;
  to.out = a.out;
  to.out_dtype = a.out_dtype;
  to.out_vec = 1;
  store_out4(to, row * 256 + 4 * lane, out_f32x4{r[0], r[1], r[2], r[3]});
}

// How the two launches are cut: tiles of rows at most, whatever the lengths, and the parts
// that a tile's tokens are cut into. A part of the first launch costs a row 8 bytes: it takes
// what makes 1024 workgroups of them, two of which share a compute unit, but no more than 8
// unless they are needed to fill the chip. (256 / 512 / 1024 / 2048 workgroups, us a call: three
// 8B prompts 132 / 132 / 123 / 132, one of 4096 tokens 255 / 256 / 239 / 249; two chunks
// of 33 and 65 tokens, where 1024 would be 64 parts, 58 / 58 / 64 / 63.)
struct Cut {
  int64_t stat_tiles, mul_tiles;
  int stat_splits, mul_splits;
};
Cut cut_of(const PromptArgs& a) {
  const int64_t most = int64_t(a.max_blocks) * a.block_size / 256;
  const int mul_rows = a.full ? kMulRows<2> : kMulRows<1>;
  Cut c;
  c.stat_tiles = tile_bound(a, kStatRows);
  c.mul_tiles = tile_bound(a, mul_rows);
  const int64_t groups = c.stat_tiles * a.kv_heads;
  c.stat_splits = int(std::max<int64_t>(
      1, std::min<int64_t>({1024 / groups, std::max<int64_t>(8, 256 / groups), most, 64})));
  c.mul_splits = split_parts(a, c.mul_tiles * (a.kv_heads / 2));
  return c;
}

template <bool BF16, int BSC, int NP>
hipError_t launch(const PromptArgs& a, const Cut& c, hipStream_t stream) {
  hipLaunchKernelGGL((diff_stats<BF16, BSC>),
                     dim3(unsigned(c.stat_tiles * a.kv_heads * c.stat_splits)), dim3(kStatThreads),
                     0, stream, a, c.stat_splits);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((diff_multiply<BF16, BSC, NP>),
                     dim3(unsigned(c.mul_tiles * (a.kv_heads / 2) * c.mul_splits)),
                     dim3(kMulWaves<NP> * 64), 0, stream, a, c.stat_splits, c.mul_splits);
  return hipGetLastError();
}

template <bool BF16, int NP>
hipError_t launch_sizes(const PromptArgs& a, const Cut& c, hipStream_t stream) {
  return a.block_size == 16   ? launch<BF16, 16, NP>(a, c, stream)
         : a.block_size == 32 ? launch<BF16, 32, NP>(a, c, stream)
                              : launch<BF16, 64, NP>(a, c, stream);
}

}  // namespace

size_t diff_prompt_workspace(const PromptArgs& a) {
  // how the weights are kept is not known here: the larger of the two cuts
  PromptArgs b = a;
  size_t most = 0;
  for (int full : {0, 1}) {
    b.full = full;
    const Cut c = cut_of(b);
    size_t n = size_t(stat_room(c.stat_splits)) * a.tokens * a.q_heads * 2;
    if (c.mul_splits > 1) n += size_t(c.mul_splits) * a.tokens * (a.q_heads / 2) * 256;
    most = std::max(most, n);
  }
  return most * 4;
}

hipError_t launch_diff_prompt_attention(const PromptArgs& a, hipStream_t stream) {
  const Cut c = cut_of(a);
  hipError_t e;
  if (!a.full)
    e = a.dtype == 1 ? launch_sizes<true, 1>(a, c, stream) : launch_sizes<false, 1>(a, c, stream);
  else
    e = a.dtype == 1 ? launch_sizes<true, 3>(a, c, stream) : launch_sizes<false, 2>(a, c, stream);
  if (e != hipSuccess || c.mul_splits == 1) return e;
  const int64_t rows = int64_t(a.tokens) * (a.q_heads / 2);
  hipLaunchKernelGGL(diff_add, dim3(unsigned((rows + 3) / 4)), dim3(256), 0, stream, a,
                     c.stat_splits, c.mul_splits);
  return hipGetLastError();
}

}  // namespace ema
