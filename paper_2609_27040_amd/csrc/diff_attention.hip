// Differential attention of one token per sequence over the paged cache, on the
// matrix cores.
//
// The two maps of the G heads that share a pair of KV heads are columns of one tile of
// scores S^T[token][map, head], with both maps' queries side by side as the B operand: the
// columns of map 1 are taken from K1 . [Q1 | Q2], those of map 2 from K2 . [Q1 | Q2]
// (G <= 8: one 16-wide tile; above, a tile for each map). Softmax runs per column as in plain
// decode; O^T[channel][map, head] += [V1 V2]^T . P^T has 256 channels and reads V once
// for both maps. At the end o = o1 / l1 - lambda o2 / l2 and, where asked, its norm over
// the 256 channels. Weights keep NP 16-bit parts, each rounded to nearest (two for
// 16-bit outputs, since the maps' difference is smaller than the maps; for 32-bit outputs
// two in f16, 22 bits, and three in bf16, 24). In f16 weights and their sum are 2^15 times as
// large, so that the smallest step, 2^-24, is 2^-39 of the largest weight (without: a row whose
// first token has all the weight and no value, 12 above the other scores, was off by 7e-4).
//
// Work: 32-token tiles of one (sequence, KV pair), 32 KiB each, all of them in a row
// cut into equal ranges, one per workgroup, one workgroup to a CU. The four waves of a
// workgroup take a segment's tiles in turn. Operands go straight into LDS, each wave's own
// 32 KiB of it and each lane's where the lane will read them, so that a whole tile is
// always on its way without a register held for it: K of the next tile is sent for as
// soon as the scores are done, V as soon as its product is. At a segment's end the waves merge
// in the place of V, with the next segment's first K already under way. A segment that is a
// whole pair is written, a part of one goes to the workspace, and a second launch joins those.
//
// 1024 operations per 1 KiB of K and V: bound by HBM. 64 sequences of 1024-4096 tokens, 8 KV
// heads, 672 MB: 114 us, 5.9 TB/s. One
// sequence of 60001 tokens, 61 MB: 27 us, 16 of them this kernel (3.8 TB/s: 14 tiles a
// workgroup do not hide its start) and 10 the join of 235 parts.
#include "prompt_common.h"

#include <algorithm>

namespace ema {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = kWaves * 64;
constexpr int kIt = 32;                  // tokens of a tile
constexpr int kCh = 256;                 // channels of a pair's values
// Tiles that a segment costs a workgroup beyond its own: its queries, its first tile's way from
// HBM, its merge. (2 / 4 / 8 / 16, us: 64 sequences of 1024-4096 tokens 116 / 114 / 117 / 122,
// 200 of 10-900 tokens 91 / 83 / 83 / 90.)
constexpr int kSegCost = 4;
constexpr int kMaxGrid = 256;
constexpr int kJoinWaves = 16;
constexpr int kJoinBatch = 4;            // parts a wave reads at once

// Records for the join: by pair where there are no more pairs than workgroups (its
// first workgroup, -1: none; its last), so that few pairs take few blocks; else by workgroup
// (the pair that begins there and goes on past it, -1: none; its last workgroup).
__host__ __device__ __forceinline__ bool by_pair(const PromptArgs& a, int grid) {
  return int64_t(a.batch) * (a.kv_heads / 2) <= grid;
}

template <bool BF16>
__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

__device__ __forceinline__ int clamp_len(const PromptArgs& a, int len) {
  return max(0, min(len, a.max_blocks * a.block_size));
}

// A run of tiles [j0, j1) of one (sequence, pair).
struct Segment {
  int b, pair, len, nt, j0, j1;
};

// Writes head `head` of sequence b from the merged maps: this lane's four channels of
// each (unnormalised o1, o2; sums l1, l2). All 64 lanes of a wave call it together.
__device__ __forceinline__ void write_head(const PromptArgs& a, int b, int head, int lane,
                                           f32x4 o1, float l1, f32x4 o2, float l2) {
  const float i1 = l1 == 0.0f ? 0.0f : 1.0f / l1, i2 = l2 == 0.0f ? 0.0f : a.lam[head] / l2;
  f32x4 r = o1 * i1 - o2 * i2;
  if (a.norm_weight) {
    float sq = r[0] * r[0] + r[1] * r[1] + r[2] * r[2] + r[3] * r[3];
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sq += __shfl_xor(sq, o);
    const float inv = sq == 0.0f ? 0.0f : 1.0f / sqrtf(sq / float(kCh) + a.norm_eps);
    const f32x4 w = *reinterpret_cast<const f32x4*>(a.norm_weight + 4 * lane);
    r = r * inv * w;
  }
  AttnArgs st;
  st.out = a.out;
  st.out_dtype = a.out_dtype;
  st.out_vec = 1;
  store_out4(st, (int64_t(b) * (a.q_heads / 2) + head) * kCh + 4 * lane,
             out_f32x4{r[0], r[1], r[2], r[3]});
}

// CT: column tiles (1: both maps in one, 8 columns each; 2: one for each map).
template <int CT, int BSC, bool BF16, int NP>
__global__ __launch_bounds__(kThreads, CT == 1 ? 2 : 1) void diff_kernel(PromptArgs a) {
  constexpr int kCols = CT == 1 ? 16 : 32;           // columns of a partial
  constexpr int kMap2 = kCols / 2;                   // map 2's first column
  // K and V are read once: streamed, except where a tile reads a part of a line whose
  // rest comes with the next tile (block size 64 on).
  constexpr bool kStream = BSC < 64;
  // Fragments of 64 x 16 bytes: V (16 a wave) of all waves, then K. Partials take the place
  // of V or, two column tiles, of both.
  __shared__ __attribute__((aligned(16))) u32x4 s_frag[2][kWaves][16][64];
  __shared__ float s_m[kWaves][kCols], s_l[kWaves][kCols];
  __shared__ int s_sum[kWaves], s_start[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int r16 = lane & 15, q4 = lane >> 4;
  const int B = a.batch, P = a.kv_heads / 2, G = a.q_heads / a.kv_heads;
  const int wg = blockIdx.x, grid = gridDim.x;

  // Units of all sequences before each thread's own ones; empty ones give zeros.
  auto units = [&](int len) {
    const int nt = (len + kIt - 1) / kIt;
    return nt > 0 ? (nt + kSegCost) * P : 0;
  };
  const int per_t = (B + kThreads - 1) / kThreads;
  const int b0 = min(B, tid * per_t), b1 = min(B, b0 + per_t);
  int mine = 0;
  for (int b = b0; b < b1; ++b) {
    const int given = a.seq_lens[b], len = clamp_len(a, given);
    if (wg == 0 && given != len) atomicAdd(a.err_count, 1);
    mine += units(len);
  }
  int incl = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int x = __shfl_up(incl, o);
    if (lane >= o) incl += x;
  }
  if (lane == 63) s_sum[wave] = incl;
  if (tid == 0) s_start[0] = -1;
  __syncthreads();
  int before = incl - mine, U = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += s_sum[w];
    U += s_sum[w];
  }
  const int per = (U + grid - 1) / grid;
  const int u0 = wg * per, u1 = min(U, u0 + per);
  for (int b = b0, at = before; b < b1; ++b) {
    const int n = units(clamp_len(a, a.seq_lens[b]));
    if (u0 >= at && u0 < at + n) {
      s_start[0] = b;
      s_start[1] = u0 - at;
    }
    at += n;
  }
  int32_t* const info = reinterpret_cast<int32_t*>(
      a.ws + int64_t(2) * grid * 2 * G * (kCh + 2));         // [grid][2]
  const bool pairwise = by_pair(a, grid);
  if (!pairwise && tid == 0) info[2 * wg] = -1;
  for (int b = wg; b < B; b += grid)
    if (a.seq_lens[b] <= 0 || a.max_blocks == 0) {
      for (int h = wave; h < a.q_heads / 2; h += kWaves)
        write_head(a, b, h, lane, f32x4{}, 0.0f, f32x4{}, 0.0f);
      if (pairwise && tid < P) info[2 * (b * P + tid)] = -1;
    }
  __syncthreads();
  const int b_first = uniform(s_start[0]);
  if (b_first < 0) return;

  int left = u1 - u0;                    // units of the range not yet handed out
  auto take = [&](Segment& g, int r) {   // from unit r of the pair (its cost first)
    const int cost = max(0, kSegCost - r);
    if (left <= cost) return false;
    left -= cost;
    g.j0 = max(0, r - kSegCost);
    g.j1 = min(g.nt, g.j0 + left);
    left -= g.j1 - g.j0;
    return true;
  };
  auto set_len = [&](Segment& g) {
    g.len = uniform(clamp_len(a, a.seq_lens[g.b]));
    g.nt = (g.len + kIt - 1) / kIt;
  };
  auto next_segment = [&](Segment& g) {
    if (left <= kSegCost) return false;
    if (++g.pair == P) {
      g.pair = 0;
      do {
        if (++g.b >= B) return false;
        set_len(g);
      } while (g.len == 0);
    }
    return take(g, 0);
  };

  const int64_t Bb = a.block_bytes;
  const int BS = a.block_size;
  u32x4 q[CT][4];
  const uint32_t lds_v = lds_address(&s_frag[0][wave][0][0]);
  const uint32_t lds_k = lds_address(&s_frag[1][wave][0][0]);
  f32x4* const part = reinterpret_cast<f32x4*>(&s_frag[0][0][0][0]);
  // Four channels 4f .. 4f + 3 of a wave's partial, its columns off each other's banks.
  auto part_at = [&](int w, int c, int f) -> f32x4& {
    return part[(w * kCols + c) * 64 + (f ^ (c & 15))];
  };
  // Where this wave's tile j of a segment begins: 16-token halves in blocks id[0], id[1]
  // (the same one from block size 32 on).
  struct Place {
    const char* at[2];
    int ok;                              // bit h: the half's block is of the pool
  };
  auto locate = [&](IdWindow& w, const Segment& g, int j) {
    Place p;
    const int t0 = j * kIt;
    w.seek(min(t0 >> a.block_shift, w.last));
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (h == 1 && BSC > 16) {
        p.at[1] = p.at[0];
        continue;
      }
      p.at[h] = a.local + int64_t(w.get(min((t0 >> a.block_shift) + h, w.last))) * Bb;
    }
    p.ok = 3;
    if (w.bad != 0) {
      p.ok = 0;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int tok = t0 + 16 * h;
        if (w.good(tok >> a.block_shift)) p.ok |= 1 << h;
        else if (g.pair == 0 && lane == 0 && tok < g.len && (tok & (BS - 1)) == 0)
          atomicAdd(a.err_count, 1);     // the tile that the block begins in
      }
    }
    return p;
  };
  // K rows: subtile t, row r16 -> token t0 + 8 * (r16 / 4) + 4t + r16 % 4 (every lane ends
  // up with the scores of 8 consecutive tokens of its column). Rows past the length
  // re-read the tile's first ones and are masked.
  auto load_k = [&](const Segment& g, const Place& p, int j) {
    const int t0 = j * kIt, n = g.len - t0;
    const int tb = BSC > 16 ? t0 & (BS - 1) : 0;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int tok = 8 * (r16 >> 2) + 4 * t + (r16 & 3);
      const int row = tok < n ? tok : 0;
      const char* base = row >= 16 ? p.at[1] : p.at[0];
      const int in = BSC == 16 ? row & 15 : tb + row;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const char* s = base + (((2 * g.pair + x) * BS + in) * 128 + q4 * 8) * 2;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
          load_lane_to_lds<kStream>(s + kk * 64, lds_k + ((x * 2 + t) * 4 + kk) * 1024);
      }
    }
  };
  // V^T rows: channel tile n, row 16n + r16, tokens t0 + 8 q4 .. + 8.
  auto load_v = [&](const Segment& g, const Place& p, int j) {
    const int t0 = j * kIt, n = g.len - t0;
    const int tb = BSC > 16 ? t0 & (BS - 1) : 0;
    const int tok = 8 * q4 < n ? 8 * q4 : 0;
    const char* base = tok >= 16 ? p.at[1] : p.at[0];
    const int in = BSC == 16 ? tok & 15 : tb + tok;
    const char* s = base + Bb / 2 + ((int64_t(2 * g.pair) * 128 + r16) * BS + in) * 2;
#pragma unroll
    for (int c = 0; c < 16; ++c) load_lane_to_lds<kStream>(s + c * 32 * BS, lds_v + c * 1024);
  };
  // Q^T as the B operand: lane (column r16, q4) holds channels 32 kk + 8 q4 .. + 8.
  auto load_q = [&](const Segment& g) {
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      const int map = CT == 1 ? r16 >> 3 : ct, head = CT == 1 ? r16 & 7 : r16;
      const bool on = head < G;
      const char* p = a.q + (int64_t(g.b) * a.q_stride +
                             (2 * (g.pair * G + (on ? head : 0)) + map) * 128 + q4 * 8) * 2;
#pragma unroll
      for (int kk = 0; kk < 4; ++kk) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(p + kk * 64);
        q[ct][kk] = on ? x : u32x4{0, 0, 0, 0};
      }
    }
  };

  f32x4 o[CT][16];
  float m[CT], l[CT];
  auto clear = [&] {
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      m[ct] = -INFINITY;
      l[ct] = 0.0f;
#pragma unroll
      for (int c = 0; c < 16; ++c) o[ct][c] = f32x4{};
    }
  };

  Segment g;
  g.b = b_first;
  set_len(g);
  const int into = uniform(s_start[1]);
  g.pair = into / (g.nt + kSegCost);
  bool have = take(g, into - g.pair * (g.nt + kSegCost));
  if (!have) have = next_segment(g);
  IdWindow win;
  Place at;
  auto open = [&](const Segment& s) {
    if (s.j0 + wave >= s.j1) return;
    win.open(a, s.b, ((s.j0 + wave) * kIt) >> a.block_shift, (s.len - 1) >> a.block_shift);
    at = locate(win, s, s.j0 + wave);
    load_k(s, at, s.j0 + wave);
  };
  auto open_v = [&](const Segment& s) {
    if (s.j0 + wave < s.j1) load_v(s, at, s.j0 + wave);
  };
  if (have) {
    load_q(g);
    open(g);
    open_v(g);
  }
  while (have) {
    clear();
    for (int j = g.j0 + wave; j < g.j1; j += kWaves) {
      const Place here = at;
      const bool more = j + kWaves < g.j1;
      // scores of tokens 8 q4 + 4t + i of column r16
      u32x4 k[2][2][4];
      loads_arrived_but_16();            // V of this tile is still on its way
#pragma unroll
      for (int x = 0; x < 16; ++x) k[x >> 3][(x >> 2) & 1][x & 3] = s_frag[1][wave][x][lane];
      f32x4 s[CT][2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if constexpr (CT == 1) {
          // each map's keys by all columns, of which the other map's are not looked at: with
          // zeros there for a query an infinite key would reach them as NaN
          f32x4 x = f32x4{}, y = f32x4{};
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) {
            x = mfma16<BF16>(k[0][t][kk], q[0][kk], x);
            y = mfma16<BF16>(k[1][t][kk], q[0][kk], y);
          }
          s[0][t] = r16 < 8 ? x : y;
        } else {
#pragma unroll
          for (int ct = 0; ct < 2; ++ct) {
            s[ct][t] = f32x4{};
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
              s[ct][t] = mfma16<BF16>(k[ct][t][kk], q[ct][kk], s[ct][t]);
          }
        }
      }
      reads_done();
      if (more) {
        at = locate(win, g, j + kWaves);
        load_k(g, at, j + kWaves);
      }
      const int n = g.len - j * kIt - 8 * q4;        // valid tokens of this lane's 8
      const int nv = (here.ok >> (q4 >> 1)) & 1 ? n : 0;
      u32x4 p[CT][NP];
      float alpha[CT];
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        float sv[8], mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          sv[i] = i < nv ? s[ct][i >> 2][i & 3] * a.scale_log2 : -INFINITY;
          mx = fmaxf(mx, sv[i]);
        }
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float m_new = fmaxf(m[ct], mx);
        const float ref = m_new == -INFINITY ? 0.0f : m_new;
        alpha[ct] = __builtin_amdgcn_exp2f(m[ct] - ref);
        m[ct] = m_new;
        const float low = BF16 ? ref : ref - 15.0f;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float x = __builtin_amdgcn_exp2f(sv[2 * i] - low);
          float y = __builtin_amdgcn_exp2f(sv[2 * i + 1] - low);
          sum += x + y;
#pragma unroll
          for (int r = 0; r < NP; ++r) {
            const uint32_t w = pack16<BF16>(x, y);
            p[ct][r][i] = w;
            x -= low16<BF16>(w);
            y -= high16<BF16>(w);
          }
        }
        l[ct] = fmaf(l[ct], alpha[ct], sum);
      }
      u32x4 keep;                        // what is masked may hold NaN
#pragma unroll
      for (int i = 0; i < 4; ++i)
        keep[i] = (2 * i < nv ? 0xffffu : 0u) | (2 * i + 1 < nv ? 0xffff0000u : 0u);
      if (more) loads_arrived_but_16();  // the next tile's K is still on its way
      else loads_arrived();
      // A tile's sum from zero, then added: the matrix cores round at what they add to.
#pragma unroll
      for (int c = 0; c < 16; ++c) {
        const u32x4 v = s_frag[0][wave][c][lane] & keep;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          f32x4 t = f32x4{};
#pragma unroll
          for (int r = NP - 1; r >= 0; --r) t = mfma16<BF16>(v, p[ct][r], t);
          o[ct][c] = o[ct][c] * alpha[ct] + t;
        }
      }
      reads_done();
      if (more) load_v(g, at, j + kWaves);
    }
    // merge the four waves
    __syncthreads();                     // all are done with their operands
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      const int colx = ct * 16 + r16;
      float sum = l[ct];
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      if (q4 == 0) {
        s_m[wave][colx] = m[ct];
        s_l[wave][colx] = sum;
      }
#pragma unroll
      for (int c = 0; c < 16; ++c)
        part_at(wave, colx, 4 * c + q4) = o[ct][c];
    }
    const Segment done = g;
    have = next_segment(g);
    if (have) {
      load_q(g);
      if (CT == 1) open(g);
    }
    __syncthreads();
    const bool begins = done.j0 == 0, ends = done.j1 == done.nt;
    const int slot = 2 * wg + (begins ? 1 : 0);
    for (int h = wave; h < G; h += kWaves) {
      f32x4 O[2];
      float M[2], L[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int c = x * kMap2 + h;
        M[x] = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) M[x] = fmaxf(M[x], s_m[w][c]);
        const float ref = M[x] == -INFINITY ? 0.0f : M[x];
        L[x] = 0.0f;
        O[x] = f32x4{};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          const float f = __builtin_amdgcn_exp2f(s_m[w][c] - ref);
          L[x] = fmaf(f, s_l[w][c], L[x]);
          O[x] += part_at(w, c, lane) * f;
        }
      }
      if (begins && ends) {
        write_head(a, done.b, done.pair * G + h, lane, O[0], L[0], O[1], L[1]);
        continue;
      }
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int64_t row = (int64_t(slot) * 2 + x) * G + h;
        *reinterpret_cast<f32x4*>(a.ws + row * kCh + 4 * lane) = O[x];
        if (lane == 0) {
          float* ml = a.ws + int64_t(2) * grid * 2 * G * kCh + row * 2;
          ml[0] = M[x];
          ml[1] = L[x];
        }
      }
    }
    if (begins && tid == 0) {
      const int pair = done.b * P + done.pair;
      // a part: the range ends with this segment
      const int last = (u1 + (done.nt - done.j1) - 1) / per;
      if (pairwise) {
        info[2 * pair] = ends ? -1 : wg;
        info[2 * pair + 1] = last;
      } else if (!ends) {
        info[2 * wg] = pair;
        info[2 * wg + 1] = last;
      }
    }
    __syncthreads();
    if (have) {
      if (CT == 2) open(g);
      open_v(g);
    }
  }
}

// Joins the parts of a pair: a block for (record, head), whose waves share out the parts,
// kJoinBatch of them in a round trip; the first wave joins the waves'. (One document of 60001
// tokens leaves 235 parts: with four waves the call took 44.7 us, with
// sixteen 27.0; eight parts in a round trip: 27.5.)
__global__ __launch_bounds__(kJoinWaves * 64) void diff_join(PromptArgs a, int grid, bool pairwise) {
  __shared__ __attribute__((aligned(16))) f32x4 s_o[kJoinWaves][2][64];
  __shared__ float s_ml[kJoinWaves][2][2];
  const int h = blockIdx.y, lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int G = a.q_heads / a.kv_heads, P = a.kv_heads / 2;
  const int32_t* info = reinterpret_cast<const int32_t*>(
      a.ws + int64_t(2) * grid * 2 * G * (kCh + 2));
  const int rec = info[2 * blockIdx.x], last = info[2 * blockIdx.x + 1];
  if (rec < 0) return;
  const int w0 = pairwise ? rec : int(blockIdx.x), pair = pairwise ? int(blockIdx.x) : rec;
  const float* mls = a.ws + int64_t(2) * grid * 2 * G * kCh;
  const int n = last - w0 + 1, waves = blockDim.x >> 6;
  float M[2] = {-INFINITY, -INFINITY}, L[2] = {0.0f, 0.0f};
  f32x4 O[2] = {f32x4{}, f32x4{}};
  for (int i0 = wave; i0 < n; i0 += kJoinBatch * waves) {
    f32x4 po[kJoinBatch][2];
    float pm[kJoinBatch][2], pl[kJoinBatch][2];
#pragma unroll
    for (int y = 0; y < kJoinBatch; ++y) {
      const int i = min(i0 + y * waves, n - 1);
      const int slot = i == 0 ? 2 * w0 + 1 : 2 * (w0 + i);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int64_t row = (int64_t(slot) * 2 + x) * G + h;
        po[y][x] = *reinterpret_cast<const f32x4*>(a.ws + row * kCh + 4 * lane);
        pm[y][x] = mls[row * 2];
        pl[y][x] = mls[row * 2 + 1];
      }
    }
#pragma unroll
    for (int y = 0; y < kJoinBatch; ++y) {
      if (i0 + y * waves >= n) break;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const float M_new = fmaxf(M[x], pm[y][x]);
        const float ref = M_new == -INFINITY ? 0.0f : M_new;
        const float f = __builtin_amdgcn_exp2f(M[x] - ref), e = __builtin_amdgcn_exp2f(pm[y][x] - ref);
        M[x] = M_new;
        L[x] = L[x] * f + pl[y][x] * e;
        O[x] = O[x] * f + po[y][x] * e;
      }
    }
  }
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    s_o[wave][x][lane] = O[x];
    if (lane == 0) {
      s_ml[wave][x][0] = M[x];
      s_ml[wave][x][1] = L[x];
    }
  }
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    float top = -INFINITY;
#pragma unroll 4
    for (int w = 0; w < waves; ++w) top = fmaxf(top, s_ml[w][x][0]);
    const float ref = top == -INFINITY ? 0.0f : top;
    L[x] = 0.0f;
    O[x] = f32x4{};
#pragma unroll 4
    for (int w = 0; w < waves; ++w) {
      const float f = __builtin_amdgcn_exp2f(s_ml[w][x][0] - ref);
      L[x] = fmaf(f, s_ml[w][x][1], L[x]);
      O[x] += s_o[w][x][lane] * f;
    }
  }
  const int b = pair / P;
  write_head(a, b, (pair - b * P) * G + h, lane, O[0], L[0], O[1], L[1]);
}

template <int CT, int BSC, bool BF16, int NP>
void launch_kernel(const PromptArgs& a, int grid, hipStream_t stream) {
  hipLaunchKernelGGL((diff_kernel<CT, BSC, BF16, NP>), dim3(grid), dim3(kThreads), 0, stream, a);
}

template <int CT, bool BF16, int NP>
void launch_sizes(const PromptArgs& a, int grid, hipStream_t stream) {
  if (a.block_size == 16) launch_kernel<CT, 16, BF16, NP>(a, grid, stream);
  else if (a.block_size == 32) launch_kernel<CT, 32, BF16, NP>(a, grid, stream);
  else launch_kernel<CT, 64, BF16, NP>(a, grid, stream);
}

template <int CT>
void launch_types(const PromptArgs& a, int grid, hipStream_t stream) {
  if (a.dtype == 0) launch_sizes<CT, false, 2>(a, grid, stream);
  else if (a.full) launch_sizes<CT, true, 3>(a, grid, stream);
  else launch_sizes<CT, true, 2>(a, grid, stream);
}

// Workgroups: one to a CU, and no more than there can be tiles.
int grid_of(const PromptArgs& a) {
  const int64_t tiles = int64_t(a.batch) * (a.kv_heads / 2) *
                        ((int64_t(a.max_blocks) * a.block_size + kIt - 1) / kIt);
  return int(std::max<int64_t>(1, std::min<int64_t>(kMaxGrid, tiles)));
}

}  // namespace

size_t diff_workspace(const PromptArgs& a) {
  const size_t G = a.q_heads / a.kv_heads, grid = grid_of(a);
  return 2 * grid * 2 * G * (kCh + 2) * 4 + grid * 8;
}

hipError_t launch_diff_attention(const PromptArgs& a, hipStream_t stream) {
  if (a.tokens <= 0) return hipSuccess;
  const int grid = grid_of(a);
  if (a.q_heads / a.kv_heads <= 8) launch_types<1>(a, grid, stream);
  else launch_types<2>(a, grid, stream);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const bool pairwise = by_pair(a, grid);
  const int records = pairwise ? a.batch * (a.kv_heads / 2) : grid;
  const int waves = std::max(4, std::min(kJoinWaves, grid / records));   // as parts to a record
  hipLaunchKernelGGL(diff_join, dim3(records, a.q_heads / a.kv_heads), dim3(waves * 64), 0, stream,
                     a, grid, pairwise);
  return hipGetLastError();
}

}  // namespace ema
