// Attention of drafted trees over the paged cache, on the matrix cores.
//
// The G query heads that share a KV head are rows beside each other: row r of a
// request's n nodes is (node r / G, head r % G). 64, 128 or 256 rows (an item) go past the
// request's tokens in tiles of 64 staged in LDS, 32 rows to a wave:
//   scores   S^T[token][row] = K . Q^T     v_mfma_f32_32x32x16, A = 32 K rows, B = Q^T
//            in registers; the rows of A are taken in an order that leaves every
//            lane with 8 consecutive tokens of one row twice over
//   softmax  online, in the log2 domain: every lane has 32 of its row's 64 scores
//            and the lane 32 away the others
//   output   O^T[channel][row] += V^T . P^T   A = 32 channels of the transposed V
//            block, B = P as the scores left it: nothing moves between lanes
// Weights, their scale in f16 and the slack of the rescaling are those of the prompt
// kernels (put_weights; below 2^8, with two f16 parts 2^4).
//
// What bounds it goes by the rows. 4 * 128 operations per (row, token): a KV head's token, 512
// bytes, takes as long from HBM as some 200 rows' products. So an item has all rows of a tree,
// up to 256 (a second tile of rows reads K and V again: 18 nodes of 4 heads behind 64 contexts take
// 147 us as one item of 128 rows, 259 as two of 64), and as many workgroups run on a CU as their
// tiles leave room for: two with 64 KiB of tiles each up to 128 rows, bound by HBM; one of two groups
// of waves in turns with 256, bound by the matrix cores and HBM together. 64 trees of 16 nodes behind
// 1024-4080 tokens (32 and 8 heads, bf16, 690 MB): 131 us, 5.3 TB/s; its loads alone take 128, its
// products and softmax alone 70. 32 trees of 64 nodes behind 3000: 136 us, 740 TFLOP/s at 3.2 TB/s;
// loads alone 83, products and softmax alone 100, and what keeps them from overlapping better is
// not known (a place more, later waits: the same).
//
// Weights of 32-bit accuracy do not fit beside outputs and scores: in three parts (bf16) every form
// spills, 12 to 120 bytes a lane, in two (f16) four of nine, up to 52; in one part none does. The
// 64 trees of 16 nodes with 32-bit outputs: 170 us (f16 158), of 64 nodes 356 for 255.
//
// Work: all items' tiles in a row, cut into equal shares, one a workgroup; items that several
// share are joined by a second launch. Where whole items leave no workgroup with much more than
// that, they stay whole: parts cost their rows' way to the workspace and back (64 trees of 16
// nodes: 152 us shared, 136 whole). Work is cut by lengths, not by the
// table's width, but for tables of at most 512 tokens, whose items all stay whole.
//
// Only tiles that reach past the older tokens look at the mask: 64 bits of it, those of
// the tile's tokens, are shifted into place from two words of the row's. There V is
// cleaned of what is not finite, since 0 times it would be NaN for rows that do not attend
// it; where something was, the rows are looked at again at the end, value by value, and those
// that do attend one get NaN in its channel.
//
// What did not help: 64 rows to a wave, one wave to a SIMD (half the LDS reads, but the registers
// spill: 405 us for 254); 32-row items of four waves with a tile each (1 node 119 us for 124, but 8
// nodes 131 for 126 and 4 nodes behind 200 contexts 163 for 145); ends of shares moved to the near
// ends of items (152 for 150); eight waves or four workgroups on a CU for 64 rows (142, 150 for 135).
#include "prompt_common.h"
#include "tree_kernels.h"

#include <algorithm>

namespace ema {
namespace {

// Loads a tile of K or V into LDS, in the places of prompt_common.h. Its 16 pieces of 1 KiB are
// shared out to RW waves; a lane's part of an address is the same for all of them but for the four
// (K) or two (V) ways in which their 16-byte parts are turned, the rest is the wave's.
template <int BSC, int RW>
struct TileLoader {
  static constexpr int kPieces = 16 / RW;
  struct Blocks {
    const char* at[4];                     // the blocks of the tile's 16-token groups
  };
  const char* local;
  int64_t block_bytes, v_at;               // v_at: the head's V in a block
  int shift, mask, last, k_at, row_bytes;
  uint32_t k_lane[4], v_lane[2];
  IdWindow window;

  // Once: what does not depend on the segment. rw: the wave's number among those of a tile.
  __device__ __forceinline__ void init(const PromptArgs& a, int rw) {
    const int lane = threadIdx.x & 63, l16 = lane >> 4;
    local = a.local;
    block_bytes = a.block_bytes;
    shift = a.block_shift;
    mask = a.block_size - 1;
    row_bytes = a.block_size * 2;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = ((rw * kPieces + i) & 3) * 4 + l16;
      k_lane[i] = row * 256 + ((lane ^ row) & 15) * 16;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      constexpr int r = BSC / 8;           // pieces of a channel's row
      const int turn = BSC == 64 ? i * 4 + l16 : BSC == 32 ? l16 : l16 & 1;
      v_lane[i] = lane / r * row_bytes + ((lane % r) ^ turn) * 16;
    }
  }
  __device__ __forceinline__ void open(const PromptArgs& a, int b, int kvh, int j, int end) {
    last = (end - 1) >> shift;
    k_at = kvh * 256 * a.block_size;
    v_at = block_bytes / 2 + k_at;
    window.open(a, b, (j * kKT) >> shift, last);
  }
  // Where tile j's tokens are; tiles in ascending order.
  __device__ __forceinline__ Blocks blocks(int j) {
    Blocks t;
    const int first = (j * kKT) >> shift;
    window.seek(min(first, last));
#pragma unroll
    for (int i = 0; i < 4; ++i)
      t.at[i] = local + int64_t(window.get(min(first + i * 16 / BSC, last))) * block_bytes;
    return t;
  }
  __device__ __forceinline__ void load_k(uint32_t to, int j, const Blocks& t, int rw) const {
    const int in = k_at + (BSC == 64 ? ((j * kKT) & mask) * 256 : 0);
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int x = rw * kPieces + i, row = (x >> 2) * 16 & (BSC - 1);
      load_to_lds<true>(pick(t, x >> 2) + in + row * 256, k_lane[i & 3], to + x * 1024);
    }
  }
  __device__ __forceinline__ void load_v(uint32_t to, int j, const Blocks& t, int rw) const {
    const int64_t in = v_at + (BSC == 64 ? ((j * kKT) & mask) * 2 : 0);
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int x = rw * kPieces + i;
      constexpr int per = BSC / 4;         // pieces of a block: 4, 8 or 16
      const int group = x / per * (BSC / 16);
      load_to_lds<true>(pick(t, group) + in + int64_t(x % per * (64 / (BSC / 8))) * row_bytes,
                  v_lane[BSC == 64 ? i & 1 : 0], to + x * 1024);
    }
  }
  // (selected, not indexed: the array stays in registers)
  static __device__ __forceinline__ const char* pick(const Blocks& t, int i) {
    const char* lo = i & 1 ? t.at[1] : t.at[0];
    const char* hi = i & 1 ? t.at[3] : t.at[2];
    return i & 2 ? hi : lo;
  }
  // Which tokens of tile j are of blocks of the pool and before token `end`.
  __device__ __forceinline__ uint64_t there(int j, int end) const {
    const int t0 = j * kKT, n = end - t0;
    uint64_t x = n < 64 ? (1ull << n) - 1ull : ~0ull;
    if (window.bad != 0)
#pragma unroll
      for (int i = 0; i < 4; ++i)          // 16 tokens, in one block
        if (!window.good((t0 + 16 * i) >> shift)) x &= ~(0xffffull << (16 * i));
    return x;
  }
  // In the pieces of V tile j that this lane has loaded: what is not `there` becomes 0, and so
  // does what is not finite; whether there was any of that.
  template <bool BF16>
  __device__ __forceinline__ bool clean_v(u32x4* tile, uint64_t there, int rw) const {
    constexpr uint32_t kExp = BF16 ? 0x7f80u : 0x7c00u;
    constexpr int r = BSC / 8, per = BSC / 4;
    const int lane = threadIdx.x & 63, l16 = lane >> 4;
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int x = rw * kPieces + i;
      const int turn = BSC == 64 ? (i & 1) * 4 + l16 : BSC == 32 ? l16 : l16 & 1;
      const uint32_t bits = uint32_t(there >> (x / per * BSC + ((lane % r) ^ turn) * 8));
      u32x4 v = tile[x * 64 + lane];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        v[k] &= (bits >> (2 * k) & 1 ? 0xffffu : 0u) | (bits >> (2 * k + 1) & 1 ? 0xffff0000u : 0u);
        const uint32_t drop = ((v[k] & kExp) == kExp ? 0xffffu : 0u) |
                              ((v[k] >> 16 & kExp) == kExp ? 0xffff0000u : 0u);
        any |= drop;
        v[k] &= ~drop;
      }
      tile[x * 64 + lane] = v;
    }
    return any != 0;
  }
  // Counts the entries of tile j whose block begins there, before token `end`, and is not of the
  // pool; one wave of those that see a sequence's tiles does. (window.bad takes whole windows, of
  // which a part of the tiles holds some only.)
  __device__ __forceinline__ void count_bad(const PromptArgs& a, int j, int end) const {
    const int lane = threadIdx.x & 63, tok = j * kKT + lane * 16;
    const bool bad = lane < kKT / 16 && tok < end && (tok & mask) == 0 && !window.good(tok >> shift);
    const int n = __popcll(__ballot(bad));
    if (n > 0 && lane == 0) atomicAdd(a.err_count, n);
  }
};

// Tiles that a segment costs a workgroup beyond its own: its queries, its first tiles' way from
// HBM, its merge. (8: within 2 % of 4 on eleven sizes.)
constexpr int kSegCost = 4;
constexpr int kCus = 256;
constexpr int kWholeTiles = 8;           // tables of at most so many tiles: items are not shared, and
                                         // there is no second launch
constexpr int kRecord = 6;               // ints: see Record
constexpr int kJoinRows = 8;
constexpr int kJoinGrid = 4096;          // workgroups of the join that run at once

// Inclusive prefix sum over the wave's 64 lanes, by DPP moves: within rows of 16 lanes, then
// the row totals carried over.
__device__ __forceinline__ int wave_inclusive_sum(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);    // row_shr 1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // lane 15 of rows 0, 2 to 1, 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // lane 31 to rows 2, 3
  return x;
}

// An item: a row tile of one (request, KV head). What the join needs of one that several
// workgroups share.
struct Record {
  int from, to;                          // its first workgroup (-1: not shared), its last one
  int row0, rows, first, kvh;            // the request's first row, its rows, the tile's first
};

// How a call is cut: by its sizes alone.
struct Cut {
  int64_t bound;                         // items at most
  int rows;                              // of an item
  int grid;
  int whole;                             // an item to a workgroup; else equal shares of all tiles
  int least;                             // units of a share at least: parts of few tiles cost more
                                         // than they save
  int uneven;                            // ... or whole items, where no workgroup has more than
                                         // this many quarters of such a share
};

// Records are kept by item where there are no more of them than that, else by the workgroup in
// which an item begins.
__host__ __device__ __forceinline__ bool by_item(const Cut& c) { return c.bound <= 2 * c.grid; }

// A run of tiles [j0, j1) of one item.
struct Segment {
  int b, row0, n, len, nt;               // the request, its rows in q, its tokens
  int item, items;                       // of the request's
  int index;                             // of all items
  int j0, j1;
};

// The shapes of a workgroup: RW waves share a tile, 32 rows each, and kWaves / RW groups of such
// waves take a segment's tiles in turn, each with kPlaces places of its own for tiles.
template <int ROWS>
struct Shape;
template <>
struct Shape<64> { static constexpr int kWaves = 4, kPlaces = 1, kPerCu = 2; };
template <>
struct Shape<128> { static constexpr int kWaves = 4, kPlaces = 2, kPerCu = 2; };
template <>
struct Shape<256> { static constexpr int kWaves = 8, kPlaces = 4, kPerCu = 1; };

template <bool BF16, int BSC, int NP, int ROWS>
__global__ __launch_bounds__(Shape<ROWS>::kWaves * 64, 2) void tree_kernel(TreeAttnArgs a, Cut cut) {
  constexpr int kWaves = Shape<ROWS>::kWaves, kThreads = kWaves * 64, kPlaces = Shape<ROWS>::kPlaces;
  constexpr int RW = ROWS / 32, kGroups = kWaves / RW, kRows = ROWS;
  // The groups' K and V tiles; at a segment's end 16 KiB of each wave's outputs
  static_assert(kGroups * kPlaces * 2 >= kWaves, "the outputs take the tiles' place");
  __shared__ __attribute__((aligned(16))) u32x4 s_kv[kGroups * kPlaces][2][kTilePieces];
  __shared__ float s_m[kWaves][32], s_l[kWaves][32];
  __shared__ int s_sum[kWaves][2], s_most[kWaves], s_flags[kWaves], s_row[ROWS];
  __shared__ int s_start[6], s_odd[2];       // s_odd: 1 values that are not finite, 2 bad blocks
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int rw = wave % RW, group = wave / RW;
  const int col = lane & 31, half = lane >> 5;
  const int B = a.batch, G = a.q_heads / a.kv_heads, H = a.kv_heads;
  // Workgroups go round the eight XCDs: an XCD's take items that follow each other.
  const int grid = gridDim.x, id = blockIdx.x;
  const int wg = grid % 8 == 0 ? id % 8 * (grid / 8) + id / 8 : id;
  const bool itemwise = by_item(cut);
  float* const ws_ml = a.ws + int64_t(2) * grid * kRows * 128;
  int32_t* const info = reinterpret_cast<int32_t*>(ws_ml + int64_t(2) * grid * kRows * 2);

  // ---- the workgroup's range: equal shares of all items' tiles ---------------------------
  auto clamp_len = [&](int len) { return max(0, min(len, a.max_blocks * a.block_size)); };
  auto items_of = [&](int n, int len) { return len > 0 ? (n * G + kRows - 1) / kRows * H : 0; };
  auto units_of = [&](int n, int len) {
    return items_of(n, len) * ((len + kKT - 1) / kKT + kSegCost);
  };
  const int per_t = (B + kThreads - 1) / kThreads;
  const int b0 = min(B, tid * per_t), b1 = min(B, b0 + per_t);
  int units = 0, items = 0, most = 0;        // most: units of an item
  float roughly = 0.0f;                      // the units
  int row0 = 0, n = 0, len = 0;              // of the thread's last request; mostly its only one
  bool wrong = false, empty = false;         // bad starts; a request without tokens
  for (int b = b0; b < b1; ++b) {
    const int bad = row_range(a, b, row0, n), given = a.seq_lens[b];
    len = clamp_len(given);
    if (wg == 0 && bad > 0) atomicAdd(a.err_count, 1);
    if (wg == 0 && n > 0 && (len < n || len != given)) atomicAdd(a.err_count, 1);
    const int x = units_of(n, len);
    units = int(uint32_t(units) + uint32_t(x));
    roughly += float(x);
    items += items_of(n, len);
    wrong |= bad > 0;
    empty |= n > 0 && len == 0;
    if (n > 0 && len > 0) most = max(most, (len + kKT - 1) / kKT + kSegCost);
  }
  int incl[2] = {wave_inclusive_sum(units), wave_inclusive_sum(items)};
  most = wave_max(most);
  if (lane == 63) {
    s_sum[wave][0] = incl[0];
    s_sum[wave][1] = incl[1];
    s_most[wave] = most;
  }
  const int flags = (__ballot(wrong) ? 1 : 0) | (__ballot(empty) ? 2 : 0);
  if (lane == 0) s_flags[wave] = flags;
  if (tid == 0) {
    s_start[0] = -1;
    s_odd[0] = s_odd[1] = 0;
  }
  __syncthreads();
  int before = incl[0] - units, index = incl[1] - items, U = 0, all_items = 0, flagged = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) {
      before += s_sum[w][0];
      index += s_sum[w][1];
    }
    U += s_sum[w][0];
    all_items += s_sum[w][1];
    most = max(most, s_most[w]);
    flagged |= s_flags[w];
  }
  if (flagged & 1) {                         // requests of many rows in common, by bad starts
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) roughly += __shfl_xor(roughly, x);
    __syncthreads();
    if (lane == 0) s_m[wave][0] = roughly;
    __syncthreads();
    float total = 0.0f;
    for (int w = 0; w < kWaves; ++w) total += s_m[w][0];
    if (total > 1.5f * (1 << 30)) {
      if (!cut.whole && wg == 0 && tid == 0) info[0] = 0;
      return;
    }
  }
  const int share = max((U - 1) / grid + 1, cut.least), rounds = (all_items + grid - 1) / grid;
  const bool whole = cut.whole || int64_t(rounds) * most * 4 <= int64_t(share) * (rounds == 1 ? cut.uneven : 5);
  const int per = whole ? rounds : share, all = whole ? all_items : U;
  // (a range may begin past the last unit: compared without adding to it)
  const int u0 = int(min(int64_t(wg) * per, int64_t(all))), u1 = u0 + min(per, all - u0);
  if (whole) before = index;
  for (int b = b0; b < b1; ++b) {
    if (per_t > 1) {
      row_range(a, b, row0, n);
      len = clamp_len(a.seq_lens[b]);
    }
    const int x = whole ? items_of(n, len) : units_of(n, len);
    if (u0 >= before && u0 - before < x) {
      s_start[0] = b;
      s_start[1] = index;
      s_start[2] = row0;
      s_start[3] = n;
      s_start[4] = len;
      s_start[5] = u0 - before;
    }
    before += x;
    index += items_of(n, len);
  }
  if (!cut.whole && wg == 0 && tid == 0) info[0] = whole ? 0 : itemwise ? int(min(int64_t(all_items), cut.bound)) : grid;
  if (!cut.whole && !itemwise && tid == 0) info[1 + wg * kRecord] = -1;
  for (int b = wg; flagged & 2 && b < B; b += grid) {      // requests without tokens
    if (a.seq_lens[b] > 0 && a.max_blocks > 0) continue;
    int s, n;
    row_range(a, b, s, n);
    AttnArgs out;
    out.out = a.out;
    out.out_dtype = a.out_dtype;
    out.out_vec = 1;
    for (int64_t x = tid; x < int64_t(n) * a.q_heads * 32; x += kThreads)
      store_out4(out, int64_t(s) * a.q_heads * 128 + 4 * x, out_f32x4{});
  }
  __syncthreads();
  if (uniform(s_start[0]) < 0) return;

  int left = u1 - u0;                        // units (whole: items) not yet handed out
  auto take = [&](Segment& g, int r) {       // from unit r of the item (its cost first)
    if (whole) {
      g.j0 = 0;
      g.j1 = g.nt;
      return left-- > 0;
    }
    const int cost = max(0, kSegCost - r);
    if (left <= cost) return false;
    left -= cost;
    g.j0 = max(0, r - kSegCost);
    g.j1 = min(g.nt, g.j0 + left);
    left -= g.j1 - g.j0;
    return true;
  };
  auto set_request = [&](Segment& g, int s, int n, int len) {
    g.row0 = uniform(s);
    g.n = uniform(n);
    g.len = uniform(len);
    g.nt = (g.len + kKT - 1) / kKT;
    g.items = items_of(g.n, g.len);
  };
  auto next_segment = [&](Segment& g) {
    if (left <= (whole ? 0 : kSegCost)) return false;
    ++g.index;
    if (++g.item == g.items) {
      g.item = 0;
      do {
        if (++g.b >= B) return false;
        int s, n;
        row_range(a, g.b, s, n);
        set_request(g, s, n, clamp_len(a.seq_lens[g.b]));
      } while (g.items == 0);
    }
    return take(g, 0);
  };

  // ---- a segment's rows and tiles ----------------------------------------------------------
  int kvh = 0, first = 0, base = 0;          // of segment g; base: tokens before the nodes
  bool alive = false;                        // the wave has rows
  int tok = -1, out_row = -1;                // the node of this lane's row, its row of out; -1: none
  const uint64_t inverse = (1ull << 32) / G + 1;         // x * inverse >> 32 = x / G for x < 2^16
  u32x4 q[8];
  TileLoader<BSC, RW> st;
  typename TileLoader<BSC, RW>::Blocks at;
  st.init(a, rw);
  auto load_q = [&](const Segment& g) {
    const int tiles = g.items / H;
    kvh = g.item / tiles;
    first = (g.item - kvh * tiles) * kRows;
    base = g.len - g.n;
    const int r = first + rw * 32 + col, node0 = first / G, x = first - node0 * G + rw * 32 + col;
    const bool live = r < g.n * G;
    const int node = live ? node0 + int(x * inverse >> 32) : 0, h = live ? r - node * G : 0;
    // (with 128 rows the branches cost more than the idle waves' products: 32 nodes of 4 heads behind
    // 64 contexts 164 us for 155)
    alive = ROWS == 128 || first + rw * 32 < g.n * G;
    tok = live ? node : -1;
    out_row = live ? (g.row0 + node) * a.q_heads + kvh * G + h : -1;
    const char* p = a.q + (int64_t(g.row0 + node) * a.q_stride + (kvh * G + h) * 128 + half * 8) * 2;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) q[ks] = *reinterpret_cast<const u32x4*>(p + ks * 32);
  };

  // Which tokens from t0 on a node attends, a bit each, but for those that are not there.
  auto attended = [&](const Segment& g, int node, int t0) -> uint64_t {
    const int before = g.len - g.n, j = t0 - before;   // j: the node at the first of them
    if (node < 0 || before + node < 0) return 0;
    if (j <= -64) return ~0ull;
    const uint64_t* words = a.mask + int64_t(g.row0 + node) * a.words;
    if (j < 0) return (words[0] << -j) | ((1ull << -j) - 1ull);
    const int w = j >> 6, by = j & 63;
    uint64_t x = w < a.words ? words[w] >> by : 0;
    if (by > 0 && w + 1 < a.words) x |= words[w + 1] << (64 - by);
    return x;
  };

  // ---- a tile ------------------------------------------------------------------------------
  f32x16 o[4], s[2];
  float m, l;                                // l: this lane's half of the tokens
  Weights<NP> w;
  bool odd = false;                          // V that is not finite in tiles that are masked in part
  const int arow = score_row(col);
  constexpr float kSlack = BF16 || NP == 1 ? 8.0f : 4.0f, kUp = BF16 ? 0.0f : 15.0f - kSlack;
  auto scores = [&](const u32x4* K) {
#pragma unroll
    for (int ks = 0; ks < 8; ++ks)
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
        s[tt] = mfma32<BF16>(K[k_place(tt * 32 + arow, ks * 2 + half)], q[ks],
                             ks == 0 ? f32x16{} : s[tt]);
  };
  auto hide = [&](const Segment& g, int j, uint64_t there) {
    const uint64_t sees = attended(g, tok, j * kKT) & there;
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      const uint32_t bits = uint32_t(sees >> (tt * 32 + half * 8));
#pragma unroll
      for (int i = 0; i < 16; ++i)
        s[tt][i] = (bits >> ((i >> 3) * 16 + (i & 7))) & 1 ? s[tt][i] : -INFINITY;
    }
  };
  auto softmax = [&] {
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
  auto values = [&](const u32x4* V) {
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const u32x4 v = V[v_place<BSC>(c * 32 + col, ks * 2 + half)];
#pragma unroll
        for (int n = 0; n < NP; ++n) o[c] = mfma32<BF16>(v, w.p[n][ks], o[c]);
      }
  };
  // The tile before's values weighed and this one's scores, in one run of products whose operands
  // are read ahead.
  auto products = [&](bool pv, const u32x4* V, bool qk, const u32x4* K) {
    constexpr int kAhead = NP == 3 ? 4 : 6;
    auto read_k = [&](int i) { return K[k_place((i & 1) * 32 + arow, (i >> 1) * 2 + half)]; };
    __builtin_amdgcn_s_setprio(1);
    u32x4 f[16], ahead[kAhead];
    if (pv) {
#pragma unroll
      for (int i = 0; i < 16; ++i) f[i] = V[v_place<BSC>((i & 3) * 32 + col, (i >> 2) * 2 + half)];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) ahead[i] = read_k(i);     // not used where !qk
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int n = 0; n < NP; ++n) o[i & 3] = mfma32<BF16>(f[i], w.p[n][i >> 2], o[i & 3]);
      EMA_SCHED_LDS_READ(kAhead);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        EMA_SCHED_MFMA(NP);
        EMA_SCHED_LDS_READ(1);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) ahead[i] = read_k(i);
    }
    if (qk) {
#pragma unroll
      for (int i = 0; i < 16; ++i) f[i] = i < kAhead ? ahead[i] : read_k(i);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        s[i & 1] = mfma32<BF16>(f[i], q[i >> 1], i < 2 ? f32x16{} : s[i & 1]);
#pragma unroll
      for (int i = 0; i < 16 - kAhead; ++i) {
        EMA_SCHED_MFMA(1);
        EMA_SCHED_LDS_READ(1);
      }
      EMA_SCHED_MFMA(kAhead);
    }
    __builtin_amdgcn_s_setprio(0);
  };
  // A tile masked in part: by the nodes' mask, the request's end or blocks out of range.
  auto is_partly = [&](int j) { return (j + 1) * kKT > base || st.window.bad != 0; };

  auto tile = [&](int place, int v) -> u32x4* { return s_kv[group * kPlaces + place][v]; };
  auto load_k = [&](int j, int place) { st.load_k(lds_address(tile(place, 0)), j, at, rw); };
  auto load_v = [&](int j, int place) { st.load_v(lds_address(tile(place, 1)), j, at, rw); };
  // This wave's part of V tile j has arrived: cleaned where some row masks some of it.
  auto clean = [&](const Segment& g, int j, int place) {
    if (is_partly(j)) odd |= st.template clean_v<BF16>(tile(place, 1), st.there(j, g.len), rw);
  };
  auto open = [&](const Segment& g) {        // the first tiles' loads
    const int j = g.j0 + group;
    if (j >= g.j1) return;
    st.open(a, g.b, kvh, j, g.len);
    at = st.blocks(j);
    load_k(j, 0);
    constexpr int kFirst = RW == 8 ? kPlaces - 1 : kPlaces;
#pragma unroll
    for (int i = 1; i < kFirst; ++i) {
      load_v(j + (i - 1) * kGroups, i - 1);
      if (j + i * kGroups >= g.j1) return;
      at = st.blocks(j + i * kGroups);
      load_k(j + i * kGroups, i);
    }
  };

  Segment g;
  g.b = uniform(s_start[0]);
  g.index = uniform(s_start[1]);
  set_request(g, s_start[2], s_start[3], s_start[4]);
  {
    const int into = uniform(s_start[5]), each = whole ? 1 : g.nt + kSegCost;
    g.item = uniform(into / each);
    g.index += g.item;
    if (!take(g, into - g.item * each) && !next_segment(g)) return;
  }
  bool have = true;
  int turn = 0;                              // whose s_odd is this segment's
  load_q(g);
  open(g);
  while (have) {
    m = -INFINITY;
    l = 0.0f;
#pragma unroll
    for (int c = 0; c < 4; ++c) o[c] = f32x16{};
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) arrived(q[ks]);
    const bool counts = kvh == 0 && first == 0 && rw == 0;
    const int turns = (g.j1 - g.j0 + kGroups - 1) / kGroups;
    if constexpr (RW == 8) {
      // The eight waves are two groups, one of each to a SIMD, that take turns: while one has the
      // matrix cores (products), the other works its scores into weights and sends for later tiles,
      // V of the next but one and K of the one after it, into the places that the turns before were
      // the last to read. The second group is one turn behind.
      constexpr int kTurn = 2 * 16 / RW;     // a wave's loads of a turn
      const int late = wave >= kWaves / 2 ? 1 : 0;
      auto place = [&](int j) { return (j - g.j0) & (kPlaces - 1); };
      auto send = [&](int j) {               // for V of tile j + 2 and K of j + 3
        if (j + 2 < g.j1) load_v(j + 2, place(j + 2));
        if (j + 3 < g.j1) {
          at = st.blocks(j + 3);
          load_k(j + 3, place(j + 3));
        }
      };
      auto arrive = [&](int j) {             // V of tile j, K of j + 1
        if (j >= g.j1) return;
        if (j + 3 < g.j1) loads_arrived_but<2 * kTurn>();
        else loads_arrived();
        clean(g, j, place(j));
        if (counts && st.window.bad != 0) st.count_bad(a, j, g.len);
      };
      if (g.j0 + 2 < g.j1) loads_arrived_but<2 * kTurn>();
      else loads_arrived();
      __syncthreads();
      if (late) {
        send(g.j0);
        arrive(g.j0);
        __syncthreads();
      }
      for (int j = g.j0; j < g.j1; ++j) {
        if (alive) products(j > g.j0, tile(place(j - 1), 1), true, tile(place(j), 0));
        __syncthreads();
        send(j + late);
        if (alive) {
          if (is_partly(j)) hide(g, j, st.there(j, g.len));
          softmax();
        }
        arrive(j + late);
        __syncthreads();
      }
      if (alive) products(true, tile(place(g.j1 - 1), 1), false, tile(0, 0));
      if (!late) __syncthreads();
    } else {
      // K of a tile is sent for as soon as all are done with the scores of the one whose place it
      // takes, V with the product of that one's: both are on their way nearly all of the time. A
      // barrier tells that loads have arrived for all, and that all are done with a place.
      constexpr int kNewer = kPlaces == 1 ? 16 / RW : 2 * (kPlaces - 1) * 16 / RW;
      int place = 0;
      for (int i = 0; i < turns; ++i) {
        const int j = g.j0 + group + i * kGroups, last = j + (kPlaces - 1) * kGroups;
        const int before = place == 0 ? kPlaces - 1 : place - 1;
        const bool here = j < g.j1, more = last + kGroups < g.j1;
        if (kPlaces > 1 && last < g.j1) loads_arrived_but<kNewer>();
        else loads_arrived();
        __syncthreads();
        if (last < g.j1) {
          // (blocks are looked up in ascending order: `at` is tile last's still)
          load_v(last, before);
        }
        if (here) {
          if (counts && st.window.bad != 0) st.count_bad(a, j, g.len);
          if (alive) {
            scores(tile(place, 0));
            if (is_partly(j)) hide(g, j, st.there(j, g.len));
          }
        }
        reads_done();
        if (kPlaces > 1) {
          if (last < g.j1) loads_arrived_but<kNewer>();
          else loads_arrived();
          if (here) clean(g, j, place);
        }
        __syncthreads();
        if (more) {
          at = st.blocks(last + kGroups);
          load_k(last + kGroups, place);
        }
        if (here && alive) softmax();
        if (kPlaces == 1) {
          if (more) loads_arrived_but<kNewer>();
          else loads_arrived();
          if (here) clean(g, j, place);
          __syncthreads();
        }
        if (here && alive) values(tile(place, 1));
        place = place == kPlaces - 1 ? 0 : place + 1;
      }
    }

    // ---- the waves' parts of a row -----------------------------------------------------
    if (__ballot(odd) && lane == 0) atomicOr(&s_odd[turn], st.window.bad != 0 ? 3 : 1);
    odd = false;
    __syncthreads();                         // all are done with their tiles
    f32x4* const part = reinterpret_cast<f32x4*>(&s_kv[0][0][0]);
    // Four channels 4f .. 4f + 3 of a wave's row, rows off each other's banks.
    auto part_at = [&](int w, int r, int f) -> f32x4& {
      return part[w * kTilePieces + r * 32 + (f ^ r)];
    };
    const float sum = l + other_half(l);
    if (half == 0) {
      s_m[wave][col] = m;
      s_l[wave][col] = sum;
      if (group == 0) s_row[rw * 32 + col] = out_row;
    }
#pragma unroll
    for (int c = 0; c < 4; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        part_at(wave, col, c * 8 + i * 2 + half) =
            f32x4{o[c][4 * i], o[c][4 * i + 1], o[c][4 * i + 2], o[c][4 * i + 3]};
    const Segment done = g;
    const int done_first = first, done_kvh = kvh;
    have = next_segment(g);
    if (have) load_q(g);
    __syncthreads();
    const int odds = s_odd[turn];
    turn ^= 1;
    if (tid == 0) s_odd[turn] = 0;           // (read before the last barrier but one)
    const bool begins = done.j0 == 0, ends = done.j1 == done.nt;
    const int64_t slot = 2 * wg + (begins ? 1 : 0);
    AttnArgs out;
    out.out = a.out;
    out.out_dtype = a.out_dtype;
    out.out_vec = 1;
    for (int x = tid; x < kRows * 32; x += kThreads) {
      const int r = x >> 5, f = x & 31, w0 = r >> 5, wr = r & 31;
      const int row = s_row[r];
      if (row < 0) break;
      float M = -INFINITY, L = 0.0f;
#pragma unroll
      for (int y = 0; y < kGroups; ++y) M = fmaxf(M, s_m[y * RW + w0][wr]);
      const float ref = M == -INFINITY ? 0.0f : M;
      f32x4 O = f32x4{};
#pragma unroll
      for (int y = 0; y < kGroups; ++y) {
        const float by = __builtin_amdgcn_exp2f(s_m[y * RW + w0][wr] - ref);
        L = fmaf(by, s_l[y * RW + w0][wr], L);
        O += part_at(y * RW + w0, wr, f) * by;
      }
      if (odds != 0) {
        const int node = (done_first + r) / G;
        // V was cleaned of what is not finite: a row that attends such a value gets NaN
        const int32_t* ids = a.table + int64_t(done.b) * a.max_blocks;
        const int begin = max(done.j0 * kKT, odds & 2 ? 0 : (done.len - done.n) & ~(kKT - 1));
        for (int t = begin; t < min(done.j1 * kKT, done.len); ++t) {
          const int id = ids[t >> a.block_shift];
          if (!(attended(done, node, t & ~(kKT - 1)) >> (t & (kKT - 1)) & 1)) continue;
          if (uint32_t(id) >= uint32_t(a.n_local)) continue;
          const uint16_t* v = reinterpret_cast<const uint16_t*>(
              a.local + int64_t(id) * a.block_bytes + a.block_bytes / 2) +
              int64_t(done_kvh * 128 + 4 * f) * a.block_size + (t & (a.block_size - 1));
          constexpr uint32_t kExp = BF16 ? 0x7f80u : 0x7c00u;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if ((v[i * a.block_size] & kExp) == kExp) O[i] = NAN;
        }
      }
      if (!(begins && ends)) {
        *reinterpret_cast<f32x4*>(a.ws + (slot * kRows + r) * 128 + 4 * f) = O;
        if (f == 0) {
          ws_ml[(slot * kRows + r) * 2] = M;
          ws_ml[(slot * kRows + r) * 2 + 1] = L;
        }
        continue;
      }
      const float inv = L == 0.0f ? 0.0f : 1.0f / L;
      store_out4(out, int64_t(row) * 128 + 4 * f,
                 out_f32x4{O[0] * inv, O[1] * inv, O[2] * inv, O[3] * inv});
    }
    if (!whole && begins && tid == 0 && (itemwise ? done.index < cut.bound : !ends)) {
      int32_t* const rec = info + 1 + (itemwise ? done.index : wg) * kRecord;
      rec[0] = ends ? -1 : wg;
      // a part: the range ends with this segment
      rec[1] = (u1 + (done.nt - done.j1) - 1) / per;
      rec[2] = done.row0;
      rec[3] = done.n * G;
      rec[4] = done_first;
      rec[5] = done_kvh;
    }
    __syncthreads();
    if (have) open(g);
  }
}

// Joins the parts of shared items: 32 lanes to a row, four channels a lane; `share` such groups
// of a workgroup take a row's parts in turn. Bound by the parts' way from memory and by its chain of
// loads: 41 MB of 16 trees of 48-64 nodes 16 us, 4.6 where nothing is shared.
__global__ __launch_bounds__(kJoinRows * 32) void tree_join(TreeAttnArgs a, int grid, int rows,
                                                            int share) {
  __shared__ __attribute__((aligned(16))) f32x4 s_o[kJoinRows][32];
  __shared__ float s_m[kJoinRows], s_l[kJoinRows];
  const float* ws_ml = a.ws + int64_t(2) * grid * rows * 128;
  const int32_t* info = reinterpret_cast<const int32_t*>(ws_ml + int64_t(2) * grid * rows * 2);
  const int each = rows * share / kJoinRows, tasks = info[0] * each;
  const int f = threadIdx.x & 31, group = threadIdx.x >> 5;
  const int G = a.q_heads / a.kv_heads;
  for (int task = blockIdx.x; task < tasks; task += gridDim.x) {
    const int32_t* rec = info + 1 + task / each * kRecord;
    const int w0 = rec[0], n = rec[1] - w0 + 1;
    const int r = task % each * (kJoinRows / share) + group / share;
    if (w0 < 0 || rec[4] + r - group / share >= rec[3]) continue;      // (the same for all)
    const bool live = rec[4] + r < rec[3];
    float M = -INFINITY, L = 0.0f;
    f32x4 O = f32x4{};
    constexpr int kAtOnce = 4;
    for (int i0 = group % share; live && i0 < n; i0 += kAtOnce * share) {
      f32x4 po[kAtOnce];
      float pm[kAtOnce], pl[kAtOnce];
#pragma unroll
      for (int y = 0; y < kAtOnce; ++y) {
        const int i = i0 + y * share;
        if (i >= n) break;
        const int64_t at = int64_t(i == 0 ? 2 * w0 + 1 : 2 * (w0 + i)) * rows + r;
        po[y] = *reinterpret_cast<const f32x4*>(a.ws + at * 128 + 4 * f);
        pm[y] = ws_ml[at * 2];
        pl[y] = ws_ml[at * 2 + 1];
      }
#pragma unroll
      for (int y = 0; y < kAtOnce; ++y) {
        if (i0 + y * share >= n) break;
        const float M_new = fmaxf(M, pm[y]);
        const float ref = M_new == -INFINITY ? 0.0f : M_new;
        const float d = __builtin_amdgcn_exp2f(M - ref), e = __builtin_amdgcn_exp2f(pm[y] - ref);
        M = M_new;
        L = L * d + pl[y] * e;
        O = O * d + po[y] * e;
      }
    }
    if (share > 1) {
      __syncthreads();                       // the task before is done with them
      s_o[group][f] = O;
      if (f == 0) {
        s_m[group] = M;
        s_l[group] = L;
      }
      __syncthreads();
      if (group % share != 0) continue;
      float top = -INFINITY;
      for (int y = 0; y < share; ++y) top = fmaxf(top, s_m[group + y]);
      const float ref = top == -INFINITY ? 0.0f : top;
      L = 0.0f;
      O = f32x4{};
      for (int y = 0; y < share; ++y) {
        const float d = __builtin_amdgcn_exp2f(s_m[group + y] - ref);
        L = fmaf(d, s_l[group + y], L);
        O += s_o[group + y][f] * d;
      }
    }
    if (!live) continue;
    AttnArgs out;
    out.out = a.out;
    out.out_dtype = a.out_dtype;
    out.out_vec = 1;
    const float inv = L == 0.0f ? 0.0f : 1.0f / L;
    const int node = (rec[4] + r) / G, h = rec[4] + r - node * G;
    store_out4(out, (int64_t(rec[2] + node) * a.q_heads + rec[5] * G + h) * 128 + 4 * f,
               out_f32x4{O[0] * inv, O[1] * inv, O[2] * inv, O[3] * inv});
  }
}

Cut cut_of(const PromptArgs& a) {
  Cut c;
  const int64_t mean = (int64_t(a.tokens) + a.batch - 1) / a.batch * (a.q_heads / a.kv_heads);
  c.rows = 64;
  while (c.rows < 256 && c.rows < mean) c.rows *= 2;
  c.bound = tile_bound(a, c.rows) * a.kv_heads;
  // (the most that there can be tiles)
  const int64_t tiles = (int64_t(a.max_blocks) * a.block_size + kKT - 1) / kKT;
  // (one request of 8 and 1 heads. 7 nodes behind 32001 tokens: 29.5 us with 2 units, 24.4 with 4,
  // 23.3 with 6, 23.9 with 8, 29.2 with 16; behind 8001: 19.5, 18.4, 19.7, 21.4, 28.0. 15 nodes: 38.6,
  // 31.8, 32.1, 33.8, 44.9 and 23.3, 24.5, 26.9, 30.1, 43.5. 31 nodes, 256 rows, behind 32001: 41.1,
  // 37.1, 37.2, 39.8, 49.6. So 6 is at most 3 % off the best behind long contexts, and some 2 us
  // behind shorter ones, where 4 or fewer would do)
  c.least = c.rows < 256 ? 6 : 4;
  // (64 rows: HBM is full with half of the workgroups; 256: each has its own time. Several rounds of
  // items are as uneven as one workgroup is alone with them: 200 requests, 8 heads, 204 us for 175)
  c.uneven = c.rows < 256 ? 8 : 5;
  const int64_t most_wgs = kCus * (c.rows == 64 ? Shape<64>::kPerCu : c.rows == 128 ? Shape<128>::kPerCu : 1);
  c.whole = tiles <= kWholeTiles && c.bound <= 1 << 16;
  c.grid = c.whole ? int(c.bound)
                   : int(std::max<int64_t>(1, c.bound > most_wgs || tiles > most_wgs
                                                  ? most_wgs
                                                  : std::min(most_wgs, c.bound * tiles)));
  return c;
}
int64_t records(const Cut& c) { return by_item(c) ? c.bound : c.grid; }

template <bool BF16, int NP, int ROWS>
void launch_sizes(const TreeAttnArgs& a, const Cut& c, hipStream_t stream) {
  const dim3 grid(unsigned(c.grid)), threads(Shape<ROWS>::kWaves * 64);
  if (a.block_size == 16)
    hipLaunchKernelGGL((tree_kernel<BF16, 16, NP, ROWS>), grid, threads, 0, stream, a, c);
  else if (a.block_size == 32)
    hipLaunchKernelGGL((tree_kernel<BF16, 32, NP, ROWS>), grid, threads, 0, stream, a, c);
  else
    hipLaunchKernelGGL((tree_kernel<BF16, 64, NP, ROWS>), grid, threads, 0, stream, a, c);
}

template <bool BF16, int NP>
void launch_rows(const TreeAttnArgs& a, const Cut& c, hipStream_t stream) {
  switch (c.rows) {
    case 64:
      launch_sizes<BF16, NP, 64>(a, c, stream);
      break;
    case 128:
      launch_sizes<BF16, NP, 128>(a, c, stream);
      break;
    default:
      launch_sizes<BF16, NP, 256>(a, c, stream);
  }
}

}  // namespace

bool tree_fits(const PromptArgs& a) {
  const int64_t tiles = (int64_t(a.max_blocks) * a.block_size + kKT - 1) / kKT;
  return (tile_bound(a, 64) * a.kv_heads) * (tiles + kSegCost) < int64_t(1) << 30;
}

size_t tree_workspace(const PromptArgs& a) {
  const Cut c = cut_of(a);
  if (c.whole) return 0;
  return (size_t(2) * c.grid * c.rows * 130 + 1 + size_t(records(c)) * kRecord) * 4;
}

hipError_t launch_tree_attention(const TreeAttnArgs& a, hipStream_t stream) {
  const Cut c = cut_of(a);
  if (a.dtype == 1) {
    if (a.full) launch_rows<true, 3>(a, c, stream);
    else launch_rows<true, 1>(a, c, stream);
  } else {
    if (a.full) launch_rows<false, 2>(a, c, stream);
    else launch_rows<false, 1>(a, c, stream);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || c.whole) return e;
  const int64_t recs = records(c);
  // as many groups to a row as it has parts, roughly
  const int share = recs * 8 <= c.grid ? 8 : recs * 3 <= c.grid ? 4 : 1;
  const int64_t tasks = recs * (c.rows * share / kJoinRows);
  hipLaunchKernelGGL(tree_join, dim3(unsigned(std::min<int64_t>(tasks, kJoinGrid))),
                     dim3(kJoinRows * 32), 0, stream, a, c.grid, c.rows, share);
  return hipGetLastError();
}

}  // namespace ema
