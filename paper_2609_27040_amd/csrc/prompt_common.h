// What the matrix-core kernels of prompt chunks share (device code only): finding
// a workgroup's rows, staging K and V tiles in LDS, and their operands.
#pragma once

#include "attn_store.h"
#include "op_kernels.h"

#include <algorithm>

namespace ema {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kKT = 64;                 // tokens of a staged tile

constexpr int kTilePieces = kKT * 16;   // 16-byte pieces of a tile's K, and of its V

// Tiles of `rows` rows of all sequences at most, whatever their lengths: a sequence of n tokens
// and G heads a KV head has ceil(n * G / rows) of them, which is neither more than n times those of
// one token nor, added up, more than all rows' and one for every further sequence.
inline int64_t tile_bound(const PromptArgs& a, int rows) {
  const int64_t group = a.q_heads / a.kv_heads;
  return std::min<int64_t>(a.tokens * ((group + rows - 1) / rows),
                           (a.tokens * group + rows - 1) / rows + a.batch - 1);
}

// Parts that the tokens of a launch's `groups` row tiles are cut into, each of 256 tokens at
// least where the table is full: the number with the least time by this estimate, in tiles of
// 1.7 us. A workgroup takes its tiles and some 5 more (it starts and writes its rows); 256 run
// at once, longest first, and the last, shortest ones leave half of the chip idle; a
// part's outputs, as many bytes as the rows have in 32 bits, are written and read at 5 TB/s in
// a further launch. (As many as fit on the chip at once, against this: 2 chunks of some 1250
// tokens behind 2250, 16 query and 2 KV heads, 157 workgroups, 1 part 112 us, 2 parts 92. Not
// counting the idle half takes 3 parts for 2 chunks of 200 behind 20000, 64 and 8 heads, where
// 2 fill the chip: 347 us for 274.)
inline int split_parts(const PromptArgs& a, int64_t groups) {
  const double tiles = double(a.max_blocks) * a.block_size / kKT;
  const double chunk = double(a.tokens) / a.batch / kKT;
  const double mean = std::max(1.0, tiles - chunk / 2), last = std::max(1.0, tiles - chunk);
  const double join = 2.0 * a.tokens * a.q_heads * 128 * 4 / 5e6 / 1.7;
  int best = 1;
  double least = 0.0;
  // (the last bound keeps grids far below 2^32 threads)
  for (int s = 1; s == 1 || (s <= 64 && s * 4 <= tiles && groups * s <= 1 << 18); ++s) {
    const double work = double(groups) * s / 256 * (mean / s + 5);
    const double t = std::max(tiles / s + 5, groups * s <= 256 ? 0 : work + (last / s + 5) / 2) +
                     (s > 1 ? s * join + 2 : 0);
    if (s == 1 || t < least) {
      best = s;
      least = t;
    }
  }
  return best;
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

template <bool BF16>
__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
  if constexpr (BF16)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// MFMA row i of a 32-token tile of scores is this token of it: every lane then has 8
// consecutive tokens, 8 * (lane / 32) on, of both 16-token halves.
__device__ __forceinline__ int score_row(int i) {
  return (i >> 4) * 16 + ((i >> 2) & 1) * 8 + ((i >> 3) & 1) * 4 + (i & 3);
}

// Two floats rounded to nearest into 16-bit halves of a word, and back.
template <bool BF16>
__device__ __forceinline__ uint32_t pack16(float x, float y) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  if constexpr (BF16) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x, y}), bf16x2));
  } else {
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, f16x2{_Float16(x), _Float16(y)});
  }
}
template <bool BF16>
__device__ __forceinline__ float low16(uint32_t w) {
  if constexpr (BF16) return __builtin_bit_cast(float, w << 16);
  else return float(__builtin_bit_cast(_Float16, uint16_t(w)));
}
template <bool BF16>
__device__ __forceinline__ float high16(uint32_t w) {
  if constexpr (BF16) return __builtin_bit_cast(float, w & 0xffff0000u);
  else return float(__builtin_bit_cast(_Float16, uint16_t(w >> 16)));
}

// The value of the lane 32 away.
__device__ __forceinline__ float other_half(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x),
                                                  __builtin_bit_cast(uint32_t, x), false, false);
  // r[0]: the lower half's values in both halves; r[1]: the upper half's
  return __builtin_bit_cast(float, (threadIdx.x & 32) ? r[0] : r[1]);
}

// Whether any of a piece's eight 16-bit values is an infinity or NaN.
template <bool BF16>
__device__ __forceinline__ bool not_finite(u32x4 v) {
  constexpr uint32_t kExp = BF16 ? 0x7f80u : 0x7c00u;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    bad |= (v[i] & kExp) == kExp || ((v[i] >> 16) & kExp) == kExp;
  return bad;
}

// Zeroes the values of a piece of V (eight tokens from `tok` on, of one channel)
// that are not finite and notes the first of them. In a tile that some rows mask in
// part, 0 times them would be NaN for rows that do not attend them; the rows that do
// get NaN at the end instead.
template <bool BF16>
__device__ __forceinline__ void drop_not_finite(u32x4& v, int tok, int* first, int* any) {
  constexpr uint32_t kExp = BF16 ? 0x7f80u : 0x7c00u;
  atomicMin(any, tok);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if ((v[i] & kExp) == kExp) {
      atomicMin(first, tok + 2 * i);
      v[i] &= 0xffff0000u;
    }
    if (((v[i] >> 16) & kExp) == kExp) {
      atomicMin(first, tok + 2 * i + 1);
      v[i] &= 0xffffu;
    }
  }
}

// A workgroup's rows: (token, query head of the group) pairs of one sequence and KV
// head, `rows` to a workgroup, in token order.
struct RowTile {
  int b;          // sequence; -1: no such tile
  int row0;       // its first row in q and out
  int n;          // its rows (tokens)
  int first;      // first (token, head) pair of the tile
  int len;        // tokens of the sequence
  int given;      // its length as it is given
  int wrong;      // of the sequences this thread looked at: those whose rows are no range of q's
};

// Rows of sequence b in q, clamped to what is there; 1 if the starts are out of range.
__device__ __forceinline__ int row_range(const PromptArgs& a, int b, int& s, int& n) {
  const int from = a.starts[b], to = a.starts[b + 1];
  s = min(max(from, 0), a.tokens);
  n = max(0, min(to, a.tokens) - s);
  return from < 0 || to < from || to > a.tokens || (b == 0 && from != 0);
}

// Sum and maximum (of values >= 0) over the wave's 64 lanes, uniform: DPP moves within
// rows of 16 lanes, the row totals carried over to the last lane.
template <typename Op>
__device__ __forceinline__ int wave_reduce(int x, Op&& op) {
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true));    // row_shr 1, 2, 4, 8
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true));
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true));
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true));
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));   // lane 15 of rows 0, 2 to 1, 3
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));   // lane 31 to rows 2, 3
  return __builtin_amdgcn_readlane(x, 63);
}
__device__ __forceinline__ int wave_sum(int x) {
  return wave_reduce(x, [](int p, int q) { return p + q; });
}
__device__ __forceinline__ int wave_max(int x) {
  return wave_reduce(x, [](int p, int q) { return max(p, q); });
}

// Tile `index` of all sequences' tiles, those that see the most tokens first (they take
// the longest, and what is left over at the end of the launch should be short ones):
// a tile's level is how many tiles of rows its last token lies before the longest
// sequence's end, so a sequence has one tile at most of each level. (Four prompts of
// 257-3841 tokens, sequence by sequence: 246-270 us by their order, the last tile of each
// first: 240, so: 215.) Every wave searches alone, 64 sequences at a time.
constexpr int kLevelBatch = 512;         // eight sequences a lane, in registers
// Sequences up to which a level is found 64 at a time, not by bisection: 4 prompts of 257-3841
// tokens 210 us (by bisection 216), 16 of 100-500 tokens 49.5 (49.2).
constexpr int kWideBatch = 8;
template <int ROWS>
__device__ __forceinline__ RowTile find_by_level(const PromptArgs& a, int group, int index) {
  constexpr int N = kLevelBatch / 64;
  const int lane = threadIdx.x & 63;
  int tiles[N], start[N], rows[N], len[N], skip[N];   // of sequences 64 * i + lane
  int total = 0, longest = 0;
  RowTile r;
  r.wrong = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    tiles[i] = rows[i] = start[i] = len[i] = 0;
    if (i * 64 >= a.batch) continue;
    const int b = i * 64 + lane;
    if (b < a.batch) {
      r.wrong += row_range(a, b, start[i], rows[i]);
      len[i] = a.seq_lens[b];
    }
    tiles[i] = (rows[i] * group + ROWS - 1) / ROWS;
    total += tiles[i];
    if (tiles[i] > 0) longest = max(longest, len[i]);
  }
  if (threadIdx.x >= 64) r.wrong = 0;    // every wave looks at all sequences
  r.b = -1;
  if (index >= wave_sum(total)) return r;
  longest = wave_max(longest);
  int most = 0;                          // levels
#pragma unroll
  for (int i = 0; i < N; ++i) {          // the level of a sequence's last tile
    skip[i] = 0;
    if (i * 64 >= a.batch) continue;
    skip[i] = min(int64_t(longest - max(len[i], 0)) * group / ROWS, int64_t(1) << 24);
    if (tiles[i] > 0) most = max(most, skip[i] + tiles[i]);
  }
  auto below = [&](int level) {          // tiles at levels under this one
    int t = 0;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i * 64 < a.batch) t += max(0, min(tiles[i], level - skip[i]));
    return wave_sum(t);
  };
  int lo = 0, hi = wave_max(most), at = 0;     // below(lo) <= index < below(hi)
  if (a.batch <= kWideBatch) {
    // each lane takes one of 64 levels and adds up its tiles sequence by sequence
    while (hi - lo > 1) {
      const int step = (hi - lo + 63) / 64, c = min(lo + (lane + 1) * step, hi);
      int t = 0;
      for (int b = 0; b < a.batch; ++b)
        t += max(0, min(__builtin_amdgcn_readlane(tiles[0], b),
                        c - __builtin_amdgcn_readlane(skip[0], b)));
      const int n = __popcll(__ballot(t <= index));    // the first n lanes
      if (n > 0) at = __builtin_amdgcn_readlane(t, n - 1);
      lo += n * step;
      hi = min(hi, lo + step);
    }
  }
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1, t = below(mid);
    if (t <= index) {
      lo = mid;
      at = t;
    } else {
      hi = mid;
    }
  }
  int k = index - at;                    // the k-th sequence with a tile of level lo
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (i * 64 >= a.batch || r.b >= 0) continue;
    const bool has = lo >= skip[i] && lo - skip[i] < tiles[i];
    const unsigned long long m = __ballot(has);
    const int c = __popcll(m);
    if (k < c) {
      const unsigned long long hit = __ballot(has && __popcll(m & ((1ull << lane) - 1ull)) == k);
      const int l = __builtin_ctzll(hit);
      r.b = i * 64 + l;
      r.first = (__builtin_amdgcn_readlane(tiles[i] + skip[i], l) - 1 - lo) * ROWS;
      r.row0 = __builtin_amdgcn_readlane(start[i], l);
      r.n = __builtin_amdgcn_readlane(rows[i], l);
      r.len = __builtin_amdgcn_readlane(len[i], l);
    }
    k -= c;
  }
  r.b = uniform(r.b);
  r.first = uniform(r.first);
  r.row0 = uniform(r.row0);
  r.n = uniform(r.n);
  r.given = uniform(r.len);
  r.len = max(0, min(r.given, a.max_blocks * a.block_size));
  return r;
}

// Tile `index` sequence by sequence, for batches above kLevelBatch: the workgroup
// walks the starts together, thread t consecutive sequences.
template <int THREADS, int ROWS>
__device__ __forceinline__ RowTile find_in_order(const PromptArgs& a, int group, int index,
                                                 int* s_scratch) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = (a.batch + THREADS - 1) / THREADS;
  const int b0 = min(a.batch, tid * per), b1 = min(a.batch, b0 + per);
  int total = 0;
  RowTile r;
  r.wrong = 0;
  for (int b = b0; b < b1; ++b) {
    int s, n;
    r.wrong += row_range(a, b, s, n);
    total += (n * group + ROWS - 1) / ROWS;
  }
  int incl = total;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int x = __shfl_up(incl, o);
    if (lane >= o) incl += x;
  }
  if (lane == 63) s_scratch[wave] = incl;
  if (tid == 0) s_scratch[THREADS / 64] = -1;
  __syncthreads();
  int at = incl - total;
  for (int w = 0; w < wave; ++w) at += s_scratch[w];
  int* out = s_scratch + THREADS / 64;
  if (index >= at && index < at + total) {
    for (int b = b0; b < b1; ++b) {
      int s, n;
      row_range(a, b, s, n);
      const int t = (n * group + ROWS - 1) / ROWS;
      if (index < at + t) {
        out[0] = b;
        out[1] = s;
        out[2] = n;
        out[3] = (index - at) * ROWS;
        break;
      }
      at += t;
    }
  }
  __syncthreads();
  r.b = uniform(out[0]);
  if (r.b < 0) return r;
  r.row0 = uniform(out[1]);
  r.n = uniform(out[2]);
  r.first = uniform(out[3]);
  r.given = uniform(a.seq_lens[r.b]);
  r.len = max(0, min(r.given, a.max_blocks * a.block_size));
  return r;
}

template <int THREADS, int ROWS>
__device__ __forceinline__ RowTile find_tile(const PromptArgs& a, int group, int index,
                                             int* s_scratch) {
  return a.batch <= kLevelBatch ? find_by_level<ROWS>(a, group, index)
                                : find_in_order<THREADS, ROWS>(a, group, index, s_scratch);
}
constexpr int kFindScratch = 16 + 4;

// The row of a lane and the tokens that it, its wave's 32 rows and its workgroup look at.
struct Reach {
  bool live;              // there is such a row
  int tok, g;             // its token of the chunk, its head of the group
  int pos;                // it attends tokens 0 .. pos
  int end, from;          // workgroup: tokens looked at; position of its first row
  int wave_end, wave_from;
  int j0, j1;             // tiles of this split
};
// `first`: the wave's first row, counted from the sequence's.
template <int ROWS>
__device__ __forceinline__ Reach reach_of(const RowTile& R, int group, int first, int split,
                                          int splits) {
  Reach x;
  const int past = R.len - R.n, rows = R.n * group;  // tokens before the chunk
  const int r = first + (threadIdx.x & 31);
  x.live = r < rows;
  x.tok = x.live ? r / group : 0;
  x.g = x.live ? r - x.tok * group : 0;
  x.pos = x.live ? past + x.tok : -1;
  x.end = uniform(max(0, past + (min(rows, R.first + ROWS) - 1) / group + 1));
  x.from = uniform(past + R.first / group);
  x.wave_end = uniform(first >= rows ? 0 : max(0, past + min(rows - 1, first + 31) / group + 1));
  x.wave_from = uniform(past + first / group);
  const int tiles = (x.end + 63) / 64;
  x.j0 = uniform(int(int64_t(tiles) * split / splits));
  x.j1 = uniform(int(int64_t(tiles) * (split + 1) / splits));
  return x;
}

// ---- staged tiles --------------------------------------------------------------------
//
// K: row t (256 bytes, 16 pieces) as it is, its pieces permuted by t so that the 16
// rows a quarter of a wave reads one piece of lie in different banks. V^T: rows of
// a block have r = min(block size, 64) / 8 pieces; a block's rows follow each other, a
// row's pieces permuted by its channel to the same end.
__device__ __forceinline__ int k_place(int tok, int piece) {
  return tok * 16 + (piece ^ (tok & 15));
}
template <int BSC>
__device__ __forceinline__ int v_turn(int ch) {
  constexpr int r = BSC / 8;
  return r == 8 ? (ch >> 1) & 7 : r == 4 ? (ch >> 2) & 3 : (ch >> 3) & 1;
}
template <int BSC>
__device__ __forceinline__ int v_place(int ch, int group) {   // group: eight tokens of the tile
  constexpr int r = BSC / 8;
  return group / r * (128 * r) + ch * r + ((group % r) ^ v_turn<BSC>(ch));
}

// The block ids of a row of the table, 64 at a time in the lanes of a register (and
// the 64 after them, on their way), read tile by tile in ascending order. Past block
// `last`, that one again (its rows are masked there). An id outside the local pool reads
// as block 0, which always exists, and leaves its mark in `bad`.
struct IdWindow {
  const int32_t* row;
  int last, at;          // at: first block of the window, a multiple of 64
  int n_local = 0, bad = 0;      // bad: ids out of range so far
  int32_t cur, next;
  __device__ __forceinline__ void open(const PromptArgs& a, int b, int first, int last_block) {
    row = a.table + int64_t(b) * a.max_blocks;
    n_local = a.n_local;
    last = last_block;
    at = first & ~63;
    bad = 0;
    cur = checked(fetch(at));
    next = fetch(at + 64);
  }
  __device__ __forceinline__ int32_t fetch(int block) const {
    return row[min(block + int(threadIdx.x & 63), last)];
  }
  __device__ __forceinline__ int32_t checked(int32_t id) {
    const bool ok = uint32_t(id) < uint32_t(n_local);
    bad += __popcll(__ballot(!ok && at + int(threadIdx.x & 63) <= last));
    return ok ? id : 0;
  }
  __device__ __forceinline__ void seek(int block) {
    if (block >= at + 64) {
      at += 64;
      cur = checked(next);
      next = fetch(at + 64);
    }
  }
  __device__ __forceinline__ int get(int block) const {
    return __builtin_amdgcn_readlane(cur, block & 63);
  }
  // Whether the table names a block of the pool there (only asked where bad > 0).
  __device__ __forceinline__ bool good(int block) const {
    return uint32_t(row[min(block, last)]) < uint32_t(n_local);
  }
};

// 16 bytes a lane from `base` (uniform) + `off` straight into LDS, at byte `lds` (uniform)
// + 16 * lane. Nothing is written to registers; loads_arrived() waits for all of the
// wave's.
__device__ __forceinline__ void load_to_lds(const char* base, uint32_t off, uint32_t lds) {
  const uint64_t b = reinterpret_cast<uint64_t>(base);
  const uint64_t ub = uint64_t(uint32_t(uniform(int(uint32_t(b))))) |
                      uint64_t(uint32_t(uniform(int(uint32_t(b >> 32))))) << 32;
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :: "s"(uniform(int(lds))), "v"(off), "s"(ub) : "memory", "m0");
}
// The same from an address per lane; NT: streamed past the caches.
template <bool NT>
__device__ __forceinline__ void load_lane_to_lds(const char* p, uint32_t lds) {
  if constexpr (NT)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt"
                 :: "s"(uniform(int(lds))), "v"(p) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                 :: "s"(uniform(int(lds))), "v"(p) : "memory", "m0");
}
// All of the wave's loads but the newest 16 have arrived.
__device__ __forceinline__ void loads_arrived_but_16() {
  asm volatile("s_waitcnt vmcnt(16)" ::: "memory");
}
// Nothing of the wave still reads LDS.
__device__ __forceinline__ void reads_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void loads_arrived() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return uint32_t(reinterpret_cast<uintptr_t>(
      (const __attribute__((address_space(3))) void*)p));
}

// Loads tiles of K and V of a workgroup's sequence into LDS, by THREADS of its threads. Place p
// of a tile is loaded by the (p % THREADS)-th of them; which piece belongs there is in the
// offsets. A wave's 64 places of one round lie in one block, the same for K and V. `head` counts from the workgroup's first KV
// head: a head's K and V both take 256 * block_size bytes.
template <int BSC, int THREADS>
struct Staging {
  static constexpr int kPieces = kTilePieces / THREADS;
  static constexpr int kPer = 16 * BSC;              // pieces of a block
  struct Blocks {
    const char* at[kPieces];                         // the blocks of this wave's places
  };
  const char* local;
  int64_t block_bytes;
  int shift, mask, last, head_bytes, wave;
  uint32_t k_off[kPieces], v_off[kPieces];           // bytes in the block
  IdWindow window;

  static __device__ __forceinline__ int thread() { return int(threadIdx.x) % THREADS; }
  // Of sequence b, whose first `end` tokens (one at least) are looked at, from tile j0 on.
  __device__ __forceinline__ void open(const PromptArgs& a, int b, int kvh, int j0, int end) {
    const int tid = thread();
    local = a.local;
    block_bytes = a.block_bytes;
    shift = a.block_shift;
    mask = a.block_size - 1;
    head_bytes = 256 * a.block_size;
    wave = uniform(tid >> 6);
    last = (end - 1) >> shift;
#pragma unroll
    for (int x = 0; x < kPieces; ++x) {
      const int p = x * THREADS + tid, kt = p >> 4;
      k_off[x] = kvh * head_bytes + (kt % BSC * 128 + ((p ^ kt) & 15) * 8) * 2;
      v_off[x] = uint32_t(a.block_bytes / 2) + kvh * head_bytes +
                 (channel(x) * a.block_size + group(x) * 8) * 2;
    }
    window.open(a, b, (j0 * kKT) >> shift, last);
  }
  // The channel, the eight tokens of its block and the first token of the tile that piece x of
  // this thread's V is.
  static __device__ __forceinline__ int channel(int x) {
    return (x * THREADS + thread()) % kPer / (BSC / 8);
  }
  static __device__ __forceinline__ int group(int x) {
    return (x * THREADS + thread()) % (BSC / 8) ^ v_turn<BSC>(channel(x));
  }
  static __device__ __forceinline__ int token(int x) {
    return (x * THREADS + thread()) / kPer * BSC + group(x) * 8;
  }
  // Where tile j's pieces are; tiles in ascending order.
  __device__ __forceinline__ Blocks blocks(int j) {
    Blocks t;
    const int first = (j * kKT) >> shift;
    window.seek(min(first, last));
#pragma unroll
    for (int x = 0; x < kPieces; ++x)
      t.at[x] = local + int64_t(window.get(min(first + (x * THREADS + wave * 64) / kPer, last))) *
                            block_bytes;
    return t;
  }
  // On to tile j, for a wave that loads none of it.
  __device__ __forceinline__ void pass(int j) { window.seek(min((j * kKT) >> shift, last)); }
  // Counts the entries of tile j whose block begins there, before token `end`, and is not of the
  // pool; one wave of those that see a sequence's tiles does. (window.bad takes whole windows, of
  // which a part of the tiles holds some only.)
  __device__ __forceinline__ void count_bad(const PromptArgs& a, int j, int end) const {
    const int lane = threadIdx.x & 63, tok = j * kKT + lane * 16;
    const bool bad = lane < kKT / 16 && tok < end && (tok & mask) == 0 && !window.good(tok >> shift);
    const int n = __popcll(__ballot(bad));
    if (n > 0 && lane == 0) atomicAdd(a.err_count, n);
  }
  // `to`: the tile's address in LDS.
  __device__ __forceinline__ void load_k(uint32_t to, int j, const Blocks& t, int head) const {
    const int in = BSC == 64 ? ((j * kKT) & mask) * 256 : 0;   // of block size 128 and more
#pragma unroll
    for (int x = 0; x < kPieces; ++x)
      load_to_lds(t.at[x] + in + head * head_bytes, k_off[x], to + (x * THREADS + wave * 64) * 16);
  }
  __device__ __forceinline__ void load_v(uint32_t to, int j, const Blocks& t, int head) const {
    const int in = BSC == 64 ? ((j * kKT) & mask) * 2 : 0;
#pragma unroll
    for (int x = 0; x < kPieces; ++x)
      load_to_lds(t.at[x] + in + head * head_bytes, v_off[x], to + (x * THREADS + wave * 64) * 16);
  }
  // In the pieces this thread has loaded of V tile j: V of tokens from `end` on or in no block
  // of the pool becomes 0, and so does what is not finite (noted in first[channel], any).
  template <bool BF16>
  __device__ __forceinline__ void clean_v(u32x4* tile, int j, int end, int* first, int* any) const {
#pragma unroll
    for (int x = 0; x < kPieces; ++x) {
      u32x4* at = tile + x * THREADS + thread();
      u32x4 v = *at;
      const int tok = j * kKT + token(x);
      const int left = window.bad == 0 || window.good(tok >> shift) ? end - tok : 0;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        v[i] &= (2 * i < left ? 0xffffu : 0u) | (2 * i + 1 < left ? 0xffff0000u : 0u);
      if (not_finite<BF16>(v)) drop_not_finite<BF16>(v, tok, first + channel(x), any);
      *at = v;
    }
  }
};

// Writes a wave's 32 rows of 128 channels (o: the lane's row lane % 32, channels 32c + 8i +
// 4 * (lane / 32) + k in o[c][4i + k]) through `lds`, 8 KiB of the wave's own, so that 16
// lanes store a row's 256 bytes side by side. row: of the output, -1 for none; rows of
// `row_channels`, the first of them `channel`. Straight from the registers a workgroup took 5 us
// here, with its compute unit idle.
__device__ __forceinline__ void write_rows(u32x4* lds, const f32x16 (&o)[4], float by, int row,
                                           int row_channels, int channel, void* out,
                                           int out_dtype) {
  const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
  const int piece = lane & 15;
  auto store = [&](int bytes) {          // 32 rows of 256 bytes, `bytes` into the output's rows
#pragma unroll
    for (int it = 0; it < 8; ++it) {
      const int r = it * 4 + (lane >> 4);
      const u32x4 x = lds[r * 16 + (piece ^ (r & 15))];
      const int to = __shfl(row, r);
      const int64_t at = int64_t(to) * row_channels + channel;
      if (to >= 0)
        *reinterpret_cast<u32x4*>(static_cast<char*>(out) + at * (out_dtype == kOutF32 ? 4 : 2) +
                                  bytes + piece * 16) = x;
    }
  };
  if (out_dtype == kOutF32) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const f32x16& x = o[2 * h + c];
          lds[col * 16 + ((c * 8 + i * 2 + half) ^ (col & 15))] = __builtin_bit_cast(
              u32x4, f32x4{x[4 * i] * by, x[4 * i + 1] * by, x[4 * i + 2] * by, x[4 * i + 3] * by});
        }
      store(h * 256);
    }
    return;
  }
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int c = 0; c < 4; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = o[c][4 * i] * by, y = o[c][4 * i + 1] * by, z = o[c][4 * i + 2] * by,
                  w = o[c][4 * i + 3] * by;
      reinterpret_cast<u32x2*>(lds)[(col * 16 + ((c * 4 + i) ^ (col & 15))) * 2 + half] =
          out_dtype == kOutBF16 ? u32x2{pack16<true>(x, y), pack16<true>(z, w)}
                                : u32x2{pack16<false>(x, y), pack16<false>(z, w)};
    }
  store(0);
}

// Order of what the scheduler lays out next, `n` instructions at a time.
#define EMA_SCHED_VALU(n) __builtin_amdgcn_sched_group_barrier(0x2, n, 0)
#define EMA_SCHED_MFMA(n) __builtin_amdgcn_sched_group_barrier(0x8, n, 0)
#define EMA_SCHED_LDS_READ(n) __builtin_amdgcn_sched_group_barrier(0x100, n, 0)

// Makes the compiler wait here for a value that is still being loaded, instead of at
// its first use inside a loop, where the wait would catch the loop's own loads.
template <typename T>
__device__ __forceinline__ void arrived(T& x) {
  asm volatile("" : "+v"(x));
}

}  // namespace ema
