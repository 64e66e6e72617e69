// What the matrix-core kernels of prompt chunks share (device code only): finding
// a workgroup's rows, staging K and V tiles in LDS, and their operands.
#pragma once

#include "attn_store.h"
#include "op_kernels.h"

namespace ema {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kKT = 64;                 // tokens of a staged tile
constexpr int kTilePieces = kKT * 16;   // 16-byte pieces of a tile's K, and of its V

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
__device__ __forceinline__ void drop_not_finite(u32x4& v, int tok, int* first) {
  constexpr uint32_t kExp = BF16 ? 0x7f80u : 0x7c00u;
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
};

// Which sequence holds tile `tile` of all sequences' tiles: every workgroup walks
// the starts, thread t `per` consecutive sequences.
template <int THREADS>
__device__ __forceinline__ RowTile find_tile(const PromptArgs& a, int group, int rows, int tile,
                                             int* s_scratch) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = (a.batch + THREADS - 1) / THREADS;
  const int b0 = min(a.batch, tid * per), b1 = min(a.batch, b0 + per);
  auto range = [&](int b, int& s, int& n) {
    if (!a.starts) {
      s = b;
      n = 1;
      return;
    }
    s = min(max(a.starts[b], 0), a.tokens);
    n = max(0, min(a.starts[b + 1], a.tokens) - s);
  };
  int total = 0;
  for (int b = b0; b < b1; ++b) {
    int s, n;
    range(b, s, n);
    total += (n * group + rows - 1) / rows;
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
  if (tile >= at && tile < at + total) {
    for (int b = b0; b < b1; ++b) {
      int s, n;
      range(b, s, n);
      const int t = (n * group + rows - 1) / rows;
      if (tile < at + t) {
        int* out = s_scratch + THREADS / 64;
        out[0] = b;
        out[1] = s;
        out[2] = n;
        out[3] = (tile - at) * rows;
        break;
      }
      at += t;
    }
  }
  __syncthreads();
  const int* in = s_scratch + THREADS / 64;
  RowTile r;
  r.b = uniform(in[0]);
  if (r.b < 0) return r;
  r.row0 = uniform(in[1]);
  r.n = uniform(in[2]);
  r.first = uniform(in[3]);
  r.len = uniform(max(0, min(a.seq_lens[r.b], a.max_blocks * a.block_size)));
  return r;
}
constexpr int kFindScratch = 16 + 4;

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
__device__ __forceinline__ int v_place(int ch, int group) {   // group: eight tokens of the tile
  constexpr int r = BSC / 8;
  const int f = r == 8 ? (ch >> 1) & 7 : r == 4 ? (ch >> 2) & 3 : (ch >> 3) & 1;
  return group / r * (128 * r) + ch * r + ((group % r) ^ f);
}

// Block ids of a tile, uniform over the wave: -1 for one that is out of range.
template <int BSC>
struct TileIds {
  static constexpr int N = kKT / BSC;    // blocks of a tile (one, of block size 64 on)
  int id[N];
};

// Ids of the tile at token t0, of which `end` tokens are there.
template <int BSC>
__device__ __forceinline__ TileIds<BSC> load_ids(const PromptArgs& a, const int32_t* row, int t0,
                                                 int end) {
  TileIds<BSC> r;
  const int last = (max(end, 1) - 1) / a.block_size;
#pragma unroll
  for (int i = 0; i < TileIds<BSC>::N; ++i) {
    // past the end: the last block again, whose rows are masked there
    const int j = min((t0 + i * BSC) / a.block_size, last);
    r.id[i] = row[j];
  }
  return r;
}

template <int BSC>
__device__ __forceinline__ void check_ids(const PromptArgs& a, TileIds<BSC>& t) {
#pragma unroll
  for (int i = 0; i < TileIds<BSC>::N; ++i)
    t.id[i] = uint32_t(t.id[i]) < uint32_t(a.n_local) ? t.id[i] : -1;
}

}  // namespace ema
