// Kept tokens moved together in the cache, in place: token base + k becomes what token
// base + keep[k] was. keep[k] >= k, and both ascend, so no place that a token is
// written to is read for a later one: a (layer, request, head) goes through its list
// in order, a chunk of it read before any of it is written, and the next chunk's loads
// are on their way while it is written.
//
// K is a row of 256 bytes per token and head in either layout. V is such a row in the
// token-major one, else a column of 128 elements, a row apart each: there a token shares every
// 32 to 128 bytes with its neighbours, and memory moves them whole.
//
// No arithmetic: bound by memory's lines and, long lists, by the chain list - table - tokens of a
// chunk. Accepted paths of 64 requests (4 of 16 nodes, 32 layers, 8 heads, 50 MB of K and V): 50-57
// us, nearly all of them the kernel, which writes 112 MB for V's lines (WRITE_SIZE) and reads 58 to
// 115 (FETCH_SIZE, or twice: it counts half of wide reads, and is not calibrated for narrow ones).
// 43 us where the call before has left the lines in the last-level cache. The same paths in an array
// of ten columns or more are a long list's work: 390 us.
// 8 contexts of 901-3501 tokens thinned to half (80 layers, 718 MB): 205 us, 3.5 TB/s.
#include "tree_kernels.h"

#include <algorithm>
#include <climits>

namespace ema {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;            // that move
// Columns of `keep` up to which the lists are short ones, whatever is in them. That there is such a
// border: 64 requests, 32 layers, 8 heads, all lists of 4 entries 50 us as short ones, 388 as long
// ones; of 9, 92 and 409. It is not the best one: short lists' form takes 126 us for 12 entries, 160
// for 16 and 272 for 28 (with room for 32), the long ones' 415, 422 and 442.
constexpr int kShort = 9;
constexpr int kBuffers = 4;

// Where a token is read or written.
struct Place {
  uint16_t* block;                       // nullptr: nothing to move
  int tok;                               // in the block
  int nhd;
};

// A request's list in one layer.
struct List {
  const int32_t *keep, *table;
  int base, n;                           // n: given, clamped
  int most;                              // entries before the end of the table
  int64_t room;                          // tokens of the table
  __device__ __forceinline__ List(const CompactArgs& a, int l, int b) {
    keep = a.keep + int64_t(b) * a.cap;
    table = a.table + (int64_t(l) * a.batch + b) * a.max_blocks;
    base = a.base[b];
    n = max(0, min(a.n_keep[b], a.cap));
    room = int64_t(a.max_blocks) << a.block_shift;
    most = base < 0 || base >= room ? 0 : int(min(int64_t(n), room - base));
  }
  // Where entry k's token comes from, in tokens from base on; k: it stays, or is out of range.
  __device__ __forceinline__ int source(int k, int& wrong) const {
    const int from = keep[k], before = k > 0 ? keep[k - 1] : -1;
    if (from >= k && from > before && int64_t(base) + from < room) return from;
    ++wrong;
    return k;
  }
  __device__ __forceinline__ bool place(const CompactArgs& a, int64_t t, Place& p) const {
    const PoolView& pv = a.pools;
    const int id = table[t >> a.block_shift];
    p.tok = int(t) & (pv.block_size - 1);
    p.nhd = id >= pv.n_local ? pv.slice_layout : 0;
    p.block = reinterpret_cast<uint16_t*>(
        id < 0 || id >= pv.n_local + pv.n_slice ? nullptr
        : id < pv.n_local ? pv.local + int64_t(id) * pv.block_bytes
                          : pv.slice + int64_t(id - pv.n_local) * pv.block_bytes);
    return p.block != nullptr;
  }
  // The places of entry k's move, if it has one; one that cannot be made is counted.
  __device__ __forceinline__ bool move(const CompactArgs& a, int k, bool counts, Place& src,
                                       Place& dst) const {
    int ignored = 0;
    const int from = source(k, ignored);
    if (from == k) return false;
    const bool s = place(a, int64_t(base) + from, src), d = place(a, int64_t(base) + k, dst);
    if (s && d) return true;
    if (counts) atomicAdd(a.err_count, 1);
    return false;
  }
  // What is out of range in the list itself, and the new length; by `threads` threads of the
  // request's first workgroup.
  __device__ __forceinline__ void report(const CompactArgs& a, int b, int threads) const {
    int wrong = 0;
    if (threadIdx.x == 0) {
      if (a.new_lens) a.new_lens[b] = int(uint32_t(base) + uint32_t(n));
      wrong = (base < 0) + (n != a.n_keep[b]);
    }
    if (base >= 0)
      for (int k = threadIdx.x; k < n; k += threads) source(k, wrong);
    if (wrong > 0) atomicAdd(a.err_count, wrong);
  }
};

// Elements of a place's K and V, of the block's head h.
struct Layout {
  int BS, H;
  int64_t half;
  __device__ __forceinline__ explicit Layout(const PoolView& pv)
      : BS(pv.block_size), H(pv.kv_heads), half(int64_t(pv.block_size) * pv.kv_heads * 128) {}
  __device__ __forceinline__ uint16_t* k(const Place& p, int h) const {
    return p.block + (p.nhd ? p.tok * H + h : h * BS + p.tok) * 128;
  }
  __device__ __forceinline__ uint16_t* v_row(const Place& p, int h) const {       // token-major
    return p.block + half + (p.tok * H + h) * 128;
  }
  __device__ __forceinline__ uint16_t* v_col(uint16_t* block, int tok, int h, int ch) const {
    return block + half + (h * 128 + ch) * BS + tok;
  }
};

// ---- short lists: an accepted path -------------------------------------------------------
//
// A workgroup takes heads of one (layer, request), as many at once as its threads hold of their
// elements: all is read, then all is written. Such a call is a chain of loads (list, table, tokens),
// so as many workgroups as possible run at once.
constexpr int kElements = 16;            // of V, of a thread

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

__global__ __launch_bounds__(kThreads, 8) void compact_short(CompactArgs a, int l0, int b0) {
  __shared__ Place s_src[kShort], s_dst[kShort];
  __shared__ int s_moves;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const int part = blockIdx.x, parts = gridDim.x, b = b0 + blockIdx.z, l = l0 + blockIdx.y;
  const Layout at(a.pools);
  const List list(a, l, b);
  if (part == 0 && l == 0) list.report(a, b, kThreads);
  if (tid < 64) {
    Place src{}, dst{};
    const bool moves = tid < list.most && list.move(a, tid, part == 0, src, dst);
    const unsigned long long m = __ballot(moves);
    if (moves) {
      const int e = __popcll(m & ((1ull << tid) - 1ull));
      s_src[e] = src;
      s_dst[e] = dst;
    }
    if (tid == 0) s_moves = __popcll(m);
  }
  __syncthreads();
  const int moves = uniform(s_moves);
  if (moves == 0) return;
  const int first = at.H * part / parts, end = at.H * (part + 1) / parts;
  const int each = kElements * kThreads / 128 / moves;     // heads at once
  const int inverse = 65536 / moves + 1;                   // r * inverse >> 16 = r / moves, r < 64
  // A row of V is half a workgroup's, so it is the same for all lanes of a wave.
  auto same = [&](const Place& p) {
    const uint64_t x = reinterpret_cast<uint64_t>(p.block);
    return Place{reinterpret_cast<uint16_t*>(uint64_t(uint32_t(uniform(int(uint32_t(x))))) |
                                             uint64_t(uint32_t(uniform(int(uint32_t(x >> 32))))) << 32),
                 uniform(p.tok), uniform(p.nhd)};
  };
  const int ch = (wave & 1) * 64 + lane;
  for (int h0 = first; h0 < end; h0 += each) {
    const int rows = min(each, end - h0) * moves;          // row r: head r / moves, entry r % moves
    u32x4 kx[2];
    uint16_t vx[kElements];
    auto v_at = [&](const Place& p, int h) -> uint16_t& {
      return p.nhd ? at.v_row(p, h)[ch] : at.v_col(p.block, p.tok, h, 0)[ch * at.BS];
    };
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = (i * kThreads + tid) >> 4, h = r * inverse >> 16;
      if (r < rows)
        kx[i] = *reinterpret_cast<const u32x4*>(at.k(s_src[r - h * moves], h0 + h) + (tid & 15) * 8);
    }
#pragma unroll
    for (int i = 0; i < kElements; ++i) {
      const int r = i * 2 + (wave >> 1), h = r * inverse >> 16;
      if (r < rows) vx[i] = v_at(same(s_src[r - h * moves]), h0 + h);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // read before any wave writes
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = (i * kThreads + tid) >> 4, h = r * inverse >> 16;
      if (r < rows)
        *reinterpret_cast<u32x4*>(at.k(s_dst[r - h * moves], h0 + h) + (tid & 15) * 8) = kx[i];
    }
#pragma unroll
    for (int i = 0; i < kElements; ++i) {
      const int r = i * 2 + (wave >> 1), h = r * inverse >> 16;
      if (r < rows) v_at(same(s_dst[r - h * moves]), h0 + h) = vx[i];
    }
  }
}

// ---- long lists ----------------------------------------------------------------------------
//
// A workgroup takes half of the channels, one a lane, of one head of a (layer, request) and goes
// through the list in chunks of up to 64 places. One wave makes the chunks, two ahead: the
// addresses of rows and pieces, and where in LDS a kept element will be. Four move them: what is
// the same for a wave's channels stays in scalar registers, because the instructions that find the
// places are what such a call has most of: with places in structures and a test for every element
// thinning took 507 us, so 301, and with the longest lists first 205.
constexpr int kChunk = 64;               // places
constexpr int kHalf = 64;                // channels
constexpr int kPieces = 24;              // of eight tokens, that a chunk reads at most
constexpr int kMovers = kThreads / 64;

struct Chunk {
  const char *k_src[kChunk], *piece[kChunk];   // rows of K; pieces of V, of channel 0
  char *k_dst[kChunk], *v_dst[kChunk];         // V: the piece of an entry's place, of channel 0
  int at[kChunk];                        // of an entry's V: bytes from channel 0's in LDS
  int pieces, last;
  unsigned long long moves, src_rows, dst_rows;   // entries to move; whose source, place is token-major
};

// A value of lane i, the same for all.
__device__ __forceinline__ uint64_t lane64(uint64_t x, int i) {
  return uint64_t(uint32_t(__builtin_amdgcn_readlane(int(uint32_t(x)), i))) |
         uint64_t(uint32_t(__builtin_amdgcn_readlane(int(uint32_t(x >> 32)), i))) << 32;
}

template <bool NHD>
__global__ __launch_bounds__(kThreads + 64, 4) void compact_long(CompactArgs a, int l0, int b0) {
  constexpr int kRowLoads = kChunk / 8 / kMovers;        // 8 rows of 128 bytes at once
  __shared__ Chunk s_list[kBuffers];
  // V: pieces as [piece][two tokens][channel], then rows as [entry][channel]
  constexpr int kRowsAt = kPieces * 4 * kHalf * 4;
  __shared__ __attribute__((aligned(16))) char s_v[kRowsAt + (NHD ? kChunk * kHalf * 2 : 0)];
  __shared__ int s_first;
  const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
  const bool maker = wave == kMovers;
  const Layout at(a.pools);
  const int h = int(blockIdx.x) >> 1, ch0 = (int(blockIdx.x) & 1) * kHalf;
  const int l = l0 + blockIdx.y;
  const bool counts = blockIdx.x == 0;
  // The longest lists first: they take the longest, and what is left over at the end of the launch
  // should be short ones.
  int b = b0 + blockIdx.z;
  if (a.batch <= kThreads) {
    int32_t* const counted = reinterpret_cast<int32_t*>(s_v);
    const int mine = tid < a.batch ? a.n_keep[tid] : 0;
    if (tid < a.batch) counted[tid] = mine;
    __syncthreads();
    int rank = 0;
    if (tid < a.batch) {
      for (int i = 0; i < a.batch; ++i)
        rank += counted[i] > mine || (counted[i] == mine && i < tid);
      if (rank == b0 + int(blockIdx.z)) s_first = tid;
    }
    __syncthreads();
    b = uniform(s_first);
    __syncthreads();
  }
  const List list(a, l, b);
  if (counts && l == 0) list.report(a, b, kThreads + 64);
  // the first entry that moves: all before it stay
  int k0 = 0;
  for (; k0 < list.most; k0 += kThreads + 64) {
    if (tid == 0) s_first = INT_MAX;
    __syncthreads();
    const int k = k0 + tid;
    int ignored = 0;
    const unsigned long long m = __ballot(k < list.most && list.source(k, ignored) != k);
    if (m != 0 && lane == 0) atomicMin(&s_first, k + int(__builtin_ctzll(m)));
    __syncthreads();
    const int found = s_first;
    __syncthreads();
    if (found != INT_MAX) {
      k0 = found;
      break;
    }
  }
  if (k0 >= list.most) return;
  // Chunks begin at a piece of the places that are written to.
  int64_t q = (int64_t(list.base) + k0) & ~7;            // the next one's, of the wave that makes them
  const int64_t end = int64_t(list.base) + list.most;
  auto make = [&](Chunk& x) {
    Place src{}, dst{};
    const int k = int(q + lane - list.base);
    bool moves = k >= k0 && k < list.most && list.move(a, k, false, src, dst);
    // an entry leads its piece if the one before has another; a piece's entries follow each other
    const uint64_t id = moves && !src.nhd
                            ? reinterpret_cast<uint64_t>(src.block) + uint64_t(src.tok & ~7) : 0;
    const uint64_t left = __shfl_up(id, 1);
    const bool leads = id != 0 && (lane == 0 || left != id);
    const unsigned long long lead = __ballot(leads);
    const int rank = __popcll(lead & ((2ull << lane) - 1ull)) - 1;     // of its piece
    // as many places, in eights, as have no more than kPieces
    int size = kChunk;
    while (__popcll(lead & (size == 64 ? ~0ull : (1ull << size) - 1ull)) > kPieces) size -= 8;
    moves = moves && lane < size;
    // moves that cannot be made: those of this chunk are counted now
    if (counts && k >= k0 && k < list.most && lane < size && !moves) {
      Place s2{}, d2{};
      list.move(a, k, true, s2, d2);
    }
    const unsigned long long all = __ballot(moves), sr = __ballot(moves && src.nhd),
                             dr = __ballot(moves && dst.nhd);
    if (moves) {
      x.k_src[lane] = reinterpret_cast<const char*>(at.k(src, h) + ch0);
      x.k_dst[lane] = reinterpret_cast<char*>(at.k(dst, h) + ch0);
      x.v_dst[lane] = reinterpret_cast<char*>(
          dst.nhd ? at.v_row(dst, h) + ch0 : at.v_col(dst.block, dst.tok & ~7, h, ch0));
      x.at[lane] = src.nhd ? kRowsAt + lane * kHalf * 2
                           : (rank * 4 + ((src.tok & 7) >> 1)) * kHalf * 4 + (src.tok & 1) * 2;
      if (leads)
        x.piece[rank] = reinterpret_cast<const char*>(at.v_col(src.block, src.tok & ~7, h, ch0));
    }
    q += size;
    if (lane == 0) {
      x.pieces = __popcll(lead & (size == 64 ? ~0ull : (1ull << size) - 1ull));
      x.moves = all;
      x.src_rows = sr;
      x.dst_rows = dr;
      x.last = q >= end;
    }
  };

  u32x4 kx[kRowLoads], rx[NHD ? kRowLoads : 1], vx[kPieces / kMovers];
  const int row8 = lane >> 3, part16 = (lane & 7) * 16;  // a lane's row of eight, its bytes there
  const int column = lane * at.BS * 2;                   // bytes from channel 0's to a lane's
  auto load = [&](const Chunk& x) {
    const unsigned long long moves = x.moves, rows = x.src_rows;
    const uint64_t pieces = reinterpret_cast<uint64_t>(x.piece[lane]);
    const int n = x.pieces;
#pragma unroll
    for (int i = 0; i < kRowLoads; ++i) {
      const int e = (i * kMovers + wave) * 8 + row8;
      if (moves >> e & 1) {
        const char* p = x.k_src[e] + part16;
        kx[i] = *reinterpret_cast<const u32x4*>(p);
        if (NHD && rows >> e & 1) rx[i] = *reinterpret_cast<const u32x4*>(p + at.half * 2);
      }
    }
#pragma unroll
    for (int i = 0; i < kPieces / kMovers; ++i)
      if (i * kMovers + wave < n)
        vx[i] = *reinterpret_cast<const u32x4*>(
            reinterpret_cast<const char*>(lane64(pieces, i * kMovers + wave)) + column);
  };

  if (maker) {
    make(s_list[0]);
    if (q < end) make(s_list[1]);
  }
  __syncthreads();
  if (!maker) load(s_list[0]);
  for (int buf = 0;; buf = (buf + 1) % kBuffers) {
    // A chunk is made two ahead: all are done with the one that had its place.
    const Chunk &x = s_list[buf], &next = s_list[(buf + 1) % kBuffers];
    const bool last = x.last != 0;
    if (maker) {
      if (q < end) make(s_list[(buf + 2) % kBuffers]);
      __syncthreads();
      __syncthreads();
      if (last) return;
      continue;
    }
    const unsigned long long moves = x.moves, src_rows = x.src_rows, dst_rows = x.dst_rows;
    const int n = x.pieces;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();                     // read by all; V of the chunk before has left LDS
#pragma unroll
    for (int i = 0; i < kPieces / kMovers; ++i) {
      const int p = i * kMovers + wave;
      if (p < n)
#pragma unroll
        for (int t = 0; t < 4; ++t)
          *reinterpret_cast<uint32_t*>(s_v + (p * 4 + t) * kHalf * 4 + lane * 4) = vx[i][t];
    }
#pragma unroll
    for (int i = 0; i < kRowLoads; ++i) {
      const int e = (i * kMovers + wave) * 8 + row8;
      if (!(moves >> e & 1)) continue;
      *reinterpret_cast<u32x4*>(x.k_dst[e] + part16) = kx[i];
      if (NHD && src_rows >> e & 1)
        *reinterpret_cast<u32x4*>(s_v + kRowsAt + e * kHalf * 2 + part16) = rx[i];
    }
    if (!last) load(next);
    __syncthreads();                     // the chunk's V is in LDS
    const int from = x.at[lane];
    const uint64_t to = reinterpret_cast<uint64_t>(x.v_dst[lane]);
    // entry e's element of this lane's channel
    auto element = [&](int e) {
      const int wide = NHD && src_rows >> e & 1 ? 1 : 2;
      return uint32_t(*reinterpret_cast<const uint16_t*>(
          s_v + __builtin_amdgcn_readlane(from, e) + (lane << wide)));
    };
    const unsigned long long cols = moves & ~dst_rows;
#pragma unroll
    for (int i = 0; i < kRowLoads; ++i) {
      const int e0 = (i * kMovers + wave) * 8;           // eight places of a channel
      const uint32_t in = uint32_t(cols >> e0) & 0xff;
      if (in == 0) continue;
      char* const p = reinterpret_cast<char*>(lane64(to, e0 + __builtin_ctz(in))) + column;
      if (in == 0xff) {
        uint32_t v[8];
#pragma unroll
        for (int t = 0; t < 8; ++t) v[t] = element(e0 + t);
        *reinterpret_cast<u32x4*>(p) =
            u32x4{v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16};
      } else {
        for (int t = 0; t < 8; ++t)
          if (in >> t & 1) *reinterpret_cast<uint16_t*>(p + t * 2) = uint16_t(element(e0 + t));
      }
    }
    if (NHD && dst_rows)
      for (int e = wave; e < kChunk; e += kMovers)       // a row's channels side by side
        if (dst_rows >> e & 1)
          *reinterpret_cast<uint16_t*>(reinterpret_cast<char*>(lane64(to, e)) + lane * 2) =
              uint16_t(element(e));
    if (last) return;
  }
}

template <typename Kernel>
hipError_t launch(Kernel kernel, const CompactArgs& a, int parts, int threads, hipStream_t stream) {
  // (a grid has fewer than 2^32 threads)
  const int batch = std::min(a.batch, 65535 / parts + 1);
  const int layers = std::max(1, std::min(a.layers, (1 << 22) / (parts * batch)));
  for (int l = 0; l < a.layers; l += layers)
    for (int b = 0; b < a.batch; b += batch) {
      hipLaunchKernelGGL(kernel, dim3(parts, std::min(layers, a.layers - l), std::min(batch, a.batch - b)),
                         dim3(threads), 0, stream, a, l, b);
      if (const hipError_t e = hipGetLastError()) return e;
    }
  return hipSuccess;
}

}  // namespace

hipError_t launch_kv_compact(const CompactArgs& a, hipStream_t stream) {
  if (a.batch <= 0) return hipSuccess;
  const int64_t lists = int64_t(a.layers) * a.batch;
  if (a.cap <= kShort) {
    // as many workgroups as run at once
    const int parts = int(std::max<int64_t>(1, std::min<int64_t>(a.pools.kv_heads, 2048 / lists)));
    return launch(compact_short, a, parts, kThreads, stream);
  }
  const int parts = a.pools.kv_heads * 2;
  return a.pools.slice_layout ? launch(compact_long<true>, a, parts, kThreads + 64, stream)
                              : launch(compact_long<false>, a, parts, kThreads + 64, stream);
}

}  // namespace ema
