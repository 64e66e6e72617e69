// Block tables, slot maps and swap lists of a step, from the requests' lengths.
//
// A table is walked as one array of batch x max_blocks entries per layer, cut into
// chunks of 2048 or 4096 entries, one workgroup each. Request b's blocks begin at
// the prefix sum of the block counts before it, and its new tokens at that of
// the new lengths: every workgroup adds up the requests before its chunk (a few
// kilobytes, in cache) and scans its own. The k-th slice block of a layer is staged in
// place k, so a chunk has to know how many lie before it: where a layer has more than
// one chunk, a first launch leaves each chunk's three counts (slice blocks, those
// to prefetch, those to write back) in the workspace and the second adds up those
// before its own. Within a chunk the ranks come from ballots, in entry order: the
// lists' order does not depend on timing.
//
// There is no arithmetic to speak of: one request and one layer is latency (9.1 us with the
// launch: lengths, prefix, ids, stores), 80 layers of 128 requests (65 MB) take 15 + 31 us, of
// which the instructions of ballots, prefixes and searches are the most (VALU busy half of the
// time; memory 1.4 TB/s). The quotients by a reciprocal and the lists' counts added up without
// barriers took 51 us to 46.
#include "op_kernels.h"

namespace ema {
namespace {

constexpr int kWavesOf = kTableThreads / 64;

__device__ __forceinline__ int clampi(int x, int lo, int hi) {
  return x < lo ? lo : (x > hi ? hi : x);
}

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

// Set bits of m below the lane.
__device__ __forceinline__ int bits_below(unsigned long long m) {
  return __builtin_amdgcn_mbcnt_hi(uint32_t(m >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(m), 0));
}

// Sums of N values over the workgroup, for every thread. `s` holds N * kWavesOf ints.
template <int N>
__device__ __forceinline__ void block_sum(int (&x)[N], int* s) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int w = wave_inclusive_sum(x[n]);
    if (lane == 63) s[n * kWavesOf + wave] = w;
  }
  __syncthreads();
#pragma unroll
  for (int n = 0; n < N; ++n) {
    x[n] = 0;
#pragma unroll
    for (int w = 0; w < kWavesOf; ++w) x[n] += s[n * kWavesOf + w];
  }
}

struct Lens {
  int len, fresh;
};

// A request's lengths within what the table holds; *bad: they were not.
__device__ __forceinline__ Lens lens_of(const TablesArgs& a, int b, bool* bad) {
  const int cap = a.u.max_blocks * a.block_size;
  const int len = a.u.seq_lens[b], fresh = a.u.new_lens[b];
  const int l = clampi(len, 0, cap), f = clampi(fresh, 0, l);
  *bad = l != len || f != fresh;
  return {l, f};
}

__device__ __forceinline__ int blocks_of(const TablesArgs& a, int len) {
  return (len + a.block_size - 1) >> a.block_shift;
}

template <int ITEMS, bool COUNT>
// Registers for three workgroups to a CU: with two, large tables take a second round.
__global__ __launch_bounds__(kTableThreads, 6) void kv_tables_kernel(TablesArgs a) {
  constexpr int kChunk = kTableThreads * ITEMS;
  constexpr int kLists = ITEMS == 4 ? kChunk : kChunk / 8 + 1;  // requests of a chunk at most
  constexpr int kPer = (kLists + kTableThreads - 1) / kTableThreads;
  __shared__ int s_first[kLists + 2], s_qs[kLists + 2], s_old[kLists + 2];
  __shared__ int s_ids[kChunk];
  __shared__ int s_red[3 * kWavesOf];
  __shared__ int s_wave[3][kWavesOf];
  const ema_kv_tables_args& u = a.u;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int chunk = blockIdx.x, layer = blockIdx.y;
  const int B = u.batch, MB = u.max_blocks, BS = a.block_size;
  const int E = B * MB;                    // below 2^31: checked on the host
  const int e0 = chunk * kChunk, e1 = min(E, e0 + kChunk);
  const int b0 = E ? e0 / MB : 0;
  const int nloc = E ? (e1 - 1) / MB + 1 - b0 : 0;   // requests of the chunk, at most kLists + 1
  const bool staged = u.staging_slots > 0;

  // Everything that waits for nothing is sent for at once: the lengths of the chunk's own
  // requests (thread t takes consecutive ones), the counts of the layer's chunks, and the
  // lengths of all requests.
  const int per = (nloc + kTableThreads - 1) / kTableThreads;
  const int i0 = min(nloc, tid * per), i1 = min(nloc, i0 + per);
  Lens own[kPer + 1];
#pragma unroll
  for (int i = 0; i <= kPer; ++i) {
    own[i] = Lens{0, 0};
    bool bad;
    if (i0 + i < i1) own[i] = lens_of(a, b0 + i0 + i, &bad);
  }
  // of the layer's slice blocks, prefetches and write-backs, 0-2: those before the chunk, 3 and
  // 4: all prefetches and write-backs; every wave adds them up for itself
  int list[5] = {};
  if (!COUNT && staged && a.chunks > 1) {
    for (int c = lane; c < a.chunks; c += 64) {
#pragma unroll
      for (int x = 0; x < 3; ++x) {
        const int v = a.counts[(int64_t(layer) * a.chunks + c) * 3 + x];
        if (c < chunk) list[x] += v;
        if (x > 0) list[2 + x] += v;
      }
    }
#pragma unroll
    for (int x = 0; x < 5; ++x)
      list[x] = __builtin_amdgcn_readlane(wave_inclusive_sum(list[x]), 63);
  }
  // 0: blocks, 1: new tokens of the requests before the chunk; 2: new tokens of all
  int sum[3] = {};
  for (int b = tid; b < B; b += kTableThreads) {
    bool bad;
    const Lens l = lens_of(a, b, &bad);
    if (!COUNT && bad && chunk == 0 && layer == 0) atomicAdd(a.err_count, 1);
    if (b < b0) {
      sum[0] += blocks_of(a, l.len);
      sum[1] += l.fresh;
    }
    sum[2] += l.fresh;
  }
  int nb = 0, nf = 0;
#pragma unroll
  for (int i = 0; i <= kPer; ++i) {
    nb += blocks_of(a, own[i].len);
    nf += own[i].fresh;
    if (i0 + i < i1) s_old[i0 + i] = own[i].len - own[i].fresh;
  }
  const int ib = wave_inclusive_sum(nb), jf = wave_inclusive_sum(nf);
  if (lane == 63) {
    s_wave[0][wave] = ib;
    s_wave[1][wave] = jf;
  }
  block_sum(sum, s_red);                    // also makes s_wave visible
  const int total_new = sum[2];
  {
    int at_b = sum[0] + ib - nb, at_f = sum[1] + jf - nf;
    for (int w = 0; w < wave; ++w) {
      at_b += s_wave[0][w];
      at_f += s_wave[1][w];
    }
#pragma unroll
    for (int i = 0; i <= kPer; ++i) {
      if (i0 + i >= i1) continue;
      s_first[i0 + i] = at_b;
      s_qs[i0 + i] = at_f;
      at_b += blocks_of(a, own[i].len);
      at_f += own[i].fresh;
      if (i0 + i == nloc - 1) {
        s_first[nloc] = at_b;
        s_qs[nloc] = at_f;
      }
    }
    if (nloc == 0 && tid == 0) s_qs[0] = 0;
  }
  __syncthreads();

  // the entries: wave w takes ITEMS runs of 64 consecutive ones. Entry x of those from request
  // b0 on is request x / MB's, at most 4096 requests on: in 32-bit floats with a reciprocal off
  // by one step the quotient is off by 2^-10 at most, so its whole part by one.
  const int x0 = e0 - b0 * MB;
  const float inv_mb = __builtin_amdgcn_rcpf(float(MB));
  int id[ITEMS], rank[ITEMS][3];
  bool is[ITEMS][3];                 // in the slice; to prefetch; to write back
  int n[3] = {0, 0, 0};
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    const int e = e0 + (wave * ITEMS + k) * 64 + lane;
    id[k] = -1;
    bool away = false, older = false, touched = false;
    if (e < e1) {
      const int x = x0 + (e - e0);
      int i = int(float(x) * inv_mb), j = x - i * MB;
      if (j < 0) {
        --i;
        j += MB;
      } else if (j >= MB) {
        ++i;
        j -= MB;
      }
      const int f = s_first[i] + j;
      if (f < s_first[i + 1]) {
        const int v = f < u.n_ids ? u.block_ids[int64_t(layer) * u.n_ids + f] : -1;
        const bool ok = v >= 0 && v < a.n_total;
        if (!COUNT && !ok) atomicAdd(a.err_count, 1);
        id[k] = ok ? v : -1;
        away = staged && ok && v >= a.n_local;
        older = away && j * BS < s_old[i];
        touched = away && (j + 1) * BS > s_old[i] && s_qs[i + 1] > s_qs[i];
      }
    }
    is[k][0] = away;
    is[k][1] = older;
    is[k][2] = touched;
#pragma unroll
    for (int c = 0; c < 3; ++c) {
      const unsigned long long m = __ballot(is[k][c]);
      rank[k][c] = n[c] + bits_below(m);
      n[c] += __popcll(m);
    }
  }
  if (staged) {
    if (lane == 0) {
#pragma unroll
      for (int c = 0; c < 3; ++c) s_wave[c][wave] = n[c];
    }
    __syncthreads();
  }
  if constexpr (COUNT) {
    if (tid < 3) {
      int t = 0;
      for (int w = 0; w < kWavesOf; ++w) t += s_wave[tid][w];
      a.counts[(int64_t(layer) * a.chunks + chunk) * 3 + tid] = t;
    }
    return;
  }

  if (staged) {
    if (a.chunks == 1) {
#pragma unroll
      for (int x = 1; x < 3; ++x)
        for (int w = 0; w < kWavesOf; ++w) list[2 + x] += s_wave[x][w];
    }
    int base[3];
#pragma unroll
    for (int x = 0; x < 3; ++x) {
      base[x] = list[x];
      for (int w = 0; w < wave; ++w) base[x] += s_wave[x][w];
    }
    const int64_t pl = int64_t(layer) * u.stage_n, wl = int64_t(layer) * u.writeback_cap;
    const int32_t* places = u.staging_ids + int64_t(layer % u.staging_slots) * u.stage_n;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const int e = e0 + (wave * ITEMS + k) * 64 + lane;
      int entry = id[k];
      if (is[k][0]) {
        const int r = base[0] + rank[k][0];
        entry = r < u.stage_n ? places[r] : -1;
        if (entry < 0 || entry >= a.n_local) {
          atomicAdd(a.err_count, 1);
          entry = -1;
        }
        const int rp = base[1] + rank[k][1], rw = base[2] + rank[k][2];
        if (is[k][1] && rp < u.stage_n) {
          u.prefetch_src[pl + rp] = id[k];
          u.prefetch_dst[pl + rp] = entry;
        }
        if (is[k][2]) {
          if (rw < u.writeback_cap) {
            u.writeback_src[wl + rw] = entry;
            u.writeback_dst[wl + rw] = id[k];
          } else {
            atomicAdd(a.err_count, 1);
          }
        }
      }
      if (e < e1) {
        const int64_t at = int64_t(layer) * E + e;
        u.block_table[at] = entry;
        if (u.canon_table) u.canon_table[at] = id[k];
        s_ids[e - e0] = entry;
      }
    }
    const int n_pf = min(list[3], u.stage_n), n_wb = min(list[4], u.writeback_cap);
    if (chunk == 0 && tid == 0) {
      u.prefetch_n[layer] = n_pf;
      u.writeback_n[layer] = n_wb;
    }
    // -1 behind the lists, each chunk's share
    for (int64_t p = n_pf + int64_t(chunk) * kTableThreads + tid; p < u.stage_n;
         p += int64_t(a.chunks) * kTableThreads)
      u.prefetch_src[pl + p] = u.prefetch_dst[pl + p] = -1;
    for (int64_t p = n_wb + int64_t(chunk) * kTableThreads + tid; p < u.writeback_cap;
         p += int64_t(a.chunks) * kTableThreads)
      u.writeback_src[wl + p] = u.writeback_dst[wl + p] = -1;
  } else {
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
      const int e = e0 + (wave * ITEMS + k) * 64 + lane;
      if (e >= e1) continue;
      const int64_t at = int64_t(layer) * E + e;
      u.block_table[at] = id[k];
      if (u.canon_table) u.canon_table[at] = id[k];
      s_ids[e - e0] = id[k];
    }
  }
  __syncthreads();

  // slots of the new tokens in the chunk's blocks: a contiguous range of them
  auto token_at = [&](int e, int i) {      // first new token in entry e, of request b0 + i, or later
    const int f = s_qs[i + 1] - s_qs[i];
    return s_qs[i] + clampi((e - (b0 + i) * MB) * BS - s_old[i], 0, f);
  };
  const int t0 = E ? token_at(e0, 0) : 0;
  const int t1 = E ? (e1 == (b0 + nloc) * MB ? s_qs[nloc] : token_at(e1, nloc - 1)) : 0;
  int32_t* slots = u.slot_map + int64_t(layer) * u.n_slots;
  for (int t = t0 + tid; t < t1; t += kTableThreads) {
    int lo = 0, hi = nloc;                 // s_qs[lo] <= t < s_qs[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (s_qs[mid] <= t) lo = mid; else hi = mid;
    }
    const int p = s_old[lo] + t - s_qs[lo], j = p >> a.block_shift;
    const int v = s_ids[(b0 + lo) * MB + j - e0];
    const bool ok = v >= 0 && v < a.n_local;
    if (!ok || t >= u.n_slots) atomicAdd(a.err_count, 1);
    if (t < u.n_slots) slots[t] = ok ? v * BS + (p - j * BS) : -1;
  }
  for (int64_t t = total_new + int64_t(chunk) * kTableThreads + tid; t < u.n_slots;
       t += int64_t(a.chunks) * kTableThreads)
    slots[t] = -1;
  if (layer == 0) {
    for (int i = tid; i < nloc; i += kTableThreads)
      if ((b0 + i) * MB >= e0) u.query_start[b0 + i] = s_qs[i];
    if (chunk == 0 && tid == 0) u.query_start[B] = total_new;
  }
}

}  // namespace

namespace {

template <int ITEMS>
hipError_t launch(const TablesArgs& a, hipStream_t stream) {
  const dim3 grid(a.chunks, a.u.layers);
  if (a.chunks > 1 && a.u.staging_slots > 0) {
    hipLaunchKernelGGL((kv_tables_kernel<ITEMS, true>), grid, dim3(kTableThreads), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((kv_tables_kernel<ITEMS, false>), grid, dim3(kTableThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_tables(const TablesArgs& a, hipStream_t stream) {
  return table_items(a.u.layers, a.u.batch, a.u.max_blocks) == 4 ? launch<4>(a, stream)
                                                                : launch<8>(a, stream);
}

}  // namespace ema
