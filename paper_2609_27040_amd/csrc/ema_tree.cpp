// Entry points of the trees and the compaction declared in include/ema_tree.h:
// argument checks, then one launcher each. (Attention: ema_ops.cpp.)
#include "ema_tree.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <initializer_list>
#include <utility>
#include <vector>

#include "op_checks.h"
#include "slice_handle.h"
#include "tree_kernels.h"

using ema::DeviceScope;
using ema::HostInts;
using ema::internal_error;
using ema::inval;
using ema::log2_of;
using ema::must_check;

namespace {

constexpr int32_t kMostBatch = 65535;

// n elements of an array, which may be missing.
struct Span {
  uintptr_t from, to;
  template <typename T>
  Span(const T* p, int64_t n)
      : from(reinterpret_cast<uintptr_t>(p)), to(p && n > 0 ? from + uintptr_t(n) * sizeof(T) : from) {}
  bool meets(const Span& o) const { return from < o.to && o.from < to; }
};

// Outputs that overlap each other or an input: a workgroup would read what another has written.
bool overlap(std::initializer_list<Span> outputs, std::initializer_list<Span> inputs) {
  for (const Span* a = outputs.begin(); a != outputs.end(); ++a) {
    for (const Span* b = a + 1; b != outputs.end(); ++b)
      if (a->meets(*b)) return true;
    for (const Span& b : inputs)
      if (a->meets(b)) return true;
  }
  return false;
}

// The starts and, of the nodes that are looked at, the parents.
int check_trees(const ema_slice* h, const char* what, const int32_t* parents,
                const int32_t* query_start, const int32_t* seq_lens, int32_t tokens, int32_t batch,
                int32_t most, hipStream_t st) {
  HostInts starts, up, lens;
  int rc;
  if ((rc = starts.get(h, query_start, int64_t(batch) + 1, st)) ||
      (rc = up.get(h, parents, tokens, st)) ||
      (seq_lens && (rc = lens.get(h, seq_lens, batch, st))))
    return rc;
  if (starts[0] != 0 || starts[batch] > tokens)
    return inval(what, "query_start must run from 0 to at most the number of tokens");
  for (int32_t b = 0; b < batch; ++b) {
    // (compared before they are subtracted; an entry past the last one would be read if the
    // starts did not ascend)
    if (starts[b + 1] < starts[b] || starts[b + 1] > tokens)
      return inval(what, "query_start descends");
    const int32_t n = starts[b + 1] - starts[b];
    if (seq_lens && lens[b] < n) return inval(what, "more nodes than the request has tokens");
    if (n > most) return inval(what, "more nodes than are looked at");
    for (int32_t i = 0; i < n; ++i)
      if (up[starts[b] + i] < -1 || up[starts[b] + i] >= i)
        return inval(what, "a parent that is not below its node");
  }
  return EMA_OK;
}

int check_lists(const ema_slice* h, const int32_t* block_table, const int32_t* base,
                const int32_t* keep, const int32_t* n_keep, int32_t layers, int32_t batch,
                int32_t max_blocks, int32_t keep_cap, hipStream_t st) {
  const char* what = "kv_compact";
  HostInts table, first, list, count;
  int rc;
  if ((rc = table.get(h, block_table, int64_t(layers) * batch * max_blocks, st)) ||
      (rc = first.get(h, base, batch, st)) ||
      (rc = list.get(h, keep, int64_t(batch) * keep_cap, st)) ||
      (rc = count.get(h, n_keep, batch, st)))
    return rc;
  const int32_t bs = h->shape.block_size, all = h->book.n_local() + h->book.n_slice();
  std::vector<std::pair<int32_t, int64_t>> used;   // a block, the entry that names it
  for (int32_t b = 0; b < batch; ++b) {
    const auto mine = int64_t(used.size());
    if (first[b] < 0) return inval(what, "a negative base");
    if (count[b] < 0 || count[b] > keep_cap) return inval(what, "n_keep outside [0, keep_cap]");
    for (int32_t k = 0; k < count[b]; ++k) {
      const int64_t e = int64_t(b) * keep_cap + k;
      if (list[e] < k || (k > 0 && list[e] <= list[e - 1]))
        return inval(what, "keep does not ascend");
      const int64_t from = int64_t(first[b]) + list[e];
      if (from >= int64_t(max_blocks) * bs) return inval(what, "a kept token past the table");
      if (list[e] == k) continue;
      for (int32_t l = 0; l < layers; ++l)
        for (int64_t t : {from, int64_t(first[b]) + k}) {
          const int64_t at = (int64_t(l) * batch + b) * max_blocks + t / bs;
          if (table[at] < 0 || table[at] >= all)
            return inval(what, "a table entry outside both pools");
          used.emplace_back(table[at], at);
        }
    }
    std::sort(used.begin() + mine, used.end());    // (a block has many tokens)
    used.erase(std::unique(used.begin() + mine, used.end()), used.end());
  }
  std::sort(used.begin(), used.end());
  for (size_t i = 1; i < used.size(); ++i)
    if (used[i].first == used[i - 1].first) return inval(what, "a block named twice");
  return EMA_OK;
}

}  // namespace

extern "C" {

int ema_tree_tables(ema_slice_t h, const int32_t* parents, const int32_t* query_start,
                    const int32_t* seq_lens, int32_t tokens, int32_t batch, uint64_t* mask,
                    int32_t mask_words, int32_t* positions, int32_t* base, void* stream) try {
  const char* what = "tree_tables";
  if (!h) return inval(what, "NULL handle");
  if (tokens < 0 || batch < 0 || batch > kMostBatch) return inval(what, "a size out of range");
  if (mask_words < 1 || mask_words > EMA_TREE_WORDS)
    return inval(what, "mask_words must be in [1, EMA_TREE_WORDS]");
  if (batch == 0) return EMA_OK;
  if (!query_start || !seq_lens || (tokens > 0 && !parents)) return inval(what, "NULL array");
  if (!h->host_only && tokens > 0 && (!mask || reinterpret_cast<uintptr_t>(mask) % 8 != 0))
    return inval(what, "mask missing or not 8-byte aligned");
  if (overlap({{mask, int64_t(tokens) * mask_words}, {positions, tokens}, {base, batch}},
              {{parents, tokens}, {query_start, int64_t(batch) + 1}, {seq_lens, batch}}))
    return inval(what, "an output overlaps another or an input");
  hipStream_t st = static_cast<hipStream_t>(stream);
  DeviceScope ds;
  if (!h->host_only)
    if (int rc = ds.enter(h)) return rc;
  bool check = false;
  if (int rc = must_check(h, st, what, &check)) return rc;
  if (check)
    if (int rc = check_trees(h, what, parents, query_start, seq_lens, tokens, batch,
                             64 * mask_words, st))
      return rc;
  if (h->host_only) return EMA_OK;
  ema::TreeTablesArgs a{};
  a.parents = parents;
  a.starts = query_start;
  a.seq_lens = seq_lens;
  a.mask = mask;
  a.positions = positions;
  a.base = base;
  a.err_count = h->d_err;
  a.tokens = tokens;
  a.batch = batch;
  a.words = mask_words;
  HIP_TRY(ema::launch_tree_tables(a, st), what);
  return EMA_OK;
} catch (...) {
  return internal_error();
}

int ema_tree_accept(ema_slice_t h, const int32_t* parents, const int32_t* query_start,
                    const int32_t* drafted, const int32_t* choice, const int32_t* root_choice,
                    int32_t tokens, int32_t batch, int32_t path_cap, int32_t* path,
                    int32_t* n_path, int32_t* next, void* stream) try {
  const char* what = "tree_accept";
  if (!h) return inval(what, "NULL handle");
  if (tokens < 0 || batch < 0 || batch > kMostBatch || path_cap < 1)
    return inval(what, "a size out of range");
  if (batch == 0) return EMA_OK;
  if (!query_start || (tokens > 0 && !parents)) return inval(what, "NULL array");
  if (!h->host_only && ((tokens > 0 && (!drafted || !choice)) || !path || !n_path || !next))
    return inval(what, "NULL array");
  if (overlap({{path, int64_t(batch) * path_cap}, {n_path, batch}, {next, batch}},
              {{parents, tokens}, {query_start, int64_t(batch) + 1}, {drafted, tokens},
               {choice, tokens}, {root_choice, batch}}))
    return inval(what, "an output overlaps another or an input");
  hipStream_t st = static_cast<hipStream_t>(stream);
  DeviceScope ds;
  if (!h->host_only)
    if (int rc = ds.enter(h)) return rc;
  bool check = false;
  if (int rc = must_check(h, st, what, &check)) return rc;
  if (check)
    if (int rc = check_trees(h, what, parents, query_start, nullptr, tokens, batch,
                             EMA_TREE_NODES, st))
      return rc;
  if (h->host_only) return EMA_OK;
  ema::TreeAcceptArgs a{};
  a.parents = parents;
  a.starts = query_start;
  a.drafted = drafted;
  a.choice = choice;
  a.root_choice = root_choice;
  a.path = path;
  a.n_path = n_path;
  a.next = next;
  a.err_count = h->d_err;
  a.tokens = tokens;
  a.batch = batch;
  a.cap = path_cap;
  HIP_TRY(ema::launch_tree_accept(a, st), what);
  return EMA_OK;
} catch (...) {
  return internal_error();
}

int ema_kv_compact(ema_slice_t h, const int32_t* block_table, const int32_t* base,
                   const int32_t* keep, const int32_t* n_keep, int32_t layers, int32_t batch,
                   int32_t max_blocks, int32_t keep_cap, int32_t* new_lens, void* stream) try {
  const char* what = "kv_compact";
  if (!h) return inval(what, "NULL handle");
  if (layers < 1 || layers > 65535 || batch < 0 || batch > kMostBatch || max_blocks < 0 ||
      keep_cap < 0)
    return inval(what, "a size out of range");
  if (batch == 0) return EMA_OK;
  if (int64_t(batch) * max_blocks * h->shape.block_size >= (int64_t(1) << 31))
    return inval(what, "batch * max_blocks * block_size must be below 2^31");
  if (!base || !n_keep || (keep_cap > 0 && !keep) || (max_blocks > 0 && !block_table))
    return inval(what, "NULL array");
  if (overlap({{new_lens, batch}},
              {{block_table, int64_t(layers) * batch * max_blocks}, {base, batch},
               {keep, int64_t(batch) * keep_cap}, {n_keep, batch}}))
    return inval(what, "new_lens overlaps an input");
  hipStream_t st = static_cast<hipStream_t>(stream);
  DeviceScope ds;
  if (!h->host_only)
    if (int rc = ds.enter(h)) return rc;
  bool check = false;
  if (int rc = must_check(h, st, what, &check)) return rc;
  if (check)
    if (int rc = check_lists(h, block_table, base, keep, n_keep, layers, batch, max_blocks,
                             keep_cap, st))
      return rc;
  if (h->host_only) return EMA_OK;
  ema::CompactArgs a{};
  a.pools = ema::pool_view(h);
  a.table = block_table;
  a.base = base;
  a.keep = keep;
  a.n_keep = n_keep;
  a.new_lens = new_lens;
  a.err_count = h->d_err;
  a.layers = layers;
  a.batch = batch;
  a.max_blocks = max_blocks;
  a.cap = keep_cap;
  a.block_shift = log2_of(h->shape.block_size);
  HIP_TRY(ema::launch_kv_compact(a, st), what);
  return EMA_OK;
} catch (...) {
  return internal_error();
}

}  // extern "C"
