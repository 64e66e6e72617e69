// Launchers of the operators declared in ema_tree.h. All take device pointers and
// enqueue on `stream`; none allocates.
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>

#include "ema_tree.h"
#include "op_kernels.h"

namespace ema {

struct TreeTablesArgs {
  const int32_t* parents;      // [tokens]
  const int32_t* starts;       // [batch + 1]
  const int32_t* seq_lens;     // [batch]
  uint64_t* mask;              // [tokens][words]
  int32_t* positions;          // [tokens] or nullptr
  int32_t* base;               // [batch] or nullptr
  int32_t* err_count;
  int32_t tokens, batch, words;
};
hipError_t launch_tree_tables(const TreeTablesArgs& a, hipStream_t stream);

struct TreeAcceptArgs {
  const int32_t* parents;      // [tokens]
  const int32_t* starts;       // [batch + 1]
  const int32_t* drafted;      // [tokens]
  const int32_t* choice;       // [tokens]
  const int32_t* root_choice;  // [batch] or nullptr
  int32_t* path;               // [batch][cap]
  int32_t* n_path;             // [batch]
  int32_t* next;               // [batch]
  int32_t* err_count;
  int32_t tokens, batch, cap;
};
hipError_t launch_tree_accept(const TreeAcceptArgs& a, hipStream_t stream);

struct TreeAttnArgs : PromptArgs {
  const uint64_t* mask;        // [tokens][words]
  int32_t words;
};
// Whether the items' tiles, all added up, are below 2^30 (sizes of a launch set).
bool tree_fits(const PromptArgs& a);
size_t tree_workspace(const PromptArgs& a);
hipError_t launch_tree_attention(const TreeAttnArgs& a, hipStream_t stream);

struct CompactArgs {
  PoolView pools;
  const int32_t* table;        // [layers][batch][max_blocks]
  const int32_t* base;         // [batch]
  const int32_t* keep;         // [batch][cap]
  const int32_t* n_keep;       // [batch]
  int32_t* new_lens;           // [batch] or nullptr
  int32_t* err_count;
  int32_t layers, batch, max_blocks, cap;
  int32_t block_shift;         // log2(block_size)
};
hipError_t launch_kv_compact(const CompactArgs& a, hipStream_t stream);

}  // namespace ema
