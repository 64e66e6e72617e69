// Launchers of the operators declared in ema_ops.h. All take device pointers and
// enqueue on `stream`; none allocates.
#pragma once

#include <hip/hip_runtime.h>
#include <cstdint>

#include "ema_ops.h"
#include "kernels.h"

namespace ema {

// ---- tables ------------------------------------------------------------------------

constexpr int kTableThreads = 512;

// Table entries that a thread takes, and with it a workgroup. Eight where there are enough of
// them for 512 workgroups and the rows are not too short for a workgroup's list of its
// requests, else four, so that small tables still spread over the chip. 80 layers of 128
// requests of up to 504 blocks, us a call with four / eight: 53 / 45.
inline int32_t table_items(int64_t layers, int64_t batch, int64_t max_blocks) {
  return max_blocks >= 8 && layers * batch * max_blocks >= 512 * kTableThreads * 8 ? 8 : 4;
}
inline int32_t table_chunks(int64_t layers, int64_t batch, int64_t max_blocks) {
  const int64_t chunk = kTableThreads * table_items(layers, batch, max_blocks);
  const int64_t n = (batch * max_blocks + chunk - 1) / chunk;
  return int32_t(n > 0 ? n : 1);
}
struct TablesArgs {
  ema_kv_tables_args u;
  int32_t n_local, n_total, block_size, block_shift;
  int32_t chunks;        // workgroups of a layer
  int32_t* counts;       // [layers][chunks][3] slice, prefetch and write-back entries
  int32_t* err_count;
};
hipError_t launch_kv_tables(const TablesArgs& a, hipStream_t stream);

// ---- store --------------------------------------------------------------------------

struct StoreArgs {
  const uint16_t* k;
  const uint16_t* v;
  int64_t k_stride, v_stride;   // elements between tokens
  const int32_t* slots;         // [tokens]
  int32_t* err_count;
  char* local;
  int64_t block_bytes;
  int32_t n_slots;              // rows of the local pool
  int32_t tokens, kv_heads, block_size;
  int32_t block_shift;          // log2(block_size)
};
hipError_t launch_kv_store(const StoreArgs& a, hipStream_t stream);

// ---- attention of chunks and differential attention -----------------------------------

struct PromptArgs {
  const char* q;               // 16-bit
  int64_t q_stride;            // elements between tokens
  const int32_t* starts;       // [batch + 1] rows of each sequence; nullptr: row b is sequence b
  const int32_t* table;        // [batch][max_blocks]
  const int32_t* seq_lens;     // [batch]
  void* out;
  const float* lam;            // [q_heads / 2]
  const float* norm_weight;    // [256] or nullptr
  float norm_eps;
  float scale_log2;            // softmax scale times log2(e)
  int32_t* err_count;
  const char* local;
  int64_t block_bytes;
  float* ws;
  int32_t n_local, tokens, batch, q_heads, kv_heads, block_size, max_blocks;
  int32_t block_shift;         // log2(block_size)
  int32_t dtype;               // 0 f16, 1 bf16
  int32_t out_dtype;           // kOutF32, kOutF16 or kOutBF16
  int32_t full;                // softmax weights of 32-bit accuracy
};
size_t prompt_workspace(const PromptArgs& a);
hipError_t launch_prompt_attention(const PromptArgs& a, hipStream_t stream);
size_t diff_workspace(const PromptArgs& a);
hipError_t launch_diff_attention(const PromptArgs& a, hipStream_t stream);
size_t diff_prompt_workspace(const PromptArgs& a);
hipError_t launch_diff_prompt_attention(const PromptArgs& a, hipStream_t stream);

}  // namespace ema
