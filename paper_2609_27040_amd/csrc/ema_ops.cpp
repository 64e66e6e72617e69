// Entry points of the operators declared in include/ema_ops.h, and of the attention of
// include/ema_tree.h: argument checks, then one launcher each.
#include "ema_ops.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <vector>

#include "op_checks.h"
#include "op_kernels.h"
#include "slice_handle.h"
#include "tree_kernels.h"

using ema::aligned16;
using ema::DeviceScope;
using ema::HostInts;
using ema::internal_error;
using ema::inval;
using ema::log2_of;
using ema::must_check;

namespace {

// ---- tables ---------------------------------------------------------------------

int tables_sizes(const ema_slice* h, const ema_kv_tables_args* u) {
  const char* what = "kv_tables";
  if (!h || !u) return inval(what, "NULL argument");
  if (u->layers < 1 || u->layers > 65535 || u->batch < 0 || u->max_blocks < 0 || u->n_ids < 0 ||
      u->n_slots < 0 || u->staging_slots < 0 || u->stage_n < 0 || u->writeback_cap < 0)
    return inval(what, "a size out of range");
  if (int64_t(u->batch) * u->max_blocks * h->shape.block_size >= (int64_t(1) << 31) ||
      (u->batch > 0 && u->max_blocks == 0))
    return inval(what, "batch * max_blocks * block_size must be in [1, 2^31)");
  if (int64_t(h->book.n_local()) * h->shape.block_size >= (int64_t(1) << 31))
    return inval(what, "the local pool has 2^31 rows or more");
  return EMA_OK;
}

size_t tables_bytes(const ema_kv_tables_args* u) {
  const int64_t chunks = ema::table_chunks(u->layers, u->batch, u->max_blocks);
  return u->staging_slots > 0 && chunks > 1 ? size_t(chunks) * u->layers * 3 * 4 : 0;
}

int check_tables(const ema_slice* h, const ema_kv_tables_args* u, hipStream_t st) {
  const char* what = "kv_tables";
  HostInts lens, fresh, ids, places;
  int rc;
  if ((rc = lens.get(h, u->seq_lens, u->batch, st)) ||
      (rc = fresh.get(h, u->new_lens, u->batch, st)) ||
      (rc = ids.get(h, u->block_ids, int64_t(u->layers) * u->n_ids, st)) ||
      (rc = places.get(h, u->staging_ids, int64_t(u->staging_slots) * u->stage_n, st)))
    return rc;
  const int32_t bs = h->shape.block_size, nl = h->book.n_local(), nt = nl + h->book.n_slice();
  int64_t blocks = 0, tokens = 0;
  for (int32_t b = 0; b < u->batch; ++b) {
    if (lens[b] < 0 || lens[b] > int64_t(u->max_blocks) * bs)
      return inval(what, "a length outside the table");
    if (fresh[b] < 0 || fresh[b] > lens[b]) return inval(what, "a new length outside its length");
    blocks += (lens[b] + bs - 1) / bs;
    tokens += fresh[b];
  }
  if (blocks > u->n_ids) return inval(what, "more blocks than block_ids holds");
  if (tokens > u->n_slots) return inval(what, "more new tokens than slot_map holds");
  for (int64_t i = 0; i < int64_t(u->staging_slots) * u->stage_n; ++i)
    if (places[i] < 0 || places[i] >= nl) return inval(what, "a staging id is not a local block");
  for (int32_t l = 0; l < u->layers; ++l) {
    int64_t f = int64_t(l) * u->n_ids, away = 0, back = 0;
    for (int32_t b = 0; b < u->batch; ++b) {
      const int32_t nb = (lens[b] + bs - 1) / bs, old = lens[b] - fresh[b];
      for (int32_t j = 0; j < nb; ++j, ++f) {
        if (ids[f] < 0 || ids[f] >= nt) return inval(what, "a block id outside both pools");
        const bool touched = fresh[b] > 0 && int64_t(j + 1) * bs > old;
        if (ids[f] < nl) continue;
        ++away;
        back += touched;
        if (touched && u->staging_slots == 0)
          return inval(what, "a new token in a slice block without staging");
      }
    }
    if (u->staging_slots > 0 && away > u->stage_n)
      return inval(what, "more slice blocks than stage_n");
    if (u->staging_slots > 0 && back > u->writeback_cap)
      return inval(what, "more write-backs than writeback_cap");
  }
  return EMA_OK;
}

// ---- attention -------------------------------------------------------------------

struct AttnCall {
  const char* what;
  int32_t maps;                  // 1 plain, 2 differential
  bool chunks;                   // query_start given
  ema_slice_t h;
  const void* q;
  int64_t q_stride;
  const int32_t *query_start, *block_table, *seq_lens;
  int32_t tokens, batch, num_q_heads, max_blocks;
  float scale;
  const float *lambda, *norm_weight;
  float norm_eps;
  void* out;
  int32_t out_dtype;
  void* workspace;
  size_t workspace_bytes;
  void* stream;
  bool tree = false;             // mask given
  const uint64_t* mask = nullptr;
  int32_t mask_words = 0;
};

int attn_sizes(const AttnCall& c) {
  if (!c.h) return inval(c.what, "NULL handle");
  const int32_t hkv = c.h->shape.num_kv_heads;
  if (c.tokens < 0 || c.batch < 0 || c.max_blocks < 0 || c.num_q_heads < hkv ||
      c.num_q_heads % hkv != 0 || c.num_q_heads > 4096)
    return inval(c.what, "bad tokens, batch, max_blocks or head counts");
  if (c.maps == 2 && hkv % 2 != 0) return inval(c.what, "the KV heads must pair up");
  if (!c.chunks && c.num_q_heads / hkv > 16)
    return inval(c.what, "more than 16 query heads per KV head");
  if (c.batch > 65535) return inval(c.what, "batch above 65535");
  if (int64_t(c.tokens) * c.num_q_heads >= (int64_t(1) << 29))
    return inval(c.what, "tokens * query heads must be below 2^29");
  if (int64_t(c.max_blocks) * c.h->shape.block_size > (int64_t(1) << 30))
    return inval(c.what, "max_blocks too large");
  // tiles of 32 tokens and a few more per (request, KV pair) are counted in 32 bits
  const int64_t tiles = int64_t(c.max_blocks) * c.h->shape.block_size / 32 + 8;
  if (!c.chunks && c.batch * tiles * (hkv / 2) >= (int64_t(1) << 31))
    return inval(c.what, "batch * max_blocks too large");
  if (c.tree && c.tokens > 0 && c.batch > 0) {
    ema::PromptArgs a{};
    a.tokens = c.tokens;
    a.batch = c.batch;
    a.q_heads = c.num_q_heads;
    a.kv_heads = hkv;
    a.block_size = c.h->shape.block_size;
    a.max_blocks = c.max_blocks;
    if (!ema::tree_fits(a)) return inval(c.what, "tokens or batch times max_blocks too large");
  }
  return EMA_OK;
}

ema::PromptArgs kernel_args(const AttnCall& c) {
  const ema_slice* h = c.h;
  ema::PromptArgs a{};
  a.q = static_cast<const char*>(c.q);
  a.q_stride = c.q_stride;
  a.starts = c.query_start;
  a.table = c.block_table;
  a.seq_lens = c.seq_lens;
  a.out = c.out;
  a.lam = c.lambda;
  a.norm_weight = c.norm_weight;
  a.norm_eps = c.norm_eps;
  const float sc = c.scale > 0.0f ? c.scale : 1.0f / std::sqrt(float(h->shape.head_dim));
  a.scale_log2 = sc * 1.4426950408889634f;
  a.err_count = h->d_err;
  a.local = h->local;
  a.block_bytes = h->bb;
  a.ws = static_cast<float*>(c.workspace);
  a.n_local = h->book.n_local();
  a.tokens = c.tokens;
  a.batch = c.batch;
  a.q_heads = c.num_q_heads;
  a.kv_heads = h->shape.num_kv_heads;
  a.block_size = h->shape.block_size;
  a.max_blocks = c.max_blocks;
  a.block_shift = log2_of(a.block_size);
  a.dtype = h->shape.dtype;
  a.out_dtype = c.out_dtype & ~EMA_FULL_WEIGHTS;
  a.full = c.out_dtype == EMA_F32 || (c.out_dtype & EMA_FULL_WEIGHTS) != 0;
  return a;
}

size_t attn_bytes(const AttnCall& c) {
  if (c.h->host_only || c.tokens == 0 || c.batch == 0) return 0;
  const ema::PromptArgs a = kernel_args(c);
  if (c.tree) return ema::tree_workspace(a);
  return c.maps == 1 ? ema::prompt_workspace(a)
                     : (c.chunks ? ema::diff_prompt_workspace(a) : ema::diff_workspace(a));
}

int workspace_call(const AttnCall& c, size_t* bytes) {
  if (!bytes) return inval(c.what, "NULL argument");
  if (int rc = attn_sizes(c)) return rc;
  *bytes = attn_bytes(c);
  return EMA_OK;
}

int check_attention(const AttnCall& c, hipStream_t st) {
  const ema_slice* h = c.h;
  HostInts starts, lens, table;
  int rc;
  if ((c.chunks && (rc = starts.get(h, c.query_start, int64_t(c.batch) + 1, st))) ||
      (rc = lens.get(h, c.seq_lens, c.batch, st)) ||
      (rc = table.get(h, c.block_table, int64_t(c.batch) * c.max_blocks, st)))
    return rc;
  const int32_t bs = h->shape.block_size;
  if (c.chunks && (starts[0] != 0 || starts[c.batch] > c.tokens))
    return inval(c.what, "query_start must run from 0 to at most the number of tokens");
  for (int32_t b = 0; b < c.batch; ++b) {
    if (lens[b] < 0 || lens[b] > int64_t(c.max_blocks) * bs)
      return inval(c.what, "a length outside the table");
    if (c.chunks && (starts[b + 1] < starts[b] || starts[b + 1] - starts[b] > lens[b]))
      return inval(c.what, "query_start descends, or has more queries than the request tokens");
    if (c.chunks && starts[b + 1] == starts[b]) continue;
    for (int32_t j = 0; j < (lens[b] + bs - 1) / bs; ++j) {
      const int32_t id = table[int64_t(b) * c.max_blocks + j];
      if (id < 0 || id >= h->book.n_local())
        return inval(c.what, "a block table entry is not a local block");
    }
  }
  return EMA_OK;
}

int attention(const AttnCall& c) {
  if (int rc = attn_sizes(c)) return rc;
  const ema_slice* h = c.h;
  const int32_t type = c.out_dtype & ~EMA_FULL_WEIGHTS;
  if (type != EMA_F32 && type != EMA_F16 && type != EMA_BF16)
    return inval(c.what, "out_dtype must be EMA_F32, EMA_F16 or EMA_BF16");
  if (!(c.norm_eps >= 0.0f)) return inval(c.what, "norm_eps must not be negative");
  if (c.tree && (c.mask_words < 1 || c.mask_words > EMA_TREE_WORDS))
    return inval(c.what, "mask_words must be in [1, EMA_TREE_WORDS]");
  if (c.tokens > 0 && c.batch > 0) {
    if ((!h->host_only && (!c.q || !c.out)) ||
        (!c.block_table && (!c.tree || c.max_blocks > 0)) || !c.seq_lens ||
        (c.chunks && !c.query_start) || (c.maps == 2 && !h->host_only && !c.lambda))
      return inval(c.what, "NULL array");
    if (c.q_stride < int64_t(c.num_q_heads) * h->shape.head_dim || c.q_stride % 8 != 0)
      return inval(c.what, "q_stride must be a multiple of 8 that holds a token's heads");
    if (!h->host_only && (!aligned16(c.q) || !aligned16(c.out) || !aligned16(c.norm_weight)))
      return inval(c.what, "q, out and norm_weight must be 16-byte aligned");
    if (c.tree && !h->host_only && (!c.mask || reinterpret_cast<uintptr_t>(c.mask) % 8 != 0))
      return inval(c.what, "mask missing or not 8-byte aligned");
  }
  if (c.tokens == 0 || c.batch == 0) return EMA_OK;
  if (!h->host_only && h->book.n_local() == 0) return inval(c.what, "the local pool is empty");
  hipStream_t st = static_cast<hipStream_t>(c.stream);
  DeviceScope ds;
  if (!h->host_only)
    if (int rc = ds.enter(h)) return rc;
  bool check = false;
  if (int rc = must_check(h, st, c.what, &check)) return rc;
  if (check)
    if (int rc = check_attention(c, st)) return rc;
  if (h->host_only) return EMA_OK;
  const size_t need = attn_bytes(c);
  if (need > 0 && (!c.workspace || c.workspace_bytes < need || !aligned16(c.workspace)))
    return inval(c.what, "workspace missing, too small or not 16-byte aligned");
  const ema::PromptArgs a = kernel_args(c);
  if (c.tree) {
    ema::TreeAttnArgs t{};
    static_cast<ema::PromptArgs&>(t) = a;
    t.mask = c.mask;
    t.words = c.mask_words;
    HIP_TRY(ema::launch_tree_attention(t, st), c.what);
    return EMA_OK;
  }
  HIP_TRY(c.maps == 1 ? ema::launch_prompt_attention(a, st)
                      : (c.chunks ? ema::launch_diff_prompt_attention(a, st)
                                  : ema::launch_diff_attention(a, st)),
          c.what);
  return EMA_OK;
}

}  // namespace

extern "C" {

int ema_kv_tables_workspace(ema_slice_t h, const ema_kv_tables_args* args, size_t* bytes) try {
  if (int rc = tables_sizes(h, args)) return rc;
  if (!bytes) return inval("kv_tables", "NULL argument");
  *bytes = h->host_only ? 0 : tables_bytes(args);
  return EMA_OK;
} catch (...) {
  return internal_error();
}

int ema_kv_tables(ema_slice_t h, const ema_kv_tables_args* args, void* workspace,
                  size_t workspace_bytes, void* stream) try {
  const char* what = "kv_tables";
  if (int rc = tables_sizes(h, args)) return rc;
  const ema_kv_tables_args& u = *args;
  const bool blocks = u.batch > 0;
  if (blocks && ((u.n_ids > 0 && !u.block_ids) || !u.seq_lens || !u.new_lens))
    return inval(what, "NULL array");
  if (u.staging_slots > 0 && u.stage_n > 0 && !u.staging_ids) return inval(what, "NULL array");
  if (!h->host_only) {
    if ((blocks && !u.block_table) || !u.query_start ||
        (u.n_slots > 0 && !u.slot_map))
      return inval(what, "NULL output");
    if (u.staging_slots > 0 &&
        (!u.prefetch_n || !u.writeback_n || (u.stage_n > 0 && (!u.prefetch_src || !u.prefetch_dst)) ||
         (u.writeback_cap > 0 && (!u.writeback_src || !u.writeback_dst))))
      return inval(what, "NULL list");
  }
  hipStream_t st = static_cast<hipStream_t>(stream);
  DeviceScope ds;
  if (!h->host_only)
    if (int rc = ds.enter(h)) return rc;
  bool check = false;
  if (int rc = must_check(h, st, what, &check)) return rc;
  if (check && u.batch > 0)
    if (int rc = check_tables(h, args, st)) return rc;
  if (h->host_only) return EMA_OK;
  const size_t need = tables_bytes(args);
  if (need > 0 && (!workspace || workspace_bytes < need || !aligned16(workspace)))
    return inval(what, "workspace missing, too small or not 16-byte aligned");
  ema::TablesArgs a{};
  a.u = u;
  a.n_local = h->book.n_local();
  a.n_total = a.n_local + h->book.n_slice();
  a.block_size = h->shape.block_size;
  a.block_shift = log2_of(a.block_size);
  a.chunks = ema::table_chunks(u.layers, u.batch, u.max_blocks);
  a.counts = static_cast<int32_t*>(workspace);
  a.err_count = h->d_err;
  HIP_TRY(ema::launch_kv_tables(a, st), what);
  return EMA_OK;
} catch (...) {
  return internal_error();
}

int ema_kv_store(ema_slice_t h, const void* k_new, int64_t k_stride, const void* v_new,
                 int64_t v_stride, const int32_t* slot_map, int32_t tokens, void* stream) try {
  const char* what = "kv_store";
  if (!h) return inval(what, "NULL handle");
  if (tokens < 0 || tokens >= 1 << 29) return inval(what, "tokens must be in [0, 2^29)");
  if (tokens == 0) return EMA_OK;
  const int64_t row = int64_t(h->shape.num_kv_heads) * h->shape.head_dim;
  if (!slot_map || (!h->host_only && (!k_new || !v_new))) return inval(what, "NULL array");
  if (k_stride < row || v_stride < row || k_stride % 8 != 0 || v_stride % 8 != 0)
    return inval(what, "a stride must be a multiple of 8 that holds a token's heads");
  if (!h->host_only && (!aligned16(k_new) || !aligned16(v_new)))
    return inval(what, "k_new and v_new must be 16-byte aligned");
  const int64_t rows = int64_t(h->book.n_local()) * h->shape.block_size;
  if (rows >= (int64_t(1) << 31)) return inval(what, "the local pool has 2^31 rows or more");
  hipStream_t st = static_cast<hipStream_t>(stream);
  DeviceScope ds;
  if (!h->host_only)
    if (int rc = ds.enter(h)) return rc;
  bool check = false;
  if (int rc = must_check(h, st, what, &check)) return rc;
  if (check) {
    HostInts slots;
    if (int rc = slots.get(h, slot_map, tokens, st)) return rc;
    std::vector<int32_t> used;
    for (int32_t t = 0; t < tokens; ++t) {
      if (slots[t] < -1 || slots[t] >= rows) return inval(what, "a slot past the local pool");
      if (slots[t] >= 0) used.push_back(slots[t]);
    }
    std::sort(used.begin(), used.end());
    if (std::adjacent_find(used.begin(), used.end()) != used.end())
      return inval(what, "a slot named twice");
  }
  if (h->host_only) return EMA_OK;
  ema::StoreArgs a{};
  a.k = static_cast<const uint16_t*>(k_new);
  a.v = static_cast<const uint16_t*>(v_new);
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.slots = slot_map;
  a.err_count = h->d_err;
  a.local = h->local;
  a.block_bytes = h->bb;
  a.n_slots = int32_t(rows);
  a.tokens = tokens;
  a.kv_heads = h->shape.num_kv_heads;
  a.block_size = h->shape.block_size;
  a.block_shift = log2_of(a.block_size);
  HIP_TRY(ema::launch_kv_store(a, st), what);
  return EMA_OK;
} catch (...) {
  return internal_error();
}

int ema_paged_prompt_workspace(ema_slice_t h, int32_t tokens, int32_t batch, int32_t num_q_heads,
                               int32_t max_blocks, size_t* bytes) try {
  AttnCall c{};
  c.what = "prompt_attention";
  c.maps = 1;
  c.chunks = true;
  c.h = h;
  c.tokens = tokens;
  c.batch = batch;
  c.num_q_heads = num_q_heads;
  c.max_blocks = max_blocks;
  return workspace_call(c, bytes);
} catch (...) {
  return internal_error();
}

int ema_paged_prompt_attention(ema_slice_t h, const void* q, int64_t q_stride,
                               const int32_t* query_start, const int32_t* block_table,
                               const int32_t* seq_lens, int32_t tokens, int32_t batch,
                               int32_t num_q_heads, int32_t max_blocks, float scale, void* out,
                               int32_t out_dtype, void* workspace, size_t workspace_bytes,
                               void* stream) try {
  return attention({"prompt_attention", 1, true, h, q, q_stride, query_start, block_table, seq_lens,
                    tokens, batch, num_q_heads, max_blocks, scale, nullptr, nullptr, 0.0f, out,
                    out_dtype, workspace, workspace_bytes, stream});
} catch (...) {
  return internal_error();
}

int ema_paged_diff_workspace(ema_slice_t h, int32_t batch, int32_t num_q_heads,
                             int32_t max_blocks, size_t* bytes) try {
  AttnCall c{};
  c.what = "diff_attention";
  c.maps = 2;
  c.h = h;
  c.tokens = c.batch = batch;
  c.num_q_heads = num_q_heads;
  c.max_blocks = max_blocks;
  return workspace_call(c, bytes);
} catch (...) {
  return internal_error();
}

int ema_paged_diff_attention(ema_slice_t h, const void* q, int64_t q_stride,
                             const int32_t* block_table, const int32_t* seq_lens, int32_t batch,
                             int32_t num_q_heads, int32_t max_blocks, float scale,
                             const float* lambda, const float* norm_weight, float norm_eps,
                             void* out, int32_t out_dtype, void* workspace,
                             size_t workspace_bytes, void* stream) try {
  return attention({"diff_attention", 2, false, h, q, q_stride, nullptr, block_table, seq_lens,
                    batch, batch, num_q_heads, max_blocks, scale, lambda, norm_weight, norm_eps, out,
                    out_dtype, workspace, workspace_bytes, stream});
} catch (...) {
  return internal_error();
}

int ema_paged_diff_prompt_workspace(ema_slice_t h, int32_t tokens, int32_t batch,
                                    int32_t num_q_heads, int32_t max_blocks, size_t* bytes) try {
  AttnCall c{};
  c.what = "diff_prompt_attention";
  c.maps = 2;
  c.chunks = true;
  c.h = h;
  c.tokens = tokens;
  c.batch = batch;
  c.num_q_heads = num_q_heads;
  c.max_blocks = max_blocks;
  return workspace_call(c, bytes);
} catch (...) {
  return internal_error();
}

int ema_paged_diff_prompt_attention(ema_slice_t h, const void* q, int64_t q_stride,
                                    const int32_t* query_start, const int32_t* block_table,
                                    const int32_t* seq_lens, int32_t tokens, int32_t batch,
                                    int32_t num_q_heads, int32_t max_blocks, float scale,
                                    const float* lambda, const float* norm_weight, float norm_eps,
                                    void* out, int32_t out_dtype, void* workspace,
                                    size_t workspace_bytes, void* stream) try {
  return attention({"diff_prompt_attention", 2, true, h, q, q_stride, query_start, block_table,
                    seq_lens, tokens, batch, num_q_heads, max_blocks, scale, lambda, norm_weight,
                    norm_eps, out, out_dtype, workspace, workspace_bytes, stream});
} catch (...) {
  return internal_error();
}

int ema_paged_tree_workspace(ema_slice_t h, int32_t tokens, int32_t batch, int32_t num_q_heads,
                             int32_t max_blocks, size_t* bytes) try {
  AttnCall c{};
  c.what = "tree_attention";
  c.maps = 1;
  c.chunks = true;
  c.tree = true;
  c.h = h;
  c.tokens = tokens;
  c.batch = batch;
  c.num_q_heads = num_q_heads;
  c.max_blocks = max_blocks;
  return workspace_call(c, bytes);
} catch (...) {
  return internal_error();
}

int ema_paged_tree_attention(ema_slice_t h, const void* q, int64_t q_stride,
                             const int32_t* query_start, const int32_t* block_table,
                             const int32_t* seq_lens, const uint64_t* mask, int32_t mask_words,
                             int32_t tokens, int32_t batch, int32_t num_q_heads,
                             int32_t max_blocks, float scale, void* out, int32_t out_dtype,
                             void* workspace, size_t workspace_bytes, void* stream) try {
  return attention({"tree_attention", 1, true, h, q, q_stride, query_start, block_table, seq_lens,
                    tokens, batch, num_q_heads, max_blocks, scale, nullptr, nullptr, 0.0f, out,
                    out_dtype, workspace, workspace_bytes, stream, true, mask, mask_words});
} catch (...) {
  return internal_error();
}

}  // extern "C"
