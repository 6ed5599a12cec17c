// Rows beside the decode step (mpk_rows_*) and trees of drafted tokens (mpk_tree_*): what the host side hands to the kernels of
// rows.hip and tree.hip.
#pragma once
#include <hip/hip_runtime.h>

#include "mpk_internal.h"

namespace mpk {

constexpr uint32_t kMaxRowSeqs = 16;   // sequences of a call: at most a graph's batch
constexpr uint32_t kTreeNodes = MPK_TREE_MAX_NODES;   // nodes of a tree
// A graph's counters of the workgroups that have finished their part of a row, zero between calls; each on a line of its own (16
// rows of 32 parts: 11.0 us, counted on one line 15.4).
constexpr uint32_t kRowsArrivals = 1024, kArrivalStride = 32;

// The sequences of a call, on a layer's cache.
struct RowSeqs {
  const int32_t* row_begin;   // [n_seqs + 1]
  const int32_t* slots;       // [n_seqs] or null
  const int32_t* positions;   // [n_seqs]
  uint32_t n_seqs, n_rows;
  uint16_t* k;                // the layer's rows: [slot][kv head][max_seq][d], or pages [page][kv head][1 << page_shift][d]
  uint16_t* v;
  const int32_t* table;       // paged cache: [slot][blocks], else null
  uint32_t page_shift, n_pages, blocks;
  uint32_t n_q, n_kv, head_dim, batch, max_seq;
  uint32_t* err;
};

struct AppendArgs {
  RowSeqs s;
  const void* qkv;
  uint16_t* q_out;
  size_t qkv_stride, q_stride;   // elements
  const uint16_t *q_norm, *k_norm;   // null: no norm
  const double* inv_freq;
  float eps;
  const int32_t* parents;   // [n_rows]: the rows are nodes of trees; else null
};

struct AttendArgs {
  RowSeqs s;
  const uint16_t* q;
  uint16_t* out;
  size_t q_stride, out_stride;   // elements
  void* work;
  const int32_t* parents;   // as above
};

struct LogprobArgs {
  const void* logits;
  size_t stride;   // elements
  const int32_t* tokens;
  float *logprobs, *entropy;
  int32_t* top_tokens;
  float* top_logprobs;
  uint32_t n_rows, vocab, n_top;
  void* work;
  uint32_t *err, *arrivals;
};

// What the workgroups of a sequence exchange (tree.hip): the graph's own memory, for what an earlier call left there must not pass for a
// word of this one.
constexpr uint32_t kVerifyChunks = 128, kVerifyDepth = 4;   // chunks of a row at most
struct VerifySync {
  uint32_t tag, left;   // of the last round of the last call; workgroups that have left this one
  uint32_t pad[30];
  uint64_t word[kVerifyDepth][kVerifyChunks][8];   // of a round and those before it
};

struct VerifyArgs {
  const int32_t* row_begin;   // [n_seqs + 1]
  const int32_t *parents, *tokens;   // [n_rows]
  uint32_t n_seqs, n_rows, vocab, flags;
  const void* logits;
  const float* draft;            // null: the tokens were chosen, not drawn
  size_t stride, draft_stride;   // elements
  const float *temperatures, *uniforms;   // null: greedy
  int32_t *lengths, *path, *next;
  float* logprobs;   // or null
  uint32_t* err;
  VerifySync* sync;   // [n_seqs]
  bool jitter;        // delays at random (MPK_DEBUG_JITTER)
};

struct KeepArgs {
  RowSeqs s;   // (k, v: of layer 0)
  uint32_t n_layers;
  size_t layer_stride;   // elements of a layer's K or V
  const int32_t *lengths, *path;
  int32_t* positions_out;   // or null
};

// Before any of the others, with the device current: what the kernels need beyond the defaults, once per device.
hipError_t rows_prepare(int device);
// Each checks nothing (the entry points have) and launches on `stream`.
hipError_t launch_rows_append(const AppendArgs& a, bool f32, hipStream_t stream);   // (trees where a.parents is given, here and next)
hipError_t launch_rows_attend(const AttendArgs& a, hipStream_t stream);
hipError_t launch_rows_logprobs(const LogprobArgs& a, bool f32, hipStream_t stream);

hipError_t launch_tree_verify(const VerifyArgs& a, bool f32, hipStream_t stream);
hipError_t launch_tree_keep(const KeepArgs& a, hipStream_t stream);

}  // namespace mpk
