// What the kernels of rows.hip and tree.hip share: the sequences of a call, checked, and the cache's rows.
#pragma once
#include "rows.h"

#include "kernels.h"

namespace mpk {

__device__ __forceinline__ void report_rows(uint32_t* err, uint32_t code, uint32_t d0, uint32_t d1) {
  if (atomicCAS(&err[0], 0u, code) == 0u) {
    err[2] = d0;
    err[3] = d1;
  }
}

// The sequences of a call, checked: lane i of the wavefront holds sequence i.  A sequence that is left out has no rows
// (begin == end).  Every wavefront of every workgroup does this for itself: the loads are one round trip.
struct SeqLanes {
  int32_t begin, end, slot, pos;
};
template <bool TREE = false>   // TREE: a sequence's rows are a tree's nodes, kTreeNodes at most
__device__ __forceinline__ SeqLanes load_seqs(const RowSeqs& s, bool tell) {
  const int lane = threadIdx.x & 63;
  SeqLanes q = {0, 0, -1, 0};
  if ((uint32_t)lane < s.n_seqs) {
    q.begin = as_global(s.row_begin)[lane];
    q.end = as_global(s.row_begin)[lane + 1];
    q.slot = s.slots ? as_global(s.slots)[lane] : lane;
    q.pos = as_global(s.positions)[lane];
  }
  const uint64_t bad = __ballot(q.begin < 0 || q.end < q.begin || (uint32_t)q.end > s.n_rows);
  if (bad) {   // no row of the call belongs to anybody for sure
    const int at = __builtin_ctzll(bad);
    if (tell && lane == at) report_rows(s.err, DE_BAD_ROWS, (uint32_t)lane, (uint32_t)q.end);
    return SeqLanes{0, 0, -1, 0};
  }
  const int32_t n = q.end - q.begin;
  uint32_t wrong = DE_NONE, what = 0;
  if (n > 0) {
    if (q.slot < 0 || (uint32_t)q.slot >= s.batch) { wrong = DE_BAD_SLOT; what = (uint32_t)q.slot; }
    else if (q.pos < 0 || (uint32_t)q.pos >= s.max_seq || (uint32_t)n > s.max_seq - (uint32_t)q.pos) {
      wrong = DE_BAD_POSITION;
      what = q.pos < 0 || (uint32_t)q.pos >= s.max_seq ? (uint32_t)q.pos : s.max_seq;
    }
    else if (TREE && (uint32_t)n > kTreeNodes) { wrong = DE_BAD_TREE; what = (uint32_t)n; }
  }
  for (uint32_t i = 0; s.slots && i + 1 < s.n_seqs; ++i) {   // (a slot that an earlier sequence with rows has)
    const int32_t other = __builtin_amdgcn_readlane(q.slot, i), rows = __builtin_amdgcn_readlane(n, i);
    if (rows > 0 && n > 0 && (uint32_t)lane > i && q.slot == other && !wrong) { wrong = DE_BAD_SLOT; what = (uint32_t)q.slot; }
  }
  if (wrong) {
    if (tell) report_rows(s.err, wrong, (uint32_t)lane, what);
    q.end = q.begin;
  }
  return q;
}

__device__ __forceinline__ float uniform_f32(float v) { return __uint_as_float(uniform_u32(__float_as_uint(v))); }

// The sequence that row r belongs to (the last that begins at or before it and has it), 64: none.
__device__ __forceinline__ uint32_t seq_of_row(const SeqLanes& q, uint32_t r) {
  const uint64_t m = __ballot((uint32_t)q.begin <= r && r < (uint32_t)q.end);
  return m ? (uint32_t)__builtin_ctzll(m) : 64u;
}

// Element offset of cache row `row` of (slot, kv head); false: its page is outside the pool.
__device__ __forceinline__ bool cache_row(const RowSeqs& s, uint32_t slot, uint32_t kvh, uint32_t row, size_t* at) {
  if (!s.table) {
    *at = (((size_t)slot * s.n_kv + kvh) * s.max_seq + row) * s.head_dim;
    return true;
  }
  const int32_t page = as_global(s.table)[(size_t)slot * s.blocks + (row >> s.page_shift)];
  if (page < 0 || (uint32_t)page >= s.n_pages) return false;
  *at = ((((size_t)page * s.n_kv + kvh) << s.page_shift) + (row & ((1u << s.page_shift) - 1u))) * s.head_dim;
  return true;
}

// The parents of a tree's nodes, a wavefront's: lane l holds those of the nodes l, 64 + l, 128 + l and 192 + l (-1 behind the last).
struct TreeLanes {
  int32_t of[kTreeNodes / 64];
};
// A node's parent is an earlier node, or -1.  Returns the first node that has another, or the number of nodes.
__device__ __forceinline__ uint32_t load_tree(const int32_t* parents, uint32_t nodes, TreeLanes* tree) {
  const uint32_t lane = threadIdx.x & 63u;
  uint32_t wrong = nodes;
#pragma unroll
  for (uint32_t i = 0; i < kTreeNodes / 64u; ++i) {
    const uint32_t t = 64u * i + lane;
    tree->of[i] = t < nodes ? as_global(parents)[t] : -1;
  }
#pragma unroll
  for (uint32_t i = kTreeNodes / 64u; i-- > 0;) {
    const uint64_t bad = __ballot(tree->of[i] < -1 || tree->of[i] >= (int32_t)(64u * i + lane));
    if (bad) wrong = 64u * i + (uint32_t)__builtin_ctzll(bad);
  }
  return wrong;
}
// The parent of node t, the same for the wavefront.
__device__ __forceinline__ int32_t parent_of(const TreeLanes& tree, uint32_t t) {
  const uint32_t i = t >> 6;
  return __builtin_amdgcn_readlane(i == 0u ? tree.of[0] : i == 1u ? tree.of[1] : i == 2u ? tree.of[2] : tree.of[3], t & 63u);
}
// Ancestors of node t: its depth.
__device__ __forceinline__ uint32_t depth_of(const TreeLanes& tree, uint32_t t) {
  uint32_t depth = 0;
  for (int32_t p = parent_of(tree, t); p >= 0; p = parent_of(tree, (uint32_t)p)) ++depth;
  return depth;
}

}  // namespace mpk
