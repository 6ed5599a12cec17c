// Rows beside the decode step (mpk_rows_append, mpk_rows_attend, mpk_rows_logprobs): kernels and launches.
#include "rows.h"

#include <algorithm>
#include <mutex>
#include <vector>

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

// ------------------------------------------------------------------------------------ append
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) { return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b}); }   // to nearest even

// 8 neighbouring elements as fp32
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
  if constexpr (sizeof(T) == 4) {
    const u32x4 a = ((const MPK_GLOBAL u32x4*)p)[0], b = ((const MPK_GLOBAL u32x4*)p)[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[i] = __uint_as_float(a[i]); x[4 + i] = __uint_as_float(b[i]); }
  } else {
    const u32x4 a = *(const MPK_GLOBAL u32x4*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = bf16_lo(a[i]); x[2 * i + 1] = bf16_hi(a[i]); }
  }
}
__device__ __forceinline__ void store8(uint16_t* p, const float (&x)[8]) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
  *(MPK_GLOBAL u32x4*)p = w;
}

// q and k of a head, normed if the model has gains (x gain / sqrt(mean(x^2) + eps)), then pairs (x_i, x_{i + d/2}) turned by the
// angle position inv_freq[i], which is worked out and reduced to one turn in 64 bits.
// A wavefront takes one row and G groups of its heads; a group is 64 / LPH heads, a head LPH lanes, a lane 8
// elements of the head's lower half and the 8 they are rotated with.  Bound by memory: 8192 rows of 64 + 2 x 8 heads of 128, 336 MB
// read and written, 60 us, 5.6 TB/s (a copy of 1 GiB reaches 5.07: part of this fits the last cache).  Queries leave in bf16 whatever
// they come in, as the matrix cores take them.
template <typename T, int D, uint32_t G>
__global__ void __launch_bounds__(256) rows_append_kernel(AppendArgs a, uint32_t waves_per_row) {
  constexpr uint32_t LPH = D / 16, HPG = 64 / LPH, HALF = D / 2;
  __shared__ float2 angles[4][HALF];
  const RowSeqs& s = a.s;
  const uint32_t lane = threadIdx.x & 63u, wave = uniform_u32(threadIdx.x >> 6);
  const SeqLanes q = load_seqs(s, blockIdx.x == 0 && wave == 0);
  const uint32_t unit = blockIdx.x * 4u + wave, row = unit / waves_per_row, part = unit - row * waves_per_row;
  if (row >= s.n_rows) return;
  const uint32_t seq = seq_of_row(q, row);
  if (seq == 64u) return;
  const uint32_t pos = (uint32_t)__builtin_amdgcn_readlane(q.pos, seq) + row - (uint32_t)__builtin_amdgcn_readlane(q.begin, seq);
  const uint32_t slot = (uint32_t)__builtin_amdgcn_readlane(q.slot, seq);
  const uint32_t sub = lane & (LPH - 1u), heads = s.n_q + 2u * s.n_kv, e = 8u * sub;
  const T* x = (const T*)a.qkv + (size_t)row * a.qkv_stride;
  float lo[G][8], hi[G][8];   // (on their way while the angles are worked out)
#pragma unroll
  for (uint32_t g = 0; g < G; ++g) {
    const uint32_t h = min((part * G + g) * HPG + lane / LPH, heads - 1u);
    load8(x + (size_t)h * D + e, lo[g]);
    load8(x + (size_t)h * D + HALF + e, hi[g]);
  }
  if (lane < HALF) {
    const double two_pi = 6.283185307179586476925286766559;
    double ang = (double)(int32_t)pos * as_global(a.inv_freq)[lane];
    ang -= two_pi * rint(ang / two_pi);
    double sn, cs;
    sincos(ang, &sn, &cs);
    angles[wave][lane] = make_float2((float)cs, (float)sn);
  }
  float2 cs[8];
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int i = 0; i < 8; ++i) cs[i] = angles[wave][e + i];
  size_t at = 0;
  const bool cached = cache_row(s, slot, 0, pos, &at);
  if (!cached && lane == 0 && part == 0) report_rows(s.err, DE_BAD_PAGE, seq, pos);
  const size_t kv_head = s.table ? (size_t)D << s.page_shift : (size_t)D * s.max_seq;
#pragma unroll
  for (uint32_t g = 0; g < G; ++g) {
    const uint32_t h = (part * G + g) * HPG + lane / LPH;
    if (h >= heads) continue;
    const bool is_v = h >= s.n_q + s.n_kv, is_q = h < s.n_q;
    if (!is_v) {
      const uint16_t* gain = is_q ? a.q_norm : a.k_norm;
      if (gain) {
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = fmaf(hi[g][i], hi[g][i], fmaf(lo[g][i], lo[g][i], ss));
#pragma unroll
        for (uint32_t o = 1; o < LPH; o *= 2) ss += __shfl_xor(ss, o, 64);
        const float inv = 1.0f / sqrtf(ss * (1.0f / (float)D) + a.eps);
        float gl[8], gh[8];
        load8(gain + e, gl);
        load8(gain + HALF + e, gh);
#pragma unroll
        for (int i = 0; i < 8; ++i) { lo[g][i] = lo[g][i] * inv * gl[i]; hi[g][i] = hi[g][i] * inv * gh[i]; }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float l = lo[g][i], u = hi[g][i];
        lo[g][i] = fmaf(l, cs[i].x, -(u * cs[i].y));
        hi[g][i] = fmaf(u, cs[i].x, l * cs[i].y);
      }
    }
    uint16_t* to = nullptr;
    if (is_q) to = a.q_out + (size_t)row * a.q_stride + (size_t)h * D;
    else if (cached) to = (is_v ? s.v + at + (size_t)(h - s.n_q - s.n_kv) * kv_head : s.k + at + (size_t)(h - s.n_q) * kv_head);
    if (to) {
      store8(to + e, lo[g]);
      store8(to + HALF + e, hi[g]);
    }
  }
}

template <typename T, int D>
static hipError_t launch_append(const AppendArgs& a, hipStream_t stream) {
  const uint32_t groups = (a.s.n_q + 2u * a.s.n_kv + 1024u / D - 1u) / (1024u / D);
  // A wavefront more a row works out the row's angles once more; a group more a wavefront has fewer of them.  One / two / four groups a
  // wavefront (32 + 2 x 8 heads of 128, bf16): 256 rows 3.8 / 4.3 / - us, 512 4.7 / 5.1 / -, 1024 7.0 / 6.7 / 7.4, 2048 11.8 / 11.0 / 11.5,
  // 4096 19.7 / 18.4 / 19.9.
  const uint32_t per_wave = a.s.n_rows <= 512u ? 1u : 2u, waves_per_row = (groups + per_wave - 1u) / per_wave;
  const dim3 blocks((uint32_t)(((uint64_t)a.s.n_rows * waves_per_row + 3u) / 4u));
  if (per_wave == 1u) rows_append_kernel<T, D, 1><<<blocks, dim3(256), 0, stream>>>(a, waves_per_row);
  else rows_append_kernel<T, D, 2><<<blocks, dim3(256), 0, stream>>>(a, waves_per_row);
  return hipGetLastError();
}
hipError_t launch_rows_append(const AppendArgs& a, bool f32, hipStream_t stream) {
  if (a.s.head_dim == 128u) return f32 ? launch_append<float, 128>(a, stream) : launch_append<uint16_t, 128>(a, stream);
  return f32 ? launch_append<float, 64>(a, stream) : launch_append<uint16_t, 64>(a, stream);
}

// ------------------------------------------------------------------------------------ attend
// Queries of one KV head are rows of one product: row r of a sequence's T x grp is query head r % grp of token r / grp, so a
// tile of 128 rows reads each key once for all heads of the group.  A workgroup takes a tile and a run of blocks of 64 keys
// (a unit); its four wavefronts have 32 rows each.
//   S^T = K Q^T on v_mfma_f32_32x32x16_bf16: a lane then holds 16 keys of ONE row (lane & 31), so maximum, exponentials and
//   sum need one exchange between the two halves of the wavefront, and the probabilities, rounded to bf16, already are the
//   other operand of O^T = V^T P^T if the keys of a step are counted 8 (j / 4) + 4 half + j % 4.  V^T comes out of the row-major
//   tile by ds_read_b64_tr_b16.
// K and V tiles go from memory straight into LDS, the next block's while this one is worked on, their 16-byte pieces permuted
// (place ^ swizzle(row)) so that neither 16 rows at one place nor 4 rows at 64 bytes share a bank.
// What bounds it: many rows, the card's power, which takes the clock down to 1.8 GHz (2048 tokens over 14000 cached, 64 heads on 8 of 128,
// 1.01 TFLOP: 868 to 911 us, 1.11 to 1.16 PFLOP/s; a product of 8192^3 reaches 1.15 to 1.20 on such values in a long run, 1.42 in a short
// one, 1.71 on zeros).  Few rows, the cache's bytes behind 4.5 us to the first of them and 4 us of the join (8 sequences of up to 4096,
// 75.7 MB: 17.5 to 19.2 us on a cache that the last call left behind, 21 to 23 over ten layers' in turn).
// Rounded: the queries, which come in bf16, and the probabilities; all else is fp32.  In one term of bf16 a probability costs the output 0.0016
// of its size beside the 0.0016 of its own rounding (0.0018 to 0.0024 together, against 64 bits).  In two terms, V P_hi + V P_lo, 0.0016 in
// all, and half as many products again: one / two terms, 4096 tokens 136 / 192 us, 2048 over 14000 907 / 1311, 16 ragged prompts 147 / 200,
// 8 x 1 token 19.2 / 19.9, 5 over 30000 18.1 / 19.8.  (A decode step, which waits for memory, has three and fp32 queries.)
constexpr uint32_t kTileRows = 128, kBlockKeys = 64;
constexpr uint32_t kAttendMinBlocks = 3, kAttendMostChunks = 256;   // blocks of a run at least, runs of a tile at most
constexpr uint32_t kAttendJoinBlocks = 5;   // what the join costs, in blocks
constexpr float kAttendShare = 1.8e-4f;      // ... and a row's partial result
constexpr uint32_t kJoinWorkgroups = 1024;
// Rows and heads, up to as many as there are compute units, that get a workgroup each in the join (a wavefront / a workgroup each: 1 token
// over 30000, 32 heads of 128, 30.6 / 26.0 us; 5 over 30000 of 64 20.1 / 17.9; 8 over 8000, 256 of them, 18.4 / 17.0; 512 18.8 / 19.3; 1024 14.7 / 16.7).
constexpr uint32_t kJoinFewItems = 256;
constexpr uint32_t kAttendHeader = 1024;   // floats of the workspace in front of the partial results
constexpr uint32_t kAttendSlots = 512;   // workgroups that run at once: two a compute unit
// Calls of one tile a sequence wait for memory, and heads of 64 have room for three a compute unit (two / three: 16 x 1 token over 4000
// 29.6 / 26.6 us, over 12000 72.1 / 66.9, 8 x 1 over 512 to 4096 14.5 / 13.5; four: 26.7, 67.3, 13.7, but 5 over 30000 18.2 / 18.3 / 19.0).
constexpr uint32_t attend_slots(uint32_t D, bool once) { return D == 64u && once ? 768u : kAttendSlots; }
constexpr uint32_t kAttendFewChunks = 64;   // runs of such a tile at most, what a workgroup of the join reads at once (5 over 30000, 87 / 59 runs: 19.5 / 18.3)

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t lds_u32 __attribute__((address_space(3)));

// How a call's work is cut: every wavefront works it out for itself from the lanes' sequences (a lane each, 16 at most: a row of
// lanes).
struct Deal {
  uint32_t tiles, chunks, blocks;   // of the lane's sequence: row tiles, runs of blocks that the longest is cut into, blocks of a run
  uint32_t whole, units;            // runs that all tiles have; units, of one KV head
  uint32_t first_unit;              // units in front of the sequence's (of all KV heads)
  uint32_t part;                    // floats of the workspace in front of the sequence's partial results
  uint32_t total;                   // units of all
};
template <typename T, class Op>
__device__ __forceinline__ T row16_reduce(T v, Op op) {   // over the lane's row of 16
  auto dpp = [](T x, auto ctrl) { return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xF, 0xF, true)); };
  v = op(v, dpp(v, std::integral_constant<int, 0xB1>{}));
  v = op(v, dpp(v, std::integral_constant<int, 0x4E>{}));
  v = op(v, dpp(v, std::integral_constant<int, 0x141>{}));
  return op(v, dpp(v, std::integral_constant<int, 0x140>{}));
}
// Sum over the lanes in front, in the lane's row of 16.
__device__ __forceinline__ uint32_t row16_before(uint32_t v) {
  uint32_t x = v;
  auto add = [&](auto ctrl) { x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, 0xF, 0xF, true); };
  add(std::integral_constant<int, 0x111>{});   // row_shr 1, 2, 4, 8
  add(std::integral_constant<int, 0x112>{});
  add(std::integral_constant<int, 0x114>{});
  add(std::integral_constant<int, 0x118>{});
  return x - v;
}
// n / d for n below 2^24 (blocks of keys: the host refuses a max_seq above 2^28).  The compiler's division, right for any number, is forty
// operations, and there were six in front of a call's first load.
__device__ __forceinline__ uint32_t quotient(uint32_t n, uint32_t d) {
  uint32_t q = (uint32_t)((float)n * __builtin_amdgcn_rcpf((float)d));
  const int32_t r = (int32_t)(n - q * d);
  return r < 0 ? q - 1u : (uint32_t)r >= d ? q + 1u : q;
}
// First of the tiles that have a run k (of `blocks` blocks), for a run that not all have: a tile's last row sees key k blocks 64.
__device__ __forceinline__ uint32_t first_tile_of_run(uint32_t k, uint32_t blocks, uint32_t pos, uint32_t lg) {
  return ((k * blocks * kBlockKeys - pos) << lg) / kTileRows;
}
template <int D, bool ONCE>   // ONCE: no sequence has more than one tile
__device__ __forceinline__ Deal deal_units(const RowSeqs& s, const SeqLanes& q, uint32_t lg) {
  const uint32_t lane = threadIdx.x & 63u, T = (uint32_t)(q.end - q.begin), rows = T << lg;
  auto add = [](auto x, auto y) { return x + y; };
  constexpr uint32_t kSlots = attend_slots(D, ONCE);
  Deal d;
  d.tiles = ONCE ? min(T, 1u) : (rows + kTileRows - 1u) / kTileRows;
  const uint32_t nb = T ? ((uint32_t)q.pos + T + kBlockKeys - 1u) / kBlockKeys : 0u;
  const uint32_t few = row16_reduce(d.tiles, add) * s.n_kv;
  const float work = row16_reduce(T ? (float)d.tiles * (float)(((uint32_t)q.pos + T / 2u) / kBlockKeys + 1u) : 0.f, add) * (float)s.n_kv;
  // few tiles: at most as many units as run at once, all about as long (in 32 bits; no sequence has 2^22 blocks)
  uint32_t c = 1u + (uint32_t)(uniform_f32(work) * __builtin_amdgcn_rcpf((float)(few <= kSlots / 2u ? kSlots - few : kSlots)));
  // (That counts a whole run for the last of a tile.  As it is / shorter where that still fits: 4 x 1 token over 3000 15.9 / 15.3 us, 16 x 1 over 1000
  // 18.7 / 17.6, 8 x 1 over 512 to 4096 19.8 / 19.4.)
  if (ONCE && uniform_u32(few) <= kSlots / 2u && c > 1u) {
    if (uniform_u32(row16_reduce(d.tiles * quotient(nb + c - 2u, c - 1u), add)) * s.n_kv <= kSlots) c -= 1u;
  }
  // A run more is a partial result more of every tile, written and read: in blocks' time `share`, with all tiles of the call; and the
  // first cut is a second kernel.  So a run is no shorter than the square root that has blocks and partial results cost the same,
  // and a tile is cut only where that saves more than it costs.  Where a sequence has one tile at most and all run at once, the kernel
  // is not counted if another sequence needs it (counted / not: 8 x 1 token over 512 to 4096 21.8 / 19.8 us, heads of 64 17.2 / 14.5; with
  // several tiles a sequence 4 x 200 to 300 over 1000 to 3000 83 / 88).  (Cut into as many runs as run at once / as here: 512 tokens 25.6 /
  // 17.6 us, eight times 200 over 300 51 / 24; tiles of up to 22 blocks never cut / as here: 64 tokens over 1000 27.6 / 15.3.)
  const uint32_t held = min(rows, kTileRows);
  const float share = (float)few * (float)held * kAttendShare;
  c = max(min(max(c, kAttendMinBlocks), 1u << 22), 1u + (uint32_t)__builtin_amdgcn_sqrtf((float)nb * share));
  if (ONCE) c = max(c, (nb + kAttendFewChunks - 1u) / kAttendFewChunks);
  for (;; c *= 2u) {   // (long enough that the partial results fit the workspace, and a tile's weights the LDS of the join)
    d.chunks = quotient(nb + c - 1u, c);
    const float saved = (float)nb - (float)c - share * (float)d.chunks;
    if (saved < (ONCE && __any(saved >= (float)kAttendJoinBlocks) ? 0.f : (float)kAttendJoinBlocks)) d.chunks = 1u;
    const bool cut = T && d.chunks > 1u;
    const float need = cut ? (float)d.tiles * (float)d.chunks * (float)s.n_kv * (float)(held * (D + 2u)) : 0.f;
    if (uniform_f32(row16_reduce(need, add)) <= 0.99f * (float)(MPK_ROWS_WORKSPACE_BYTES / 4u) && __all(d.chunks <= kAttendMostChunks)) break;
  }
  d.blocks = max(1u, quotient(nb + d.chunks - 1u, d.chunks));
  d.chunks = T ? quotient(nb + d.blocks - 1u, d.blocks) : 0u;
  // a run whose first key lies behind the sequence's first new row is not every tile's
  if constexpr (ONCE) d.whole = d.units = d.chunks;
  else {
    d.whole = T ? min(d.chunks, quotient((uint32_t)q.pos / kBlockKeys, d.blocks) + 1u) : 0u;
    d.units = d.tiles * d.whole;
    for (uint32_t k = d.whole; k < d.chunks; ++k) d.units += d.tiles - first_tile_of_run(k, d.blocks, (uint32_t)q.pos, lg);
  }
  const uint32_t units = d.units * s.n_kv, floats = d.chunks > 1u ? d.tiles * d.chunks * s.n_kv * held * (D + 2u) : 0u;
  d.total = row16_reduce(units, add);
  d.part = row16_before(floats);
  d.first_unit = row16_before(units);
  if (uniform_u32(d.total) > kSlots) {   // not all at once: the sequences with more blocks first
    d.first_unit = 0;
    for (uint32_t i = 0; i < s.n_seqs; ++i) {
      const uint32_t onb = __builtin_amdgcn_readlane(nb, i), ou = __builtin_amdgcn_readlane(units, i);
      if (onb > nb || (onb == nb && i < lane)) d.first_unit += ou;
    }
  }
  return d;
}
// Blocks of keys that the rows of a tile see.
__device__ __forceinline__ uint32_t tile_blocks(uint32_t pos, uint32_t T, uint32_t tile, uint32_t lg) {
  const uint32_t t = min(T - 1u, (tile * kTileRows + kTileRows - 1u) >> lg);
  return (pos + t) / kBlockKeys + 1u;
}

template <int D>
__device__ __forceinline__ uint32_t swizzle(uint32_t row) {   // 16-byte piece c of a row of the tile lies at place c ^ swizzle(row)
  return D == 128 ? ((row & 3u) << 2) | ((row >> 2) & 3u) : (((row >> 1) & 1u) << 2) | ((row >> 2) & 3u);
}

// 1 KB of the wavefront's lanes' 16 bytes each into LDS at `to` (lane after lane).  Assembly text, for the compiler waits for a
// load into LDS before any later read of LDS that it cannot tell apart; who issues it waits (drain_vmem).  The text has the wait states
// that the compiler does not insert for it: five behind a vector operation that wrote the scalar registers (one would do for m0);
// m0 is named as lost, for the compiler joins writes of m0 across what it takes to leave it (the warning: m0 is not its to preserve).
// ONCE: what is read leaves the caches first.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
template <bool ONCE>
__device__ __forceinline__ void load_to_lds(const void* base, uint32_t off, uint32_t to) {
  const uint64_t p = (uint64_t)base;
  const u32x4 rsrc = {uniform_u32((uint32_t)p), uniform_u32((uint32_t)(p >> 32) & 0xFFFFu), 0x7FFFFFFFu, 0x00020000u};
  if constexpr (ONCE) asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds" ::"s"(uniform_u32(to)), "v"(off), "s"(rsrc) : "memory", "m0");
  else asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(uniform_u32(to)), "v"(off), "s"(rsrc) : "memory", "m0");
}
#pragma clang diagnostic pop

// The largest of three, a NaN left out; one operation, v_max3_f32.  Not as assembly text: the compiler puts the wait states between a
// matrix instruction and the first reader of its results only where it knows the reader.
__device__ __forceinline__ float max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }

__device__ __forceinline__ uint32_t nonfinite(uint32_t w) { return ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u; }   // bit 15 / 31: lower / upper

// ONCE: no sequence has more than one tile, so that a unit's keys are its own.
template <int D, bool PAGED, bool ONCE>
__global__ void __launch_bounds__(256, 2) rows_attend_kernel(AttendArgs a, uint32_t lg) {
  constexpr uint32_t KS = D / 16, NT = D / 32, CPR = D / 8, RPI = 64 / CPR, IPW = 16 / RPI, ROWB = D * 2, TILE = kBlockKeys * ROWB;
  extern __shared__ __align__(16) unsigned char tiles_lds[];   // K, V of the even blocks, K, V of the odd ones, a flag
  uint32_t& flag = *(uint32_t*)(tiles_lds + 4u * TILE);
  const RowSeqs& s = a.s;
  const uint32_t lane = threadIdx.x & 63u, wave = uniform_u32(threadIdx.x >> 6), l31 = lane & 31u, half = lane >> 5;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)tiles_lds;
  __builtin_amdgcn_s_setprio(3);   // (until the unit's first requests are out: 8 x 1 token 20.3 / 19.6 us)
  const SeqLanes q = load_seqs(s, blockIdx.x == 0 && wave == 0);
  const Deal d = deal_units<D, ONCE>(s, q, lg);
  const uint32_t total = uniform_u32(d.total);
  if (blockIdx.x == 0 && threadIdx.x < kMaxRowSeqs) {   // what the join needs of it
    MPK_GLOBAL u32x4* to = as_global((u32x4*)a.work) + 2u * threadIdx.x;
    to[0] = u32x4{(uint32_t)q.begin, (uint32_t)q.end, (uint32_t)q.pos, d.chunks};
    to[1] = u32x4{d.blocks, d.part, 0u, 0u};
  }
  const float scale2 = 1.44269504088896340736f / sqrtf((float)D);   // scores count in powers of two

  for (uint32_t u = blockIdx.x; u < total; u += gridDim.x) {
    // ---- the unit: sequence, tile of rows (the longest first), run of blocks, KV head (the one that neighbours in time share an L2 for)
    const uint32_t mine = d.units * s.n_kv;
    const uint32_t seq = (uint32_t)__builtin_ctzll(__ballot(mine && u >= d.first_unit && u < d.first_unit + mine));
    const uint32_t T = __builtin_amdgcn_readlane((uint32_t)(q.end - q.begin), seq), pos0 = __builtin_amdgcn_readlane(q.pos, seq);
    const uint32_t slot = __builtin_amdgcn_readlane(q.slot, seq), begin = __builtin_amdgcn_readlane(q.begin, seq);
    const uint32_t chunks = __builtin_amdgcn_readlane(d.chunks, seq), per = __builtin_amdgcn_readlane(d.blocks, seq);
    const uint32_t tiles = __builtin_amdgcn_readlane(d.tiles, seq), whole = __builtin_amdgcn_readlane(d.whole, seq);
    const uint32_t v = u - __builtin_amdgcn_readlane(d.first_unit, seq), kvh = v % s.n_kv;
    uint32_t w = v / s.n_kv, chunk = w / tiles;
    if (ONCE) { chunk = w; w = 0; }
    else if (chunk < whole) w -= chunk * tiles;
    else {
      w -= whole * tiles;
      for (chunk = whole;; ++chunk) {
        const uint32_t n = tiles - first_tile_of_run(chunk, per, pos0, lg);
        if (w < n) break;
        w -= n;
      }
    }
    const uint32_t tile = ONCE ? 0u : tiles - 1u - w;
    const uint32_t nb = tile_blocks(pos0, T, tile, lg), b0 = chunk * per, b1 = min(nb, b0 + per);
    const uint32_t rows = T << lg, last = pos0 + T - 1u;   // the sequence's last row in the cache
    const uint32_t w0 = tile * kTileRows + wave * 32u;   // the wavefront's rows: none behind `rows`
    const bool have = w0 < rows;
    const uint32_t pos_lo = pos0 + (min(w0, rows - 1u) >> lg), pos_hi = pos0 + (min(w0 + 31u, rows - 1u) >> lg);
    const uint32_t tile_lo = pos0 + ((tile * kTileRows) >> lg);
    // ---- tiles of keys and values: this wavefront's 16 rows of a block
    const uint16_t *kbase, *vbase;
    const size_t head_at = PAGED ? ((size_t)kvh << s.page_shift) * D : ((size_t)slot * s.n_kv + kvh) * s.max_seq * D;
    kbase = s.k + head_at;
    vbase = s.v + head_at;
    uint32_t voff[IPW], jrow[IPW];
#pragma unroll
    for (uint32_t i = 0; i < IPW; ++i) {
      jrow[i] = lane / CPR;
      voff[i] = ((lane % CPR) ^ swizzle<D>(wave * 16u + i * RPI + lane / CPR)) * 16u;
    }
    uint32_t page[2] = {0, 0};
    auto fetch_pages = [&](uint32_t b) {   // of the two runs of 8 rows (a page has 8 at least)
      if constexpr (PAGED) {
#pragma unroll
        for (uint32_t g = 0; g < 2; ++g)
          page[g] = ld_u32c((const uint32_t*)s.table + (size_t)slot * s.blocks + (min(b * kBlockKeys + wave * 16u + g * 8u, last) >> s.page_shift));
      }
    };
    auto request = [&](uint32_t b, uint32_t buf) {
      uint32_t pg[2] = {page[0], page[1]};
      if constexpr (PAGED) {
#pragma unroll
        for (uint32_t g = 0; g < 2; ++g)
          if (pg[g] >= s.n_pages) {
            if (lane == 0) report_rows(s.err, DE_BAD_PAGE, seq, min(b * kBlockKeys + wave * 16u + g * 8u, last));
            pg[g] = 0;
          }
      }
      const bool whole = b * kBlockKeys + kBlockKeys - 1u <= last;
#pragma unroll
      for (uint32_t i = 0; i < IPW; ++i) {
        const uint32_t r0 = b * kBlockKeys + wave * 16u + i * RPI, c0 = min(r0, last);
        // rows behind the last one are the last one: nothing beyond what has been appended is ever read
        const uint32_t j = whole ? jrow[i] : min(r0 + jrow[i], last) - c0;
        const size_t at = PAGED ? (((size_t)pg[i * RPI / 8u] * s.n_kv << s.page_shift) + (c0 & ((1u << s.page_shift) - 1u))) * D : (size_t)c0 * D;
        const uint32_t to = lds0 + buf * 2u * TILE + (wave * IPW + i) * 1024u, off = j * ROWB + voff[i];
        load_to_lds<ONCE>(kbase + at, off, to);
        load_to_lds<ONCE>(vbase + at, off, to + TILE);
      }
    };
    fetch_pages(b0);
    request(b0, 0);
    fetch_pages(min(b0 + 1u, b1 - 1u));
    // ---- queries: B operand, lane = row, 8 columns a step and half
    const uint32_t r = tile * kTileRows + wave * 32u + l31, rr = min(r, rows - 1u), t = rr >> lg;
    const uint32_t head = (kvh << lg) + (rr & ((1u << lg) - 1u)), pos = pos0 + t;
    u32x4 qf[KS];
    {
      const uint16_t* p = a.q + (size_t)(begin + t) * a.q_stride + (size_t)head * D + 8u * half;
#pragma unroll
      for (uint32_t k = 0; k < KS; ++k) qf[k] = *as_global((const u32x4*)(p + 16u * k));
    }

    f32x16 o[NT];
#pragma unroll
    for (uint32_t n = 0; n < NT; ++n) o[n] = f32x16{};
    float m = -3.402823466e38f, lsum = 0.f;   // of the lane's row (the sum: of the lane's keys)
    const uint32_t krow = l31 * ROWB, kx = (half ^ swizzle<D>(l31)) * 16u;
    const uint32_t rl = (lane & 15u) >> 2, un = 2u * ((lane >> 4) & 1u) + ((lane & 3u) >> 1);
    uint32_t vat[NT][2];   // of the lane's 8 bytes of a step of 16 keys: columns 32 n .., keys 8 x + 4 half ..
#pragma unroll
    for (uint32_t n = 0; n < NT; ++n)
#pragma unroll
      for (uint32_t x = 0; x < 2; ++x) {
        const uint32_t place = ((n ^ (D == 128 ? rl : rl >> 1)) << 2) | (un ^ (half + 2u * x));
        vat[n][x] = (8u * x + 4u * half + rl) * ROWB + place * 16u + 8u * (lane & 1u);
      }
    __builtin_amdgcn_s_setprio(0);
    drain_vmem();
    __syncthreads();

    for (uint32_t b = b0; b < b1; ++b) {
      const uint32_t buf = (b - b0) & 1u, kv0 = b * kBlockKeys;
      if (b + 1u < b1) {
        request(b + 1u, buf ^ 1u);
        fetch_pages(min(b + 2u, b1 - 1u));
      }
      const uint32_t kt = lds0 + buf * 2u * TILE, vt = kt + TILE;
      bool poisoned = false;
      if (kv0 + kBlockKeys - 1u > tile_lo) {   // some row does not see all of the block
        // 0 x NaN is NaN: a value that is not finite must not meet the zero probability of a row that does not see it.  Such
        // values are taken out of the tile and added below to the rows that do.
        lds_u32* p = (lds_u32*)(uintptr_t)(vt + threadIdx.x * (TILE / 256u));
        uint32_t bad = 0;
#pragma unroll
        for (uint32_t i = 0; i < TILE / 1024u; ++i) bad |= nonfinite(p[i]);
        if (threadIdx.x == 0) flag = 0;
        __syncthreads();
        if (bad) flag = 1;
        __syncthreads();
        poisoned = flag != 0;
        if (__builtin_expect(poisoned, 0)) {
          for (uint32_t i = 0; i < TILE / 1024u; ++i) {
            const uint32_t x = p[i], n = nonfinite(x);
            p[i] = x & ~(((n & 0x8000u) ? 0xFFFFu : 0u) | ((n & 0x80000000u) ? 0xFFFF0000u : 0u));
          }
          __syncthreads();
        }
      }
      if (have && kv0 <= pos_hi) {
        // A SIMD has a wavefront of each of two workgroups.  One that multiplies goes first, one that works out probabilities before
        // one that requests or waits: the matrix pipe is fed while the other's vector operations fill its gaps (priorities all
        // alike / as here: 4096 tokens 156 / 144 us, 2048 over 14000 976 / 915; multiplies alone preferred 153 / 969).
        __builtin_amdgcn_s_setprio(2);
        f32x16 sc[2] = {f32x16{}, f32x16{}};
#pragma unroll
        for (uint32_t k = 0; k < KS; ++k) {
#pragma unroll
          for (uint32_t n = 0; n < 2; ++n) {
            const u32x4 kf = *(__attribute__((address_space(3))) u32x4*)(uintptr_t)(kt + ((krow + kx) ^ (32u * k)) + n * 32u * ROWB);
            sc[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf), __builtin_bit_cast(bf16x8, qf[k]), sc[n], 0, 0, 0);
          }
        }
        // (keys are read two steps ahead of their products, 2048 tokens over 14000 942 -> 918 us; one step, left to itself, three as two)
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
        for (uint32_t k = 2; k < KS; ++k) {
          __builtin_amdgcn_sched_group_barrier(0x8, 2, 0);
          __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x8, 4, 0);
        __builtin_amdgcn_s_setprio(1);
        if (kv0 + kBlockKeys - 1u > pos_lo) {
          const int32_t seen = (int32_t)(pos - kv0 - 4u * half);
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[n][i] = 32 * n + 8 * (i >> 2) + (i & 3) > seen ? -INFINITY : sc[n][i];
        }
        float mx = -INFINITY;
#pragma unroll
        for (uint32_t i = 0; i < 16; ++i) mx = max3(mx, sc[0][i], sc[1][i]);
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
        mx = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
        // The reference m may stay behind the maximum by 2^8 (probabilities up to 256 lose nothing in bf16): with the exact one
        // every other block of 32 rows has a row whose maximum grows, and rescales all outputs.
        if (__any((mx - m) * scale2 > 8.f)) {
          const float mn = fmaxf(m, mx), f = __builtin_amdgcn_exp2f((m - mn) * scale2);
          lsum *= f;
          m = mn;
#pragma unroll
          for (uint32_t n = 0; n < NT; ++n) o[n] *= f;
        }
        const float ms = m * scale2;
        bf16x8 pf[4];
#pragma unroll
        for (uint32_t n = 0; n < 2; ++n)
#pragma unroll
          for (uint32_t i = 0; i < 16; ++i) {
            pf[2 * n + (i >> 3)][i & 7u] = (__bf16)__builtin_amdgcn_exp2f(fmaf(sc[n][i], scale2, -ms));
          }
        __builtin_amdgcn_s_setprio(2);
#pragma unroll
        for (uint32_t k = 0; k < 4; ++k)
#pragma unroll
          for (uint32_t n = 0; n < NT; ++n) {
            union { s16x4 h[2]; bf16x8 v; } vf;
#pragma unroll
            for (uint32_t x = 0; x < 2; ++x) {
              vf.h[x] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(uintptr_t)(vt + vat[n][x]) + 16u * k * ROWB / 8u);
            }
            o[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf.v, pf[k], o[n], 0, 0, 0);
          }
        __builtin_amdgcn_s_setprio(0);
        // The sum is of the rounded ones: the weights add up to one.  Behind the products, in the shadow of the last of them (in
        // front of them: 2048 tokens over 14000 992 us instead of 936).
        float part_sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (uint32_t i = 0; i < 8; i += 2)
#pragma unroll
          for (uint32_t k = 0; k < 4; ++k)
            part_sum[k] = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{pf[k][i], pf[k][i + 1]}, bf16x2{(__bf16)1.0f, (__bf16)1.0f}, part_sum[k], false);
        lsum += (part_sum[0] + part_sum[1]) + (part_sum[2] + part_sum[3]);
        if (__builtin_expect(poisoned, 0)) {
          for (uint32_t j = 0; j < kBlockKeys && kv0 + j <= pos_hi; ++j) {
            size_t at = 0;
            if (!cache_row(s, slot, kvh, kv0 + j, &at) || kv0 + j > pos) continue;
#pragma unroll
            for (uint32_t n = 0; n < NT; ++n)
#pragma unroll
              for (uint32_t i = 0; i < 16; ++i) {
                const uint32_t x = as_global(s.v)[at + 32u * n + 8u * (i >> 2) + 4u * half + (i & 3u)];
                if ((x & 0x7F80u) == 0x7F80u) o[n][i] += bf16_to_f32((uint16_t)x);
              }
          }
        }
      }
      drain_vmem();
      __syncthreads();
    }
    __builtin_amdgcn_s_setprio(3);
    // ---- the end: the row's sum of both halves; the output, or the unit's partial result
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(lsum), __float_as_uint(lsum), false, false);
    const float l = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
    if (r < rows) {
      if (nb <= per) {
        const float inv = 1.0f / l;
        uint16_t* to = a.out + (size_t)(begin + t) * a.out_stride + (size_t)head * D + 8u * half;
#pragma unroll
        for (uint32_t n = 0; n < NT; ++n)
#pragma unroll
          for (uint32_t i = 0; i < 16; i += 8) {   // a lane has 4 of 8 columns, the other half's lane the others: 8 of one lane, 8 of the other
            const auto x = __builtin_amdgcn_permlane32_swap(pack_bf16(o[n][i] * inv, o[n][i + 1] * inv), pack_bf16(o[n][i + 4] * inv, o[n][i + 5] * inv), false, false);
            const auto y = __builtin_amdgcn_permlane32_swap(pack_bf16(o[n][i + 2] * inv, o[n][i + 3] * inv), pack_bf16(o[n][i + 6] * inv, o[n][i + 7] * inv), false, false);
            *as_global((u32x4*)(to + 32u * n + 2u * i)) = u32x4{x[0], y[0], x[1], y[1]};
          }
      } else {
        const uint32_t held = min(rows, kTileRows), in_tile = r - tile * kTileRows;
        float* part = (float*)a.work + kAttendHeader + __builtin_amdgcn_readlane(d.part, seq) + (size_t)((tile * chunks + chunk) * s.n_kv + kvh) * held * (D + 2u);
        float* to = part + (size_t)in_tile * D + 4u * half;
#pragma unroll
        for (uint32_t n = 0; n < NT; ++n)
#pragma unroll
          for (uint32_t i = 0; i < 4; ++i) *as_global((f32x4*)(to + 32u * n + 8u * i)) = f32x4{o[n][4 * i], o[n][4 * i + 1], o[n][4 * i + 2], o[n][4 * i + 3]};
        if (half == 0) *as_global((f32x2*)(part + (size_t)held * D + 2u * in_tile)) = f32x2{m * scale2, l};
      }
    }
  }
}

// Joins the partial results of a row whose tile was cut into runs, in their order: W wavefronts per row and query head, every W-th
// run each.
template <int D, uint32_t W>
__global__ void __launch_bounds__(256) rows_attend_join_kernel(AttendArgs a, uint32_t lg) {
  __shared__ float parts[4][D];
  __shared__ float weight[4][kAttendMostChunks + 16u * W];
  const RowSeqs& s = a.s;
  const uint32_t lane = threadIdx.x & 63u, wave = uniform_u32(threadIdx.x >> 6);
  SeqLanes q = {0, 0, -1, 0};
  uint32_t seq_chunks = 0, blocks = 0, seq_part = 0;
  if (lane < kMaxRowSeqs) {
    const u32x4 x = as_global((const u32x4*)a.work)[2u * lane], y = as_global((const u32x4*)a.work)[2u * lane + 1u];
    q.begin = (int32_t)x[0]; q.end = (int32_t)x[1]; q.pos = (int32_t)x[2];
    seq_chunks = x[3]; blocks = y[0]; seq_part = y[1];
  }
  if (!__ballot(seq_chunks > 1u)) return;
  const uint32_t mine = W == 1 ? 0u : wave;   // first run
  for (uint64_t item = W == 1 ? blockIdx.x * 4u + wave : blockIdx.x; item < (uint64_t)s.n_rows * s.n_q; item += gridDim.x * (4u / W)) {
  const uint32_t row = (uint32_t)(item / s.n_q), head = (uint32_t)(item - (uint64_t)row * s.n_q);
  const uint32_t seq = seq_of_row(q, row);
  if (seq == 64u) continue;
  const uint32_t T = __builtin_amdgcn_readlane((uint32_t)(q.end - q.begin), seq), pos0 = __builtin_amdgcn_readlane(q.pos, seq);
  const uint32_t chunks = __builtin_amdgcn_readlane(seq_chunks, seq), per = __builtin_amdgcn_readlane(blocks, seq);
  if (chunks <= 1u) continue;
  const uint32_t r = ((row - __builtin_amdgcn_readlane(q.begin, seq)) << lg) + (head & ((1u << lg) - 1u)), tile = r / kTileRows;
  const uint32_t n = uniform_u32(quotient(tile_blocks(pos0, T, tile, lg) + per - 1u, per));
  if (n <= 1u) continue;
  const uint32_t held = min(T << lg, kTileRows), in_tile = r - tile * kTileRows;
  const size_t stride = (size_t)s.n_kv * held * (D + 2u);
  const float* part = (const float*)a.work + kAttendHeader + __builtin_amdgcn_readlane(seq_part, seq) +
                      (size_t)(tile * chunks * s.n_kv + (head >> lg)) * held * (D + 2u);
  // outputs of 16 runs in flight at once, the first with the maxima and sums, a lane a run (and the 64th, .. after it): their weights go by LDS
  const float* p = part + (size_t)in_tile * D + (D / 64) * lane;
  float M = -INFINITY, l = 0.f, o[D / 64] = {}, v[16][D / 64];
  f32x2 ml[kAttendMostChunks / 64];
  auto request = [&](uint32_t c) {
#pragma unroll
    for (uint32_t j = 0; j < 16; ++j)
#pragma unroll
      for (int e = 0; e < D / 64; ++e) v[j][e] = as_global(p)[min(mine + W * (c + j), n - 1u) * stride + e];
  };
#pragma unroll
  for (uint32_t i = 0; i < kAttendMostChunks / 64; ++i) {
    ml[i] = f32x2{-INFINITY, 0.f};
    if (64u * i + lane < n) ml[i] = *as_global((const f32x2*)(part + (64u * i + lane) * stride + (size_t)held * D + 2u * in_tile));
  }
  request(0);
#pragma unroll
  for (uint32_t i = 0; i < kAttendMostChunks / 64; ++i) M = fmaxf(M, ml[i].x);
  M = wave_max_dpp(M);
#pragma unroll
  for (uint32_t i = 0; i < kAttendMostChunks / 64; ++i) {
    const float f = __builtin_amdgcn_exp2f(ml[i].x - M);
    l = fmaf(ml[i].y, f, l);
    weight[wave][64u * i + lane] = f;
  }
  l = wave_sum_dpp(l);
  for (uint32_t c = 0;;) {
#pragma unroll
    for (uint32_t j = 0; j < 16; ++j)
#pragma unroll
      for (int e = 0; e < D / 64; ++e) o[e] = mine + W * (c + j) < n ? fmaf(v[j][e], weight[wave][mine + W * (c + j)], o[e]) : o[e];
    c += 16u;
    if (mine + W * c >= n) break;
    request(c);
  }
  if constexpr (W > 1) {
#pragma unroll
    for (int e = 0; e < D / 64; ++e) parts[wave][(D / 64) * lane + e] = o[e];
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int e = 0; e < D / 64; ++e) {
      const float* q = &parts[0][(D / 64) * lane + e];
      o[e] = (q[0] + q[D]) + (q[2 * D] + q[3 * D]);
    }
  }
  const float inv = 1.0f / l;
  uint16_t* to = a.out + (size_t)row * a.out_stride + (size_t)head * D + (D / 64) * lane;
  if constexpr (D == 128) *as_global((uint32_t*)to) = pack_bf16(o[0] * inv, o[1] * inv);
  else *as_global(to) = (uint16_t)pack_bf16(o[0] * inv, 0.f);
  }
}

constexpr uint32_t attend_lds(uint32_t D) { return 4u * kBlockKeys * D * 2u + 16u; }
hipError_t rows_prepare(int device) {
  static std::mutex mu;
  static std::vector<bool> done;
  std::lock_guard<std::mutex> lock(mu);
  if ((size_t)device < done.size() && done[device]) return hipSuccess;
  hipError_t e = hipSuccess;
  for (const void* fn : {(const void*)rows_attend_kernel<128, false, false>, (const void*)rows_attend_kernel<128, true, false>,
                         (const void*)rows_attend_kernel<128, false, true>, (const void*)rows_attend_kernel<128, true, true>})
    if (e == hipSuccess) e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, (int)attend_lds(128));
  if (e == hipSuccess) {
    done.resize(std::max(done.size(), (size_t)device + 1u));
    done[device] = true;
  }
  return e;
}

template <int D, bool PAGED>
static hipError_t launch_attend(const AttendArgs& a, uint32_t lg, hipStream_t stream) {
  // units: one per tile, and up to kAttendSlots more where tiles are cut (a workgroup without one has worked that out for nothing;
  // one takes several where there are more)
  const uint64_t tiles = (((uint64_t)a.s.n_rows << lg) / kTileRows + a.s.n_seqs) * a.s.n_kv;
  const uint32_t grid = (uint32_t)std::min<uint64_t>(tiles <= kAttendSlots / 2u ? kAttendSlots : tiles + (tiles <= 2u * kAttendSlots ? kAttendSlots : kAttendSlots / 4u), 1u << 20);
  // Rows of one tile at most: keys that are kept would only drive out others from the caches.  (Kept / not, 10 layers' caches in turn: 8 x 1
  // token over 512 to 4096 24.7 / 22.8 us, 16 x 1 over 4000 52.6 / 47.9; one call's cache, which stays in the last cache, 21.9 / 21.9.  Several
  // tiles a sequence, 16 ragged prompts: 147 / 159.)  By the rows of the call, for the host does not see the sequences': more rows than a tile
  // has, of sequences that have one tile each, go the other way, as do few rows in a call with many to spare (8 x 4 / 8 x 5 tokens over 4000,
  // 26.0 / 27.8 us; 16 x 2 / 16 x 3 over 2000, heads of 64, 15.3 / 19.0).
  if (a.s.n_rows << lg <= kTileRows) {
    const uint32_t runs = std::min(kAttendFewChunks, a.s.max_seq / (kAttendMinBlocks * kBlockKeys) + 1u);
    rows_attend_kernel<D, PAGED, true><<<dim3(std::min(attend_slots(D, true), a.s.n_seqs * a.s.n_kv * runs)), dim3(256), attend_lds(D), stream>>>(a, lg);
  }
  else rows_attend_kernel<D, PAGED, false><<<dim3(grid), dim3(256), attend_lds(D), stream>>>(a, lg);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.s.max_seq < (kAttendMinBlocks + kAttendJoinBlocks) * kBlockKeys) return e;   // (never cut)
  // On a longer cache the host cannot tell whether anything was cut, so a call that was not pays for the launch (64 tokens, max_seq 64 / 4096:
  // 7.5 / 10.1 us).
  const uint64_t items = (uint64_t)a.s.n_rows * a.s.n_q;
  if (items <= kJoinFewItems) rows_attend_join_kernel<D, 4><<<dim3((uint32_t)items), dim3(256), 0, stream>>>(a, lg);
  else rows_attend_join_kernel<D, 1><<<dim3((uint32_t)std::min<uint64_t>((items + 3u) / 4u, kJoinWorkgroups)), dim3(256), 0, stream>>>(a, lg);
  return hipGetLastError();
}
hipError_t launch_rows_attend(const AttendArgs& a, hipStream_t stream) {
  uint32_t lg = 0;
  while ((1u << lg) < a.s.n_q / a.s.n_kv) ++lg;
  if (a.s.head_dim == 128u) return a.s.table ? launch_attend<128, true>(a, lg, stream) : launch_attend<128, false>(a, lg, stream);
  return a.s.table ? launch_attend<64, true>(a, lg, stream) : launch_attend<64, false>(a, lg, stream);
}

// ------------------------------------------------------------------------------------ log probabilities
// One pass over a row.  A wavefront reads 16 logits a lane and step and keeps, against the largest m that it has seen,
//   s = sum e^(x - m) without one of the largest, t = sum e^(x - m) (x - m)
// (ln p = x - m - log1p(s): nothing is lost of a token that is all but certain; entropy = log1p(s) - t / (1 + s)), and its
// best logits, sorted, one a lane.  A step none of whose logits beats the last of these, most of them, is sums alone.
// With few rows a row is cut into runs of steps, one a workgroup, and the one that arrives last joins these.
// What bounds it: many rows, the vector operations (an unpack, a half of a maximum, a fused product, an exponential at a quarter of
// the rate, a floor, a fused product and a sum a logit, and what a load takes: 118 for the 16 logits of a lane's step.  Of the 5500 of a
// row of 32000 that is two thirds; the others are the steps, ten or so of 32 with 4 alternatives, that have one to offer or a new maximum.
// 4096 rows of 32000 bf16, 262 MB, 53 to 58 us with 4 alternatives, 50 with none); in fp32 memory (4096 rows with 5 83 us, 6.3 TB/s).
// One row of 151936 with 20, 11 us: what waits for what, a fifth of it each the first logits, the first step's alternatives, a run's
// join, its way to the others and the row's join.
constexpr uint32_t kLogprobChunks = 64;   // runs of a row at most: a lane each when they are joined
// Workgroups that a call is cut into where its rows are fewer.  512 / 1024 / 1536 with 20 alternatives: 32 rows of 151936 19.2 / 18.2 /
// 16.9 us, 64 23.2 / 23.7 / 23.2, 200 37.0 / 35.8 / 40.1; 200 of 32000 20.2 / 18.9 / 20.6, 512 23.7 / 25.8 / 32.0.
constexpr uint32_t kLogprobWorkgroups = 1024;
// A wavefront a row from here on.  Four / one, 32000 in bf16 with 4 alternatives: 1536 rows 32.5 / 35.1 us, 2048 38.4 / 36.0, 4096
// 68 / 56; with 20 43 / 52, 51 / 54, 88 / 76.
constexpr uint32_t kLogprobManyRows = 2048;
constexpr uint32_t kLogprobLane = 16;   // logits of a lane and step
static_assert(kLogprobWorkgroups == kRowsArrivals, "a counter for each row of a call that cuts its rows: there are fewer of them than this");
constexpr uint32_t kNotLast = 0xFFFFFFFFu;

// A logit and its token as one number: larger logits first, of equal ones the lower token.  0: none.
__device__ __forceinline__ uint64_t entry_of(float x, uint32_t token) {
  const uint32_t u = __float_as_uint(x + 0.0f);   // (-0 is 0)
  return ((uint64_t)(u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u)) << 32) | (0xFFFFFFFFu - token);
}
__device__ __forceinline__ float entry_logit(uint64_t e) {
  const uint32_t k = (uint32_t)(e >> 32);
  return __uint_as_float(k ^ ((k & 0x80000000u) ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ __forceinline__ uint64_t readlane64(uint64_t v, uint32_t lane) {
  return ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32) | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
}

struct RowSum {
  float m, s, t;
};
// The sums of the wavefront's first n lanes, as one (in every lane).
__device__ __forceinline__ RowSum join_sums(const RowSum& a, uint32_t n) {
  const uint32_t lane = threadIdx.x & 63u;
  const float mine = lane < n ? a.m : -INFINITY, m = wave_max_dpp(mine);
  const uint64_t holds = __ballot(lane < n && a.m == m);
  float s = 0.f, t = 0.f;
  if (holds && lane == (uint32_t)__builtin_ctzll(holds)) { s = a.s; t = a.t; }
  else if (lane < n) {
    if (a.m == -INFINITY) s = a.s;   // (nothing: 0, or NaN)
    else {
      const float d = fmaxf(a.m - m, -200.f), f = __expf(d);
      s = (a.s + 1.f) * f;
      t = (a.t + (a.s + 1.f) * d) * f;
    }
  }
  return RowSum{m, wave_sum_dpp(s), wave_sum_dpp(t)};
}

// The best k of n entries in LDS, in order, into best [k] (empty before).  Called by whole wavefronts, WAVES of them, this one the
// wave-th: an entry's place is the number of entries above it, eight lanes count an eighth of them each.
template <uint32_t WAVES>
__device__ __forceinline__ void rank_entries(uint32_t wave, const uint64_t* list, uint32_t n, uint32_t k, uint64_t* best) {
  for (uint32_t i0 = 0; i0 < n; i0 += 8u * WAVES) {
    const uint32_t i = i0 + 8u * wave + ((threadIdx.x & 63u) >> 3);
    const uint64_t mine = i < n ? list[i] : 0;
    uint32_t rank = 0;
#pragma unroll 4
    for (uint32_t j = threadIdx.x & 7u; j < n; j += 8u) rank += list[j] > mine;
    rank += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)rank, 0xB1, 0xF, 0xF, true);    // lane ^ 1
    rank += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)rank, 0x4E, 0xF, 0xF, true);    // lane ^ 2
    rank += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)rank, 0x141, 0xF, 0xF, true);   // mirror of 8
    if (mine && rank < k && (threadIdx.x & 7u) == 0) best[rank] = mine;
  }
}
// A lower bound, its upper 16 bits, of the n-th largest of the lanes' numbers (0 where fewer have any).
__device__ __forceinline__ uint32_t nth_largest(uint32_t key, uint32_t n) {
  uint32_t p = 0;
#pragma unroll 1
  for (uint32_t bit = 0x40000000u; bit > 0x8000u; bit >>= 2) {   // two bits a time: three counts that do not wait for each other
    const uint32_t a = (uint32_t)__popcll(__ballot(key >= (p | bit))), b = (uint32_t)__popcll(__ballot(key >= (p | 2u * bit))),
                   c = (uint32_t)__popcll(__ballot(key >= (p | 3u * bit)));
    p |= c >= n ? 3u * bit : b >= n ? 2u * bit : a >= n ? bit : 0u;
  }
  return p;
}

// ln(1 + s), s >= 0, in a few operations: 2 artanh(s / (2 + s)) as a series below one (the rest of it is under 2e-8 of the
// value), the logarithm above.
__device__ __forceinline__ float log1p_fast(float s) {
  const float z = s / (2.f + s), y = z * z;
  const float p = fmaf(fmaf(fmaf(fmaf(fmaf(fmaf(fmaf(y, 1.f / 15, 1.f / 13), y, 1.f / 11), y, 1.f / 9), y, 1.f / 7), y, 1.f / 5), y, 1.f / 3), y, 1.f);
  return s < 1.f ? 2.f * z * p : __logf(1.f + s);
}

// What is written for a row, by one wavefront: `mine` is lane j's j-th best entry, empty ones last.
__device__ __forceinline__ void write_row(const LogprobArgs& a, uint32_t row, const RowSum& r, float asked, uint64_t mine) {
  const uint32_t lane = threadIdx.x & 63u;
  const bool none = !(r.m > -INFINITY) || r.m == INFINITY || r.s != r.s;
  const float norm = log1p_fast(r.s), nan = __uint_as_float(0x7FC00000u);
  if (lane == 0) {
    if (a.entropy) as_global(a.entropy)[row] = none ? nan : norm - r.t / (1.f + r.s);
    if (a.tokens) {
      const int32_t t = as_global(a.tokens)[row];
      float lp = nan;
      if (t == -1) lp = 0.f;
      else if (t < 0 || (uint32_t)t >= a.vocab) report_rows(a.err, DE_BAD_ROW_TOKEN, row, (uint32_t)t);
      else if (!none) lp = asked - r.m - norm;
      as_global(a.logprobs)[row] = lp;
    }
  }
  if (!a.n_top) return;
  mine = lane < a.n_top ? mine : 0;
  const uint32_t real = (uint32_t)__popcll(__ballot(mine != 0));
  uint32_t id = 0xFFFFFFFFu - (uint32_t)mine;
  if (real < a.n_top) {   // fewer tokens above -inf than asked for: the lowest of the others
    bool listed = false;
    for (uint32_t j = 0; j < real; ++j) listed |= (uint32_t)__builtin_amdgcn_readlane((int)id, j) == lane;
    uint32_t at = real;
    for (uint64_t b = __ballot(!listed); b && at < a.n_top; b &= b - 1, ++at)
      if (lane == at) id = (uint32_t)__builtin_ctzll(b);
  }
  if (lane < a.n_top) {
    as_global(a.top_tokens)[(size_t)row * a.n_top + lane] = none ? -1 : (int32_t)id;
    as_global(a.top_logprobs)[(size_t)row * a.n_top + lane] = none ? nan : (mine ? entry_logit(mine) : -INFINITY) - r.m - norm;
  }
}

template <typename T>
__device__ __forceinline__ float logit_at(const T* p, size_t i) {
  if constexpr (sizeof(T) == 4) return as_global(p)[i];
  else return bf16_to_f32(as_global(p)[i]);
}
// The logit asked about, 0 for no token or a wrong one.
template <typename T>
__device__ __forceinline__ float asked_logit(const LogprobArgs& a, uint32_t row) {
  if (!a.tokens) return 0.f;
  const int32_t t = as_global(a.tokens)[row];
  return t >= 0 && (uint32_t)t < a.vocab ? logit_at((const T*)a.logits + (size_t)row * a.stride, (size_t)t) : 0.f;
}

// A wavefront's best entries so far: lane j holds the j-th.  A few that a step has to offer are put in place one by one, the
// lanes behind shifted.  More are gathered in LDS (fresh [128]) and joined with them 64 at a time: an entry's place is the
// number of entries above it.  (All joined / up to kLogprobFew put in place, 4096 rows of 32000: 4 alternatives 63.7 / 59.5 us, 20
// 89 / 75; 2048 rows of 151936 with 20 180 / 150.  With up to 1, 4, 16 or 64: 84, 77, 76, 75 and 159, 149, 150, 150.)
constexpr uint32_t kLogprobFew = 8;
struct Best {
  uint64_t mine = 0, last = 0;   // last: the n_top-th, 0 while there are fewer
  uint32_t count = 0, waiting = 0;
  __device__ __forceinline__ void insert(uint64_t e, uint32_t n_top) {
    const uint32_t lane = threadIdx.x & 63u, place = (uint32_t)__popcll(__ballot(mine > e));
    auto lane_before = [](uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x138, 0xF, 0xF, true); };   // wave_shr 1
    const uint64_t before = (uint64_t)lane_before((uint32_t)(mine >> 32)) << 32 | lane_before((uint32_t)mine);
    count = min(n_top, count + 1u);
    mine = lane >= count ? 0 : lane == place ? e : lane > place ? before : mine;
  }
  __device__ __forceinline__ void join(uint64_t* fresh, uint64_t* sorted, uint32_t n_top) {
    const uint32_t lane = threadIdx.x & 63u;
    for (uint32_t at = 0; at < waiting; at += 64u) {
      const uint32_t n = min(64u, waiting - at);
      const uint64_t now = lane < n ? fresh[at + lane] : 0;
      uint32_t place_now = 0, place_old = lane;
#pragma unroll 4
      for (uint32_t i = 0; i < n; ++i) {
        const uint64_t e = fresh[at + i];
        place_now += e > now;
        place_old += e > mine;
      }
#pragma unroll 2
      for (uint32_t i = 0; i < count; ++i) place_now += sorted[i] > now;
      if (lane < n && place_now < n_top) sorted[place_now] = now;
      if (lane < count && place_old < n_top) sorted[place_old] = mine;
      count = min(n_top, count + n);
      mine = lane < count ? sorted[lane] : 0;
    }
    waiting = 0;
    last = count == n_top ? readlane64(mine, n_top - 1u) : 0;
  }
};

// The workgroup's run of a row (sums r and the lanes' best entries, in wavefront 0) to the device's coherence point; the
// workgroup that arrives last at the row's counter, and it alone, goes on with all of them: true, r and `mine` the row's.
__device__ __forceinline__ bool join_runs(const LogprobArgs& a, uint32_t row, uint32_t chunk, uint32_t chunks, RowSum& r, uint64_t& mine, uint64_t* lds) {
  uint64_t *best = lds, &least = lds[MPK_ROWS_MAX_TOP], *list = lds + MPK_ROWS_MAX_TOP + 2;   // list: [chunks * k]
  uint32_t& n = (uint32_t&)lds[MPK_ROWS_MAX_TOP + 1];
  const uint32_t lane = threadIdx.x & 63u, k = a.n_top;
  uint64_t *sums = (uint64_t*)a.work + (size_t)row * chunks * (2u + k), *entries = sums + 2u * chunks;   // [chunks][2], [chunks][k]
  if (threadIdx.x < 64u) {
    if (lane == 0) { st_act2((float*)(sums + 2u * chunk), r.m, r.s); st_act((float*)(sums + 2u * chunk + 1u), r.t); }
    if (lane < k) __hip_atomic_store(as_global(entries + chunk * k + lane), mine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    drain_vmem();
    if (lane == 0) {
      uint32_t* arrived = a.arrivals + (size_t)row * kArrivalStride;
      const bool last = __hip_atomic_fetch_add(as_global(arrived), 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1u == chunks;
      if (last) st_act_u32(arrived, 0u);   // as the next call finds it
      n = last ? 0u : kNotLast;
    }
  }
  __syncthreads();
  if (n == kNotLast) return false;
  // everything that the runs left, in one round of loads
  constexpr uint32_t kPer = kLogprobChunks * MPK_ROWS_MAX_TOP / 256u;
  uint64_t e[kPer];
  const uint32_t nth = min(k, (2u * k + chunks - 1u) / chunks);
#pragma unroll
  for (uint32_t j = 0; j < kPer; ++j) e[j] = threadIdx.x + 256u * j < chunks * k ? ld_relaxed64(entries + threadIdx.x + 256u * j) : 0;
  if (threadIdx.x < 64u) {   // (the sums: the first wavefront writes them)
    r = RowSum{-INFINITY, 0.f, 0.f};
    if (lane < chunks) {
      const float2 ms = ld_act2((const float*)(sums + 2u * lane));
      r.m = ms.x; r.s = ms.y; r.t = ld_act((const float*)(sums + 2u * lane + 1u));
    }
    r = join_sums(r, chunks);
  } else if (k && threadIdx.x < 128u) {   // (beside it)
    // ceil(k / nth) runs have nth entries at or above the one that this many runs' nth entries are not below: k of the row are,
    // and few others where about half of the runs have one
    const uint64_t nth_best = lane < chunks ? ld_relaxed64(entries + lane * k + nth - 1u) : 0;
    const uint32_t p = nth_largest((uint32_t)(nth_best >> 32), (k + nth - 1u) / nth);
    if (lane == 0) least = (uint64_t)p << 32;
    if (lane < k) best[lane] = 0;
  }
  __syncthreads();
#pragma unroll
  for (uint32_t j = 0; j < kPer; ++j)
    if (256u * j < chunks * k && e[j] && e[j] >= least) list[atomicAdd(&n, 1u)] = e[j];   // (in any order: an entry's rank goes by all of them)
  __syncthreads();
  rank_entries<4>(threadIdx.x >> 6, list, n, k, best);
  __syncthreads();
  mine = lane < k ? best[lane] : 0;
  return true;
}

// W wavefronts of a workgroup share a run: 4, or 1 and the run is a row.
template <typename T, uint32_t W>
__global__ void __launch_bounds__(256) rows_logprobs_kernel(LogprobArgs a, uint32_t chunks, uint32_t share) {
  constexpr uint32_t N = kLogprobLane, E = 16 / sizeof(T), V = N / E, kStep = 64 * N;   // logits of 16 bytes, such loads of a step, logits of a step
  __shared__ uint64_t fresh[4][128], sorted[4][MPK_ROWS_MAX_TOP], list[4 * MPK_ROWS_MAX_TOP], first_best[MPK_ROWS_MAX_TOP];
  // what hot steps pass from lane to lane (4 more: reads of the logits of several lanes spread over the banks), then the entries of the join
  __shared__ __align__(16) uint64_t lists[4 * 64 * (N + 4) / 2];
  float(*offered)[64][N + 4] = (float(*)[64][N + 4])lists;
  static_assert(W == 1 || sizeof(lists) >= (kLogprobChunks * MPK_ROWS_MAX_TOP + MPK_ROWS_MAX_TOP + 2) * 8, "entries of all runs");
  __shared__ RowSum sums[4];
  __shared__ __align__(16) uint32_t bounds[4];   // of each wavefront: no larger than its (k / W)-th largest logit, as entries count them
  const uint32_t lane = threadIdx.x & 63u, wave = uniform_u32(threadIdx.x >> 6), part_of = W == 1 ? 0u : wave;
  const uint32_t unit = W == 1 ? blockIdx.x * 4u + wave : blockIdx.x, row = unit / chunks, chunk = unit - row * chunks, k = a.n_top;
  if (W == 1 && row >= a.n_rows) return;
  const T* x = (const T*)a.logits + (size_t)row * a.stride;
  const uint32_t head = min(a.vocab, (uint32_t)((16u - ((uintptr_t)x & 15u)) & 15u) / (uint32_t)sizeof(T));   // logits in front of a 16-byte boundary
  const uint32_t nvec = (a.vocab - head) / E, tail = a.vocab - head - nvec * E;
  const MPK_GLOBAL u32x4* xv = (const MPK_GLOBAL u32x4*)(x + head);
  const uint32_t v0 = chunk * share, v1 = min(nvec, v0 + share);
  float asked = 0.f;

  // The sums count in powers of two from c = log2(e) (m - shift) as rounded, so that an exponent is one fused operation; shift is 0
  // but for logits so large that the rounding of c would show, which are then taken less it.
  const float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
  float c = 0.f, shift = 0.f;
  RowSum r = {-INFINITY, 0.f, 0.f};
  Best best;
  // What lies at or below `bound` is no alternative of the row; `limit` is that, or the last of the best.  Without alternatives there
  // is the largest to beat alone.
  float bound = -INFINITY, limit = -INFINITY;
  // Read once, so not to be kept (kept / not: 1024 rows of 151936 108 / 97 us, 4096 of 32000 91 / 83, in bf16 58.4 / 58.0; few rows alike).
  u32x4 next[V];
  auto request = [&](uint32_t first) {
#pragma unroll
    for (uint32_t j = 0; j < V; ++j) next[j] = __builtin_nontemporal_load(xv + min(first + j * 64u + lane, v1 - 1u));
  };
  uint32_t at = v0 + part_of * (kStep / E);
  if (at < v1) request(at);
  if (part_of == 0) asked = asked_logit<T>(a, row);
  // The row's edges, what lies in front of the first and behind the last load of 16 bytes, come last, as one step.
  bool edges = false, start = W > 1;
  for (;;) {
    float y[N];
    const uint32_t first = at;
    if (at < v1) {
      u32x4 now[V];
#pragma unroll
      for (uint32_t j = 0; j < V; ++j) now[j] = next[j];
      at += W * (kStep / E);
      if (at < v1) request(at);
#pragma unroll
      for (uint32_t j = 0; j < V; ++j)
#pragma unroll
        for (uint32_t e = 0; e < 4; ++e) {
          if constexpr (E == 4) y[4 * j + e] = __uint_as_float(now[j][e]);
          else { y[8 * j + 2 * e] = bf16_lo(now[j][e]); y[8 * j + 2 * e + 1] = bf16_hi(now[j][e]); }
        }
      if (first + kStep / E > v1) {
#pragma unroll
        for (uint32_t j = 0; j < N; ++j)
          if (first + (j / E) * 64u + lane >= v1) y[j] = -INFINITY;
      }
    } else {
#pragma unroll
      for (uint32_t j = 0; j < N; ++j) y[j] = -INFINITY;
      if (!start) {
        if (edges || chunk || part_of || !(head + tail)) break;
        edges = true;
      }
      if (edges && lane < head + tail) y[0] = logit_at(x, lane < head ? lane : a.vocab - tail + (lane - head));
    }
    float mx = -INFINITY;
#pragma unroll
    for (uint32_t j = 0; j < N; j += 2) mx = max3(mx, y[j], y[j + 1]);
    if (W > 1 && k) {
      // No less than k logits of the row are at or above the least of the wavefronts' bounds, so what lies below is no answer (an
      // equal logit may be, hence the number below).  It is never above this wavefront's own largest.  The first step's bounds
      // together: a quarter of the alternatives each; later ones as they are by now, whatever the others have got to.  (The first
      // ones alone / all: 200 rows of 151936 with 20 alternatives 43 / 35 us, 1024 115 / 111, in bf16 84 / 76.)
      if (start) {
        const uint32_t p = nth_largest(mx == mx ? (uint32_t)(entry_of(mx, 0) >> 32) : 0u, (k + W - 1u) / W);
        if (lane == 0) bounds[wave] = p;
        __syncthreads();
      }
      const u32x4 b = *(volatile __attribute__((address_space(3))) u32x4*)(__attribute__((address_space(3))) uint32_t*)bounds;
      const uint32_t all = uniform_u32(min(min(b[0], b[1]), min(b[2], b[3])));
      if (all > 0x007FFFFFu) {
        bound = fmaxf(bound, entry_logit((uint64_t)(all - (all == 0x80000000u ? 2u : 1u)) << 32));   // (below 0 lies -0, which is not less)
        limit = fmaxf(limit, bound);
      }
    }
    start = false;
    float least = fmaxf(bound, -3.402823466e38f);
    uint64_t hot = __ballot(mx > limit || (edges && mx == limit));   // (tokens ascend, so an equal logit does not beat the last; the edges come out of order)
    if (hot) {
      const float m = wave_max_dpp(mx);
      const bool more = m > r.m;
      if (more) {
        const float sn = fabsf(m) < 1048576.f ? 0.f : m, cn = (m - sn) * kLog2e;
        if (r.m != -INFINITY) {
          const float d = fmaxf(fmaf(shift - sn, kLog2e, c - cn), -300.f), f = __builtin_amdgcn_exp2f(d);
          if (lane == 0) {   // the largest until now is one of many
            const float e = fmaf(r.m - shift, kLog2e, -c), p = __builtin_amdgcn_exp2f(e);
            r.s += p;
            r.t = fmaf(p, e, r.t);
          }
          r.t = fmaf(r.s, d, r.t) * f;
          r.s *= f;
        }
        r.m = m; c = cn; shift = sn;
      }
      if (k) {
        if ((uint32_t)__popcll(hot) > k) {
          // more lanes than places: k logits are at or above the k-th largest of the lanes' largest (its upper 16 bits)
          const uint32_t p = nth_largest(mx == mx ? (uint32_t)(entry_of(mx, 0) >> 32) : 0u, k);
          if (p > 0x007FFFFFu) least = fmaxf(least, entry_logit((uint64_t)p << 32));
          hot = __ballot(mx >= least);
        }
        if (hot >> lane & 1u) {
#pragma unroll
          for (uint32_t j = 0; j < N; j += 4) *(float4*)&offered[wave][lane][j] = make_float4(y[j], y[j + 1], y[j + 2], y[j + 3]);
        }
        while (hot) {   // four such lanes at a time, or two
          uint32_t from = 64u;
#pragma unroll
          for (uint32_t g = 0; g < 64u / N; ++g) {
            if (hot && lane / N == g) from = (uint32_t)__builtin_ctzll(hot);
            hot &= hot - 1ull;
          }
          const uint32_t j = lane % N;
          const float v = offered[wave][from & 63u][j];
          const uint32_t token = edges ? (from < head ? from : a.vocab - tail + (from - head)) : head + (first + (j / E) * 64u + from) * E + j % E;
          const uint64_t e = entry_of(v, token);
          uint64_t b = __ballot(from < 64u && v >= least && e > best.last);
          if (!best.waiting && !hot && (uint32_t)__popcll(b) <= kLogprobFew) {
            for (; b; b &= b - 1ull) best.insert(readlane64(e, (uint32_t)__builtin_ctzll(b)), k);
            if (lane < best.count) sorted[wave][lane] = best.mine;
            best.last = best.count == k ? readlane64(best.mine, k - 1u) : 0;
            break;
          }
          if (b >> lane & 1u) fresh[wave][best.waiting + (uint32_t)__popcll(b & ((1ull << lane) - 1u))] = e;
          best.waiting += (uint32_t)__popcll(b);
          if (best.waiting >= 64u || !hot) best.join(fresh[wave], sorted[wave], k);
        }
        limit = fmaxf(bound, best.last ? entry_logit(best.last) : -INFINITY);
        if (W > 1 && best.count >= (k + W - 1u) / W) {
          const uint32_t own = (uint32_t)(readlane64(best.mine, (k + W - 1u) / W - 1u) >> 32);
          if (lane == 0) *(volatile uint32_t*)&bounds[wave] = own;
        }
      } else limit = r.m;
      if (more) {   // one of the largest stays out of the sum
        bool out = lane == (uint32_t)__builtin_ctzll(__ballot(mx == m));
#pragma unroll
        for (uint32_t j = 0; j < N; ++j) {
          const bool it = out && y[j] == m;
          y[j] = it ? -INFINITY : y[j];
          out = out && !it;
        }
      }
    }
    if (__builtin_expect(shift != 0.f, 0)) {
#pragma unroll
      for (uint32_t j = 0; j < N; ++j) y[j] -= shift;
    }
    float s = 0.f, t = 0.f;
#pragma unroll
    for (uint32_t j = 0; j < N; ++j) {
      const float d = fmaf(y[j], kLog2e, -c), e = __builtin_amdgcn_exp2f(d);
      s += e;
      t = fmaf(e, fmaxf(d, -300.f), t);
    }
    r.s += s;
    r.t += t;
  }
  // ---- the lanes' and the wavefronts' results together
  r.s = wave_sum_dpp(r.s);
  r.t = wave_sum_dpp(r.t);
  if (r.m != -INFINITY) {   // from powers of two and c to those of e and m
    const float e = fmaf(r.m - shift, kLog2e, -c), f = __builtin_amdgcn_exp2f(-e);
    r.t = fmaf(-e, r.s, r.t) * f * kLn2;
    r.s *= f;
  }
  uint64_t mine = best.mine;
  if constexpr (W > 1) {
    if (lane == 0) sums[wave] = r;
    if (lane < k) list[wave * k + lane] = mine;
    if (wave == 1 && lane < k) first_best[lane] = 0;
    __syncthreads();
    if (wave == 0) r = join_sums(sums[lane & 3u], 4);   // (who writes them; the others meanwhile)
    if (k) {
      if (wave) rank_entries<3>(wave - 1u, list, 4u * k, k, first_best);
      __syncthreads();
    }
    if (lane < k) mine = first_best[lane];
    if (chunks > 1u && !join_runs(a, row, chunk, chunks, r, mine, lists)) return;
    if (wave) return;
  }
  write_row(a, row, r, asked, mine);
}

template <typename T>
static hipError_t launch_logprobs(const LogprobArgs& a, hipStream_t stream) {
  constexpr uint32_t E = 16 / sizeof(T);
  // a workgroup's share, in loads of 16 bytes: a whole row where there are rows enough for all compute units, else 4096 logits or
  // more, alike for all (filled one after the other, the last one's wavefronts without logits have no bound on the alternatives:
  // one row of 151936 with 20 12.1 us instead of 11.8)
  if (a.n_rows >= kLogprobManyRows) {
    rows_logprobs_kernel<T, 1><<<dim3((a.n_rows + 3u) / 4u), dim3(256), 0, stream>>>(a, 1u, a.vocab / E);
    return hipGetLastError();
  }
  constexpr uint32_t kRound = 4u * 64u * kLogprobLane;   // logits that a workgroup takes at once
  const uint32_t all = (a.vocab + kRound - 1u) / kRound, want = (kLogprobWorkgroups + a.n_rows - 1u) / a.n_rows;
  const uint32_t n = std::min(std::min(want, all), kLogprobChunks), rounds = (all + n - 1u) / n, chunks = (all + rounds - 1u) / rounds;
  rows_logprobs_kernel<T, 4><<<dim3(a.n_rows * chunks), dim3(256), 0, stream>>>(a, chunks, (a.vocab / E + chunks - 1u) / chunks);
  return hipGetLastError();
}
hipError_t launch_rows_logprobs(const LogprobArgs& a, bool f32, hipStream_t stream) {
  return f32 ? launch_logprobs<float>(a, stream) : launch_logprobs<uint16_t>(a, stream);
}

}  // namespace mpk
