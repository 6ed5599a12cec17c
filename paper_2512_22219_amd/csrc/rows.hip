// Rows beside the decode step (mpk_rows_append, mpk_rows_attend, mpk_rows_logprobs): kernels and launches.
#include "rows.h"

#include <algorithm>

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
  for (uint32_t i = 0; i + 1 < s.n_seqs; ++i) {   // (a slot that an earlier sequence with rows has)
    const int32_t other = __builtin_amdgcn_readlane(q.slot, i), rows = __builtin_amdgcn_readlane(n, i);
    if (rows > 0 && n > 0 && (uint32_t)lane > i && q.slot == other && !wrong) { wrong = DE_BAD_SLOT; what = (uint32_t)q.slot; }
  }
  if (wrong) {
    if (tell) report_rows(s.err, wrong, (uint32_t)lane, what);
    q.end = q.begin;
  }
  return q;
}

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
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) { return (uint32_t)f32_to_bf16(a) | ((uint32_t)f32_to_bf16(b) << 16); }

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

// A wavefront takes one row and a run of `per_wave` groups of its heads; a group is 64 / LPH heads, a head LPH lanes, a lane 8
// elements of the head's lower half and the 8 they are rotated with.
template <typename T, int D>
__global__ void __launch_bounds__(256) rows_append_kernel(AppendArgs a, uint32_t per_wave, uint32_t waves_per_row) {
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
  if (lane < HALF) {
    const double two_pi = 6.283185307179586476925286766559;
    double ang = (double)(int32_t)pos * as_global(a.inv_freq)[lane];
    ang -= two_pi * rint(ang / two_pi);
    double sn, cs;
    sincos(ang, &sn, &cs);
    angles[wave][lane] = make_float2((float)cs, (float)sn);
  }
  const uint32_t sub = lane & (LPH - 1u), heads = s.n_q + 2u * s.n_kv, e = 8u * sub;
  float2 cs[8];
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int i = 0; i < 8; ++i) cs[i] = angles[wave][e + i];
  const T* x = (const T*)a.qkv + (size_t)row * a.qkv_stride;
  size_t at = 0;
  const bool cached = cache_row(s, slot, 0, pos, &at);
  if (!cached && lane == 0 && part == 0) report_rows(s.err, DE_BAD_PAGE, seq, pos);
  const size_t kv_head = s.table ? (size_t)D << s.page_shift : (size_t)D * s.max_seq;
  for (uint32_t g = 0; g < per_wave; ++g) {
    const uint32_t h = (part * per_wave + g) * HPG + lane / LPH;
    if (h >= heads) continue;
    float lo[8], hi[8];
    load8(x + (size_t)h * D + e, lo);
    load8(x + (size_t)h * D + HALF + e, hi);
    const bool is_v = h >= s.n_q + s.n_kv, is_q = h < s.n_q;
    if (!is_v) {
      const uint16_t* gain = is_q ? a.q_norm : a.k_norm;
      if (gain) {
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = fmaf(hi[i], hi[i], fmaf(lo[i], lo[i], ss));
#pragma unroll
        for (uint32_t o = 1; o < LPH; o *= 2) ss += __shfl_xor(ss, o, 64);
        const float inv = 1.0f / sqrtf(ss * (1.0f / (float)D) + a.eps);
        float gl[8], gh[8];
        load8(gain + e, gl);
        load8(gain + HALF + e, gh);
#pragma unroll
        for (int i = 0; i < 8; ++i) { lo[i] = lo[i] * inv * gl[i]; hi[i] = hi[i] * inv * gh[i]; }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float l = lo[i], u = hi[i];
        lo[i] = fmaf(l, cs[i].x, -(u * cs[i].y));
        hi[i] = fmaf(u, cs[i].x, l * cs[i].y);
      }
    }
    uint16_t* to = nullptr;
    if (is_q) to = a.q_out + (size_t)row * a.q_stride + (size_t)h * D;
    else if (cached) to = (is_v ? s.v + at + (size_t)(h - s.n_q - s.n_kv) * kv_head : s.k + at + (size_t)(h - s.n_q) * kv_head);
    if (to) {
      store8(to + e, lo);
      store8(to + HALF + e, hi);
    }
  }
}

template <typename T, int D>
static hipError_t launch_append(const AppendArgs& a, hipStream_t stream) {
  const uint32_t groups = (a.s.n_q + 2u * a.s.n_kv + 1024u / D - 1u) / (1024u / D);
  const uint32_t per_wave = a.s.n_rows <= 256u ? 1u : groups, waves_per_row = (groups + per_wave - 1u) / per_wave;
  const uint64_t blocks = ((uint64_t)a.s.n_rows * waves_per_row + 3u) / 4u;
  rows_append_kernel<T, D><<<dim3((uint32_t)blocks), dim3(256), 0, stream>>>(a, per_wave, waves_per_row);
  return hipGetLastError();
}
hipError_t launch_rows_append(const AppendArgs& a, bool f32, hipStream_t stream) {
  if (a.s.head_dim == 128u) return f32 ? launch_append<float, 128>(a, stream) : launch_append<uint16_t, 128>(a, stream);
  return f32 ? launch_append<float, 64>(a, stream) : launch_append<uint16_t, 64>(a, stream);
}

// ------------------------------------------------------------------------------------ attend
// One wavefront per row and query head: 64 keys at a time, a lane a key for the scores, a lane D / 64 columns for the product.
template <int D>
__global__ void __launch_bounds__(64) rows_attend_kernel(AttendArgs a) {
  __shared__ float qs[D], ps[64];
  __shared__ uint64_t vat[64];
  const RowSeqs& s = a.s;
  const uint32_t lane = threadIdx.x, row = blockIdx.x / s.n_q, h = blockIdx.x - row * s.n_q;
  const SeqLanes q = load_seqs(s, blockIdx.x == 0);
  const uint32_t seq = seq_of_row(q, row);
  if (seq == 64u) return;
  const uint32_t pos = (uint32_t)__builtin_amdgcn_readlane(q.pos, seq) + row - (uint32_t)__builtin_amdgcn_readlane(q.begin, seq);
  const uint32_t slot = (uint32_t)__builtin_amdgcn_readlane(q.slot, seq), kvh = h / (s.n_q / s.n_kv);
  for (uint32_t i = lane; i < D; i += 64) qs[i] = bf16_to_f32(as_global(a.q)[(size_t)row * a.q_stride + (size_t)h * D + i]);
  __syncthreads();
  float m = -INFINITY, l = 0.f, o[D / 64] = {};
  for (uint32_t j0 = 0; j0 <= pos; j0 += 64) {
    const uint32_t j = j0 + lane;
    float sc = -INFINITY;
    size_t at = 0;
    bool there = false;
    if (j <= pos) {
      there = cache_row(s, slot, kvh, j, &at);
      if (!there) report_rows(s.err, DE_BAD_PAGE, seq, j);
      if (there) {
        sc = 0.f;
        for (int e = 0; e < D; e += 8) {
          float kk[8];
          load8(s.k + at + e, kk);
#pragma unroll
          for (int i = 0; i < 8; ++i) sc = fmaf(qs[e + i], kk[i], sc);
        }
        sc *= 1.0f / sqrtf((float)D);
      }
    }
    const float mn = fmaxf(m, wave_max(sc)), scale = m == mn ? 1.f : expf(m - mn);
    const float p = sc == -INFINITY ? 0.f : expf(sc - mn);
    l = l * scale + wave_sum(p);
    m = mn;
    ps[lane] = p;
    vat[lane] = there ? at : ~0ull;
    __syncthreads();
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
      o[c] *= scale;
      for (int i = 0; i < 64; ++i)
        if (vat[i] != ~0ull) o[c] = fmaf(ps[i], bf16_to_f32(as_global(s.v)[vat[i] + c * 64 + lane]), o[c]);
    }
    __syncthreads();
  }
#pragma unroll
  for (int c = 0; c < D / 64; ++c) as_global(a.out)[(size_t)row * a.out_stride + (size_t)h * D + c * 64 + lane] = f32_to_bf16(o[c] / l);
}
hipError_t launch_rows_attend(const AttendArgs& a, hipStream_t stream) {
  const dim3 grid(a.s.n_rows * a.s.n_q);
  if (a.s.head_dim == 128u) rows_attend_kernel<128><<<grid, dim3(64), 0, stream>>>(a);
  else rows_attend_kernel<64><<<grid, dim3(64), 0, stream>>>(a);
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------ log probabilities
template <typename T>
__device__ __forceinline__ float logit_at(const T* p, size_t i) {
  if constexpr (sizeof(T) == 4) return as_global(p)[i];
  else return bf16_to_f32(as_global(p)[i]);
}
// One workgroup per row, a pass for the largest, one for the sums, one for each alternative.
template <typename T>
__global__ void __launch_bounds__(512) rows_logprobs_kernel(LogprobArgs a) {
  __shared__ float red[16];
  __shared__ uint64_t best[8];
  const uint32_t row = blockIdx.x, tid = threadIdx.x;
  const T* x = (const T*)a.logits + (size_t)row * a.stride;
  float m = -INFINITY, bad = 0.f;
  for (uint32_t i = tid; i < a.vocab; i += 512) {
    const float v = logit_at(x, i);
    if (!(v < INFINITY)) bad = 1.f;
    m = fmaxf(m, v);
  }
  bad = block_sum(bad, red);
  m = wave_max(m);
  __syncthreads();
  if ((tid & 63) == 0) red[tid >> 6] = m;
  __syncthreads();
  for (int i = 0; i < 8; ++i) m = fmaxf(m, red[i]);
  float sum = 0.f, dot = 0.f;
  for (uint32_t i = tid; i < a.vocab; i += 512) {
    const float d = fmaxf(logit_at(x, i) - m, -200.f), e = expf(d);
    sum += e;
    dot = fmaf(e, d, dot);
  }
  sum = block_sum(sum, red);
  dot = block_sum(dot, red);
  const bool none = bad != 0.f || m == -INFINITY;
  const float norm = logf(sum), nan = __uint_as_float(0x7FC00000u);
  if (tid == 0) {
    if (a.entropy) a.entropy[row] = none ? nan : norm - dot / sum;
    if (a.tokens) {
      const int32_t t = a.tokens[row];
      float lp = nan;
      if (t == -1) lp = 0.f;
      else if (t < 0 || (uint32_t)t >= a.vocab) report_rows(a.err, DE_BAD_TOKEN, row, (uint32_t)t);
      else if (!none) lp = logit_at(x, (uint32_t)t) - m - norm;
      a.logprobs[row] = lp;
    }
  }
  uint64_t last = ~0ull;
  for (uint32_t k = 0; k < a.n_top; ++k) {
    uint64_t b = 0;
    for (uint32_t i = tid; i < a.vocab; i += 512) {
      const uint32_t u = __float_as_uint(logit_at(x, i) + 0.0f);
      const uint64_t key = ((uint64_t)(u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u)) << 32) | (0xFFFFFFFFu - i);
      if (key < last && key > b) b = key;
    }
    for (int o = 32; o > 0; o >>= 1) {
      const uint64_t other = __shfl_xor((unsigned long long)b, o, 64);
      b = other > b ? other : b;
    }
    __syncthreads();
    if ((tid & 63) == 0) best[tid >> 6] = b;
    __syncthreads();
    for (int i = 0; i < 8; ++i) b = best[i] > b ? best[i] : b;
    last = b;
    if (tid == 0) {
      const uint32_t i = 0xFFFFFFFFu - (uint32_t)b;
      a.top_tokens[(size_t)row * a.n_top + k] = none ? -1 : (int32_t)i;
      a.top_logprobs[(size_t)row * a.n_top + k] = none ? nan : logit_at(x, i) - m - norm;
    }
  }
}
hipError_t launch_rows_logprobs(const LogprobArgs& a, bool f32, hipStream_t stream) {
  if (f32) rows_logprobs_kernel<float><<<dim3(a.n_rows), dim3(512), 0, stream>>>(a);
  else rows_logprobs_kernel<uint16_t><<<dim3(a.n_rows), dim3(512), 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace mpk
