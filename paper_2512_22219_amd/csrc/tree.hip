// Trees of drafted tokens: which of them stay (mpk_tree_verify), and their rows in the cache closed up (mpk_tree_keep).
#include <algorithm>

#include "rows_device.h"

namespace mpk {

// ------------------------------------------------------------------------------------ verify
constexpr uint32_t kVerifyThreads = 1024, kVerifyWaves = kVerifyThreads / 64;

template <typename T>
__device__ __forceinline__ float logit_of(const T* p, size_t i) {
  if constexpr (sizeof(T) == 4) return as_global(p)[i];
  else return bf16_to_f32(as_global(p)[i]);
}
// The sum over the workgroup, in every thread, and in *before that over the threads in front.
__device__ __forceinline__ double block_sum64(double v, double* red, double* before = nullptr) {
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
  double in = v;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const double x = __shfl_up(in, o, 64);
    if (lane >= (uint32_t)o) in += x;
  }
  __syncthreads();
  if (lane == 63u) red[wave] = in;
  __syncthreads();
  double all = 0., front = 0.;
  for (uint32_t i = 0; i < kVerifyWaves; ++i) {
    if (i == wave) front = all;
    all += red[i];
  }
  if (before) *before = front + (in - v);
  return all;
}

// The walk of one sequence from the root on.  p = softmax(row / temperature) in 64 bits: a random number is compared with sums
// of up to a vocabulary of weights, and which side it falls on is a token.
template <typename T>
__global__ void __launch_bounds__(kVerifyThreads) tree_verify_kernel(VerifyArgs a) {
  __shared__ double red[kVerifyWaves], scale[kTreeNodes], over[kTreeNodes];
  __shared__ uint64_t best[kVerifyWaves];
  __shared__ int32_t parent[kTreeNodes], gone[kTreeNodes];
  __shared__ int32_t found[2];
  const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, seq = blockIdx.x;
  int32_t b = 0, e = 0;
  if (lane < a.n_seqs) {
    b = as_global(a.row_begin)[lane];
    e = as_global(a.row_begin)[lane + 1];
  }
  const uint64_t bad = __ballot(b < 0 || e < b || (uint32_t)e > a.n_rows);
  if (bad) {
    if (seq == 0 && wave == 0 && lane == (uint32_t)__builtin_ctzll(bad)) report_rows(a.err, DE_BAD_ROWS, lane, (uint32_t)e);
    b = e = 0;
  }
  const uint32_t begin = (uint32_t)__builtin_amdgcn_readlane(b, seq), nodes = (uint32_t)__builtin_amdgcn_readlane(e, seq) - begin;
  uint32_t length = 0;
  int32_t next = -1;
  bool out = nodes == 0;
  if (nodes > kTreeNodes) {
    if (threadIdx.x == 0) report_rows(a.err, DE_BAD_TREE, seq, nodes);
    out = true;
  }
  float temperature = 0.f;
  if (!out) {
    TreeLanes tree;
    uint32_t wrong = load_tree(a.parents + begin, nodes, &tree);
    for (uint32_t t = 1; t < wrong; ++t)
      if (parent_of(tree, t) < 0) wrong = t;   // (one root)
    if (wrong < nodes) {
      if (threadIdx.x == 0) report_rows(a.err, DE_BAD_PARENT, seq, wrong);
      out = true;
    }
    if (threadIdx.x < nodes) parent[threadIdx.x] = as_global(a.parents)[begin + threadIdx.x];
    if (a.temperatures) temperature = as_global(a.temperatures)[seq];
    if (!(temperature >= 0.f && temperature < INFINITY)) {
      if (threadIdx.x == 0) report_rows(a.err, DE_BAD_TEMPERATURE, seq, __float_as_uint(temperature));
      out = true;
    }
    __syncthreads();
  }
  const bool greedy = temperature == 0.f;
  const double inv_t = greedy ? 1. : 1. / (double)temperature;
  uint32_t at = 0;
  while (!out) {
    const T* x = (const T*)a.logits + (size_t)(begin + at) * a.stride;
    const float* q = a.draft && !greedy ? a.draft + (size_t)(begin + at) * a.draft_stride : nullptr;
    if (threadIdx.x == 0) as_global(a.path)[begin + length] = (int32_t)at;
    ++length;
    // ---- the largest logit, of equal ones the first
    uint64_t top = 0;
    bool none = false;
    for (uint32_t v = threadIdx.x; v < a.vocab; v += kVerifyThreads) {
      const float y = logit_of(x, v);
      none |= !(y < INFINITY);
      const uint32_t u = __float_as_uint(y + 0.0f);
      const uint64_t key = ((uint64_t)(u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u)) << 32) | (0xFFFFFFFFu - v);
      if (y > -INFINITY) top = max(top, key);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = max(top, (uint64_t)__shfl_xor((unsigned long long)top, o, 64));
    __syncthreads();
    if (lane == 0) best[wave] = top;
    none = __syncthreads_or(none);
    for (uint32_t i = 0; i < kVerifyWaves; ++i) top = max(top, best[i]);
    if (none || !top) {   // no distribution
      if (threadIdx.x == 0 && a.logprobs) as_global(a.logprobs)[begin + length - 1u] = __uint_as_float(0x7FC00000u);
      break;
    }
    const int32_t largest = (int32_t)(0xFFFFFFFFu - (uint32_t)top);
    const double m = (double)logit_of(x, (size_t)largest);
    double total = 0.;
    if (!greedy || a.logprobs) {
      double s = 0.;
      for (uint32_t v = threadIdx.x; v < a.vocab; v += kVerifyThreads) s += exp(((double)logit_of(x, v) - m) * inv_t);
      total = block_sum64(s, red);
    }
    // ---- its children in turn
    uint32_t n_gone = 0;       // tokens that are ruled out (no draft distribution), or subtractions made (one)
    double drawn = 0., mass = total;
    // what is left of the row's distribution at v, not normed: mass is its sum
    auto rest = [&](uint32_t v) {
      double r = exp(((double)logit_of(x, v) - m) * inv_t);
      if (q) {
        const double qv = (double)as_global(q)[v];
        for (uint32_t i = 0; i < n_gone; ++i) r = fmax(0., r * over[i] - scale[i] * qv);
      } else {
        for (uint32_t i = 0; i < n_gone; ++i) r = gone[i] == (int32_t)v ? 0. : r;
      }
      return r;
    };
    int32_t taken = -1;
    for (uint32_t t = at + 1u; t < nodes && taken < 0; ++t) {
      if (parent[t] != (int32_t)at) continue;
      const int32_t token = as_global(a.tokens)[begin + t];
      if (token < 0 || (uint32_t)token >= a.vocab) {
        if (threadIdx.x == 0) report_rows(a.err, DE_BAD_TOKEN, seq, (uint32_t)token);
        continue;
      }
      if (greedy) {
        if (token == largest) taken = (int32_t)t;
        continue;
      }
      const double u = (double)as_global(a.uniforms)[begin + t], r = rest((uint32_t)token);
      if (!q) {
        if (u * mass < r) { taken = (int32_t)t; continue; }
        if (mass - r > 0.) {
          mass -= r;
          if (threadIdx.x == 0) gone[n_gone] = token;
          ++n_gone;
        }
        __syncthreads();
        continue;
      }
      if (a.flags & MPK_TREE_DRAWN_ONCE && drawn >= 1.) continue;   // (the distribution has no more tokens)
      const double mine = (double)as_global(q)[token], norm = a.flags & MPK_TREE_DRAWN_ONCE ? 1. / (1. - drawn) : 1.;
      if (u * norm * mine * mass < r) { taken = (int32_t)t; continue; }
      drawn += mine;
      __syncthreads();
      if (threadIdx.x == 0) { over[n_gone] = 1. / mass; scale[n_gone] = norm; }
      __syncthreads();
      ++n_gone;
      double s = 0.;
      for (uint32_t v = threadIdx.x; v < a.vocab; v += kVerifyThreads) s += rest(v);
      s = block_sum64(s, red);
      if (s > 0.) mass = s;
      else --n_gone;   // (nothing left: as it was)
    }
    if (taken >= 0) {
      const int32_t token = as_global(a.tokens)[begin + taken];
      if (threadIdx.x == 0 && a.logprobs) as_global(a.logprobs)[begin + length - 1u] = (float)(((double)logit_of(x, (size_t)token) - m) * inv_t - log(total));
      at = (uint32_t)taken;
      __syncthreads();
      continue;
    }
    // ---- the end of the walk: the token that follows
    if (greedy) next = largest;
    else {
      const uint32_t share = (a.vocab + kVerifyThreads - 1u) / kVerifyThreads, v0 = min(a.vocab, threadIdx.x * share), v1 = min(a.vocab, v0 + share);
      double s = 0.;
      for (uint32_t v = v0; v < v1; ++v) s += rest(v);
      double before;
      const double all = block_sum64(s, red, &before), goal = (double)as_global(a.uniforms)[begin] * all;
      // the first thread whose end is beyond the goal; by rounding there may be none: the last that has anything
      const uint64_t beyond = __ballot(s > 0. && before + s > goal), any = __ballot(s > 0.);
      if (threadIdx.x == 0) { found[0] = 0x7FFFFFFF; found[1] = -1; }
      __syncthreads();
      if (lane == 0 && beyond) atomicMin(&found[0], (int32_t)(64u * wave + (uint32_t)__builtin_ctzll(beyond)));
      if (lane == 0 && any) atomicMax(&found[1], (int32_t)(64u * wave + 63u - (uint32_t)__builtin_clzll(any)));
      __syncthreads();
      const int32_t who = found[0] != 0x7FFFFFFF ? found[0] : found[1];
      __syncthreads();
      if ((int32_t)threadIdx.x == who) {
        double c = before;
        for (uint32_t v = v0; v < v1; ++v) {
          const double r = rest(v);
          if (r > 0.) next = (int32_t)v;
          c += r;
          if (r > 0. && c > goal) break;
        }
        found[0] = next;
      }
      __syncthreads();
      next = found[0];
    }
    if (threadIdx.x == 0 && a.logprobs) as_global(a.logprobs)[begin + length - 1u] = (float)(((double)logit_of(x, (size_t)next) - m) * inv_t - log(total));
    break;
  }
  if (threadIdx.x == 0) {
    as_global(a.lengths)[seq] = (int32_t)length;
    as_global(a.next)[seq] = next;
  }
  for (uint32_t t = length + threadIdx.x; t < nodes; t += kVerifyThreads) {
    as_global(a.path)[begin + t] = -1;
    if (a.logprobs) as_global(a.logprobs)[begin + t] = 0.f;
  }
}

hipError_t launch_tree_verify(const VerifyArgs& a, bool f32, hipStream_t stream) {
  if (f32) tree_verify_kernel<float><<<dim3(a.n_seqs), dim3(kVerifyThreads), 0, stream>>>(a);
  else tree_verify_kernel<uint16_t><<<dim3(a.n_seqs), dim3(kVerifyThreads), 0, stream>>>(a);
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------ keep
// The rows of a path, place t_k behind the cached rows, to place k.  t_k >= k and ascends, so a row that is written is never one still
// to be read if they are moved in ascending order: a wavefront moves those of one layer, K or V, sequence and KV head, 16 (of 64
// elements 32) at a time, all read before any is written.
template <int D>
__global__ void __launch_bounds__(256) tree_keep_kernel(KeepArgs a) {
  constexpr uint32_t LPR = D / 8, RPI = 64 / LPR, N = 4;   // lanes of a row, rows of a load, loads in flight
  const RowSeqs& s = a.s;
  const uint32_t lane = threadIdx.x & 63u, unit = uniform_u32(blockIdx.x * 4u + (threadIdx.x >> 6));
  if (unit >= s.n_seqs * s.n_kv * 2u * a.n_layers) return;
  const uint32_t seq = unit % s.n_seqs, head = unit / s.n_seqs % s.n_kv, part = unit / (s.n_seqs * s.n_kv), layer = part >> 1;
  const bool first = head == 0 && part == 0;   // of the sequence
  const SeqLanes q = load_seqs<true>(s, unit == 0);
  const uint32_t begin = (uint32_t)__builtin_amdgcn_readlane(q.begin, seq), nodes = (uint32_t)__builtin_amdgcn_readlane(q.end, seq) - begin;
  const uint32_t slot = (uint32_t)__builtin_amdgcn_readlane(q.slot, seq);
  int32_t pos = (int32_t)as_global(s.positions)[seq];
  if (nodes) {
    const int32_t said = as_global(a.lengths)[seq];
    const uint32_t n = said < 0 || (uint32_t)said > nodes ? 0u : (uint32_t)said;
    int32_t path[kTreeNodes / 64], last = -1;
    uint32_t wrong = (uint32_t)said == n ? n : 0u;
    bool fine = (uint32_t)said == n;
#pragma unroll
    for (uint32_t i = 0; i < kTreeNodes / 64u; ++i) {
      const uint32_t k = 64u * i + lane;
      path[i] = k < n ? as_global(a.path)[begin + k] : 0x7FFFFFFF;
      int32_t before = __shfl_up(path[i], 1, 64);
      if (lane == 0) before = last;
      last = __builtin_amdgcn_readlane(path[i], 63);
      const uint64_t bad = __ballot(k < n && (path[i] <= before || (uint32_t)path[i] >= nodes));
      if (bad && fine) {
        wrong = 64u * i + (uint32_t)__builtin_ctzll(bad);
        fine = false;
      }
    }
    if (!fine) {
      if (first && lane == 0) report_rows(s.err, DE_BAD_PATH, seq, wrong);
    } else {
      uint16_t* cache = (part & 1u ? s.v : s.k) + layer * a.layer_stride;
      const uint32_t col = (lane % LPR) * 8u;
      for (uint32_t k0 = 0; k0 < n; k0 += N * RPI) {
        const uint32_t i = k0 >> 6;
        const int32_t mine = i == 0u ? path[0] : i == 1u ? path[1] : i == 2u ? path[2] : path[3];
        u32x4 row[N];
        size_t to[N];
        bool moves[N];
#pragma unroll
        for (uint32_t j = 0; j < N; ++j) {
          const uint32_t k = k0 + j * RPI + lane / LPR;
          const uint32_t t = (uint32_t)__shfl(mine, (int)(k & 63u), 64);
          size_t from = 0;
          moves[j] = k < n && t != k;
          if (moves[j]) {
            const bool ok = cache_row(s, slot, head, (uint32_t)pos + t, &from), ok_to = cache_row(s, slot, head, (uint32_t)pos + k, &to[j]);
            if (!ok || !ok_to) {
              if (first && lane % LPR == 0) report_rows(s.err, DE_BAD_PAGE, seq, (uint32_t)pos + (ok ? k : t));
              moves[j] = false;
            }
          }
          if (moves[j]) row[j] = *as_global((const u32x4*)(cache + from + col));
        }
        drain_vmem();
#pragma unroll
        for (uint32_t j = 0; j < N; ++j)
          if (moves[j]) *as_global((u32x4*)(cache + to[j] + col)) = row[j];
      }
      pos += (int32_t)n;
    }
  }
  if (first && lane == 0 && a.positions_out) as_global(a.positions_out)[seq] = pos;
}

hipError_t launch_tree_keep(const KeepArgs& a, hipStream_t stream) {
  const uint32_t units = a.s.n_seqs * a.s.n_kv * 2u * a.n_layers;
  if (a.s.head_dim == 128u) tree_keep_kernel<128><<<dim3((units + 3u) / 4u), dim3(256), 0, stream>>>(a);
  else tree_keep_kernel<64><<<dim3((units + 3u) / 4u), dim3(256), 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace mpk
