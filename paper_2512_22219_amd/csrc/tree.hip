// Trees of drafted tokens: which of them stay (mpk_tree_verify), and their rows in the cache closed up (mpk_tree_keep).
#include <algorithm>
#include <type_traits>

#include "rows_device.h"

namespace mpk {

// ------------------------------------------------------------------------------------ verify
// The walk needs, of each node that it comes to, the largest logit m and Z = sum 2^(k (x - m)), k = log2(e) / temperature, in 64 bits: a random
// number is compared with sums of up to a vocabulary of weights, and which side it falls on is a token.
// It goes in rounds.  A round is a node of the walk or what is left of the node's distribution behind refused children: with a draft
// distribution behind each; of chosen tokens, whose weights are taken off the row's sum meanwhile, where hardly anything is left
// (kVerifyLeft).  A row is cut into chunks, one for each of the sequence's workgroups.  Each leaves its sums where all of them read them,
// reads all of them, and works out for itself how the walk goes on.
// So a round is one pass over a chunk and one exchange between the compute units, and nobody waits for a decision to be passed on.
// Nor does anybody depend on workgroups that may not run yet: sums that have not come after a while are worked out by
// who needs them (the same operations in the same order, the same bits), so that each workgroup alone comes to the end.  It takes its
// time: beside products that fill the device a call waits for room, 64 nodes 280 to 520 us.
//
// Bound by the latency of the rounds, one behind the other; a row of 150000 logits is read in a fraction of a microsecond.  A round of one
// sequence takes 4.4 us: the chunk's logits 0.6 to 0.9, weights 0.5, sums over the workgroup 0.5, the exchange 1.4 to 1.8, the row's sums
// and the children 1; beside the rounds 2 us at the start (lists, the root's row) and 3 to 4 where a token is drawn.  A chain of 6 takes,
// greedy, 8.4 / 12.6 / 17.1 / 21.3 / 25.7 / 29.9 us with 0 / 1 / 2 / 3 / 4 / 5 tokens accepted, sampled 10.3 to 29.0.  Sampled, with one or two
// accepted, 64 nodes 15 to 19; with three or four in the longest walk, 8 x 25 drawn nodes over 128256 logits in bf16 35 to 49, 16 x 64 33 to 40.
// A workgroup a sequence took 505, 650 and 653 us for the last three, 81 for a chain.
// No better were (as it is / so):
//   - units handed out by a counter, whoever comes last deciding (atomics on one address take 20 ns each): 64 nodes 21 / 30
//   - two or three nodes of the tree in a round (1 / 2 / 3): 64 nodes 20.8 / 20.6 / 20.8, 8 x 25 drawn 48 / 59 / 68, a chain of 6, up to two
//     accepted, 8.5 to 17.4 / 10.4 to 17.3 / 11.6
//   - the chunk of the child that is tried next requested while the others' sums come: no change, the slowest of all decides; or summed as
//     well: a chain 16.7 / 16.8, 64 nodes 18.2 / 19.7, 8 x 25 34.8 / 37.3, 16 x 64 40.5 / 43.4
//   - that by four wavefronts while a fifth leads: a round 4.3 / 3.5 where that child is accepted, but 0.5 more once and two workgroups a
//     compute unit instead of three: a chain 8.1 to 16.7 / 8.5 to 15.6, 64 nodes 18.2 / 19.2, 8 x 25 35.5 / 37.4
//   - what is left of a chunk kept in LDS from one refused child to the next: no change, but 48.4 / 42.1 for 13 trees of 55 nodes with ten
//     children a node; 2 % more in the mean of 64 calls
//   - a sequence's workgroups on one XCD: one over 150000 logits 16.7 / 21.0, 13 over 19000 58.3 / 55.3; by a rule on chunks an XCD 0.6 % less in
//     52 calls' mean
//   - words read by 16 bytes: no change
constexpr uint32_t kVerifyThreads = 256, kVerifyWaves = kVerifyThreads / 64;
// Logits of a thread and of a workgroup at once.  Chunks of 2048 / 4096: 64 nodes 18.2 / 21.7 us, 8 x 25 drawn
// 35.5 / 38.3.
constexpr uint32_t kVerifyLane = 8, kVerifyStep = kVerifyThreads * kVerifyLane;
constexpr uint32_t kVerifyEach = kVerifyChunks / 64;   // chunks of a lane when they are joined: the lane-th, the 64 + lane-th
constexpr uint32_t kVerifyWorkgroups = 768;   // of a call at most: as many as run at once, three a compute unit
// Ticks of 10 ns until others' sums are worked out: several rounds, and more by the steps of a chunk and the subtractions in them, so that it happens
// only where a workgroup does not run.  (16 rows of 4 million logits, 43 steps, in bf16 and drawn, 412 us, with 20 us whatever the steps 654; 8 million
// in fp32, sampled, 271, 323.)
constexpr uint32_t kVerifyPatience = 2000, kVerifyPatienceStep = 200, kVerifyPatienceLess = 20;
// Refused chosen tokens are taken off the sums until less than this is left of them; then what is left is summed anew, against its own largest logit.
// A difference has the sums' error, some 1e-13 of what they began with, so what is compared with random numbers and drawn from stays within 1e-10.  A
// node comes to this with the same probability: its numbers have refused all the rest.
constexpr double kVerifyLeft = 1. / 1024.;
constexpr uint32_t kVerifyTags = 1u << 30, kVerifyTagsJitter = 64u;   // rounds until tags start over (MPK_DEBUG_JITTER: often)

struct VerifyPlan {
  uint32_t chunks, steps;   // of a row: a workgroup each; of a chunk
};
// What became of a node's children: one of them was accepted (its place), or none (the walk ends), the row has no distribution, or the
// next is to be tried on what is left behind one refused.
enum : int32_t { kNone = -1, kNoDistribution = -2, kRefused = -3 };

__device__ __forceinline__ void put64(uint64_t* p, uint64_t v) { __hip_atomic_store(as_global(p), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// 2^d for d <= 0, 0 below -1000 (and for -inf): a polynomial p of degree 9 on [-1/2, 1/2], within 2.1e-14 of the value, and the power of two
// added to the exponent.  p(0) = 1 exactly, p'(0) = ln 2: the points of p are +-sqrt(y), y the zeros of the Chebyshev polynomial of degree 5 over the
// interval [0, 1/4] of squares, moved so that the least is 0.  So the weight of a row's largest logit is 1, however many sums it goes through.
template <bool ZERO = true>   // false: d is not below -1000
__device__ __forceinline__ double exp2_64(double d) {
  const double big = 6755399441055744.0;   // 1.5 x 2^52: the sum's low bits are d as a whole number
  const double t = d + big, f = d - (t - big);
  double p = 0x1.b64f6fecb838ep-24;
  p = fma(p, f, 0x1.63e7f7eb368ffp-20);
  p = fma(p, f, 0x1.ffcb7f06ad7afp-17);
  p = fma(p, f, 0x1.430896a28d2bbp-13);
  p = fma(p, f, 0x1.5d87fe8d66e50p-10);
  p = fma(p, f, 0x1.3b2ab724d2acep-7);
  p = fma(p, f, 0x1.c6b08d7045c65p-5);
  p = fma(p, f, 0x1.ebfbdff81b648p-3);
  p = fma(p, f, 0x1.62e42fefa39efp-1);
  p = fma(p, f, 1.0);
  const uint32_t hi = (uint32_t)__double2hiint(p) + ((uint32_t)__double2loint(t) << 20);
  return ZERO && d < -1000. ? 0. : __hiloint2double((int)hi, __double2loint(p));
}
// (x and m as they are in 64 bits: their difference loses nothing that shows)
__device__ __forceinline__ double weight(float x, double m, double k) { return exp2_64(((double)x - m) * k); }

__device__ __forceinline__ double lane64(double v, uint32_t lane) {
  return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), lane), __builtin_amdgcn_readlane(__double2loint(v), lane));
}
template <int CTRL>
__device__ __forceinline__ double dpp64(double v) {
  return __hiloint2double(__builtin_amdgcn_update_dpp(0, __double2hiint(v), CTRL, 0xF, 0xF, true), __builtin_amdgcn_update_dpp(0, __double2loint(v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ double wave_sum64(double v) {
  v += dpp64<0xB1>(v);    // lane ^ 1
  v += dpp64<0x4E>(v);    // lane ^ 2
  v += dpp64<0x141>(v);   // mirror of 8
  v += dpp64<0x140>(v);   // mirror of 16
  return (lane64(v, 0) + lane64(v, 16)) + (lane64(v, 32) + lane64(v, 48));
}
__device__ __forceinline__ double wave_before64(double v, double* all) {   // the sum over the lanes in front, and over all
  const uint32_t row = (threadIdx.x & 63u) >> 4;
  double x = v;
  x += dpp64<0x111>(x);   // from 1, 2, 4 and 8 lanes in front, in a row of 16
  x += dpp64<0x112>(x);
  x += dpp64<0x114>(x);
  x += dpp64<0x118>(x);
  const double r0 = lane64(x, 15), r1 = r0 + lane64(x, 31), r2 = r1 + lane64(x, 47);
  *all = r2 + lane64(x, 63);
  return dpp64<0x111>(x) + (row == 0u ? 0. : row == 1u ? r0 : row == 2u ? r1 : r2);
}

template <typename T>
__device__ __forceinline__ float logit_of(const T* p, size_t i) {
  if constexpr (sizeof(T) == 4) return as_global(p)[i];
  else return bf16_to_f32(as_global(p)[i]);
}
// 16 bytes from an address of any alignment of the elements.
typedef uint32_t u32x4_of4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_of2 __attribute__((ext_vector_type(4), aligned(2)));
// N neighbouring elements of a row of n from the i-th on as fp32, `fill` behind the last; by loads of E of them, the row's last E where some of
// these lie behind its end.
template <uint32_t N, uint32_t E, typename T>
__device__ __forceinline__ void load_row(const T* x, uint32_t i, uint32_t n, float fill, float* y) {
  constexpr uint32_t PER = 16 / sizeof(T);
  using Bytes = std::conditional_t<sizeof(T) == 4, u32x4_of4, u32x4_of2>;
  if (n < E) {
#pragma unroll
    for (uint32_t j = 0; j < N; ++j) y[j] = j < E && i + j < n ? logit_of(x, i + j) : fill;
    return;
  }
#pragma unroll
  for (uint32_t j = 0; j < N; j += E) {
    const uint32_t at = min(i + j, n - E);
#pragma unroll
    for (uint32_t l = 0; l < E; l += PER) {
      const u32x4 b = *(const MPK_GLOBAL Bytes*)(x + at + l);
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) {
        if constexpr (PER == 4) y[j + l + e] = __uint_as_float(b[e]);
        else { y[j + l + 2 * e] = bf16_lo(b[e]); y[j + l + 2 * e + 1] = bf16_hi(b[e]); }
      }
    }
    if (__any(at != i + j)) {   // (elements in front of the i-th have been read too: they are another load's)
#pragma unroll
      for (uint32_t e = 0; e < E; ++e) y[j + e] = at + e < i + j ? fill : y[j + e];
    }
  }
}
// Where the load of the i-th element (a multiple of E from a load's first) starts.
__device__ __forceinline__ uint32_t row_start(uint32_t i, uint32_t n, uint32_t E) { return n < E ? i : min(i, n - E); }

// T: the logits; DRAFT: there are draft distributions.
template <typename T, bool DRAFT>
__global__ void __launch_bounds__(kVerifyThreads, 3) tree_verify_kernel(VerifyArgs a, VerifyPlan p) {
  constexpr uint32_t E = 16 / sizeof(T), V = kVerifyLane / E;   // logits of a load, loads of a step
  __shared__ double part_sum[kVerifyChunks], total[kTreeNodes], over[kTreeNodes], scale[kTreeNodes], sums[kVerifyWaves];
  __shared__ float top[kTreeNodes], maxima[kVerifyWaves], hit_logit[kVerifyWaves];
  __shared__ uint32_t places[kVerifyWaves], hit[kVerifyWaves], last[kVerifyWaves], zeros[kVerifyThreads];
  __shared__ struct { int32_t code; uint32_t lack, place, child, subtracted; float most; } told;   // by wavefront 0 (most: what weights are against)
  __shared__ uint8_t path[kTreeNodes];
  __shared__ int32_t tokens[kTreeNodes];   // -1: none; wavefront 0 has them at once, the others behind the first round
  __shared__ float uniforms[kTreeNodes];
  const uint32_t lane = threadIdx.x & 63u, wave = uniform_u32(threadIdx.x >> 6), seq = blockIdx.x % a.n_seqs, own = blockIdx.x / a.n_seqs;   // its chunk
  VerifySync& sync = a.sync[seq];

  // ---- the sequence, checked by every wavefront for itself
  int32_t b = 0, e = 0;
  if (lane < a.n_seqs) {
    b = as_global(a.row_begin)[lane];
    e = as_global(a.row_begin)[lane + 1];
  }
  float temperature = 0.f;
  if (a.temperatures) temperature = as_global(a.temperatures)[seq];
  uint32_t tag = uniform_u32(ld_relaxed(&sync.tag));   // of the last round of the call before
  const bool teller = own == 0u && wave == 0u;
  const uint64_t bad = __ballot(b < 0 || e < b || (uint32_t)e > a.n_rows);
  if (bad) {
    if (teller && seq == 0 && lane == (uint32_t)__builtin_ctzll(bad)) report_rows(a.err, DE_BAD_ROWS, lane, (uint32_t)e);
    b = e = 0;
  }
  const uint32_t begin = (uint32_t)__builtin_amdgcn_readlane(b, seq), nodes = (uint32_t)__builtin_amdgcn_readlane(e, seq) - begin;
  bool out = nodes == 0;
  float y[kVerifyLane];   // a chunk's first logits: the root's are on their way meanwhile
  auto row_of = [&](uint32_t node) { return (const T*)a.logits + (size_t)(begin + node) * a.stride; };
  const uint32_t chunk_logits = p.steps * kVerifyStep;
  auto request = [&](uint32_t node, uint32_t chunk, uint32_t step, float (&y)[kVerifyLane]) {
    const T* x = row_of(node);
    const uint32_t v0 = chunk * chunk_logits + step * kVerifyStep + threadIdx.x * E;
#pragma unroll
    for (uint32_t j = 0; j < V; ++j) load_row<E, E>(x, v0 + j * kVerifyThreads * E, a.vocab, -INFINITY, y + j * E);
  };
  if (!out) request(0u, own, 0u, y);
  TreeLanes tree;
  int32_t token[kTreeNodes / 64u] = {};   // (on their way beside the parents: a round waits for the children's logits alone, 2 % of a call)
  float number[kTreeNodes / 64u] = {};
  if (wave == 0 && nodes <= kTreeNodes) {
#pragma unroll
    for (uint32_t i = 0; i < kTreeNodes / 64u; ++i) {
      const uint32_t t = 64u * i + lane;
      if (t > 0u && t < nodes) {
        token[i] = as_global(a.tokens)[begin + t];
        if (a.temperatures) number[i] = as_global(a.uniforms)[begin + t];
      }
    }
  }
  if (nodes > kTreeNodes) {
    if (teller && lane == 0) report_rows(a.err, DE_BAD_TREE, seq, nodes);
    out = true;
  } else if (!out) {
    uint32_t wrong = load_tree(a.parents + begin, nodes, &tree);
#pragma unroll
    for (uint32_t i = kTreeNodes / 64u; i-- > 0;) {   // (one root)
      const uint64_t roots = __ballot(tree.of[i] < 0 && 64u * i + lane < nodes) & ~(uint64_t)(i == 0u);
      if (roots) wrong = min(wrong, 64u * i + (uint32_t)__builtin_ctzll(roots));
    }
    if (wrong < nodes) {
      if (teller && lane == 0) report_rows(a.err, DE_BAD_PARENT, seq, wrong);
      out = true;
    } else if (wave == 0) {
#pragma unroll
      for (uint32_t i = 0; i < kTreeNodes / 64u; ++i) {
        const uint32_t t = 64u * i + lane;
        const bool fine = (uint32_t)token[i] < a.vocab;
        if (!fine && teller) report_rows(a.err, DE_BAD_TOKEN, seq, (uint32_t)token[i]);
        tokens[t] = fine ? token[i] : -1;
        uniforms[t] = number[i];
      }
    }
    if (!(temperature >= 0.f && temperature < INFINITY)) {
      if (teller && lane == 0) report_rows(a.err, DE_BAD_TEMPERATURE, seq, __float_as_uint(temperature));
      out = true;
    }
  }
  if (out) {
    if (own) return;
    if (threadIdx.x == 0) {
      as_global(a.lengths)[seq] = 0;
      as_global(a.next)[seq] = -1;
    }
    for (uint32_t t = threadIdx.x; t < nodes; t += kVerifyThreads) {
      as_global(a.path)[begin + t] = -1;
      if (a.logprobs) as_global(a.logprobs)[begin + t] = 0.f;
    }
    return;
  }
  const bool greedy = temperature == 0.f, weigh = !greedy || a.logprobs;
  const double k = 1.4426950408889634 / (greedy ? 1. : (double)temperature);
  auto draft_of = [&](uint32_t node) { return a.draft + (size_t)(begin + node) * a.draft_stride; };
  auto parents_of = [&](uint32_t i) { return i == 0u ? tree.of[0] : i == 1u ? tree.of[1] : i == 2u ? tree.of[2] : tree.of[3]; };   // of the nodes 64 i + lane

  // ---- tokens that were chosen and refused: of the node's children in front of the `from`-th, a thread each (-1: none)
  auto refused = [&](uint32_t node, uint32_t from) {
    return threadIdx.x < nodes && threadIdx.x < from && parents_of(wave) == (int32_t)node ? tokens[threadIdx.x] : -1;
  };
  // Which of a thread's elements of the step from v0 on are the token of another thread (or its own): a bit each, in `zeros` of the thread that load
  // (of E elements) number n of the step belongs to, thread_of(n), from first_of(n) on.  By all threads.
  auto mark = [&](int32_t gone, uint32_t v0, auto thread_of, auto first_of) {
    zeros[threadIdx.x] = 0;
    __syncthreads();
    const uint32_t n = ((uint32_t)gone - v0) / E;
    if (gone >= 0 && (uint32_t)gone >= v0 && n < kVerifyStep / E) atomicOr(&zeros[thread_of(n)], 1u << (first_of(n) + (uint32_t)gone - row_start(v0 + n * E, a.vocab, E)));
    __syncthreads();
    return zeros[threadIdx.x];
  };

  // ---- a chunk of a node's row, by the workgroup: a wavefront's largest logit, its first place, and the sum of the weights against that; then, in
  // wavefront 0, the chunk's (in m a NaN: the row has no distribution).  The first step's logits may be there already.  less: without the
  // tokens that are gone.
  auto sum_weights = [&](uint32_t node, uint32_t chunk, float (&ahead)[kVerifyLane], bool there, bool less, int32_t gone, float& m, double& sum, uint32_t& first) {
    float most = -INFINITY;
    uint32_t at = 0xFFFFFFFFu;
    double s = 0.;
    bool none = false;
    if (!there) request(node, chunk, 0u, ahead);
    for (uint32_t step = 0; step < p.steps; ++step) {
      float y[kVerifyLane];
#pragma unroll
      for (uint32_t j = 0; j < kVerifyLane; ++j) y[j] = ahead[j];
      if (!DRAFT && less) {
        const uint32_t out = mark(gone, chunk * chunk_logits + step * kVerifyStep, [](uint32_t n) { return n % kVerifyThreads; }, [](uint32_t n) { return n / kVerifyThreads * E; });
#pragma unroll
        for (uint32_t j = 0; j < kVerifyLane; ++j) y[j] = out >> j & 1u ? -INFINITY : y[j];
      }
      if (step + 1u < p.steps) request(node, chunk, step + 1u, ahead);   // (one step ahead / not: 16 x 64 nodes 33 to 41 / 36 to 43 us)
      float mx = y[0];
#pragma unroll
      for (uint32_t j = 0; j < kVerifyLane; ++j) {
        mx = fmaxf(mx, y[j]);
        none |= !(y[j] < INFINITY);
      }
      const float wm = wave_max_dpp(mx);
      if (greedy && wm > most) {
        uint32_t j = kVerifyLane;
#pragma unroll
        for (uint32_t l = kVerifyLane; l-- > 0;) j = y[l] == wm ? l : j;
        at = j < kVerifyLane ? row_start(chunk * chunk_logits + step * kVerifyStep + (j / E * kVerifyThreads + threadIdx.x) * E, a.vocab, E) + j % E : 0xFFFFFFFFu;
      }
      if (wm > most) {
        if (most > -INFINITY) s *= exp2_64(((double)most - (double)wm) * k);
        most = wm;
      }
      if (weigh && most > -INFINITY) {
        // (a weight below 2^-1000 is that here: neither shows in the sum)
#pragma unroll
        for (uint32_t j = 0; j < kVerifyLane; ++j) s += exp2_64<false>(fmax(((double)y[j] - (double)most) * k, -1000.));
      }
    }
    s = wave_sum64(s);
    if (greedy) at = wave_min_u32(at);
    none = __any(none);
    if (lane == 0) { maxima[wave] = none ? __uint_as_float(0x7FC00000u) : most; sums[wave] = s; places[wave] = at; }
    __syncthreads();
    if (wave) return;
    m = maxima[0];
    none = m != m;
#pragma unroll
    for (uint32_t i = 1; i < kVerifyWaves; ++i) { none |= maxima[i] != maxima[i]; m = fmaxf(m, maxima[i]); }
    const float mine = maxima[lane % kVerifyWaves];   // (a lane each)
    s = mine > -INFINITY ? sums[lane % kVerifyWaves] * weight(mine, (double)m, k) : 0.;
    first = 0xFFFFFFFFu;
    sum = 0.;
#pragma unroll
    for (uint32_t i = 0; i < kVerifyWaves; ++i) {
      sum += lane64(s, i);
      if (maxima[i] == m) first = min(first, places[i]);
    }
    if (none) m = __uint_as_float(0x7FC00000u);
  };
  // ... and what is left of it after n subtractions.
  auto sum_rest = [&](uint32_t node, uint32_t chunk, uint32_t n, float (&ahead)[kVerifyLane], double& sum) {
    const float* q = draft_of(node);
    const uint32_t v0 = chunk * chunk_logits + threadIdx.x * E;
    const double m = (double)top[node];
    double s = 0.;
    float z_ahead[kVerifyLane];
    auto request_both = [&](uint32_t step) {
      request(node, chunk, step, ahead);
#pragma unroll
      for (uint32_t j = 0; j < V; ++j) load_row<E, E>(q, v0 + step * kVerifyStep + j * kVerifyThreads * E, a.vocab, 0.f, z_ahead + j * E);
    };
    request_both(0u);
    for (uint32_t step = 0; step < p.steps; ++step) {
      float y[kVerifyLane], z[kVerifyLane];
#pragma unroll
      for (uint32_t j = 0; j < kVerifyLane; ++j) { y[j] = ahead[j]; z[j] = z_ahead[j]; }
      if (step + 1u < p.steps) request_both(step + 1u);
      double r[kVerifyLane];
#pragma unroll
      for (uint32_t j = 0; j < kVerifyLane; ++j) r[j] = weight(y[j], m, k);
      for (uint32_t i = 0; i < n; ++i) {
        const double o = over[i], f = scale[i];
#pragma unroll
        for (uint32_t j = 0; j < kVerifyLane; ++j) r[j] = fmax(0., r[j] * o - (double)z[j] * f);
      }
#pragma unroll
      for (uint32_t j = 0; j < kVerifyLane; ++j) s += r[j];
    }
    s = wave_sum64(s);
    if (lane == 0) sums[wave] = s;
    __syncthreads();
    if (wave == 0) sum = (sums[0] + sums[1]) + (sums[2] + sums[3]);
  };

  // ---- a wavefront: a node's children in turn.  Its lanes have the children among 64 nodes: token (-1: none), the token's logit, random number, draft.
  struct Children {
    int32_t token;
    float x, u, q;
  };
  auto children_of = [&](uint32_t node, uint32_t i) {
    const uint32_t t = 64u * i + lane;
    Children c = {-1, 0.f, 0.f, 0.f};
    if (t < nodes && parents_of(i) == (int32_t)node) c.token = tokens[t];
    if (c.token >= 0 && !greedy) {
      c.x = logit_of(row_of(node), (size_t)c.token);
      c.u = uniforms[t];
      if constexpr (DRAFT) c.q = as_global(draft_of(node))[c.token];
    }
    return c;
  };
  // Tokens that were chosen: r is w without the refused tokens, mass its sum; part are the sums of the lane's chunks, and lose them too.  The children
  // from `child` on, until one is accepted or what is left is to be summed anew.  near: those among the nodes that `child` is among.
  auto try_chosen = [&](uint32_t node, const Children& near, double m, uint32_t largest, uint32_t& child, double mass, double (&part)[kVerifyEach]) -> int32_t {
    const double enough = mass * kVerifyLeft;
#pragma unroll 1
    for (uint32_t i = child >> 6; i * 64u < nodes; ++i) {
      const Children c = i == child >> 6 ? near : children_of(node, i);
      if (greedy) {
        const uint64_t same = __ballot(c.token >= 0 && (uint32_t)c.token == largest);
        if (same) return (int32_t)(64u * i + (uint32_t)__builtin_ctzll(same));
        continue;
      }
      const double w = c.token >= 0 ? weight(c.x, m, k) : 0.;
      for (uint64_t set = __ballot(c.token >= 0 && 64u * i + lane >= child); set; set &= set - 1ull) {
        const uint32_t j = (uint32_t)__builtin_ctzll(set);
        const int32_t mine = __builtin_amdgcn_readlane(c.token, j);
        bool twin = lane < j && c.token == mine;   // of an earlier child: ruled out by now
        for (uint32_t g = node >> 6; g < i; ++g) twin |= parents_of(g) == (int32_t)node && 64u * g + lane < nodes && tokens[64u * g + lane] == mine;
        const double r = __any(twin) ? 0. : lane64(w, j), u = (double)__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(c.u), j));
        if (u * mass < r || r >= mass) return (int32_t)(64u * i + j);   // (r is mass where no other token is left: u < 1)
        mass -= r;
        const uint32_t of = (uint32_t)mine / chunk_logits;   // (something: what is left of a chunk may be lost in the difference, and u = 0 draws it)
#pragma unroll
        for (uint32_t h = 0; h < kVerifyEach; ++h) part[h] = of == 64u * h + lane ? fmax(0x1p-1000, part[h] - r) : part[h];
        if (mass < enough) {
          child = 64u * i + j + 1u;
          return kRefused;
        }
      }
    }
    return kNone;
  };
  // Tokens that were drawn: r is w after n subtractions, mass its sum; the children from `child` on, until one is accepted or refused.  near:
  // the children among the nodes that `child` is among.  norm: what a refused one's subtraction takes the draft times.
  auto try_drawn = [&](uint32_t node, const Children& near, double m, double mass, uint32_t n, uint32_t& child, double& drawn, double& norm) -> int32_t {
#pragma unroll 1
    for (uint32_t i = child >> 6; i * 64u < nodes; ++i) {
      const Children c = i == child >> 6 ? near : children_of(node, i);
      const uint64_t set = __ballot(c.token >= 0 && 64u * i + lane >= child);
      if (!set) continue;
      if (a.flags & MPK_TREE_DRAWN_ONCE && drawn >= 1.) return kNone;   // (the distribution has no more tokens)
      const uint32_t j = (uint32_t)__builtin_ctzll(set);
      auto of_it = [&](float v) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), j)); };
      double r = weight(of_it(c.x), m, k);
      const double share = (double)of_it(c.q), u = (double)of_it(c.u);
      for (uint32_t s = 0; s < n; ++s) r = fmax(0., r * over[s] - share * scale[s]);
      norm = a.flags & MPK_TREE_DRAWN_ONCE ? 1. / (1. - drawn) : 1.;
      if (u * norm * share * mass < r) return (int32_t)(64u * i + j);
      drawn += share;
      child = 64u * i + j + 1u;
      return kRefused;
    }
    return kNone;
  };

  // ---- the exchange: a chunk's sums in words that have the round's tag each (the place where something is greedy)
  const uint32_t words = greedy ? 4u : 3u;
  // (a line of 64 bytes a chunk: side by side 8 x 25 drawn took 39 to 51 us, so 30 to 46)
  auto leave = [&](float m, double sum, uint32_t first) {
    if (lane < words) {
      const uint32_t v = lane == 0u ? __float_as_uint(m) : lane == 1u ? (uint32_t)__double2hiint(sum) : lane == 2u ? (uint32_t)__double2loint(sum) : first;
      put64(&sync.word[tag % kVerifyDepth][own][lane], (uint64_t)tag << 32 | v);
    }
  };

  // ---- rounds
  uint32_t at = 0, length = 1, child = 0, subtracted = 0;   // the walk's node, its nodes; the children to be tried, from here on; the node's subtractions
  int32_t ended;
  const double uniform = greedy ? 0. : (double)as_global(a.uniforms)[begin];   // of the root: for the next token
  if (threadIdx.x == 0) path[0] = 0;
  bool there = true, rest = false;   // the chunk's first logits are on their way; the round is of what is left of the node's row
  double now[kVerifyEach] = {}, drawn = 0., mass = 0.;   // wavefront 0: the lane's chunks, the draft's share of the refused tokens, the sum of the chunks
  for (;;) {
    ++tag;
    if (a.jitter) {   // (MPK_DEBUG_JITTER: up to twice the others' patience)
      const uint64_t t0 = wall_clock64(), wait = (uint64_t)((tag * 2654435761u ^ blockIdx.x * 2246822519u) >> 16) % (2u * kVerifyPatience);
      while (wall_clock64() - t0 < wait) __builtin_amdgcn_s_sleep(8);
    }
    // The children and their logits are on their way beside the chunk
    Children near = {-1, 0.f, 0.f, 0.f};
    if (wave == 0) near = children_of(at, child >> 6);
    // ---- this workgroup's chunk, then the others' sums: wavefront 0 gets them
    float part_max[kVerifyEach];
    double part[kVerifyEach];
    uint32_t part_place[kVerifyEach], chunk = own;
    bool got[kVerifyEach];
#pragma unroll
    for (uint32_t h = 0; h < kVerifyEach; ++h) {
      got[h] = 64u * h + lane >= p.chunks;
      part_max[h] = -INFINITY;
      part[h] = 0.;
      part_place[h] = 0xFFFFFFFFu;
    }
    for (uint32_t patience = kVerifyPatience + (p.steps - 1u) * kVerifyPatienceStep + (DRAFT && rest ? p.steps * subtracted * kVerifyPatienceLess : 0u);; patience = 0) {
      float m = 0.f;
      double sum = 0.;
      uint32_t first = 0;
      if (DRAFT && rest) sum_rest(at, chunk, subtracted, y, sum);
      else sum_weights(at, chunk, y, there && patience, rest, rest ? refused(at, child) : -1, m, sum, first);
      there = false;
      if (patience) {
        if (wave == 0) leave(m, sum, first);
      } else {
#pragma unroll
        for (uint32_t h = 0; h < kVerifyEach; ++h)
          if (64u * h + lane == chunk) { part_max[h] = m; part[h] = sum; part_place[h] = first; got[h] = true; }
      }
      if (wave == 0) {
        uint64_t since = 0;
        uint32_t lack;
        for (;;) {
          bool ahead = false;   // (others are a round ahead: it will not come)
          uint64_t w[kVerifyEach][4];
#pragma unroll
          for (uint32_t h = 0; h < kVerifyEach; ++h)
            if (!got[h]) {
#pragma unroll
              for (uint32_t l = 0; l < 4; ++l) w[h][l] = l < words ? ld_relaxed64(&sync.word[tag % kVerifyDepth][64u * h + lane][l]) : (uint64_t)tag << 32;
            }
          lack = kVerifyChunks;
#pragma unroll
          for (uint32_t h = kVerifyEach; h-- > 0;) {
            if (!got[h]) {
              got[h] = true;
#pragma unroll
              for (uint32_t l = 0; l < 4; ++l) got[h] &= (uint32_t)(w[h][l] >> 32) == tag;
              ahead |= (int32_t)((uint32_t)(w[h][0] >> 32) - tag) > 0;
              part_max[h] = __uint_as_float((uint32_t)w[h][0]);
              part[h] = __hiloint2double((int)(uint32_t)w[h][1], (int)(uint32_t)w[h][2]);
              part_place[h] = (uint32_t)w[h][3];
            }
            const uint64_t lacks = __ballot(!got[h]);
            if (lacks) lack = 64u * h + (uint32_t)__builtin_ctzll(lacks);
          }
          if (lack == kVerifyChunks || __any(ahead)) break;
          if (!since) since = wall_clock64();
          else if (wall_clock64() - since > patience) break;
        }
        if (lane == 0) told.lack = lack;
        if (lack == kVerifyChunks) {
          // ---- the row's sums over its chunks, and the node's children
          int32_t c = kNoDistribution;
          double m;
          if (!DRAFT || !rest) {
            float mc = part_max[0];
            bool none = part_max[0] != part_max[0];
#pragma unroll
            for (uint32_t h = 1; h < kVerifyEach; ++h) { mc = fmaxf(mc, part_max[h]); none |= part_max[h] != part_max[h]; }
            const float most = wave_max_dpp(mc);
            m = (double)most;
            double s = 0.;
            uint32_t place = 0xFFFFFFFFu;
#pragma unroll
            for (uint32_t h = 0; h < kVerifyEach; ++h) {
              now[h] = part_max[h] > -INFINITY ? part[h] * weight(part_max[h], m, k) : 0.;
              s += now[h];
              if (part_max[h] == most) place = min(place, part_place[h]);
            }
            mass = wave_sum64(s);
            drawn = 0.;
            const uint32_t largest = greedy ? wave_min_u32(place) : 0u;
            if (lane == 0) {
              if (!rest) {
                top[at] = most;
                total[at] = mass;
              }
              told.most = most;
              told.place = largest;
            }
            if (!__any(none) && most > -INFINITY) c = !DRAFT || greedy ? try_chosen(at, near, m, largest, child, mass, now) : kRefused;
            if (!DRAFT && lane == 0) told.child = child;
          } else {
            m = (double)top[at];
            double s = 0.;
#pragma unroll
            for (uint32_t h = 0; h < kVerifyEach; ++h) s += part[h];
            s = wave_sum64(s);
            if (s > 0.) {
              mass = s;
#pragma unroll
              for (uint32_t h = 0; h < kVerifyEach; ++h) now[h] = part[h];
            } else --subtracted;   // (nothing would be left: as it was)
            c = kRefused;
          }
          if (DRAFT && c == kRefused) {
            double norm;
            c = try_drawn(at, near, m, mass, subtracted, child, drawn, norm);
            if (lane == 0) {
              if (c == kRefused) { over[subtracted] = 1. / mass; scale[subtracted] = norm; }
              told.child = child;
              told.subtracted = subtracted;
            }
          }
          if (lane == 0) told.code = c;
        }
      }
      __syncthreads();
      chunk = uniform_u32(told.lack);
      if (chunk == kVerifyChunks) break;   // (else one that is not there after a while: worked out here)
      __syncthreads();
    }
    // ---- the walk
    ended = (int32_t)uniform_u32((uint32_t)told.code);
    rest = ended == kRefused;
    if (DRAFT) subtracted = uniform_u32(told.subtracted);
    if (DRAFT || rest) child = uniform_u32(told.child);
    if (rest) {
      ++subtracted;
      continue;
    }
    if (ended < 0) break;
    at = (uint32_t)ended;
    child = at & ~63u;
    subtracted = 0;
    if (threadIdx.x == 0) path[length] = (uint8_t)at;
    ++length;
  }
  uint32_t left = 0;   // how many workgroups are through, their words (wavefront 0's stores) in place
  if (wave == 0) {
    drain_vmem();
    if (lane == 0) left = __hip_atomic_fetch_add(as_global(&sync.left), 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1u;
#pragma unroll
    for (uint32_t h = 0; h < kVerifyEach; ++h) part_sum[64u * h + lane] = now[h];
  }
  __syncthreads();

  // ---- the end of the walk: the token that follows is drawn from what is left of the last node's row, in the first chunk that ends beyond
  // the goal (by rounding there may be none: the last that has anything).  The workgroup that has this chunk writes the results.
  const bool draws = ended == kNone && !greedy;
  uint32_t chunk = 0;
  double goal = 0.;
  auto choose = [&]() {
    double front = 0.;   // (the lanes' first chunks, then their second ones)
    double before[kVerifyEach], mine[kVerifyEach];
#pragma unroll
    for (uint32_t h = 0; h < kVerifyEach; ++h) {
      double all;
      mine[h] = part_sum[64u * h + lane];
      before[h] = front + wave_before64(mine[h], &all);
      front += all;
    }
    const double aim = uniform * front;
    uint32_t beyond = kVerifyChunks, last = kVerifyChunks;
#pragma unroll
    for (uint32_t h = kVerifyEach; h-- > 0;) {
      const uint64_t any = __ballot(mine[h] > 0.), set = __ballot(mine[h] > 0. && before[h] + mine[h] > aim);
      if (set) beyond = 64u * h + (uint32_t)__builtin_ctzll(set);
      if (any && last == kVerifyChunks) last = 64u * h + 63u - (uint32_t)__builtin_clzll(any);
    }
    chunk = beyond != kVerifyChunks ? beyond : last;
#pragma unroll
    for (uint32_t h = 0; h < kVerifyEach; ++h)
      if (chunk >> 6 == h) goal = aim - lane64(before[h], chunk & 63u);
  };
  if (draws) choose();
  if (own == (chunk == kVerifyChunks ? 0u : chunk)) {
    // (what the path's nodes say about the tokens behind them, a thread each: on its way meanwhile)
    float said = 0.f;
    const uint32_t here = threadIdx.x < length ? path[threadIdx.x] : 0u;
    if (a.logprobs && threadIdx.x + 1u < length) said = logit_of(row_of(here), (size_t)tokens[path[threadIdx.x + 1u]]);
    int32_t token = ended == kNone && greedy ? (int32_t)told.place : -1;
    float logit = 0.f;   // the token's
    if (draws) {
      const int32_t gone = DRAFT ? -1 : refused(at, nodes);   // (all children have been refused)
      for (; chunk != kVerifyChunks; choose()) {
        if (lane == 0) { hit[wave] = 0xFFFFFFFFu; last[wave] = 0; }
        double front = 0.;
        uint32_t late = 0;   // the last token that has anything, + 1
        for (uint32_t step = 0; step < p.steps; ++step) {
          const uint32_t v0 = chunk * chunk_logits + step * kVerifyStep, v = v0 + threadIdx.x * kVerifyLane;
          float z[kVerifyLane];
          load_row<kVerifyLane, E>(row_of(at), v, a.vocab, -INFINITY, y);
          if (DRAFT && subtracted) load_row<kVerifyLane, E>(draft_of(at), v, a.vocab, 0.f, z);
          const uint32_t zero = DRAFT ? 0u : mark(gone, v0, [](uint32_t n) { return n / V; }, [](uint32_t n) { return n % V * E; });
          double r[kVerifyLane], s = 0.;
          const double m = (double)told.most;
#pragma unroll
          for (uint32_t j = 0; j < kVerifyLane; ++j) r[j] = weight(y[j], m, k);   // (of one that is gone it may be anything)
          if constexpr (DRAFT) {
            for (uint32_t i = 0; i < subtracted; ++i) {
              const double o = over[i], f = scale[i];
#pragma unroll
              for (uint32_t j = 0; j < kVerifyLane; ++j) r[j] = fmax(0., r[j] * o - (double)z[j] * f);
            }
          } else {
#pragma unroll
            for (uint32_t j = 0; j < kVerifyLane; ++j) r[j] = zero >> j & 1u ? 0. : r[j];
          }
#pragma unroll
          for (uint32_t j = 0; j < kVerifyLane; ++j) s += r[j];
          double all, before = wave_before64(s, &all);
          if (lane == 0) sums[wave] = all;
          __syncthreads();
          before += front;
#pragma unroll
          for (uint32_t i = 0; i < kVerifyWaves; ++i) {
            if (i < wave) before += sums[i];
            front += sums[i];
          }
          const bool crosses = s > 0. && before + s > goal;
          const uint64_t any = __ballot(s > 0.), cross = __ballot(crosses);
          // the wavefront's first thread that ends beyond the goal, or its last that has anything: a token and its logit
          if (any && lane == (cross ? (uint32_t)__builtin_ctzll(cross) : 63u - (uint32_t)__builtin_clzll(any))) {
            uint32_t which = 0xFFFFFFFFu;
            float logit = 0.f;
            bool over_it = false;
            double sum = before;
#pragma unroll
            for (uint32_t j = 0; j < kVerifyLane; ++j) {
              sum += r[j];
              if (r[j] > 0. && !over_it) {
                which = row_start(v + j / E * E, a.vocab, E) + j % E;
                logit = y[j];
                over_it = crosses && sum > goal;
              }
            }
            (crosses ? hit : last)[wave] = crosses ? which : which + 1u;
            hit_logit[wave] = logit;
          }
          __syncthreads();
          token = -1;
#pragma unroll
          for (uint32_t i = 0; i < kVerifyWaves; ++i)
            if (token < 0 && hit[i] != 0xFFFFFFFFu) { token = (int32_t)hit[i]; logit = hit_logit[i]; }
          if (token >= 0) break;
#pragma unroll
          for (uint32_t i = 0; i < kVerifyWaves; ++i)
            if (last[i] > late) { late = last[i]; logit = hit_logit[i]; }
          __syncthreads();
        }
        if (token < 0) token = (int32_t)late - 1;
        if (token >= 0) break;
        if (threadIdx.x == 0) part_sum[chunk] = 0.;   // (nothing was left of it)
        __syncthreads();
      }
    }
    if (threadIdx.x == 0) {
      as_global(a.lengths)[seq] = (int32_t)length;
      as_global(a.next)[seq] = token;
    }
    if (threadIdx.x + 1u == length && token >= 0) said = greedy ? top[at] : logit;
    if (threadIdx.x < nodes) {
      const uint32_t t = threadIdx.x;
      as_global(a.path)[begin + t] = t < length ? (int32_t)here : -1;
      if (a.logprobs) {
        float lp = 0.f;
        if (t < length) {
          lp = (float)(((double)said - (double)top[here]) * k * 0.69314718055994531 - log(total[here]));
          if (t + 1u == length && token < 0) lp = __uint_as_float(0x7FC00000u);
        }
        as_global(a.logprobs)[begin + t] = lp;
      }
    }
  }
  // ---- who has been counted last leaves the tag for the next call.  Tags start over before they run out, with the words cleared: nobody looks
  // at these any more.
  if (wave || uniform_u32(left) != p.chunks) return;
  if (tag >= (a.jitter ? kVerifyTagsJitter : kVerifyTags)) {
    for (uint32_t i = lane; i < kVerifyDepth * kVerifyChunks * 8u; i += 64u) put64(&sync.word[0][0][0] + i, 0ull);
    tag = 0;
  }
  if (lane == 0) {
    st_act_u32(&sync.left, 0u);
    st_act_u32(&sync.tag, tag);
  }
}

hipError_t launch_tree_verify(const VerifyArgs& a, bool f32, hipStream_t stream) {
  VerifyPlan p{};
  const uint32_t most = std::min(kVerifyChunks, kVerifyWorkgroups / a.n_seqs);
  p.steps = (a.vocab + most * kVerifyStep - 1u) / (most * kVerifyStep);
  p.chunks = (a.vocab + p.steps * kVerifyStep - 1u) / (p.steps * kVerifyStep);
  auto run = [&](auto kernel) { kernel<<<dim3(p.chunks * a.n_seqs), dim3(kVerifyThreads), 0, stream>>>(a, p); };
  if (a.draft) run(f32 ? tree_verify_kernel<float, true> : tree_verify_kernel<uint16_t, true>);
  else run(f32 ? tree_verify_kernel<float, false> : tree_verify_kernel<uint16_t, false>);
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------ keep
// The rows of a path, place t_k behind the cached rows, to place k.  t_k >= k and ascends, so a row that is written is never one still
// to be read if they are moved in ascending order: a wavefront moves those of one layer, K or V, sequence and KV head, 16 (of 64
// elements 32) at a time, all read before any is written.  Bound by latency (lists, path, pages, rows, one behind the other): 5 of 32 nodes in 36
// layers 3.4 us, 16 paths on pages, 9 MB read and written, 7.0 (a copy takes 1.8).  The path requested beside its length: 3.4, 7.1.
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
