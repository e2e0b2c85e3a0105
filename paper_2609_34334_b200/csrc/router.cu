// The router of an expert-parallel layer: softmax, the topk experts of each token, their counts (which an all-to-allv is made of) and the
// balance loss, forward and backward.  (The paper has no counterpart.)
//
// A row of logits is held by L lanes with V logits each, in registers, for all that is done with it: one read of the logits, no second pass.  Sums over
// the tokens (the probability of each expert, how often it was chosen) stay in a lane's registers and the CTA's shared memory until the CTA has done its rows;
// its sums then go to scratch and one cluster of CTAs adds them in a fixed order, so that the same call gives the same bits.
// Both directions are bound by the issue of instructions and the latency of steps that depend on each other, not by HBM: 32,000 rows of 256 binary32 logits, topk 8, take
// 26 us forward (35.6 MB, 5.4 us at the copy rate; 450 instructions a row) and 16.4 to 17.8 us backward (69 MB, 10.5 us; 340).
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "comm.h"
#include "device_common.cuh"

using namespace hoccl;

namespace hoccl {
namespace {

namespace cg = cooperative_groups;

constexpr int kMaxExperts = 1024, kMaxTopk = 32;
// Warps of a CTA: many, so that few CTAs leave sums behind (32,000 rows of 256 experts: 28.4 us with 8, 25.8 with 16), as far as the candidates' room allows.
template <int V>
constexpr int kWarpsFor = V <= 8 ? 16 : V == 16 ? 8 : 4;
constexpr int kRouteCtas = 2 * kAllSms;          // CTAs of a launch besides one for each rank, one wave; bounds the scratch
constexpr int kEndCtas = 8;                      // one cluster
constexpr int kClusterRanks = 8;                 // ranks up to which a grid may be one cluster that ends by itself

struct RouteArgs {
  int R, experts, topk, groups;
  unsigned long long ld, dld;
  unsigned rows_per_cta;
  int normalize;
  double balance, z, per_choice; // forward: balance_coef * experts, z_coef, 1 / topk
  float* partial;                // forward: see PartialSums; null if the grid is one cluster, which needs none
  float *loss, *saved_out;       // forward
  const float* saved;            // backward
  const float* dloss;
  unsigned first[kMaxRanks + 1]; // prefix sums of CTAs
  unsigned tokens[kMaxRanks];
  const void* logits[kMaxRanks];
  int* indices[kMaxRanks];
  float* weights[kMaxRanks];     // backward: their gradients
  void* dlogits[kMaxRanks];      // forward: the counts
};

// Over the L lanes of a row; a NaN counts only where there is nothing else.
template <int L>
__device__ __forceinline__ float lanes_max(float x) {
  if constexpr (L == 32) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
    return r;
  } else {
#pragma unroll
    for (int d = L / 2; d; d >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
    return x;
  }
}
template <int L>
__device__ __forceinline__ unsigned lanes_min(unsigned x) {
  if constexpr (L == 32) {
    return __reduce_min_sync(0xffffffffu, x);
  } else {
#pragma unroll
    for (int d = L / 2; d; d >>= 1) x = min(x, __shfl_xor_sync(0xffffffffu, x, d));
    return x;
  }
}
template <int L>
__device__ __forceinline__ float lanes_sum(float x) {
#pragma unroll
  for (int d = L / 2; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
  return x;
}
// e^x, off by 2 + |1.17 x| units in the last place; 0 where that is below the least normal number.  (expf is off by 2; its steps for the range of x cost a few
// instructions for each logit in kernels that are bound by their issue, and what they add matters least: it counts for probabilities far below the row's largest.)
__device__ __forceinline__ float exp_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x * 1.4426950408889634f));
  return r;
}
template <int V>
__device__ __forceinline__ float largest(const float* x) {
  float m = x[0];
#pragma unroll
  for (int i = 1; i < V; i++) m = fmaxf(m, x[i]);
  return m;
}

// Which expert lane `lane`'s i-th logit belongs to.  VEC (rows that are whole, aligned vectors): V consecutive ones; else spread for coalescing.
template <int V, int L, bool VEC>
__device__ __forceinline__ int expert_of(int lane, int i) {
  return VEC ? lane * V + i : i * L + lane;
}

template <int DT, int V, int L, bool VEC>
__device__ __forceinline__ void load_row(const void* base, unsigned long long at, int experts, int lane, float* x) {
  if (VEC) {
    constexpr int VE = Traits<DT>::VE;
    const uint4* p = reinterpret_cast<const uint4*>(static_cast<const char*>(base) + at * Traits<DT>::E);
#pragma unroll
    for (int j = 0; j < V / VE; j++) {
      const bool in = (lane * V + j * VE) < experts;
      const uint4 r = in ? __ldcs(p + lane * (V / VE) + j) : make_uint4(0, 0, 0, 0);
      const unsigned w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
      for (int i = 0; i < 4; i++) {
        if (DT == 0) {
          x[j * VE + i] = in ? __uint_as_float(w[i]) : -INFINITY;
        } else {
          x[j * VE + 2 * i] = in ? __uint_as_float(w[i] << 16) : -INFINITY;
          x[j * VE + 2 * i + 1] = in ? __uint_as_float(w[i] & 0xffff0000u) : -INFINITY;
        }
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; i++) {
      const int e = expert_of<V, L, VEC>(lane, i);
      if (DT == 0) x[i] = e < experts ? __ldcs(static_cast<const float*>(base) + at + e) : -INFINITY;
      else x[i] = e < experts ? __uint_as_float((unsigned)__ldcs(static_cast<const unsigned short*>(base) + at + e) << 16) : -INFINITY;
    }
  }
}

// Row whose largest logit is `top`: x -> exp(x - top); their sum and its reciprocal.  A row without a logit above -infinity:
// 0, NaN where the logit is; their sum 0 or NaN, inv 1, and false (top is set to 0).
template <int V, int L>
__device__ __forceinline__ bool softmax_row(float* x, float* top, float* total, float* inv) {
  const bool open = *top > -INFINITY;
  if (!open) *top = 0.0f;
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < V; i++) sum += x[i] = exp_fast(x[i] - *top);
  sum = lanes_sum<L>(sum);
  *inv = open ? __fdividef(1.0f, sum) : 1.0f;
  *total = sum;
  return open;
}

// What the CTAs of a forward launch leave for its end: sums of p, counts of the chosen, rows and the sum of squared logarithms.  In memory,
// CTA after CTA, or in the shared memory of a grid that is one cluster.
// The sums are binary32 all the way: a lane adds a number for each of its rows (tokens / 19,000 of 64 experts at topk 4, / 4,700 of 256), then lanes, warps and CTAs follow in a few
// levels, and the terms are positive, so a sum is off by at most that many roundings, 2^-24 each (measured: the losses by 1e-8 to 3e-7, for 32,000 to 32 million rows).
// Binary64 sums would take a lane 2 V registers instead of V of the 64 that two CTAs an SM leave it.
struct PartialSums {
  static constexpr int kFlight = 16;   // CTAs whose sums a thread has on their way at a time: the latency of one counts
  const float* at;
  int experts;
  __device__ __forceinline__ const float* of(unsigned cta) const { return at + cta * (2 * (size_t)experts + 2); }
  __device__ __forceinline__ float p(unsigned cta, int e) const { return __ldcg(of(cta) + e); }
  __device__ __forceinline__ int count(unsigned cta, int e) const { return __float_as_int(__ldcg(of(cta) + experts + e)); }
  __device__ __forceinline__ float squares(unsigned cta) const { return __ldcg(of(cta) + 2 * experts + 1); }
};
template <class T>
__device__ __forceinline__ T* in_cluster(T* own, unsigned cta) {
  return gridDim.x > 1 ? cg::this_cluster().map_shared_rank(own, cta) : own;
}
struct ClusterSums {
  static constexpr int kFlight = 1;
  float *sums, *sq;   // this CTA's
  int* counts;
  int experts;
  __device__ __forceinline__ float p(unsigned cta, int e) const { return in_cluster(sums, cta)[e]; }
  __device__ __forceinline__ int count(unsigned cta, int e) const { return in_cluster(counts, cta)[e]; }
  __device__ __forceinline__ float squares(unsigned cta) const { return *in_cluster(sq, cta); }
};

// Adds the CTAs' sums in a fixed order.  The CTAs of the grid, one cluster, take 32 experts at a time each, a lane each; a CTA's warps share the ranks, and a rank's
// forward CTAs where there are fewer ranks than warps; beside its expert a lane reads what one forward CTA left of rows and squares.  Each CTA puts its parts of
// the losses into the first one's shared memory, which adds them.  shared: end_words(R, warps) words.
__host__ __device__ constexpr int end_words(int R, int warps) { return (4 + kEndCtas) * kMaxRanks + 64 * R + 66 * warps; }
template <class Sums>
__device__ __forceinline__ void route_end(const RouteArgs& a, const Sums& in, float* shared) {
  constexpr int F = Sums::kFlight;
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, warps = blockDim.x / 32, ctas = gridDim.x;
  double* per_row = reinterpret_cast<double*>(shared);                  // [kMaxRanks]: 1 / rows of a group
  float* parts = shared + 2 * kMaxRanks;                                // [kEndCtas][kMaxRanks], filled in the first CTA
  int* rows = reinterpret_cast<int*>(parts + kEndCtas * kMaxRanks);     // [kMaxRanks]
  float* logs = parts + (kEndCtas + 1) * kMaxRanks;                     // [kMaxRanks]
  float* p_rank = logs + kMaxRanks;                                     // [R][32]
  int* c_rank = reinterpret_cast<int*>(p_rank + 32 * a.R);
  float* p_part = p_rank + 64 * a.R;                                    // [warps][32], then [warps]: squares
  int* c_part = reinterpret_cast<int*>(p_part + 33 * warps);            // [warps][32], then [warps]: rows
  int split = 1;
  while (split * 2 * a.R <= warps) split *= 2;                          // warps of one rank
  constexpr int kGroups = 2;                                            // of a warp: 64 ranks on 32 warps, kClusterRanks on 4
  float loss[kGroups];                                                  // of group warp + i * warps, in this CTA's experts
#pragma unroll
  for (int i = 0; i < kGroups; i++) loss[i] = 0.0f;
  for (int e0 = 32 * (int)blockIdx.x; e0 < a.experts; e0 += 32 * ctas) {
    const int e = e0 + lane;
    for (int r0 = 0; r0 < a.R; r0 += warps / split) {
      const int r = r0 + warp / split;
      float p = 0, z = 0;
      int n = 0, m = 0;
      if (r < a.R) {
        for (unsigned b0 = a.first[r] + warp % split; b0 < a.first[r + 1]; b0 += F * split) {
          float ps[F];
          int ns[F];
#pragma unroll
          for (int u = 0; u < F; u++) {
            const unsigned b = b0 + u * split;
            const bool some = b < a.first[r + 1] && e < a.experts;
            ps[u] = some ? in.p(b, e) : 0.0f;
            ns[u] = some ? in.count(b, e) : 0;
          }
          const unsigned b = b0 + lane * split;
          if (lane < F && b < a.first[r + 1]) {
            m += in.count(b, a.experts);
            z += in.squares(b);
          }
#pragma unroll
          for (int u = 0; u < F; u++) {
            p += ps[u];
            n += ns[u];
          }
        }
      }
      m = __reduce_add_sync(0xffffffffu, m);
      z = lanes_sum<32>(z);
      if (split > 1) {
        p_part[warp * 32 + lane] = p;
        c_part[warp * 32 + lane] = n;
        if (lane == 0) {
          p_part[32 * warps + warp] = z;
          c_part[32 * warps + warp] = m;
        }
        __syncthreads();
        if (warp % split == 0 && r < a.R)
          for (int w = 1; w < split; w++) {
            p += p_part[(warp + w) * 32 + lane];
            n += c_part[(warp + w) * 32 + lane];
            z += p_part[32 * warps + warp + w];
            m += c_part[32 * warps + warp + w];
          }
      }
      if (warp % split == 0 && r < a.R) {
        p_rank[r * 32 + lane] = p;
        c_rank[r * 32 + lane] = n;
        if (lane == 0) {
          rows[r] = m;
          logs[r] = z;
        }
        if (e < a.experts) static_cast<int*>(a.dlogits[r])[e] = n;
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kGroups; i++) {
      const int g = warp + i * warps;
      if (g >= a.groups) break;
      const int r0 = a.groups > 1 ? g : 0, r1 = a.groups > 1 ? g + 1 : a.R;
      float p = 0;
      long long c = 0, n = 0;
#pragma unroll 8
      for (int r = r0; r < r1; r++) {
        p += p_rank[r * 32 + lane];
        c += c_rank[r * 32 + lane];
        n += rows[r];
      }
      // 1 / n by a step of Newton's iteration from binary32's: off by 2^-44, and what comes of it is rounded to binary32 once
      const double guess = n ? (double)__frcp_rn((float)n) : 0.0, each = guess * (2.0 - (double)n * guess), f = (double)c * each * a.per_choice;
      if (e < a.experts) a.saved_out[(size_t)g * (a.experts + 1) + e] = (float)(a.balance * f * each);
      loss[i] += n ? (float)(f * each) * p : p;                         // no rows: 0, or NaN
      if (lane == 0) per_row[g] = each;
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < kGroups; i++) {
    const int g = warp + i * warps;
    if (g >= a.groups) break;
    const float part = lanes_sum<32>(loss[i]);
    if (lane == 0) in_cluster(parts, 0)[blockIdx.x * kMaxRanks + g] = part;
  }
  if (ctas > 1) cg::this_cluster().sync();
  else __syncthreads();
  if (blockIdx.x != 0) return;
  for (int r = threadIdx.x; r < a.R; r += blockDim.x) static_cast<int*>(a.dlogits[r])[a.experts] = rows[r];
  for (int g = threadIdx.x; g < a.groups; g += blockDim.x) {
    const int r0 = a.groups > 1 ? g : 0, r1 = a.groups > 1 ? g + 1 : a.R;
    float l = 0.0f, z = 0.0f;
#pragma unroll
    for (int c = 0; c < kEndCtas; c++) l += c < ctas ? parts[c * kMaxRanks + g] : 0.0f;
#pragma unroll 8
    for (int r = r0; r < r1; r++) z += logs[r];
    a.loss[2 * g] = (float)(a.balance * l);
    a.loss[2 * g + 1] = a.z == 0.0 ? 0.0f : (float)(a.z * per_row[g] * z);   // (the sum of squares may be infinite)
    a.saved_out[(size_t)g * (a.experts + 1) + a.experts] = (float)(2.0 * a.z * per_row[g]);
  }
}

__global__ void __launch_bounds__(1024) route_end_kernel(const __grid_constant__ RouteArgs a) {
  __shared__ __align__(16) float shared[end_words(kMaxRanks, 32)];
  cg::this_cluster().sync();   // every CTA has started, so the first one's shared memory is there; over before the forward's kernel is
  wait_for_stream();
  route_end(a, PartialSums{a.partial, a.experts}, shared);
}

// The topk largest of a row without a pass over it for each: the topk-th largest of the lanes' own largest logits is a bar that at least topk logits reach, and
// few more do (a dozen for 8 of 256); those are collected.  Where a lane can hold each of them and no two are alike, a maximum over the warp finds one after
// the other; up to twice as many, or with some alike, each counts the ones in front of it.  More of them (rows of many equal logits, the bar of which few are
// below; up to all experts) are searched topk times, each lane its share: counting would take the square of their number.
// us for 8 ranks of n rows with counting up to 1, 2 and 4 times the lanes, and whatever the number: 128 experts, topk 8, n = 2048 18.8, 16.7, 16.7, 16.7;
// 256 experts, topk 32, n = 4096 130, 129, 144, 168; 256 experts, topk 8, n = 4096 26.6 each, all logits alike 74, 74, 74, 629.
// (One search of the whole row for each choice took 1090 instructions a row of 256 and 50 us for
// 32,000 rows, most of it on the half-rate integer pipe; this form takes 23 us, 6 of them for ranking and writing, 5.3 for the bar and the collecting.)
template <int DT, int V, int L, bool VEC>
__global__ void __launch_bounds__(kWarpsFor<V> * 32, V <= 8 ? 2 : 1) route_kernel(const __grid_constant__ RouteArgs a) {
  constexpr int W = kWarpsFor<V>, G = 32 / L, kRows = W * G;     // rows of a warp, of the CTA, at a time
  constexpr int kFound = kRows * L * V;
  constexpr int kEnd = W * L * V + end_words(kClusterRanks, W);  // words of the sums and of their end, which reuse the candidates' room
  __shared__ __align__(16) uint2 found[kFound > kEnd / 2 ? kFound : (kEnd + 1) / 2];   // {bits of the logit, expert} of a row's candidates, L * V for each row
  __shared__ int count[L * V + 1];
  __shared__ uint2 chosen[kRows][L];                              // (topk <= L: see kShapes)
  __shared__ int candidates[kRows];
  __shared__ float squares[W];
  static_assert(W * L * V % 2 == 0, "8-byte words in the end's room");
  const int warp = threadIdx.x / 32, lane = threadIdx.x % L, group = threadIdx.x % 32 / L, slot = warp * G + group;
  uint2* mine = found + slot * (L * V);
  for (int e = threadIdx.x; e <= a.experts; e += W * 32) count[e] = 0;
  if (lane == 0) candidates[slot] = 0;
  int r = 0;
  while (blockIdx.x >= a.first[r + 1]) r++;
  const unsigned row0 = (blockIdx.x - a.first[r]) * a.rows_per_cta, row1 = min(a.tokens[r], row0 + a.rows_per_cta);
  wait_for_stream();
  __syncthreads();
  float p_sum[V] = {}, z_sum = 0.0f, log_top = 0.0f, log_total = 1.0f;   // the last: of one of the rows since their logarithms were taken
  int turn = 0;
  for (unsigned base = row0 + warp * G; base < row1; base += kRows) {
    const unsigned row = base + group;
    const bool real = row < row1;
    float x[V], total, inv;
    if (real) {
      load_row<DT, V, L, VEC>(a.logits[r], row * a.ld, a.experts, lane, x);
    } else {
#pragma unroll
      for (int i = 0; i < V; i++) x[i] = -INFINITY;
    }
    float best = largest<V>(x), top = lanes_max<L>(best), bar = top;
    for (int k = 1; k < a.topk; k++) {   // equal ones fall together: the bar only gets lower
      if (best == bar) best = -INFINITY;
      bar = lanes_max<L>(best);
    }
    bar = fmaxf(bar, -3.402823466e38f);
    int here = 0;
#pragma unroll
    for (int i = 0; i < V; i++) here += x[i] >= bar;
    if (here) {   // in places that no order of the lanes is promised for: what follows goes by value and expert alone
      int to = slot * (L * V) + atomicAdd(&candidates[slot], here);
#pragma unroll
      for (int i = 0; i < V; i++)
        if (x[i] >= bar) found[to++] = make_uint2(__float_as_uint(x[i]), expert_of<V, L, VEC>(lane, i));
    }
    __syncwarp();
    const int n = candidates[slot], have = min(n, a.topk);
    const bool open = softmax_row<V, L>(x, &top, &total, &inv);
#pragma unroll
    for (int i = 0; i < V; i++) p_sum[i] += x[i] * inv;
    if (lane == turn) {                  // a logarithm takes as long for one lane as for all: each lane keeps a row's until all have one
      log_top = top;
      log_total = open ? total : total + 1.0f;   // closed: 1, or NaN
    }
    if (++turn == L) {
      const float s = log_top + logf(log_total);
      z_sum += s * s;
      log_top = 0.0f;
      log_total = 1.0f;
      turn = 0;
    }
    const unsigned long long at = (unsigned long long)row * a.topk;
    bool done = false;
    if (__all_sync(0xffffffffu, n <= L)) {
      const uint2 own = lane < n ? mine[lane] : make_uint2(0x7fc00000u, 0);
      const float y = __uint_as_float(own.x);
      float v = y;   // NaN: none, or taken
      int rank = -1;
      for (int k = 0; k < a.topk; k++)
        if (v == lanes_max<L>(v)) {
          rank = k;
          v = __uint_as_float(0x7fc00000u);
        }
      // equal ones fell together unless as many have a rank as there are ranks, and one has the last
      constexpr unsigned kLanes = L == 32 ? 0xffffffffu : (1u << (L & 31)) - 1;
      const unsigned ranked = __ballot_sync(0xffffffffu, rank >= 0) >> (L == 32 ? 0 : group * L) & kLanes;
      const unsigned last = __ballot_sync(0xffffffffu, rank == have - 1 && have) >> (L == 32 ? 0 : group * L) & kLanes;
      done = __all_sync(0xffffffffu, __popc(ranked) == have && (last || !have));
      if (done && rank >= 0) {
        chosen[slot][rank] = own;
        atomicAdd(&count[own.y], 1);
      }
    }
    if (!done && (V <= 2 || __all_sync(0xffffffffu, n <= 2 * L))) {
      for (int c = lane; c < n; c += L) {
        const uint2 own = mine[c];
        const float y = __uint_as_float(own.x);
        int before = 0;
        for (int j = 0; j < n; j++) {
          const uint2 o = mine[j];
          before += __uint_as_float(o.x) > y || (__uint_as_float(o.x) == y && o.y < own.y);
        }
        if (before < a.topk) {
          chosen[slot][before] = own;
          atomicAdd(&count[own.y], 1);
        }
      }
    } else if (V > 2 && !done) {
      // a lane offers the first of its share of what is left
      float best;
      unsigned first, from;
      const auto offer = [&] {
        best = -INFINITY;
        first = ~0u;
        for (unsigned c = lane; c < (unsigned)n; c += L) {
          const uint2 o = mine[c];
          const float y = __uint_as_float(o.x);
          if (y > best || (y == best && o.y < first)) {
            best = y;
            first = o.y;
            from = c;
          }
        }
      };
      offer();
      for (int k = 0; k < a.topk; k++) {
        const float v = lanes_max<L>(best);
        const unsigned e = lanes_min<L>(best == v ? first : ~0u);
        if (first == e && e != ~0u) {   // one lane, as an expert has one place; none where nothing is left
          chosen[slot][k] = make_uint2(__float_as_uint(best), e);
          atomicAdd(&count[e], 1);
          mine[from].x = 0x7fc00000u;
          offer();
        }
      }
    }
    __syncwarp();
    // the chosen are added in the order of their ranks: the candidates' places, and so the lanes that ranked them, are in no certain order
    const uint2 own = lane < have ? chosen[slot][lane] : make_uint2(0, 0xffffffffu);
    const float ex = lane < have ? exp_fast(__uint_as_float(own.x) - top) : 0.0f;
    const float part = a.normalize ? lanes_sum<L>(ex) : 1.0f;
    if (real && lane < a.topk) {
      a.indices[r][at + lane] = (int)own.y;
      // 0 * inv: a NaN in the row reaches its weights either way
      a.weights[r][at + lane] = lane < have ? ex * (a.normalize ? __fdividef(1.0f, part) + 0.0f * inv : inv) : 0.0f;
    }
    if (lane == 0) {
      candidates[slot] = 0;
      if (n) atomicAdd(&count[a.experts], 1);
    }
    __syncwarp();
  }
  {
    const float s = log_top + logf(log_total);
    z_sum += s * s;
  }
  // the CTA's sums: lanes of one expert, then warps, in order
  __syncthreads();
  float* sums = reinterpret_cast<float*>(found);   // [W][experts], the first one the CTA's in the end
#pragma unroll
  for (int i = 0; i < V; i++) {
#pragma unroll
    for (int d = L; d < 32; d <<= 1) p_sum[i] += __shfl_xor_sync(0xffffffffu, p_sum[i], d);
    const int e = expert_of<V, L, VEC>(lane, i);
    if (group == 0 && e < a.experts) sums[warp * a.experts + e] = p_sum[i];
  }
  z_sum = lanes_sum<32>(z_sum);
  if (threadIdx.x % 32 == 0) squares[warp] = z_sum;
  __syncthreads();
  float* out = a.partial ? a.partial + (size_t)blockIdx.x * (2 * a.experts + 2) : nullptr;
  for (int e = threadIdx.x; e < a.experts; e += W * 32) {
    float s = 0.0f;
    for (int w = 0; w < W; w++) s += sums[w * a.experts + e];
    if (out) {
      out[e] = s;
      out[a.experts + e] = __int_as_float(count[e]);
    } else {
      sums[e] = s;
    }
  }
  if (threadIdx.x == 0) {
    float z = 0.0f;
    for (int w = 0; w < W; w++) z += squares[w];
    if (out) {
      out[2 * a.experts] = __int_as_float(count[a.experts]);
      out[2 * a.experts + 1] = z;
    } else {
      squares[0] = z;
    }
  }
  if (out) return;
  if (gridDim.x > 1) cg::this_cluster().sync();
  else __syncthreads();
  route_end(a, ClusterSums{sums, squares, count, a.experts}, sums + W * L * V);
}

template <int DT>
__device__ __forceinline__ float logit_at(const void* base, unsigned long long at) {
  return DT == 0 ? static_cast<const float*>(base)[at] : __uint_as_float((unsigned)static_cast<const unsigned short*>(base)[at] << 16);
}

// dlogits_j = p_j (c_j - shift) + what the weights' gradient adds to the chosen.  The latter comes through shared memory, where expert e of a row lies at
// the place that its lane reads without a bank conflict; what was added is set back to zero behind the row.
template <int DT, int V, int L, bool VEC>
__global__ void __launch_bounds__(kWarpsFor<V> * 32, V <= 8 ? 2 : 1) route_backward_kernel(const __grid_constant__ RouteArgs a) {
  constexpr int W = kWarpsFor<V>, G = 32 / L, kRows = W * G;
  __shared__ float extra[kRows][L * V];
  __shared__ unsigned char seen[kRows][L * V];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % L, group = threadIdx.x % 32 / L, slot = warp * G + group;
  const auto place = [](int e) { return VEC ? e % V * L + e / V : e; };
  int r = 0;
  while (blockIdx.x >= a.first[r + 1]) r++;
  const unsigned row0 = (blockIdx.x - a.first[r]) * a.rows_per_cta, row1 = min(a.tokens[r], row0 + a.rows_per_cta);
  const bool with = a.weights[r] != nullptr;
#pragma unroll
  for (int i = 0; i < V; i++) extra[slot][i * L + lane] = 0.0f;
  wait_for_stream();
  const int g = a.groups > 1 ? r : 0;
  const float scale = a.dloss ? a.dloss[g] : 1.0f, z = a.saved[(size_t)g * (a.experts + 1) + a.experts] * scale;
  float c[V];
#pragma unroll
  for (int i = 0; i < V; i++) {
    const int e = expert_of<V, L, VEC>(lane, i);
    c[i] = e < a.experts ? a.saved[(size_t)g * (a.experts + 1) + e] * scale : 0.0f;
  }
  // a row's logits, this lane's choice of it (expert and gradient of its weight): the next row's are on their way while one is worked on
  float next[V], next_dw = 0.0f;
  int next_e = -1;
  const auto fetch = [&](unsigned row) {
    next_e = -1;
    if (row < row1) {
      if (with && lane < a.topk) {
        next_e = a.indices[r][(unsigned long long)row * a.topk + lane];
        next_dw = a.weights[r][(unsigned long long)row * a.topk + lane];
      }
      load_row<DT, V, L, VEC>(a.logits[r], row * a.ld, a.experts, lane, next);
    } else {
#pragma unroll
      for (int i = 0; i < V; i++) next[i] = -INFINITY;
    }
  };
  fetch(row0 + slot);
  for (unsigned base = row0 + warp * G; base < row1; base += kRows) {
    const unsigned row = base + group;
    const bool real = row < row1;
    const unsigned long long logits_at = row * a.ld;
    const int e = next_e;
    const float dw = next_dw;
    const bool valid = (unsigned)e < (unsigned)a.experts;
    float x[V], total, inv, y = 0.0f;
    if (valid) y = logit_at<DT>(a.logits[r], logits_at + e);
#pragma unroll
    for (int i = 0; i < V; i++) x[i] = next[i];
    fetch(row + kRows);
    float top = lanes_max<L>(largest<V>(x));
    const bool open = softmax_row<V, L>(x, &top, &total, &inv);
    float mean = 0.0f;   // of c under p
#pragma unroll
    for (int i = 0; i < V; i++) mean += (x[i] *= inv) * c[i];
    mean = lanes_sum<L>(mean);
    float shift = mean - (z != 0.0f && open ? z * (top + logf(total)) : 0.0f);
    if (with) {
      const float w = valid ? exp_fast(y - top) * inv : 0.0f, dws = valid ? w * dw : 0.0f;
      const float w_sum = lanes_sum<L>(w), dw_sum = lanes_sum<L>(dws);
      const float per = a.normalize ? (w_sum > 0.0f ? 1.0f / w_sum : w_sum) : 1.0f;   // 0 or NaN stays
      const float inner = dw_sum * per, less = a.normalize ? inner : 0.0f;
      // an index that comes twice in a row adds twice, one after the other in the order of k
      const float add = w * per * (dw - less);
      if (valid) seen[slot][e] = (unsigned char)lane;   // of two lanes that leave their number in one place, one does not find it there
      __syncwarp();
      if (!__any_sync(0xffffffffu, valid && seen[slot][e] != lane)) {
        if (valid) extra[slot][place(e)] = add;
      } else {
        for (int k = 0; k < a.topk; k++) {
          if (valid && lane == k) extra[slot][place(e)] += add;
          __syncwarp();
        }
      }
      if (!a.normalize) shift += inner;
      __syncwarp();
    }
#pragma unroll
    for (int i = 0; i < V; i++) x[i] *= c[i] - shift;
    if (with) {
#pragma unroll
      for (int i = 0; i < V; i++) x[i] += extra[slot][i * L + lane];
      __syncwarp();
      if (valid) extra[slot][place(e)] = 0.0f;
      __syncwarp();
    }
    if (real) {
      const unsigned long long at = row * a.dld;
      if (VEC) {
        constexpr int VE = Traits<DT>::VE;
        uint4* p = reinterpret_cast<uint4*>(static_cast<char*>(a.dlogits[r]) + at * Traits<DT>::E);
#pragma unroll
        for (int j = 0; j < V / VE; j++)
          if (lane * V + j * VE < a.experts) {
            unsigned w[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
              if (DT == 0) w[i] = __float_as_uint(x[j * VE + i]);
              else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(x[j * VE + 2 * i + 1]), "f"(x[j * VE + 2 * i]));
            }
            __stcs(p + lane * (V / VE) + j, make_uint4(w[0], w[1], w[2], w[3]));
          }
      } else {
#pragma unroll
        for (int i = 0; i < V; i++) {
          const int to = expert_of<V, L, VEC>(lane, i);
          if (to < a.experts) {
            if (DT == 0) static_cast<float*>(a.dlogits[r])[at + to] = x[i];
            else static_cast<__nv_bfloat16*>(a.dlogits[r])[at + to] = __float2bfloat16_rn(x[i]);
          }
        }
      }
    }
  }
}

// ---------------------------------------------------------------- host

// Shapes: 8, 16 or 32 lanes a row with 1, 2, 4 or 8 logits each, 32 lanes with 16 or 32.  topk is at most the lanes, so a lane holds one of a row's chosen.
// Fewer lanes put more rows into a warp, which then share what an instruction does for a row beside its logits; more lanes end a row sooner.  us for 8 ranks
// of n rows, forward and backward, with 32 lanes and with the fewest: 32 experts, topk 4, n = 16 5.9 + 2.3 and 6.1 + 2.5, n = 512 9.6 + 2.9 and 9.5 + 2.8,
// n = 8192 27.5 + 18.4 and 17.8 + 8.7; 128 experts, topk 8, n = 16 6.8 + 2.7 and 7.8 + 3.0, n = 512 11.5 + 3.5 and 11.7 + 3.4, n = 8192 40.3 + 24.0 and 35.6 + 15.4.
constexpr int kShapes = 14;
constexpr unsigned long long kFewRows = 4096;   // of all ranks
int shape_with(int lanes, int experts) {        // -1: none
  int log_v = 0;
  while ((lanes << log_v) < experts) log_v++;
  if (lanes == 32) return 8 + log_v;
  return log_v > 3 ? -1 : (lanes == 8 ? 0 : 4) + log_v;
}
int lanes_of(int shape) { return shape < 4 ? 8 : shape < 8 ? 16 : 32; }
int warps_of(int shape) { return shape <= 11 ? kWarpsFor<8> : shape == 12 ? kWarpsFor<16> : kWarpsFor<32>; }
size_t rows_at_once(int shape) { return (size_t)warps_of(shape) * (32 / lanes_of(shape)); }
// The shape with the fewest lanes, of which there are at least `least`.
int compact_shape(int experts, int least) {
  for (int lanes = 8; lanes < 32; lanes *= 2)
    if (lanes >= least && shape_with(lanes, experts) >= 0) return shape_with(lanes, experts);
  return shape_with(32, experts);
}

template <int DT, bool VEC>
const void* route_entry_of(int shape, bool backward) {
  // a lane's logits are at least a vector of 16 bytes
#define ROW(V, L) {reinterpret_cast<const void*>(&route_kernel<DT, V, L, (VEC && V >= Traits<DT>::VE)>), reinterpret_cast<const void*>(&route_backward_kernel<DT, V, L, (VEC && V >= Traits<DT>::VE)>)}
  static const void* const fns[kShapes][2] = {ROW(1, 8),  ROW(2, 8),  ROW(4, 8),  ROW(8, 8),  ROW(1, 16), ROW(2, 16),  ROW(4, 16),
                                              ROW(8, 16), ROW(1, 32), ROW(2, 32), ROW(4, 32), ROW(8, 32), ROW(16, 32), ROW(32, 32)};
#undef ROW
  return fns[shape][backward];
}
const void* route_entry(int dtype, int shape, bool vec, bool backward) {
  if (dtype == HOCCL_FLOAT32) return vec ? route_entry_of<0, true>(shape, backward) : route_entry_of<0, false>(shape, backward);
  return vec ? route_entry_of<1, true>(shape, backward) : route_entry_of<1, false>(shape, backward);
}

bool aligned_to(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

struct Span {
  const char* at;
  size_t bytes;
  bool written;
};
bool spans_clash(std::vector<Span>* v) {
  std::sort(v->begin(), v->end(), [](const Span& a, const Span& b) { return a.at < b.at; });
  const char *end = nullptr, *written_end = nullptr;
  for (const Span& s : *v) {
    if (!s.bytes) continue;
    if (s.at < written_end || (s.written && s.at < end)) return true;
    end = std::max(end, s.at + s.bytes);
    if (s.written) written_end = std::max(written_end, s.at + s.bytes);
  }
  return false;
}
size_t rows_bytes(size_t rows, size_t ld, size_t width, size_t e) { return rows ? ((rows - 1) * ld + width) * e : 0; }

hoccl_result_t check_config(const hoccl_comm* c, const hoccl_route_config_t* f, const void* logits, size_t ld, const size_t* tokens) {
  if (!c || !f || !logits || !tokens) return HOCCL_ERR_INVALID_ARG;
  if (!dtype_size((int)f->dtype)) return HOCCL_ERR_UNSUPPORTED;
  if (f->experts < 1 || f->experts > kMaxExperts || f->topk < 1 || f->topk > kMaxTopk || f->topk > f->experts || ld < (size_t)f->experts || ld > 1ull << 31) return HOCCL_ERR_INVALID_ARG;
  if ((f->normalize | f->per_rank) & ~1) return HOCCL_ERR_INVALID_ARG;
  for (int r = 0; r < c->R; r++)
    if (tokens[r] >= 1ull << 31) return HOCCL_ERR_INVALID_ARG;
  return HOCCL_OK;
}

unsigned long long rows_of(const size_t* tokens, int R) {
  unsigned long long all = 0;
  for (int r = 0; r < R; r++) all += tokens[r];
  return all;
}

// Rows of one CTA and the ranks' first CTAs: as many CTAs as `most` at most, besides one for each rank, and no fewer rows in one than its warps hold.
unsigned share_rows(const size_t* tokens, int R, int shape, unsigned most, unsigned* rows_per_cta, unsigned* first) {
  const unsigned long long all = rows_of(tokens, R);
  const unsigned long long at_once = rows_at_once(shape);
  unsigned long long per = (all + most - 1) / most;
  per = std::max((per + at_once - 1) / at_once, 1ull) * at_once;
  *rows_per_cta = (unsigned)per;
  first[0] = 0;
  for (int r = 0; r < R; r++) first[r + 1] = first[r] + (unsigned)((tokens[r] + per - 1) / per);
  return first[R];
}

// The same in one cluster, if its warps have at most kClusterTurns rows then: a second launch costs as much as a few rows of a warp (8 ranks, 64 experts: 7.4 us
// for 16 rows in one cluster, 9.2 us for 33 in two launches and as much for 24 in one cluster with 3 turns).
constexpr int kClusterTurns = 2;
bool share_in_cluster(const size_t* tokens, int R, int shape, unsigned* rows_per_cta, unsigned* first) {
  if (R > kClusterRanks) return false;
  unsigned long long most = 0;
  for (int r = 0; r < R; r++) most = std::max<unsigned long long>(most, tokens[r]);
  const unsigned long long at_once = rows_at_once(shape), ctas = kEndCtas / R, per = std::max(((most + ctas - 1) / ctas + at_once - 1) / at_once, 1ull) * at_once;
  if (per > kClusterTurns * at_once) return false;
  *rows_per_cta = (unsigned)per;
  first[0] = 0;
  for (int r = 0; r < R; r++) first[r + 1] = first[r] + (unsigned)((tokens[r] + per - 1) / per);
  return true;
}

}  // namespace

void add_router_kernels(std::vector<const void*>* fns) {
  for (int dtype = 0; dtype < 2; dtype++)
    for (int shape = 0; shape < kShapes; shape++)
      for (int form = 0; form < 4; form++) fns->push_back(route_entry(dtype, shape, form & 1, form & 2));
  fns->push_back(reinterpret_cast<const void*>(&route_end_kernel));
}

}  // namespace hoccl

extern "C" {

size_t hoccl_route_scratch_bytes(int R, size_t max_tokens, int experts) {
  if (R < 1 || R > kMaxRanks || experts < 1 || experts > kMaxExperts) return 0;
  const size_t at_once = rows_at_once(shape_with(32, experts));   // the fewest of the shapes it may take
  const size_t ctas = std::min((size_t)R * ((max_tokens + at_once - 1) / at_once), (size_t)kRouteCtas + R);
  return (ctas * (2 * (size_t)experts + 2) * sizeof(float) + 255) / 256 * 256;
}

hoccl_result_t hoccl_route(const void* const* logits, size_t ld, const size_t* tokens, const hoccl_route_config_t* f, int32_t* const* indices,
                           float* const* weights, int32_t* const* counts, float* loss, float* saved, hoccl_comm_t c, hoccl_stream_t stream) {
  const double t0 = now_us();
  hoccl_result_t rc = check_config(c, f, logits, ld, tokens);
  if (rc != HOCCL_OK) return rc;
  if (!indices || !weights || !counts || !loss || !saved || !aligned_to(loss, 4) || !aligned_to(saved, 4)) return HOCCL_ERR_INVALID_ARG;
  if (!std::isfinite(f->balance_coef) || !std::isfinite(f->z_coef)) return HOCCL_ERR_INVALID_ARG;
  const size_t e = dtype_size((int)f->dtype);
  const int groups = f->per_rank ? c->R : 1;
  RouteArgs a = {};
  a.R = c->R;
  a.experts = f->experts;
  a.topk = f->topk;
  a.groups = groups;
  a.ld = ld;
  a.normalize = f->normalize;
  a.balance = f->balance_coef * f->experts;
  a.z = f->z_coef;
  a.per_choice = 1.0 / f->topk;
  a.loss = loss;
  a.saved_out = saved;
  // the bar of the choice is the topk-th of as many numbers as there are lanes: few of them would let many logits over it
  const int wide = shape_with(32, f->experts), compact = compact_shape(f->experts, 2 * f->topk);
  int shape = wide;
  unsigned grid = share_rows(tokens, c->R, wide, kRouteCtas, &a.rows_per_cta, a.first);
  const size_t need = (size_t)grid * (2 * (size_t)f->experts + 2) * sizeof(float);
  bool vec = (f->experts * e) % 16 == 0 && (ld * e) % 16 == 0;
  try {
    std::vector<Span> spans = {{(const char*)loss, 8u * (size_t)groups, true}, {(const char*)saved, (size_t)groups * (f->experts + 1) * 4, true}};
    for (int r = 0; r < c->R; r++) {
      if (!counts[r] || !aligned_to(counts[r], 4)) return HOCCL_ERR_INVALID_ARG;
      a.dlogits[r] = counts[r];
      spans.push_back({(const char*)counts[r], (size_t)(f->experts + 1) * 4, true});
      if (!tokens[r]) continue;
      if (!logits[r] || !indices[r] || !weights[r] || !aligned_to(logits[r], e) || !aligned_to(indices[r], 4) || !aligned_to(weights[r], 4)) return HOCCL_ERR_INVALID_ARG;
      a.tokens[r] = (unsigned)tokens[r];
      a.logits[r] = logits[r];
      a.indices[r] = indices[r];
      a.weights[r] = weights[r];
      vec = vec && aligned_to(logits[r], 16);
      spans.push_back({(const char*)logits[r], rows_bytes(tokens[r], ld, f->experts, e), false});
      spans.push_back({(const char*)indices[r], tokens[r] * f->topk * 4, true});
      spans.push_back({(const char*)weights[r], tokens[r] * f->topk * 4, true});
    }
    if (c->scratch) spans.push_back({(const char*)c->scratch, need, true});
    if (spans_clash(&spans)) return HOCCL_ERR_INVALID_ARG;
  } catch (const std::bad_alloc&) {
    return HOCCL_ERR_INTERNAL;
  }
  bool one_cluster = grid && share_in_cluster(tokens, c->R, wide, &a.rows_per_cta, a.first);   // ends by itself
  if (grid && !one_cluster && compact != wide) {
    one_cluster = share_in_cluster(tokens, c->R, compact, &a.rows_per_cta, a.first);
    if (one_cluster || rows_of(tokens, c->R) > kFewRows) shape = compact;
  }
  grid = one_cluster ? a.first[c->R] : share_rows(tokens, c->R, shape, kRouteCtas, &a.rows_per_cta, a.first);
  if (need && (!c->scratch || c->scratch_bytes < need)) return HOCCL_ERR_SCRATCH;
  a.partial = one_cluster ? nullptr : static_cast<float*>(c->scratch);
  c->stats = hoccl_stats_t{};
  DeviceScope scope(c->device);
  CU_TRY(c, scope.err);
  void* params[1] = {&a};
  if (grid)
    CU_TRY(c, launch_in_order_params(route_entry((int)f->dtype, shape, vec, false), (int)grid, 32 * warps_of(shape), params, (cudaStream_t)stream, 0, one_cluster ? (int)grid : 1));
  if (!one_cluster) {
    const int ctas = std::min(kEndCtas, (f->experts + 31) / 32);   // (one CTA for 256 experts takes 32 us where 8 take 13)
    CU_TRY(c, launch_in_order_params(reinterpret_cast<const void*>(&route_end_kernel), ctas, 1024, params, (cudaStream_t)stream, 0, ctas));
  }
  c->stats.host_launch_us = now_us() - t0;
  return HOCCL_OK;
}

hoccl_result_t hoccl_route_backward(const void* const* logits, size_t ld, const size_t* tokens, const hoccl_route_config_t* f, const int32_t* const* indices,
                                    const float* saved, const float* const* dweights, const float* dloss, void* const* dlogits, size_t dld, hoccl_comm_t c,
                                    hoccl_stream_t stream) {
  const double t0 = now_us();
  hoccl_result_t rc = check_config(c, f, logits, ld, tokens);
  if (rc != HOCCL_OK) return rc;
  if ((dweights && !indices) || !saved || !dlogits || !aligned_to(saved, 4) || !aligned_to(dloss, 4) || dld < (size_t)f->experts || dld > 1ull << 31) return HOCCL_ERR_INVALID_ARG;
  const size_t e = dtype_size((int)f->dtype);
  const int groups = f->per_rank ? c->R : 1;
  RouteArgs a = {};
  a.R = c->R;
  a.experts = f->experts;
  a.topk = f->topk;
  a.groups = groups;
  a.ld = ld;
  a.dld = dld;
  a.saved = saved;
  a.dloss = dloss;
  a.normalize = f->normalize;
  bool vec = (f->experts * e) % 16 == 0 && (ld * e) % 16 == 0 && (dld * e) % 16 == 0;
  try {
    std::vector<Span> spans = {{(const char*)saved, (size_t)groups * (f->experts + 1) * 4, false}};
    if (dloss) spans.push_back({(const char*)dloss, (size_t)groups * 4, false});
    for (int r = 0; r < c->R; r++) {
      if (!tokens[r]) continue;
      if (!logits[r] || !dlogits[r] || !aligned_to(logits[r], e) || !aligned_to(dlogits[r], e)) return HOCCL_ERR_INVALID_ARG;
      if (dweights && (!indices[r] || !dweights[r] || !aligned_to(indices[r], 4) || !aligned_to(dweights[r], 4))) return HOCCL_ERR_INVALID_ARG;
      a.tokens[r] = (unsigned)tokens[r];
      a.logits[r] = logits[r];
      a.dlogits[r] = dlogits[r];
      a.indices[r] = dweights ? const_cast<int32_t*>(indices[r]) : nullptr;
      a.weights[r] = dweights ? const_cast<float*>(dweights[r]) : nullptr;
      vec = vec && aligned_to(logits[r], 16) && aligned_to(dlogits[r], 16);
      // in place: a row is read by the lanes that write it, before they do
      if (!(dlogits[r] == logits[r] && dld == ld)) spans.push_back({(const char*)logits[r], rows_bytes(tokens[r], ld, f->experts, e), false});
      spans.push_back({(const char*)dlogits[r], rows_bytes(tokens[r], dld, f->experts, e), true});
      if (dweights) {
        spans.push_back({(const char*)indices[r], tokens[r] * f->topk * 4, false});
        spans.push_back({(const char*)dweights[r], tokens[r] * f->topk * 4, false});
      }
    }
    if (spans_clash(&spans)) return HOCCL_ERR_INVALID_ARG;
  } catch (const std::bad_alloc&) {
    return HOCCL_ERR_INTERNAL;
  }
  c->stats = hoccl_stats_t{};
  const int shape = rows_of(tokens, c->R) > kFewRows ? compact_shape(f->experts, f->topk) : shape_with(32, f->experts);
  const unsigned grid = share_rows(tokens, c->R, shape, kRouteCtas, &a.rows_per_cta, a.first);
  if (!grid) return HOCCL_OK;
  DeviceScope scope(c->device);
  CU_TRY(c, scope.err);
  CU_TRY(c, launch_in_order(route_entry((int)f->dtype, shape, vec, true), (int)grid, 32 * warps_of(shape), &a, (cudaStream_t)stream));
  c->stats.host_launch_us = now_us() - t0;
  return HOCCL_OK;
}

}  // extern "C"
