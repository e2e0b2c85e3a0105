// The operators of a training step that read gradients: the AdamW step over many tensors, the same step on R ranks with sharded
// state (reduce-scatter, update, all-gather in one kernel) and the gradient norm.  (The paper has no counterpart.)
//
// All three stream.  An element of a bf16 weight with a binary32 master and states moves 28 bytes (gradient 2, master, m and v 4 in and 4 out, weight 2 out) and
// takes 35 instructions: HBM bounds it (201 M weights 821 us, 6.87 TB/s).  With 8-bit states it moves 16 bytes and takes 70: the issue of
// instructions bounds it (548 to 573 us with the same arrays again and again, 585 to 591 with three sets in turn: 5.5 TB/s), so its arithmetic goes two numbers an
// instruction and every step of the rounding is counted.
// The unit of work is a block of 256 elements, one warp's: the elements that share a scale in 8-bit states, so that a block's
// largest value is one warp reduction and states of either kind have one shape.  In an aligned, whole block lane l holds elements 8 l .. 8 l + 7 (32-byte
// accesses of binary32 arrays, 16 of bf16, 8 of codes); in any other one elements l, l + 32, ...  Both run the same arithmetic: alignment changes no bit.
// A CTA's warps take the blocks of one tile of one tensor, so that which tensor, and where in its arrays, is the same for the whole CTA: addresses are a
// uniform base and the thread's own constant offset (found by each warp for itself they were a third of the instructions of a step with 8-bit states).
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "comm.h"
#include "device_common.cuh"

using namespace hoccl;

namespace hoccl {
namespace {

namespace cg = cooperative_groups;

constexpr int kBlock = HOCCL_STATE_BLOCK;
constexpr int kWarps = 4, kOptThreads = 32 * kWarps, kTile = kWarps * kBlock;
static_assert(kBlock == 256, "a warp holds a block with 8 elements a lane");

// weights: binary32; bf16; bf16 beside a binary32 master
enum { W_FP32 = 0, W_BF16 = 1, W_MASTER = 2 };

// Twice the same number, as an operand of two operations at once: in the kernel's parameters it takes neither registers nor moves.
struct Pair {
  unsigned long long w;
};
struct AdamScalars {
  Pair beta1, grad1, beta2, grad2;   // grad1 = 1 - beta1, grad2 = 1 - beta2, rounded once
  Pair eps, one, half, minus_half, minus_one;   // one: see add2
  float lr, step_size, root_scale;   // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
  float grad_scale;
  unsigned seed;
  const float* factor;
  const hoccl_adamw_rates_t* rates;
};

struct AdamRow {
  void *param, *m, *v;
  const void* grad;
  float *master, *m_scale, *v_scale;
  unsigned long long n;
  float decay;
  unsigned flags;   // bit 0: aligned for eight elements at a time; the rest: number of the tensor in the caller's table
};
// Tensors by value: a launch carries up to 32 (2.4 KB of parameters; a call takes 2.9 us of the host's time), 128 (9.4 KB, 3.1 us) or 420 (31 KB, about the most
// there is, 3.9 us).  With 64 in the middle a call of 96 tensors takes 3.9 us, with 96 3.0, with 128 3.1, with 192 3.3; one of 128 tensors 3.9, 3.9, 3.1 and 3.3.
template <int N>
struct AdamTableT {
  int n, pad;
  AdamRow row[N];
  unsigned first[N + 1];        // prefix sums of tiles: a CTA each
};
using AdamTableSmall = AdamTableT<32>;
using AdamTableMiddle = AdamTableT<128>;
using AdamTable = AdamTableT<420>;
static_assert(sizeof(AdamTable) + sizeof(AdamScalars) <= 32764, "kernel parameters");

struct ShardedArgs {
  int R;
  float decay;
  unsigned per_rank;             // tiles of a full chunk: a CTA each
  unsigned long long count, q;
  unsigned long long aligned, paired;   // bit c: chunk c, for eight and for two elements at a time
  const void* grad[kMaxRanks];
  void* param[kMaxRanks];
  void *m[kMaxRanks], *v[kMaxRanks];
  float *master[kMaxRanks], *m_scale[kMaxRanks], *v_scale[kMaxRanks];
};

// ---------------------------------------------------------------- device: memory

// Eight consecutive elements of an aligned array, read or written once: no reuse to keep lines for.
__device__ __forceinline__ void load8(const float* p, float* x) {
  asm volatile("ld.global.L1::no_allocate.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7])
               : "l"(p)
               : "memory");
}
__device__ __forceinline__ void store8(float* p, const float* x) {
  asm volatile("st.global.L1::no_allocate.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]),
               "f"(x[5]), "f"(x[6]), "f"(x[7])
               : "memory");
}
__device__ __forceinline__ void widen8(uint4 r, float* x) {
  const unsigned w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; i++) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ unsigned pack_bf16(float lo, float hi) {
  unsigned d;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}

// Two binary32 operations in one instruction, each rounded by itself: the step is bound by the issue of instructions, not by the lanes.
struct Two {
  unsigned long long w;
};
__device__ __forceinline__ Two two(float a, float b) {
  Two r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r.w) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ Two two(float a) { return two(a, a); }
__device__ __forceinline__ Two two(Pair a) { return Two{a.w}; }
__device__ __forceinline__ void split(Two x, float* a) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a[0]), "=f"(a[1]) : "l"(x.w)); }
__device__ __forceinline__ Two mul2(Two a, Two b) {
  Two r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.w) : "l"(a.w), "l"(b.w));
  return r;
}
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
  Two r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.w) : "l"(a.w), "l"(b.w), "l"(c.w));
  return r;
}

// a + b: the compiler turns a product and a packed sum into one fused operation, however each is marked; times a 1 that it cannot see through it does not.
__device__ __forceinline__ Two add2(Two a, Two b, Pair one) { return fma2(a, two(one), b); }

// Square roots rounded to nearest, of numbers within kRootLow .. kRootHigh: an approximate reciprocal root, one step of Goldschmidt's iteration for the
// root and half the reciprocal, and the remainder's correction (P. Markstein, "Computation of elementary functions on the IBM RISC System/6000
// processor", 1990).  hoccl_selftest_root compares every number of the range with __fsqrt_rn.
constexpr float kRootLow = 0x1p-96f, kRootHigh = 0x1p96f;
__device__ __forceinline__ Two root_in_range(Two x, Two half, Two minus_half, Two minus_one) {
  float a[2], y[2];
  split(x, a);
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y[0]) : "f"(a[0]));
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y[1]) : "f"(a[1]));
  const Two yy = two(y[0], y[1]);
  Two g = mul2(x, yy), h = mul2(yy, minus_half);
  const Two r = fma2(g, h, half);
  g = fma2(g, r, g);
  h = fma2(h, r, h);
  return fma2(fma2(g, g, mul2(x, minus_one)), h, g);
}

__device__ __forceinline__ float max_nan(float a, float b) {   // NaN if either is
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// How a block is read and written: element by element within the array's end, element by element all of it, two elements at a time (arrays that start on two
// elements' boundary; the sharded step alone: half as many accesses of every rank's arrays), or eight (on 8 elements').  The plain step takes elements one by one
// wherever it cannot take eight.  Pairs would serve arrays on two elements' boundary alone: 50 M weights there, one by one and in pairs, bf16 with master
// 213 and 208 us, without 179 and 162, with 8-bit states 166 and 144; arrays one element off 213, 180 and 166.
enum Mode { ENDS, WHOLE, PAIRS, VECTORS };
// Where a thread's eight elements lie in its tile, and whether they exist where `left` elements do.
template <Mode MODE>
__device__ __forceinline__ unsigned element(int i) {
  if (MODE == VECTORS) return threadIdx.x * 8 + i;
  const unsigned warp = (threadIdx.x & ~31u) * 8, lane = threadIdx.x & 31;
  return MODE == PAIRS ? warp + i / 2 * 64 + lane * 2 + i % 2 : warp + i * 32 + lane;
}
template <Mode MODE>
__device__ __forceinline__ bool exists(int i, unsigned left) {
  return MODE != ENDS || element<MODE>(i) < left;
}

// DT 0 binary32, 1 bf16.  base: the tile's first element; `left`: elements of the array from there on (a block that is not ENDS lies within them).
template <int DT, Mode MODE>
__device__ __forceinline__ void load_floats(const void* base, unsigned left, float* x) {
  if (DT == 0) {
    const float* p = static_cast<const float*>(base);
    if (MODE == VECTORS) {
      load8(p + threadIdx.x * 8, x);
    } else if (MODE == PAIRS) {
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const float2 r = __ldcs(reinterpret_cast<const float2*>(p + element<MODE>(i)));
        x[i] = r.x;
        x[i + 1] = r.y;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; i++) x[i] = exists<MODE>(i, left) ? __ldcs(p + element<MODE>(i)) : 0.0f;
    }
  } else {
    const unsigned short* p = static_cast<const unsigned short*>(base);
    if (MODE == VECTORS) {
      widen8(__ldcs(reinterpret_cast<const uint4*>(p) + threadIdx.x), x);
    } else if (MODE == PAIRS) {
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const unsigned r = __ldcs(reinterpret_cast<const unsigned*>(p + element<MODE>(i)));
        x[i] = __uint_as_float(r << 16);
        x[i + 1] = __uint_as_float(r & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; i++) x[i] = exists<MODE>(i, left) ? __uint_as_float((unsigned)__ldcs(p + element<MODE>(i)) << 16) : 0.0f;
    }
  }
}
// A thread's eight gradients: as vectors of 16 bytes where they can be, so that those of several ranks fit the registers.
template <int DT, Mode MODE>
struct Raw {
  float x[8];
  __device__ __forceinline__ void load(const void* base, unsigned left) { load_floats<DT, MODE>(base, left, x); }
  __device__ __forceinline__ void widen(float* y) const {
#pragma unroll
    for (int i = 0; i < 8; i++) y[i] = x[i];
  }
};
template <>
struct Raw<1, PAIRS> {
  unsigned r[4];
  __device__ __forceinline__ void load(const void* base, unsigned) {
#pragma unroll
    for (int i = 0; i < 4; i++) r[i] = __ldcs(reinterpret_cast<const unsigned*>(static_cast<const unsigned short*>(base) + element<PAIRS>(2 * i)));
  }
  __device__ __forceinline__ void widen(float* y) const { widen8(make_uint4(r[0], r[1], r[2], r[3]), y); }
};
template <>
struct Raw<1, VECTORS> {
  uint4 r;
  __device__ __forceinline__ void load(const void* base, unsigned) { r = __ldcs(static_cast<const uint4*>(base) + threadIdx.x); }
  __device__ __forceinline__ void widen(float* y) const { widen8(r, y); }
};
template <int DT, Mode MODE>
__device__ __forceinline__ void store_floats(void* base, unsigned left, const float* x) {
  if (DT == 0) {
    float* p = static_cast<float*>(base);
    if (MODE == VECTORS) {
      store8(p + threadIdx.x * 8, x);
    } else if (MODE == PAIRS) {
#pragma unroll
      for (int i = 0; i < 8; i += 2) __stcs(reinterpret_cast<float2*>(p + element<MODE>(i)), make_float2(x[i], x[i + 1]));
    } else {
#pragma unroll
      for (int i = 0; i < 8; i++)
        if (exists<MODE>(i, left)) __stcs(p + element<MODE>(i), x[i]);
    }
  } else {
    unsigned short* p = static_cast<unsigned short*>(base);
    if (MODE == VECTORS) {
      __stcs(reinterpret_cast<uint4*>(p) + threadIdx.x, make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])));
    } else if (MODE == PAIRS) {
#pragma unroll
      for (int i = 0; i < 8; i += 2) __stcs(reinterpret_cast<unsigned*>(p + element<MODE>(i)), pack_bf16(x[i], x[i + 1]));
    } else {
#pragma unroll
      for (int i = 0; i < 8; i++)
        if (exists<MODE>(i, left)) __stcs(p + element<MODE>(i), __bfloat16_as_ushort(__float2bfloat16_rn(x[i])));
    }
  }
}

// ---------------------------------------------------------------- device: 8-bit states

// The 32-bit finalizer of MurmurHash3 (Appleby, public domain), as far as before its last step, h ^ (h >> 16).
__device__ __forceinline__ unsigned mix_most(unsigned h) {
  h = (h ^ (h >> 16)) * 0x85EBCA6Bu;
  return (h ^ (h >> 13)) * 0xC2B2AE35u;
}
__device__ __forceinline__ unsigned mix(unsigned h) {
  h = mix_most(h);
  return h ^ (h >> 16);
}
__device__ __forceinline__ unsigned tensor_key(unsigned seed, unsigned tensor) { return mix(seed + tensor * 0x9E3779B9u); }
// The two halves of a finished word: what m and what the root are rounded with.  (h >> 16 as a permutation of bytes: the shift would be merged with the one
// that places the bits, and the mask that this needs costs an instruction a number.)
struct Halves {
  unsigned m, root;
};
__device__ __forceinline__ Halves halves(unsigned h) {
  h = mix_most(h);
  const unsigned high = __byte_perm(h, 0, 0x4432);
  return Halves{(h ^ high) & 0xffffu, high};
}
// Of the elements of a tile that starts at element `at` of its tensor: mix(tile_key + offset).  (A tile does not straddle a multiple of 2^32.)
__device__ __forceinline__ unsigned tile_key(unsigned key, unsigned long long at) { return (unsigned)at + (unsigned)(at >> 32) * 0x632BE5ABu + key; }

template <Mode MODE>
__device__ __forceinline__ void load_codes(const void* base, unsigned left, float scale, float* x) {
  const unsigned char* p = static_cast<const unsigned char*>(base);
  unsigned short pair[4];
  if (MODE == VECTORS) {
    const uint2 r = __ldcs(reinterpret_cast<const uint2*>(p) + threadIdx.x);
    pair[0] = (unsigned short)r.x;
    pair[1] = (unsigned short)(r.x >> 16);
    pair[2] = (unsigned short)r.y;
    pair[3] = (unsigned short)(r.y >> 16);
  } else if (MODE == PAIRS) {
#pragma unroll
    for (int i = 0; i < 4; i++) pair[i] = __ldcs(reinterpret_cast<const unsigned short*>(p + element<MODE>(2 * i)));
  } else {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const unsigned lo = exists<MODE>(2 * i, left) ? __ldcs(p + element<MODE>(2 * i)) : 0, hi = exists<MODE>(2 * i + 1, left) ? __ldcs(p + element<MODE>(2 * i + 1)) : 0;
      pair[i] = (unsigned short)(lo | hi << 8);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const float2 f = __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2(pair[i], __NV_E4M3)));
    split(mul2(two(f.x, f.y), two(scale)), x + 2 * i);
  }
}

// One number on the grid of e4m3 (3 bits of mantissa from 2^-6 on, steps of 2^-9 below), rounded towards zero or, with the chance of what is
// cut off, away from it.  rnd: 16 random bits, which come to lie just below the mantissa's third bit.  Adding 2^-6 to a number below
// 2^-6 puts it where binary32's own grid of 3 bits has those steps.
__device__ __forceinline__ float round_normal(float u, unsigned rnd) { return __uint_as_float((__float_as_uint(u) + rnd * 16) & 0xfff00000u); }
__device__ __forceinline__ float round_any(float u, unsigned rnd) {
  const float shift = fabsf(u) < 0.015625f ? copysignf(0.015625f, u) : 0.0f;
  return copysignf(round_normal(u + shift, rnd) - shift, u);
}
// Stores a block (x >= 0 for the root) and its scale.  The whole warp takes part.  A block without a number below 2^-6 of the codes' range, the usual
// one, does without the steps for those: 4 instructions a number instead of 9.
template <Mode MODE, bool ROOT>
__device__ __forceinline__ void store_codes(void* base, float* scales, unsigned left, const float* x, const Halves* word) {
  float top = fabsf(x[0]), low = top;
#pragma unroll
  for (int i = 1; i < 8; i++) {
    top = max_nan(top, fabsf(x[i]));
    low = fminf(low, fabsf(x[i]));
  }
  top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top)));   // of non-negative numbers and NaN the words have their order
  const bool some = top > 1e-35f;
  const float inv = some ? __frcp_rn(top) * 448.0f : 0.0f;
  if ((threadIdx.x & 31) == 0) scales[threadIdx.x / 32] = some ? top * (1.0f / 448.0f) : top == top ? 0.0f : top;
  float q[8];
  if (__any_sync(0xffffffffu, low * inv < 0.015625f)) {
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const float u = x[i] * inv;
      q[i] = round_any(u, ROOT ? word[i].root : word[i].m);
      if (ROOT && u > 0.0f) q[i] = fmaxf(q[i], 0.001953125f);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      split(mul2(two(x[i], x[i + 1]), two(inv)), q + i);
#pragma unroll
      for (int j = i; j < i + 2; j++) q[j] = round_normal(q[j], ROOT ? word[j].root : word[j].m);
    }
  }
  unsigned short pair[4];
#pragma unroll
  for (int i = 0; i < 4; i++) pair[i] = __nv_cvt_float2_to_fp8x2(make_float2(q[2 * i], q[2 * i + 1]), __NV_SATFINITE, __NV_E4M3);
  unsigned char* p = static_cast<unsigned char*>(base);
  if (MODE == VECTORS) {
    __stcs(reinterpret_cast<uint2*>(p) + threadIdx.x, make_uint2(pair[0] | (unsigned)pair[1] << 16, pair[2] | (unsigned)pair[3] << 16));
  } else if (MODE == PAIRS) {
#pragma unroll
    for (int i = 0; i < 4; i++) __stcs(reinterpret_cast<unsigned short*>(p + element<MODE>(2 * i)), pair[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++)
      if (exists<MODE>(i, left)) p[element<MODE>(i)] = (unsigned char)(pair[i / 2] >> (i % 2 * 8));
  }
}

// ---------------------------------------------------------------- device: the step

struct Rates {
  float lr, step_size, root_scale, scale;
  unsigned seed;
  bool skip;
};
__device__ __forceinline__ Rates read_rates(const AdamScalars& s) {
  Rates r{s.lr, s.step_size, s.root_scale, s.grad_scale, s.seed, false};
  if (s.rates) {
    const uint4 x = *reinterpret_cast<const uint4*>(s.rates);
    r.lr = __uint_as_float(x.x);
    r.step_size = r.lr / __uint_as_float(x.y);
    r.root_scale = 1.0f / sqrtf(__uint_as_float(x.z));
    r.seed = x.w;
  }
  if (s.factor) {
    const float f = *s.factor;
    r.skip = f != f;
    r.scale *= f;
  }
  return r;
}

// The arrays of one tensor (shard) from one tile on.
struct Place {
  void *m, *v;
  float *master, *m_scale, *v_scale;
  unsigned left, key;   // elements from the tile's start on; tile_key
};
__device__ __forceinline__ Place place_of(void* m, void* v, float* master, float* ms, float* vs, unsigned long long n, unsigned long long at, int w, int state,
                                          unsigned seed, unsigned tensor) {
  const size_t e = state == HOCCL_STATE_FLOAT32 ? 4 : 1;
  Place p;
  p.m = static_cast<char*>(m) + at * e;
  p.v = static_cast<char*>(v) + at * e;
  p.master = w == W_MASTER ? master + at : nullptr;
  p.m_scale = state == HOCCL_STATE_8BIT ? ms + at / kBlock : nullptr;
  p.v_scale = state == HOCCL_STATE_8BIT ? vs + at / kBlock : nullptr;
  p.left = (unsigned)min(n - at, (unsigned long long)kTile);
  p.key = state == HOCCL_STATE_8BIT ? tile_key(tensor_key(seed, tensor), at) : 0;
  return p;
}

// What a block's state and weight need besides its gradient.
template <int W, int STATE, Mode MODE>
struct Held {
  float p[8], m[8], v[8];
  // weights: W_MASTER from the master, else from param
  __device__ __forceinline__ void load(const void* param, const Place& a) {
    if (W == W_MASTER) load_floats<0, MODE>(a.master, a.left, p);
    else load_floats<W == W_FP32 ? 0 : 1, MODE>(param, a.left, p);
    if (STATE == HOCCL_STATE_FLOAT32) {
      load_floats<0, MODE>(a.m, a.left, m);
      load_floats<0, MODE>(a.v, a.left, v);
    } else {
      load_codes<MODE>(a.m, a.left, a.m_scale[threadIdx.x / 32], m);
      load_codes<MODE>(a.v, a.left, a.v_scale[threadIdx.x / 32], v);
    }
  }
  // g: the gradients as they were read.  Afterwards p holds the new weights, which the caller stores; the state is stored here.
  __device__ __forceinline__ void step(const float* g, const AdamScalars& s, const Rates& r, float keep, const Place& a) {
    // states: every operation rounded by itself, as the header has it, so that 8-bit codes can be told bit for bit
    float root[8];
    float low = 3.4e38f, high = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      const Two x = mul2(two(g[i], g[i + 1]), two(r.scale));
      Two vv = two(v[i], v[i + 1]);
      if (STATE == HOCCL_STATE_8BIT) vv = mul2(vv, vv);
      split(add2(mul2(two(m[i], m[i + 1]), two(s.beta1)), mul2(x, two(s.grad1)), s.one), m + i);
      split(add2(mul2(vv, two(s.beta2)), mul2(mul2(x, x), two(s.grad2)), s.one), v + i);
      low = fminf(low, fminf(v[i], v[i + 1]));
      high = max_nan(high, max_nan(v[i], v[i + 1]));
    }
    if (!__any_sync(0xffffffffu, !(low >= kRootLow && high <= kRootHigh))) {
#pragma unroll
      for (int i = 0; i < 8; i += 2) split(root_in_range(two(v[i], v[i + 1]), two(s.half), two(s.minus_half), two(s.minus_one)), root + i);
    } else {
#pragma unroll
      for (int i = 0; i < 8; i++) root[i] = __fsqrt_rn(v[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      float below[2], over[2];
      split(fma2(two(root[i], root[i + 1]), two(r.root_scale), two(s.eps)), below);
      asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(over[0]) : "f"(below[0]));   // eps is a normal number
      asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(over[1]) : "f"(below[1]));
      split(fma2(mul2(two(m[i], m[i + 1]), two(over[0], over[1])), two(-r.step_size), mul2(two(p[i], p[i + 1]), two(keep))), p + i);
    }
    if (W == W_MASTER) store_floats<0, MODE>(a.master, a.left, p);
    if (STATE == HOCCL_STATE_FLOAT32) {
      store_floats<0, MODE>(a.m, a.left, m);
      store_floats<0, MODE>(a.v, a.left, v);
    } else {
      Halves word[8];
#pragma unroll
      for (int i = 0; i < 8; i++) word[i] = halves(a.key + element<MODE>(i));
      store_codes<MODE, false>(a.m, a.m_scale, a.left, m, word);
      store_codes<MODE, true>(a.v, a.v_scale, a.left, root, word);
    }
  }
};

template <int GT, int W, int STATE, Mode MODE>
__device__ __forceinline__ void tensor_block(const void* grad, void* param, const Place& a, const AdamScalars& s, const Rates& r, float keep) {
  Held<W, STATE, MODE> h;
  float g[8];
  load_floats<GT, MODE>(grad, a.left, g);
  h.load(param, a);
  h.step(g, s, r, keep, a);
  store_floats<W == W_FP32 ? 0 : 1, MODE>(param, a.left, h.p);
}

template <int GT, int W, int STATE, class Table>
__global__ void __launch_bounds__(kOptThreads, 32 / kWarps) adamw_kernel(const __grid_constant__ Table t, const __grid_constant__ AdamScalars s) {
  wait_for_stream();
  const Rates r = read_rates(s);
  if (r.skip) return;
  const unsigned tile = blockIdx.x, here = (threadIdx.x & ~31u) * 8;
  int k = 0;
  for (int step = t.n <= 32 ? 16 : t.n <= 128 ? 64 : 256; step; step >>= 1)   // the tensor the tile lies in
    if (k + step < t.n && t.first[k + step] <= tile) k += step;
  const AdamRow& row = t.row[k];
  const unsigned long long at = (unsigned long long)(tile - t.first[k]) * kTile;
  const Place a = place_of(row.m, row.v, row.master, row.m_scale, row.v_scale, row.n, at, W, STATE, r.seed, row.flags >> 1);
  const void* grad = static_cast<const char*>(row.grad) + at * (GT == 0 ? 4 : 2);
  void* param = static_cast<char*>(row.param) + at * (W == W_FP32 ? 4 : 2);
  const float keep = fmaf(-r.lr, row.decay, 1.0f);
  if (here >= a.left) return;
  if (here + kBlock > a.left) tensor_block<GT, W, STATE, ENDS>(grad, param, a, s, r, keep);
  else if (row.flags & 1) tensor_block<GT, W, STATE, VECTORS>(grad, param, a, s, r, keep);
  else tensor_block<GT, W, STATE, WHOLE>(grad, param, a, s, r, keep);
}

// The gradients of a block are read from every rank at once and its new weights stored to every rank: the reads and writes of an all-reduce, with the state's in
// between.  13.1 M bf16 weights over 8 ranks: 117 us, 6.3 TB/s (with four of eight gradients in flight and 170 registers 278 us; the pair of collectives alone 211);
// one weight more, which puts chunks off 32 bytes, 129 us (two elements at a time in every other chunk, one in the rest; 139 with one in all; 146 with 80 registers
// instead of 64, 175 with 128 and all eight gradients in flight).  64 registers make ten of the twelve forms spill, 8 to 44 bytes: 2 us more for the aligned
// weights, 7 less for the others, taken one at a time.
template <int GT, int W, int STATE, Mode MODE>
__device__ __forceinline__ void sharded_block(const ShardedArgs& args, const AdamScalars& s, const Rates& r, int c, unsigned long long lo, const Place& a) {
  // the ring's order: c + 1, c + 2, ..., c; the gradients of kFlight ranks in flight at a time, as they lie in memory
  constexpr int kFlight = MODE < PAIRS ? 2 : GT == 0 ? 4 : MODE == PAIRS ? 4 : 8;
  float g[8];
  int from = c;
  for (int j0 = 0; j0 < args.R; j0 += kFlight) {
    Raw<GT, MODE> x[kFlight];
#pragma unroll
    for (int j = 0; j < kFlight; j++)
      if (j0 + j < args.R) {
        from = from + 1 < args.R ? from + 1 : 0;
        x[j].load(static_cast<const char*>(args.grad[from]) + lo * (GT == 0 ? 4 : 2), a.left);
      }
#pragma unroll
    for (int j = 0; j < kFlight; j++)
      if (j0 + j < args.R) {
        float y[8];
        x[j].widen(y);
#pragma unroll
        for (int i = 0; i < 8; i++) g[i] = j0 + j ? __fadd_rn(g[i], y[i]) : y[i];
      }
  }
  constexpr int kWeight = W == W_FP32 ? 4 : 2;
  Held<W, STATE, MODE> h;
  h.load(static_cast<const char*>(args.param[c]) + lo * kWeight, a);
  h.step(g, s, r, fmaf(-r.lr, args.decay, 1.0f), a);
  for (int to = 0; to < args.R; to++) store_floats<W == W_FP32 ? 0 : 1, MODE>(static_cast<char*>(args.param[to]) + lo * kWeight, a.left, h.p);
}

template <int GT, int W, int STATE>
__global__ void __launch_bounds__(kOptThreads, 32 / kWarps) sharded_adamw_kernel(const __grid_constant__ ShardedArgs args, const __grid_constant__ AdamScalars s) {
  wait_for_stream();
  const Rates r = read_rates(s);
  if (r.skip) return;
  const unsigned here = (threadIdx.x & ~31u) * 8;
  const int c = (int)(blockIdx.x / args.per_rank);
  const unsigned long long at = (unsigned long long)(blockIdx.x - c * args.per_rank) * kTile, lo = min(c * args.q, args.count), n = min(args.q, args.count - lo);
  if (at + here >= n) return;   // the short chunks at the end have fewer tiles
  const Place a = place_of(args.m[c], args.v[c], args.master[c], args.m_scale[c], args.v_scale[c], n, at, W, STATE, r.seed, (unsigned)c);
  if (here + kBlock > a.left) sharded_block<GT, W, STATE, ENDS>(args, s, r, c, lo + at, a);
  else if (args.aligned >> c & 1) sharded_block<GT, W, STATE, VECTORS>(args, s, r, c, lo + at, a);
  else if (args.paired >> c & 1) sharded_block<GT, W, STATE, PAIRS>(args, s, r, c, lo + at, a);
  else sharded_block<GT, W, STATE, WHOLE>(args, s, r, c, lo + at, a);
}

// ---------------------------------------------------------------- device: the norm

constexpr int kNormThreads = 256, kNormCtas = 8 * kAllSms, kNormTile = 4 * kNormThreads;   // vectors of 16 bytes in a tile
struct NormRow {
  const void* p;
  unsigned long long n;
};
struct NormEndArgs {
  const double* partial;
  int n;
  double max_norm;
  float* out;
};
template <int N>
struct NormTableT {
  int n, first_launch;
  double* partial;               // one for each CTA: launches of one call add to it one after the other
  NormEndArgs end;               // of a grid that is one cluster and ends by itself
  NormRow row[N];
  unsigned first[N + 1];         // prefix sums of tiles
};
constexpr int kNormRows = 1024;
// Few tiles are summed by one cluster in one launch, which ends by itself: a second launch costs more than the SMs that stay idle (one tensor of 4096: 3.1 us in two
// launches, 2.3 in one, the call's host time 4.5 and 2.9; 8 of them 3.4 and 2.7; 32 tiles are 4 for a CTA).
constexpr int kNormCluster = 8, kNormClusterTiles = 4 * kNormCluster;
using NormTableSmall = NormTableT<64>;
using NormTable = NormTableT<kNormRows>;
static_assert(sizeof(NormTable) <= 32764, "kernel parameters");

// 201 M bf16 gradients: 62 to 69 us from one GPU to another, 6.5 to 5.8 TB/s.  Squares in binary64: the square of any binary32 number is there, and a long sum keeps its bits.
template <int DT>
__device__ __forceinline__ double squares(uint4 r) {
  float x[8];
  if (DT == 1) {
    widen8(r, x);
  } else {
    x[0] = __uint_as_float(r.x);
    x[1] = __uint_as_float(r.y);
    x[2] = __uint_as_float(r.z);
    x[3] = __uint_as_float(r.w);
  }
  double s = 0;
#pragma unroll
  for (int i = 0; i < (DT == 1 ? 8 : 4); i++) s = fma((double)x[i], (double)x[i], s);
  return s;
}
template <int DT>
__device__ __forceinline__ double square_of(const void* p, unsigned long long i) {
  const float x = DT == 1 ? __uint_as_float((unsigned)static_cast<const unsigned short*>(p)[i] << 16) : static_cast<const float*>(p)[i];
  return (double)x * (double)x;
}

__device__ __forceinline__ double warp_sum(double s) {
#pragma unroll
  for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
  return s;
}
__device__ __forceinline__ double cta_sum(double s, double* shared) {   // in a fixed order; valid in the first warp
  const int lane = threadIdx.x & 31;
  s = warp_sum(s);
  if (lane == 0) shared[threadIdx.x / 32] = s;
  __syncthreads();
  return threadIdx.x < 32 ? warp_sum(lane < (int)blockDim.x / 32 ? shared[lane] : 0.0) : 0.0;
}

__device__ __forceinline__ void norm_out(double sum, const NormEndArgs& a) {
  const double norm = sqrt(sum);
  a.out[0] = (float)norm;
  a.out[1] = isfinite(norm) ? (float)fmin(1.0, a.max_norm / (norm + 1e-6)) : __uint_as_float(0x7fc00000u);
}

template <int DT, class Table, bool CLUSTER>
__global__ void __launch_bounds__(kNormThreads) norm_kernel(const __grid_constant__ Table t) {
  using T = Traits<DT>;
  __shared__ double shared[kNormThreads / 32];
  if constexpr (CLUSTER) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");   // this CTA has started
  wait_for_stream();
  double sum = 0;
  const unsigned tiles = t.first[t.n];
  int k = 0;
  for (unsigned tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    if (tile >= t.first[k + 1])
      for (int step = t.n <= 64 ? 32 : 512; step; step >>= 1)
        if (k + step < t.n && t.first[k + step] <= tile) k += step;
    const NormRow row = t.row[k];
    const unsigned head = min((unsigned long long)((16u - ((unsigned)(uintptr_t)row.p & 15u)) & 15u) / T::E, row.n);
    const unsigned long long nvec = (row.n - head) / T::VE, at = (unsigned long long)(tile - t.first[k]) * kNormTile;
    const uint4* p = reinterpret_cast<const uint4*>(static_cast<const char*>(row.p) + (size_t)head * T::E) + at;
    const unsigned here = at < nvec ? (unsigned)min(nvec - at, (unsigned long long)kNormTile) : 0;
    uint4 v[4];
#pragma unroll
    for (int u = 0; u < 4; u++) v[u] = threadIdx.x + u * kNormThreads < here ? __ldcs(p + threadIdx.x + u * kNormThreads) : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int u = 0; u < 4; u++) sum += squares<DT>(v[u]);
    const unsigned ends = (unsigned)(row.n - nvec * T::VE);   // elements before and behind the vectors
    if (at == 0 && threadIdx.x < ends) sum += square_of<DT>(row.p, threadIdx.x < head ? threadIdx.x : nvec * T::VE + threadIdx.x);
  }
  sum = cta_sum(sum, shared);
  if constexpr (CLUSTER) {
    __shared__ double parts[kNormCluster];
    cg::cluster_group cluster = cg::this_cluster();
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");   // the first CTA has started too, so its shared memory is there
    if (threadIdx.x == 0) cluster.map_shared_rank(parts, 0)[blockIdx.x] = sum;   // into the first CTA's shared memory
    cluster.sync();
    if (blockIdx.x == 0 && threadIdx.x == 0) {
      double all = 0;
      for (int c = 0; c < kNormCluster; c++) all += parts[c];
      norm_out(all, t.end);
    }
  } else if (threadIdx.x == 0) {
    t.partial[blockIdx.x] = t.first_launch ? sum : t.partial[blockIdx.x] + sum;
  }
}

constexpr int kNormEndThreads = 512;
__global__ void __launch_bounds__(kNormEndThreads) norm_end_kernel(const __grid_constant__ NormEndArgs a) {
  __shared__ double shared[kNormEndThreads / 32];
  constexpr int kEach = (kNormCtas + kNormEndThreads - 1) / kNormEndThreads;
  wait_for_stream();
  double x[kEach], s = 0;
#pragma unroll
  for (int i = 0; i < kEach; i++) x[i] = (int)threadIdx.x + i * kNormEndThreads < a.n ? __ldcg(a.partial + threadIdx.x + i * kNormEndThreads) : 0.0;
#pragma unroll
  for (int i = 0; i < kEach; i++) s += x[i];
  s = cta_sum(s, shared);
  if (threadIdx.x == 0) norm_out(s, a);
}

// Every number of kRootLow .. kRootHigh: counts[0] += roots that differ from __fsqrt_rn's, counts[1] += numbers.
__global__ void __launch_bounds__(256) root_selftest_kernel(unsigned long long* counts) {
  const unsigned lo = __float_as_uint(kRootLow), hi = __float_as_uint(kRootHigh);
  unsigned long long wrong = 0, seen = 0;
  for (unsigned b = lo + blockIdx.x * 256 + threadIdx.x; b <= hi; b += gridDim.x * 256) {
    float r[2];
    split(root_in_range(two(__uint_as_float(b), __uint_as_float(hi - (b - lo))), two(0.5f), two(-0.5f), two(-1.0f)), r);
    wrong += __float_as_uint(r[0]) != __float_as_uint(__fsqrt_rn(__uint_as_float(b)));
    wrong += __float_as_uint(r[1]) != __float_as_uint(__fsqrt_rn(__uint_as_float(hi - (b - lo))));
    seen++;
  }
  atomicAdd(counts, wrong);
  atomicAdd(counts + 1, seen);
}

// ---------------------------------------------------------------- host: dispatch

template <class Table>
const void* adamw_entry(int gt, int w, int state) {
#define ROW(G, W) {reinterpret_cast<const void*>(&adamw_kernel<G, W, 0, Table>), reinterpret_cast<const void*>(&adamw_kernel<G, W, 1, Table>)}
  static const void* const fns[2][3][2] = {{ROW(0, 0), ROW(0, 1), ROW(0, 2)}, {ROW(1, 0), ROW(1, 1), ROW(1, 2)}};
#undef ROW
  return fns[gt][w][state];
}
const void* sharded_entry(int gt, int w, int state) {
#define ROW(G, W) {reinterpret_cast<const void*>(&sharded_adamw_kernel<G, W, 0>), reinterpret_cast<const void*>(&sharded_adamw_kernel<G, W, 1>)}
  static const void* const fns[2][3][2] = {{ROW(0, 0), ROW(0, 1), ROW(0, 2)}, {ROW(1, 0), ROW(1, 1), ROW(1, 2)}};
#undef ROW
  return fns[gt][w][state];
}
const void* norm_entry(int dtype, bool small, bool one_cluster) {
#define ROW(D) {reinterpret_cast<const void*>(&norm_kernel<D, NormTable, false>), reinterpret_cast<const void*>(&norm_kernel<D, NormTableSmall, false>), \
                reinterpret_cast<const void*>(&norm_kernel<D, NormTableSmall, true>)}
  static const void* const fns[2][3] = {ROW(0), ROW(1)};
#undef ROW
  return fns[dtype][one_cluster ? 2 : small];
}

bool aligned_to(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

bool fill_scalars(const hoccl_adamw_config_t& c, AdamScalars* s) {
  for (double x : {c.lr, c.beta1, c.beta2, c.eps, c.grad_scale})
    if (!std::isfinite(x)) return false;
  if (c.beta1 < 0 || c.beta1 >= 1 || c.beta2 < 0 || c.beta2 >= 1 || !(c.eps > 0) || c.step < 1) return false;
  if (!aligned_to(c.factor, 4) || !aligned_to(c.rates, 16)) return false;
  // 1 - beta^t by way of the logarithm: no cancellation for beta near 1; beta = 0 gives 1
  const double bias1 = -std::expm1((double)c.step * std::log(c.beta1)), bias2 = -std::expm1((double)c.step * std::log(c.beta2));
  s->lr = (float)c.lr;
  s->step_size = (float)(c.lr / bias1);
  s->root_scale = (float)(1.0 / std::sqrt(bias2));
  const float eps = (float)c.eps;
  const auto pair = [](double x) {
    const float f = (float)x;
    unsigned w;
    std::memcpy(&w, &f, 4);
    return Pair{(unsigned long long)w << 32 | w};
  };
  s->beta1 = pair(c.beta1);
  s->grad1 = pair(1.0 - c.beta1);
  s->beta2 = pair(c.beta2);
  s->grad2 = pair(1.0 - c.beta2);
  s->eps = pair(c.eps);
  s->one = pair(1.0);
  s->half = pair(0.5);
  s->minus_half = pair(-0.5);
  s->minus_one = pair(-1.0);
  s->grad_scale = (float)c.grad_scale;
  s->seed = c.seed;
  s->factor = c.factor;
  s->rates = c.rates;
  for (float x : {s->lr, s->step_size, s->root_scale, s->grad_scale})
    if (!std::isfinite(x)) return false;
  return eps >= 0x1p-126f && eps <= 0x1p126f;   // the kernels divide by numbers from eps on with a reciprocal that takes and gives normal ones, else 0
}

struct Region {
  const char* at;
  size_t bytes;
  bool written;
};
// Whether a region that is written overlaps any other one.
bool regions_clash(std::vector<Region>* regions) {
  std::sort(regions->begin(), regions->end(), [](const Region& a, const Region& b) { return a.at < b.at; });
  const char *end = nullptr, *written_end = nullptr;   // of what came before
  for (const Region& r : *regions) {
    if (!r.bytes) continue;
    if (r.at < written_end || (r.written && r.at < end)) return true;
    end = std::max(end, r.at + r.bytes);
    if (r.written) written_end = std::max(written_end, r.at + r.bytes);
  }
  return false;
}

// What a set of arrays shares: bit 0 if all start on an access of eight elements, bit 1 of two.
unsigned phase_of(const void* p, size_t e) { return (aligned_to(p, 8 * e) ? 1u : 0u) | (aligned_to(p, 2 * e) ? 2u : 0u); }

// Checks one tensor's (shard's) state and adds its regions; *phase loses what its arrays do not have.
bool state_fits(const void* m, const void* v, const float* master, const float* ms, const float* vs, size_t n, int state, std::vector<Region>* regions, unsigned* phase) {
  const size_t e = state == HOCCL_STATE_FLOAT32 ? 4 : 1;
  if (!m || !v || !aligned_to(m, e) || !aligned_to(v, e) || !aligned_to(master, 4)) return false;
  *phase &= phase_of(m, e) & phase_of(v, e) & phase_of(master, 4);
  regions->push_back({(const char*)m, n * e, true});
  regions->push_back({(const char*)v, n * e, true});
  if (master) regions->push_back({(const char*)master, n * 4, true});
  if (state == HOCCL_STATE_8BIT) {
    if (!ms || !vs || !aligned_to(ms, 4) || !aligned_to(vs, 4)) return false;
    const size_t bytes = (n + kBlock - 1) / kBlock * 4;
    regions->push_back({(const char*)ms, bytes, true});
    regions->push_back({(const char*)vs, bytes, true});
  }
  return true;
}

}  // namespace

cudaError_t launch_root_selftest(unsigned long long* counts, cudaStream_t stream) {
  root_selftest_kernel<<<8 * kAllSms, 256, 0, stream>>>(counts);
  return cudaGetLastError();
}

void add_optim_kernels(std::vector<const void*>* fns) {
  for (int gt = 0; gt < 2; gt++) {
    for (int w = 0; w < 3; w++)
      for (int state = 0; state < 2; state++)
        for (const void* f : {adamw_entry<AdamTableSmall>(gt, w, state), adamw_entry<AdamTableMiddle>(gt, w, state), adamw_entry<AdamTable>(gt, w, state), sharded_entry(gt, w, state)}) fns->push_back(f);
    for (int form = 0; form < 3; form++) fns->push_back(norm_entry(gt, form > 0, form == 2));
  }
  fns->push_back(reinterpret_cast<const void*>(&norm_end_kernel));
}

}  // namespace hoccl

// Tables ready to launch.
struct hoccl_adamw_plan {
  int grad_dtype, weights, state;
  std::vector<AdamTableSmall> small;
  std::vector<AdamTableMiddle> middle;
  std::vector<AdamTable> large;
};

namespace {

constexpr size_t kMaxTensorElements = 1ull << 39;   // 2^29 tiles; with those of 64 ranks' chunks a grid holds them

template <class Table>
void append_table(const std::vector<AdamRow>& rows, size_t from, size_t n, std::vector<Table>* out) {
  out->emplace_back();
  Table& t = out->back();
  t.n = (int)n;
  t.pad = 0;
  t.first[0] = 0;
  for (size_t k = 0; k < n; k++) {
    t.row[k] = rows[from + k];
    t.first[k + 1] = t.first[k] + (unsigned)((t.row[k].n + kTile - 1) / kTile);
  }
}

hoccl_result_t make_plan(hoccl_adamw_plan_t* out, const hoccl_adamw_tensor_t* tensors, int n, int param_dtype, int grad_dtype, int state) {
  const size_t pe = dtype_size(param_dtype), ge = dtype_size(grad_dtype);
  std::vector<AdamRow> rows;
  std::vector<Region> regions;
  bool with = false, without = false;
  for (int k = 0; k < n; k++) {
    const hoccl_adamw_tensor_t& t = tensors[k];
    if (t.count == 0) continue;
    if (t.count > kMaxTensorElements || !t.param || !t.grad || !aligned_to(t.param, pe) || !aligned_to(t.grad, ge) || !std::isfinite(t.weight_decay)) return HOCCL_ERR_INVALID_ARG;
    (t.master ? with : without) = true;
    unsigned phase = phase_of(t.param, pe) & phase_of(t.grad, ge);
    if (!state_fits(t.exp_avg, t.exp_avg_sq, t.master, t.exp_avg_scale, t.exp_avg_sq_scale, t.count, state, &regions, &phase)) return HOCCL_ERR_INVALID_ARG;
    regions.push_back({(const char*)t.param, t.count * pe, true});
    regions.push_back({(const char*)t.grad, t.count * ge, false});
    rows.push_back(AdamRow{t.param, t.exp_avg, t.exp_avg_sq, t.grad, t.master, t.exp_avg_scale, t.exp_avg_sq_scale, (unsigned long long)t.count, t.weight_decay,
                           (unsigned)k << 1 | (phase & 1)});
  }
  if (with && without) return HOCCL_ERR_INVALID_ARG;
  if (with && param_dtype != HOCCL_BFLOAT16) return HOCCL_ERR_UNSUPPORTED;
  if (regions_clash(&regions)) return HOCCL_ERR_INVALID_ARG;
  hoccl_adamw_plan* p = new hoccl_adamw_plan();
  *out = p;   // the caller frees it if filling it runs out of memory
  p->grad_dtype = grad_dtype;
  p->state = state;
  p->weights = param_dtype == HOCCL_FLOAT32 ? W_FP32 : with ? W_MASTER : W_BF16;
  constexpr size_t kLarge = sizeof(AdamTable::row) / sizeof(AdamRow), kMiddle = sizeof(AdamTableMiddle::row) / sizeof(AdamRow),
                   kSmall = sizeof(AdamTableSmall::row) / sizeof(AdamRow);
  for (size_t from = 0; from < rows.size();) {
    unsigned long long tiles = 0;
    size_t here = 0;   // as many as a table and a grid hold
    while (here < kLarge && from + here < rows.size()) {
      const unsigned long long more = (rows[from + here].n + kTile - 1) / kTile;
      if (here && tiles + more >= 1ull << 31) break;
      tiles += more;
      here++;
    }
    if (here <= kSmall) append_table(rows, from, here, &p->small);
    else if (here <= kMiddle) append_table(rows, from, here, &p->middle);
    else append_table(rows, from, here, &p->large);
    from += here;
  }
  return HOCCL_OK;
}

template <class Table>
cudaError_t launch_tables(const std::vector<Table>& tables, const hoccl_adamw_plan& p, AdamScalars* s, cudaStream_t stream) {
  for (const Table& t : tables) {
    void* params[2] = {const_cast<Table*>(&t), s};
    const cudaError_t e = launch_in_order_params(adamw_entry<Table>(p.grad_dtype, p.weights, p.state), (int)t.first[t.n], kOptThreads, params, stream);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

bool known_state(int state) { return state == HOCCL_STATE_FLOAT32 || state == HOCCL_STATE_8BIT; }

}  // namespace

extern "C" {

hoccl_result_t hoccl_adamw_create(hoccl_adamw_plan_t* plan, const hoccl_adamw_tensor_t* tensors, int n, hoccl_dtype_t param_dtype, hoccl_dtype_t grad_dtype,
                                  hoccl_state_t state) {
  if (!plan) return HOCCL_ERR_INVALID_ARG;
  *plan = nullptr;
  if (n < 0 || (n && !tensors)) return HOCCL_ERR_INVALID_ARG;
  if (!dtype_size((int)param_dtype) || !dtype_size((int)grad_dtype) || !known_state((int)state)) return HOCCL_ERR_UNSUPPORTED;
  hoccl_result_t rc;
  try {
    rc = make_plan(plan, tensors, n, (int)param_dtype, (int)grad_dtype, (int)state);
  } catch (const std::bad_alloc&) {
    rc = HOCCL_ERR_INTERNAL;
  }
  if (rc != HOCCL_OK) {
    delete *plan;
    *plan = nullptr;
  }
  return rc;
}

void hoccl_adamw_destroy(hoccl_adamw_plan_t plan) { delete plan; }

hoccl_result_t hoccl_adamw_step(hoccl_adamw_plan_t plan, const hoccl_adamw_config_t* config, hoccl_comm_t c, hoccl_stream_t stream) {
  const double t0 = now_us();
  AdamScalars s;
  if (!plan || !config || !c || !fill_scalars(*config, &s)) return HOCCL_ERR_INVALID_ARG;
  c->stats = hoccl_stats_t{};
  DeviceScope scope(c->device);
  CU_TRY(c, scope.err);
  CU_TRY(c, launch_tables(plan->small, *plan, &s, (cudaStream_t)stream));
  CU_TRY(c, launch_tables(plan->middle, *plan, &s, (cudaStream_t)stream));
  CU_TRY(c, launch_tables(plan->large, *plan, &s, (cudaStream_t)stream));
  c->stats.host_launch_us = now_us() - t0;
  return HOCCL_OK;
}

hoccl_result_t hoccl_sharded_adamw(const void* const* grads, void* const* params, void* const* exp_avg, void* const* exp_avg_sq, float* const* master,
                                   float* const* exp_avg_scale, float* const* exp_avg_sq_scale, size_t count, hoccl_dtype_t param_dtype,
                                   hoccl_dtype_t grad_dtype, hoccl_state_t state, float weight_decay, const hoccl_adamw_config_t* config, hoccl_comm_t c,
                                   hoccl_stream_t stream) {
  const double t0 = now_us();
  AdamScalars s;
  const size_t pe = dtype_size((int)param_dtype), ge = dtype_size((int)grad_dtype);
  const bool eight = state == HOCCL_STATE_8BIT;
  if (!c || !config || !grads || !params || !exp_avg || !exp_avg_sq || (eight && (!exp_avg_scale || !exp_avg_sq_scale))) return HOCCL_ERR_INVALID_ARG;
  if (!pe || !ge || !known_state((int)state) || (master && param_dtype != HOCCL_BFLOAT16)) return HOCCL_ERR_UNSUPPORTED;
  if (!fill_scalars(*config, &s) || !std::isfinite(weight_decay) || count > kMaxTensorElements) return HOCCL_ERR_INVALID_ARG;
  c->stats = hoccl_stats_t{};
  if (count == 0) return HOCCL_OK;
  ShardedArgs a = {};
  a.R = c->R;
  a.decay = weight_decay;
  a.count = count;
  a.q = (count + (size_t)c->R - 1) / (size_t)c->R;
  a.per_rank = (unsigned)((a.q + kTile - 1) / kTile);
  try {
    std::vector<Region> regions;
    for (int r = 0; r < c->R; r++) {
      if (!grads[r] || !params[r] || !aligned_to(grads[r], ge) || !aligned_to(params[r], pe)) return HOCCL_ERR_INVALID_ARG;
      a.grad[r] = grads[r];
      a.param[r] = params[r];
      regions.push_back({(const char*)grads[r], count * ge, false});
      regions.push_back({(const char*)params[r], count * pe, true});
      const size_t lo = std::min((size_t)(r * a.q), count), n = std::min((size_t)a.q, count - lo);
      if (!n) continue;
      a.m[r] = exp_avg[r];
      a.v[r] = exp_avg_sq[r];
      a.master[r] = master ? master[r] : nullptr;
      a.m_scale[r] = eight ? exp_avg_scale[r] : nullptr;
      a.v_scale[r] = eight ? exp_avg_sq_scale[r] : nullptr;
      unsigned phase = 3;
      if ((master && !master[r]) || !state_fits(a.m[r], a.v[r], a.master[r], a.m_scale[r], a.v_scale[r], n, (int)state, &regions, &phase)) return HOCCL_ERR_INVALID_ARG;
      for (int k = 0; k < c->R; k++) phase &= phase_of((const char*)grads[k] + lo * ge, ge) & phase_of((const char*)params[k] + lo * pe, pe);
      if (phase & 1) a.aligned |= 1ull << r;
      if (phase & 2) a.paired |= 1ull << r;
    }
    if (regions_clash(&regions)) return HOCCL_ERR_INVALID_ARG;
  } catch (const std::bad_alloc&) {
    return HOCCL_ERR_INTERNAL;
  }
  DeviceScope scope(c->device);
  CU_TRY(c, scope.err);
  void* launch[2] = {&a, &s};
  const int weights = param_dtype == HOCCL_FLOAT32 ? W_FP32 : master ? W_MASTER : W_BF16;
  CU_TRY(c, launch_in_order_params(sharded_entry((int)grad_dtype, weights, (int)state), (int)(a.per_rank * (unsigned)c->R), kOptThreads, launch, (cudaStream_t)stream));
  c->stats.host_launch_us = now_us() - t0;
  return HOCCL_OK;
}

size_t hoccl_grad_norm_scratch_bytes(void) { return kNormCtas * sizeof(double); }

}  // extern "C"

namespace {

unsigned long long norm_tiles(size_t count, size_t e) { return std::max<unsigned long long>((count * e / 16 + kNormTile - 1) / kNormTile, 1); }

// Launches one table of vectors after the other; all launches of a call have the same grid, so that CTA b adds to partial b in order.
template <class Table>
cudaError_t norm_launches(const void* const* grads, const size_t* counts, int n, size_t cap, int dtype, int grid, const NormEndArgs& end, bool one_cluster, cudaStream_t stream) {
  Table t;
  const size_t e = dtype_size(dtype);
  t.partial = const_cast<double*>(end.partial);
  t.end = end;
  t.first_launch = 1;
  int k = 0;
  do {
    t.n = 0;
    t.first[0] = 0;
    for (; k < n && t.n < (int)cap; k++) {
      if (!counts[k]) continue;
      t.row[t.n] = NormRow{grads[k], (unsigned long long)counts[k]};
      t.first[t.n + 1] = t.first[t.n] + (unsigned)norm_tiles(counts[k], e);
      t.n++;
    }
    void* params[1] = {&t};
    const cudaError_t err = launch_in_order_params(norm_entry(dtype, sizeof(Table) == sizeof(NormTableSmall), one_cluster), grid, kNormThreads, params, stream, 0, one_cluster ? grid : 1);
    if (err != cudaSuccess) return err;
    t.first_launch = 0;
  } while (k < n);
  return cudaSuccess;
}

}  // namespace

extern "C" hoccl_result_t hoccl_grad_norm(const void* const* grads, const size_t* counts, int n, hoccl_dtype_t dtype, double max_norm, float* out, hoccl_comm_t c,
                                          hoccl_stream_t stream) {
  const double t0 = now_us();
  const size_t e = dtype_size((int)dtype);
  if (!c || !out || n < 0 || (n && (!grads || !counts)) || !aligned_to(out, 4) || !(max_norm > 0)) return HOCCL_ERR_INVALID_ARG;
  if (!e) return HOCCL_ERR_UNSUPPORTED;
  unsigned long long tiles = 0;
  int vectors = 0;
  const size_t need = hoccl_grad_norm_scratch_bytes();
  const auto in_scratch = [&](const void* p, size_t bytes) { return c->scratch && ranges_overlap((const char*)c->scratch, need, (const char*)p, bytes); };
  if (in_scratch(out, 8)) return HOCCL_ERR_INVALID_ARG;
  for (int k = 0; k < n; k++) {
    if (!counts[k]) continue;
    if (!grads[k] || !aligned_to(grads[k], e) || counts[k] > kMaxTensorElements || in_scratch(grads[k], counts[k] * e)) return HOCCL_ERR_INVALID_ARG;
    tiles += norm_tiles(counts[k], e);
    vectors++;
  }
  if (tiles >= (1ull << 32) - kNormCtas) return HOCCL_ERR_INVALID_ARG;   // (a CTA's tile number passes the last one by a grid)
  if (!c->scratch || c->scratch_bytes < need) return HOCCL_ERR_SCRATCH;
  c->stats = hoccl_stats_t{};
  DeviceScope scope(c->device);
  CU_TRY(c, scope.err);
  const bool one_cluster = tiles <= kNormClusterTiles;
  const int grid = one_cluster ? kNormCluster : (int)std::min<unsigned long long>(tiles, kNormCtas);
  NormEndArgs end{static_cast<double*>(c->scratch), grid, max_norm, out};
  if (vectors <= 64) CU_TRY(c, norm_launches<NormTableSmall>(grads, counts, n, 64, (int)dtype, grid, end, one_cluster, (cudaStream_t)stream));
  else CU_TRY(c, norm_launches<NormTable>(grads, counts, n, kNormRows, (int)dtype, grid, end, false, (cudaStream_t)stream));
  if (!one_cluster) CU_TRY(c, launch_in_order(reinterpret_cast<const void*>(&norm_end_kernel), 1, kNormEndThreads, &end, (cudaStream_t)stream));
  c->stats.host_launch_us = now_us() - t0;
  return HOCCL_OK;
}
