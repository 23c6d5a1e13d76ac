// adamw.hpp -- one AdamW step over many tensors (bart_ops.h has the formulas).
// Bound by memory: 1e8 f32 elements with 32-bit states 531 us (28 bytes an
// element, 5.3 TB/s); 3e8 bf16 elements with 8-bit states 525 to 580 us (10.06
// bytes, 5.2 to 5.7 TB/s, 56 instructions an element beside it).  A small model
// takes 5.2 us here: a workgroup reads its chunk, then the tensor, then the data.
#pragma once
#include <float.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "bart_ops.h"
#include "lanes.hpp"
#include "scalar.hpp"

namespace bart {

constexpr int kStateBlock = 256;      // elements that share a scale
constexpr int kChunk = 4096;          // elements of one workgroup
constexpr float kE4m3Max = 448.f;
constexpr float kLeast = 0x1p-100f;   // blocks of nothing larger are held as zeros

struct AdamwChunk {
  int32_t tensor, chunk;
};

// What changes from step to step.
struct AdamwStep {
  float b1, c1, b2, c2;   // betas and 1 - betas
  float eps, grad_scale;
  float root;             // 1 / sqrt(1 - beta2^t)
  double lr, first;       // lr; 1 / (1 - beta1^t)
  uint32_t dither;        // the step's term of the threshold sequence
};

// Two e4m3 codes, the low or the high half of a word, widened; the nearest codes
// of two values, written there (NaN to the NaN code).
template <bool HIGH>
__device__ __forceinline__ void e4m3_wide(uint32_t word, float *out) {
  typedef float two __attribute__((ext_vector_type(2)));
  const two v = __builtin_amdgcn_cvt_pk_f32_fp8((int)word, HIGH);
  out[0] = v.x;
  out[1] = v.y;
}
// The values are at most 448 (1 + 2^-22) in size: that is nearest to 448.
template <bool HIGH>
__device__ __forceinline__ uint32_t e4m3_nearest(uint32_t word, float a, float b) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, (int)word, HIGH);
}

// The e4m3 code of q >= 0 rounded up iff its distance to the value below, as
// a share of the spacing, plus threshold / 2^20 reaches 1; at least 1 where q
// is positive.  q x 2^-120 has e4m3's exponents, gradual underflow included, in
// f32's lowest ones: its upper 12 bits are the code.  A NaN ends above every
// code and becomes the NaN code.
__device__ __forceinline__ uint32_t e4m3_dithered(float q, uint32_t threshold) {
  q = __builtin_elementwise_minimum(q, kE4m3Max);  // keeps NaN
  const uint32_t code = (__float_as_uint(q * 0x1p-120f) + threshold) >> 20;
  const uint32_t least = min(__float_as_uint(q), 1u);
  return min(max(code, least), 0x7fu);
}

// The square root rounded correctly, for v = 0 and v >= 2^-96: the hardware's is
// within an ulp, and sqrt v lies below the middle of two neighbours r' < r iff
// v <= r' r (Tuckerman's test), whose sign the multiply-add gives exactly.
constexpr float kRootFrom = 0x1p-96f;
__device__ __forceinline__ float root_of(float v) {
  const float r = __builtin_amdgcn_sqrtf(v);
  const float down = __uint_as_float(__float_as_uint(r) - 1);
  const float up = __uint_as_float(__float_as_uint(r) + 1);
  const bool lower = __builtin_fmaf(-down, r, v) <= 0.f;  // 0: down is NaN, r stays
  const bool higher = __builtin_fmaf(-up, r, v) > 0.f;
  return higher ? up : lower ? down : r;
}

// 20-bit thresholds: the two-dimensional equidistributed sequence
// frac(i a + t b) with a, b the powers of the real root of x^3 = x + 1.
constexpr uint32_t kThresholdStep = 0xC13FA9A9u;

// Device memory whose address was read from memory: told so, the compiler
// loads and stores it as such and not as what might be LDS.
template <class T>
using dev = __attribute__((address_space(1))) T *;
template <class T>
__device__ __forceinline__ dev<T> on_device(const void *p) {
  return (dev<T>)(uintptr_t)p;
}

// G neighbours of one type, at any address of such elements.
template <class T, int G>
struct Some {
  typedef T vec __attribute__((ext_vector_type(G), aligned(sizeof(T))));
};

// Elements i ... i + G - 1 of an array; without FULL, `here` of them (the others
// are 0).
template <int DT, int G, bool FULL>
__device__ __forceinline__ void read_some(float *to, const void *from, int64_t i, int here) {
  using S = Scalar<DT>;
  using U = typename std::conditional<DT == BART_F32, uint32_t, uint16_t>::type;
  const auto p = on_device<const U>(from) + i;
  typename Some<U, G>::vec v = 0;
  if (FULL || here >= G) {
    v = *(dev<const typename Some<U, G>::vec>)p;
  } else {
#pragma unroll
    for (int e = 0; e < G; ++e)
      if (e < here) v[e] = p[e];
  }
#pragma unroll
  for (int e = 0; e < G; ++e) {
    const U u = v[e];
    to[e] = S::wide(__builtin_bit_cast(typename S::T, u));
  }
}
template <int DT, int G, bool FULL>
__device__ __forceinline__ void write_some(void *to, int64_t i, const float *from, int here) {
  using S = Scalar<DT>;
  using U = typename std::conditional<DT == BART_F32, uint32_t, uint16_t>::type;
  const auto p = on_device<U>(to) + i;
  typename Some<U, G>::vec v;
#pragma unroll
  for (int e = 0; e < G; ++e) v[e] = __builtin_bit_cast(U, S::narrow(from[e]));
  if (FULL || here >= G) {
    *(dev<typename Some<U, G>::vec>)p = v;
  } else {
#pragma unroll
    for (int e = 0; e < G; ++e)
      if (e < here) p[e] = v[e];
  }
}
// 8 codes of one byte.
template <bool FULL>
__device__ __forceinline__ void read_codes(uint32_t (&w)[2], const void *from, int64_t i,
                                           int here) {
  const auto p = on_device<const uint8_t>(from) + i;
  typedef uint32_t two __attribute__((ext_vector_type(2), aligned(1)));
  if (FULL || here >= 8) {
    const two v = *(dev<const two>)p;
    w[0] = v.x;
    w[1] = v.y;
  } else {
    w[0] = w[1] = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < here) w[e >> 2] |= (uint32_t)p[e] << (e & 3) * 8;
  }
}
template <bool FULL>
__device__ __forceinline__ void write_codes(void *to, int64_t i, const uint32_t (&w)[2],
                                            int here) {
  const auto p = on_device<uint8_t>(to) + i;
  typedef uint32_t two __attribute__((ext_vector_type(2), aligned(1)));
  if (FULL || here >= 8) {
    *(dev<two>)p = two{w[0], w[1]};
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < here) p[e] = (uint8_t)(w[e >> 2] >> (e & 3) * 8);
  }
}

// A workgroup of 256 lanes takes kChunk elements, a lane G neighbouring ones
// at a time: 16 bytes of the widest array, or with 8-bit states 8 elements, so
// that the 32 lanes of half a wave hold the block that shares a scale.  All
// loads of a lane's kChunk / 256 elements are under way before the first is
// used.  FULL: the chunk does not reach past the tensor's end.
template <int PT, int GT, int BITS, bool FULL>
__device__ __forceinline__ void adamw_chunk(const bart_adamw_tensor &t, int64_t base,
                                            const AdamwStep &K) {
  constexpr int G = BITS == 8 ? 8 : 4, N = kChunk / 256 / G;
  float p[N][G], g[N][G], m[N][G], v[N][G], sm[N], sr[N];
  uint32_t mc[N][2], rc[N][2];
  int here[N];
  const bool master = PT != BART_F32 && t.master;
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int64_t i = base + (n * 256 + (int)threadIdx.x) * G;
    here[n] = FULL ? G : (int)max(min(t.n - i, (int64_t)G), (int64_t)0);
    read_some<GT, G, FULL>(g[n], t.grad, i, here[n]);
    if (master)
      read_some<BART_F32, G, FULL>(p[n], t.master, i, here[n]);
    else
      read_some<PT, G, FULL>(p[n], t.param, i, here[n]);
    if constexpr (BITS == 32) {
      read_some<BART_F32, G, FULL>(m[n], t.m, i, here[n]);
      read_some<BART_F32, G, FULL>(v[n], t.v, i, here[n]);
    } else {
      read_codes<FULL>(mc[n], t.m, i, here[n]);
      read_codes<FULL>(rc[n], t.v, i, here[n]);
      sm[n] = FULL || here[n] ? on_device<const float>(t.m_scale)[i / kStateBlock] : 0.f;
      sr[n] = FULL || here[n] ? on_device<const float>(t.v_scale)[i / kStateBlock] : 0.f;
    }
  }
  const double lr = K.lr * (double)t.lr_scale;
  const float keep = (float)(1.0 - lr * (double)t.weight_decay);
  const float rate = (float)(lr * K.first);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int64_t i = base + (n * 256 + (int)threadIdx.x) * G;
    float r[G];
    if constexpr (BITS == 8) {
#pragma unroll
      for (int e = 0; e < 8; e += 4) {
        e4m3_wide<false>(mc[n][e / 4], m[n] + e);
        e4m3_wide<true>(mc[n][e / 4], m[n] + e + 2);
        e4m3_wide<false>(rc[n][e / 4], r + e);
        e4m3_wide<true>(rc[n][e / 4], r + e + 2);
      }
#pragma unroll
      for (int e = 0; e < G; ++e) {
        m[n][e] *= sm[n];
        r[e] *= sr[n];
        v[n][e] = r[e] * r[e];
      }
    }
    uint32_t least = ~0u;  // of the positive v, less 1
#pragma unroll
    for (int e = 0; e < G; ++e) {
      const float ge = g[n][e] * K.grad_scale;
      m[n][e] = m[n][e] * K.b1 + ge * K.c1;
      v[n][e] = v[n][e] * K.b2 + ge * ge * K.c2;
      least = min(least, __float_as_uint(v[n][e]) - 1);
    }
    // the root that is held in 8 bits is rounded correctly, so that its code is
    // that of the definition; where only the update uses it, 1 ulp serves, but
    // the hardware's root takes what is below the normal range as 0
    constexpr float kFrom = BITS == 8 ? kRootFrom : FLT_MIN;
    if (__any(least < __float_as_uint(kFrom) - 1)) {
#pragma unroll
      for (int e = 0; e < G; ++e) r[e] = sqrtf(v[n][e]);
    } else {
#pragma unroll
      for (int e = 0; e < G; ++e)
        r[e] = BITS == 8 ? root_of(v[n][e]) : __builtin_amdgcn_sqrtf(v[n][e]);
    }
#pragma unroll
    for (int e = 0; e < G; ++e) {
      const float step = m[n][e] * __builtin_amdgcn_rcpf(__builtin_fmaf(r[e], K.root, K.eps));
      p[n][e] = __builtin_fmaf(p[n][e], keep, -(step * rate));
    }
    if (master) write_some<BART_F32, G, FULL>(t.master, i, p[n], here[n]);
    write_some<PT, G, FULL>(t.param, i, p[n], here[n]);
    if constexpr (BITS == 32) {
      write_some<BART_F32, G, FULL>(t.m, i, m[n], here[n]);
      write_some<BART_F32, G, FULL>(t.v, i, v[n], here[n]);
    } else {
      // every lane takes part; past the tensor's end all is 0
      float tm = 0.f, tr = 0.f;
#pragma unroll
      for (int e = 0; e < G; ++e) {
        tm = fmaxf(tm, fabsf(m[n][e]));
        tr = fmaxf(tr, r[e]);
      }
      tm = lanes_max<32>(tm);
      tr = lanes_max<32>(tr);
      // below kLeast 448 / top would overflow
      if (tm < kLeast) tm = 0.f;
      if (tr < kLeast) tr = 0.f;
      const float um = tm > 0.f ? kE4m3Max / tm : 0.f, ur = tr > 0.f ? kE4m3Max / tr : 0.f;
      const uint32_t first = (uint32_t)i * kThresholdStep + K.dither;
#pragma unroll
      for (int e = 0; e < 8; e += 4) {
        uint32_t w = e4m3_nearest<false>(0, m[n][e] * um, m[n][e + 1] * um);
        mc[n][e / 4] = e4m3_nearest<true>(w, m[n][e + 2] * um, m[n][e + 3] * um);
        w = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q)
          w |= e4m3_dithered(r[e + q] * ur, (first + (e + q) * kThresholdStep) >> 12) << q * 8;
        rc[n][e / 4] = w;
      }
      write_codes<FULL>(t.m, i, mc[n], here[n]);
      write_codes<FULL>(t.v, i, rc[n], here[n]);
      if (threadIdx.x % 32 == 0 && (FULL || here[n])) {
        on_device<float>(t.m_scale)[i / kStateBlock] = tm * (1.f / kE4m3Max);
        on_device<float>(t.v_scale)[i / kStateBlock] = tr * (1.f / kE4m3Max);
      }
    }
  }
}

template <int PT, int GT, int BITS>
__global__ __launch_bounds__(256) void k_adamw(const bart_adamw_tensor *tensors,
                                               const AdamwChunk *chunks, AdamwStep K) {
  const AdamwChunk at = chunks[blockIdx.x];
  const bart_adamw_tensor t = tensors[at.tensor];
  const int64_t base = (int64_t)at.chunk * kChunk;
  if (base + kChunk <= t.n)
    adamw_chunk<PT, GT, BITS, true>(t, base, K);
  else
    adamw_chunk<PT, GT, BITS, false>(t, base, K);
}

}  // namespace bart
