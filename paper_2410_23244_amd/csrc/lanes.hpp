// lanes.hpp -- reductions over neighbouring lanes of a wave, by lane moves of
// the vector unit (no LDS round trips); every lane of a group gets the result.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace bart {

// 2^x by the transcendental unit (1 ulp; results below the normal range are 0)
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// f(v of one half of a group of D lanes, v of the other), D = 2 ... 64: given
// groups of D / 2 lanes that already agree among themselves, groups of D
// lanes agree afterwards, and every lane combines in the same order.
template <int D, class F>
__device__ __forceinline__ uint32_t lane_step(uint32_t v, F f) {
  if constexpr (D == 2)  // the other lane of a pair
    return f(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xf, 0xf, true));
  if constexpr (D == 4)  // the other pair of four
    return f(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xf, 0xf, true));
  if constexpr (D == 8)  // eight lanes mirrored
    return f(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xf, 0xf, true));
  if constexpr (D == 16)  // sixteen lanes mirrored
    return f(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x140, 0xf, 0xf, true));
  if constexpr (D == 32) {
    const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return f(p[0], p[1]);
  }
  const auto p = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return f(p[0], p[1]);
}

template <int T, class F>
__device__ __forceinline__ uint32_t lane_reduce(uint32_t v, F f) {
  if constexpr (T >= 2) v = lane_step<2>(v, f);
  if constexpr (T >= 4) v = lane_step<4>(v, f);
  if constexpr (T >= 8) v = lane_step<8>(v, f);
  if constexpr (T >= 16) v = lane_step<16>(v, f);
  if constexpr (T >= 32) v = lane_step<32>(v, f);
  if constexpr (T >= 64) v = lane_step<64>(v, f);
  return v;
}

template <int T>
__device__ __forceinline__ float lanes_max(float v) {
  return __uint_as_float(lane_reduce<T>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
    return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  }));
}

// The sum of two values does not depend on their order, so all lanes of a
// group hold the same bits.
template <int T>
__device__ __forceinline__ float lanes_sum(float v) {
  return __uint_as_float(lane_reduce<T>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
    return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
  }));
}

template <int T>
__device__ __forceinline__ uint32_t lanes_max_u32(uint32_t v) {
  return lane_reduce<T>(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}

// The largest 64-bit word: the largest high word, then the largest low word
// among the lanes that hold it.
template <int T>
__device__ __forceinline__ uint64_t lanes_max_u64(uint64_t v) {
  const uint32_t hi = lanes_max_u32<T>((uint32_t)(v >> 32));
  const uint32_t lo = lanes_max_u32<T>((uint32_t)(v >> 32) == hi ? (uint32_t)v : 0u);
  return (uint64_t)hi << 32 | lo;
}

// How many of the lanes in `who` come before this one.
__device__ __forceinline__ uint32_t lanes_before(uint64_t who) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32),
                                   __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
}

// A value that is the same in all lanes of a wave, when T >= 64: known to be
// so, it lives in scalar registers and its branches are scalar ones.
template <int T>
__device__ __forceinline__ int uniform(int v) {
  return T >= 64 ? __builtin_amdgcn_readfirstlane(v) : v;
}

// The same of a word that all lanes of a whole wave agree on.
__device__ __forceinline__ uint64_t uniform64(uint64_t v) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v);
  return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(v >> 32)) << 32 | lo;
}

// A scalar that the compiler knows nothing of: addresses derived from it are
// computed where they are used instead of being kept, one register pair each,
// from one turn of a loop to the next.
__device__ __forceinline__ int opaque(int v) {
  v = __builtin_amdgcn_readfirstlane(v);
  asm volatile("" : "+s"(v));
  return v;
}

// Orders LDS accesses among the T lanes of a group: a workgroup's barrier, or
// within one wave, whose lanes run together, only the order of its accesses.
template <int T>
__device__ __forceinline__ void group_sync() {
  if constexpr (T > 64) {
    __syncthreads();
  } else {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

}  // namespace bart
