// rows.hpp -- kernels over rows of class scores: log probability of the given
// class, entropy, best alternatives, and the gradient of the first two.  The
// definitions, and the rows that need a rule, are in bart_ops.h.
#pragma once
#include <float.h>
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "bart_ops.h"
#include "keysearch.hpp"
#include "lanes.hpp"
#include "scalar.hpp"

namespace bart {

struct RowsArgs {
  bart_rows r;
  bart_rows_out o;
  bart_rows_grad g;
  float inv_t;  // 1 / T
  int64_t first;  // row of the launch's first workgroup
};

constexpr float kNegInf = -INFINITY;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// ------------------------------------------------------------------ chunks
//
// A row is read as chunks of 16 bytes.  Groups of 8 and more lanes count them
// from the 16-byte boundary at or before the row's first class (rows of an odd
// stride begin anywhere, and loads that straddle a boundary cost a training
// step over 50001 bf16 classes a sixth of its time); smaller groups, whose
// lanes read rows of their own, from the row's beginning.  The first and the
// last chunk of a row, where the classes do not fill them, are read from the
// row's beginning and up to its end, never outside it: what they share with
// the chunk beside them is set to -inf, as is every class that is not allowed.
// From then on a chunk needs no bounds and no mask: -inf has probability 0 and
// is no alternative.  A chunk is named by the class it begins with, which may
// be below 0 or past the row.

template <int DT>
struct Chunk {
  using S = Scalar<DT>;
  using T = typename S::T;
  static constexpr int V = 16 / sizeof(T);  // elements
  uint32_t w[4];

  __device__ __forceinline__ float get(int e) const {
    if constexpr (DT == BART_F32)
      return __uint_as_float(w[e]);
    else if constexpr (DT == BART_BF16)
      return __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
    else
      return S::wide(__builtin_bit_cast(T, (uint16_t)(w[e >> 1] >> (e & 1) * 16)));
  }
  __device__ __forceinline__ void set(int e, T v) {
    if constexpr (DT == BART_F32) {
      w[e] = __float_as_uint(v);
    } else {
      const uint32_t u = __builtin_bit_cast(uint16_t, v);
      w[e >> 1] = e & 1 ? (w[e >> 1] & 0xffffu) | u << 16 : (w[e >> 1] & 0xffff0000u) | u;
    }
  }
  __device__ __forceinline__ void rule_out(int e) {
    if constexpr (DT == BART_F32)
      w[e] = 0xff800000u;
    else
      set(e, __builtin_bit_cast(T, (uint16_t)(DT == BART_BF16 ? 0xff80 : 0xfc00)));
  }
  __device__ __forceinline__ void load(const T *p) { __builtin_memcpy(w, p, 16); }
  // Makes the compiler forget what it derived from the chunk: widened again
  // where it is needed again, a chunk stays in 4 registers in between.
  __device__ __forceinline__ void forget() {
    asm volatile("" : "+v"(w[0]), "+v"(w[1]), "+v"(w[2]), "+v"(w[3]));
  }
  static __device__ __forceinline__ void store(T *p, const float *d) {
    T v[V];
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = S::narrow(d[e]);
    __builtin_memcpy(p, v, 16);
  }
};

// One row's memory, for groups of T lanes.
template <int DT, int T_>
struct Row {
  using K = Chunk<DT>;
  using T = typename K::T;
  static constexpr int V = K::V;
  static constexpr bool kShort = T_ == 1;  // rows may be shorter than a chunk
  const T *x;
  const uint8_t *mask;
  int C;
  int head;  // classes between the first chunk's beginning and the row's

  __device__ __forceinline__ Row(const RowsArgs &A, int64_t i)
      : x((const T *)A.r.x + i * A.r.ld),
        mask(A.r.mask ? A.r.mask + i * A.r.ld_mask : nullptr),
        C(A.r.n_class),
        head(T_ >= 8 ? (int)((uintptr_t)x / sizeof(T) % V) : 0) {}

  // Where the chunk that begins with class j0 is read.
  __device__ __forceinline__ int base(int j0) const { return max(min(j0, C - V), 0); }

  // The chunks that begin with classes j, j + step, ...: all their loads are
  // under way before the first is looked at.
  template <int N>
  __device__ __forceinline__ void load(K (&c)[N], int j, int step) const {
    if (kShort && C < V) {
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const int at = j + n * step + e, k = min(at, C - 1);
          c[n].set(e, x[k]);
          if (at >= C || (mask && !mask[k])) c[n].rule_out(e);
        }
      return;
    }
#pragma unroll
    for (int n = 0; n < N; ++n) c[n].load(x + base(j + n * step));
    if (mask) {
      uint32_t ok[N][V / 4];
#pragma unroll
      for (int n = 0; n < N; ++n) __builtin_memcpy(ok[n], mask + base(j + n * step), V);
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (!(ok[n][e >> 2] & 0xffu << (e & 3) * 8)) c[n].rule_out(e);
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int j0 = j + n * step, b = base(j0);
      if (b != j0) {  // a row's first or last chunk, or none
#pragma unroll
        for (int e = 0; e < V; ++e)
          if ((uint32_t)(b + e - j0) >= (uint32_t)V) c[n].rule_out(e);
      }
    }
  }

  // The score of one class, -inf where it is not allowed.
  __device__ __forceinline__ float at(int j) const {
    return !mask || mask[j] ? Scalar<DT>::wide(x[j]) : kNegInf;
  }
};

// ----------------------------------------------------- statistics of a row
//
// With a = log2(e) / T: m = the largest score, M = a number next to m a (its
// rounded product, kept within 2^26), s = sum 2^z and t = sum z 2^z with z = x a
// - M.  Any M near m a serves; taken as it is, z is one multiply-add, rounded
// once.  Two such sets are joined by moving the one with the smaller M to the
// larger: the running maximum and sum of one pass.
// Beyond 2^26 a rounded product could be off by more than exponents can bear.
// Scores far below -2^26 (masks by large negative numbers) then have z far below 0
// and count for nothing; where they are all that a row has, or the largest is
// above 2^26, m a and M are apart by more than rounding (at most 4), and the
// row is summed again by differences x - m (`careful`).  A NaN among the scores
// shows as s = NaN, and a row without any as m = -inf.

constexpr float kMostRef = 0x1p26f;

struct Stats {
  float m, M, s, t;
};

__device__ __forceinline__ Stats no_stats() { return {kNegInf, -kMostRef, 0.f, 0.f}; }

__device__ __forceinline__ float ref_of(float m, float a) {
  return fminf(fmaxf(m * a, -kMostRef), kMostRef);
}

// Moves q to the reference M >= q.M.
__device__ __forceinline__ void move_to(Stats &q, float M) {
  const float z = q.M - M;
  const float f = exp2_fast(z);
  q.t = f == 0.f ? 0.f : f * (q.t + z * q.s);
  q.s *= f;
  q.M = M;
}

// The larger of three by one instruction (the compiler would quiet each
// operand first; a NaN among them shows in the sums).
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
  return d;
}

template <int DT, int N>
__device__ __forceinline__ float max_of(float m, const Chunk<DT> (&c)[N]) {
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int e = 0; e < Chunk<DT>::V; e += 2) m = max3(m, c[n].get(e), c[n].get(e + 1));
  return m;
}

// Adds the chunks to q, whose reference already covers them; without ENT, t
// is not kept.
template <bool ENT, int DT, int N>
__device__ __forceinline__ void sum_chunks(Stats &q, const Chunk<DT> (&c)[N], float a) {
  float s1 = 0.f, t1 = 0.f, M = q.M;
  // with and without ENT are two sides of a branch: were they seen to share their
  // exponentials, these would all be computed before it and kept (93 -> 188
  // registers with 64 elements a lane)
  if (ENT) asm("" : "+v"(M));
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int e = 0; e < Chunk<DT>::V; e += 2) {
      const float z0 = __builtin_fmaf(c[n].get(e), a, -M);
      const float z1 = __builtin_fmaf(c[n].get(e + 1), a, -M);
      const float p0 = exp2_fast(z0), p1 = exp2_fast(z1);
      q.s += p0;
      s1 += p1;
      if (ENT) {  // z of a score -inf is -inf: 0 x that would be NaN
        q.t = __builtin_fmaf(p0, fmaxf(z0, -1e4f), q.t);
        t1 = __builtin_fmaf(p1, fmaxf(z1, -1e4f), t1);
      }
    }
  q.s += s1;
  q.t += t1;
}

// Adds chunks that q's reference may not cover yet.
template <int DT, int N>
__device__ __forceinline__ void add_chunks(Stats &q, const Chunk<DT> (&c)[N], float a, bool ent) {
  q.m = max_of(q.m, c);
  move_to(q, ref_of(q.m, a));
  if (ent)
    sum_chunks<true>(q, c, a);
  else
    sum_chunks<false>(q, c, a);
}

// Joins the sets of T neighbouring lanes, all of which get the result.
template <int T>
__device__ __forceinline__ void join_lanes(Stats &q, bool ent) {
  q.m = lanes_max<T>(q.m);
  move_to(q, lanes_max<T>(q.M));
  q.s = lanes_sum<T>(q.s);
  if (ent) q.t = lanes_sum<T>(q.t);
}

// Joins the sets of the waves of a workgroup of W waves.
template <int W>
__device__ __forceinline__ void join_waves(Stats &q, bool ent, Stats *part) {
  if constexpr (W > 1) {
    __syncthreads();  // what was there has been read
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = q;
    __syncthreads();
    q = part[threadIdx.x % W];
    join_lanes<W>(q, ent);
  }
}

// What a call returns of one row, and what its gradient needs.
struct RowEnd {
  float m, logs, H;  // logs = ln sum exp((x - m) / T)
};

// Sums a row that has a score above -inf and no NaN by differences x - m,
// element by element.
template <int DT, int T>
__device__ __forceinline__ RowEnd careful(const Row<DT, T> &row, float inv_t, int lane,
                                          Stats *part) {
  constexpr int W = T > 64 ? T / 64 : 1, L = T > 64 ? 64 : T;
  auto all_max = [&](float v) {
    v = lanes_max<L>(v);
    if constexpr (W > 1) {
      __syncthreads();
      if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6].m = v;
      __syncthreads();
      v = lanes_max<W>(part[threadIdx.x % W].m);
    }
    return v;
  };
  auto all_sum = [&](float v) {
    v = lanes_sum<L>(v);
    if constexpr (W > 1) {
      __syncthreads();
      if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6].s = v;
      __syncthreads();
      v = lanes_sum<W>(part[threadIdx.x % W].s);
    }
    return v;
  };
  float m = kNegInf;
  for (int64_t j = lane; j < row.C; j += T) m = fmaxf(m, row.at((int)j));
  m = all_max(m);
  float s = 0.f, t = 0.f;
  for (int64_t j = lane; j < row.C; j += T) {
    const float z = (row.at((int)j) - m) * inv_t;
    const float p = exp2_fast(z * kLog2e);
    s += p;
    t += p * fmaxf(z, -1e4f);
  }
  s = all_sum(s);
  t = all_sum(t);
  const float logs = logf(s);
  return {m, logs, logs - t / s};
}

// A row's end from its joined statistics.
template <int DT, int T>
__device__ __forceinline__ RowEnd row_end(const RowsArgs &A, const Row<DT, T> &row, const Stats &q,
                                          float a, int lane, Stats *part) {
  const float off = __builtin_fmaf(q.m, a, -q.M);
  if (!uniform<T>(fabsf(off) <= 4.f && q.s < INFINITY)) {
    if (uniform<T>(q.s != q.s)) return {q.m, NAN, NAN};  // a NaN
    if (uniform<T>(q.m == kNegInf)) return {q.m, kNegInf, 0.f};  // nothing allowed
    return careful(row, A.inv_t, lane, part);
  }
  const float ln = logf(q.s);
  return {q.m, ln - kLn2 * off, ln - q.t * kLn2 / q.s};
}

__device__ __forceinline__ int64_t row_label(const RowsArgs &A, int64_t i) {
  return A.r.label ? A.r.label[i * A.r.label_stride] : -1;
}

// One lane writes a row's numbers; xl: the score of its label (anything where
// there is none).
__device__ __forceinline__ void write_row(const RowsArgs &A, int64_t i, const RowEnd &r,
                                          int64_t label, float xl) {
  if (A.o.logp) {
    float lp = 0.f;
    if (label >= A.r.n_class)
      lp = NAN;
    else if (label >= 0)
      lp = r.logs == kNegInf ? kNegInf : (xl - r.m) * A.inv_t - r.logs;
    A.o.logp[i] = lp;
  }
  if (A.o.entropy) A.o.entropy[i] = r.H;
  if (A.o.norm) {
    A.o.norm[2 * i] = r.m;
    A.o.norm[2 * i + 1] = r.logs;
  }
}

// ------------------------------------------------------------ alternatives
//
// A score and its class as one word that orders as the alternatives do:
// larger score first, lower class first among equal ones.  0 is below every
// score above -inf.

__device__ __forceinline__ uint64_t top_key(float x, uint32_t j) {
  const uint32_t b = __float_as_uint(x + 0.f);  // -0 and 0 are equal scores
  const uint32_t u = b & 0x80000000u ? ~b : b | 0x80000000u;
  return (uint64_t)u << 32 | (uint32_t)~j;
}
__device__ __forceinline__ float key_score(uint64_t k) {
  const uint32_t u = (uint32_t)(k >> 32);
  return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ int32_t key_class(uint64_t k) { return (int32_t)~(uint32_t)k; }
// The last class whose key with key_score(k) reaches k, which need not be a
// key: classes end before 2^30, and the score -0, which no key has, stands for 0.
__device__ __forceinline__ int32_t key_last(uint64_t k) {
  return k >> 32 == 0x7fffffffu ? INT32_MAX : (int32_t)min(~(uint32_t)k, (uint32_t)INT32_MAX);
}

// Alternative c of row i, or that there is none (key 0).
__device__ __forceinline__ void write_top(const RowsArgs &A, int64_t i, int c, uint64_t key,
                                          const RowEnd &r) {
  const float none = r.logs != r.logs ? NAN : kNegInf;
  const int64_t at = i * A.o.k + c;
  if (A.o.top_logp) A.o.top_logp[at] = key ? (key_score(key) - r.m) * A.inv_t - r.logs : none;
  if (A.o.top_class) A.o.top_class[at] = key ? key_class(key) : -1;
}

// The alternatives of a row by T < 64 lanes that hold it in registers (a
// lane's chunks begin with classes j0, j0 + T V, ...), one after the other: the
// largest score, its lowest class, then without it.
template <int DT, int N, int T>
__device__ __forceinline__ void top_by_rounds(const RowsArgs &A, int64_t i, const Row<DT, T> &row,
                                              const RowEnd &r, const Chunk<DT> (&c)[N], int lane,
                                              int j0) {
  constexpr int V = Chunk<DT>::V, E = N * V;
  float v[E];
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int e = 0; e < V; ++e) v[n * V + e] = c[n].get(e);
  const bool none = r.logs != r.logs || r.logs == kNegInf;
  for (int q = 0; q < A.o.k; ++q) {
    float own = kNegInf;
#pragma unroll
    for (int e = 0; e < E; e += 2) own = max3(own, v[e], v[e + 1]);
    const float best = lanes_max<T>(own);
    int at = -1;  // the first place that holds it
#pragma unroll
    for (int e = E - 1; e >= 0; --e) at = v[e] == best ? e : at;
    uint32_t j = ~0u;
    if (at >= 0) j = row.base(j0 + at / V * (T * V)) + at % V;
    const uint32_t first = ~lanes_max_u32<T>(~j);
    if (j != first) at = -1;
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = e == at ? kNegInf : v[e];
    if (lane == 0) write_top(A, i, q, none || best == kNegInf ? 0 : top_key(best, first), r);
  }
}

// Candidates for a row's alternatives, in LDS: a list that holds every score
// at or above a threshold that at least k scores reach.  The threshold is the
// k-th largest of the maxima of 64 columns (lane l of every wave that works on
// the row forms column l; 256 columns for k > 40 on 256 lanes and more), so on
// scores in no particular order the list gets about 64 ln(64 / (64 - k))
// entries, 24 for k = 20.  Where more scores reach it than the list holds (long
// runs of equal scores, large scores in fewer than k columns, k as large as the
// number of columns), the list is made anew above a tighter threshold, a key.
// Keys are read two at a time: at a multiple of 16 bytes by one instruction (64 of
// 65536 x 1000 f32 398 us, 502 otherwise).
template <int CAP>
struct alignas(16) TopList {
  uint64_t key[CAP];
  uint32_t count;
  uint32_t lanes;   // lanes that hold a candidate, their numbers in cols
  float theta;      // the threshold, where not every wave finds it
  uint64_t least;   // the tighter one
};

// The k-th largest of 64 lanes' values, k <= 64: by k rounds while they are
// few, else each lane counts the values above its own (cols: the 64 values in
// LDS).
__device__ __forceinline__ float kth_of_lanes(float u, int k, const float *cols) {
  const int lane = threadIdx.x & 63;
  if (k <= 8) {
    float best = kNegInf;
    for (int q = 0; q < k; ++q) {
      best = lanes_max<64>(u);
      if (lane == __ffsll((unsigned long long)__ballot(u == best)) - 1) u = kNegInf;
    }
    return best;
  }
  int above = 0;
#pragma unroll 16
  for (int i = 0; i < 64; ++i) {
    const float v = cols[i];
    above += v > u || (v == u && i < lane) ? 1 : 0;
  }
  return __shfl(u, __ffsll((unsigned long long)__ballot(above == k - 1)) - 1);
}

// Puts this wave's scores >= theta on the list (TIGHT: those equal to theta up
// to class `last`); count: its entries so far, where no other wave (T > 64)
// appends to it.
template <int T, bool TIGHT, int DT, int CAP>
__device__ __forceinline__ void list_chunk(TopList<CAP> &list, uint32_t &count,
                                           const Chunk<DT> &c, int base, float theta, int last) {
#pragma unroll
  for (int e = 0; e < Chunk<DT>::V; ++e) {
    const float v = c.get(e);
    const bool in = v >= theta && v > kNegInf && (!TIGHT || v > theta || base + e <= last);
    const uint64_t who = __ballot(in);
    if (!who) continue;
    uint32_t at = count;
    if constexpr (T > 64) {
      const int first = __ffsll((unsigned long long)who) - 1;
      if ((threadIdx.x & 63) == first) at = atomicAdd(&list.count, (uint32_t)__popcll(who));
      at = __builtin_amdgcn_readlane(at, first);
    } else {
      count += __popcll(who);
    }
    at += lanes_before(who);
    if (in && at < CAP) list.key[at] = top_key(v, base + e);
  }
}

// Lists the scores of the chunks of the lanes that have one to list (mine),
// spread over all lanes.  The list's count is that of all, also where it does
// not hold them.  cols gets those lanes' numbers; list.count and list.lanes are
// 0 before.
template <bool TIGHT, int DT, int T, int CAP>
__device__ __forceinline__ void list_row(const Row<DT, T> &row, int from, int to, bool mine,
                                         float theta, int last, int lane, float *cols,
                                         TopList<CAP> &list) {
  constexpr int V = Chunk<DT>::V;
  if (const uint64_t who = __ballot(mine)) {
    const int first = __ffsll((unsigned long long)who) - 1;
    uint32_t at = 0;
    if ((lane & 63) == first) at = atomicAdd(&list.lanes, (uint32_t)__popcll(who));
    at = __builtin_amdgcn_readlane(at, first) + lanes_before(who);
    if (mine) cols[at] = __uint_as_float(lane);
  }
  group_sync<T>();
  const uint32_t lanes = uniform<T>(list.lanes);
  uint32_t count = 0;
  const uint32_t items = lanes * (uint32_t)((to - from + T * V - 1) / (T * V));
  for (uint32_t it = lane; it - lane < items; it += T) {
    const uint32_t turn = it / max(lanes, 1u);  // the lane's chunk number `turn`
    int64_t j = to;
    if (it < items)
      j = from + ((int64_t)turn * T + __float_as_uint(cols[it - turn * lanes])) * V;
    Chunk<DT> c[1];
    const int j0 = j < to ? (int)j : row.C;  // past the row: nothing
    row.load(c, j0, 0);
    list_chunk<T, TIGHT>(list, count, c[0], row.base(j0), theta, last);
  }
  if (T == 64 && lane == 0) list.count = count;
  group_sync<T>();
}

// Gives put the list's best k in order (and 0 for those it lacks), T lanes.
template <int CAP, class PUT>
__device__ __forceinline__ void put_ranked(const TopList<CAP> &list, int lane, int T, int k,
                                           PUT put) {
  const int n = min(list.count, (uint32_t)CAP);
  for (int c = lane; c < n; c += T) {
    const uint64_t key = list.key[c];
    int rank = 0;
    for (int q = 0; q < n; ++q) rank += list.key[q] > key ? 1 : 0;
    if (rank < k) put(rank, key);
  }
  for (int c = n + lane; c < k; c += T) put(c, (uint64_t)0);
}

// The k best of a row's chunks that begin in [from, to) by T >= 64 lanes; own:
// the largest score this lane has seen of its chunks (every T-th).  put(c, key)
// takes alternative c (key 0: there is none).  The chunks of the few lanes
// that hold a candidate are read again, spread over all lanes (one after the
// other by their own lanes, 4096 x 32768 bf16 with 5 alternatives took 85 us
// instead of 55).  cols: T floats, list: in LDS.
template <int DT, int T, int CAP, class PUT>
__device__ __forceinline__ void top_by_list(const Row<DT, T> &row, int k, int from, int to,
                                            float own, int lane, float *cols, TopList<CAP> &list,
                                            PUT put) {
  constexpr int W = T / 64;
  cols[lane] = own;
  if (lane == 0) list.count = list.lanes = 0;
  group_sync<T>();
  float theta;
  if (W >= 4 && k > 40) {
    constexpr int kCols = W >= 4 ? 256 : 64;
    float u = own;
    if (lane < kCols)
      for (int w = 1; w < T / kCols; ++w) u = fmaxf(u, cols[w * kCols + lane]);
    __syncthreads();
    if (lane < kCols) cols[lane] = u;
    __syncthreads();
    if (lane < kCols) {
      int above = 0;
#pragma unroll 16
      for (int i = 0; i < kCols; ++i) {
        const float v = cols[i];
        above += v > u || (v == u && i < lane) ? 1 : 0;
      }
      if (above == k - 1) list.theta = u;
    }
    __syncthreads();
    theta = list.theta;
  } else {
    if constexpr (W > 1) {
      if (lane < 64) {
        float u = own;
        for (int w = 1; w < W; ++w) u = fmaxf(u, cols[w * 64 + lane]);
        cols[lane] = u;
      }
      __syncthreads();
    }
    theta = kth_of_lanes(cols[lane & 63], k, cols);
    group_sync<T>();  // cols have been read
  }
  list_row<false>(row, from, to, own >= theta && own > kNegInf, theta, 0, lane, cols, list);
  // An overflowing list is made anew above the k-th best of its first entries:
  // where they come in no particular order, one in 256 / k of them remains.  After
  // kSamples such lists the threshold is searched for by counting what reaches
  // it, at most 64 times however the scores lie.
  constexpr int kSample = 256, kSamples = 3;
  static_assert(kSample <= CAP && kSample > BART_MAX_TOP, "a tighter threshold exists");
  KeySearch s{0, ~(uint64_t)0};
  uint32_t count = uniform<T>(list.count);
  for (int pass = 0;
       pass < kSamples + 64 && (count > CAP || (pass > kSamples && count < (uint32_t)k)); ++pass) {
    if (pass < kSamples) {
      for (int c = lane; c < kSample; c += T) {
        const uint64_t key = list.key[c];
        int rank = 0;
#pragma unroll 8
        for (int q = 0; q < kSample; ++q) rank += list.key[q] > key ? 1 : 0;
        if (rank == k - 1) list.least = key;
      }
      group_sync<T>();
      s.lo = uniform64(list.least);
    }
    const uint64_t least = pass < kSamples ? s.lo : s.probe();
    if (lane == 0) list.count = list.lanes = 0;
    group_sync<T>();
    theta = key_score(least);
    list_row<true>(row, from, to, own >= theta, theta, key_last(least), lane, cols, list);
    count = uniform<T>(list.count);
    if (pass >= kSamples) s.take(least, count, k);
    group_sync<T>();  // the count has been read
  }
  put_ranked(list, lane, T, k, put);
}

// The alternatives of a whole row.
template <int DT, int T, int CAP>
__device__ __forceinline__ void top_of_row(const RowsArgs &A, int64_t i, const Row<DT, T> &row,
                                           const RowEnd &r, float own, int lane, float *cols,
                                           TopList<CAP> &list) {
  auto put = [&](int c, uint64_t key) { write_top(A, i, c, key, r); };
  if (r.logs != r.logs || r.logs == kNegInf) {
    for (int c = lane; c < A.o.k; c += T) put(c, 0);
    return;
  }
  top_by_list<DT, T>(row, A.o.k, -row.head, row.C, own, lane, cols, list, put);
}

// ---------------------------------------------------------------- gradient

// What the gradient of a row needs to know of it.  kind 0: zeros; 1: the
// formula, with p = 2^z / s; 2: NaN wherever the score is above -inf; 3: the
// formula by differences, for scores too large for z.
struct RowGrad {
  int kind;
  float m, a, M, nl2;  // log2 p = x a - M + nl2
  float c, h, K;       // d = 2^z (c + h (z + K))
  float at_label;      // added at the label
  int label;
  int has_h;           // h is not 0
};

template <int T>
__device__ __forceinline__ RowGrad row_grad(const RowsArgs &A, int64_t i, int64_t label,
                                            const RowEnd &r) {
  RowGrad q;
  const float w = A.g.w_logp && label >= 0 ? A.g.w_logp[i * A.g.w_logp_stride] : 0.f;
  const float h = A.g.w_entropy ? A.g.w_entropy[i * A.g.w_entropy_stride] : 0.f;
  q.m = r.m;
  q.a = A.inv_t * kLog2e;
  q.M = ref_of(r.m, q.a);
  const bool big = fabsf(q.M) >= kMostRef;
  q.kind = (w == 0.f && h == 0.f) || r.logs == kNegInf ? 0 : r.logs != r.logs ? 2 : big ? 3 : 1;
  if (w != 0.f && label >= A.r.n_class) q.kind = 2;
  q.nl2 = -r.logs * kLog2e;
  if (q.kind == 1) q.nl2 -= __builtin_fmaf(r.m, q.a, -q.M);
  const float p0 = exp2_fast(q.nl2);  // 1 / s
  q.c = -w * A.inv_t * p0;
  q.h = -h * A.inv_t * kLn2 * p0;
  q.K = h != 0.f ? r.H * kLog2e + q.nl2 : 0.f;  // no H is kept without w_entropy
  q.at_label = w * A.inv_t;
  // a weight that is not finite: NaN, but not where there is no probability
  if (q.kind & 1 && !(fabsf(q.c) + fabsf(q.h) + fabsf(q.at_label) < INFINITY)) q.kind = 2;
  q.label = label >= 0 && label < A.r.n_class ? (int)label : -1;
  q.kind = uniform<T>(q.kind);
  q.has_h = uniform<T>(q.h != 0.f);
  return q;
}

// The gradient of the chunk that begins with class j0, written to its place
// in out.
template <int DT, int T>
__device__ __forceinline__ void grad_chunk(const Row<DT, T> &row, typename Scalar<DT>::T *out,
                                           const RowGrad &q, const Chunk<DT> &c, int j0) {
  using K = Chunk<DT>;
  constexpr int V = K::V;
  const int b = row.kShort && row.C < V ? j0 : row.base(j0);
  float d[V];
  if (q.kind == 1) {
    if (!q.has_h) {
#pragma unroll
      for (int e = 0; e < V; ++e) d[e] = q.c * exp2_fast(__builtin_fmaf(c.get(e), q.a, -q.M));
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float z = __builtin_fmaf(c.get(e), q.a, -q.M);
        d[e] = exp2_fast(z) * __builtin_fmaf(q.h, fmaxf(z, -1e4f) + q.K, q.c);
      }
    }
  } else if (q.kind == 3) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float z = (c.get(e) - q.m) * q.a;
      d[e] = exp2_fast(z) * __builtin_fmaf(q.h, fmaxf(z, -1e4f) + q.K, q.c);
    }
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) d[e] = q.kind == 0 || c.get(e) == kNegInf ? 0.f : NAN;
  }
  if (q.kind & 1 && (uint32_t)(q.label - b) < (uint32_t)V) {
#pragma unroll
    for (int e = 0; e < V; ++e)
      if (b + e == q.label && c.get(e) != kNegInf) d[e] += q.at_label;
  }
  if (j0 >= 0 && j0 + V <= row.C) {
    K::store(out + j0, d);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e)
      if ((uint32_t)(b + e - j0) < (uint32_t)V && b + e < row.C)
        out[b + e] = Scalar<DT>::narrow(d[e]);
  }
}

// ----------------------------------------------------------------- kernels

// T lanes hold a row in registers, E elements each: every score is read once,
// and the gradient written from what was read.  T <= 64: 256 / T rows per
// workgroup; T > 64: one.  STATS false: the gradient alone, from norm and
// entropy.  There is no loop over rows: the compiler would keep each chunk's
// address and bounds in registers from row to row (65536 x 1000 f32 77 us
// instead of 44).  Bound by memory: 65536 x 1000 f32 44 us (6.0 TB/s), 8192 x
// 32768 bf16 with the gradient 189 us (5.7 TB/s), gradient alone 30011 x 1000
// f32 48 us (5.0 TB/s); 1e6 x 10 f32 with 3 alternatives 17.7 us (4.5 TB/s),
// where the alternatives' rounds issue beside the loads.
template <int DT, int T, int E, bool STATS>
__global__ __launch_bounds__(T > 256 ? T : 256) void k_rows(RowsArgs A, const float *norm,
                                                           const float *entropy) {
  using K = Chunk<DT>;
  constexpr int V = K::V, N = E / V, B = T > 256 ? T : 256, W = T > 64 ? T / 64 : 1;
  constexpr int CAP = T > 64 ? 1024 : 256;
  constexpr bool kLists = STATS && T >= 64;
  __shared__ Stats part[W];
  __shared__ float cols[kLists ? B : 1];
  __shared__ TopList<kLists ? CAP : 1> lists[kLists ? B / T : 1];
  const int lane = threadIdx.x % T;
  const float a = A.inv_t * kLog2e;
  const int64_t i = A.first + (int64_t)blockIdx.x * (B / T) + uniform<T>(threadIdx.x / T);
  if (i >= A.r.n) return;  // T > 64: not taken, there is one row per workgroup
  const Row<DT, T> row(A, i);
  const int64_t label = row_label(A, i);
  K c[N];
  const int j0 = lane * V - row.head;
  row.load(c, j0, T * V);
  RowEnd r;
  if constexpr (STATS) {
    const float xl = label >= 0 && label < row.C ? row.at((int)label) : 0.f;
    const bool ent = A.o.entropy || A.g.w_entropy;
    Stats q = no_stats();
    const float own = q.m = max_of(q.m, c);
    q.M = ref_of(q.m, a);
    if (N > 4) {
#pragma unroll
      for (int n = 0; n < N; ++n) c[n].forget();
    }
    if (ent)
      sum_chunks<true>(q, c, a);
    else
      sum_chunks<false>(q, c, a);
    join_lanes<(T < 64 ? T : 64)>(q, ent);
    join_waves<W>(q, ent, part);
    r = row_end(A, row, q, a, lane, part);
    if (lane == 0) write_row(A, i, r, label, xl);
    if (A.o.k) {
      if constexpr (T < 64)
        top_by_rounds<DT, N, T>(A, i, row, r, c, lane, j0);
      else
        top_of_row<DT, T>(A, i, row, r, own, lane, cols + threadIdx.x / T * T,
                          lists[threadIdx.x / T]);
    }
  } else {
    r = {norm[2 * i], norm[2 * i + 1], A.g.w_entropy ? entropy[i] : 0.f};
  }
  if (A.g.grad) {
    if (N > 4) {
#pragma unroll
      for (int n = 0; n < N; ++n) c[n].forget();
    }
    // in place: every read of the row before its place may be overwritten
    if (STATS) group_sync<(T < 64 ? 64 : T)>();
    const RowGrad q = row_grad<T>(A, i, label, r);
    auto *out = (typename K::T *)A.g.grad + i * A.g.ld_grad;
#pragma unroll
    for (int n = 0; n < N; ++n)
      if (j0 + n * T * V < row.C) grad_chunk(row, out, q, c[n], j0 + n * T * V);
  }
}

// Rows of any length: T lanes read a row's chunks 4 at a time, and a second
// time for the gradient, except the last H chunks of each lane, which stay in
// registers.  Bound by memory: 16384 x 131072 bf16 701 us (6.1 TB/s at 8
// instructions per score); with the gradient by what is read twice, which
// reaches the caches beyond the compute unit's own at the rate of memory:
// 8192 x 50001 bf16 361 us (4.5 TB/s of operands).
template <int DT, int T, int H>
__global__ __launch_bounds__(T) void k_rows_stream(RowsArgs A) {
  using K = Chunk<DT>;
  constexpr int V = K::V, W = T / 64, N = 4, CAP = 1024;
  __shared__ Stats part[W];
  __shared__ float cols[T];
  __shared__ TopList<CAP> list;
  const int lane = threadIdx.x;
  const float a = A.inv_t * kLog2e;
  const bool ent = A.o.entropy || A.g.w_entropy;
  const int64_t i = A.first + blockIdx.x;
  const Row<DT, T> row(A, i);
  const int64_t label = row_label(A, i);
  const float xl = label >= 0 && label < row.C ? row.at((int)label) : 0.f;
  const int j0 = lane * V - row.head;
  Stats q = no_stats();
  constexpr int kPiece = N * T * V;
  // the pieces that are read twice end where the held chunks begin
  const int pieces = (max(row.C + row.head - H * T * V, 0) + kPiece - 1) / kPiece;
  for (int p = 0; p < pieces; ++p) {
    K c[N];
    row.load(c, opaque(p * kPiece) + j0, T * V);
    add_chunks(q, c, a, ent);
  }
  K held[H ? H : 1];
  const int jh = opaque(pieces * kPiece) + j0;
  if constexpr (H > 0) {
    row.load(held, jh, T * V);
    add_chunks(q, held, a, ent);
  }
  const float own = q.m;
  join_lanes<64>(q, ent);
  join_waves<W>(q, ent, part);
  const RowEnd r = row_end(A, row, q, a, lane, part);
  if (lane == 0) write_row(A, i, r, label, xl);
  if (A.o.k) top_of_row<DT, T>(A, i, row, r, own, lane, cols, list);
  if (A.g.grad) {
    __syncthreads();  // every read of the row before its place may be overwritten
    const RowGrad g = row_grad<T>(A, i, label, r);
    auto *out = (typename K::T *)A.g.grad + i * A.g.ld_grad;
    if constexpr (H > 0) {
#pragma unroll
      for (int n = 0; n < H; ++n) {
        held[n].forget();
        if (jh + n * T * V < row.C) grad_chunk(row, out, g, held[n], jh + n * T * V);
      }
    }
    // last piece first: what was read last is the likeliest to be near
    for (int p = pieces - 1; p >= 0; --p) {
      K c[N];
      const int j = opaque(p * kPiece) + j0;
      row.load(c, j, T * V);
#pragma unroll
      for (int n = 0; n < N; ++n)
        if (j + n * T * V < row.C) grad_chunk(row, out, g, c[n], j + n * T * V);
    }
  }
}

// Few long rows: each row's chunks are split over S workgroups of 256 lanes,
// `length` classes (a multiple of 256 V) each, that leave their statistics
// and their k best keys in part [n][S] and keys [n][S][k].  Bound by latency:
// one row of 131101 bf16 classes 3.4 us here and 2.4 in the join, 8.3 and 4.2
// with 20 alternatives, whose candidates are read again and ranked here.
template <int DT>
__global__ __launch_bounds__(256) void k_rows_part(RowsArgs A, int S, int length, Stats *part_out,
                                                  uint64_t *keys) {
  using K = Chunk<DT>;
  constexpr int V = K::V, T = 256, W = T / 64, N = 2, CAP = 1024;
  __shared__ Stats part[W];
  __shared__ float cols[T];
  __shared__ TopList<CAP> list;
  const int lane = threadIdx.x;
  const float a = A.inv_t * kLog2e;
  const bool ent = A.o.entropy || A.g.w_entropy;
  const int64_t i = A.first + blockIdx.x / (uint32_t)S;
  const int s = (int)(blockIdx.x % (uint32_t)S);
  const Row<DT, T> row(A, i);
  const int from = (int)min((int64_t)s * length - row.head, (int64_t)row.C);
  const int to = (int)min((int64_t)from + length, (int64_t)row.C);
  Stats q = no_stats();
  for (int64_t j = from; j < to; j += N * T * V) {
    K c[N];
    row.load(c, (int)j + lane * V, T * V);
    if (j + N * T * V > to) {  // the chunks of the next workgroup
#pragma unroll
      for (int n = 0; n < N; ++n)
        if (j + n * T * V + lane * V >= to) {
#pragma unroll
          for (int e = 0; e < V; ++e) c[n].rule_out(e);
        }
    }
    add_chunks(q, c, a, ent);
  }
  const float own = q.m;
  join_lanes<64>(q, ent);
  join_waves<W>(q, ent, part);
  const int64_t at = i * S + s;
  if (lane == 0) part_out[at] = q;
  if (A.o.k)
    top_by_list<DT, T>(row, A.o.k, from, to, own, lane, cols, list,
                       [&](int c, uint64_t key) { keys[at * A.o.k + c] = key; });
}

// Joins the parts of each row, S <= kMaxParts; norm and entropy, where not
// NULL, get what the gradient needs.  With r = ceil(k / S), at least k keys
// reach the ceil(k / r)-th largest of the parts' r-th keys; those that do are
// ranked (about k of them where the parts are alike).
constexpr int kMaxParts = 32;

template <int DT>
__global__ __launch_bounds__(256) void k_rows_join(RowsArgs A, int S, const Stats *part_in,
                                                  const uint64_t *keys, float *norm,
                                                  float *entropy) {
  constexpr int T = 256, W = T / 64;
  __shared__ Stats part[W];
  __shared__ TopList<kMaxParts * BART_MAX_TOP> list;
  __shared__ uint64_t nth[kMaxParts];
  const int lane = threadIdx.x, k = A.o.k;
  const int64_t i = A.first + blockIdx.x;
  keys += i * S * k;
  // of the keys, the first a lane looks at are loaded beside the rest
  const uint64_t early = lane < S * k ? keys[lane] : 0;
  const int r_th = (k + S - 1) / S;
  if (k && lane < S) nth[lane] = keys[lane * k + r_th - 1];
  const Row<DT, T> row(A, i);
  const int64_t label = row_label(A, i);
  const float xl = label >= 0 && label < row.C ? row.at((int)label) : 0.f;
  Stats q = (lane & 63) < S ? part_in[i * S + (lane & 63)] : no_stats();
  join_lanes<64>(q, true);
  const RowEnd r = row_end(A, row, q, A.inv_t * kLog2e, lane, part);
  if (lane == 0) {
    write_row(A, i, r, label, xl);
    if (norm) {
      norm[2 * i] = r.m;
      norm[2 * i + 1] = r.logs;
      entropy[i] = r.H;
    }
    list.count = 0;
  }
  __syncthreads();
  if (k == 0) return;
  if (!(r.logs != r.logs || r.logs == kNegInf)) {
    // equal keys do not occur, except 0: no score
    const uint64_t mine = nth[min(lane & 63, S - 1)];
    int above = 0;
    for (int p = 0; p < S; ++p) above += nth[p] > mine ? 1 : 0;
    const uint64_t theta = max(
        lanes_max_u64<64>(above >= (k + r_th - 1) / r_th - 1 ? mine : 0), (uint64_t)1);
    for (int q = lane; q < S * k; q += T) {
      const uint64_t key = q < T ? early : keys[q];
      if (key >= theta) list.key[atomicAdd(&list.count, 1u)] = key;
    }
  }
  __syncthreads();
  put_ranked(list, lane, T, k, [&](int c, uint64_t key) { write_top(A, i, c, key, r); });
}

// The gradient alone of rows of many classes: workgroups of 256 lanes take
// pieces of 4 chunks a lane.  Bound by memory: 2047 x 50001 bf16 73.5 us (5.6
// TB/s).
template <int DT>
__global__ __launch_bounds__(256) void k_grad_wide(RowsArgs A, const float *norm,
                                                  const float *entropy, int pieces) {
  using K = Chunk<DT>;
  constexpr int V = K::V, N = 4;
  const int64_t i = A.first + blockIdx.x / (uint32_t)pieces;
  const Row<DT, 256> row(A, i);
  const int j = (int)(blockIdx.x % (uint32_t)pieces) * (N * 256 * V) + (int)threadIdx.x * V -
                row.head;
  K c[N];
  row.load(c, j, 256 * V);
  const RowGrad q = row_grad<256>(A, i, row_label(A, i),
                             {norm[2 * i], norm[2 * i + 1], A.g.w_entropy ? entropy[i] : 0.f});
  auto *out = (typename K::T *)A.g.grad + i * A.g.ld_grad;
#pragma unroll
  for (int n = 0; n < N; ++n)
    if (j + n * 256 * V < row.C) grad_chunk(row, out, q, c[n], j + n * 256 * V);
}

}  // namespace bart
