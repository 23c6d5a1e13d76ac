// ops.hip -- host side of the entry points of bart_ops.h: checks, plans,
// launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <exception>
#include <iterator>
#include <vector>

#include "adamw.hpp"
#include "bart.h"
#include "bart_ops.h"
#include "error.hpp"
#include "rows.hpp"

using namespace bart;

namespace {

#define HIP_TRY(expr)                                                              \
  do {                                                                             \
    hipError_t e_ = (expr);                                                        \
    if (e_ != hipSuccess)                                                          \
      return fail(BART_EHIP, "%s failed: %s", #expr, hipGetErrorString(e_));       \
  } while (0)

// Makes a device the current one until the end of a call, for a plan that keeps
// the device it was made on.
struct OnDevice {
  int before = -1;
  hipError_t enter(int device) {
    int now = 0;
    if (const hipError_t e = hipGetDevice(&now); e != hipSuccess) return e;
    if (now == device) return hipSuccess;
    before = now;
    return hipSetDevice(device);
  }
  ~OnDevice() {
    if (before >= 0) (void)hipSetDevice(before);
  }
};

constexpr int64_t kMaxRows = (int64_t)1 << 40;
constexpr int64_t kMaxLd = (int64_t)1 << 40;

// Whether the rows [a, a + bytes of n rows) of two buffers share memory.
bool overlap(const void *a, int64_t abytes, const void *b, int64_t bbytes) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + (uintptr_t)bbytes && y < x + (uintptr_t)abytes;
}

// Whether rows of `row` bytes that begin `stride` bytes apart at a lie in the gaps
// between such rows at b.
bool between(const void *a, const void *b, int64_t row, int64_t stride) {
  if (stride == 0) return false;
  const int64_t off = (int64_t)((uintptr_t)a - (uintptr_t)b) % stride;
  const int64_t at = off < 0 ? off + stride : off;
  return at >= row && at <= stride - row;
}

// Whether n steps of a stride reach past what an address computation holds.
bool too_far(int64_t n, int64_t stride) { return stride > 0 && n > ((int64_t)1 << 60) / stride; }

const char *check_rows(const bart_rows *r) {
  if (!r) return "rows is NULL";
  if (r->n < 0 || r->n > kMaxRows) return "n must be in [0, 2^40]";
  if (r->n_class < 1 || r->n_class > (1 << 30)) return "n_class must be in [1, 2^30]";
  if (!dtype_ok(r->dtype)) return "dtype must be BART_F32, BART_F16 or BART_BF16";
  if (r->ld < 0 || r->ld > kMaxLd) return "ld must be in [0, 2^40]";
  if (r->n > 0 && !r->x) return "x is NULL";
  if ((uintptr_t)r->x % dtype_bytes(r->dtype)) return "x is not aligned to its elements";
  if (too_far(r->n, r->ld)) return "n x ld must not exceed 2^60";
  if (r->label && (r->label_stride < 0 || too_far(r->n, r->label_stride)))
    return "label_stride must be >= 0, n x label_stride at most 2^60";
  if ((uintptr_t)r->label % 8) return "label is not aligned to its elements";
  if (r->mask && (r->ld_mask < 0 || r->ld_mask > kMaxLd || too_far(r->n, r->ld_mask)))
    return "ld_mask must be in [0, 2^40], n x ld_mask at most 2^60";
  if (!(r->temperature >= 1e-30 && r->temperature <= 1e30))
    return "temperature must be in [1e-30, 1e30]";
  return nullptr;
}

const char *check_grad(const bart_rows *r, const bart_rows_grad *g) {
  if (r->n > 0 && !g->grad) return "grad is NULL";
  if (r->n > 0 && !g->w_logp && !g->w_entropy) return "a gradient needs w_logp or w_entropy";
  if (g->w_logp && (g->w_logp_stride < 0 || too_far(r->n, g->w_logp_stride)))
    return "w_logp_stride must be >= 0, n x w_logp_stride at most 2^60";
  if (g->w_entropy && (g->w_entropy_stride < 0 || too_far(r->n, g->w_entropy_stride)))
    return "w_entropy_stride must be >= 0, n x w_entropy_stride at most 2^60";
  if (r->n > 0 && g->w_logp && !r->label) return "w_logp needs labels";
  if (g->ld_grad < r->n_class || g->ld_grad > kMaxLd || too_far(r->n, g->ld_grad))
    return "ld_grad must be in [n_class, 2^40], n x ld_grad at most 2^60";
  if ((uintptr_t)g->grad % dtype_bytes(r->dtype)) return "grad is not aligned to its elements";
  if (((uintptr_t)g->w_logp | (uintptr_t)g->w_entropy) % 4)
    return "the weights are not aligned to their elements";
  if (r->n == 0) return nullptr;
  const int64_t es = dtype_bytes(r->dtype);
  const bool same = g->grad == r->x && (g->ld_grad == r->ld || r->n == 1);
  const bool apart = g->ld_grad == r->ld && between(g->grad, r->x, r->n_class * es, r->ld * es);
  if (!same && !apart && overlap(r->x, ((r->n - 1) * r->ld + r->n_class) * es, g->grad,
                       ((r->n - 1) * g->ld_grad + r->n_class) * es))
    return "grad overlaps the scores without being them";
  return nullptr;
}

RowsArgs rows_args(const bart_rows *r, const bart_rows_out *o, const bart_rows_grad *g) {
  RowsArgs A;
  A.r = *r;
  A.o = o ? *o : bart_rows_out{};
  A.g = g ? *g : bart_rows_grad{};
  A.inv_t = (float)(1.0 / r->temperature);
  A.first = 0;
  return A;
}

using RowsFn = void (*)(RowsArgs, const float *, const float *);
struct RowsLaunch {
  RowsFn fn;
  int per_block, block;  // rows and lanes of a workgroup
};

// Classes that the chunks of a row have to hold room for: where not every row
// begins on a 16-byte boundary, its first chunk begins before it.
int64_t span_of(const bart_rows &r) {
  const int es = dtype_bytes(r.dtype);
  const bool aligned = (uintptr_t)r.x % 16 == 0 && (r.n == 1 || r.ld * es % 16 == 0);
  return r.n_class + (aligned ? 0 : 16 / es - 1);
}

// Rows held in registers (fn NULL: longer than that pays).  Measured, us:
//  - 512 classes and many alternatives: 64 lanes and a list against 32 lanes
//    and a round for each: 65536 x 500 f32, k = 8 69 / 65, k = 20 88 / 138;
//  - 1024: 32 elements a lane of 32 against 16 of 64: 65536 x 1000 bf16, k = 0
//    26 / 33, k = 2 43 / 58, k = 5 72 / 70, f32 44 / 44, 55 / 61, 78 / 70;
//  - 4096: 64 a lane of 64 against 16 of 256: 32768 x 4096 bf16 53 / 63, with
//    a gradient 101 / 113, f32 94 / 86 and 210 / 188, with 5 alternatives 109 /
//    127;
//  - 16384 with a gradient: 64 a lane of 256 against a stream: 8192 x 16384
//    f32 209 / 239; without one a stream is as fast (94);
//  - 32768 with a gradient: 64 a lane of 512 against 32 of 1024: 8192 x 32768
//    bf16 194 / 224, f32 (twice the registers) 4096 x 32768 230 / 195;
//  - beyond: a stream that holds a part against 64 a lane of 1024: 8192 x 50001
//    bf16 361 / 460.
template <int DT>
RowsLaunch rows_in_registers(const RowsArgs &A) {
  const int64_t C = span_of(A.r);
  if (A.r.n_class <= 16) return {k_rows<DT, 1, 16, true>, 256, 256};
  if (A.r.n_class <= 32) return {k_rows<DT, 2, 16, true>, 128, 256};
  if (A.r.n_class <= 64) return {k_rows<DT, 4, 16, true>, 64, 256};
  if (C <= 128) return {k_rows<DT, 8, 16, true>, 32, 256};
  if (C <= 256) return {k_rows<DT, 16, 16, true>, 16, 256};
  if (C <= 512 && A.o.k <= 10) return {k_rows<DT, 32, 16, true>, 8, 256};
  if (C <= 1024 && A.o.k <= 2) return {k_rows<DT, 32, 32, true>, 8, 256};
  if (C <= 1024) return {k_rows<DT, 64, 16, true>, 4, 256};
  if (C <= 2048) return {k_rows<DT, 64, 32, true>, 4, 256};
  if constexpr (DT == BART_F32)
    if (C <= 4096 && !A.o.k) return {k_rows<DT, 256, 16, true>, 1, 256};
  if (C <= 4096) return {k_rows<DT, 64, 64, true>, 4, 256};
  if (C <= 8192) return {k_rows<DT, 256, 32, true>, 1, 256};
  if (!A.g.grad) return {};
  if (C <= 16384) return {k_rows<DT, 256, 64, true>, 1, 256};
  if (C > 32768) return {};
  if constexpr (DT == BART_F32)
    return {k_rows<DT, 1024, 32, true>, 1, 1024};
  else
    return {k_rows<DT, 512, 64, true>, 1, 512};
}

// The gradient alone: rows that 2048 elements a wave hold; longer ones are cut
// into pieces.
template <int DT>
RowsLaunch grad_in_registers(const RowsArgs &A) {
  const int64_t C = span_of(A.r);
  if (A.r.n_class <= 16) return {k_rows<DT, 1, 16, false>, 256, 256};
  if (A.r.n_class <= 32) return {k_rows<DT, 2, 16, false>, 128, 256};
  if (A.r.n_class <= 64) return {k_rows<DT, 4, 16, false>, 64, 256};
  if (C <= 128) return {k_rows<DT, 8, 16, false>, 32, 256};
  if (C <= 256) return {k_rows<DT, 16, 16, false>, 16, 256};
  if (C <= 512) return {k_rows<DT, 32, 16, false>, 8, 256};
  if (C <= 1024) return {k_rows<DT, 64, 16, false>, 4, 256};
  if (C <= 2048) return {k_rows<DT, 64, 32, false>, 4, 256};
  return {};
}

// Few long rows are split over workgroups: parts of a row and classes of a
// part (S = 1: not split).  A second launch joins the parts, and a gradient is a
// third; each also costs the caller 3 us, so it pays where one workgroup would
// read for long: 131072 bf16 classes, us on the device of 1 / 32 / 64 / 128
// rows: split 5.2 / 6.3 / 8.4 / 11.7, a row per workgroup 10 / 10 / 11 / 12;
// 100000 classes, 1 row, without and with 20 alternatives: 5.1 and 11.4, 9.8 and
// 14.6.  At 65536, forward / with 20 alternatives / with the gradient, split
// against a row per workgroup: 1 row bf16 5.3 / 11.6 / 8.8 against 6.6 / 10.4 /
// 10.0, f32 5.0 / 10.8 / 8.4 against 6.7 / 10.8 / 11.8; 64 rows bf16 6.4 / 12.6 /
// 11.7 against 7.3 / 11.6 / 11.5, f32 7.6 / 13.6 / 15.8 against 8.0 / 12.4 / 14.3.
// What up to 16 rows without alternatives gain there is less than the launches
// cost; at 40000 classes the gain is below 1 us and alternatives lose 2 to 3.
struct Split {
  int S, length;
};

Split split_of(const bart_rows &r) {
  if (r.n > 64 || r.n_class <= 65536) return {1, 0};
  const int step = 256 * 16 / dtype_bytes(r.dtype);  // a chunk a lane
  const int64_t span = span_of(r);
  int64_t S = std::min<int64_t>({kMaxParts, (span + step - 1) / step, 512 / std::max<int64_t>(r.n, 1)});
  if (S < 2) return {1, 0};
  const int64_t length = ((span + S - 1) / S + step - 1) / step * step;
  return {(int)((span + length - 1) / length), (int)length};
}

// Workspace of a split call: statistics, keys, and what the gradient needs.
struct SplitSpace {
  size_t part, keys, norm, entropy, total;
};

SplitSpace split_space(const bart_rows &r, int S, int k, bool grad) {
  SplitSpace w;
  auto up = [](size_t v) { return (v + 15) / 16 * 16; };
  w.part = 0;
  w.keys = w.part + up(sizeof(Stats) * r.n * S);
  w.norm = w.keys + up(sizeof(uint64_t) * r.n * S * k);
  w.entropy = w.norm + (grad ? up(sizeof(float) * 2 * r.n) : 0);
  w.total = w.entropy + (grad ? up(sizeof(float) * r.n) : 0);
  return w;
}

// Launches f(args, grid) over n rows, per_block rows and `pieces` workgroups at
// a time: a grid holds fewer than 2^32 threads.
template <class F>
void over_rows(RowsArgs A, int per_block, int block, int pieces, F f) {
  const int64_t most = std::max<int64_t>(1, ((int64_t)1 << 31) / block / pieces);  // row groups
  const int64_t groups = (A.r.n + per_block - 1) / per_block;
  for (int64_t g = 0; g < groups; g += most) {
    A.first = g * per_block;
    f(A, (unsigned)(std::min(most, groups - g) * pieces));
  }
}

template <int DT>
void launch_grad(const RowsArgs &A, const float *norm, const float *entropy, hipStream_t st) {
  if (const RowsLaunch L = grad_in_registers<DT>(A); L.fn) {
    over_rows(A, L.per_block, L.block, 1, [&](const RowsArgs &a, unsigned grid) {
      L.fn<<<grid, L.block, 0, st>>>(a, norm, entropy);
    });
    return;
  }
  constexpr int kPiece = 4 * 256 * Chunk<DT>::V;
  const int pieces = (int)((span_of(A.r) + kPiece - 1) / kPiece);
  over_rows(A, 1, 256, pieces, [&](const RowsArgs &a, unsigned grid) {
    k_grad_wide<DT><<<grid, 256, 0, st>>>(a, norm, entropy, pieces);
  });
}

template <int DT>
void launch_split(RowsArgs A, const Split &p, char *ws, hipStream_t st) {
  const SplitSpace w = split_space(A.r, p.S, A.o.k, A.g.grad);
  Stats *part = (Stats *)(ws + w.part);
  uint64_t *keys = (uint64_t *)(ws + w.keys);
  float *norm = A.g.grad ? (float *)(ws + w.norm) : nullptr;
  float *entropy = A.g.grad ? (float *)(ws + w.entropy) : nullptr;
  const int n = (int)A.r.n;
  k_rows_part<DT><<<n * p.S, 256, 0, st>>>(A, p.S, p.length, part, keys);
  k_rows_join<DT><<<n, 256, 0, st>>>(A, p.S, part, keys, norm, entropy);
  if (A.g.grad) launch_grad<DT>(A, norm, entropy, st);
}

template <int DT>
void launch_logprob(const RowsArgs &A, char *ws, hipStream_t st) {
  if (const Split p = split_of(A.r); p.S > 1) {
    launch_split<DT>(A, p, ws, st);
    return;
  }
  if (const RowsLaunch L = rows_in_registers<DT>(A); L.fn) {
    over_rows(A, L.per_block, L.block, 1, [&](const RowsArgs &a, unsigned grid) {
      L.fn<<<grid, L.block, 0, st>>>(a, nullptr, nullptr);
    });
    return;
  }
  // With a gradient, which reads again what is not held: fewer rows at once
  // keep more of each in the caches, against less overlap between rows.  us of
  // (lanes, held chunks), 16 bits: 8192 x 50001 (256, 0) 425, (512, 0) 376,
  // (512, 4) 361, (1024, 4) 376; 8192 x 65536 532, 464, 439, 422; 2048 x 131072
  // 305, 274, 268, 234; f32: 8192 x 40000 712, 623, 605, 542 and (1024, 8) 502.
  // Without one: 256 lanes, unless there are too few rows to fill the device
  // (131072 bf16 classes: 128 rows 16.2 us with 256 lanes, 12.2 with 512; 512
  // rows 22 and 25).
  const bool grad = A.g.grad, wide = A.r.n_class > (56 << 10);
  const int T = grad ? (DT == BART_F32 || wide ? 1024 : 512) : A.r.n <= 256 ? 512 : 256;
  over_rows(A, 1, T, 1, [&](const RowsArgs &a, unsigned grid) {
    if (!grad && T == 512)
      k_rows_stream<DT, 512, 0><<<grid, T, 0, st>>>(a);
    else if (!grad)
      k_rows_stream<DT, 256, 0><<<grid, T, 0, st>>>(a);
    else if constexpr (DT == BART_F32)
      k_rows_stream<DT, 1024, 8><<<grid, T, 0, st>>>(a);
    else if (wide)
      k_rows_stream<DT, 1024, 4><<<grid, T, 0, st>>>(a);
    else
      k_rows_stream<DT, 512, 4><<<grid, T, 0, st>>>(a);
  });
}

const char *check_logprob(const bart_rows *r, const bart_rows_out *o, const bart_rows_grad *g) {
  if (const char *e = check_rows(r)) return e;
  if (!o) return "out is NULL";
  if (o->k < 0 || o->k > BART_MAX_TOP) return "k must be in [0, 64]";
  if (((uintptr_t)o->logp | (uintptr_t)o->entropy | (uintptr_t)o->norm | (uintptr_t)o->top_logp |
       (uintptr_t)o->top_class) % 4)
    return "an output is not aligned to its elements";
  if (r->n == 0) return g ? check_grad(r, g) : nullptr;
  if (o->k > 0 && !o->top_logp && !o->top_class) return "k > 0 needs top_logp or top_class";
  if (o->logp && !r->label) return "logp needs labels";
  if (!o->logp && !o->entropy && !o->norm && !o->k && !g) return "nothing is asked for";
  return g ? check_grad(r, g) : nullptr;
}

// ------------------------------------------------------------------- AdamW

const char *check_tensors(const bart_adamw_tensor *t, int32_t n, int32_t bits) {
  if (!t) return "tensors is NULL";
  if (n < 1) return "n_tensors must be >= 1";
  if (bits != 32 && bits != 8) return "state_bits must be 32 or 8";
  for (int32_t i = 0; i < n; ++i) {
    const bart_adamw_tensor &q = t[i];
    if (q.n < 0 || q.n > ((int64_t)1 << 40)) return "a tensor's n must be in [0, 2^40]";
    if (!dtype_ok(q.param_dtype)) return "param_dtype must be BART_F32, BART_F16 or BART_BF16";
    if (q.grad_dtype != q.param_dtype && q.grad_dtype != BART_F32)
      return "grad_dtype must be param_dtype or BART_F32";
    if (q.master && q.param_dtype == BART_F32)
      return "a master copy stands beside 16-bit weights only";
    if (!std::isfinite(q.weight_decay)) return "weight_decay must be finite";
    if (!std::isfinite(q.lr_scale)) return "lr_scale must be finite";
    if (q.n == 0) continue;
    if (!q.param || !q.grad || !q.m || !q.v) return "a tensor has a NULL array";
    if (bits == 8 && (!q.m_scale || !q.v_scale)) return "8-bit states need their scales";
    if (bits == 32 && (q.m_scale || q.v_scale)) return "32-bit states have no scales";
    if ((uintptr_t)q.param % dtype_bytes(q.param_dtype) ||
        (uintptr_t)q.grad % dtype_bytes(q.grad_dtype) || (uintptr_t)q.master % 4 ||
        (uintptr_t)q.m_scale % 4 || (uintptr_t)q.v_scale % 4 ||
        (bits == 32 && ((uintptr_t)q.m | (uintptr_t)q.v) % 4))
      return "an array is not aligned to its elements";
  }
  return nullptr;
}

// Whether an array that one tensor's step writes shares memory with an array of
// another tensor.  (Two tensors may have one gradient.)
bool tensors_overlap(const bart_adamw_tensor *t, int32_t n, int32_t bits) {
  struct Range {
    uintptr_t from, to;
    int32_t tensor;
  };
  std::vector<Range> out, in;
  for (int32_t i = 0; i < n; ++i) {
    const bart_adamw_tensor &q = t[i];
    if (q.n == 0) continue;
    const int64_t state = bits == 32 ? 4 : 1, blocks = (q.n + kStateBlock - 1) / kStateBlock;
    auto add = [&](std::vector<Range> &to, const void *p, int64_t bytes) {
      if (p) to.push_back({(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes, i});
    };
    add(out, q.param, q.n * dtype_bytes(q.param_dtype));
    add(out, q.master, q.n * 4);
    add(out, q.m, q.n * state);
    add(out, q.v, q.n * state);
    add(out, q.m_scale, blocks * 4);
    add(out, q.v_scale, blocks * 4);
    add(in, q.grad, q.n * dtype_bytes(q.grad_dtype));
  }
  auto before = [](const Range &a, const Range &b) { return a.from < b.from; };
  std::sort(out.begin(), out.end(), before);
  std::vector<Range> parts;  // apart and in order; a tensor's own ones that touch are one
  for (const Range &r : out) {
    if (!parts.empty() && r.from < parts.back().to) {
      if (r.tensor != parts.back().tensor) return true;
      parts.back().to = std::max(parts.back().to, r.to);
    } else {
      parts.push_back(r);
    }
  }
  for (const Range &r : in) {
    auto p = std::upper_bound(parts.begin(), parts.end(), r, before);
    if (p != parts.begin() && std::prev(p)->to > r.from) --p;
    for (; p != parts.end() && p->from < r.to; ++p)
      if (p->tensor != r.tensor) return true;
  }
  return false;
}

// The kernels differ by the types of a tensor: tensors of equal types form a
// group, and a group is one launch.
int group_of(const bart_adamw_tensor &t) { return t.param_dtype * 2 + (t.grad_dtype != t.param_dtype); }
constexpr int kGroups = 6;

int64_t chunks_of(int64_t n) { return (n + kChunk - 1) / kChunk; }

size_t table_bytes(int32_t n_tensors) {
  return (n_tensors * sizeof(bart_adamw_tensor) + 15) / 16 * 16;
}

using AdamwFn = void (*)(const bart_adamw_tensor *, const AdamwChunk *, AdamwStep);

template <int BITS>
AdamwFn adamw_fn(int group) {
  switch (group) {
    case 0: return k_adamw<BART_F32, BART_F32, BITS>;
    case 2: return k_adamw<BART_F16, BART_F16, BITS>;
    case 3: return k_adamw<BART_F16, BART_F32, BITS>;
    case 4: return k_adamw<BART_BF16, BART_BF16, BITS>;
    case 5: return k_adamw<BART_BF16, BART_F32, BITS>;
  }
  return nullptr;
}

}  // namespace

struct bart_adamw {
  int device = 0;
  int32_t bits = 32;
  const bart_adamw_tensor *tensors = nullptr;  // device
  const AdamwChunk *chunks = nullptr;          // device, group by group
  int64_t first[kGroups + 1] = {};
};

extern "C" {

size_t bart_logprob_workspace_bytes(const bart_rows *r, const bart_rows_out *o,
                                    const bart_rows_grad *g) {
  if (check_logprob(r, o, g) || r->n == 0) return 0;
  const Split p = split_of(*r);
  return p.S > 1 ? split_space(*r, p.S, o->k, g != nullptr).total : 0;
}

int bart_logprob(const bart_rows *r, const bart_rows_out *o, const bart_rows_grad *g,
                 void *workspace, size_t ws_bytes, void *stream) {
  if (const char *e = check_logprob(r, o, g)) return fail(BART_EINVAL, "%s", e);
  if (r->n == 0) return BART_OK;
  if (const size_t need = bart_logprob_workspace_bytes(r, o, g)) {
    if (!workspace) return fail(BART_EINVAL, "workspace is NULL");
    if ((uintptr_t)workspace % 16) return fail(BART_ENOSPACE, "workspace must be 16-byte aligned");
    if (ws_bytes < need)
      return fail(BART_ENOSPACE, "workspace holds %zu bytes, %zu are needed", ws_bytes, need);
  }
  const RowsArgs A = rows_args(r, o, g);
  char *ws = (char *)workspace;
  switch (r->dtype) {
    case BART_F32: launch_logprob<BART_F32>(A, ws, (hipStream_t)stream); break;
    case BART_F16: launch_logprob<BART_F16>(A, ws, (hipStream_t)stream); break;
    default: launch_logprob<BART_BF16>(A, ws, (hipStream_t)stream);
  }
  HIP_TRY(hipGetLastError());
  return BART_OK;
}

int bart_logprob_grad(const bart_rows *r, const float *norm, const float *entropy,
                      const bart_rows_grad *g, void *stream) {
  if (const char *e = check_rows(r)) return fail(BART_EINVAL, "%s", e);
  if (!g) return fail(BART_EINVAL, "grad is NULL");
  if (const char *e = check_grad(r, g)) return fail(BART_EINVAL, "%s", e);
  if (r->n == 0) return BART_OK;
  if (!norm) return fail(BART_EINVAL, "norm is NULL");
  if (g->w_entropy && !entropy) return fail(BART_EINVAL, "w_entropy needs the entropies");
  if (((uintptr_t)norm | (uintptr_t)entropy) % 4)
    return fail(BART_EINVAL, "norm or entropy is not aligned to its elements");
  const RowsArgs A = rows_args(r, nullptr, g);
  switch (r->dtype) {
    case BART_F32: launch_grad<BART_F32>(A, norm, entropy, (hipStream_t)stream); break;
    case BART_F16: launch_grad<BART_F16>(A, norm, entropy, (hipStream_t)stream); break;
    default: launch_grad<BART_BF16>(A, norm, entropy, (hipStream_t)stream);
  }
  HIP_TRY(hipGetLastError());
  return BART_OK;
}

size_t bart_adamw_workspace_bytes(const bart_adamw_tensor *t, int32_t n_tensors,
                                  int32_t state_bits) {
  if (check_tensors(t, n_tensors, state_bits)) return 0;
  int64_t chunks = 0;
  for (int32_t i = 0; i < n_tensors; ++i) chunks += chunks_of(t[i].n);
  return table_bytes(n_tensors) + std::max<int64_t>(chunks, 1) * sizeof(AdamwChunk);
}

int bart_adamw_init(const bart_adamw_tensor *t, int32_t n_tensors, int32_t state_bits,
                    void *workspace, size_t ws_bytes, void *stream, bart_adamw **out) {
  if (!out) return fail(BART_EINVAL, "out is NULL");
  *out = nullptr;
  if (const char *e = check_tensors(t, n_tensors, state_bits)) return fail(BART_EINVAL, "%s", e);
  if (!workspace) return fail(BART_EINVAL, "workspace is NULL");
  bart_adamw *h = nullptr;
  try {
    if (tensors_overlap(t, n_tensors, state_bits))
      return fail(BART_EINVAL, "arrays of different tensors overlap");
    if ((uintptr_t)workspace % 16) return fail(BART_ENOSPACE, "workspace must be 16-byte aligned");
    const size_t need = bart_adamw_workspace_bytes(t, n_tensors, state_bits);
    if (ws_bytes < need)
      return fail(BART_ENOSPACE, "workspace holds %zu bytes, %zu are needed", ws_bytes, need);
    h = new bart_adamw;
    std::vector<AdamwChunk> chunks;
    chunks.reserve((need - table_bytes(n_tensors)) / sizeof(AdamwChunk));
    for (int g = 0; g < kGroups; ++g) {
      for (int32_t i = 0; i < n_tensors; ++i)
        if (group_of(t[i]) == g)
          for (int64_t c = 0; c < chunks_of(t[i].n); ++c) chunks.push_back({i, (int32_t)c});
      h->first[g + 1] = (int64_t)chunks.size();
    }
    h->bits = state_bits;
    h->tensors = (const bart_adamw_tensor *)workspace;
    h->chunks = (const AdamwChunk *)((char *)workspace + table_bytes(n_tensors));
    const int rc = [&]() -> int {
      hipStream_t st = (hipStream_t)stream;
      HIP_TRY(hipGetDevice(&h->device));
      HIP_TRY(hipMemcpyAsync(workspace, t, n_tensors * sizeof *t, hipMemcpyHostToDevice, st));
      if (!chunks.empty())
        HIP_TRY(hipMemcpyAsync((void *)h->chunks, chunks.data(), chunks.size() * sizeof(AdamwChunk),
                               hipMemcpyHostToDevice, st));
      // the host tables must stay valid until the copies ran
      HIP_TRY(hipStreamSynchronize(st));
      return BART_OK;
    }();
    if (rc) {
      delete h;
      return rc;
    }
  } catch (const std::exception &e) {
    delete h;
    return fail(BART_ENOSPACE, "no host memory for the plan: %s", e.what());
  }
  *out = h;
  return BART_OK;
}

int bart_adamw_step(bart_adamw *h, const bart_adamw_hyper *y, void *stream) {
  if (!h) return fail(BART_EINVAL, "plan is NULL");
  if (!y) return fail(BART_EINVAL, "hyper is NULL");
  if (!std::isfinite((float)y->lr)) return fail(BART_EINVAL, "lr must be finite in 32 bits");
  if (!(y->beta1 >= 0.0 && y->beta1 < 1.0 && y->beta2 >= 0.0 && y->beta2 < 1.0))
    return fail(BART_EINVAL, "betas must be in [0, 1)");
  if (!(y->eps >= 1e-37 && std::isfinite(y->eps))) return fail(BART_EINVAL, "eps must be >= 1e-37");
  if (!std::isfinite((float)y->grad_scale))
    return fail(BART_EINVAL, "grad_scale must be finite in 32 bits");
  if (y->step < 1) return fail(BART_EINVAL, "step must be >= 1");
  OnDevice here;
  HIP_TRY(here.enter(h->device));
  AdamwStep K;
  K.b1 = (float)y->beta1;
  K.c1 = (float)(1.0 - y->beta1);
  K.b2 = (float)y->beta2;
  K.c2 = (float)(1.0 - y->beta2);
  K.eps = (float)y->eps;
  K.grad_scale = (float)y->grad_scale;
  K.root = (float)(1.0 / std::sqrt(1.0 - std::pow(y->beta2, (double)y->step)));
  K.lr = y->lr;
  K.first = 1.0 / (1.0 - std::pow(y->beta1, (double)y->step));
  K.dither = (uint32_t)((uint64_t)y->step * 0x91E10DA5u);
  for (int g = 0; g < kGroups; ++g) {
    const int64_t a = h->first[g], b = h->first[g + 1];
    // a grid holds fewer than 2^32 threads
    for (int64_t c = a; c < b; c += 1 << 23) {
      const int grid = (int)std::min<int64_t>(b - c, 1 << 23);
      AdamwFn fn = h->bits == 32 ? adamw_fn<32>(g) : adamw_fn<8>(g);
      fn<<<grid, 256, 0, (hipStream_t)stream>>>(h->tensors, h->chunks + c, K);
      HIP_TRY(hipGetLastError());
    }
  }
  return BART_OK;
}

void bart_adamw_destroy(bart_adamw *h) { delete h; }

}  // extern "C"
