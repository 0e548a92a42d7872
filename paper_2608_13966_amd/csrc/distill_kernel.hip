// distill_kernel.hip -- the loss against a teacher's top logits and its
// gradient (quasar_ops.h).
//
// The listed classes of a row are few: every workgroup that works on a row
// takes them into LDS and normalises the teacher's side itself.  The student's
// row is what costs: it is read for lse as a running maximum and a sum of
// exponentials (rescaled when the maximum grows), and for the gradient again.
#include "ops_common.h"
#include "ops_internal.h"

namespace quasar {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kListed = QUASAR_DISTILL_MAX_LISTED;

// max and sum of exp2((z - max) c) of a set of logits; an empty set is (-inf, 0)
struct MaxSum {
  float m, s;
};
// -inf - -inf would be NaN: two sets of -inf have their sums at exponent 0
__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b, float c) {
  const float m = fmaxf(a.m, b.m);
  // a NaN of either sum stays; a NaN logit has made its sum NaN
  const float fa = a.m == m ? 1.0f : __builtin_amdgcn_exp2f((a.m - m) * c);
  const float fb = b.m == m ? 1.0f : __builtin_amdgcn_exp2f((b.m - m) * c);
  return MaxSum{m, a.s * fa + b.s * fb};
}

struct Listed {
  int index[kListed];   // -1: no entry
  float p[kListed];     // the teacher's probability
};

// Loads row `row`'s list; the teacher's probabilities are in l.p after the
// call (a barrier ends it).  False: no entry has p > 0, or row_weight is 0.
// plogp: sum of p log p.
__device__ bool load_listed(const quasar_distill& a, int64_t row, Listed& l, float* red, float& plogp) {
  const int K = a.listed;
  const float it = 1.0f / a.temperature;
  if (a.row_weight && a.row_weight[row] == 0.0f) return false;
  float m = -INFINITY;
  bool nan = false;
  for (int k = threadIdx.x; k < K; k += kThreads) {
    const int64_t e = row * K + k;
    const int64_t ix = a.index_bits == 64 ? reinterpret_cast<const int64_t*>(a.index)[e]
                                          : (int64_t) reinterpret_cast<const int32_t*>(a.index)[e];
    const bool ok = ix >= 0 && ix < a.classes;
    const float t = ok ? elem(a.teacher, e, a.teacher_dtype == QUASAR_BF16) * it : -INFINITY;
    l.index[k] = ok ? (int)ix : -1;
    l.p[k] = t;
    m = fmaxf(m, t);
    nan |= t != t;
  }
  m = group_reduce<kWaves>(m, red, MaxOp());
  const bool any_nan = __syncthreads_or(nan);
  if (m == -INFINITY && !any_nan) return false;
  float s = 0.0f;
  for (int k = threadIdx.x; k < K; k += kThreads) s += __builtin_amdgcn_exp2f((l.p[k] - m) * kLog2e);
  s = group_reduce<kWaves>(s, red + kWaves, SumOp());
  const float ls = __logf(s), is = 1.0f / s;
  float h = 0.0f;
  for (int k = threadIdx.x; k < K; k += kThreads) {
    const float t = l.p[k] - m, p = __builtin_amdgcn_exp2f(t * kLog2e) * is;
    l.p[k] = p;
    if (!(p == 0.0f)) h += p * (t - ls);
  }
  plogp = group_reduce<kWaves>(h, red + 2 * kWaves, SumOp());
  return true;
}

// max and sum over the elements [e0, e1) of a row (base: the row's first element)
template <int T>
__device__ MaxSum scan(const void* z, int64_t base, int e0, int e1, float c) {
  MaxSum r{-INFINITY, 0.0f};
  for (int e = e0 + (int)threadIdx.x * 8; e < e1; e += kThreads * 8) {
    Piece<T> p;
    p.load(z, base + e, e1 - e, 0xff80);  // -inf past the end
    float m = r.m;
#pragma unroll
    for (int i = 0; i < 8; i++) m = fmaxf(m, p.get(i));
    if (m == -INFINITY) {  // nothing but -inf so far: no exponent to take, but a NaN among them stays
#pragma unroll
      for (int i = 0; i < 8; i++) r.s += p.get(i) != p.get(i) ? p.get(i) : 0.0f;
      continue;
    }
    if (m != r.m) {
      r.s *= r.m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((r.m - m) * c);
      r.m = m;
    }
#pragma unroll
    for (int i = 0; i < 8; i++) r.s += __builtin_amdgcn_exp2f((p.get(i) - m) * c);
  }
  return r;
}

__device__ __forceinline__ MaxSum group_join(MaxSum r, float c, MaxSum* s) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const MaxSum b{__shfl_xor(r.m, o, 64), __shfl_xor(r.s, o, 64)};
    r = join(r, b, c);
  }
  if ((threadIdx.x & 63) == 0) s[wave_index()] = r;
  __syncthreads();
  r = s[0];
#pragma unroll
  for (int i = 1; i < kWaves; i++) r = join(r, s[i], c);
  return r;
}

__device__ __forceinline__ float lse_of(MaxSum r, float it) { return r.m * it + __logf(r.s); }

// Workgroup b works on part b % parts of row b / parts.
// Partial maximum and sum of one part of a row, into part[b].
template <int T>
__global__ __launch_bounds__(kThreads) void distill_scan_kernel(quasar_distill a, int per, int parts, MaxSum* part) {
  __shared__ MaxSum s[kWaves];
  const int row = blockIdx.x / (unsigned)parts, at = blockIdx.x % (unsigned)parts;
  const float c = kLog2e / a.temperature;
  const int e0 = at * per, V = (int)a.classes, e1 = e0 + per < V ? e0 + per : V;
  const MaxSum r = group_join(scan<T>(a.logits, row * a.logits_stride, e0, e1, c), c, s);
  if (threadIdx.x == 0) part[blockIdx.x] = r;
}

// One part of a row's gradient, and (part 0) its loss and lse.  lse is joined
// from the row's `sums` partial ones, or (0) taken from a.lse.
template <int T>
__global__ __launch_bounds__(kThreads) void distill_row_kernel(quasar_distill a, int what, int per, int parts,
                                                               const MaxSum* part, int sums) {
  __shared__ Listed l;
  __shared__ float red[4 * kWaves];
  const int64_t row = blockIdx.x / (unsigned)parts, base = row * a.logits_stride, gbase = row * a.grad_stride;
  const int at = blockIdx.x % (unsigned)parts;
  const float it = 1.0f / a.temperature, c = kLog2e / a.temperature;
  const int V = (int)a.classes;
  const int e0 = at * per, e1 = e0 + per < V ? e0 + per : V;
  float plogp = 0.0f;
  const bool live = load_listed(a, row, l, red, plogp);
  if (!live) {
    if (what != 1 && at == 0 && threadIdx.x == 0) a.loss[row] = a.lse[row] = 0.0f;
    if (what == 0) return;
    const float zero[8] = {};
    for (int e = e0 + (int)threadIdx.x * 8; e < e1; e += kThreads * 8)
      store_piece<T == kElemBF16>(a.grad, gbase + e, zero, e1 - e);
    return;
  }
  const float weight = a.row_weight ? a.row_weight[row] : 1.0f;
  float lse;
  if (sums > 0) {
    MaxSum r = part[row * sums];
    for (int i = 1; i < sums; i++) r = join(r, part[row * sums + i], c);
    lse = lse_of(r, it);
  } else {
    lse = a.lse[row];
  }
  if (what != 1 && at == 0) {
    float s = 0.0f;
    for (int k = threadIdx.x; k < a.listed; k += kThreads)
      if (l.index[k] >= 0 && !(l.p[k] == 0.0f))
        s += l.p[k] * (lse - elem(a.logits, base + l.index[k], T == kElemBF16) * it);
    s = group_reduce<kWaves>(s, red + 3 * kWaves, SumOp());
    if (threadIdx.x == 0) {
      a.loss[row] = weight * (plogp + s);
      a.lse[row] = lse;
    }
  }
  if (what == 0) return;
  const float g = (a.grad_loss ? a.grad_loss[row] : a.grad_scale) * weight * it;
  const float off = lse * kLog2e;
  // the listed classes' gradients, from their logits before `grad` may overwrite them
  constexpr int kPer = kListed / kThreads;
  float mine[kPer];
#pragma unroll
  for (int j = 0; j < kPer; j++) {
    const int k = threadIdx.x + j * kThreads;
    mine[j] = 0.0f;
    if (k >= a.listed) continue;
    const int ix = l.index[k];
    if (ix < e0 || ix >= e1) continue;
    float p = 0.0f;
    for (int i = 0; i < a.listed; i++) p += l.index[i] == ix ? l.p[i] : 0.0f;
    mine[j] = g * (__builtin_amdgcn_exp2f(elem(a.logits, base + ix, T == kElemBF16) * c - off) - p);
  }
  __syncthreads();
  for (int e = e0 + (int)threadIdx.x * 8; e < e1; e += kThreads * 8) {
    Piece<T> p;
    p.load(a.logits, base + e, e1 - e);
    float d[8];
#pragma unroll
    for (int i = 0; i < 8; i++) d[i] = g * __builtin_amdgcn_exp2f(__builtin_fmaf(p.get(i), c, -off));
    store_piece<T == kElemBF16>(a.grad, gbase + e, d, e1 - e);
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kPer; j++) {
    const int k = threadIdx.x + j * kThreads;
    if (k >= a.listed) continue;
    const int ix = l.index[k];
    if (ix >= e0 && ix < e1) put_elem(a.grad, gbase + ix, mine[j], T == kElemBF16);
  }
}

constexpr int kPart = 16384;  // classes a workgroup takes

int parts_of(int64_t classes) { return (int)((classes + kPart - 1) / kPart); }

}  // namespace

size_t distill_workspace(int64_t rows, int64_t classes) { return (size_t)rows * parts_of(classes) * sizeof(MaxSum); }

hipError_t launch_distill(const quasar_distill& a, int what, hipStream_t stream) {
  const int parts = parts_of(a.classes);
  const unsigned blocks = (unsigned)(a.rows * parts);
  MaxSum* ws = reinterpret_cast<MaxSum*>(a.workspace);
  const bool bf16 = a.logits_dtype == QUASAR_BF16;
  const auto row_kernel = [&](int w, int n, int sums) {
    if (bf16)
      distill_row_kernel<kElemBF16><<<dim3((unsigned)(a.rows * n)), dim3(kThreads), 0, stream>>>(
          a, w, n == 1 ? (int)a.classes : kPart, n, ws, sums);
    else
      distill_row_kernel<kElemF32><<<dim3((unsigned)(a.rows * n)), dim3(kThreads), 0, stream>>>(
          a, w, n == 1 ? (int)a.classes : kPart, n, ws, sums);
    return hipGetLastError();
  };
  if (what != 1) {
    if (bf16)
      distill_scan_kernel<kElemBF16><<<dim3(blocks), dim3(kThreads), 0, stream>>>(a, kPart, parts, ws);
    else
      distill_scan_kernel<kElemF32><<<dim3(blocks), dim3(kThreads), 0, stream>>>(a, kPart, parts, ws);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    // in place, the loss is taken before another part's gradient overwrites a listed logit
    if (what == 2 && parts > 1 && a.grad == a.logits) {
      e = row_kernel(0, 1, parts);
      return e != hipSuccess ? e : row_kernel(1, parts, 0);
    }
  }
  return what == 1 ? row_kernel(1, parts, 0) : row_kernel(what, what == 0 ? 1 : parts, parts);
}

}  // namespace quasar
