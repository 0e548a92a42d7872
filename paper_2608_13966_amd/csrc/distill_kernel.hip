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
constexpr int kMostPart = 16384;

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

// The probability of class ix: all entries of it.
__device__ __forceinline__ float listed_p(const Listed& l, int K, int ix) {
  float p = 0.0f;
#pragma unroll 4
  for (int i = 0; i < K; i++)
    if (l.index[i] == ix) p += l.p[i];
  return p;
}

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

// r joined with eight more logits
template <int T>
__device__ __forceinline__ void take(MaxSum& r, const Piece<T>& p, float c) {
  float m = r.m;
#pragma unroll
  for (int i = 0; i < 8; i++) m = fmaxf(m, p.get(i));
  if (m == -INFINITY) {  // nothing but -inf so far: no exponent to take, but a NaN among them stays
#pragma unroll
    for (int i = 0; i < 8; i++) r.s += p.get(i) != p.get(i) ? p.get(i) : 0.0f;
    return;
  }
  if (m != r.m) {
    r.s *= r.m == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f((r.m - m) * c);
    r.m = m;
  }
  float e[8];
#pragma unroll
  for (int i = 0; i < 8; i++) e[i] = __builtin_amdgcn_exp2f((p.get(i) - m) * c);
  r.s += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
}

// max and sum over the elements [e0, e1) of a row (base: the row's first element)
template <int T>
__device__ MaxSum scan(const void* z, int64_t base, int e0, int e1, float c) {
  MaxSum r{-INFINITY, 0.0f};
  for (int e = e0 + (int)threadIdx.x * 8; e < e1; e += kThreads * 8) {
    Piece<T> p;
    p.load(z, base + e, e1 - e, 0xff80);  // -inf past the end
    take(r, p, c);
  }
  return r;
}

template <int WAVES = kWaves>
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
  for (int i = 1; i < WAVES; i++) r = join(r, s[i], c);
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
  // the student's probability; z / tau and lse may be large, their difference is taken first
  const auto soft = [&](float z) { return __builtin_amdgcn_exp2f(__builtin_fmaf(z, it, -lse) * kLog2e); };
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
    mine[j] = g * (soft(elem(a.logits, base + ix, T == kElemBF16)) - listed_p(l, a.listed, ix));
  }
  __syncthreads();
  for (int e = e0 + (int)threadIdx.x * 8; e < e1; e += kThreads * 8) {
    Piece<T> p;
    p.load(a.logits, base + e, e1 - e);
    float d[8];
#pragma unroll
    for (int i = 0; i < 8; i++) d[i] = g * soft(p.get(i));
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

// ---- a row in registers ---------------------------------------------------------
// One workgroup takes whole rows, NV pieces of eight classes a thread, which stay
// in registers from their only read to the gradient; each piece's registers take
// the next row's as soon as its gradient is stored (without a gradient: as soon
// as it is summed), so loads and stores overlap.  The lists are a row ahead too,
// their entries' loads before the row's (loads return in order: an entry asked
// for after them would come after them, and hold the first wavefront up).
// WHAT: 0 the loss, 1 the gradient from a.lse, 2 both.
template <int T, int NT, int NV, int WHAT>
__global__ __launch_bounds__(NT) void distill_resident_kernel(quasar_distill a) {
  constexpr bool GRAD = WHAT != 0, SUM = WHAT != 1;
  constexpr int kPer = kListed / NT;  // entries a thread fetches
  struct Row {  // of rows in turn
    Listed l;
    float z[kListed];
    MaxSum s[NT / 64];
    float plogp;
    int live;
  };
  __shared__ Row rows[2];
  const int tid = threadIdx.x, lane = tid & 63, V = (int)a.classes, K = a.listed;
  const float it = 1.0f / a.temperature, c = kLog2e / a.temperature;
  Piece<T> pc[NV];
  // pieces are whole (all lanes' where the row goes that far); the row's last V % 8 classes are one a thread
  const auto whole = [&](int v) { return (v + 1) * NT * 8 <= V || (v * NT + tid + 1) * 8 <= V; };
  const auto load = [&](int v, int64_t row) {
    pc[v].load(a.logits, row * a.logits_stride + (v * NT + tid) * 8, whole(v) ? 8 : 0, 0xff80);
  };
  const int rest = (V & ~7) + tid;
  float last = -INFINITY;
  const auto load_last = [&](int64_t row) {
    if (rest < V) last = elem(a.logits, row * a.logits_stride + rest, T == kElemBF16);
  };
  // the list of a row: entries, then (in LDS, with the teacher's logits / tau) their logits
  int64_t ix[kPer];
  float te[kPer], ze[kPer];
  const auto load_list = [&](int64_t row) {
#pragma unroll
    for (int j = 0; j < kPer; j++) {
      const int k = tid + j * NT;
      const int64_t e = row * K + k;
      if (k < K) {
        ix[j] = a.index_bits == 64 ? reinterpret_cast<const int64_t*>(a.index)[e]
                                   : (int64_t) reinterpret_cast<const int32_t*>(a.index)[e];
        te[j] = elem(a.teacher, e, a.teacher_dtype == QUASAR_BF16);
      }
    }
  };
  const auto put_list = [&](Row& o, int64_t row) {
#pragma unroll
    for (int j = 0; j < kPer; j++) {
      const int k = tid + j * NT;
      if (k < K) {
        const bool ok = ix[j] >= 0 && ix[j] < V;
        o.l.index[k] = ok ? (int)ix[j] : -1;
        o.l.p[k] = ok ? te[j] * it : -INFINITY;
        ze[j] = elem(a.logits, row * a.logits_stride + (ok ? ix[j] : 0), T == kElemBF16);
      }
    }
  };
  const auto put_logits = [&](Row& o) {
#pragma unroll
    for (int j = 0; j < kPer; j++)
      if (tid + j * NT < K) o.z[tid + j * NT] = ze[j];
  };
  if (blockIdx.x < a.rows) {
    load_list(blockIdx.x);
#pragma unroll
    for (int v = 0; v < NV; v++) load(v, blockIdx.x);
    load_last(blockIdx.x);
    put_list(rows[0], blockIdx.x);
    put_logits(rows[0]);
  }
  __syncthreads();
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    Row &o = rows[turn], &n = rows[turn ^ 1];
    const int64_t next = row + gridDim.x;
    const float weight = a.row_weight ? a.row_weight[row] : 1.0f;
    if (next < a.rows) load_list(next);
    float lse = SUM ? 0.0f : a.lse[row];
    MaxSum r{-INFINITY, 0.0f};
    if constexpr (SUM) {
#pragma unroll
      for (int v = 0; v < NV; v++) {
        take(r, pc[v], c);
        if (!GRAD && next < a.rows) load(v, next);
      }
    }
    if (SUM && rest < V) r = join(r, last == -INFINITY ? MaxSum{last, 0.0f} : MaxSum{last, last == last ? 1.0f : last}, c);
    if (!GRAD && next < a.rows) load_last(next);
    if (tid < 64) {
      float m = -INFINITY, s = 0.0f, h = 0.0f;
      bool nan = false;
      for (int k = lane; k < K; k += 64) {
        m = fmaxf(m, o.l.p[k]);
        nan |= o.l.p[k] != o.l.p[k];
      }
      m = wave_reduce(m, MaxOp());
      const bool live = weight != 0.0f && (m != -INFINITY || __ballot(nan) != 0);
      if (live) {
        for (int k = lane; k < K; k += 64) s += __builtin_amdgcn_exp2f((o.l.p[k] - m) * kLog2e);
        s = wave_reduce(s, SumOp());
        const float ls = __logf(s), is = 1.0f / s;
        for (int k = lane; k < K; k += 64) {
          const float t = o.l.p[k] - m, p = __builtin_amdgcn_exp2f(t * kLog2e) * is;
          o.l.p[k] = p;
          if (!(p == 0.0f)) h += p * (t - ls);
        }
        h = wave_reduce(h, SumOp());
      }
      if (lane == 0) {
        o.plogp = h;
        o.live = live;
      }
    }
    if constexpr (SUM) {
      r = group_join<NT / 64>(r, c, o.s);  // its barrier shows the list too
      lse = lse_of(r, it);
    } else {
      __syncthreads();
    }
    const bool live = o.live;
    if (SUM && tid < 64) {
      float s = 0.0f;
      if (live)
        for (int k = lane; k < K; k += 64)
          if (o.l.index[k] >= 0 && !(o.l.p[k] == 0.0f)) s += o.l.p[k] * (lse - o.z[k] * it);
      s = wave_reduce(s, SumOp());
      if (lane == 0) {
        a.loss[row] = live ? weight * (o.plogp + s) : 0.0f;
        a.lse[row] = live ? lse : 0.0f;
      }
    }
    if (next < a.rows) put_list(n, next);
    if constexpr (GRAD) {
      const int64_t gbase = row * a.grad_stride;
      const float g = (!SUM && a.grad_loss ? a.grad_loss[row] : a.grad_scale) * weight * it;
      const float ls = SUM ? __builtin_amdgcn_logf(r.s) : 0.0f;
      // the student's probability; the logits and lse may be large, their difference is taken first
      const auto soft = [&](float z) {
        return __builtin_amdgcn_exp2f(SUM ? __builtin_fmaf(z - r.m, c, -ls) : __builtin_fmaf(z, it, -lse) * kLog2e);
      };
#pragma unroll
      for (int v = 0; v < NV; v++) {
        float d[8];
        pc[v].refresh();
#pragma unroll
        for (int i = 0; i < 8; i++) d[i] = soft(pc[v].get(i));
#pragma unroll
        for (int i = 0; i < 8; i++) d[i] = live ? g * d[i] : 0.0f;
        if (whole(v)) store_piece<T == kElemBF16>(a.grad, gbase + (v * NT + tid) * 8, d, 8);
        if (next < a.rows) load(v, next);
      }
      if (rest < V) put_elem(a.grad, gbase + rest, live ? g * soft(last) : 0.0f, T == kElemBF16);
      if (next < a.rows) load_last(next);
      __syncthreads();  // the listed classes' gradients over the others'
      if (live) {
        for (int k = tid; k < K; k += NT) {
          const int at = o.l.index[k];
          if (at >= 0)
            put_elem(a.grad, gbase + at, g * (soft(o.z[k]) - listed_p(o.l, K, at)), T == kElemBF16);
        }
      }
      if (next < a.rows) put_logits(n);
    } else {
      if (next < a.rows) put_logits(n);
      __syncthreads();
    }
  }
}

// The split form: classes a workgroup takes, so that about four run on a CU,
// 2048 at least (a piece of eight a thread) and 16384 at most.
int part_of(int64_t rows, int64_t classes) {
  const int64_t want = rows >= 4096 ? kMostPart : rows * classes / (4 * kCUs);
  return (int)(want <= 2048 ? 2048 : want >= kMostPart ? kMostPart : (want + 2047) / 2048 * 2048);
}
int parts_of(int64_t rows, int64_t classes) {
  const int per = part_of(rows, classes);
  return (int)((classes + per - 1) / per);
}

// The pieces a thread holds, 64 registers of them at the most.
template <int T>
constexpr int kMostPieces = T == kElemBF16 ? 16 : 8;

bool resident(int64_t rows, int64_t classes, bool bf16) {
  const int64_t most = 1024 * 8 * (bf16 ? kMostPieces<kElemBF16> : kMostPieces<kElemF32>);
  return classes <= most && (rows >= kCUs || classes <= kMostPart);
}

template <int T, int WHAT>
hipError_t launch_resident(const quasar_distill& a, hipStream_t stream) {
#define QUASAR_RESIDENT(NT, NV)                                                                     \
  if (a.classes <= (NT) * 8 * (NV)) {                                                               \
    const int64_t most = (int64_t)kCUs * (1024 / (NT));                                             \
    distill_resident_kernel<T, NT, NV, WHAT>                                                        \
        <<<dim3((unsigned)(a.rows < most ? a.rows : most)), dim3(NT), 0, stream>>>(a);              \
    return hipGetLastError();                                                                       \
  }
  constexpr int P = kMostPieces<T>;
  QUASAR_RESIDENT(256, 2)
  QUASAR_RESIDENT(256, P / 2)
  QUASAR_RESIDENT(256, P)
  QUASAR_RESIDENT(512, P)
  QUASAR_RESIDENT(1024, P * 3 / 4)
  QUASAR_RESIDENT(1024, P)
#undef QUASAR_RESIDENT
  return hipErrorInvalidValue;
}

}  // namespace

size_t distill_workspace(int64_t rows, int64_t classes) {
  return (size_t)rows * parts_of(rows, classes) * sizeof(MaxSum);
}

hipError_t launch_distill(const quasar_distill& a, int what, hipStream_t stream) {
  const bool bf16 = a.logits_dtype == QUASAR_BF16;
  if (resident(a.rows, a.classes, bf16)) {
    if (bf16)
      return what == 0   ? launch_resident<kElemBF16, 0>(a, stream)
             : what == 1 ? launch_resident<kElemBF16, 1>(a, stream)
                         : launch_resident<kElemBF16, 2>(a, stream);
    return what == 0   ? launch_resident<kElemF32, 0>(a, stream)
           : what == 1 ? launch_resident<kElemF32, 1>(a, stream)
                       : launch_resident<kElemF32, 2>(a, stream);
  }
  const int parts = parts_of(a.rows, a.classes), per = part_of(a.rows, a.classes);
  MaxSum* ws = reinterpret_cast<MaxSum*>(a.workspace);
  const auto row_kernel = [&](int w, int n, int sums) {
    const dim3 grid((unsigned)(a.rows * n)), block(kThreads);
    const int each = n == 1 ? (int)a.classes : per;
    if (bf16)
      distill_row_kernel<kElemBF16><<<grid, block, 0, stream>>>(a, w, each, n, ws, sums);
    else
      distill_row_kernel<kElemF32><<<grid, block, 0, stream>>>(a, w, each, n, ws, sums);
    return hipGetLastError();
  };
  if (what != 1) {
    const dim3 grid((unsigned)(a.rows * parts)), block(kThreads);
    if (bf16)
      distill_scan_kernel<kElemBF16><<<grid, block, 0, stream>>>(a, per, parts, ws);
    else
      distill_scan_kernel<kElemF32><<<grid, block, 0, stream>>>(a, per, parts, ws);
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
