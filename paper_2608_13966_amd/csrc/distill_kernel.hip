// distill_kernel.hip -- the loss against a teacher's top logits and its
// gradient (quasar_ops.h).
//
// The listed classes of a row are few: one wavefront of every workgroup that
// works on a row takes them into LDS and normalises the teacher's side.  The
// student's row is what costs: it is read for lse as a running maximum and a sum
// of exponentials (rescaled when the maximum grows), and needed for the gradient
// again: a row that fits one workgroup's registers stays there (resident
// kernel), others, and rows too few to fill the CUs, go in parts twice.
//
// Bound by memory: bf16, 64 listed, loss and gradient of 4096 x 131072 469 us, 4.6
// TB/s (a copy of 4 GiB: 4.8); the gradient alone of 4096 x 32000 100 us, 5.3 TB/s.
// In parts the row is read twice: loss and gradient of 4096 x 151936 677 us (481 at
// the copy's rate).  Few rows are latency: 48 x 50021 in fp32 4.1 + 7.4 us.
#include "ops_common.h"
#include "ops_internal.h"

namespace quasar {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kListed = QUASAR_DISTILL_MAX_LISTED;
constexpr int kListedWave = 256;  // where one wavefront takes a row

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

// A row's list in LDS, K entries.
//
// The gradient of a class takes the probabilities of all its entries, but few
// lists name a class twice.  `seen` tells: a hash table of the classes (open
// addressing, at most half full), each with kTwice once a second entry has come
// to it.  Only those classes look through the list (all of them doing so took
// 10 us of a row of 197 entries); the sum is in the list's order either way.
struct RowList {
  static constexpr uint32_t kNone = 0xffffffffu, kTwice = 0x80000000u;
  struct One {
    int index;  // -1: no entry
    float p;    // the teacher's probability
    float z;    // the student's logit
    int slot;   // in seen
  };
  One* e;
  float* logp;     // the logarithms of the entries' p
  uint32_t* seen;  // 2^bits slots
  float* some;     // whether the row is not masked (row_weight 0, or no entry with p > 0)
  int bits;

  static __host__ __device__ __forceinline__ int bits_of(int K) {
    int b = 5;
    while ((1 << b) < 2 * K) b++;
    return b;
  }
  // floats of LDS, in whole entries
  static __host__ __device__ __forceinline__ int size(int K) { return ((5 * K + 3) & ~3) + (1 << bits_of(K)) + 4; }
  __device__ __forceinline__ RowList(float* lds, int K)
      : e(reinterpret_cast<One*>(lds)),
        logp(lds + 4 * K),
        seen(reinterpret_cast<uint32_t*>(lds + ((5 * K + 3) & ~3))),
        some(lds + size(K) - 4),
        bits(bits_of(K)) {}

  __device__ __forceinline__ bool live() const { return *some != 0.0f; }
  // a barrier between clear(), note() and probability()
  template <int NT>
  __device__ __forceinline__ void clear() const {
    for (int i = threadIdx.x; i < 1 << bits; i += NT) seen[i] = kNone;
  }
  __device__ __forceinline__ void note(int k) const {
    const uint32_t ix = (uint32_t)e[k].index;
    for (uint32_t i = ix * 0x9e3779b1u >> (32 - bits);; i = (i + 1) & ((1u << bits) - 1u)) {
      const uint32_t had = atomicCAS(&seen[i], kNone, ix);
      if (had == kNone || (had & ~kTwice) == ix) {
        if (had != kNone) atomicOr(&seen[i], kTwice);
        e[k].slot = (int)i;
        return;
      }
    }
  }
  // of the class of entry k, which has been noted
  __device__ __forceinline__ float probability(int k, int K) const {
    if (!(seen[e[k].slot] & kTwice)) return e[k].p;
    const int ix = e[k].index;
    float sum = 0.0f;
    for (int j = 0; j < K; j++)
      if (e[j].index == ix) sum += e[j].p;
    return sum;
  }
};
// Entry k of a row's list as it lies in memory: the same loads for either type
// of index and of teacher, without a branch.
struct Entry {
  int32_t lo, hi;
  uint16_t top, low;
  __device__ __forceinline__ Entry() {}
  __device__ __forceinline__ Entry(const quasar_distill& a, int64_t row, int k) {
    const int64_t e = row * a.listed + k;
    const bool wide = a.index_bits == 64, tb = a.teacher_dtype == QUASAR_BF16;
    const int32_t* const i = reinterpret_cast<const int32_t*>(a.index) + (wide ? 2 * e : e);
    lo = i[0];
    hi = i[wide ? 1 : 0];
    const uint16_t* const t = reinterpret_cast<const uint16_t*>(a.teacher) + (tb ? e : 2 * e);
    top = t[tb ? 0 : 1];
    low = t[0];
  }
  // the class, or -1
  __device__ __forceinline__ int at(const quasar_distill& a) const {
    return lo >= 0 && lo < (int)a.classes && (a.index_bits == 32 || hi == 0) ? lo : -1;
  }
  __device__ __forceinline__ float teacher(const quasar_distill& a) const {
    return as_f32((uint32_t)top << 16 | (a.teacher_dtype == QUASAR_BF16 ? 0u : low));
  }
  // into the list; its logit as well
  template <int T>
  __device__ __forceinline__ void put(const quasar_distill& a, const RowList& o, int k, int64_t base) const {
    const int ix = at(a);
    o.e[k].index = ix;
    o.e[k].p = ix >= 0 ? teacher(a) : -INFINITY;
    o.e[k].z = elem(a.logits, base + (ix >= 0 ? ix : 0), T == kElemBF16);
  }
};

// From the entries' teacher logits in o.p to their probabilities and the logarithms of them.
__device__ __forceinline__ void normalise(const RowList& o, int K, float weight, Divisor tau) {
  const int lane = threadIdx.x & 63;
  wave_lds_fence();
  float m = -INFINITY, s = 0.0f;
  bool nan = false;
  for (int k = lane; k < K; k += 64) {
    m = fmaxf(m, o.e[k].p);
    nan |= o.e[k].p != o.e[k].p;
  }
  m = wave_reduce(m, MaxOp());
  const bool live = weight != 0.0f && (m != -INFINITY || __ballot(nan) != 0);
  if (live) {
    for (int k = lane; k < K; k += 64) {
      const float t = tau.of(o.e[k].p - m), e = exp_of(t);
      o.logp[k] = t;
      o.e[k].p = e;
      s += e;
    }
    s = wave_reduce(s, SumOp());
    const float ls = log_of(s), is = 1.0f / s;
    for (int k = lane; k < K; k += 64) {
      o.e[k].p *= is;
      o.logp[k] -= ls;
    }
  }
  if (lane == 0) *o.some = live ? 1.0f : 0.0f;
}
// The row's loss; the first wavefront's lanes get it.  An entry's two
// logarithms, each from its own maximum on, are subtracted before anything is
// summed: sum p log p and sum p log q are large against a small loss (300
// rows of 1200 classes, 200 listed, tau 0.7, against the formula in 64 bits: off by
// 3.3e-7, the difference of the two sums by 1.0e-6).
__device__ __forceinline__ float loss_of(const RowList& o, int K, float weight, float m, float log_sum, Divisor tau) {
  float s = 0.0f;
  const bool live = o.live();
  if (live)
    for (int k = threadIdx.x & 63; k < K; k += 64) {
      const float p = o.e[k].p;
      if (o.e[k].index >= 0 && !(p == 0.0f)) s += p * (o.logp[k] - (tau.of(o.e[k].z - m) - log_sum));
    }
  s = wave_reduce(s, SumOp());
  return live ? weight * s : 0.0f;
}

// r joined with eight more logits
template <int T>
__device__ __forceinline__ void take(MaxSum& r, const Piece<T>& p, float c) {
  float m = r.m;
#pragma unroll
  for (int i = 0; i < 8; i++) m = fmaxf(m, p.get(i));
  // no exponent to take: of nothing but -inf nothing counts, beside +inf it alone does, and a NaN stays
  if (fabsf(m) == INFINITY) {
    if (m != r.m && r.s == r.s) r.s = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; i++) r.s += p.get(i) != p.get(i) ? p.get(i) : p.get(i) == INFINITY ? 1.0f : 0.0f;
    r.m = m;
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

// NV pieces a thread of a part of a row: classes [e0, e0 + 2048 NV), whole
// pieces only; the last part has the V % 8 classes past them, one a thread.  All
// loads are in flight at once.
template <int T, int NV>
struct Part {
  static constexpr int kClasses = kThreads * 8 * NV, kSize = elem_size<T>();
  Piece<T> p[NV];
  float last;
  int at, bytes, rest;  // this thread's first byte, the part's bytes, the class past the pieces (or V)

  __device__ __forceinline__ Part(int V, int e0) {
    const int left = (V & ~7) - e0;
    at = (int)threadIdx.x * 8 * kSize;
    bytes = (left < kClasses ? left : kClasses) * kSize;
    rest = e0 + kClasses >= V ? (V & ~7) + (int)threadIdx.x : V;
    last = -INFINITY;
  }
  __device__ __forceinline__ bool whole(int v) const { return v * kThreads * 8 * kSize + at < bytes; }
  __device__ __forceinline__ void load(const void* row, int V, int e0) {
    const __amdgpu_buffer_rsrc_t b = wave_buffer(const_cast<char*>(reinterpret_cast<const char*>(row)) + (int64_t)e0 * kSize, bytes);
#pragma unroll
    for (int v = 0; v < NV; v++) load_piece<T>(p[v], b, at + v * kThreads * 8 * kSize);
    if (rest < V) last = elem(row, rest, T == kElemBF16);
  }
};
// r joined with one more logit
__device__ __forceinline__ MaxSum take_one(MaxSum r, float z, float c) {
  return join(r, z == -INFINITY ? MaxSum{z, 0.0f} : MaxSum{z, z == z ? 1.0f : z}, c);
}

__device__ __forceinline__ MaxSum wave_join(MaxSum r, float c) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const MaxSum b{__shfl_xor(r.m, o, 64), __shfl_xor(r.s, o, 64)};
    r = join(r, b, c);
  }
  return r;
}
template <int WAVES = kWaves>
__device__ __forceinline__ MaxSum group_join(MaxSum r, float c, MaxSum* s) {
  r = wave_join(r, c);
  if ((threadIdx.x & 63) == 0) s[wave_index()] = r;
  __syncthreads();
  r = s[0];
#pragma unroll
  for (int i = 1; i < WAVES; i++) r = join(r, s[i], c);
  return r;
}

__device__ __forceinline__ float lse_of(float m, float log_sum, Divisor tau) { return tau.of(m) + log_sum; }

// Workgroup b works on part b % parts of row b / parts.
// Partial maximum and sum of one part of a row, into part[b].
template <int T, int NV>
__global__ __launch_bounds__(kThreads) void distill_scan_kernel(quasar_distill a, int parts, MaxSum* part) {
  __shared__ MaxSum s[kWaves];
  const int row = blockIdx.x / (unsigned)parts, e0 = blockIdx.x % (unsigned)parts * Part<T, NV>::kClasses;
  const float c = kLog2e / a.temperature;
  const int V = (int)a.classes;
  Part<T, NV> z(V, e0);
  z.load(reinterpret_cast<const char*>(a.logits) + row * a.logits_stride * elem_size<T>(), V, e0);
  MaxSum r{-INFINITY, 0.0f};
#pragma unroll
  for (int v = 0; v < NV; v++)
    if (z.whole(v)) take(r, z.p[v], c);
  if (z.rest < V) r = take_one(r, z.last, c);
  r = group_join(r, c, s);
  if (threadIdx.x == 0) part[blockIdx.x] = r;
}

// One part of a row's gradient, and (part 0) its loss and lse.  what: 0 the loss
// alone (one workgroup a row), 1 the gradient alone, 2 both.  lse is joined from
// the row's `sums` partial ones, or (0) taken from a.lse.
template <int T, int NV>
__global__ __launch_bounds__(kThreads) void distill_row_kernel(quasar_distill a, int what, int parts, const MaxSum* part,
                                                               int sums) {
  extern __shared__ float lds[];
  const int64_t row = blockIdx.x / (unsigned)parts, base = row * a.logits_stride, gbase = row * a.grad_stride;
  const int at = blockIdx.x % (unsigned)parts, e0 = at * Part<T, NV>::kClasses;
  const Divisor tau(a.temperature);
  const float it = tau.hi, c = uniform_f32(kLog2e / a.temperature);
  const int V = (int)a.classes, K = a.listed;
  const RowList o(lds, K);
  const float weight = a.row_weight ? a.row_weight[row] : 1.0f;
  // the list's first 64 entries are asked for before the row, whose loads would hold them up
  const int lane = threadIdx.x & 63;
  const Entry first(a, row, lane < K ? lane : 0);
  Part<T, NV> z(V, e0);
  if (what != 0) z.load(reinterpret_cast<const char*>(a.logits) + base * elem_size<T>(), V, e0);
  if (threadIdx.x < 64) {
    if (lane < K) first.put<T>(a, o, lane, base);
    for (int k = lane + 64; k < K; k += 64) Entry(a, row, k).put<T>(a, o, k, base);
  }
  if (what != 0) o.clear<kThreads>();
  MaxSum r{-INFINITY, 0.0f};  // of the row's parts: each wavefront joins them
  for (int i = threadIdx.x & 63; i < sums; i += 64) r = join(r, part[row * sums + i], c);
  if (threadIdx.x < 64) normalise(o, K, weight, tau);
  if (sums > 0) r = wave_join(r, c);
  const float lse = sums > 0 ? lse_of(r.m, log_of(r.s), tau) : a.lse[row];
  __syncthreads();
  const bool live = o.live();
  if (what != 1 && at == 0 && threadIdx.x < 64) {
    const float loss = loss_of(o, K, weight, r.m, log_of(r.s), tau);
    if (threadIdx.x == 0) {
      a.loss[row] = loss;
      a.lse[row] = live ? lse : 0.0f;
    }
  }
  if (what == 0) return;
  const float g = (a.grad_loss ? a.grad_loss[row] : a.grad_scale) * weight * it;
  // the student's probability; z / tau and lse may be large, their difference is taken first
  const auto soft = [&](float z) { return __builtin_amdgcn_exp2f(__builtin_fmaf(z, it, -lse) * kLog2e); };
  const int e1 = e0 + Part<T, NV>::kClasses < V ? e0 + Part<T, NV>::kClasses : V;
  for (int k = threadIdx.x; k < K; k += kThreads)
    if (o.e[k].index >= e0 && o.e[k].index < e1) o.note(k);
  const __amdgpu_buffer_rsrc_t out =
      wave_buffer(reinterpret_cast<char*>(a.grad) + (gbase + e0) * elem_size<T>(), z.bytes);
#pragma unroll
  for (int v = 0; v < NV; v++) {
    float d[8];
#pragma unroll
    for (int i = 0; i < 8; i++) d[i] = soft(z.p[v].get(i));
#pragma unroll
    for (int i = 0; i < 8; i++) d[i] = live ? g * d[i] : 0.0f;
    store_piece<T == kElemBF16>(out, z.at + v * kThreads * 8 * elem_size<T>(), d);
  }
  if (z.rest < V) put_elem(a.grad, gbase + z.rest, live ? g * soft(z.last) : 0.0f, T == kElemBF16);
  __syncthreads();  // the listed classes' gradients over the others'
  if (!live) return;
  for (int k = threadIdx.x; k < K; k += kThreads) {
    const int ix = o.e[k].index;
    if (ix >= e0 && ix < e1) put_elem(a.grad, gbase + ix, g * (soft(o.e[k].z) - o.probability(k, K)), T == kElemBF16);
  }
}

// ---- a row in registers ---------------------------------------------------------
// One workgroup (or wavefront) takes whole rows, NV pieces of eight classes a thread, which stay
// in registers from their only read to the gradient; each piece's registers take
// the next row's as soon as its gradient is stored (without a gradient: as soon
// as it is summed), so loads and stores overlap.  The lists are a row ahead too,
// their entries' loads before the row's (loads return in order: an entry asked
// for after them would come after them, and hold the first wavefront up).
// GRAD: the gradient too.
template <int T, int NT, int NV, bool GRAD>
__global__ __launch_bounds__(NT) void distill_resident_kernel(quasar_distill a) {
  constexpr int kPer = (NT == 64 ? kListedWave : kListed) / NT;  // entries a thread fetches
  extern __shared__ float lds[];
  __shared__ MaxSum sums[2][NT / 64];
  const int tid = threadIdx.x, V = (int)a.classes, K = a.listed;
  const auto list = [&](int turn) { return RowList(lds + turn * RowList::size(K), K); };  // of rows in turn
  const Divisor tau(a.temperature);
  const float it = tau.hi, c = uniform_f32(kLog2e / a.temperature);
  Piece<T> pc[NV];
  // Pieces are whole: a row's buffer ends with its last one; the V % 8 classes past it are one a thread.  No load or
  // store stands behind a branch: the compiler would make the first use of any load wait for all of them.  A
  // workgroup without a next row loads its own again.
  constexpr int kSize = elem_size<T>();
  const int mine = tid * 8 * kSize, bytes = (V & ~7) * kSize;
  const auto whole = [&](int v) { return v * NT * 8 * kSize + mine < bytes; };
  const auto buffer = [&](const void* p, int64_t stride, int64_t row) {
    return wave_buffer(const_cast<char*>(reinterpret_cast<const char*>(p)) + row * stride * kSize, bytes);
  };
  const auto load = [&](int v, __amdgpu_buffer_rsrc_t b) { load_piece<T>(pc[v], b, mine + v * NT * 8 * kSize); };
  const int rest = (V & ~7) + tid;
  float last = -INFINITY;
  const auto load_last = [&](int64_t row) {
    last = elem(a.logits, row * a.logits_stride + (rest < V ? rest : 0), T == kElemBF16);
  };
  // the list of a row: entries, then (in LDS, with the teacher's logits) their logits
  Entry en[kPer];
  float ze[kPer];
  const auto load_list = [&](int64_t row) {
#pragma unroll
    for (int j = 0; j < kPer; j++) en[j] = Entry(a, row, tid + j * NT < K ? tid + j * NT : 0);
  };
  const auto put_list = [&](const RowList& o, int64_t row) {
#pragma unroll
    for (int j = 0; j < kPer; j++) {
      const int k = tid + j * NT, ix = en[j].at(a);
      if (k < K) {
        o.e[k].index = ix;
        o.e[k].p = ix >= 0 ? en[j].teacher(a) : -INFINITY;
      }
      ze[j] = elem(a.logits, row * a.logits_stride + (ix >= 0 ? ix : 0), T == kElemBF16);
    }
  };
  const auto put_logits = [&](const RowList& o) {
#pragma unroll
    for (int j = 0; j < kPer; j++)
      if (tid + j * NT < K) o.e[tid + j * NT].z = ze[j];
  };
  if (blockIdx.x < a.rows) {
    load_list(blockIdx.x);
#pragma unroll
    for (int v = 0; v < NV; v++) load(v, buffer(a.logits, a.logits_stride, blockIdx.x));
    load_last(blockIdx.x);
    put_list(list(0), blockIdx.x);
    put_logits(list(0));
    if constexpr (GRAD) list(0).template clear<NT>();
  }
  __syncthreads();
  int turn = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
    const RowList o = list(turn), n = list(turn ^ 1);
    const int64_t next = row + gridDim.x < a.rows ? row + gridDim.x : row;
    const float weight = a.row_weight ? a.row_weight[row] : 1.0f;
    const __amdgpu_buffer_rsrc_t coming = buffer(a.logits, a.logits_stride, next);
    load_list(next);
    MaxSum r{-INFINITY, 0.0f};
#pragma unroll
    for (int v = 0; v < NV; v++) {
      if (whole(v)) take(r, pc[v], c);
      if constexpr (!GRAD) load(v, coming);
    }
    if (rest < V) r = take_one(r, last, c);
    if constexpr (!GRAD) load_last(next);
    if (tid < 64) normalise(o, K, weight, tau);
    r = group_join<NT / 64>(r, c, sums[turn]);  // its barrier shows the list too
    const bool live = o.live();
    if (tid < 64) {
      // of their own to the compiler: it began what follows ahead of the branch, in every wavefront, and spilled pieces
      // for it (the loss of 4096 x 131072 took 227 us, so 195)
      float rm = r.m, rs = r.s;
      asm volatile("" : "+v"(rm), "+v"(rs));
      const float log_sum = log_of(rs);
      const float loss = loss_of(o, K, weight, rm, log_sum, tau);
      if (tid == 0) {
        a.loss[row] = loss;
        a.lse[row] = live ? lse_of(rm, log_sum, tau) : 0.0f;
      }
    }
    put_list(n, next);
    if constexpr (GRAD) {
      n.template clear<NT>();
      // the last wavefronts: the first one has had the loss to make
      for (int k = NT - 1 - tid; k < K; k += NT)
        if (o.e[k].index >= 0) o.note(k);
      const int64_t gbase = row * a.grad_stride;
      const __amdgpu_buffer_rsrc_t going = buffer(a.grad, a.grad_stride, row);
      const float g = a.grad_scale * weight * it, ls = __builtin_amdgcn_logf(r.s);
      const auto soft = [&](float z) { return __builtin_amdgcn_exp2f(__builtin_fmaf(z - r.m, c, -ls)); };
#pragma unroll
      for (int v = 0; v < NV; v++) {
        float d[8];
        pc[v].refresh();
#pragma unroll
        for (int i = 0; i < 8; i++) d[i] = soft(pc[v].get(i));
#pragma unroll
        for (int i = 0; i < 8; i++) d[i] = live ? g * d[i] : 0.0f;
        store_piece<T == kElemBF16>(going, mine + v * NT * 8 * kSize, d);
        load(v, coming);
      }
      if (rest < V) put_elem(a.grad, gbase + rest, live ? g * soft(last) : 0.0f, T == kElemBF16);
      load_last(next);
      __syncthreads();  // the listed classes' gradients over the others'
      if (live) {
        for (int k = NT - 1 - tid; k < K; k += NT) {
          const int at = o.e[k].index;
          if (at >= 0) put_elem(a.grad, gbase + at, g * (soft(o.e[k].z) - o.probability(k, K)), T == kElemBF16);
        }
      }
      put_logits(n);
    } else {
      put_logits(n);
      __syncthreads();
    }
  }
}

// The split form: pieces a thread takes (1, 2, 4 or 8), so that two
// workgroups or more run on a CU.
int part_pieces(int64_t rows, int64_t classes) {
  int nv = 8;
  while (nv > 1 && rows * ((classes + 2048 * nv - 1) / (2048 * nv)) < 2 * kCUs) nv /= 2;
  while (nv > 1 && 1024 * nv >= classes) nv /= 2;  // pieces past the row cost as many instructions
  return nv;
}
int parts_of(int64_t rows, int64_t classes) {
  const int per = 2048 * part_pieces(rows, classes);
  return (int)((classes + per - 1) / per);
}

// The pieces a thread holds, 64 registers of them at the most.
template <int T>
constexpr int kMostPieces = T == kElemBF16 ? 16 : 8;

// Rows in registers (one launch, one read) where they fill the CUs or are short;
// in parts where a few long ones would leave CUs idle.  Loss and gradient (the loss
// alone), us, bf16 with 64 listed, this form against the parts: 48 x 4000 6.8 against
// 7.4 (4.9, 6.5); 48 x 16384 8.2, 7.7 (6.3, 6.7); 16 x 32000 10.6, 7.1 (8.0, 6.4); 48 x
// 50021 in fp32 15.1, 10.4 (8.2, 7.4); 4096 x 32000 121, 159 (59, 56); 4096 x 131072
// 469, 590 (194, 189).  Between them the rule is not always the faster one: 180 x 50000
// 12.9, 15.9 (7.8, 9.5) but in parts, and a row of more than 65536 classes (fp32: 32768)
// has a CU to itself, so 257 of them take nearly as long as 512: 257 x 131072 51, 37
// (29, 18), 512 x 131072 68, 68 (37, 27).
bool resident(int64_t rows, int64_t classes, bool bf16) {
  const int64_t most = 1024 * 8 * (bf16 ? kMostPieces<kElemBF16> : kMostPieces<kElemF32>);
  return classes <= most && (rows >= kCUs || classes <= 16384);
}

// A row that one wavefront holds takes one where there are rows enough for them
// (four a CU): no wavefront waits for another then.  Loss and gradient, us, against
// 256 threads a row: 8192 x 4000 with 64 listed 32.9, 42.4; 8192 x 1200 20.8, 35.4;
// but 300 x 4000 with 256 listed 13.0, 9.4.
//
// Wavefronts a CU, by what a thread holds (more than fit only queue): 8192 x 4000, 256
// threads a row, 46.6 with 16, 43.6 with 20, 42.4 with 24, 44.3 with 32; one wavefront a
// row 37.0 with 8, 32.9 with 12, 36.1 with 16, 40.3 with 24.
template <int T, bool GRAD>
hipError_t launch_resident(const quasar_distill& a, hipStream_t stream) {
  const size_t lds = 2 * RowList::size(a.listed) * sizeof(float);
#define QUASAR_RESIDENT(NT, NV)                                                                     \
  if (a.classes <= (NT) * 8 * (NV)) {                                                               \
    constexpr int held = (NV) * 8 * elem_size<T>();                                                 \
    constexpr int waves = (NT) == 64 ? 12 : (NT) > 256 || held > 64 ? 16 : held > 32 ? 20 : 24;     \
    const int64_t most = (int64_t)kCUs * (waves * 64 / (NT));                                       \
    distill_resident_kernel<T, NT, NV, GRAD>                                                        \
        <<<dim3((unsigned)(a.rows < most ? a.rows : most)), dim3(NT), lds, stream>>>(a);            \
    return hipGetLastError();                                                                       \
  }
  constexpr int P = kMostPieces<T>;
  if (a.rows >= 4 * kCUs && a.listed <= kListedWave) {
    QUASAR_RESIDENT(64, P / 4)
    QUASAR_RESIDENT(64, P / 2)
  }
  QUASAR_RESIDENT(256, 2)
  if constexpr (P / 4 > 2) QUASAR_RESIDENT(256, P / 4)
  QUASAR_RESIDENT(256, P / 2)
  QUASAR_RESIDENT(256, P)
  QUASAR_RESIDENT(512, P)
  QUASAR_RESIDENT(1024, P * 3 / 4)
  QUASAR_RESIDENT(1024, P)
#undef QUASAR_RESIDENT
  return hipErrorInvalidValue;
}

// n rows from row r on
quasar_distill rows_of(quasar_distill a, int64_t r, int64_t n, int parts) {
  const int64_t size = size_of(a.logits_dtype);
  a.rows = n;
  a.logits = rows_on(a.logits, r, a.logits_stride, size);
  a.grad = rows_on(a.grad, r, a.grad_stride, size);
  a.index = rows_on(a.index, r, a.listed, a.index_bits / 8);
  a.teacher = rows_on(a.teacher, r, a.listed, size_of(a.teacher_dtype));
  a.row_weight = rows_on(a.row_weight, r, 1, 4);
  a.grad_loss = rows_on(a.grad_loss, r, 1, 4);
  a.loss = rows_on(a.loss, r, 1, 4);
  a.lse = rows_on(a.lse, r, 1, 4);
  a.workspace = rows_on(a.workspace, r, parts, sizeof(MaxSum));
  return a;
}

template <int T, int NV>
hipError_t launch_split_rows(const quasar_distill& a, int what, int parts, hipStream_t stream) {
  const dim3 grid((unsigned)(a.rows * parts)), block(kThreads);
  const size_t lds = RowList::size(a.listed) * sizeof(float);
  MaxSum* ws = reinterpret_cast<MaxSum*>(a.workspace);
  const auto row_kernel = [&](int w, int sums) {
    distill_row_kernel<T, NV><<<w == 0 ? dim3((unsigned)a.rows) : grid, block, lds, stream>>>(a, w, w == 0 ? 1 : parts, ws,
                                                                                            sums);
    return hipGetLastError();
  };
  if (what == 1) return row_kernel(1, 0);
  distill_scan_kernel<T, NV><<<grid, block, 0, stream>>>(a, parts, ws);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // in place, the loss is taken before another part's gradient overwrites a listed logit
  if (what == 2 && parts > 1 && a.grad == a.logits) {
    e = row_kernel(0, parts);
    return e != hipSuccess ? e : row_kernel(1, 0);
  }
  return row_kernel(what, parts);
}

template <int T, int NV>
hipError_t launch_split(const quasar_distill& a, int what, hipStream_t stream) {
  const int parts = parts_of(a.rows, a.classes);
  const int64_t most = most_groups(kThreads) / parts;
  for (int64_t r = 0; r < a.rows; r += most) {
    const hipError_t e = launch_split_rows<T, NV>(rows_of(a, r, a.rows - r < most ? a.rows - r : most, parts), what, parts, stream);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <int T>
hipError_t launch_type(const quasar_distill& a, int what, hipStream_t stream) {
  if (what != 1 && resident(a.rows, a.classes, T == kElemBF16))
    return what == 0 ? launch_resident<T, false>(a, stream) : launch_resident<T, true>(a, stream);
  switch (part_pieces(a.rows, a.classes)) {
    case 1: return launch_split<T, 1>(a, what, stream);
    case 2: return launch_split<T, 2>(a, what, stream);
    case 4: return launch_split<T, 4>(a, what, stream);
    default: return launch_split<T, 8>(a, what, stream);
  }
}

}  // namespace

size_t distill_workspace(int64_t rows, int64_t classes) {
  return (size_t)rows * parts_of(rows, classes) * sizeof(MaxSum);
}

hipError_t launch_distill(const quasar_distill& a, int what, hipStream_t stream) {
  return a.logits_dtype == QUASAR_BF16 ? launch_type<kElemBF16>(a, what, stream) : launch_type<kElemF32>(a, what, stream);
}

}  // namespace quasar
