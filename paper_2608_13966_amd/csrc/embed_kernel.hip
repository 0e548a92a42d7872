// embed_kernel.hip -- the embedding: rows of a table by token, and the table's
// gradient (quasar_ops.h).
//
// The lookup moves rows.  The gradient first sorts the tokens (a stable radix
// sort of token and position), so that a token's rows stand together and in
// order; then stretches of the sorted list of the same length are summed, however
// the tokens are distributed: a stretch writes the rows of the table whose tokens
// lie in it whole, and leaves what it has of the others (its first and its last
// at most) to a last launch that joins them.  No float atomics: the order of every
// sum follows from the tokens.
//
// Rows that no token has are zeros.  Where there are few tokens for the table, all of
// it is filled with zeros beside the sort, whose few workgroups mostly wait; else the
// sort marks the rows that tokens have, and further workgroups of the summing launch
// write zeros into the others.  Short lists and small tables take one launch, in which
// each workgroup sorts for itself.
//
// All of it is bound by memory but for the launches.  32768 tokens of 131072 x 4096 in
// bf16: lookup 64 us; gradient 243 (the bytes at a copy's rate 259, a fill of the table
// alone 157).  8 tokens, lookup 2.7; 1999 of 50021 x 1537 in fp32, gradient 68 into three
// tables in turn, 57 into one (a fill 45); 46151 of 538 x 1130 in bf16 56 (its bytes 21),
// nearly half of it the sort's four launches.
#include "ops_common.h"
#include "ops_internal.h"

namespace quasar {
namespace {

constexpr int kThreads = 256;

// The token at i as a row of the table, or `rows` for none.
__device__ __forceinline__ uint32_t token_at(const void* index, int bits, int64_t i, uint32_t rows) {
  if (bits == 64) {
    const uint64_t t = reinterpret_cast<const uint64_t*>(index)[i];
    return t < rows ? (uint32_t)t : rows;
  }
  const uint32_t t = reinterpret_cast<const uint32_t*>(index)[i];
  return t < rows ? t : rows;
}

// ---- lookup -------------------------------------------------------------------
// L lanes (8 columns each) a row, NV pieces a lane.  An output that the last-level
// cache does not hold goes past it: 32768 tokens of 4096 in bf16 65 us, else 76 (four
// pieces a lane 66, one 100).
// WHOLE: a row has eight columns or more, and the lane that its end cuts moves the last eight, some of them the lane's
// before too.
template <int WT, int L, int NV, bool NT, bool WHOLE>
__global__ __launch_bounds__(kThreads) void embed_kernel(quasar_embedding a, int64_t units, Divide per) {
  const int lane = threadIdx.x & (L - 1);
  const int64_t u = (int64_t)blockIdx.x * (kThreads / L) + threadIdx.x / L;
  if (u >= units) return;
  const uint32_t t = per.of((uint32_t)u), part = (uint32_t)u - t * per.by, rows = (uint32_t)a.rows;
  const uint32_t row = token_at(a.index, a.index_bits, t, rows);
  Piece<WT> p[NV];
#pragma unroll
  for (int v = 0; v < NV; v++) {
    int c = ((int)part * NV + v) * (8 * L) + lane * 8;
    if constexpr (WHOLE) {
      c = c < (int)a.cols - 8 ? c : (int)a.cols - 8;
      p[v].load(a.weight, (row < rows ? row : 0) * a.weight_stride + c, 8);
    } else {
      p[v].load(a.weight, row < rows ? row * a.weight_stride + c : 0, row < rows ? (int)a.cols - c : 0);
    }
  }
#pragma unroll
  for (int v = 0; v < NV; v++) {
    int c = ((int)part * NV + v) * (8 * L) + lane * 8;
    if (WHOLE) {
      if (c >= (int)a.cols) continue;
      c = c < (int)a.cols - 8 ? c : (int)a.cols - 8;
    }
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; i++) f[i] = row < rows ? p[v].get(i) * a.scale : 0.0f;
    store_piece<NT>(a.y, t * a.y_stride + c, f, (int)a.cols - c, a.y_dtype == QUASAR_BF16);
  }
}

// ---- sort -----------------------------------------------------------------------
constexpr int kMaxBins = 512, kMaxChunks = 256, kRound = 1024;  // digits; chunks of the list; keys a workgroup ranks at once

struct Sort {
  const void* index;     // the first pass reads the tokens,
  const uint2* from;     // later ones (token, position) pairs
  uint2* to;
  uint32_t* counts;      // [chunks][bins]
  uint8_t* touched;      // [rows], 1 where a token has the row; or NULL
  int index_bits, tokens, chunk;
  uint32_t rows;
  int shift, width, bins;
};

// A table to be filled with zeros, in units of 16 bytes a thread.  A fill of 1 GiB
// takes 157 us in workgroups of 4 KB, 173 of 8 KB, 190 of 32 KB.
struct Fill {
  char* p;
  int64_t bytes;
  int size;  // of an element
  bool nt;   // past the caches: more than half of what the last level holds (10000 tokens of 40000 x 4096, bf16 87 us, else 97)
};
// Units a .. b - 1, by the workgroups from `group` on, `groups` in all.
template <int THREADS>
__device__ __forceinline__ void fill_units(const Fill& f, int64_t a, int64_t b, int64_t group, int64_t groups) {
  for (int64_t u = a + group; u < b; u += groups) {
    int64_t at = (u * THREADS + threadIdx.x) * 16;
    if (at + 16 <= f.bytes) {
      if (f.nt)
        st16_any_nt(f.p + at, make_uint4(0u, 0u, 0u, 0u));
      else
        st16_any(f.p + at, make_uint4(0u, 0u, 0u, 0u));
    } else {
      for (; at < f.bytes; at += f.size) {
        if (f.size == 2)
          *reinterpret_cast<uint16_t*>(f.p + at) = 0;
        else
          *reinterpret_cast<uint32_t*>(f.p + at) = 0u;
      }
    }
  }
}

// All rows are marked as untouched, by thread i of `all`.
__device__ __forceinline__ void clear_marks(const Sort& s, int64_t i, int64_t all) {
  if (!s.touched) return;
  for (; i < ((int64_t)s.rows + 15) / 16; i += all)  // the array is whole pieces of 16
    reinterpret_cast<uint4*>(s.touched)[i] = make_uint4(0u, 0u, 0u, 0u);
}

// A lane's keys of the round from i0 on, one in 64 of its wavefront's; past the end the last one, without a branch: the
// loads then run side by side.
constexpr int kKeys = kRound / kThreads;
__device__ __forceinline__ int place_in_round(int j) { return wave_index() * (64 * kKeys) + j * 64 + (int)(threadIdx.x & 63); }
__device__ __forceinline__ void round_of(const Sort& s, int64_t i0, int end, uint2 (&key)[kKeys]) {
  int at[kKeys];
#pragma unroll
  for (int j = 0; j < kKeys; j++) {
    const int64_t i = i0 + place_in_round(j);
    at[j] = (int)(i < end ? i : end - 1);
  }
  if (s.from) {
#pragma unroll
    for (int j = 0; j < kKeys; j++) key[j] = s.from[at[j]];
  } else if (s.index_bits == 64) {
#pragma unroll
    for (int j = 0; j < kKeys; j++) key[j] = make_uint2(token_at(s.index, 64, at[j], s.rows), (uint32_t)at[j]);
  } else {
#pragma unroll
    for (int j = 0; j < kKeys; j++) key[j] = make_uint2(token_at(s.index, 32, at[j], s.rows), (uint32_t)at[j]);
  }
}

// How often each digit of a pass occurs in a chunk.
__device__ __forceinline__ void count(const Sort& s, int chunks) {
  __shared__ uint32_t bin[kMaxBins];
  for (int i = threadIdx.x; i < s.bins; i += kThreads) bin[i] = 0;
  if (!s.from) clear_marks(s, (int64_t)blockIdx.x * kThreads + threadIdx.x, (int64_t)chunks * kThreads);
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * s.chunk;
  const int end = (int)(first + s.chunk < s.tokens ? first + s.chunk : s.tokens);
  for (int64_t i0 = first; i0 < end; i0 += kRound) {
    uint2 key[kKeys];
    round_of(s, i0, end, key);
#pragma unroll
    for (int j = 0; j < kKeys; j++)
      if (i0 + place_in_round(j) < end) atomicAdd(&bin[(key[j].x >> s.shift) & (s.bins - 1)], 1u);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < s.bins; i += kThreads) s.counts[(int64_t)blockIdx.x * s.bins + i] = bin[i];
}

// In both kernels the workgroups past the first `chunks` fill units a .. b - 1.
__global__ __launch_bounds__(kThreads) void count_kernel(Sort s, int chunks, Fill f, int64_t a, int64_t b) {
  if ((int)blockIdx.x < chunks)
    count(s, chunks);
  else
    fill_units<kThreads>(f, a, b, blockIdx.x - chunks, gridDim.x - chunks);
}

// For K keys a lane, one after the other: how many of the wavefront's keys so far have the key's digit, those of lower
// lanes among them; `count` has them by digit.  The lanes of the same digit are found for all K side by side.
template <int K>
__device__ __forceinline__ void ranks_of(const uint32_t (&key)[K], int bins, const bool (&has)[K], uint32_t* count, uint32_t (&rank)[K]) {
  const int lane = threadIdx.x & 63;
  uint32_t d[K];
  uint64_t same[K];
#pragma unroll
  for (int j = 0; j < K; j++) {
    d[j] = has[j] ? key[j] & (bins - 1) : 0;
    same[j] = __ballot(has[j]);
  }
  for (int b = 1; b < bins; b *= 2) {
#pragma unroll
    for (int j = 0; j < K; j++) {
      const uint64_t set = __ballot((d[j] & b) != 0);
      same[j] &= (d[j] & b) ? set : ~set;
    }
  }
#pragma unroll
  for (int j = 0; j < K; j++) {
    const uint32_t below = __popcll(same[j] & (((uint64_t)1 << lane) - 1));
    rank[j] = has[j] ? count[d[j]] + below : 0;
    wave_lds_fence();
    if (has[j] && below == 0) count[d[j]] += __popcll(same[j]);
    wave_lds_fence();
  }
}

// The sum of n over the lower lanes of a workgroup of WAVES wavefronts (s: WAVES
// numbers of LDS).
template <int WAVES>
__device__ __forceinline__ uint32_t sum_before(uint32_t n, uint32_t* s) {
  const int lane = threadIdx.x & 63, wave = wave_index();
  uint32_t run = n;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const uint32_t up = __shfl_up(run, o);
    if (lane >= o) run += up;
  }
  if (lane == 63) s[wave] = run;
  __syncthreads();
  run -= n;
  for (int w = 0; w < wave; w++) run += s[w];
  return run;
}

// Brings the keys of a chunk to their places: those of smaller digits come first,
// then those of the same digit in earlier chunks, then in earlier wavefronts and
// rounds of this one.
__device__ __forceinline__ void place(const Sort& s, int chunks) {
  constexpr int kWaves = kThreads / 64;
  __shared__ uint32_t base[kMaxBins], count[kWaves][kMaxBins], sums[kWaves];
  const int wave = wave_index(), bins = s.bins;
  const int64_t first = (int64_t)blockIdx.x * s.chunk;
  const int end = (int)(first + s.chunk < s.tokens ? first + s.chunk : s.tokens);
  uint2 key[kKeys];
  // of two digits a thread: their number before this chunk, and in all
  constexpr int kOwn = kMaxBins / kThreads;
  uint32_t before[kOwn], all[kOwn], mine = 0;
#pragma unroll
  for (int j = 0; j < kOwn; j++) before[j] = all[j] = 0;
  if ((int)threadIdx.x * kOwn < bins) {
    static_assert(kOwn == 2, "a pair of digits");
    const uint2* const own = reinterpret_cast<const uint2*>(s.counts) + threadIdx.x;
#pragma unroll 16
    for (int c = 0; c < chunks; c++) {
      const uint2 n = own[(int64_t)c * (bins / 2)];
      before[0] += c < (int)blockIdx.x ? n.x : 0;
      before[1] += c < (int)blockIdx.x ? n.y : 0;
      all[0] += n.x;
      all[1] += n.y;
    }
  }
#pragma unroll
  for (int j = 0; j < kOwn; j++) mine += all[j];
  uint32_t at = sum_before<kWaves>(mine, sums);
#pragma unroll
  for (int j = 0; j < kOwn; j++) {
    const int d = threadIdx.x * kOwn + j;
    base[d] = at + before[j];
    at += all[j];
  }
  for (int64_t i0 = first; i0 < end; i0 += kRound) {
    round_of(s, i0, end, key);
    for (int i = threadIdx.x; i < kWaves * kMaxBins; i += kThreads) (&count[0][0])[i] = 0;
    __syncthreads();
    uint32_t digit[kKeys], rank[kKeys];
    bool has[kKeys];
#pragma unroll
    for (int j = 0; j < kKeys; j++) {
      has[j] = i0 + place_in_round(j) < end;
      digit[j] = key[j].x >> s.shift;
      if (has[j] && s.touched && !s.from && key[j].x < s.rows) s.touched[key[j].x] = 1;
    }
    ranks_of(digit, bins, has, count[wave], rank);
    __syncthreads();
    // count: the keys of the wavefronts before; base: past this round
    for (int d = threadIdx.x; d < bins; d += kThreads) {
      uint32_t at = base[d];
#pragma unroll
      for (int w = 0; w < kWaves; w++) {
        const uint32_t n = count[w][d];
        count[w][d] = at;
        at += n;
      }
      base[d] = at;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kKeys; j++) {
      if (has[j]) s.to[count[wave][(key[j].x >> s.shift) & (bins - 1)] + rank[j]] = key[j];
    }
    __syncthreads();
  }
}

__global__ __launch_bounds__(kThreads) void place_kernel(Sort s, int chunks, Fill f, int64_t a, int64_t b) {
  if ((int)blockIdx.x < chunks)
    place(s, chunks);
  else
    fill_units<kThreads>(f, a, b, blockIdx.x - chunks, gridDim.x - chunks);
}

// All passes at once, for a list that one workgroup holds; the others fill.
constexpr int kSmall = 4096, kSmallRows = 1 << 18;
__global__ __launch_bounds__(1024) void sort_small_kernel(Sort s, int passes, Fill f, int64_t fills) {
  if (blockIdx.x > 0) {
    fill_units<1024>(f, 0, fills, blockIdx.x - 1, gridDim.x - 1);
    return;
  }
  constexpr int kWaves = 16, kKeys = kSmall / 1024;
  __shared__ uint2 list[kSmall];
  __shared__ uint32_t count[kWaves][kMaxBins], sums[kWaves];
  const int lane = threadIdx.x & 63, wave = wave_index(), bins = s.bins;
  uint2 key[kKeys];
#pragma unroll
  for (int j = 0; j < kKeys; j++) {
    const int i = wave * (64 * kKeys) + j * 64 + lane, at = i < s.tokens ? i : s.tokens - 1;
    key[j] = make_uint2(0u, (uint32_t)at);
    if (s.tokens > 0) key[j].x = s.index_bits == 64 ? token_at(s.index, 64, at, s.rows) : token_at(s.index, 32, at, s.rows);
  }
  clear_marks(s, threadIdx.x, 1024);
  __syncthreads();
  for (int p = 0; p < passes; p++) {
    const int shift = p * s.width;
    for (int i = threadIdx.x; i < kWaves * kMaxBins; i += 1024) (&count[0][0])[i] = 0;
    __syncthreads();
    uint32_t digit[kKeys], rank[kKeys];
    bool has[kKeys];
#pragma unroll
    for (int j = 0; j < kKeys; j++) {
      has[j] = wave * (64 * kKeys) + j * 64 + lane < s.tokens;
      digit[j] = key[j].x >> shift;
    }
    ranks_of(digit, bins, has, count[wave], rank);
    __syncthreads();
    uint32_t all = 0;
    if (threadIdx.x < kMaxBins) {
#pragma unroll
      for (int w = 0; w < kWaves; w++) {
        const uint32_t n = count[w][threadIdx.x];
        count[w][threadIdx.x] = all;
        all += n;
      }
    }
    const uint32_t at = sum_before<kWaves>(all, sums);
    if (threadIdx.x < kMaxBins) {
#pragma unroll
      for (int w = 0; w < kWaves; w++) count[w][threadIdx.x] += at;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kKeys; j++) {
      if (wave * (64 * kKeys) + j * 64 + lane < s.tokens) list[count[wave][(key[j].x >> shift) & (bins - 1)] + rank[j]] = key[j];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kKeys; j++) {
      const int i = wave * (64 * kKeys) + j * 64 + lane;
      if (i < s.tokens) key[j] = list[i];
    }
  }
#pragma unroll
  for (int j = 0; j < kKeys; j++) {
    const int i = wave * (64 * kKeys) + j * 64 + lane;
    if (i >= s.tokens) continue;
    s.to[i] = key[j];
    if (s.touched && key[j].x < s.rows) s.touched[key[j].x] = 1;
  }
}

// ---- gradient ---------------------------------------------------------------------
struct Grad {
  const void* dy;
  void* dw;
  const uint2* sorted;
  const uint8_t* touched;
  float* part;            // [stretches][2][pitch]: a stretch's sums for a row begun before it, and for one that goes on
  int64_t dy_stride, dw_stride;
  int64_t sum_groups;     // workgroups that sum; the rest write zeros
  int tokens, stretch, stretches, cols, pitch;
  uint32_t rows;
  float scale;
  int dw_bf16;
  bool nt;                // the one launch's zeros go past the caches
};

template <bool BF16>
__device__ __forceinline__ void put_row(const Grad& g, uint32_t row, int c, const float (&v)[8]) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; i++) f[i] = v[i] * g.scale;
  store_piece<BF16>(g.dw, row * g.dw_stride + c, f, g.cols - c);
}
__device__ __forceinline__ void put_row(const Grad& g, uint32_t row, int c, const float (&v)[8]) {
  if (g.dw_bf16)
    put_row<true>(g, row, c, v);
  else
    put_row<false>(g, row, c, v);
}

// Zeros in a row by `lanes` lanes: 16 bytes each, past the caches with nt.
__device__ __forceinline__ void zero_row(const Grad& g, int64_t row, int lanes = 64, bool nt = false) {
  const int lane = threadIdx.x & (lanes - 1), size = g.dw_bf16 ? 2 : 4, bytes = g.cols * size;
  char* const p = reinterpret_cast<char*>(g.dw) + row * g.dw_stride * size;
  for (int b = lane * 16; b < bytes; b += lanes * 16) {
    if (b + 16 <= bytes) {
      if (nt)
        st16_any_nt(p + b, make_uint4(0u, 0u, 0u, 0u));
      else
        st16_any(p + b, make_uint4(0u, 0u, 0u, 0u));
    } else {
      for (int e = b; e < bytes; e += size) {
        if (size == 2)
          *reinterpret_cast<uint16_t*>(p + e) = 0;
        else
          *reinterpret_cast<uint32_t*>(p + e) = 0u;
      }
    }
  }
}

// Zeros in set `set` of eight rows, where no token has them, by a wavefront.
constexpr int kSet = 8;
__device__ __forceinline__ void zero_rows(const Grad& g, int64_t set) {
  const int64_t r0 = set * kSet;
  if (r0 >= g.rows) return;
  const uint2 t = *reinterpret_cast<const uint2*>(g.touched + r0);  // whole pieces of 16 are there
#pragma unroll 1
  for (int i = 0; i < kSet; i++) {
    if (((i < 4 ? t.x : t.y) >> (8 * (i & 3)) & 0xffu) || r0 + i >= g.rows) continue;
    zero_row(g, r0 + i);
  }
}

constexpr int kMaxStretch = 32;

// L lanes (8 columns each) take a stretch of the sorted list.  WHOLE: a row has eight columns or more, and the lane
// that its end cuts takes its last eight, some of them the lane's before too (the same sums), so that no load has a
// branch and all of a batch run side by side.
template <int GT, int L, bool WHOLE>
__global__ __launch_bounds__(kThreads) void embed_sum_kernel(Grad g, Divide per) {
  const int lane = threadIdx.x & (L - 1);
  if (blockIdx.x >= g.sum_groups) {
    for (int64_t u = blockIdx.x - g.sum_groups; u * (kThreads / 64 * kSet) < g.rows; u += gridDim.x - g.sum_groups)
      zero_rows(g, u * (kThreads / 64) + wave_index());
    return;
  }
  const int64_t u = (int64_t)blockIdx.x * (kThreads / L) + threadIdx.x / L;
  const uint32_t st = per.of((uint32_t)u), part = (uint32_t)u - st * per.by;
  if (st >= (uint32_t)g.stretches) return;
  int c = (int)part * (8 * L) + lane * 8;
  const int left = g.cols - c;
  if (WHOLE && left < 8) c = g.cols - 8;
  const int64_t p0 = (int64_t)st * g.stretch;
  const int n = (int)(g.tokens - p0 < g.stretch ? g.tokens - p0 : g.stretch);
  const uint2* const list = g.sorted + p0;
  // the row that the stretch begins in the middle of, and the one that goes on past it
  const uint32_t none = g.rows, head = p0 > 0 ? list[-1].x : none, tail = p0 + n < g.tokens ? list[n].x : none;
  // The list goes through LDS: a load of it from memory between those of dy's rows would wait for all of them.
  __shared__ uint2 pairs[kThreads / L][kMaxStretch];
  uint2* const mine = pairs[threadIdx.x / L];
  for (int i = lane; i < n; i += L) mine[i] = list[i];
  wave_lds_fence();
  if (mine[0].x >= none) return;  // and all that follow
  const uint32_t at0 = mine[0].y;
  constexpr int kAhead = 4;  // rows of a batch; the next one is in flight while one is summed
  struct Batch {
    uint32_t key[kAhead];
    Piece<GT> row[kAhead];
  } batch[2];
  const auto fetch = [&](Batch& b, int i) {
    uint2 p[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; j++) {
      p[j] = mine[i + j < n ? i + j : n - 1];
      if (i + j >= n) p[j].x = none;
    }
#pragma unroll
    for (int j = 0; j < kAhead; j++) {
      if constexpr (L == 64) {
        p[j].x = __builtin_amdgcn_readfirstlane(p[j].x);
        p[j].y = __builtin_amdgcn_readfirstlane(p[j].y);
      }
      b.key[j] = p[j].x;
      // read once: kept in no cache, where the lines of dw that are still to be written out are (118 us, so 80)
      if constexpr (WHOLE)  // a row that is none, or past the stretch: its first one again, whose sum nothing reads
        b.row[j].template load<true>(g.dy, (p[j].x < none ? p[j].y : at0) * g.dy_stride + c, 8);
      else
        b.row[j].template load<true>(g.dy, p[j].x < none ? p[j].y * g.dy_stride + c : 0, p[j].x < none ? left : 0);
    }
  };
  fetch(batch[0], 0);
  float sum[8] = {};
  uint32_t now = batch[0].key[0];
  bool begun = now == head;  // before this stretch
  const auto flush = [&](bool goes_on) {
    if (now >= none || left <= 0) return;
    if (begun || goes_on)
      store_piece<false>(g.part, ((int64_t)st * 2 + (begun ? 0 : 1)) * g.pitch + c, sum, WHOLE ? 8 : g.pitch - c);
    else
      put_row(g, now, c, sum);
  };
  const auto add = [&](const Batch& b) {
#pragma unroll
    for (int j = 0; j < kAhead; j++) {
      if (b.key[j] != now) {
        flush(false);
        now = b.key[j];
        begun = false;
#pragma unroll
        for (int k = 0; k < 8; k++) sum[k] = 0.0f;
      }
#pragma unroll
      for (int k = 0; k < 8; k++) sum[k] += b.row[j].get(k);
    }
  };
  int i = 0;
  for (; i + 2 * kAhead < n; i += 2 * kAhead) {
    fetch(batch[1], i + kAhead);
    add(batch[0]);
    fetch(batch[0], i + 2 * kAhead);
    add(batch[1]);
  }
  fetch(batch[1], i + kAhead);
  add(batch[0]);
  add(batch[1]);
  flush(now == tail);
}

// The rows that several stretches have sums of: for each stretch in which such a
// row begins, that one's and the next ones', shared out over the workgroup's lanes.
// A row that most tokens have is one workgroup's for each 512 columns: the whole gradient
// of 32768 x 4096 takes 104 us where all tokens are the same, 84 where they are 1000, of
// 300000 x 512 424 and 99.
template <int L>
__global__ __launch_bounds__(kThreads) void embed_join_kernel(Grad g, Divide per) {
  constexpr int kShares = kThreads / L;
  __shared__ float lds[kShares > 1 ? (kShares - 1) * L * 8 : 1];
  const int lane = threadIdx.x & (L - 1), share = threadIdx.x / L;
  const uint32_t st = per.of(blockIdx.x), part = blockIdx.x - st * per.by;
  const int c = (int)part * (8 * L) + lane * 8;
  const int64_t p0 = (int64_t)st * g.stretch, p1 = p0 + g.stretch;
  if (p1 >= g.tokens) return;
  const uint32_t key = g.sorted[p1].x, last = g.sorted[p1 - 1].x, first = g.sorted[p0].x, before = p0 > 0 ? g.sorted[p0 - 1].x : g.rows;
  if (key >= g.rows || last != key) return;         // none goes on
  if (first == key && before == key) return;        // it began before
  // how many stretches follow that begin with it: 64 looked at together
  int more = 1;
  for (int64_t s = (int64_t)st + 1; ; s += 64) {
    const int64_t mine = s + (threadIdx.x & 63);
    const uint64_t same = __ballot(mine < g.stretches && g.sorted[mine * g.stretch].x == key);
    const int run = ~same ? __builtin_ctzll(~same) : 64;
    more += run;
    if (run < 64) break;
  }
  float sum[8] = {};
  constexpr int kAhead = 4;
  for (int i = share; i < more; i += kShares * kAhead) {  // its sums: slot 1 of the stretch where it begins, slot 0 of the others
    Piece<kElemF32> v[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; j++) {
      const int at = i + j * kShares < more ? i + j * kShares : i;  // without a branch, as above
      v[j].load(g.part, (((int64_t)st + at) * 2 + (at == 0)) * g.pitch + (c < g.pitch ? c : 0), 8);
    }
#pragma unroll
    for (int j = 0; j < kAhead; j++)
#pragma unroll
      for (int k = 0; k < 8; k++) sum[k] += i + j * kShares < more ? v[j].get(k) : 0.0f;
  }
  if (share > 0) {
#pragma unroll
    for (int i = 0; i < 8; i++) lds[((share - 1) * 8 + i) * L + lane] = sum[i];
  }
  __syncthreads();
  if (share > 0 || c >= g.cols) return;
  for (int s = 0; s < kShares - 1; s++)
#pragma unroll
    for (int i = 0; i < 8; i++) sum[i] += lds[(s * 8 + i) * L + lane];
  put_row(g, key, c, sum);
}

// ---- gradient, one launch -----------------------------------------------------------
// For lists and tables so small that launches would take most of the time: the first
// `sum_groups` workgroups sort the whole list, each for itself, and sum the rows whose
// tokens begin in their share of it (8 L columns of them); the others write the zeros.
// Up to kFew tokens are sorted by counting the smaller keys of each: 221 of 10136 x 16
// 9 us, 13 by digits (for up to 512 counting takes as long as digits).
constexpr int kFew = 256;
constexpr int kOnceBits = 11;   // of a position: a key is row and position in 32 bits
constexpr int kOnceTokens = 1 << kOnceBits, kOnceRows = 1 << 18;

// The first of list[0 .. n - 1], ascending, that is not below v.
__device__ __forceinline__ int lower_bound(const uint32_t* list, int n, uint32_t v) {
  int at = 0;
  for (; n > 0;) {
    const int half = n >> 1;
    if (list[at + half] < v) {
      at += half + 1;
      n -= half + 1;
    } else {
      n = half;
    }
  }
  return at;
}

// KEYS tokens a thread (a wavefront's follow one another).
template <int GT, int L, int KEYS, bool WHOLE>
__global__ __launch_bounds__(1024) void embed_once_kernel(Grad g, Sort s, int passes, int parts, int each, int zero_rows_each) {
  constexpr int kWaves = 16, kShares = 1024 / L;
  __shared__ __align__(16) uint32_t list[KEYS * 1024];
  __shared__ uint32_t sums[kWaves];
  // first the digits' counts (or the rows that tokens have, one bit each), then the shares' sums
  __shared__ union {
    uint32_t count[kWaves][kMaxBins];
    uint32_t bits[kOnceRows / 32];
    float part[kShares][2][8][L];
  } u;
  const int tid = threadIdx.x, wave = wave_index(), first = wave * (64 * KEYS) + (tid & 63);  // and every 64th on
  uint32_t key[KEYS];
#pragma unroll
  for (int j = 0; j < KEYS; j++) {
    const int i = first + j * 64;
    key[j] = i < s.tokens ? token_at(s.index, s.index_bits, i, s.rows) << kOnceBits | (uint32_t)i : ~0u;
  }
  if ((int)blockIdx.x >= g.sum_groups) {
    const int r0 = (int)(blockIdx.x - g.sum_groups) * zero_rows_each, left = (int)s.rows - r0, n = left < zero_rows_each ? left : zero_rows_each;
    if (n <= 0) return;
    for (int i = tid; i < (n + 31) / 32; i += 1024) u.bits[i] = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < KEYS; j++) {
      const uint32_t own = (key[j] >> kOnceBits) - (uint32_t)r0;  // no token: past every row
      if (own < (uint32_t)n) atomicOr(&u.bits[own >> 5], 1u << (own & 31));
    }
    __syncthreads();
    const int lanes = L == 64 || g.dw_bf16 ? L : 2 * L;
    for (int r = tid / lanes; r < n; r += 1024 / lanes)
      if (!(u.bits[r >> 5] >> (r & 31) & 1u)) zero_row(g, r0 + r, lanes, g.nt);
    return;
  }
  if (KEYS == 1 && s.tokens <= kFew) {
    // a place is the number of smaller keys, each key's in shares
    constexpr int kOwn = kFew * kFew / 4096;  // pieces of four keys
    if (tid < kFew) {
      list[tid] = key[0];
      u.bits[tid] = 0;
    }
    __syncthreads();
    const uint32_t mine = list[tid & (kFew - 1)];
    uint32_t below = 0;
    const uint4* const from = reinterpret_cast<const uint4*>(list) + (tid / kFew) * kOwn;
    for (int j = 0; j < kOwn; j++) {
      const uint4 v = from[j];
      below += (v.x < mine) + (v.y < mine) + (v.z < mine) + (v.w < mine);
    }
    atomicAdd(&u.bits[tid & (kFew - 1)], below);
    __syncthreads();
    if (tid < s.tokens) list[u.bits[tid]] = mine;
    __syncthreads();
  } else {
    const int bins = s.bins;
    for (int p = 0; p < passes; p++) {
      const int shift = kOnceBits + p * s.width;
      for (int i = tid; i < kWaves * kMaxBins; i += 1024) (&u.count[0][0])[i] = 0;
      __syncthreads();
      uint32_t digit[KEYS], rank[KEYS];
      bool has[KEYS];
#pragma unroll
      for (int j = 0; j < KEYS; j++) {
        has[j] = first + j * 64 < s.tokens;
        digit[j] = key[j] >> shift;
      }
      ranks_of(digit, bins, has, u.count[wave], rank);
      __syncthreads();
      uint32_t all = 0;
      if (tid < kMaxBins) {
#pragma unroll
        for (int w = 0; w < kWaves; w++) {
          const uint32_t n = u.count[w][tid];
          u.count[w][tid] = all;
          all += n;
        }
      }
      const uint32_t at = sum_before<kWaves>(all, sums);
      if (tid < kMaxBins) {
#pragma unroll
        for (int w = 0; w < kWaves; w++) u.count[w][tid] += at;
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < KEYS; j++)
        if (first + j * 64 < s.tokens) list[u.count[wave][(key[j] >> shift) & (bins - 1)] + rank[j]] = key[j];
      __syncthreads();
#pragma unroll
      for (int j = 0; j < KEYS; j++)
        if (first + j * 64 < s.tokens) key[j] = list[first + j * 64];
    }
  }
  // the tokens a .. b - 1 of the rows that begin in this workgroup's share
  const int n = lower_bound(list, s.tokens, s.rows << kOnceBits);
  const int share = tid / L, col = tid & (L - 1), group = (int)blockIdx.x / parts;
  int c = ((int)blockIdx.x - group * parts) * (8 * L) + col * 8;
  const int left = g.cols - c;
  if (WHOLE && left < 8) c = g.cols - 8;  // as in embed_sum_kernel
  const auto row_at = [&](int i) { return list[i] >> kOnceBits; };
  const auto from_row = [&](int i) {  // i, or where the row that goes on there ends
    if (i >= n) return n;
    return i > 0 && row_at(i) == row_at(i - 1) ? lower_bound(list, n, (row_at(i) + 1) << kOnceBits) : i;
  };
  const int a = from_row(group * each), b = from_row((group + 1) * each), q = (b - a + kShares - 1) / kShares;
  const int p0 = a + share * q, p1 = p0 + q < b ? p0 + q : b;
  const bool any = p0 < p1, begun = any && p0 > a && row_at(p0) == row_at(p0 - 1), goes_on = any && p1 < b && row_at(p1) == row_at(p1 - 1);
  if (any) {
    constexpr int kAhead = 4;
    struct Batch {
      uint32_t key[kAhead];
      Piece<GT> row[kAhead];
    } batch[2];
    const auto fetch = [&](Batch& o, int i) {
#pragma unroll
      for (int j = 0; j < kAhead; j++) {
        const uint32_t v = list[i + j < p1 ? i + j : p1 - 1];
        o.key[j] = v >> kOnceBits;
        o.row[j].load(g.dy, (int64_t)(v & (kOnceTokens - 1)) * g.dy_stride + (WHOLE || left > 0 ? c : 0), WHOLE ? 8 : left);
      }
    };
    fetch(batch[0], p0);
    float sum[8] = {};
    uint32_t now = batch[0].key[0];
    bool before = begun;
    const auto flush = [&](bool on) {
      if (before || on) {
#pragma unroll
        for (int k = 0; k < 8; k++) u.part[share][before ? 0 : 1][k][col] = sum[k];
      } else if (left > 0) {
        put_row(g, now, c, sum);
      }
    };
    const auto add = [&](const Batch& o, int i) {
#pragma unroll
      for (int j = 0; j < kAhead; j++) {
        if (i + j >= p1) break;
        if (o.key[j] != now) {
          flush(false);
          now = o.key[j];
          before = false;
#pragma unroll
          for (int k = 0; k < 8; k++) sum[k] = 0.0f;
        }
#pragma unroll
        for (int k = 0; k < 8; k++) sum[k] += o.row[j].get(k);
      }
    };
    int i = p0;
    for (; i + 2 * kAhead < p1; i += 2 * kAhead) {
      fetch(batch[1], i + kAhead);
      add(batch[0], i);
      fetch(batch[0], i + 2 * kAhead);
      add(batch[1], i + kAhead);
    }
    if (i + kAhead < p1) fetch(batch[1], i + kAhead);
    add(batch[0], i);
    add(batch[1], i + kAhead);
    flush(goes_on);
  }
  __syncthreads();
  // the rows that several shares have sums of, by the one in which they begin
  if (!goes_on || left <= 0 || (begun && row_at(p0) == row_at(p1 - 1))) return;
  const uint32_t row = row_at(p1);
  float sum[8];
#pragma unroll
  for (int k = 0; k < 8; k++) sum[k] = u.part[share][1][k][col];
  const int last = (lower_bound(list, n, (row + 1) << kOnceBits) - 1 - a) / q;  // the share in which it ends
#pragma unroll 4
  for (int t = share + 1; t <= last; t++)
#pragma unroll
    for (int k = 0; k < 8; k++) sum[k] += u.part[t][0][k][col];
  put_row(g, row, c, sum);
}

// f(L) for the lanes that a row of so many columns takes
template <typename F>
hipError_t with_lanes(int64_t cols, F f) {
  using std::integral_constant;
  if (cols <= 64) return f(integral_constant<int, 8>());
  if (cols <= 128) return f(integral_constant<int, 16>());
  if (cols <= 256) return f(integral_constant<int, 32>());
  return f(integral_constant<int, 64>());
}

constexpr int64_t kCountFill = 8 << 10, kPlaceFill = 12 << 10;  // units

int64_t least_of(int64_t a, int64_t b) { return a < b ? a : b; }
int64_t round16(int64_t n) { return (n + 15) & ~(int64_t)15; }

constexpr int64_t kFull = 2048;  // wavefronts that sum at once
// The sort's passes and where the scratch memory's parts lie.
struct Plan {
  int passes, bits;          // digits of so many bits
  int chunk, chunks;
  int stretch, stretches, pitch;
  int64_t a, b, counts, touched, part, bytes;
  Plan(int64_t rows, int64_t cols, int64_t tokens) {
    int width = 1;
    while (((int64_t)1 << width) <= rows) width++;  // `rows` itself stands for no token
    passes = (width + 8) / 9;
    bits = (width + passes - 1) / passes;
    const int64_t rounds = tokens > 0 ? (tokens + kRound - 1) / kRound : 1, each = (rounds + kMaxChunks - 1) / kMaxChunks;
    chunk = (int)(each * kRound);
    chunks = (int)((rounds + each - 1) / each);
    // short stretches where there are few wavefronts' worth of them, so that enough run at once
    const int64_t lanes = cols <= 64 ? 8 : cols <= 128 ? 16 : cols <= 256 ? 32 : (cols + 511) / 512 * 64, waves = tokens * lanes / 64;
    stretch = waves >= 32 * kFull ? 32 : waves >= 16 * kFull ? 16 : 8;
    stretches = (int)((tokens + stretch - 1) / stretch);
    pitch = (int)((cols + 7) & ~(int64_t)7);
    a = 0;
    b = a + round16(tokens * 8);
    counts = b + round16(tokens * 8);
    touched = counts + round16((int64_t)chunks * 4 << bits);
    part = touched + round16(rows);
    bytes = part + (int64_t)stretches * 2 * pitch * 4;
  }
};

int64_t zero_groups(int64_t rows) { return least_of((rows + 4 * kSet - 1) / (4 * kSet), most_groups(kThreads) / 2); }
unsigned with_fill(int64_t others, int64_t units) { return (unsigned)(others + least_of(units, most_groups(kThreads) - others)); }

template <int GT, int L>
hipError_t launch_sum(Grad g, hipStream_t stream) {
  const int64_t per = (g.cols + 8 * L - 1) / (8 * L), each = kThreads / L;
  g.sum_groups = (g.stretches * per + each - 1) / each;
  const int64_t groups = g.sum_groups + (g.touched ? zero_groups(g.rows) : 0);
  if (groups > 0) {
    if (g.cols >= 8)
      embed_sum_kernel<GT, L, true><<<dim3((unsigned)groups), dim3(kThreads), 0, stream>>>(g, Divide((uint32_t)per));
    else
      embed_sum_kernel<GT, L, false><<<dim3((unsigned)groups), dim3(kThreads), 0, stream>>>(g, Divide((uint32_t)per));
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || g.stretches < 2) return e;
  embed_join_kernel<L><<<dim3((unsigned)((g.stretches - 1) * per)), dim3(kThreads), 0, stream>>>(g, Divide((uint32_t)per));
  return hipGetLastError();
}

template <int GT, int L, int KEYS>
hipError_t launch_once(const Grad& from, const Sort& s, int passes, hipStream_t stream) {
  Grad g = from;
  // about four tokens a share, and no more workgroups than run at once
  const int64_t parts = (g.cols + 8 * L - 1) / (8 * L), most = parts < kCUs / 2 ? kCUs / 2 / parts : 1;
  int64_t groups = (g.tokens + 4 * (1024 / L) - 1) / (4 * (1024 / L));
  groups = groups < 1 ? 1 : least_of(groups, most);
  const int64_t bytes = (int64_t)g.rows * g.cols * (g.dw_bf16 ? 2 : 4);
  const int64_t zeros = least_of((bytes + 16383) / 16384, 2 * kCUs);
  g.sum_groups = groups * parts;
  const dim3 grid((unsigned)(g.sum_groups + zeros));
  const int each = (int)((g.tokens + groups - 1) / groups), zeros_each = (int)((g.rows + zeros - 1) / zeros);
  if (g.cols >= 8)
    embed_once_kernel<GT, L, KEYS, true><<<grid, dim3(1024), 0, stream>>>(g, s, passes, (int)parts, each, zeros_each);
  else
    embed_once_kernel<GT, L, KEYS, false><<<grid, dim3(1024), 0, stream>>>(g, s, passes, (int)parts, each, zeros_each);
  return hipGetLastError();
}

template <int WT>
hipError_t launch_lookup(const quasar_embedding& a, hipStream_t stream) {
  const bool nt = a.tokens * a.cols * size_of(a.y_dtype) >= kLastLevel;
  return with_lanes(a.cols, [&](auto lanes) {
    constexpr int L = decltype(lanes)::value;
    const auto pieces = [&](auto nv) {
      constexpr int NV = decltype(nv)::value;
      constexpr int64_t each = kThreads / L, grid = most_groups(kThreads) * each;
      const int64_t per = (a.cols + 8 * L * NV - 1) / (8 * L * NV), most = (grid < (int64_t)1 << 31 ? grid : (int64_t)1 << 31) / per;
      for (int64_t t = 0; t < a.tokens; t += most) {
        quasar_embedding s = a;
        s.tokens = a.tokens - t < most ? a.tokens - t : most;
        s.index = reinterpret_cast<const char*>(a.index) + t * (a.index_bits / 8);
        s.y = rows_on(a.y, t, a.y_stride, size_of(a.y_dtype));
        const int64_t units = s.tokens * per, groups = (units + each - 1) / each;
        const auto run = [&](auto past, auto whole) {
          embed_kernel<WT, L, NV, decltype(past)::value, decltype(whole)::value>
              <<<dim3((unsigned)groups), dim3(kThreads), 0, stream>>>(s, units, Divide((uint32_t)per));
        };
        if (a.cols < 8)
          run(std::false_type(), std::false_type());
        else if (nt)
          run(std::true_type(), std::true_type());
        else
          run(std::false_type(), std::true_type());
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
      }
      return hipSuccess;
    };
    return a.cols > 512 ? pieces(std::integral_constant<int, 2>()) : pieces(std::integral_constant<int, 1>());
  });
}

}  // namespace

hipError_t launch_embed(const quasar_embedding& a, hipStream_t stream) {
  return a.weight_dtype == QUASAR_BF16 ? launch_lookup<kElemBF16>(a, stream) : launch_lookup<kElemF32>(a, stream);
}

bool embed_backward_fits(int64_t rows, int64_t cols, int64_t tokens, size_t& workspace) {
  const Plan p(rows, cols, tokens);
  workspace = (size_t)p.bytes;
  bool fits = true;
  (void)with_lanes(cols, [&](auto lanes) {
    constexpr int L = decltype(lanes)::value;
    // the join's workgroups; the sums are 256 / L of these to one, and the zeros' at most half a grid
    fits = ((int64_t)p.stretches - 1) * ((cols + 8 * L - 1) / (8 * L)) <= most_groups(kThreads);
    return hipSuccess;
  });
  return fits;
}

hipError_t launch_embed_backward(const quasar_embedding_backward& a, hipStream_t stream) {
  const Plan p(a.rows, a.cols, a.tokens);
  char* const ws = reinterpret_cast<char*>(a.workspace);
  uint2* const bufs[2] = {reinterpret_cast<uint2*>(ws + p.a), reinterpret_cast<uint2*>(ws + p.b)};
  Sort s{};
  s.index = a.index;
  s.counts = reinterpret_cast<uint32_t*>(ws + p.counts);
  s.touched = reinterpret_cast<uint8_t*>(ws + p.touched);
  s.index_bits = a.index_bits;
  s.tokens = (int)a.tokens;
  s.chunk = p.chunk;
  s.rows = (uint32_t)a.rows;
  s.bins = 1 << p.bits;
  s.width = p.bits;
  Grad g{};
  g.dy = a.dy;
  g.dw = a.dweight;
  g.sorted = bufs[(p.passes - 1) & 1];
  g.part = reinterpret_cast<float*>(ws + p.part);
  g.dy_stride = a.dy_stride;
  g.dw_stride = a.dweight_stride;
  g.tokens = (int)a.tokens;
  g.stretch = p.stretch;
  g.stretches = p.stretches;
  g.cols = (int)a.cols;
  g.pitch = p.pitch;
  g.rows = s.rows;
  g.scale = a.scale;
  g.dw_bf16 = a.dweight_dtype == QUASAR_BF16;
  const int64_t bytes = a.rows * a.cols * size_of(a.dweight_dtype);
  // One launch (us, against three): 221 tokens of 10136 x 16 9, 22; 1000 of 1545 x 654 13, 19; 1024 of 10000 x 8192 25, 34;
  // 1076 of 38447 x 128 14, 20; 2048 of 10000 x 8192 28, 38; 1999 of 50021 x 1537 in fp32 57, 57.  In tables of which the
  // last-level cache holds less than half, the fill past it decides: 8 of 131072 x 2048 in fp32 101, 94.  With all tokens the
  // same 1000 of 1000 x 1024 take 19, 22, 2048 32, 26; and more lists longer than that.
  // Its zeros go past the caches where they would take the room of a longer list's rows (into three tables in turn, 2048 of
  // 10000 x 8192 29, else 44; of 32000 x 4096 49, 54; but 8 of 40000 x 4096 65, 63, and lines that rows share 80, 68).
  if (a.tokens <= kOnceTokens && a.rows <= kOnceRows && bytes <= 2 * kLastLevel) {
    const int64_t row_bytes = a.dweight_stride * size_of(a.dweight_dtype);
    g.nt = a.tokens > kFew && bytes > kLastLevel / 2 && row_bytes % 64 == 0 && (reinterpret_cast<uintptr_t>(a.dweight) & 63) == 0;
    return with_lanes(a.cols, [&](auto lanes) {
      constexpr int L = decltype(lanes)::value;
      const auto keys = [&](auto n) {
        constexpr int KEYS = decltype(n)::value;
        return a.dy_dtype == QUASAR_BF16 ? launch_once<kElemBF16, L, KEYS>(g, s, p.passes, stream)
                                         : launch_once<kElemF32, L, KEYS>(g, s, p.passes, stream);
      };
      return a.tokens <= 1024 ? keys(std::integral_constant<int, 1>()) : keys(std::integral_constant<int, 2>());
    });
  }
  // Filling all of the table is the faster where no more than half of its rows can be touched: they are written twice, but
  // the rest without a look at the marks, and beside the sort (131072 x 4096 in bf16, us: 8 tokens 183 against 196, 32768
  // 260 against 293, 60000 317 against 358; 65536 tokens of 50000 x 2048 130 against 126).
  const Fill f{reinterpret_cast<char*>(a.dweight), bytes, (int)size_of(a.dweight_dtype), bytes > kLastLevel / 2};
  const bool fill = a.tokens <= a.rows / 2 && (a.rows == 1 || a.dweight_stride == a.cols);
  if (fill) s.touched = nullptr;
  g.touched = s.touched;
  hipError_t e;
  if (a.tokens <= kSmall && a.rows <= kSmallRows) {
    const int64_t units = fill ? (bytes + 1024 * 16 - 1) / (1024 * 16) : 0;
    s.to = bufs[(p.passes - 1) & 1];
    sort_small_kernel<<<dim3((unsigned)(1 + least_of(units, most_groups(1024) - 1))), dim3(1024), 0, stream>>>(s, p.passes, f, units);
    e = hipGetLastError();
  } else {
    // shares of the fill that take about as long as the sort's part
    const int64_t units = fill ? (bytes + kThreads * 16 - 1) / (kThreads * 16) : 0;
    int64_t done = 0;
    const auto share = [&](int64_t n) {
      const int64_t a0 = done;
      done = least_of(done + n, units);
      return a0;
    };
    e = hipSuccess;
    for (int i = 0; i < p.passes && e == hipSuccess; i++) {
      s.from = i == 0 ? nullptr : bufs[(i - 1) & 1];
      s.to = bufs[i & 1];
      s.shift = i * p.bits;
      int64_t from = share(kCountFill);
      count_kernel<<<dim3(with_fill(p.chunks, done - from)), dim3(kThreads), 0, stream>>>(s, p.chunks, f, from, done);
      e = hipGetLastError();
      if (e != hipSuccess) break;
      from = share(i == p.passes - 1 ? units : kPlaceFill);
      place_kernel<<<dim3(with_fill(p.chunks, done - from)), dim3(kThreads), 0, stream>>>(s, p.chunks, f, from, done);
      e = hipGetLastError();
    }
  }
  if (e != hipSuccess) return e;
  return with_lanes(a.cols, [&](auto lanes) {
    constexpr int L = decltype(lanes)::value;
    return a.dy_dtype == QUASAR_BF16 ? launch_sum<kElemBF16, L>(g, stream) : launch_sum<kElemF32, L>(g, stream);
  });
}

}  // namespace quasar
