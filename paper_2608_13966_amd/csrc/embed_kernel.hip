// embed_kernel.hip -- the embedding: rows of a table by token, and the table's
// gradient (quasar_ops.h).
//
// The lookup moves rows.  The gradient first sorts the tokens (a stable radix
// sort of token and position), so that a token's rows stand together and in
// order; then stretches of the sorted list of the same length are summed, however
// the tokens are distributed: a stretch writes the rows of the table whose tokens
// lie in it whole, and leaves what it has of the others (its first and its last
// at most) to a last launch that joins them.  Rows that no token has are written as
// zeros by further workgroups of the summing launch.  No float atomics: the order
// of every sum follows from the tokens.
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
// L lanes (8 columns each) a row, NV pieces a lane.
template <int WT, int L, int NV>
__global__ __launch_bounds__(kThreads) void embed_kernel(quasar_embedding a, int64_t units, Divide per) {
  const int lane = threadIdx.x & (L - 1);
  const int64_t u = (int64_t)blockIdx.x * (kThreads / L) + threadIdx.x / L;
  if (u >= units) return;
  const uint32_t t = per.of((uint32_t)u), part = (uint32_t)u - t * per.by, rows = (uint32_t)a.rows;
  const uint32_t row = token_at(a.index, a.index_bits, t, rows);
  Piece<WT> p[NV];
#pragma unroll
  for (int v = 0; v < NV; v++) {
    const int c = ((int)part * NV + v) * (8 * L) + lane * 8;
    p[v].load(a.weight, row < rows ? row * a.weight_stride + c : 0, row < rows ? (int)a.cols - c : 0);
  }
#pragma unroll
  for (int v = 0; v < NV; v++) {
    const int c = ((int)part * NV + v) * (8 * L) + lane * 8;
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; i++) f[i] = row < rows ? p[v].get(i) * a.scale : 0.0f;
    store_piece(a.y, t * a.y_stride + c, f, (int)a.cols - c, a.y_dtype == QUASAR_BF16);
  }
}

// ---- sort -----------------------------------------------------------------------
constexpr int kMaxBins = 512, kMaxChunks = 256, kRound = 1024;  // digits; chunks of the list; keys a workgroup ranks at once

struct Sort {
  const void* index;     // the first pass reads the tokens,
  const uint2* from;     // later ones (token, position) pairs
  uint2* to;
  uint32_t* counts;      // [chunks][bins]
  uint8_t* touched;      // [rows], 1 where a token has the row
  int index_bits, tokens, chunk;
  uint32_t rows;
  int shift, bins;
};

__device__ __forceinline__ uint2 pair_at(const Sort& s, int i) {
  if (s.from) return s.from[i];
  return make_uint2(token_at(s.index, s.index_bits, i, s.rows), (uint32_t)i);
}

// How often each digit occurs in a chunk; and on the first pass all rows are marked as untouched.
__global__ __launch_bounds__(kThreads) void count_kernel(Sort s) {
  __shared__ uint32_t bin[kMaxBins];
  for (int i = threadIdx.x; i < s.bins; i += kThreads) bin[i] = 0;
  if (!s.from) {
    const uint32_t quads = (s.rows + 15) / 16;  // the array is whole pieces of 16
    for (uint32_t i = blockIdx.x * kThreads + threadIdx.x; i < quads; i += gridDim.x * kThreads)
      reinterpret_cast<uint4*>(s.touched)[i] = make_uint4(0u, 0u, 0u, 0u);
  }
  __syncthreads();
  const int64_t first = (int64_t)blockIdx.x * s.chunk;
  const int end = (int)(first + s.chunk < s.tokens ? first + s.chunk : s.tokens);
  for (int64_t i = first + threadIdx.x; i < end; i += kThreads)
    atomicAdd(&bin[(pair_at(s, (int)i).x >> s.shift) & (s.bins - 1)], 1u);
  __syncthreads();
  for (int i = threadIdx.x; i < s.bins; i += kThreads) s.counts[(int64_t)blockIdx.x * s.bins + i] = bin[i];
}

// Brings the keys of a chunk to their places: those of smaller digits come first,
// then those of the same digit in earlier chunks, then in earlier wavefronts and
// rounds of this one.
__global__ __launch_bounds__(kThreads) void place_kernel(Sort s) {
  constexpr int kWaves = kThreads / 64, kKeys = kRound / kThreads;  // keys a lane holds
  __shared__ uint32_t base[kMaxBins], count[kWaves][kMaxBins], sums[kWaves];
  const int lane = threadIdx.x & 63, wave = wave_index(), bins = s.bins;
  // of two digits a thread: their number before this chunk, and in all
  constexpr int kOwn = kMaxBins / kThreads;
  uint32_t before[kOwn], all[kOwn], mine = 0;
#pragma unroll
  for (int j = 0; j < kOwn; j++) {
    const int d = threadIdx.x * kOwn + j;
    before[j] = all[j] = 0;
    if (d < bins) {
#pragma unroll 8
      for (int c = 0; c < (int)gridDim.x; c++) {
        const uint32_t n = s.counts[(int64_t)c * bins + d];
        before[j] += c < (int)blockIdx.x ? n : 0;
        all[j] += n;
      }
    }
    mine += all[j];
  }
  // digits before this thread's: over the wavefront, then the wavefronts
  uint32_t run = mine;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const uint32_t up = __shfl_up(run, o);
    if (lane >= o) run += up;
  }
  if (lane == 63) sums[wave] = run;
  __syncthreads();
  uint32_t at = run - mine;
  for (int w = 0; w < wave; w++) at += sums[w];
#pragma unroll
  for (int j = 0; j < kOwn; j++) {
    const int d = threadIdx.x * kOwn + j;
    base[d] = at + before[j];
    at += all[j];
  }
  const int64_t first = (int64_t)blockIdx.x * s.chunk;
  const int end = (int)(first + s.chunk < s.tokens ? first + s.chunk : s.tokens);
  for (int64_t i0 = first; i0 < end; i0 += kRound) {
    for (int i = threadIdx.x; i < kWaves * kMaxBins; i += kThreads) (&count[0][0])[i] = 0;
    __syncthreads();
    uint2 key[kKeys];
    uint32_t rank[kKeys];
#pragma unroll
    for (int j = 0; j < kKeys; j++) {
      const int64_t i = i0 + wave * (64 * kKeys) + j * 64 + lane;
      const bool has = i < end;
      if (has) {
        key[j] = pair_at(s, (int)i);
        if (!s.from && key[j].x < s.rows) s.touched[key[j].x] = 1;
      }
      const uint32_t d = has ? (key[j].x >> s.shift) & (bins - 1) : 0;
      // the lanes with the same digit
      uint64_t same = __ballot(has);
      for (int b = 1; b < bins; b *= 2) {
        const uint64_t set = __ballot((d & b) != 0);
        same &= (d & b) ? set : ~set;
      }
      const uint32_t below = __popcll(same & (((uint64_t)1 << lane) - 1));
      rank[j] = has ? count[wave][d] + below : 0;
      wave_lds_fence();
      if (has && below == 0) count[wave][d] += __popcll(same);
      wave_lds_fence();
    }
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
      const int64_t i = i0 + wave * (64 * kKeys) + j * 64 + lane;
      if (i < end) s.to[count[wave][(key[j].x >> s.shift) & (bins - 1)] + rank[j]] = key[j];
    }
    __syncthreads();
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

constexpr int kZeroRows = 8;  // rows that L lanes look at for zeros

// L lanes (8 columns each) take a stretch of the sorted list; the next rows are in flight meanwhile.
template <int GT, int L>
__global__ __launch_bounds__(kThreads) void embed_sum_kernel(Grad g, Divide per) {
  const int lane = threadIdx.x & (L - 1);
  if (blockIdx.x >= g.sum_groups) {
    const int64_t u = (blockIdx.x - g.sum_groups) * (kThreads / L) + threadIdx.x / L;
    const uint32_t set = per.of((uint32_t)u), part = (uint32_t)u - set * per.by;
    const int64_t r0 = (int64_t)set * kZeroRows;
    const int c = (int)part * (8 * L) + lane * 8;
    const float zero[8] = {};
    if (c >= g.cols) return;
    if (r0 >= g.rows) return;
    uint2 t = *reinterpret_cast<const uint2*>(g.touched + r0);  // whole pieces of 16 are there
#pragma unroll
    for (int i = 0; i < kZeroRows; i++) {
      const uint32_t has = (i < 4 ? t.x : t.y) >> (8 * (i & 3)) & 0xffu;
      if (!has && r0 + i < g.rows) put_row(g, (uint32_t)r0 + i, c, zero);
    }
    return;
  }
  const int64_t u = (int64_t)blockIdx.x * (kThreads / L) + threadIdx.x / L;
  const uint32_t st = per.of((uint32_t)u), part = (uint32_t)u - st * per.by;
  if (st >= (uint32_t)g.stretches) return;
  const int c = (int)part * (8 * L) + lane * 8, left = g.cols - c;
  const int64_t p0 = (int64_t)st * g.stretch;
  const int n = (int)(g.tokens - p0 < g.stretch ? g.tokens - p0 : g.stretch);
  const uint2* const list = g.sorted + p0;
  // the row that the stretch begins in the middle of, and the one that goes on past it
  const uint32_t none = g.rows, head = p0 > 0 ? list[-1].x : none, tail = p0 + n < g.tokens ? list[n].x : none;
  constexpr int kAhead = 4;
  Piece<GT> row[kAhead];
  uint2 key[kAhead];
  const auto fetch = [&](int j, int i) {
    key[j] = i < n ? list[i] : make_uint2(none, 0u);
    row[j].load(g.dy, key[j].x < none ? key[j].y * g.dy_stride + c : 0, key[j].x < none ? left : 0);
  };
#pragma unroll
  for (int j = 0; j < kAhead; j++) fetch(j, j);
  float sum[8] = {};
  uint32_t now = key[0].x;
  bool begun = now == head;  // before this stretch
  const auto flush = [&](bool goes_on) {
    if (now >= none) return;
    if (begun || goes_on)
      store_piece<false>(g.part, ((int64_t)st * 2 + (begun ? 0 : 1)) * g.pitch + c, sum, g.pitch - c);
    else
      put_row(g, now, c, sum);
  };
  for (int i = 0; i < n; i += kAhead) {
#pragma unroll
    for (int j = 0; j < kAhead; j++) {
      if (key[j].x != now) {
        flush(false);
        now = key[j].x;
        begun = false;
#pragma unroll
        for (int k = 0; k < 8; k++) sum[k] = 0.0f;
      }
#pragma unroll
      for (int k = 0; k < 8; k++) sum[k] += row[j].get(k);
      fetch(j, i + kAhead + j);
    }
  }
  flush(now == tail);
}

// The rows that several stretches have sums of: for each stretch in which such a
// row begins, that one's and the next ones', shared out over the workgroup's lanes.
template <int L>
__global__ __launch_bounds__(kThreads) void embed_join_kernel(Grad g, Divide per) {
  constexpr int kShares = kThreads / L;
  __shared__ float lds[kShares > 1 ? (kShares - 1) * L * 8 : 1];
  const int lane = threadIdx.x & (L - 1), share = threadIdx.x / L;
  const uint32_t st = per.of(blockIdx.x), part = blockIdx.x - st * per.by;
  const int c = (int)part * (8 * L) + lane * 8;
  const int64_t p0 = (int64_t)st * g.stretch, p1 = p0 + g.stretch;
  if (p1 >= g.tokens) return;
  const uint32_t key = g.sorted[p1].x;
  if (key >= g.rows || g.sorted[p1 - 1].x != key) return;                     // none goes on
  if (g.sorted[p0].x == key && p0 > 0 && g.sorted[p0 - 1].x == key) return;  // it began before
  float sum[8] = {};
  const auto add = [&](int64_t stretch, int slot) {
    float v[8];
    load_floats(g.part, (stretch * 2 + slot) * g.pitch + c, g.pitch - c, false, v);
#pragma unroll
    for (int i = 0; i < 8; i++) sum[i] += v[i];
  };
  if (share == 0) add(st, 1);
  for (int64_t s = (int64_t)st + 1 + share; s < g.stretches && g.sorted[s * g.stretch].x == key; s += kShares) add(s, 0);
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

// f(L) for the lanes that a row of so many columns takes
template <typename F>
hipError_t with_lanes(int64_t cols, F f) {
  using std::integral_constant;
  if (cols <= 64) return f(integral_constant<int, 8>());
  if (cols <= 128) return f(integral_constant<int, 16>());
  if (cols <= 256) return f(integral_constant<int, 32>());
  return f(integral_constant<int, 64>());
}

int64_t round16(int64_t n) { return (n + 15) & ~(int64_t)15; }

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
    // short stretches where there are few tokens, so that enough of them run at once
    stretch = tokens >= 16384 ? 32 : tokens >= 4096 ? 16 : 8;
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

template <int GT, int L>
hipError_t launch_sum(Grad g, hipStream_t stream) {
  const int64_t per = (g.cols + 8 * L - 1) / (8 * L), each = kThreads / L;
  const int64_t units = g.stretches * per, zeros = ((int64_t)g.rows + kZeroRows - 1) / kZeroRows * per;
  g.sum_groups = (units + each - 1) / each;
  const int64_t groups = g.sum_groups + (zeros + each - 1) / each;
  embed_sum_kernel<GT, L><<<dim3((unsigned)groups), dim3(kThreads), 0, stream>>>(g, Divide((uint32_t)per));
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || g.stretches < 2) return e;
  embed_join_kernel<L><<<dim3((unsigned)((g.stretches - 1) * per)), dim3(kThreads), 0, stream>>>(g, Divide((uint32_t)per));
  return hipGetLastError();
}

template <int WT>
hipError_t launch_lookup(const quasar_embedding& a, hipStream_t stream) {
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
        embed_kernel<WT, L, NV><<<dim3((unsigned)groups), dim3(kThreads), 0, stream>>>(s, units, Divide((uint32_t)per));
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
    constexpr int L = decltype(lanes)::value, each = kThreads / L;
    const int64_t per = (cols + 8 * L - 1) / (8 * L), zeros = (rows + kZeroRows - 1) / kZeroRows * per;
    fits = p.stretches * per <= most_groups(kThreads) && zeros < (int64_t)1 << 31 &&
           (p.stretches * per + each - 1) / each + (zeros + each - 1) / each <= most_groups(kThreads);
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
  for (int i = 0; i < p.passes; i++) {
    s.from = i == 0 ? nullptr : bufs[(i - 1) & 1];
    s.to = bufs[i & 1];
    s.shift = i * p.bits;
    count_kernel<<<dim3(p.chunks), dim3(kThreads), 0, stream>>>(s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    place_kernel<<<dim3(p.chunks), dim3(kThreads), 0, stream>>>(s);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  Grad g{};
  g.dy = a.dy;
  g.dw = a.dweight;
  g.sorted = s.to;
  g.touched = s.touched;
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
  return with_lanes(a.cols, [&](auto lanes) {
    constexpr int L = decltype(lanes)::value;
    return a.dy_dtype == QUASAR_BF16 ? launch_sum<kElemBF16, L>(g, stream) : launch_sum<kElemF32, L>(g, stream);
  });
}

}  // namespace quasar
