// weight_grad_kernel.hip -- a linear layer's weight gradient from the input that
// was kept in 8 bits (quasar_ops.h): dweight = dy^T x, summed over the tokens.
//
// Both operands have the summed dimension in their rows, and a matrix instruction
// wants it along a lane's registers: tiles lie in LDS as they come from memory and
// are read through LDS's transposing loads (four rows of 16 columns by 16 lanes:
// each gets one column).  x becomes bf16 on the way, exactly (its exponent is a
// power of two); dy in fp32 becomes three bf16 parts, exactly, one product each.
#include "ops_common.h"
#include "ops_internal.h"

namespace quasar {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kStep = 64;                    // tokens a step takes
constexpr int64_t kMaxPitch = (1 << 22) - 1;  // elements of a row whose bytes the tile kernel reckons in 24 bits

__host__ __device__ constexpr int64_t part_pitch(int64_t cols) { return (cols + 7) & ~(int64_t)7; }

// Eight E4M3 bytes times a power of two as packed bf16, exact.
__device__ __forceinline__ uint4 kept_bf16(uint2 q, float f) {
  float v[8];
  unpack_e4m3x8(q, v);
#pragma unroll
  for (int i = 0; i < 8; i++) v[i] *= f;
  return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}

// Eight fp32 values as the sum of three bf16 ones each: cut off after eight
// significant bits twice, and what is left has eight.  NaN and infinity are the
// first part alone.
__device__ __forceinline__ void split3(const float (&v)[8], uint4 (&o)[3]) {
  uint32_t d[3][4];
#pragma unroll
  for (int i = 0; i < 4; i++) {
    uint32_t hi[2], mid[2];
    float lo[2];
#pragma unroll
    for (int j = 0; j < 2; j++) {
      const float x = v[2 * i + j];
      const bool finite = fabsf(x) < INFINITY;
      hi[j] = x == x ? as_u32(x) & 0xffff0000u : 0x7fc00000u;
      const float r = finite ? x - as_f32(hi[j]) : 0.0f;
      mid[j] = as_u32(r) & 0xffff0000u;
      lo[j] = r - as_f32(mid[j]);
    }
    d[0][i] = (hi[0] >> 16) | hi[1];
    d[1][i] = (mid[0] >> 16) | mid[1];
    d[2][i] = pack_bf16x2(lo[0], lo[1]);
  }
#pragma unroll
  for (int p = 0; p < 3; p++) o[p] = make_uint4(d[p][0], d[p][1], d[p][2], d[p][3]);
}

// In LDS a row of a tile is W columns; the 16-column unit u of row t lies at u ^
// f(t): the rows 8 g + 4 j + (0 .. 3) that a transposing load takes then lie in
// different banks, those of two groups g too.
template <int W>
__device__ __forceinline__ int spot(int t, int col) {
  const int f = ((t & 3) | ((t >> 1) & 4)) & (W / 16 - 1);
  return t * W + (((col >> 4) ^ f) << 4) + (col & 15);
}

// The operand of a 16 x 16 x 32 matrix instruction: columns col .. col + 15 of the
// 32 rows from t0 on.
template <int W>
__device__ __forceinline__ bf16x8 read_tile(const uint16_t* lds, int t0, int col, int lane) {
  const int t = t0 + 8 * (lane >> 4) + ((lane & 15) >> 2), c = col + 4 * (lane & 3);
  typedef __attribute__((address_space(3))) s16x4 lds4;
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(lds + spot<W>(t, c)));
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(lds + spot<W>(t + 4, c)));
  typedef short s16x8 __attribute__((ext_vector_type(8)));
  const s16x8 r = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  return __builtin_bit_cast(bf16x8, r);
}

// A workgroup makes B x B values of dweight (or of its share's sums in part) from
// its share of the tokens, 64 at a time: the next 64 come to registers while these
// are multiplied.  Four wavefronts of B/2 x B/2.
template <int GT, int B>
__global__ __launch_bounds__(256) void weight_grad_kernel(quasar_weight_grad a, int tiles_n, int splits, int steps_per, float* part) {
  constexpr int kParts = GT == kElemF32 ? 3 : 1, kPieces = kStep * B / 8 / 256, T = B / 32;
  __shared__ __align__(16) uint16_t lds[(kParts + 1) * kStep * B];
  uint16_t* const xs = lds + kParts * kStep * B;
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_index();
  const int split = blockIdx.x % (unsigned)splits, tile = blockIdx.x / (unsigned)splits;
  const int64_t n0 = (int64_t)(tile % tiles_n) * B, k0 = (int64_t)(tile / tiles_n) * B;
  const int64_t t0 = (int64_t)split * steps_per * kStep;
  const int64_t t1 = t0 + (int64_t)steps_per * kStep < a.tokens ? t0 + (int64_t)steps_per * kStep : a.tokens;

  // this thread's pieces: columns 8 c of rows tr + i * (rows of a round)
  constexpr int kWide = B / 8, kRound = 256 / kWide;
  const int c = (tid % kWide) * 8, tr = tid / kWide;
  const int ln = (int)(a.rows - n0 - c < 8 ? a.rows - n0 - c : 8), lk = (int)(a.cols - k0 - c < 8 ? a.cols - k0 - c : 8);
  Piece<GT> g[kPieces];
  uint2 q[kPieces];
  uint32_t e[kPieces];
  const auto fetch = [&](int64_t t) {
#pragma unroll
    for (int i = 0; i < kPieces; i++) {
      const int64_t r = t + tr + i * kRound;
      const bool has = r < t1;
      g[i].load(a.dy, has ? r * a.dy_stride + n0 + c : 0, has ? ln : 0);
      q[i] = load_bytes(has ? a.q + r * a.q_stride + k0 + c : a.q, has ? lk : 0);
      e[i] = has && lk > 0 ? a.exponent[r * a.exponent_stride + ((k0 + c) >> 7)] : 127u;
    }
  };
  f32x4 acc[T][T];
#pragma unroll
  for (int i = 0; i < T; i++)
#pragma unroll
    for (int j = 0; j < T; j++) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const int wn = (wave >> 1) * (B / 2), wk = (wave & 1) * (B / 2);
  if (t0 < t1) fetch(t0);
  for (int64_t t = t0; t < t1; t += kStep) {
    __syncthreads();  // the last step's reads are done
#pragma unroll
    for (int i = 0; i < kPieces; i++) {
      const int at = spot<B>(tr + i * kRound, c);
      if constexpr (GT == kElemF32) {
        uint4 p[3];
        split3(g[i].f, p);
#pragma unroll
        for (int j = 0; j < 3; j++) *reinterpret_cast<uint4*>(lds + j * kStep * B + at) = p[j];
      } else {
        *reinterpret_cast<uint4*>(lds + at) = make_uint4(g[i].d[0], g[i].d[1], g[i].d[2], g[i].d[3]);
      }
      *reinterpret_cast<uint4*>(xs + at) = kept_bf16(q[i], as_f32(e[i] << 23));
    }
    if (t + kStep < t1) fetch(t + kStep);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kStep; k += 32) {
      bf16x8 mx[T];
#pragma unroll
      for (int j = 0; j < T; j++) mx[j] = read_tile<B>(xs, k, wk + 16 * j, lane);
#pragma unroll
      for (int p = 0; p < kParts; p++)
#pragma unroll
        for (int i = 0; i < T; i++) {
          const bf16x8 mg = read_tile<B>(lds + p * kStep * B, k, wn + 16 * i, lane);
#pragma unroll
          for (int j = 0; j < T; j++) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(mg, mx[j], acc[i][j], 0, 0, 0);
        }
    }
  }
  // acc[i][j][e]: row 16 i + 4 (lane / 16) + e, column 16 j + lane % 16
#pragma unroll
  for (int i = 0; i < T; i++)
#pragma unroll
    for (int j = 0; j < T; j++)
#pragma unroll
      for (int r = 0; r < 4; r++) {
        const int64_t n = n0 + wn + 16 * i + 4 * (lane >> 4) + r, k = k0 + wk + 16 * j + (lane & 15);
        if (n >= a.rows || k >= a.cols) continue;
        if (part)
          part[((int64_t)split * a.rows + n) * part_pitch(a.cols) + k] = acc[i][j][r];
        else
          put_elem(a.dweight, n * a.dweight_stride + k, acc[i][j][r], a.dweight_dtype == QUASAR_BF16);
      }
}

// ---- large weights ----------------------------------------------------------------
// x in bf16 [padded tokens, kp], rows past the last token zero; and what the tile
// kernel cannot load of dy as it is: all of it in bf16 [padded tokens, np] (fp32: its
// three parts one after the other, which the products then run through as through
// three times the tokens), or the last, incomplete step's rows alone.
struct Spread {
  uint16_t *x, *dy;
  int64_t x_pieces, dy_pieces;  // of eight elements
  int64_t padded, first;        // tokens; the first that dy holds
  Divide kp8, np8;              // pieces of a row
};

template <int GT>
__global__ __launch_bounds__(256) void spread_kernel(quasar_weight_grad a, Spread s) {
  const int64_t all = s.x_pieces + s.dy_pieces, step = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += step) {
    if (i < s.x_pieces) {
      const int64_t t = i / s.kp8.by;
      const int k = (int)(i - t * s.kp8.by) * 8;
      const bool has = t < a.tokens;
      const uint2 q = load_bytes(has ? a.q + t * a.q_stride + k : a.q, has ? (int)a.cols - k : 0);
      const uint32_t e = has ? a.exponent[t * a.exponent_stride + (k >> 7)] : 127u;
      st128(s.x + i * 8, kept_bf16(q, as_f32(e << 23)));
    } else {
      const int64_t j = i - s.x_pieces, r = j / s.np8.by, t = r + s.first;
      const int n = (int)(j - r * s.np8.by) * 8;
      const bool has = t < a.tokens;
      Piece<GT> g;
      g.load(a.dy, has ? t * a.dy_stride + n : 0, has ? (int)a.rows - n : 0);
      if constexpr (GT == kElemF32) {
        uint4 p[3];
        split3(g.f, p);
#pragma unroll
        for (int q = 0; q < 3; q++) st128(s.dy + (q * s.dy_pieces + j) * 8, p[q]);
      } else {
        st128(s.dy + j * 8, make_uint4(g.d[0], g.d[1], g.d[2], g.d[3]));
      }
    }
  }
}

// The operands of the tile kernel: rows of dy up to step `whole`, then from `rest`;
// x repeats after `period` steps.
struct Operands {
  const uint16_t *dy, *rest, *x;
  int dy_stride, rest_stride, kp, np;  // elements; np: columns that dy has
  int whole, period, steps;
};

// A workgroup makes 256 x 256 values of dweight with 8 wavefronts of 128 rows x 64
// columns, 64 tokens a step.  Both operands of a step lie in LDS as two halves each
// (g0: the first 64 rows of every wavefront's 128, x0: the first 32 columns of its
// 64, x1 and g1 the rest), and a step has two phases, each with 32 matrix
// instructions a wavefront: g0 (x0 x1), g1 (x0 x1).  Two stages; a half is filled again
// as soon as both halves of the workgroup have read it.
//
// The wavefronts of a SIMD work in turn: those of wm = 1 run one barrier behind, so
// that while one multiplies the other reads its next operands.  Barriers 2p and 2p + 1
// end the reading and the multiplying of phase p for wm = 0, 2p + 1 and 2p + 2 for wm
// = 1; a wavefront has its operands before it comes to the barrier that ends the
// reading.  Hence
//  - a half filled in phase p may be one whose last reads were in phase p - 1
//    (g0, x0 and x1, read in a step's phase 0, are filled for the step after the
//    next in its phase 1; g1 in the next step's phase 0);
//  - what phase p reads has to have landed for every wavefront's own loads
//    before the barrier that ends its reading of phase p - 1: with two loads a
//    half, "at most 8 outstanding" then, either phase.
// Past the last step the loads repeat it, so that the counts hold.
constexpr int kSlabPitch = 64 + 4, kSlab = 32 * kSlabPitch;
__global__ __launch_bounds__(512, 2) void weight_grad_tile_kernel(quasar_weight_grad a, Operands op, int tiles_n, int tiles_k,
                                                                  int steps_per, float* part) {
  constexpr int kHalf = kStep * 128, kStage = 4 * kHalf;  // elements; halves g0, x0, x1, g1
  __shared__ __align__(16) uint16_t lds[2 * kStage];
  static_assert(8 * kSlab * 4 <= (int)sizeof(lds), "the epilogue's stage fits");
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)lds;
  const int lane = threadIdx.x & 63, wave = wave_index();
  const int wm = wave >> 2, wn = wave & 3;
  int tn, tk;
  const int split = blockIdx.x / (unsigned)(tiles_n * tiles_k);
  tile_of(blockIdx.x - split * tiles_n * tiles_k, tiles_n, tiles_k, tn, tk);
  const int n0 = tn * 256, k0 = tk * 256;
  const int first = split * steps_per, left = op.steps - first, steps = left < steps_per ? left : steps_per;

  // each wavefront loads 8 rows of a half, 4 an instruction; columns past the matrix repeat its last ones
  uint32_t col[4][2], row[2];
#pragma unroll
  for (int i = 0; i < 2; i++) {
    const int t = wave * 8 + i * 4 + (lane >> 4);
    const int f = (t & 3) | ((t >> 1) & 4), c = ((((lane & 15) >> 1) ^ f) << 4) + (lane & 1) * 8;
    row[i] = (uint32_t)t;
#pragma unroll
    for (int h = 0; h < 2; h++) {
      const int n = n0 + (c >> 6) * 128 + h * 64 + (c & 63), k = k0 + (c >> 5) * 64 + h * 32 + (c & 31);
      col[h == 0 ? 0 : 3][i] = 2u * (uint32_t)(n < op.np - 8 ? n : op.np - 8);
      col[h == 0 ? 1 : 2][i] = 2u * (uint32_t)(k < op.kp - 8 ? k : op.kp - 8);
    }
  }
  const auto fill = [&](int h, int step) {
    const uint32_t to = lds0 + ((step & 1) * kStage + h * kHalf + wave * 8 * 128) * 2;
    const int s = first + (step < steps ? step : steps - 1);
    const char* from;
    uint32_t pitch;
    if (h == 0 || h == 3) {
      const bool rest = s >= op.whole;
      pitch = 2u * (uint32_t)(rest ? op.rest_stride : op.dy_stride);
      from = reinterpret_cast<const char*>(rest ? op.rest : op.dy) + (int64_t)(rest ? s - op.whole : s) * kStep * pitch;
    } else {
      int sx = s;
      if (sx >= op.period) sx -= op.period;
      if (sx >= op.period) sx -= op.period;
      pitch = 2u * (uint32_t)op.kp;
      from = reinterpret_cast<const char*>(op.x) + (int64_t)sx * kStep * pitch;
    }
#pragma unroll
    for (int i = 0; i < 2; i++) load_lds16(from, __umul24(row[i], pitch) + col[h][i], to + i * 4 * 128 * 2);
  };
  f32x4 acc[8][4];
#pragma unroll
  for (int i = 0; i < 8; i++)
#pragma unroll
    for (int j = 0; j < 4; j++) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  bf16x8 fg[4][2], fx[2][2][2];
  const auto read_g = [&](int h, int stage) {
    const uint16_t* p = lds + stage * kStage + (h ? 3 : 0) * kHalf;
#pragma unroll
    for (int i = 0; i < 4; i++)
#pragma unroll
      for (int k = 0; k < 2; k++) fg[i][k] = read_tile<128>(p, 32 * k, wm * 64 + 16 * i, lane);
  };
  const auto read_x = [&](int h, int stage) {
    const uint16_t* p = lds + stage * kStage + (h ? 2 : 1) * kHalf;
#pragma unroll
    for (int j = 0; j < 2; j++)
#pragma unroll
      for (int k = 0; k < 2; k++) fx[h][j][k] = read_tile<128>(p, 32 * k, wn * 32 + 16 * j, lane);
  };
  // ends the phase's reading, multiplies by both halves of x, ends the phase
  const auto multiply = [&](int hg) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int hx = 0; hx < 2; hx++)
#pragma unroll
      for (int k = 0; k < 2; k++)
#pragma unroll
        for (int i = 0; i < 4; i++)
#pragma unroll
          for (int j = 0; j < 2; j++)
            acc[hg * 4 + i][hx * 2 + j] =
                __builtin_amdgcn_mfma_f32_16x16x32_bf16(fg[i][k], fx[hx][j][k], acc[hg * 4 + i][hx * 2 + j], 0, 0, 0);
    __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
  };
  const auto landed8 = [] { asm volatile("s_waitcnt vmcnt(8)" ::: "memory"); };

  fill(0, 0);
  fill(1, 0);
  fill(2, 0);
  fill(3, 0);
  fill(0, 1);
  fill(1, 1);
  fill(2, 1);
  landed8();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  if (wm == 1) __builtin_amdgcn_s_barrier();
  for (int s = 0; s < steps; s++) {
    const int stage = s & 1;
    read_g(0, stage);
    read_x(0, stage);
    read_x(1, stage);
    fill(3, s + 1);
    landed8();
    multiply(0);
    read_g(1, stage);
    fill(0, s + 2);
    fill(1, s + 2);
    fill(2, s + 2);
    landed8();
    multiply(1);
  }
  if (wm == 0) __builtin_amdgcn_s_barrier();
  // LDS is the epilogue's once every wavefront's loads have landed
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  // 32 rows at a time through the wavefront's part of LDS, so that a lane stores eight neighbours
  float* const st = reinterpret_cast<float*>(lds) + wave * kSlab;
  const int c = (lane & 7) * 8;
  const int64_t k = k0 + wn * 64 + c, nw = n0 + wm * 128;
  const int some = (int)(a.cols - k < 0 ? 0 : a.cols - k < 8 ? a.cols - k : 8);
#pragma unroll
  for (int s = 0; s < 4; s++) {
#pragma unroll
    for (int i = 0; i < 2; i++)
#pragma unroll
      for (int j = 0; j < 4; j++)
#pragma unroll
        for (int e = 0; e < 4; e++)
          st[(16 * i + 4 * (lane >> 4) + e) * kSlabPitch + 16 * j + (lane & 15)] = acc[2 * s + i][j][e];
    wave_lds_fence();
#pragma unroll
    for (int p = 0; p < 32; p += 8) {
      const int r = p + (lane >> 3);
      const int64_t n = nw + 32 * s + r;
      float v[8];
#pragma unroll
      for (int q = 0; q < 8; q++) v[q] = st[r * kSlabPitch + c + q];
      if (n >= a.rows) continue;
      if (part)
        store_piece<false>(part, ((int64_t)split * a.rows + n) * part_pitch(a.cols) + k, v, some);
      else
        store_piece(a.dweight, n * a.dweight_stride + k, v, some, a.dweight_dtype == QUASAR_BF16);
    }
    wave_lds_fence();
  }
}

// dweight from the sums of `splits` shares of the tokens, eight values a thread.
__global__ __launch_bounds__(256) void weight_grad_join_kernel(quasar_weight_grad a, const float* part, int splits) {
  const int64_t pitch = part_pitch(a.cols), per = pitch / 8, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t n = i / per, k = (i - n * per) * 8;
  if (n >= a.rows) return;
  float v[8] = {};
  for (int s = 0; s < splits; s += 8) {  // eight shares in flight at once
    Piece<kElemF32> p[8];
#pragma unroll
    for (int j = 0; j < 8; j++)
      if (s + j < splits) p[j].load(part, ((s + j) * a.rows + n) * pitch + k, (int)(a.cols - k));
#pragma unroll
    for (int j = 0; j < 8; j++)
      if (s + j < splits) {
#pragma unroll
        for (int q = 0; q < 8; q++) v[q] += p[j].get(q);
      }
  }
  store_piece(a.dweight, n * a.dweight_stride + k, v, (int)(a.cols - k), a.dweight_dtype == QUASAR_BF16);
}

// The tile kernel loads rows of 16-byte pieces: dy as it is, if it is that.
bool direct(const quasar_weight_grad& a) {
  return a.dy_dtype == QUASAR_BF16 && a.rows % 8 == 0 && a.dy_stride % 8 == 0 && a.dy_stride <= kMaxPitch &&
         (reinterpret_cast<uintptr_t>(a.dy) & 15) == 0;
}

struct Choice {
  int tile, splits, steps;  // values a side; shares of the tokens, and the steps of each
  int64_t tiles_n, tiles;
  int64_t padded, np, kp, parts;   // the tile kernel's tokens and columns, and the parts of dy
  int64_t rest;                    // the tokens from here on are copied
  size_t x_bytes, dy_bytes, bytes;  // workspace: x, dy, and all of it with the shares' sums
};

Choice choose(const quasar_weight_grad& a) {
  const int64_t tokens = a.tokens, rows = a.rows, cols = a.cols;
  Choice c{};
  const auto tiles_of = [&](int b) { return ((rows + b - 1) / b) * ((cols + b - 1) / b); };
  const int64_t steps = tokens > 0 ? (tokens + kStep - 1) / kStep : 1;
  c.splits = 1;
  c.parts = a.dy_dtype == QUASAR_F32 ? 3 : 1;
  int64_t all = steps;
  if (tiles_of(256) >= 128 && steps >= 8 && rows <= kMaxPitch && cols <= kMaxPitch) {
    c.tile = 256;
    c.tiles = tiles_of(256);
    c.padded = steps * kStep;
    c.np = (rows + 7) & ~(int64_t)7;
    c.kp = (cols + 7) & ~(int64_t)7;
    c.x_bytes = (size_t)(c.padded * c.kp * 2);
    c.rest = direct(a) ? tokens / kStep * kStep : 0;
    c.dy_bytes = (size_t)(c.parts * (c.padded - c.rest) * c.np * 2);
    all = c.parts * steps;
    while (c.splits < 32 && 2 * c.tiles * c.splits <= kCUs && all >= 2 * c.splits * 16) c.splits *= 2;
  } else {
    c.tile = tiles_of(128) >= kCUs && a.dy_dtype == QUASAR_BF16 ? 128 : 64;
    c.tiles = tiles_of(c.tile);
    while (c.splits < 32 && 2 * c.tiles * c.splits <= 4 * kCUs && steps >= 2 * c.splits * 4) c.splits *= 2;
  }
  c.tiles_n = (rows + c.tile - 1) / c.tile;
  c.steps = (int)((all + c.splits - 1) / c.splits);
  c.splits = (int)((all + c.steps - 1) / c.steps);
  c.bytes = c.x_bytes + c.dy_bytes;
  if (c.splits > 1) c.bytes += (size_t)c.splits * (size_t)rows * (size_t)part_pitch(cols) * 4;
  return c;
}

template <int GT, int B>
void launch_tiles(const quasar_weight_grad& a, const Choice& c, float* part, hipStream_t stream) {
  weight_grad_kernel<GT, B><<<dim3((unsigned)(c.tiles * c.splits)), dim3(256), 0, stream>>>(a, (int)c.tiles_n, c.splits, c.steps,
                                                                                            part);
}

hipError_t launch_large(const quasar_weight_grad& a, const Choice& c, float* part, hipStream_t stream) {
  char* const ws = reinterpret_cast<char*>(a.workspace);
  const int steps = (int)(c.padded / kStep);
  const int64_t copied = c.padded - c.rest;
  Spread s{reinterpret_cast<uint16_t*>(ws), reinterpret_cast<uint16_t*>(ws + c.x_bytes), c.padded * (c.kp / 8), copied * (c.np / 8),
           c.padded, c.rest, Divide((uint32_t)(c.kp / 8)), Divide((uint32_t)(c.np / 8))};
  const int64_t groups = (s.x_pieces + s.dy_pieces + 255) / 256, most = 32 * kCUs;
  const dim3 grid((unsigned)(groups < most ? groups : most));
  if (a.dy_dtype == QUASAR_F32)
    spread_kernel<kElemF32><<<grid, dim3(256), 0, stream>>>(a, s);
  else
    spread_kernel<kElemBF16><<<grid, dim3(256), 0, stream>>>(a, s);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  Operands op{reinterpret_cast<const uint16_t*>(a.dy), s.dy, s.x, (int)(c.rest > 0 ? a.dy_stride : 0), (int)c.np, (int)c.kp,
              (int)c.np, (int)(c.rest / kStep), steps, (int)c.parts * steps};
  weight_grad_tile_kernel<<<dim3((unsigned)(c.tiles * c.splits)), dim3(512), 0, stream>>>(
      a, op, (int)c.tiles_n, (int)(c.tiles / c.tiles_n), c.steps, part);
  return hipGetLastError();
}

}  // namespace

bool weight_grad_fits(const quasar_weight_grad& a, size_t& workspace) {
  const Choice c = choose(a);
  workspace = c.bytes;
  return c.tiles * c.splits <= most_groups(c.tile == 256 ? 512 : 256) && (c.splits == 1 || a.rows * (part_pitch(a.cols) / 8) <= 256 * most_groups(256));
}

hipError_t launch_weight_grad(const quasar_weight_grad& a, hipStream_t stream) {
  const Choice c = choose(a);
  float* const part = c.splits > 1 ? reinterpret_cast<float*>(reinterpret_cast<char*>(a.workspace) + c.x_bytes + c.dy_bytes) : nullptr;
  hipError_t e = hipSuccess;
  if (c.tile == 256)
    e = launch_large(a, c, part, stream);
  else if (a.dy_dtype == QUASAR_F32)
    launch_tiles<kElemF32, 64>(a, c, part, stream);
  else if (c.tile == 64)
    launch_tiles<kElemBF16, 64>(a, c, part, stream);
  else
    launch_tiles<kElemBF16, 128>(a, c, part, stream);
  if (e == hipSuccess) e = hipGetLastError();
  if (e != hipSuccess || !part) return e;
  const int64_t n = a.rows * (part_pitch(a.cols) / 8);
  weight_grad_join_kernel<<<dim3((unsigned)((n + 255) / 256)), dim3(256), 0, stream>>>(a, part, c.splits);
  return hipGetLastError();
}

}  // namespace quasar
