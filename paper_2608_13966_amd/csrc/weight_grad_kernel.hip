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
constexpr int64_t kMaxPitch = 1 << 22;       // elements of a row (no weight has more) whose bytes the tile kernel reckons in 24 bits

__host__ __device__ constexpr int64_t part_pitch(int64_t cols) { return (cols + 7) & ~(int64_t)7; }

// Eight E4M3 bytes times a power of two as packed bf16, exact.
__device__ __forceinline__ uint4 kept_bf16(uint2 q, float f) {
  return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q.x, f, false)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q.x, f, true)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q.y, f, false)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q.y, f, true)));
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
// 32 rows from t0 on.  (APART: its groups of four columns lie so far apart.)
template <int W, int APART = 4>
__device__ __forceinline__ bf16x8 read_tile(const uint16_t* lds, int t0, int col, int lane) {
  const int t = t0 + 8 * (lane >> 4) + ((lane & 15) >> 2), c = col + APART * (lane & 3);
  typedef __attribute__((address_space(3))) s16x4 lds4;
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(lds + spot<W>(t, c)));
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(lds + spot<W>(t + 4, c)));
  typedef short s16x8 __attribute__((ext_vector_type(8)));
  const s16x8 r = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  return __builtin_bit_cast(bf16x8, r);
}

// A workgroup makes 64 x 64 values of dweight (or of its share's sums in part) from
// its share of the tokens, 64 at a time: the next two steps' pieces come to registers
// while one is multiplied (with one step's, 777 tokens, 1000 x 1544 took 20.6 us, not
// 14; four steps' were no faster).  Four wavefronts of 32 x 32.
template <int GT>
__global__ __launch_bounds__(256) void weight_grad_kernel(quasar_weight_grad a, int tiles_n, int splits, int steps_per, float* part) {
  constexpr int B = 64;
  constexpr int kParts = GT == kElemF32 ? 3 : 1, kPieces = kStep * B / 8 / 256, T = B / 32;
  // two stages where they are small: the next step is written while one is read (fp32's would leave fewer workgroups)
  constexpr int kStages = GT == kElemF32 ? 1 : 2, kStage = (kParts + 1) * kStep * B, kX = kParts * kStep * B;
  __shared__ __align__(16) uint16_t lds[kStages * kStage];
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_index();
  // neighbouring tiles on an XCD, whose L2 then holds what they read: 10308 tokens, 6825 x 216 109 us, else 165; 12011, 1743 x
  // 1459 171, 269; 777, 1000 x 1544 14, 14
  const int tiles = (int)(gridDim.x / (unsigned)splits), u = stretch_of(blockIdx.x, gridDim.x), split = u / tiles;
  int tn, tk;
  tile_at(u - split * tiles, tiles_n, tiles / tiles_n, tn, tk);
  const int64_t n0 = (int64_t)tn * B, k0 = (int64_t)tk * B;
  const int64_t t0 = (int64_t)split * steps_per * kStep;
  const int64_t t1 = t0 + (int64_t)steps_per * kStep < a.tokens ? t0 + (int64_t)steps_per * kStep : a.tokens;

  // this thread's pieces: columns 8 c of rows tr + i * (rows of a round)
  constexpr int kWide = B / 8, kRound = 256 / kWide;
  const int c = (tid % kWide) * 8, tr = tid / kWide;
  const int ln = (int)(a.rows - n0 - c < 8 ? a.rows - n0 - c : 8), lk = (int)(a.cols - k0 - c < 8 ? a.cols - k0 - c : 8);
  struct Fetched {
    Piece<GT> g[kPieces];
    uint2 q[kPieces];
    uint32_t e[kPieces];
  } f[2];
  // Whole pieces without a branch (the compiler would wait for all of them where a branch ends): past a row's end is the
  // next row, and columns past the matrix reach nothing that is stored; those of a thread without any are the first ones.
  // A thread's places in a step are 32-bit offsets from the step's first row.
  const int64_t gn = ln > 0 ? n0 + c : 0, qk = lk > 0 ? k0 + c : 0;
  constexpr int kSize = elem_size<GT>();
  uint32_t g_at[kPieces], q_at[kPieces], e_at[kPieces];
#pragma unroll
  for (int i = 0; i < kPieces; i++) {
    const int64_t r = tr + i * kRound;
    g_at[i] = (uint32_t)((r * a.dy_stride + gn) * kSize);
    q_at[i] = (uint32_t)(r * a.q_stride + qk);
    e_at[i] = (uint32_t)(r * a.exponent_stride + (qk >> 7));
  }
  const auto fetch = [&](Fetched& o, int64_t t) {
    const char* const g = reinterpret_cast<const char*>(a.dy) + t * a.dy_stride * kSize;
    const uint8_t *const q = a.q + t * a.q_stride, *const e = a.exponent + t * a.exponent_stride;
#pragma unroll
    for (int i = 0; i < kPieces; i++) {
      o.g[i].load(g + g_at[i], 0, 8);
      o.q[i] = ld8_any(q + q_at[i]);
      o.e[i] = e[e_at[i]];
    }
  };
  // near the last token: nothing past it
  const auto fetch_some = [&](Fetched& o, int64_t t) {
#pragma unroll
    for (int i = 0; i < kPieces; i++) {
      const int64_t r = t + tr + i * kRound;
      const bool has = r < t1;
      o.g[i].load(a.dy, has ? r * a.dy_stride + n0 + c : 0, has ? ln : 0);
      o.q[i] = load_bytes(has ? a.q + r * a.q_stride + k0 + c : a.q, has ? lk : 0);
      o.e[i] = has && lk > 0 ? a.exponent[r * a.exponent_stride + ((k0 + c) >> 7)] : 127u;
    }
  };
  const auto stage = [&](const Fetched& o, int to) {
    uint16_t* const p = lds + to * kStage;
#pragma unroll
    for (int i = 0; i < kPieces; i++) {
      const int at = spot<B>(tr + i * kRound, c);
      if constexpr (GT == kElemF32) {
        uint4 v[3];
        split3(o.g[i].f, v);
#pragma unroll
        for (int j = 0; j < 3; j++) *reinterpret_cast<uint4*>(p + j * kStep * B + at) = v[j];
      } else {
        *reinterpret_cast<uint4*>(p + at) = make_uint4(o.g[i].d[0], o.g[i].d[1], o.g[i].d[2], o.g[i].d[3]);
      }
      *reinterpret_cast<uint4*>(p + kX + at) = kept_bf16(o.q[i], as_f32(o.e[i] << 23));
    }
  };
  f32x4 acc[T][T];
#pragma unroll
  for (int i = 0; i < T; i++)
#pragma unroll
    for (int j = 0; j < T; j++) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  const int wn = (wave >> 1) * (B / 2), wk = (wave & 1) * (B / 2);
  const auto meet = [&] {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  const auto multiply = [&](int from) {
    const uint16_t* const p = lds + from * kStage;
#pragma unroll
    for (int k = 0; k < kStep; k += 32) {
      bf16x8 mx[T];
#pragma unroll
      for (int j = 0; j < T; j++) mx[j] = read_tile<B>(p + kX, k, wk + 16 * j, lane);
#pragma unroll
      for (int q = 0; q < kParts; q++)
#pragma unroll
        for (int i = 0; i < T; i++) {
          const bf16x8 mg = read_tile<B>(p + q * kStep * B, k, wn + 16 * i, lane);
#pragma unroll
          for (int j = 0; j < T; j++) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(mg, mx[j], acc[i][j], 0, 0, 0);
        }
    }
  };
  // the steps whose pieces, eight elements past a row's end too, lie before the last token's row
  const int64_t safe = a.tokens - 8 < t1 ? a.tokens - 8 : t1;
  const bool near = a.dy_stride <= kMaxPitch && a.q_stride <= kMaxPitch && a.exponent_stride <= kMaxPitch;  // offsets fit
  const int whole = near && safe > t0 ? (int)((safe - t0) / kStep) : 0;
  const auto step_at = [&](int s) { return t0 + (int64_t)(s < whole ? s : whole - 1) * kStep; };  // past the last: it again
  if (whole > 0) {
    fetch(f[0], step_at(0));
    fetch(f[1], step_at(1));
    if constexpr (kStages == 2) {
      stage(f[0], 0);
      fetch(f[0], step_at(2));
    }
    // step s, the next one in o
    const auto step = [&](int s, Fetched& o) {
      if constexpr (kStages == 2) {
        meet();  // the step is written, and all are done with the one before
        const uint16_t* const p = lds + (s & 1) * kStage;
        bf16x8 mx[2][T], mg[2][T];
#pragma unroll
        for (int k = 0; k < 2; k++)
#pragma unroll
          for (int j = 0; j < T; j++) {
            mx[k][j] = read_tile<B>(p + kX, 32 * k, wk + 16 * j, lane);
            mg[k][j] = read_tile<B>(p, 32 * k, wn + 16 * j, lane);
          }
        stage(o, (s + 1) & 1);
        fetch(o, step_at(s + 3));
#pragma unroll
        for (int k = 0; k < 2; k++)
#pragma unroll
          for (int i = 0; i < T; i++)
#pragma unroll
            for (int j = 0; j < T; j++) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(mg[k][i], mx[k][j], acc[i][j], 0, 0, 0);
      } else {
        stage(o, 0);
        fetch(o, step_at(s + 2));
        meet();
        multiply(0);
        meet();
      }
    };
    for (int s = 0; s < whole; s += 2) {
      step(s, f[kStages == 2 ? 1 : 0]);
      if (s + 1 < whole) step(s + 1, f[kStages == 2 ? 0 : 1]);
    }
    meet();
  }
  for (int64_t t = t0 + (int64_t)whole * kStep; t < t1; t += kStep) {
    fetch_some(f[0], t);
    stage(f[0], 0);
    meet();
    multiply(0);
    meet();
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

// ---- few tokens ---------------------------------------------------------------------
// Up to 128 tokens: one step is all there is, and writing dweight is what takes the time.  A workgroup makes 128 rows x
// 256 columns (128 past 64 tokens) from operands that it stages once; a wavefront keeps its columns of x in registers,
// reads 16 rows of dy at a time and stores from where the products are: x is the first operand, so that a lane has
// neighbours of a row.  bf16, us (a fill of dweight's bytes; the other kernels): 16 tokens, 8192 x 8192 in fp32 42 (40;
// 65), in bf16 22 (20; 44); 4, 14336 x 4096 37 (35; 62); 96, 4096 x 4096 15 (10; 25).  Past the caches 73, not 42.
template <int GT, int KS>
struct Few {
  static constexpr int P = KS > 2 ? 1 : 2;                          // 32-column parts of a wavefront
  static constexpr int N = GT == kElemF32 && KS > 2 ? 64 : 128, K = 128 * P;  // rows and columns of a workgroup
};
template <int GT, int KS, bool WB>
__global__ __launch_bounds__(256) void weight_grad_few_kernel(quasar_weight_grad a, int tiles_k) {
  constexpr int N = Few<GT, KS>::N, K = Few<GT, KS>::K, P = Few<GT, KS>::P, R = 32 * KS, kParts = GT == kElemF32 ? 3 : 1;
  constexpr int kXRow = K / 8, kXRows = 256 / kXRow, kX = R / kXRows, kGRow = N / 8, kGRows = 256 / kGRow, kG = R / kGRows;
  __shared__ __align__(16) uint16_t lds[R * K + kParts * R * N];
  uint16_t* const lds_g = lds + R * K;
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_index();
  const int u = stretch_of(blockIdx.x, gridDim.x), tn = u / tiles_k;
  const int64_t n0 = (int64_t)tn * N, k0 = (int64_t)(u - tn * tiles_k) * K;
  // this thread's pieces: eight columns of a row of each round.  Whole ones without a branch: a row past the last
  // token is the last one's and becomes 0, a piece past a row's end is the row's last (nothing of it is stored)
  const int xc = (tid % kXRow) * 8, xr = tid / kXRow, gc = (tid % kGRow) * 8, gr = tid / kGRow, last = (int)a.tokens - 1;
  const int lk = (int)(a.cols - k0 - xc < 8 ? a.cols - k0 - xc : 8), ln = (int)(a.rows - n0 - gc < 8 ? a.rows - n0 - gc : 8);
  const int64_t xk = lk < 8 ? a.cols - 8 : k0 + xc, gn = ln < 8 ? a.rows - 8 : n0 + gc;
  const int64_t block = (lk > 0 ? k0 + xc : a.cols - 1) >> 7;
  uint2 q[kX];
  uint32_t e[kX];
  Piece<GT> g[kG];
#pragma unroll
  for (int i = 0; i < kX; i++) {
    const int t = xr + kXRows * i < last ? xr + kXRows * i : last;
    q[i] = ld8_any(a.q + t * a.q_stride + xk);
    e[i] = a.exponent[t * a.exponent_stride + block];
  }
#pragma unroll
  for (int i = 0; i < kG; i++) {
    const int t = gr + kGRows * i < last ? gr + kGRows * i : last;
    g[i].load(a.dy, t * a.dy_stride + gn, 8);
  }
  // a piece that the row's end cuts: its elements one by one
  if (lk > 0 && lk < 8) {
#pragma unroll
    for (int i = 0; i < kX; i++) {
      const int t = xr + kXRows * i < last ? xr + kXRows * i : last;
      const uint8_t* const p = a.q + t * a.q_stride + k0 + xc;
      uint32_t b[8];
#pragma unroll
      for (int j = 0; j < 8; j++) b[j] = p[j < lk ? j : 0];
      q[i] = make_uint2(b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24, b[4] | b[5] << 8 | b[6] << 16 | b[7] << 24);
    }
  }
  if (ln > 0 && ln < 8) {
#pragma unroll
    for (int i = 0; i < kG; i++) {
      const int t = gr + kGRows * i < last ? gr + kGRows * i : last;
      const int64_t at = t * a.dy_stride + n0 + gc;
      if constexpr (GT == kElemF32) {
#pragma unroll
        for (int j = 0; j < 8; j++) g[i].f[j] = reinterpret_cast<const float*>(a.dy)[at + (j < ln ? j : 0)];
      } else {
        const uint16_t* const p = reinterpret_cast<const uint16_t*>(a.dy) + at;
#pragma unroll
        for (int j = 0; j < 4; j++) g[i].d[j] = p[2 * j < ln ? 2 * j : 0] | (uint32_t)p[2 * j + 1 < ln ? 2 * j + 1 : 0] << 16;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kX; i++) {
    const int t = xr + kXRows * i;
    const uint4 v = kept_bf16(q[i], as_f32(e[i] << 23));
    *reinterpret_cast<uint4*>(lds + spot<K>(t, xc)) = t <= last ? v : make_uint4(0u, 0u, 0u, 0u);
  }
#pragma unroll
  for (int i = 0; i < kG; i++) {
    const int t = gr + kGRows * i;
    uint4 v[kParts];
    if constexpr (GT == kElemF32)
      split3(g[i].f, v);
    else
      v[0] = make_uint4(g[i].d[0], g[i].d[1], g[i].d[2], g[i].d[3]);
#pragma unroll
    for (int p = 0; p < kParts; p++)
      *reinterpret_cast<uint4*>(lds_g + p * R * N + spot<N>(t, gc)) = t <= last ? v[p] : make_uint4(0u, 0u, 0u, 0u);
  }
  __syncthreads();
  // Instruction h of part p has columns 32 p + 8 (0 .. 3) + 4 h + (0 .. 3), with an output in fp32 32 p + 16 h + (0 .. 15):
  // four lanes then store 64 neighbouring bytes
  constexpr int kApart = WB ? 8 : 4, kNext = WB ? 4 : 16;
  const int w0 = wave * (32 * P);
  bf16x8 mx[P][2][KS];
#pragma unroll
  for (int p = 0; p < P; p++)
#pragma unroll
    for (int h = 0; h < 2; h++)
#pragma unroll
      for (int k = 0; k < KS; k++) mx[p][h][k] = read_tile<K, kApart>(lds, 32 * k, w0 + 32 * p + kNext * h, lane);
  for (int s = 0; s < N && n0 + s < a.rows; s += 16) {
    f32x4 acc[P][2];
#pragma unroll
    for (int p = 0; p < P; p++)
#pragma unroll
      for (int h = 0; h < 2; h++) acc[p][h] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < KS; k++)
#pragma unroll
      for (int z = 0; z < kParts; z++) {
        const bf16x8 mg = read_tile<N>(lds_g + z * R * N, 32 * k, s, lane);
#pragma unroll
        for (int p = 0; p < P; p++)
#pragma unroll
          for (int h = 0; h < 2; h++) acc[p][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(mx[p][h][k], mg, acc[p][h], 0, 0, 0);
      }
    // acc[p][h][i]: row s + lane % 16, column 32 p + kNext h + kApart (lane / 16) + i
    const int64_t n = n0 + s + (lane & 15), k = k0 + w0 + kApart * (lane >> 4), at = n * a.dweight_stride + k;
    if (n >= a.rows) continue;
#pragma unroll
    for (int p = 0; p < P; p++) {
      if constexpr (WB) {
        const float v[8] = {acc[p][0][0], acc[p][0][1], acc[p][0][2], acc[p][0][3], acc[p][1][0], acc[p][1][1], acc[p][1][2], acc[p][1][3]};
        store_piece<true>(a.dweight, at + 32 * p, v, (int)(a.cols - k - 32 * p));
      } else {
#pragma unroll
        for (int h = 0; h < 2; h++) {
          const int left = (int)(a.cols - k) - 32 * p - 16 * h;
          float* const to = reinterpret_cast<float*>(a.dweight) + at + 32 * p + 16 * h;
          if (left >= 4) {
            st16_any(to, __builtin_bit_cast(uint4, acc[p][h]));
          } else {
#pragma unroll
            for (int i = 0; i < 3; i++)
              if (i < left) to[i] = acc[p][h][i];
          }
        }
      }
    }
  }
}

// ---- large weights ----------------------------------------------------------------
// x in bf16 with the tokens of a step side by side, [padded tokens / 64, kp, 64], 0 past
// the last token: a transposing load has half the rate of a plain one, so what is
// written out anyway is turned on the way.  And what the tile kernel cannot load of dy
// as it is: all of it in bf16 [padded tokens, np] (fp32: its three parts one after the
// other, which the products then run through as through three times the tokens), or the
// last, incomplete step's rows alone.
struct Spread {
  uint16_t *x, *dy;
  int64_t dy_pieces;  // of eight elements
  int64_t first;      // the first token that dy holds
  int steps, kp;
  unsigned x_groups;  // workgroups that write x: 64 tokens and 128 columns each
  Divide np8;         // pieces of a row
};

template <int GT>
__global__ __launch_bounds__(256) void spread_kernel(quasar_weight_grad a, Spread s) {
  if (blockIdx.x < s.x_groups) {
    __shared__ __align__(16) uint16_t lds[kStep * 128];
    const int step = blockIdx.x % (unsigned)s.steps, block = blockIdx.x / (unsigned)s.steps, c = (threadIdx.x & 15) * 8;
    const int left = (int)a.cols - block * 128 - c;
    uint2 q[4];
    uint32_t e[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int64_t t = (int64_t)step * kStep + (threadIdx.x >> 4) + 16 * i;
      const bool has = t < a.tokens;
      q[i] = load_bytes(has ? a.q + t * a.q_stride + block * 128 + c : a.q, has ? left : 0);
      e[i] = has ? a.exponent[t * a.exponent_stride + block] : 127u;
    }
#pragma unroll
    for (int i = 0; i < 4; i++)
      *reinterpret_cast<uint4*>(lds + spot<128>((threadIdx.x >> 4) + 16 * i, c)) = kept_bf16(q[i], as_f32(e[i] << 23));
    __syncthreads();
    const int lane = threadIdx.x & 63, wave = wave_index();
    uint16_t* const out = s.x + ((int64_t)step * s.kp + block * 128) * kStep;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int tile = wave * 2 + (i >> 1), k = tile * 16 + (lane & 15), t0 = (i & 1) * 32;
      const bf16x8 v = read_tile<128>(lds, t0, tile * 16, lane);
      if (block * 128 + k < s.kp) st128(out + k * kStep + t0 + 8 * (lane >> 4), __builtin_bit_cast(uint4, v));
    }
    return;
  }
  const int64_t step = (int64_t)(gridDim.x - s.x_groups) * 256;
  for (int64_t j = (int64_t)(blockIdx.x - s.x_groups) * 256 + threadIdx.x; j < s.dy_pieces; j += step) {
    const int64_t r = j / s.np8.by, t = r + s.first;
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

// The operands of the tile kernel: rows of dy up to step `whole`, then from `rest`;
// x repeats after `period` steps.
struct Operands {
  const uint16_t *dy, *rest, *x;
  int dy_stride, rest_stride, kp, np;  // elements; np: columns that dy has
  int whole, period, steps;
};

// In LDS, 16-byte chunk c of x's column m lies at chunk c ^ (m / 2 % 8) of the
// column's 128 bytes: the 16 columns that an operand read or a store touches at one
// chunk then lie in 16 different groups of four banks.
__device__ __forceinline__ int chunk_at(int m, int c) { return m * kStep + 8 * (c ^ ((m >> 1) & 7)); }

// A workgroup makes 256 x 256 values of dweight with 8 wavefronts of 64 rows x 128
// columns, 64 tokens a step.  Both operands of a step lie in LDS as two halves each, g0
// and x0 the first 128 rows and columns (of dy whole lines of memory), 32 and 64 of
// them a wavefront's, g1 and x1 the rest; and a step has two phases, each with 32
// matrix instructions a wavefront: x0 (g0 g1), x1 (g0 g1).  The reads are spread evenly:
// phase 0 reads x0 and g1, phase 1 x1 and the next step's g0.  Two stages; a half is
// filled again as soon as all have read it.
//
// 8192 tokens, 14336 x 4096, normal values, median of 140 passes on a busy card: the call
// takes 740 us (26 spread the operands, 18 join the shares), 1.30 PFLOP/s; beside it a
// library product of bf16 operands that lie along the summed dimension takes 631, of dy
// and x as they lie here 947.  (Cards differ: 755, 700 to 735 and 1030 on another.  After
// a rest the first twenty calls of this kernel take 706, up to 966 and 734 as the clocks
// settle.)  Matrix units are busy 73% of the time, and the card's power is part of the
// bound.  On the way, on one cool card (us): both operands through transposing loads, three
// quarters of a step's reads in its first phase 882; halves of half lines of dy 922, of
// whole ones 795; the tiles past whole rounds shared out 747; addresses that go on a step
// at a time 727; loads ahead of reads 719, and 619 with all-zero operands.  32 x 32 x 16
// instructions took 777, not 747.
//
// The wavefronts of a SIMD work in turn: those of wk = 1 run one barrier behind, so
// that while one multiplies the other reads its next operands.  Barriers 2p and 2p + 1
// end the reading and the multiplying of phase p for wk = 0, 2p + 1 and 2p + 2 for wk
// = 1; a wavefront has its operands before it comes to the barrier that ends the
// reading.  Hence
//  - a half filled in phase p may be one whose last reads were in phase p - 1: x0 and
//    g1, read in a step's phase 0, are filled for the step after the next in its phase
//    1; x1 in the next step's phase 0; g0, read in the phase 1 before, in phase 0;
//  - what phase p reads has to have landed for every wavefront's own loads before the
//    barrier that ends its reading of phase p - 1: it was filled in phase p - 3, and
//    p - 2 and p - 1 have issued four loads each since: "at most 8 outstanding".
// Past the last step the loads repeat it, so that the counts hold.
constexpr int kSlabPitch = 128 + 4, kSlab = 16 * kSlabPitch;
__global__ __launch_bounds__(512, 2) void weight_grad_tile_kernel(quasar_weight_grad a, Operands op, int tiles_n, int tiles_k,
                                                                  int whole, int shared, int splits, int steps_per, float* part) {
  constexpr int kHalf = kStep * 128, kStage = 4 * kHalf;  // elements; halves g0, g1, x0, x1
  __shared__ __align__(16) uint16_t lds[2 * kStage];
  static_assert(8 * kSlab * 4 <= (int)sizeof(lds), "the epilogue's stage fits");
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)lds;
  const int lane = threadIdx.x & 63, wave = wave_index();
  const int wk = wave >> 2, wn = wave & 3;
  // the first `whole` tiles are a workgroup's each, the last `shared` ones that of `splits`
  int tile, split = 0, tn, tk;
  if ((int)blockIdx.x < whole) {
    tile = stretch_of(blockIdx.x, whole);
    steps_per = op.steps;
    part = nullptr;
  } else {
    const int u = stretch_of(blockIdx.x - whole, shared * splits);
    split = u / shared;
    tile = whole + (u - split * shared);
    if (part) part += ((int64_t)(tile - whole) * splits + split) * (256 * 256);
  }
  tile_at(tile, tiles_n, tiles_k, tn, tk);
  const int64_t n0 = (int64_t)tn * 256, k0 = (int64_t)tk * 256;
  const int first = split * steps_per, left = op.steps - first, steps = left < steps_per ? left : steps_per;

  // each wavefront loads 8 rows of a half of dy, 4 an instruction, and 16 columns of a half of x, 8 an
  // instruction; rows and columns past the matrix repeat its last ones
  uint32_t row[2], g_col[2][2], x_at[2][2];
#pragma unroll
  for (int i = 0; i < 2; i++) {
    const int t = wave * 8 + i * 4 + (lane >> 4);
    const int f = (t & 3) | ((t >> 1) & 4), c = ((((lane & 15) >> 1) ^ f) << 4) + (lane & 1) * 8;
    const int m = wave * 16 + i * 8 + (lane >> 3);
    row[i] = (uint32_t)t;
#pragma unroll
    for (int h = 0; h < 2; h++) {
      const int n = (int)n0 + h * 128 + c, k = (int)k0 + h * 128 + m;
      g_col[h][i] = 2u * (uint32_t)(n < op.np - 8 ? n : op.np - 8);
      x_at[h][i] = 2u * (uint32_t)((k < op.kp ? k : op.kp - 1) * kStep + 8 * ((lane & 7) ^ ((m >> 1) & 7)));
    }
  }
  // where the next step to be filled lies, a step on at a time; past the last step it stays
  int g_step = first, x_step = first;
  const bool in_rest = first >= op.whole;
  uint32_t pitch = 2u * (uint32_t)(in_rest ? op.rest_stride : op.dy_stride);
  const char* g_from = reinterpret_cast<const char*>(in_rest ? op.rest : op.dy) + (int64_t)(first - (in_rest ? op.whole : 0)) * kStep * pitch;
  const int64_t g_pace = (int64_t)kStep * pitch, x_pace = (int64_t)op.kp * (2 * kStep);
  const char* x_from = reinterpret_cast<const char*>(op.x) + (int64_t)(first % op.period) * x_pace;
  int x_left = op.period - 1 - first % op.period;  // steps until x begins again
  const auto next_g = [&] {
    if (g_step + 1 >= first + steps) return;
    g_from += g_pace;
    if (++g_step == op.whole) {
      g_from = reinterpret_cast<const char*>(op.rest);
      pitch = 2u * (uint32_t)op.rest_stride;
    }
  };
  const auto next_x = [&] {
    if (x_step + 1 >= first + steps) return;
    x_step++;
    x_from += x_pace;
    if (x_left-- == 0) {
      x_from = reinterpret_cast<const char*>(op.x);
      x_left = op.period - 1;
    }
  };
  const auto fill_g = [&](int h, int stage) {
    const uint32_t to = lds0 + (stage * kStage + h * kHalf + wave * 8 * 128) * 2;
#pragma unroll
    for (int i = 0; i < 2; i++) load_lds16(g_from, __umul24(row[i], pitch) + g_col[h][i], to + i * 4 * 128 * 2);
  };
  const auto fill_x = [&](int h, int stage) {
    const uint32_t to = lds0 + (stage * kStage + (2 + h) * kHalf + wave * 16 * kStep) * 2;
#pragma unroll
    for (int i = 0; i < 2; i++) load_lds16(x_from, x_at[h][i], to + i * 8 * kStep * 2);
  };
  f32x4 acc[4][8];
#pragma unroll
  for (int i = 0; i < 4; i++)
#pragma unroll
    for (int j = 0; j < 8; j++) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  bf16x8 fg[2][2][2], next[2][2], fx[4][2];
  const auto read_g = [&](int h, int stage, bf16x8 (&to)[2][2]) {
    const uint16_t* p = lds + stage * kStage + h * kHalf;
#pragma unroll
    for (int i = 0; i < 2; i++)
#pragma unroll
      for (int k = 0; k < 2; k++) to[i][k] = read_tile<128>(p, 32 * k, wn * 32 + 16 * i, lane);
  };
  const auto read_x = [&](int h, int stage) {
    const uint16_t* p = lds + stage * kStage + (2 + h) * kHalf;
#pragma unroll
    for (int j = 0; j < 4; j++)
#pragma unroll
      for (int k = 0; k < 2; k++)
        fx[j][k] = __builtin_bit_cast(
            bf16x8, *reinterpret_cast<const uint4*>(p + chunk_at(wk * 64 + 16 * j + (lane & 15), 4 * k + (lane >> 4))));
  };
  // ends the phase's reading, multiplies by both halves of dy, ends the phase
  const auto multiply = [&](int hx) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int hg = 0; hg < 2; hg++)
#pragma unroll
      for (int k = 0; k < 2; k++)
#pragma unroll
        for (int i = 0; i < 2; i++)
#pragma unroll
          for (int j = 0; j < 4; j++)
            acc[hg * 2 + i][hx * 4 + j] =
                __builtin_amdgcn_mfma_f32_16x16x32_bf16(fg[hg][i][k], fx[j][k], acc[hg * 2 + i][hx * 4 + j], 0, 0, 0);
    __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
  };
  const auto landed8 = [] { asm volatile("s_waitcnt vmcnt(8)" ::: "memory"); };

  fill_g(0, 0);
  fill_x(0, 0);
  fill_g(1, 0);
  fill_x(1, 0);
  next_g();
  next_x();
  fill_g(0, 1);
  fill_x(0, 1);
  fill_g(1, 1);
  next_g();
  landed8();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  read_g(0, 0, fg[0]);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();  // g0 may be filled again
  asm volatile("" ::: "memory");
  if (wk == 1) __builtin_amdgcn_s_barrier();
  for (int s = 0; s < steps; s++) {
    const int stage = s & 1;
    fill_x(1, stage ^ 1);
    fill_g(0, stage);
    read_x(0, stage);
    read_g(1, stage, fg[1]);
    next_x();
    landed8();
    multiply(0);
    fill_x(0, stage);
    fill_g(1, stage);
    read_x(1, stage);
    read_g(0, stage ^ 1, next);
    next_g();
    landed8();
    multiply(1);
#pragma unroll
    for (int i = 0; i < 2; i++)
#pragma unroll
      for (int k = 0; k < 2; k++) fg[0][i][k] = next[i][k];
  }
  if (wk == 0) __builtin_amdgcn_s_barrier();
  // LDS is the epilogue's once every wavefront's loads have landed
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  // 16 rows at a time through the wavefront's part of LDS, so that a lane stores eight neighbours
  float* const st = reinterpret_cast<float*>(lds) + wave * kSlab;
  const int c = (lane & 15) * 8;
  const int64_t k = k0 + (c >> 6) * 128 + wk * 64 + (c & 63);
  const int some = (int)(a.cols - k < 0 ? 0 : a.cols - k < 8 ? a.cols - k : 8);
#pragma unroll
  for (int i = 0; i < 4; i++) {
#pragma unroll
    for (int j = 0; j < 8; j++)
#pragma unroll
      for (int e = 0; e < 4; e++) st[(4 * (lane >> 4) + e) * kSlabPitch + 16 * j + (lane & 15)] = acc[i][j][e];
    wave_lds_fence();
#pragma unroll
    for (int p = 0; p < 16; p += 4) {
      const int r = p + (lane >> 4);
      const int n = (i >> 1) * 128 + wn * 32 + (i & 1) * 16 + r;
      float v[8];
#pragma unroll
      for (int q = 0; q < 8; q++) v[q] = st[r * kSlabPitch + c + q];
      if (part)
        store_piece<false>(part, n * 256 + (k - k0), v, 8);
      else if (n0 + n < a.rows)
        store_piece(a.dweight, (n0 + n) * a.dweight_stride + k, v, some, a.dweight_dtype == QUASAR_BF16);
    }
    wave_lds_fence();
  }
}

// dweight from the shares of the tiles from `whole` on, [tiles][splits][256][256], 32 workgroups a tile.
__global__ __launch_bounds__(256) void weight_grad_tile_join_kernel(quasar_weight_grad a, const float* part, int tiles_n, int tiles_k,
                                                                    int whole, int splits) {
  const int tile = blockIdx.x >> 5, i = (blockIdx.x & 31) * 256 + threadIdx.x;
  int tn, tk;
  tile_at(whole + tile, tiles_n, tiles_k, tn, tk);
  const int64_t n = (int64_t)tn * 256 + (i >> 5), k = (int64_t)tk * 256 + (i & 31) * 8;
  const int left = (int)(a.cols - k < 8 ? a.cols - k : 8);
  if (n >= a.rows || left <= 0) return;
  part += (int64_t)tile * splits * (256 * 256) + i * 8;
  float v[8] = {};
  for (int s = 0; s < splits; s += 8) {  // eight shares in flight at once
    Piece<kElemF32> p[8];
#pragma unroll
    for (int j = 0; j < 8; j++)
      if (s + j < splits) p[j].load(part, (int64_t)(s + j) * (256 * 256), 8);
#pragma unroll
    for (int j = 0; j < 8; j++)
      if (s + j < splits) {
#pragma unroll
        for (int q = 0; q < 8; q++) v[q] += p[j].get(q);
      }
  }
  store_piece(a.dweight, n * a.dweight_stride + k, v, left, a.dweight_dtype == QUASAR_BF16);
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
  int tile, splits, steps;  // values a side, 0: the kernel for few tokens; shares of the tokens, and the steps of each
  int64_t tiles_n, tiles;           // tiles a column of them, and all
  int64_t padded, np, kp, parts;   // the tile kernel's tokens and columns, and the parts of dy
  int64_t rest;                    // the tokens from here on are copied
  int64_t whole;                   // the tiles of one workgroup each
  size_t x_bytes, dy_bytes, bytes;  // workspace: x, dy, and all of it with the shares' sums
};

// The least time of both kernels over the shares that the tokens can be cut into, from what was measured of their parts
// (us).  A step of the 64 x 64 kernel takes 0.2, and 0.23 for each workgroup that a CU has, up to four (fp32: 0.6 and 0.52),
// a round of workgroups 2, and 0.8 for each, more.  A step of the tile kernel takes 1.3, in full rounds at the clock that
// the card then holds 1.5; a round 2 and what its tiles write at 6.9 TB/s; the launch that spreads its operands 7 and what
// it moves.  Shares cost a join of 5 and 3, and what they and it move.  (bf16, 64 x 64 against tiles, each at its best: 777
// tokens, 1000 x 1544 14, 30; 4096, 256 x 256 11, 24; 8192, 1024 x 1024 48, 48; 2048, 2048 x 2048 41, 45; 8192, 2048 x 2048
// 161, 86; 200, 4096 x 4096 38, 29; 1000 78, 47; 10308, 6824 x 216 101, 58, 6825 x 216 107, 101.  A 128 x 128 form of the
// first was never better by more than a tenth.)
constexpr double kMoved = 5.2e6;  // bytes a us

// f(type of dy, steps of 32 tokens)
template <typename F>
auto with_few(const quasar_weight_grad& a, F f) {
  using std::integral_constant;
  const auto steps = [&](auto gt) {
    if (a.tokens <= 32) return f(gt, integral_constant<int, 1>());
    if (a.tokens <= 64) return f(gt, integral_constant<int, 2>());
    if (a.tokens <= 96) return f(gt, integral_constant<int, 3>());
    return f(gt, integral_constant<int, 4>());
  };
  return a.dy_dtype == QUASAR_F32 ? steps(integral_constant<int, kElemF32>()) : steps(integral_constant<int, kElemBF16>());
}

Choice choose(const quasar_weight_grad& a) {
  // The kernel for few tokens where it has workgroups for half of the CUs (us, against the others: 64 tokens of 2048 x 2048
  // in 128 of them 8.4, 8.1, with dweight in bf16 5.9, 6.6; in 256 of 2048 x 4096 9.1, 12.8; 43 of 1347 x 2606 in 121 8.8, 8.3;
  // 33 of 1000 x 1000 in 32 6.2, 5.1).
  if (a.tokens >= 1 && a.tokens <= 128 && a.rows >= 8 && a.cols >= 8) {
    Choice few{};
    few.splits = few.steps = 1;
    (void)with_few(a, [&](auto gt, auto ks) {
      using Form = Few<decltype(gt)::value, decltype(ks)::value>;
      few.tiles_n = (a.rows + Form::N - 1) / Form::N;
      few.tiles = few.tiles_n * ((a.cols + Form::K - 1) / Form::K);
      return 0;
    });
    if (few.tiles >= kCUs / 2 && few.tiles <= most_groups(256)) return few;
  }
  const int64_t steps = a.tokens > 0 ? (a.tokens + kStep - 1) / kStep : 1;
  const int64_t out = a.rows * part_pitch(a.cols) * 4;
  const bool wide = a.dy_dtype == QUASAR_F32;
  Choice c{};
  double least = 0.0;
  const auto take = [&](double us, int tile, int64_t splits) {
    if (c.tile != 0 && us >= least) return;
    least = us;
    c.tile = tile;
    c.splits = (int)splits;
  };
  const int64_t small = ((a.rows + 63) / 64) * ((a.cols + 63) / 64);
  for (int64_t s = 1, last = 0; s <= 32 && s <= steps && (s == 1 || small * s <= 16 * kCUs); s++) {
    const int64_t per = (steps + s - 1) / s, groups = small * s;
    if (per == last) continue;  // as many steps a share
    last = per;
    const int64_t full = groups / (4 * kCUs), rest = (groups % (4 * kCUs) + kCUs - 1) / kCUs;
    const auto round = [&](double n) { return n == 0 ? 0.0 : 2.0 + 0.8 * n + (double)per * (wide ? 0.6 + 0.52 * n : 0.2 + 0.23 * n); };
    take((double)full * round(4) + round((double)rest) + (s == 1 ? 0.0 : 5.0 + (double)(out * 2 * s) / kMoved), 64, s);
  }
  const int64_t tiles = ((a.rows + 255) / 256) * ((a.cols + 255) / 256), whole = tiles / kCUs * kCUs, rest = tiles - whole;
  const int64_t parts = wide ? 3 : 1, all = parts * steps, padded = steps * kStep;
  const int64_t np = (a.rows + 7) & ~(int64_t)7, kp = (a.cols + 7) & ~(int64_t)7, from = direct(a) ? a.tokens / kStep * kStep : 0;
  // where its grids take it: the spread's workgroups, and the tiles with up to 32 shares of those past whole rounds
  if (steps * ((kp + 127) / 128) + 32 * kCUs <= most_groups(256) && tiles + 32 * kCUs <= most_groups(512)) {
    constexpr double kTile = 256 * 256 * 4 / 6.9e6;
    const auto round = [&](int64_t groups, int64_t per) {
      return 2.0 + (double)per * (1.3 + 0.2 * (double)groups / kCUs) + (double)groups * kTile;
    };
    const double spread = 7.0 + (double)(padded * kp * 3 + (padded - from) * np * (wide ? 10 : 4)) / kMoved +
                          (double)(whole / kCUs) * round(kCUs, all);
    if (rest == 0) take(spread, 256, 1);
    for (int64_t s = 1; rest > 0 && s <= 32 && s <= all; s++) {
      const int64_t per = (all + s - 1) / s, groups = rest * s, full = groups / kCUs, last = groups % kCUs;
      take(spread + (double)full * round(kCUs, per) + (last == 0 ? 0.0 : round(last, per)) +
               (s == 1 ? 0.0 : 3.0 + (double)groups * kTile),
           256, s);
    }
  }
  const int64_t b = c.tile, total = c.tile == 256 ? all : steps;
  c.tiles_n = (a.rows + b - 1) / b;
  c.tiles = c.tiles_n * ((a.cols + b - 1) / b);
  c.steps = (int)((total + c.splits - 1) / c.splits);
  c.splits = (int)((total + c.steps - 1) / c.steps);
  if (c.tile == 256) {
    c.parts = parts;
    c.padded = padded;
    c.np = np;
    c.kp = kp;
    c.rest = from;
    c.whole = whole;
    c.x_bytes = (size_t)(padded * kp * 2);
    c.dy_bytes = (size_t)(parts * (padded - from) * np * 2);
  }
  c.bytes = c.x_bytes + c.dy_bytes;
  if (c.splits > 1) c.bytes += (size_t)c.splits * (size_t)(c.tile == 256 ? rest * 256 * 256 * 4 : out);
  return c;
}

hipError_t launch_large(const quasar_weight_grad& a, const Choice& c, float* part, hipStream_t stream) {
  char* const ws = reinterpret_cast<char*>(a.workspace);
  const int steps = (int)(c.padded / kStep);
  const int64_t copied = c.padded - c.rest;
  const int64_t x_groups = steps * ((c.kp + 127) / 128), pieces = copied * (c.np / 8), most = 32 * kCUs;
  Spread s{reinterpret_cast<uint16_t*>(ws), reinterpret_cast<uint16_t*>(ws + c.x_bytes), pieces, c.rest, steps, (int)c.kp,
           (unsigned)x_groups, Divide((uint32_t)(c.np / 8))};
  const int64_t dy_groups = (pieces + 255) / 256;
  const dim3 grid((unsigned)(x_groups + (dy_groups < most ? dy_groups : most)));
  if (a.dy_dtype == QUASAR_F32)
    spread_kernel<kElemF32><<<grid, dim3(256), 0, stream>>>(a, s);
  else
    spread_kernel<kElemBF16><<<grid, dim3(256), 0, stream>>>(a, s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  Operands op{reinterpret_cast<const uint16_t*>(a.dy), s.dy, s.x, (int)(c.rest > 0 ? a.dy_stride : 0), (int)c.np, (int)c.kp,
              (int)c.np, (int)(c.rest / kStep), steps, (int)c.parts * steps};
  const int tiles_n = (int)c.tiles_n, tiles_k = (int)(c.tiles / c.tiles_n), whole = (int)c.whole, shared = (int)(c.tiles - c.whole);
  weight_grad_tile_kernel<<<dim3((unsigned)(whole + shared * c.splits)), dim3(512), 0, stream>>>(a, op, tiles_n, tiles_k, whole, shared,
                                                                                                 c.splits, c.steps, part);
  e = hipGetLastError();
  if (e != hipSuccess || !part) return e;
  weight_grad_tile_join_kernel<<<dim3((unsigned)shared * 32), dim3(256), 0, stream>>>(a, part, tiles_n, tiles_k, whole, c.splits);
  return hipGetLastError();
}

}  // namespace

bool weight_grad_fits(const quasar_weight_grad& a, size_t& workspace) {
  const Choice c = choose(a);
  workspace = c.bytes;
  if (c.tile != 64) return true;
  return c.tiles * c.splits <= most_groups(256) && (c.splits == 1 || a.rows * (part_pitch(a.cols) / 8) <= 256 * most_groups(256));
}

template <int GT, int KS>
hipError_t launch_few(const quasar_weight_grad& a, const Choice& c, hipStream_t stream) {
  const dim3 grid((unsigned)c.tiles);
  const int tiles_k = (int)(c.tiles / c.tiles_n);
  if (a.dweight_dtype == QUASAR_BF16)
    weight_grad_few_kernel<GT, KS, true><<<grid, dim3(256), 0, stream>>>(a, tiles_k);
  else
    weight_grad_few_kernel<GT, KS, false><<<grid, dim3(256), 0, stream>>>(a, tiles_k);
  return hipGetLastError();
}

hipError_t launch_weight_grad(const quasar_weight_grad& a, hipStream_t stream) {
  const Choice c = choose(a);
  float* const part = c.splits > 1 ? reinterpret_cast<float*>(reinterpret_cast<char*>(a.workspace) + c.x_bytes + c.dy_bytes) : nullptr;
  if (c.tile == 0) return with_few(a, [&](auto gt, auto ks) { return launch_few<decltype(gt)::value, decltype(ks)::value>(a, c, stream); });
  if (c.tile == 256) return launch_large(a, c, part, stream);
  const dim3 grid((unsigned)(c.tiles * c.splits));
  if (a.dy_dtype == QUASAR_F32)
    weight_grad_kernel<kElemF32><<<grid, dim3(256), 0, stream>>>(a, (int)c.tiles_n, c.splits, c.steps, part);
  else
    weight_grad_kernel<kElemBF16><<<grid, dim3(256), 0, stream>>>(a, (int)c.tiles_n, c.splits, c.steps, part);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !part) return e;
  const int64_t n = a.rows * (part_pitch(a.cols) / 8);
  weight_grad_join_kernel<<<dim3((unsigned)((n + 255) / 256)), dim3(256), 0, stream>>>(a, part, c.splits);
  return hipGetLastError();
}

}  // namespace quasar
