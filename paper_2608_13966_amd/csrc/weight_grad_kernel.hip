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
constexpr int kStep = 64;
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

struct Choice {
  int tile, splits, steps;  // values a side; shares of the tokens, and the steps of each
  int64_t tiles_n, tiles;
  size_t bytes;             // workspace
};

Choice choose(int64_t tokens, int64_t rows, int64_t cols, int dy_dtype) {
  Choice c{};
  const auto tiles_of = [&](int b) { return ((rows + b - 1) / b) * ((cols + b - 1) / b); };
  c.tile = tiles_of(128) >= kCUs && dy_dtype == QUASAR_BF16 ? 128 : 64;
  c.tiles_n = (rows + c.tile - 1) / c.tile;
  c.tiles = tiles_of(c.tile);
  const int64_t steps = tokens > 0 ? (tokens + kStep - 1) / kStep : 1;
  c.splits = 1;
  while (c.splits < 32 && 2 * c.tiles * c.splits <= 4 * kCUs && steps >= 2 * c.splits * 4) c.splits *= 2;
  c.steps = (int)((steps + c.splits - 1) / c.splits);
  c.splits = (int)((steps + c.steps - 1) / c.steps);
  if (c.splits > 1) c.bytes = (size_t)c.splits * (size_t)rows * (size_t)part_pitch(cols) * 4;
  return c;
}

template <int GT, int B>
void launch_tiles(const quasar_weight_grad& a, const Choice& c, float* part, hipStream_t stream) {
  weight_grad_kernel<GT, B><<<dim3((unsigned)(c.tiles * c.splits)), dim3(256), 0, stream>>>(a, (int)c.tiles_n, c.splits, c.steps,
                                                                                            part);
}

}  // namespace

bool weight_grad_fits(int64_t tokens, int64_t rows, int64_t cols, int dy_dtype, size_t& workspace) {
  const Choice c = choose(tokens, rows, cols, dy_dtype);
  workspace = c.bytes;
  return c.tiles * c.splits <= most_groups(256) && (c.splits == 1 || rows * (part_pitch(cols) / 8) <= 256 * most_groups(256));
}

hipError_t launch_weight_grad(const quasar_weight_grad& a, hipStream_t stream) {
  const Choice c = choose(a.tokens, a.rows, a.cols, a.dy_dtype);
  float* const part = c.splits > 1 ? reinterpret_cast<float*>(a.workspace) : nullptr;
  if (a.dy_dtype == QUASAR_F32)
    launch_tiles<kElemF32, 64>(a, c, part, stream);
  else if (c.tile == 64)
    launch_tiles<kElemBF16, 64>(a, c, part, stream);
  else
    launch_tiles<kElemBF16, 128>(a, c, part, stream);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !part) return e;
  const int64_t n = a.rows * (part_pitch(a.cols) / 8);
  weight_grad_join_kernel<<<dim3((unsigned)((n + 255) / 256)), dim3(256), 0, stream>>>(a, part, c.splits);
  return hipGetLastError();
}

}  // namespace quasar
