// checkpoint_kernel.hip -- activations kept in 8 bits, and the gradient of an
// activation function from what was kept (quasar_ops.h).
//
// A stretch of 128 columns is the work of 16 lanes, eight elements (16 bytes in
// bf16) each: the largest |x| is found by four lane exchanges, its exponent bits
// give the scale, and scaling by a power of two is exact, so q is rounded once.
// Both kernels are bound by memory, but not by far: GELU is 25 instructions an
// element, a reciprocal and an exponential among them.  8192 x 14336 bf16: kept alone
// 60 us, 5.8 TB/s; with ReLU's or SiLU's output 100 and 104, GELU's 114 (5.1); back 102
// to 105 (5.6).  Rows of 64 columns use half of their lanes: 1048576 of them, GELU 111.
#include "ops_common.h"
#include "ops_internal.h"

namespace quasar {
namespace {

// The kernels' 16-lane units, `per` (the stretches of a row) a row.
struct Units {
  uint32_t count;
  Divide per;
};

constexpr int kThreads = 256;

__device__ __forceinline__ uint32_t top_of_run16(uint32_t m) {
  m = max(m, dpp_u32<kDppXor1>(m));
  m = max(m, dpp_u32<kDppXor2>(m));
  m = max(m, dpp_u32<kDppHalfMirror>(m));
  return max(m, dpp_u32<kDppMirror>(m));
}

// The bits of the largest |element|; NaN and infinity are the largest.
__device__ __forceinline__ uint32_t top_bits(const Piece<kElemF32>& p) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; i++) m = max(m, as_u32(p.f[i]) & 0x7fffffffu);
  return m;
}
__device__ __forceinline__ uint32_t top_bits(const Piece<kElemBF16>& p) {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  u16x2 m = {0, 0};
#pragma unroll
  for (int i = 0; i < 4; i++) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, p.d[i] & 0x7fff7fffu));
  return (uint32_t)max(m.x, m.y) << 16;
}

constexpr uint32_t kInfBits = 0x7f800000u;

// act(x) in x's place, in fewer instructions than the products' epilogue has room for:
// SiLU's quotient by the hardware's reciprocal and one step of Newton's (within 8 x
// 2^-24; 8192 x 14336 in bf16 125 us with the division, 104 so), GELU without a
// selection (past 32 the tail is 0, and infinity times it not a number; 116, 114).
// GELU of -infinity, which is not a number either, is the caller's to see to: as NaN.
__device__ __forceinline__ void apply(float (&v)[8], int act) {
  if (act == QUASAR_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = v[i] < 0.0f ? 0.0f : v[i];  // NaN stays
  } else if (act == QUASAR_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const float e = exp_of(-fabsf(v[i])), d = 1.0f + e, r = __builtin_amdgcn_rcpf(d);
      v[i] = (v[i] >= 0.0f ? v[i] : v[i] * e) * __builtin_fmaf(r, __builtin_fmaf(-d, r, 1.0f), r);
    }
  } else if (act == QUASAR_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const float u = fabsf(v[i]), tail = normal_tail(u);
      v[i] = __builtin_fmaf(-min_f32(u, 32.0f), tail, max_f32(v[i], 0.0f));
    }
  }
}

// U units a thread, whose loads are issued together.
template <int XT, int U>
__global__ __launch_bounds__(kThreads) void checkpoint_kernel(quasar_checkpoint a, Units units) {
  const int lane = threadIdx.x & 15, cols = (int)a.cols;
  const uint32_t first = (blockIdx.x * (uint32_t)(kThreads / 16) * U) + (threadIdx.x >> 4);
  Piece<XT> p[U];
  uint32_t row[U];
  int block[U];
#pragma unroll
  for (int j = 0; j < U; j++) {
    const uint32_t u = first + j * (kThreads / 16);
    row[j] = units.per.of(u);
    block[j] = (int)(u - row[j] * units.per.by);
    const int c = block[j] * 128 + lane * 8;
    p[j].load(a.x, u < units.count ? row[j] * a.x_stride + c : 0, u < units.count ? cols - c : 0);
  }
#pragma unroll
  for (int j = 0; j < U; j++) {
    if (first + j * (kThreads / 16) >= units.count) return;  // all 16 lanes
    const int c = block[j] * 128 + lane * 8, left = cols - c;
    float v[8], s[8];
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = p[j].get(i);
    uint32_t top = top_of_run16(top_bits(p[j]));
    const bool wild = top >= kInfBits;  // something is not finite: the largest of the rest
    if (wild) {
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const uint32_t b = as_u32(v[i]) & 0x7fffffffu;
        m = max(m, b < kInfBits ? b : 0u);
      }
      top = top_of_run16(m);
    }
    // 448 = 1.75 * 2^8: one more where the significand is larger than 1.75
    const int e = min(max((int)((top + 0x1fffffu) >> 23) - 8, 7), 247);
    const float f = as_f32((uint32_t)(254 - e) << 23);
#pragma unroll
    for (int i = 0; i < 8; i++) s[i] = v[i] * f;
    if (e == 247) {  // 256 * 2^120 would not be finite
#pragma unroll
      for (int i = 0; i < 8; i++) s[i] = fminf(fmaxf(s[i], -240.0f), 240.0f);
    }
    if (wild) {
#pragma unroll
      for (int i = 0; i < 8; i++)
        if (!(fabsf(v[i]) < INFINITY)) {
          s[i] = __builtin_nanf("");
          if (a.act == QUASAR_ACT_GELU && v[i] < 0.0f) v[i] = s[i];  // -infinity (1 + erf(-infinity)) / 2
        }
    }
    store_bytes(a.q + row[j] * a.q_stride + c, pack_e4m3x8(s), left);
    if (lane == 0) a.exponent[row[j] * a.exponent_stride + block[j]] = (uint8_t)e;
    if (a.y) {
      apply(v, a.act);
      store_piece(a.y, row[j] * a.y_stride + c, v, left, a.y_dtype == QUASAR_BF16);
    }
  }
}

// act'(x) in x's place.  x is finite or NaN.
__device__ __forceinline__ void derive(float (&v)[8], int act) {
  if (act == QUASAR_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = v[i] > 0.0f ? 1.0f : v[i] <= 0.0f ? 0.0f : v[i];
  } else if (act == QUASAR_ACT_SILU) {  // s + x s (1 - s), with e = exp(-|x|): s (1 - s) = e / (1 + e)^2
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const float e = exp_of(-fabsf(v[i])), r = __builtin_amdgcn_rcpf(1.0f + e), er = e * r;
      v[i] = __builtin_fmaf(v[i], er * r, v[i] >= 0.0f ? r : er);
    }
  } else {  // the distribution and x times the density
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const float e = normal_exp(v[i]), tail = normal_tail(fabsf(v[i]), e);
      v[i] = __builtin_fmaf(v[i] * 0.3989422804f, e, v[i] > 0.0f ? 1.0f - tail : tail);
    }
  }
}

template <int GT, int U>
__global__ __launch_bounds__(kThreads) void checkpoint_backward_kernel(quasar_checkpoint_grad a, Units units) {
  const int lane = threadIdx.x & 15, cols = (int)a.cols;
  const uint32_t first = (blockIdx.x * (uint32_t)(kThreads / 16) * U) + (threadIdx.x >> 4);
  Piece<GT> g[U];
  uint2 q[U];
  uint32_t row[U], e[U];
  int col[U];
#pragma unroll
  for (int j = 0; j < U; j++) {
    const uint32_t u = first + j * (kThreads / 16);
    const bool has = u < units.count;
    row[j] = has ? units.per.of(u) : 0;
    const int block = has ? (int)(u - row[j] * units.per.by) : 0;
    col[j] = block * 128 + lane * 8;
    const int left = has ? cols - col[j] : 0;
    g[j].load(a.dy, row[j] * a.dy_stride + col[j], left);
    q[j] = load_bytes(a.q + row[j] * a.q_stride + col[j], left);
    e[j] = a.exponent[row[j] * a.exponent_stride + block];
  }
#pragma unroll
  for (int j = 0; j < U; j++) {
    if (first + j * (kThreads / 16) >= units.count) return;
    const int left = cols - col[j];
    float v[8];
    unpack_e4m3x8(q[j], v);
    const float f = as_f32(e[j] << 23);
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] *= f;
    derive(v, a.act);
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] *= g[j].get(i);
    store_piece(a.dx, row[j] * a.dx_stride + col[j], v, left, a.dx_dtype == QUASAR_BF16);
  }
}

// kernel(n rows from row r on, their units, the grid), as often as rows and
// stretches are more than a grid takes
template <int U, typename F>
hipError_t in_units(int64_t rows, int64_t cols, F kernel) {
  constexpr int64_t group = kThreads / 16 * U, grid = most_groups(kThreads) * group;
  const int64_t per = (cols + 127) / 128, most = (grid < (int64_t)1 << 31 ? grid : (int64_t)1 << 31) / per;
  for (int64_t r = 0; r < rows; r += most) {
    const int64_t n = rows - r < most ? rows - r : most, count = n * per;
    kernel(r, n, Units{(uint32_t)count, Divide((uint32_t)per)}, dim3((unsigned)((count + group - 1) / group)));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <int XT, int U>
hipError_t launch_keep(const quasar_checkpoint& a, hipStream_t stream) {
  return in_units<U>(a.rows, a.cols, [&](int64_t r, int64_t n, const Units& units, dim3 grid) {
    quasar_checkpoint s = a;
    s.rows = n;
    s.x = rows_on(a.x, r, a.x_stride, size_of(a.x_dtype));
    s.y = rows_on(a.y, r, a.y_stride, size_of(a.y_dtype));
    s.q = rows_on(a.q, r, a.q_stride, 1);
    s.exponent = rows_on(a.exponent, r, a.exponent_stride, 1);
    checkpoint_kernel<XT, U><<<grid, dim3(kThreads), 0, stream>>>(s, units);
  });
}

template <int GT, int U>
hipError_t launch_back(const quasar_checkpoint_grad& a, hipStream_t stream) {
  return in_units<U>(a.rows, a.cols, [&](int64_t r, int64_t n, const Units& units, dim3 grid) {
    quasar_checkpoint_grad s = a;
    s.rows = n;
    s.dy = rows_on(a.dy, r, a.dy_stride, size_of(a.dy_dtype));
    s.q = rows_on(a.q, r, a.q_stride, 1);
    s.exponent = rows_on(a.exponent, r, a.exponent_stride, 1);
    s.dx = rows_on(a.dx, r, a.dx_stride, size_of(a.dx_dtype));
    checkpoint_backward_kernel<GT, U><<<grid, dim3(kThreads), 0, stream>>>(s, units);
  });
}

}  // namespace

hipError_t launch_checkpoint(const quasar_checkpoint& a, hipStream_t stream) {
  return a.x_dtype == QUASAR_BF16 ? launch_keep<kElemBF16, 2>(a, stream) : launch_keep<kElemF32, 2>(a, stream);
}
hipError_t launch_checkpoint_backward(const quasar_checkpoint_grad& a, hipStream_t stream) {
  return a.dy_dtype == QUASAR_BF16 ? launch_back<kElemBF16, 2>(a, stream) : launch_back<kElemF32, 2>(a, stream);
}

}  // namespace quasar
