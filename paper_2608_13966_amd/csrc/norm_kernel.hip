// norm_kernel.hip -- the RMS norm with the residual's addition and its
// gradients (quasar_ops.h).
//
// Both directions are bound by memory: a row is read once and kept in
// registers as its storage form widened to fp32, eight consecutive elements
// (one 16-byte load in bf16) per lane and step, so the mean of squares, the
// row's largest |y| and the outputs all come from one read.  At 16384 x 4096 in
// bf16: forward (residual, y and q) 110 us, 5.5 TB/s; backward 101 + 6.7 us, 4.9
// TB/s (a copy of 1 GiB: 5.2).  One row takes 3.2 us, little more than a launch.
// Narrow rows leave lanes of their wavefront idle, 48 of 64 at 128 columns: 524288 x
// 128, y alone 159 us (the bytes at the copy's rate: 52), backward 227 (78).
#include "ops_common.h"
#include "ops_internal.h"

namespace quasar {

// floats from one part of dweight to the next
__host__ __device__ constexpr int parts_pitch(int cols) { return (cols + 3) & ~3; }

namespace {

constexpr int kNormThreads = 256;

// TPR threads work on one row (64: a wavefront, without a barrier; more: a
// workgroup), NV pieces of eight elements each.
template <int XT, int RT, int TPR, int NV>
__global__ __launch_bounds__(TPR < kNormThreads ? kNormThreads : TPR) void norm_kernel(quasar_norm a) {
  constexpr int kWaves = TPR / 64;
  constexpr int kRows = TPR < kNormThreads ? kNormThreads / TPR : 1;
  __shared__ float red[2][kWaves];
  const int t = TPR == 64 ? threadIdx.x & 63 : threadIdx.x;
  const int64_t row = (int64_t)blockIdx.x * kRows + (kRows > 1 ? wave_index() : 0);
  if (row >= a.rows) return;  // the whole wavefront; no barrier follows where kRows > 1
  const int cols = (int)a.cols;
  float h[NV][8];
  float ss = 0.0f;
  Piece<XT> px[NV];
  Piece<RT == kElemNone ? XT : RT> pr[NV];
  const int64_t ex = row * a.x_stride, er = row * a.residual_stride;
#pragma unroll
  for (int v = 0; v < NV; v++) {
    const int c = (v * TPR + t) * 8;
    px[v].load(a.x, ex + c, cols - c);
    if constexpr (RT != kElemNone) pr[v].load(a.residual, er + c, cols - c);
  }
#pragma unroll
  for (int v = 0; v < NV; v++) {
#pragma unroll
    for (int i = 0; i < 8; i++) {
      h[v][i] = px[v].get(i);
      if constexpr (RT != kElemNone) h[v][i] += pr[v].get(i);
      ss = __builtin_fmaf(h[v][i], h[v][i], ss);
    }
  }
  ss = group_reduce<kWaves>(ss, red[0], SumOp());
  const float rstd = 1.0f / __builtin_sqrtf(ss / (float)cols + a.eps);
  if (a.rstd && t == 0) a.rstd[row] = rstd;
  if constexpr (RT != kElemNone) {
    if (a.h) {
      const int64_t eh = row * a.h_stride;
#pragma unroll
      for (int v = 0; v < NV; v++) {
        const int c = (v * TPR + t) * 8;
        store_piece<RT == kElemBF16>(a.h, eh + c, h[v], cols - c);
      }
    }
  }
  float top = 0.0f;
#pragma unroll
  for (int v = 0; v < NV; v++) {
    const int c = (v * TPR + t) * 8;
    float w[8];
    load_floats(a.weight, c, cols - c, a.weight_dtype == QUASAR_BF16, w);
#pragma unroll
    for (int i = 0; i < 8; i++) {
      h[v][i] = h[v][i] * rstd * w[i];
      top = fmaxf(top, fabsf(h[v][i]));
    }
  }
  if (a.y) {
    const int64_t ey = row * a.y_stride;
#pragma unroll
    for (int v = 0; v < NV; v++) {
      const int c = (v * TPR + t) * 8;
      store_piece(a.y, ey + c, h[v], cols - c, a.y_dtype == QUASAR_BF16);
    }
  }
  if (!a.q) return;
  top = group_reduce<kWaves>(top, red[1], MaxOp());
  // NaN for a row that is not finite
  float scale = fmaxf(top / 448.0f, 0x1p-120f);
  if (!(ss < INFINITY)) scale = __builtin_nanf("");
  if (t == 0) a.scale[row] = scale;
  const int64_t eq = row * a.q_stride;
  const float inv = 1.0f / scale;
  const bool plain = !(scale >= 0x1p-80f && scale <= 0x1p100f);  // the remainders may not be exact, or nothing finite
#pragma unroll
  for (int v = 0; v < NV; v++) {
    const int c = (v * TPR + t) * 8, n = cols - c;
    float s[8];
#pragma unroll
    for (int i = 0; i < 8; i++) s[i] = quotient(h[v][i], scale, inv);
    if (plain) {
#pragma unroll
      for (int i = 0; i < 8; i++) s[i] = h[v][i] / scale;
    }
    const uint2 b = pack_e4m3x8(s);
    uint8_t* p = a.q + eq + c;
    if (n >= 8) {
      st8_any(p, b);
    } else {
#pragma unroll
      for (int i = 0; i < 8; i++)
        if (i < n) p[i] = (uint8_t)((i < 4 ? b.x : b.y) >> (8 * (i & 3)));
    }
  }
}

// f(TPR, NV) for the widest-fitting shape: a row that one wavefront holds in
// 32 elements a lane takes one (no barrier), wider ones a workgroup.
template <typename F>
hipError_t with_shape(int64_t cols, F f) {
  using std::integral_constant;
#define QUASAR_SHAPE(T, N) \
  if (cols <= 8 * T * N) return f(integral_constant<int, T>(), integral_constant<int, N>())
  QUASAR_SHAPE(64, 1);
  QUASAR_SHAPE(64, 2);
  QUASAR_SHAPE(64, 4);
  QUASAR_SHAPE(256, 2);
  QUASAR_SHAPE(256, 4);
  QUASAR_SHAPE(1024, 2);
  QUASAR_SHAPE(1024, 4);
#undef QUASAR_SHAPE
  return hipErrorInvalidValue;
}

// n rows from row r on
quasar_norm rows_of(quasar_norm a, int64_t r, int64_t n) {
  a.rows = n;
  a.x = rows_on(a.x, r, a.x_stride, size_of(a.x_dtype));
  a.residual = rows_on(a.residual, r, a.residual_stride, size_of(a.residual_dtype));
  a.h = rows_on(a.h, r, a.h_stride, size_of(a.residual_dtype));
  a.y = rows_on(a.y, r, a.y_stride, size_of(a.y_dtype));
  a.q = rows_on(a.q, r, a.q_stride, 1);
  a.scale = rows_on(a.scale, r, 1, 4);
  a.rstd = rows_on(a.rstd, r, 1, 4);
  return a;
}

template <int XT, int RT>
hipError_t launch_norm_types(const quasar_norm& a, hipStream_t stream) {
  return with_shape(a.cols, [&](auto tpr, auto nv) {
    constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value;
    constexpr int threads = TPR < kNormThreads ? kNormThreads : TPR, rows = threads / TPR;
    constexpr int64_t most = most_groups(threads) * rows;
    for (int64_t r = 0; r < a.rows; r += most) {
      const quasar_norm s = rows_of(a, r, a.rows - r < most ? a.rows - r : most);
      norm_kernel<XT, RT, TPR, NV><<<dim3((unsigned)((s.rows + rows - 1) / rows)), dim3(threads), 0, stream>>>(s);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
    return hipSuccess;
  });
}

// ---- backward ---------------------------------------------------------------
// Row groups of TPR threads take rows in turn; a thread meets the same columns
// in every row, so its share of dweight stays in registers.  The shares of a
// workgroup's row groups meet in LDS, those of the workgroups in `parts`
// (parts_kernel sums them), in a fixed order.  That sum is what a launch more
// costs: 777 x 1537 in fp32 takes 6.9 + 3.4 us.
template <int GT, int HT, int TPR, int NV>
__global__ __launch_bounds__(TPR < kNormThreads ? kNormThreads : TPR) void norm_backward_kernel(quasar_norm_backward a,
                                                                                               float* parts) {
  constexpr int kWaves = TPR / 64;
  constexpr int kRows = TPR < kNormThreads ? kNormThreads / TPR : 1;
  __shared__ float red[2][kWaves];
  __shared__ float sdw[kRows > 1 ? (kRows - 1) * TPR * NV * 8 : 1];
  const int t = TPR == 64 ? threadIdx.x & 63 : threadIdx.x;
  const int sub = kRows > 1 ? wave_index() : 0;
  const int cols = (int)a.cols;
  const float rcols = 1.0f / (float)cols;
  float w[NV][8], dw[NV][8] = {};
#pragma unroll
  for (int v = 0; v < NV; v++) {
    const int c = (v * TPR + t) * 8;
    load_floats(a.weight, c, cols - c, a.weight_dtype == QUASAR_BF16, w[v]);
  }
  int flip = 0;
  for (int64_t row = (int64_t)blockIdx.x * kRows + sub; row < a.rows; row += (int64_t)gridDim.x * kRows) {
    Piece<GT> pg[NV];
    Piece<HT> ph[NV];
    const int64_t eg = row * a.dy_stride, eh = row * a.h_stride, ed = row * a.dh_stride, ex = row * a.dx_stride;
#pragma unroll
    for (int v = 0; v < NV; v++) {
      const int c = (v * TPR + t) * 8;
      pg[v].load(a.dy, eg + c, cols - c);
      ph[v].load(a.h, eh + c, cols - c);
    }
    // dh is asked for with the rest where there are registers for it
    constexpr bool kEarly = TPR <= 256;
    float dh[NV][8];
    if (kEarly && a.dh) {
#pragma unroll
      for (int v = 0; v < NV; v++) {
        const int c = (v * TPR + t) * 8;
        load_floats(a.dh, ed + c, cols - c, a.dx_dtype == QUASAR_BF16, dh[v]);
      }
    }
    const float rstd = a.rstd[row];
    float dot = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; v++)
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const float n = ph[v].get(i) * rstd, g = pg[v].get(i);
        dot = __builtin_fmaf(g * w[v][i], n, dot);
        dw[v][i] = __builtin_fmaf(g, n, dw[v][i]);
      }
    // two LDS rows in turn: a wavefront may be a row ahead of another's read
    dot = group_reduce<kWaves>(dot, red[flip], SumOp());
    flip ^= 1;
    const float m = dot * rcols;
#pragma unroll
    for (int v = 0; v < NV; v++) {
      const int c = (v * TPR + t) * 8, n8 = cols - c;
      float dx[8];
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const float n = ph[v].get(i) * rstd;
        dx[i] = rstd * __builtin_fmaf(-m, n, pg[v].get(i) * w[v][i]);
      }
      if (a.dh) {
        if constexpr (!kEarly) load_floats(a.dh, ed + c, n8, a.dx_dtype == QUASAR_BF16, dh[v]);
#pragma unroll
        for (int i = 0; i < 8; i++) dx[i] += dh[v][i];
      }
      store_piece(a.dx, ex + c, dx, n8, a.dx_dtype == QUASAR_BF16);
    }
  }
  if (!parts) return;
  if constexpr (kRows > 1) {
    if (sub > 0) {
#pragma unroll
      for (int v = 0; v < NV; v++)
#pragma unroll
        for (int i = 0; i < 8; i++) sdw[(((sub - 1) * NV + v) * 8 + i) * TPR + t] = dw[v][i];
    }
    __syncthreads();
    if (sub > 0) return;
#pragma unroll
    for (int s = 0; s < kRows - 1; s++)
#pragma unroll
      for (int v = 0; v < NV; v++)
#pragma unroll
        for (int i = 0; i < 8; i++) dw[v][i] += sdw[((s * NV + v) * 8 + i) * TPR + t];
  }
#pragma unroll
  for (int v = 0; v < NV; v++) {
    const int c = (v * TPR + t) * 8;
    store_piece<false>(parts, (int64_t)blockIdx.x * parts_pitch(cols) + c, dw[v], cols - c);
  }
}

// dweight[c] = sum of parts[0 .. n)[c]: 16 columns a workgroup, four a thread,
// the parts shared out over 64 rows of threads whose sums meet in LDS.
__global__ __launch_bounds__(256) void parts_kernel(const float* parts, int n, int cols, float* out) {
  __shared__ float s[64][17];
  const int x = (threadIdx.x & 3) * 4, y = threadIdx.x >> 2, c = blockIdx.x * 16 + x, pitch = parts_pitch(cols);
  float sum[4] = {};
  if (c < cols) {
#pragma unroll 8
    for (int i = y; i < n; i += 64) {
      const float4 v = *reinterpret_cast<const float4*>(parts + (int64_t)i * pitch + c);
      sum[0] += v.x;
      sum[1] += v.y;
      sum[2] += v.z;
      sum[3] += v.w;
    }
  }
#pragma unroll
  for (int i = 0; i < 4; i++) s[y][x + i] = sum[i];
  __syncthreads();
  // four threads a column sum 16 each, then meet (they are a quad)
  if (threadIdx.x < 64) {
    const int col = threadIdx.x >> 2, q = threadIdx.x & 3;
    float t = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; i++) t += s[q * 16 + i][col];
    t += dpp_f32<kDppXor1>(t);
    t += dpp_f32<kDppXor2>(t);
    if (q == 0 && blockIdx.x * 16 + col < cols) out[blockIdx.x * 16 + col] = t;
  }
}

template <int GT, int HT>
hipError_t launch_backward_types(const quasar_norm_backward& a, hipStream_t stream) {
  return with_shape(a.cols, [&](auto tpr, auto nv) {
    constexpr int TPR = decltype(tpr)::value, NV = decltype(nv)::value;
    constexpr int threads = TPR < kNormThreads ? kNormThreads : TPR;
    const int n = norm_backward_parts(a.rows, a.cols);
    float* parts = !a.dweight ? nullptr : n == 1 ? a.dweight : reinterpret_cast<float*>(a.workspace);
    norm_backward_kernel<GT, HT, TPR, NV><<<dim3(n), dim3(threads), 0, stream>>>(a, parts);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.dweight || n == 1) return e;
    parts_kernel<<<dim3((unsigned)((a.cols + 15) / 16)), dim3(256), 0, stream>>>(parts, n, (int)a.cols, a.dweight);
    return hipGetLastError();
  });
}

}  // namespace

hipError_t launch_norm(const quasar_norm& a, hipStream_t stream) {
  const bool xb = a.x_dtype == QUASAR_BF16, rb = a.residual_dtype == QUASAR_BF16;
  if (!a.residual)
    return xb ? launch_norm_types<kElemBF16, kElemNone>(a, stream) : launch_norm_types<kElemF32, kElemNone>(a, stream);
  if (rb) return xb ? launch_norm_types<kElemBF16, kElemBF16>(a, stream) : launch_norm_types<kElemF32, kElemBF16>(a, stream);
  return xb ? launch_norm_types<kElemBF16, kElemF32>(a, stream) : launch_norm_types<kElemF32, kElemF32>(a, stream);
}

size_t norm_backward_workspace(int64_t rows, int64_t cols) {
  const int n = norm_backward_parts(rows, cols);
  return n > 1 ? (size_t)n * parts_pitch((int)cols) * sizeof(float) : 0;
}

int norm_backward_parts(int64_t rows, int64_t cols) {
  const int64_t per = cols <= 2048 ? 4 : 1;           // rows a workgroup takes at once
  const int64_t most = (cols <= 8192 ? 4 : 2) * kCUs;  // what runs at once (of 1024 threads: two a CU)
  const int64_t groups = (rows + per - 1) / per, rounds = groups <= most ? 1 : (groups + most - 1) / most;
  return (int)((groups + rounds - 1) / rounds);  // no more parts than that many rounds need
}

hipError_t launch_norm_backward(const quasar_norm_backward& a, hipStream_t stream) {
  const bool gb = a.dy_dtype == QUASAR_BF16, hb = a.h_dtype == QUASAR_BF16;
  if (gb) return hb ? launch_backward_types<kElemBF16, kElemBF16>(a, stream) : launch_backward_types<kElemBF16, kElemF32>(a, stream);
  return hb ? launch_backward_types<kElemF32, kElemBF16>(a, stream) : launch_backward_types<kElemF32, kElemF32>(a, stream);
}

}  // namespace quasar
